"""Host side of the operators around the linears (blocks of 128, query and key norms, AdamW), without a GPU: sizes, refusals, plans, and the build's check of the scaled
MFMAs' operands."""
import ctypes
import struct

import pytest
import torch

from paper_2512_15306_amd import build, llmq
from tests import adamw_common as ac

P = 0x10000               # never dereferenced: every call below fails validation on the host
ODD = 0x10001


def test_scale_bytes():
    for rows, cols, want in ((1, 1, 128), (128, 128, 128), (129, 128, 256), (128, 129, 256), (300, 1000, 384 * 8), (8192, 3584, 8192 * 28)):
        assert llmq.llmq_block_scales_bytes(rows, cols) == want
    assert llmq.llmq_block_scales_bytes(0, 5) == llmq.llmq_block_scales_bytes(5, -1) == llmq.llmq_block_scales_bytes(1 << 31, 1) == 0


def test_block_calls_refuse():
    L = llmq.lib()
    q = lambda x=P, rows=4, cols=4, fmt=0, block=1, q=P, s=P, qt=P, st=P: L.llmq_quantize_fp8_blocks(x, rows, cols, fmt, block, q, s, qt, st, None)  # noqa: E731
    assert q(x=None) == q(q=None) == q(s=None) == q(qt=None) == q(st=None) == q(q=None, s=None, qt=None, st=None) == -1
    assert q(rows=0) == q(cols=-1) == q(rows=1 << 31) == q(rows=1 << 20, cols=1 << 20) == -2
    assert q(fmt=2) == -4 and q(block=64) == q(block=0) == -7
    for name in ("x", "q", "s", "qt", "st"):
        assert q(**{name: P + 8}) == -3
    g = lambda A=P, sA=P, fa=0, B=P, sB=P, fb=0, R=4, C=4, T=64, c=P, amax=None: L.llmq_fp8_gemm_blocks(A, sA, fa, B, sB, fb, R, C, T, c, 0, amax, None)  # noqa: E731
    assert g(A=None) == g(sA=None) == g(B=None) == g(sB=None) == g(c=None) == -1
    assert g(R=0) == g(C=0) == g(T=0) == g(R=1 << 31) == g(R=1 << 20, T=1 << 20) == g(R=1 << 20, C=1 << 20) == -2
    assert g(T=8, R=1 << 21) == g(T=8, C=1 << 28) == -2                  # beyond the generic kernel's grid
    assert g(fa=2) == g(fb=-1) == -4
    for name in ("A", "sA", "B", "sB", "c"):
        assert g(**{name: P + 8}) == -3
    assert g(amax=P + 2) == -3


def test_query_and_key_calls_refuse():
    L = llmq.lib()
    f = dict(x=P, xs=512, M=3, Hq=4, Hkv=2, D=64, wq=P, wk=P, eps=1e-6, pos=P, freq=P, rot=64, inter=0, q=P, qs=256, k=P, ks=128, rstd=P)

    def fwd(**o):
        a = dict(f, **o)
        return L.llmq_qk_norm_rope_fwd(a["x"], a["xs"], a["M"], a["Hq"], a["Hkv"], a["D"], a["wq"], a["wk"], a["eps"], a["pos"], a["freq"], a["rot"], a["inter"], a["q"], a["qs"], a["k"], a["ks"],
                                       a["rstd"], None)

    assert fwd(x=None) == fwd(q=None) == fwd(k=None) == fwd(wq=None) == fwd(wk=None) == fwd(pos=None) == fwd(freq=None) == -1
    assert fwd(M=0) == fwd(Hq=0) == fwd(Hkv=0) == fwd(D=0) == fwd(D=1025) == fwd(rot=65) == fwd(rot=66) == fwd(rot=-2) == fwd(Hq=1 << 17) == fwd(xs=511) == fwd(qs=255) == fwd(ks=127) == -2
    assert fwd(inter=2) == -7
    for name in ("x", "q", "k", "wq", "wk"):
        assert fwd(**{name: ODD}) == -3
    assert fwd(pos=P + 4) == fwd(freq=P + 4) == fwd(rstd=P + 2) == -3
    b = dict(dq=P, dqs=256, dk=P, dks=128, dv=P, dvs=128, x=P, xs=512, M=3, Hq=4, Hkv=2, D=64, wq=P, wk=P, rstd=P, pos=P, freq=P, rot=64, inter=0, dx=P, dxs=512, dwq=P, dwk=P, fmt=0, amax=P, scale=P,
             ws=P, bytes=llmq.llmq_qk_norm_rope_workspace_bytes(3, 4, 2, 64))

    def bwd(**o):
        a = dict(b, **o)
        return L.llmq_qk_norm_rope_bwd(a["dq"], a["dqs"], a["dk"], a["dks"], a["dv"], a["dvs"], a["x"], a["xs"], a["M"], a["Hq"], a["Hkv"], a["D"], a["wq"], a["wk"], a["rstd"], a["pos"], a["freq"],
                                       a["rot"], a["inter"], a["dx"], a["dxs"], a["dwq"], a["dwk"], 0, a["fmt"], a["amax"], a["scale"], a["ws"], ctypes.c_size_t(a["bytes"]), None)

    assert bwd(dq=None) == bwd(dk=None) == bwd(dx=None) == bwd(wk=None) == bwd(x=None) == bwd(rstd=None) == bwd(pos=None) == bwd(ws=None) == bwd(amax=None) == -1      # (a scale without absmax)
    assert bwd(wq=None, wk=None) == bwd(wq=None, wk=None, dwq=None) == bwd(wq=None, wk=None, dwk=None) == -1 and bwd(wq=None, wk=None, dwq=None, dwk=None, bytes=0) == -5      # sums without a norm
    assert bwd(M=0) == bwd(dqs=255) == bwd(dks=127) == bwd(dvs=127) == bwd(xs=511) == bwd(dxs=511) == bwd(rot=66) == -2
    assert bwd(fmt=2) == -4 and bwd(bytes=b["bytes"] - 1) == -5 and bwd(inter=-1) == -7
    assert bwd(ws=P + 8) == bwd(dwq=P + 2) == bwd(dx=ODD) == bwd(dv=ODD) == bwd(amax=P + 2) == -3
    assert llmq.llmq_qk_norm_rope_workspace_bytes(3, 4, 2, 64) >= 1024 * 2 * 64 * 4 and llmq.llmq_qk_norm_rope_workspace_bytes(0, 4, 2, 64) == 0


def entry(**o):
    """Arrays that lie apart, those of one entry from those of another too"""
    entry.at = getattr(entry, "at", P) + (1 << 24)
    e = llmq._AdamWTensor(n=10, **{name: entry.at + (k << 20) for k, name in enumerate(("w_bf16", "w_f32", "grad", "m", "v"))})
    for k, v in o.items():
        setattr(e, k, v)
    return e


def plan_of(*entries):
    L, arr = llmq.lib(), (llmq._AdamWTensor * max(len(entries), 1))(*entries)
    n = L.llmq_adamw_plan_bytes(arr, len(entries))
    buf, info = (ctypes.c_uint8 * max(n, 1))(), (ctypes.c_int64 * 4)()
    return L.llmq_adamw_plan(arr, len(entries), buf, ctypes.c_size_t(n), info), bytes(buf)[:n], list(info)


def test_plans():
    status, table, info = plan_of(entry(n=4096), entry(n=4097, first_counter=9, flags=llmq.ADAMW_STATES_8BIT, m_scale=P, v_scale=2 * P), entry(n=1, d_amax=P))
    assert status == 0 and info == [3, 10, 1, 0] and len(table) == 512 + 10 * 8
    assert [struct.unpack_from("ii", table, 512 + 8 * k) for k in range(10)] == [(0, k) for k in range(4)] + [(1, k) for k in range(5)] + [(2, 0)]
    assert plan_of(entry())[2][2] == 0
    for bad, want in ((dict(grad=None), -1), (dict(m=None), -1), (dict(v=None), -1), (dict(w_bf16=None, w_f32=None), -1), (dict(flags=2), -1), (dict(w_bf16=None, d_amax=P), -1),
                      (dict(n=0), -2), (dict(n=1 << 40), -2), (dict(first_counter=-1), -2), (dict(flags=16), -7), (dict(flags=8), -7), (dict(grad=P + 8), -3), (dict(w_f32=P + 4), -3), (dict(d_amax=P + 2), -3)):
        assert plan_of(entry(), entry(**bad))[0] == want, bad
    assert plan_of()[0] == -2
    L, arr = llmq.lib(), (llmq._AdamWTensor * 1)(entry())
    n, info = L.llmq_adamw_plan_bytes(arr, 1), (ctypes.c_int64 * 4)()
    assert L.llmq_adamw_plan(arr, 1, (ctypes.c_uint8 * n)(), ctypes.c_size_t(n - 1), info) == -5
    assert L.llmq_adamw_plan(arr, 1, None, ctypes.c_size_t(n), info) == -1
    words = (ctypes.c_uint32 * 10)()
    info[0], info[1] = 1, 1
    assert L.llmq_adamw_step(None, info, words, None, None, None) == L.llmq_adamw_step(P, None, words, None, None, None) == -1
    assert L.llmq_adamw_step(P, info, None, None, None, None) == L.llmq_adamw_step(P, info, words, P, None, None) == -1       # neither, both
    assert L.llmq_adamw_step(P + 8, info, words, None, None, None) == L.llmq_adamw_step(P, info, None, P + 2, None, None) == -3
    info[1] = 0
    assert L.llmq_adamw_step(P, info, words, None, None, None) == -2


def test_plans_of_arrays_that_overlap():
    a, b = entry(n=1000), entry(n=1000)
    assert plan_of(a, b)[0] == 0 and plan_of(a, a)[0] == -8
    bits8 = dict(flags=llmq.ADAMW_STATES_8BIT, m_scale=3 * P, v_scale=4 * P)
    for shared in (dict(w_bf16=a.w_bf16), dict(w_f32=a.w_f32 + 3984), dict(m=a.v + 3984), dict(v=a.v - 3984), dict(grad=a.w_bf16 + 1984), dict(w_bf16=a.grad + 1984), dict(w_bf16=a.w_f32, w_f32=None),
                   dict(bits8, m_scale=a.m + 3999), dict(bits8, v_scale=a.m - 7), dict(bits8, v_scale=3 * P + 7), dict(bits8, m=a.m - 992)):
        for order in ((a, entry(n=1000, **shared)), (entry(n=1000, **shared), a)):
            assert plan_of(*order)[0] == -8, shared
    for apart in (dict(w_f32=a.w_f32 + 4000), dict(v=a.v - 4000), dict(grad=a.grad + 16), dict(w_bf16=a.grad + 2000), dict(w_bf16=a.grad - 2000), dict(bits8, v_scale=a.m - 8), dict(bits8, v_scale=3 * P + 8),
                  dict(bits8, m=a.m - 1008), dict(m_scale=a.m, v_scale=a.m), dict(d_amax=P)):
        for order in ((a, entry(n=1000, **apart)), (entry(n=1000, **apart), a)):
            assert plan_of(*order)[0] == 0, apart
    assert plan_of(entry(d_amax=P), entry(d_amax=P))[0] == 0
    assert plan_of(entry(w_f32=None, m=a.m), entry(grad=a.m))[0] == plan_of(entry(n=1, m=a.grad, v=a.grad))[0] == -8
    many = [entry(n=1 + 997 * k % 5000) for k in range(500)]
    assert plan_of(*many)[0] == 0 and plan_of(*many, entry(v=many[250].v))[0] == -8


def test_the_numbers_of_a_step():
    words = llmq.llmq_adamw_hyper(7, 3e-4, 0.9, 0.95, 1e-8, 0.1, 1234)
    f = words[:8].view(torch.float32)
    want = torch.tensor([0.9, 0.95, 1 - 0.9, 1 - 0.95, 3e-4 * 0.1, 3e-4 / (1 - 0.9 ** 7), 1 / (1 - 0.95 ** 7) ** 0.5, 1e-8], dtype=torch.float64).float()
    assert torch.equal(f[[0, 1, 2, 3, 4, 7]], want[[0, 1, 2, 3, 4, 7]]) and torch.allclose(f, want, rtol=2.0 ** -23, atol=0)      # (powers may differ by a unit of binary64)
    assert int(words[8]) & 0xFFFFFFFF == ac.step_key(7, 1234)
    assert not torch.equal(words, llmq.llmq_adamw_hyper(8, 3e-4, 0.9, 0.95, 1e-8, 0.1, 1234))
    assert int(llmq.llmq_adamw_hyper(7, 3e-4, 0.9, 0.95, 1e-8, 0.1, 1235)[8]) != int(words[8])
    for bad in (dict(step=0), dict(lr=-1.0), dict(beta1=1.0), dict(beta2=float("nan")), dict(eps=0.0), dict(eps=float("inf")), dict(weight_decay=float("inf"))):
        with pytest.raises(llmq.LlmqError) as e:
            llmq.llmq_adamw_hyper(**dict(dict(step=1, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1), **bad))
        assert e.value.status == -8 and "out of range" in str(e.value)


def test_tensors_on_the_host_are_refused():
    x = torch.zeros(4, 128, dtype=torch.bfloat16)
    u = torch.zeros(4, 128, dtype=torch.uint8)
    for call in (lambda: llmq.llmq_quantize_fp8_blocks(x, 0, 1, u, u), lambda: llmq.llmq_fp8_gemm_blocks(u, u, 0, u, u, 0, x[:, :4].contiguous()),
                 lambda: llmq.llmq_qk_norm_rope_fwd(x, 2, 1, 32, None, None, 1e-6, None, None, False, x[:, :64], x[:, :32]),
                 lambda: llmq.llmq_adamw_plan([llmq.AdamWTensor(x, None, x, x.float(), x.float())])):
        with pytest.raises(ValueError, match="must live on the GPU"):
            call()


SCALED = """%s:                                ; @x
\tv_mov_b32_e32 v40, v41
\ts_nop 4
\ts_nop 0
\ts_nop 0
\tv_mfma_scale_f32_16x16x128_f8f6f4 a[0:3], v[20:27], v[10:17], a[0:3], v40, v50 op_sel_hi:[0,0,0]
\tv_mfma_scale_f32_16x16x128_f8f6f4 a[4:7], v[20:27], v[10:17], a[4:7], v40, v50 op_sel:[1,0,0] op_sel_hi:[0,0,0]
\ts_endpgm
.Lfunc_end0:
""" % "_ZN4llmq16gemm_tile_kernelILi0EEEv"


@pytest.mark.parametrize("planted", ["\tv_mov_b32_e32 v40, v60", "\tv_lshrrev_b32_e32 v50, 8, v50", "\tv_mov_b64_e32 v[26:27], v[60:61]", "\tv_add_u32_e32 v12, v1, v2"])
def test_writes_right_in_front_of_a_scaled_mfma_fail_the_build(planted):
    build.check_scale_operands("good.hip", SCALED)
    for anchor in ("\ts_nop 0\n\ts_nop 0\n", "a[0:3], v40, v50 op_sel_hi:[0,0,0]\n"):
        assert anchor in SCALED
        with pytest.raises(RuntimeError, match="scaled MFMA"):
            build.check_scale_operands("bad.hip", SCALED.replace(anchor, anchor + planted + "\n", 1))
    build.check_scale_operands("good.hip", SCALED.replace("\ts_nop 4\n", "\ts_nop 4\n\tv_mov_b32_e32 v60, v61\n"))
