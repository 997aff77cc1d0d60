"""Calls of the query and key norms and of AdamW that are refused on the host, without a GPU."""
import ctypes

import pytest
import torch

from paper_2512_15306_amd import llmq

P = 0x10000               # never dereferenced: every call below fails validation on the host


def forward(**o):
    a = dict(dict(x=P, xs=512, M=3, Hq=4, Hkv=2, D=64, wq=P, wk=P, eps=1e-6, pos=P, freq=P, rot=64, inter=0, q=P, qs=256, k=P, ks=128, rstd=P), **o)
    return llmq.lib().llmq_qk_norm_rope_fwd(a["x"], a["xs"], a["M"], a["Hq"], a["Hkv"], a["D"], a["wq"], a["wk"], a["eps"], a["pos"], a["freq"], a["rot"], a["inter"], a["q"], a["qs"], a["k"], a["ks"],
                                            a["rstd"], None)


def test_eps_has_to_be_a_number_from_zero_on():
    for eps in (float("nan"), -1e-6, float("inf"), -float("inf")):
        assert forward(eps=eps) == -8
    assert forward(eps=0.0, x=P + 1) == forward(eps=1e38, x=P + 1) == -3          # (stopped by an address at an odd byte)
    assert forward(eps=float("nan"), wq=None, wk=None, x=P + 1) == -3             # without a norm there is no eps


def backward(**o):
    a = dict(dict(dq=P, dqs=256, dk=P, dks=128, dv=P, dvs=128, x=P, xs=512, M=3, Hq=4, Hkv=2, D=64, wq=P, wk=P, rstd=P, pos=P, freq=P, rot=64, inter=0, dx=P, dxs=512, dwq=P, dwk=2 * P, fmt=0, amax=P,
                  scale=P, ws=P, bytes=llmq.llmq_qk_norm_rope_workspace_bytes(3, 4, 2, 64)), **o)
    return llmq.lib().llmq_qk_norm_rope_bwd(a["dq"], a["dqs"], a["dk"], a["dks"], a["dv"], a["dvs"], a["x"], a["xs"], a["M"], a["Hq"], a["Hkv"], a["D"], a["wq"], a["wk"], a["rstd"], a["pos"], a["freq"],
                                            a["rot"], a["inter"], a["dx"], a["dxs"], a["dwq"], a["dwk"], 0, a["fmt"], a["amax"], a["scale"], a["ws"], ctypes.c_size_t(a["bytes"]), None)


def test_the_sums_for_queries_and_keys_lie_apart():
    """One buffer for both (a weight that queries and keys share) would be written by two workgroups at once."""
    for dwk in (P, P + 4, P + 252, P - 4, P - 252):
        assert backward(dwk=dwk) == -8


def test_the_words_of_a_plan_stay_on_the_host():
    """They are read during the call; a plan moved to the device as a whole would be read there."""
    words = llmq.llmq_adamw_hyper(1, 1e-3, 0.9, 0.95, 1e-8, 0.1)
    for info in (torch.zeros(4, dtype=torch.int64, device="meta"), torch.zeros(4, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), torch.zeros(8, dtype=torch.int64)[::2]):
        with pytest.raises(ValueError, match="info"):
            llmq.llmq_adamw_step(llmq.AdamWPlan(torch.zeros(64, dtype=torch.uint8), info, ()), words)


@pytest.mark.gpu
def test_a_plan_moved_to_the_device_is_refused():
    on = dict(device="cuda:0")
    t = llmq.AdamWTensor(None, torch.zeros(64, **on), torch.zeros(64, **on), torch.zeros(64, **on), torch.zeros(64, **on))
    plan = llmq.llmq_adamw_plan([t])
    with pytest.raises(ValueError, match="info"):
        llmq.llmq_adamw_step(plan._replace(info=plan.info.to("cuda:0")), llmq.llmq_adamw_hyper(1, 1e-3, 0.9, 0.95, 1e-8, 0.1))


def test_the_numbers_of_a_step_are_finite_in_binary32():
    good = dict(step=1, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
    for bad in (dict(lr=1e39), dict(lr=1e38, beta1=0.99), dict(lr=1e20, weight_decay=1e20), dict(eps=1e39)):      # (infinities in the words, and NaN in the weights)
        with pytest.raises(llmq.LlmqError) as e:
            llmq.llmq_adamw_hyper(**dict(good, **bad))
        assert e.value.status == -8
    words = llmq.llmq_adamw_hyper(**dict(good, lr=3e37, beta1=0.9, beta2=1 - 2.0 ** -53, weight_decay=1.0))[:8].view(torch.float32)
    assert torch.isfinite(words).all() and words.max() > 1e37


def test_absmax_words_lie_in_no_array():
    n, at = 1000, 1 << 20
    arrays = dict(w_bf16=2 * n, w_f32=4 * n, grad=2 * n, m=n, v=n, m_scale=8, v_scale=8)

    def entries(word, **o):
        e = llmq._AdamWTensor(n=n, flags=llmq.ADAMW_STATES_8BIT, d_amax=word, **{name: (k + 1) * at for k, name in enumerate(arrays)})
        other = llmq._AdamWTensor(n=n, d_amax=word, w_bf16=at << 8, grad=(at << 8) + 8192, m=(at << 9), v=(at << 9) + 8192, **o)
        return e, other

    for k, size in enumerate(arrays.values()):
        first = (k + 1) * at
        for word in (first, first + (size - 1) // 4 * 4):
            with pytest.raises(ValueError, match="amax"):
                llmq._check_absmax_words(entries(word))
        for word in (first - 4, first + (size + 3) // 4 * 4):
            llmq._check_absmax_words(entries(word))
    for word in ((at << 9) + 3996, (at << 8) + 8192 + 1996):          # moments of binary32, gradients of BF16
        with pytest.raises(ValueError, match="amax"):
            llmq._check_absmax_words(entries(word))
    llmq._check_absmax_words(entries((at << 8) + 8192 + 2000))
    with pytest.raises(ValueError, match="amax"):
        llmq._check_absmax_words(entries((at << 8) + 8192 + 2000, flags=llmq.ADAMW_GRAD_F32))
    llmq._check_absmax_words(entries(None))


@pytest.mark.gpu
def test_an_absmax_word_in_a_moment_is_refused():
    on = dict(device="cuda:0")
    w, m = torch.zeros(64, dtype=torch.bfloat16, **on), torch.zeros(64, **on)
    t = llmq.AdamWTensor(w, None, torch.zeros(64, **on), m, torch.zeros(64, **on), amax=m[8:9])
    with pytest.raises(ValueError, match="amax"):
        llmq.llmq_adamw_plan([t])
    llmq.llmq_adamw_plan([t._replace(amax=torch.zeros(1, **on))])
