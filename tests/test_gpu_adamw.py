"""The AdamW step on the GPU: bit for bit against the same operations in binary32, and against binary64."""
import numpy as np
import pytest
import torch

from paper_2512_15306_amd import llmq
from tests import adamw_common as ac

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HYPER = dict(lr=1e-3, b1=0.9, b2=0.95, eps=1e-8, wd=0.1)


def hyper(t, h, seed=0):
    return llmq.llmq_adamw_hyper(t, h["lr"], h["b1"], h["b2"], h["eps"], h["wd"], seed)


class Tensor:
    """One tensor on the GPU and its state on the CPU."""

    def __init__(self, n, bits, weights, seed, grad32=False, decay=True, first=0, amax=None, grad_std=1e-3):
        rng = np.random.default_rng(seed)
        self.n, self.bits, self.decay, self.first, self.stochastic = n, bits, decay, first, weights == "stochastic"
        size = np.exp(rng.normal(size=(n + 127) // 128)).repeat(128)[:n]
        master = (rng.normal(size=n) * 0.02).astype(np.float32)
        w = ac.bf16_bits(master) if weights != "f32" else None
        keeps_master = weights in ("master", "f32")
        if bits == 8:
            m, ms = ac.codes_of((rng.normal(size=n) * size).astype(np.float32), rng.integers(0, 65536, n), False)
            v, vs = ac.codes_of(np.abs(rng.normal(size=n) * size).astype(np.float32), rng.integers(0, 65536, n), False)
            ms, vs = ms - 12, vs - 10                                        # moments of 1e-3 or so
            self.state = ac.State(w, master if keeps_master else None, (m | rng.integers(0, 2, n) * 128).astype(np.uint8), v.astype(np.uint8), ms, vs)
        else:
            self.state = ac.State(w, master if keeps_master else None, (rng.normal(size=n) * size * 3e-4).astype(np.float32), ((rng.normal(size=n) * size * 1e-3) ** 2).astype(np.float32))
        g = (rng.normal(size=n) * size * grad_std).astype(np.float32)
        self.grad = g if grad32 else ac.bf16_values(ac.bf16_bits(g))
        s = self.state
        on = lambda a, t=None: None if a is None else torch.from_numpy(a.copy()).to(DEV) if t is None else torch.from_numpy(a.view(np.int16).copy()).view(t).to(DEV)  # noqa: E731
        self.w, self.master, self.m, self.v = on(s.w, torch.bfloat16), on(s.master), on(s.m), on(s.v)
        self.ms, self.vs = on(None if s.m_scale is None else s.m_scale.astype(np.uint8)), on(None if s.v_scale is None else s.v_scale.astype(np.uint8))
        self.g = on(self.grad) if grad32 else on(ac.bf16_bits(self.grad), torch.bfloat16)
        self.amax = amax

    def entry(self):
        return llmq.AdamWTensor(self.w, self.master, self.g, self.m, self.v, self.ms, self.vs, self.first, self.decay, self.stochastic, self.amax)

    def check(self, t, h, seed=0, scale=1.0):
        want = ac.step_as_rounded(self.state, self.grad, t, seed=seed, scale=scale, decay=self.decay, stochastic=self.stochastic, first=self.first, **h)
        for name, got, exp in (("w", self.w, want.w), ("master", self.master, want.master), ("m", self.m, want.m), ("v", self.v, want.v), ("m_scale", self.ms, want.m_scale),
                               ("v_scale", self.vs, want.v_scale)):
            if exp is not None:
                a = (got.view(torch.int16) if got.dtype == torch.bfloat16 else got).cpu().numpy()
                a = a.view(np.uint16) if a.dtype == np.int16 else a
                assert np.array_equal(a, exp.astype(a.dtype)), "%s differs at %s" % (name, np.argwhere(a != exp.astype(a.dtype))[:3].ravel())
        # and by the formula, before any rounding to 16 or 8 bits, in roundings of at most 2^-24 each (of numbers as of operations): 4 of the sum of a moment's parts' magnitudes.  A weight:
        # m' 4 of |m0| b1 + |g| (1 - b1), which may be more than |m'|; v' 6 at most (g s, its square, 1 - b2, the product; the sum), so its root 3 and 1, with the factor 6, with eps 7; division,
        # lr and product 3: 14 of the step with those magnitudes in place of |m'|, less than 2^-20 of it.  Such a step has no bound in units of lr: a moment may stand beside a root that is
        # next to nothing.  Decay and the two subtractions: 2^-23 of the old weight's and the new one's magnitudes.
        w, m, v = ac.step_exact(self.state, self.grad, t, scale=scale, decay=self.decay, **h)
        m0, v0 = self.state.moments()
        step = h["lr"] / (1 - h["b1"] ** t) * (np.abs(m0.astype(np.float64)) * h["b1"] + np.abs(self.grad * scale) * (1 - h["b1"])) / (np.sqrt(v / (1 - h["b2"] ** t)) + h["eps"])
        if self.bits == 32:
            assert (np.abs(want.m - m) <= 2.0 ** -22 * (np.abs(m0) + np.abs(self.grad * scale))).all() and (np.abs(want.v - v) <= 2.0 ** -22 * v).all()
        if want.master is not None:
            assert (np.abs(want.master - w) <= 2.0 ** -20 * step + 2.0 ** -23 * (np.abs(self.state.master) + np.abs(w))).all()
        self.state = want


SIZES = [1, 7, 8, 127, 128, 129, 1000, 1023, 1024, 1025, 2048, 4095, 4096, 4097, 20000]


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("weights", ["master", "bf16", "stochastic", "f32"])
@pytest.mark.parametrize("b2", [0.95, 0.999])
def test_steps_of_many_tensors(bits, weights, b2):
    h = dict(HYPER, b2=b2)
    tensors = [Tensor(n, bits, weights, 11 + n, grad32=k % 3 == 1, decay=k % 4 != 2, first=1000000 * k) for k, n in enumerate(SIZES)]
    plan = llmq.llmq_adamw_plan([t.entry() for t in tensors])
    for t in (1, 2, 900):
        llmq.llmq_adamw_step(plan, hyper(t, h, 5))
        torch.cuda.synchronize()
        for x in tensors:
            x.check(t, h, 5)


def test_one_launch_takes_every_kind():
    kinds = [(bits, weights, g32) for bits in (8, 32) for weights in ("master", "bf16", "stochastic", "f32") for g32 in (False, True)]
    tensors = [Tensor(3000 + 17 * k, b, w, k, g32, first=10000 * k) for k, (b, w, g32) in enumerate(kinds)]
    llmq.llmq_adamw_step(llmq.llmq_adamw_plan([t.entry() for t in tensors]), hyper(3, HYPER))
    for t in tensors:
        t.check(3, HYPER)


def test_from_nothing():
    """First step with moments of zeros: every element moves by the rate, whatever its gradient's size; zero gradients leave the weight."""
    for bits in (8, 32):
        x = Tensor(1000, bits, "f32", 1)
        for t in (x.m, x.v):
            t.zero_()
        if bits == 8:
            x.ms.fill_(127), x.vs.fill_(127)
        x.g[::10] = 0
        before = x.master.clone()
        llmq.llmq_adamw_step(llmq.llmq_adamw_plan([x.entry()]), llmq.llmq_adamw_hyper(1, 1e-3, 0.9, 0.95, 1e-12, 0.0))
        moved = (x.master - before).cpu()
        assert (moved[::10] == 0).all()
        fine = x.g.float().cpu().abs() > 0
        assert torch.allclose(moved[fine], -1e-3 * torch.sign(x.g.float().cpu()[fine]), rtol=1e-3, atol=2e-9)
        assert (x.m[::10] == 0).all() and (x.v[::10] == 0).all()


@pytest.mark.parametrize("b2,most", [(0.95, 0.06), (0.99, 0.05), (0.999, 0.05)])
def test_eight_bit_moments_follow_a_steady_gradient(b2, most):
    """Gradients of fixed magnitudes and alternating signs: v must come to their squares, which it would not if codes were rounded to the nearest (it then
    stops at a thirtieth).  The mean over 8192 elements is off by the bias the header states (4 % at most up to 31/32) and by noise: a code's rounding moves v by at most
    a quarter of its value, independently from element to element, over about 1 / (1 - b2) steps of weight 1: less than 0.5 / sqrt(8192) < 1 %."""
    n, steps = 8192, int(6 / (1 - b2))
    g = torch.exp(torch.rand(n, generator=torch.Generator().manual_seed(1)) * 3 - 7).to(torch.bfloat16)
    m, v, w = torch.zeros(n, dtype=torch.uint8, device=DEV), torch.zeros(n, dtype=torch.uint8, device=DEV), torch.zeros(n, device=DEV)
    ms, vs = (torch.full((n // 128,), 127, dtype=torch.uint8, device=DEV) for _ in range(2))
    grad = g.to(DEV)
    plan = llmq.llmq_adamw_plan([llmq.AdamWTensor(None, w, grad, m, v, ms, vs)])
    for t in range(1, steps + 1):
        grad.neg_()
        llmq.llmq_adamw_step(plan, llmq.llmq_adamw_hyper(t, 1e-4, 0.9, b2, 1e-10, 0.0))
    root = ac.e4m3_values(v.cpu().numpy()) * np.repeat(np.exp2(vs.cpu().numpy().astype(np.float64) - 127), 128)
    ratio = (root / g.double().numpy()) ** 2 / (1 - b2 ** steps)
    assert abs(ratio.mean() - 1) < most, ratio.mean()


def test_random_bits_are_even():
    """Each of the 32 bits, neighbours, and steps: within 5 standard deviations of a fair coin over 2^20 counters."""
    n = 1 << 20
    c = np.arange(n, dtype=np.uint64)
    a, b = ac.mixed(c, ac.step_key(1, 0)), ac.mixed(c, ac.step_key(2, 0))
    slack = 5 * 0.5 / np.sqrt(n)
    for k in range(32):
        bit = lambda x: (x >> np.uint64(k)) & np.uint64(1)  # noqa: E731
        assert abs(bit(a).mean() - 0.5) < slack
        assert abs((bit(a)[1:] ^ bit(a)[:-1]).mean() - 0.5) < slack
        assert abs((bit(a) ^ bit(b)).mean() - 0.5) < slack


def test_stochastic_weights_keep_small_steps():
    """Steps of a hundredth of a BF16 spacing: rounded to the nearest the weights would never move."""
    n = 65536
    w, grad = torch.ones(n, dtype=torch.bfloat16, device=DEV), torch.ones(n, dtype=torch.bfloat16, device=DEV)
    m, v = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    plan = llmq.llmq_adamw_plan([llmq.AdamWTensor(w, None, grad, m, v, stochastic=True)])
    lr = 2.0 ** -8 / 100                                          # spacing of BF16 below 1: 2^-8
    for t in range(1, 101):
        llmq.llmq_adamw_step(plan, llmq.llmq_adamw_hyper(t, lr, 0.9, 0.95, 1e-12, 0.0, 7))
    # 100 steps of lr; a weight's deviation is below one spacing times sqrt(100 p (1 - p)), p = 1/100 or so: 1 spacing, over 65536 weights 2^-8 / 256; five of those
    assert abs(float(w.double().mean()) - (1 - 100 * lr)) < 5 * 2.0 ** -16


def test_absmax_of_the_new_weights():
    """Of each tensor, or of several that name the same word; with the scale it is what the quantizer would find."""
    both, own = torch.full((1,), 1e30, device=DEV), torch.full((1,), -1.0, device=DEV)
    ts = [Tensor(5000, 32, "master", 1, amax=both), Tensor(300, 8, "bf16", 2, amax=both), Tensor(70000, 8, "master", 3, amax=own), Tensor(10, 32, "bf16", 4)]
    llmq.llmq_adamw_step(llmq.llmq_adamw_plan([t.entry() for t in ts]), hyper(1, HYPER))
    assert both.item() == max(ts[0].w.abs().max().item(), ts[1].w.abs().max().item()) and own.item() == ts[2].w.abs().max().item()
    a, s, s2 = (torch.zeros(1, device=DEV) for _ in range(3))
    llmq.llmq_amax(ts[2].w, 0, a, s, torch.zeros(llmq.llmq_amax_workspace_bytes(), device=DEV, dtype=torch.uint8))
    llmq.llmq_scale_from_amax(own, 0, s2)
    assert torch.equal(a, own) and torch.equal(s, s2)
    ts[0].g[3] = float("nan")
    llmq.llmq_adamw_step(llmq.llmq_adamw_plan([t.entry() for t in ts]), hyper(2, HYPER))
    assert both.view(torch.int32).item() == 0x7FC00000 and torch.isfinite(own).all()


def test_gradients_that_are_not_finite():
    x, y = Tensor(1000, 8, "f32", 1), Tensor(1000, 32, "f32", 2)
    x.g[200], y.g[200] = float("nan"), float("inf")
    plan = llmq.llmq_adamw_plan([x.entry(), y.entry()])
    llmq.llmq_adamw_step(plan, hyper(1, HYPER))
    llmq.llmq_adamw_step(plan, hyper(2, HYPER))
    bad = torch.isnan(x.master).cpu()
    assert bad[128:256].all() and not bad[:128].any() and not bad[256:].any()         # its block
    bad = torch.isnan(y.master).cpu()
    assert bad[200] and bad.sum() == 1


@pytest.mark.parametrize("scale", [0.25, 0.0, float("nan"), float("inf")])
def test_gradient_scale(scale):
    """A factor on every gradient; where it is not finite nothing is written, not even the absmax."""
    amax = torch.full((1,), 3.0, device=DEV)
    ts = [Tensor(3000, 8, "master", 1, amax=amax), Tensor(5000, 32, "bf16", 2)]
    before = [[a.clone() for a in (t.w, t.m, t.v)] for t in ts]
    llmq.llmq_adamw_step(llmq.llmq_adamw_plan([t.entry() for t in ts]), hyper(4, HYPER), torch.full((1,), scale, device=DEV))
    if np.isfinite(scale):
        for t in ts:
            t.check(4, HYPER, scale=scale)
        assert amax.item() == ts[0].w.abs().max().item()
    else:
        assert all(torch.equal(a, b) for t, old in zip(ts, before) for a, b in zip((t.w, t.m, t.v), old)) and amax.item() == 3.0


def test_captured_steps_take_new_numbers():
    ts = [Tensor(3000, 8, "stochastic", 1), Tensor(5000, 32, "master", 2, amax=torch.zeros(1, device=DEV))]
    plan, device_hyper = llmq.llmq_adamw_plan([t.entry() for t in ts]), hyper(1, HYPER).to(DEV)
    llmq.llmq_adamw_step(plan, device_hyper)
    torch.cuda.synchronize()
    for t in ts:
        t.check(1, HYPER)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            llmq.llmq_adamw_step(plan, device_hyper)
    for step in range(2, 6):
        h = dict(HYPER, lr=1e-3 / step)
        device_hyper.copy_(hyper(step, h))
        graph.replay()
        torch.cuda.synchronize()
        for t in ts:
            t.check(step, h)
        assert ts[1].amax.item() == ts[1].w.abs().max().item()


def test_pieces_of_a_launch(monkeypatch):
    monkeypatch.setenv("LLMQ_MAX_WORKGROUPS", "8")
    ts = [Tensor(100000, 8, "master", 1), Tensor(77777, 32, "bf16", 2)]
    llmq.llmq_adamw_step(llmq.llmq_adamw_plan([t.entry() for t in ts]), hyper(2, HYPER))
    for t in ts:
        t.check(2, HYPER)


def test_bad_calls_are_refused():
    x = Tensor(300, 8, "master", 1)
    good = x.entry()
    for change in ({"m": x.m[:-1]}, {"v_scale": x.vs[:-1]}, {"w": x.w.cpu()}, {"master": x.master[::2]}, {"w": None, "master": None}, {"amax": torch.zeros(2, device=DEV)}):
        with pytest.raises(ValueError):
            llmq.llmq_adamw_plan([good._replace(**change)])
    for change in ({"grad": x.g.half()}, {"v": x.v.float()}, {"w": x.w.float()}):
        with pytest.raises(TypeError):
            llmq.llmq_adamw_plan([good._replace(**change)])
    for change in ({"m_scale": None}, {"stochastic": True}, {"first_counter": -1}, {"w": None, "amax": torch.zeros(1, device=DEV)}):
        with pytest.raises(llmq.LlmqError):
            llmq.llmq_adamw_plan([good._replace(**change)])
    with pytest.raises(llmq.LlmqError):
        llmq.llmq_adamw_plan([])
    plan = llmq.llmq_adamw_plan([good])
    with pytest.raises(ValueError):
        llmq.llmq_adamw_step(plan, hyper(1, HYPER)[:9])
    with pytest.raises(ValueError):
        llmq.llmq_adamw_step(plan, hyper(1, HYPER), torch.ones(2, device=DEV))
    for bad in (dict(step=0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(eps=1e-60), dict(weight_decay=-1.0)):
        with pytest.raises(llmq.LlmqError):
            llmq.llmq_adamw_hyper(**dict(dict(step=1, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1), **bad))
