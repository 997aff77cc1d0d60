"""8-bit moments of AdamW far below their block's largest value (E4M3 codes under 2^-6): rounding keeps the mean there too, so that moments without a gradient go to zero, weights come to rest, and
gradients that are small beside their neighbours' arrive.  On the CPU with the model that has the kernel's bits, and on the GPU."""
import numpy as np
import pytest
import torch

from tests import adamw_common as ac

HYPER = dict(lr=1e-3, b1=0.9, b2=0.95, eps=1e-10, wd=0.0)
EVERY = np.arange(65536, dtype=np.uint64)                # all values of a code's 16 random bits


@pytest.mark.parametrize("kept", ["value", "square", "root"])
@pytest.mark.parametrize("units", [2.0 ** -13, 0.01, 0.3, 0.999, 1.0, 1.9, 3.6, 4.5, 6.75, 7.99, 8.0, 8.3, 13.7, 16.0, 21.3])
def test_the_mean_over_all_random_bits(units, kept):
    """Of a code's value, or of its square (a root's below 2^-6 always), in steps of the smallest code 2^-9: 65536 draws hit a probability to 2^-16, so the mean is off by at most that share of the step between the two neighbours
    (of their squares' difference; half a draw and two roundings of binary32 more in the product that decides there: 2^-15)."""
    x = np.full(65536, units * 2.0 ** -9, dtype=np.float32)
    x[::128] = 448.0                                      # scales of one
    square, root = kept == "square", kept == "root"
    codes, b = ac.codes_of(x, EVERY, square, root)
    assert (b == 127).all()
    fine = np.arange(65536) % 128 != 0
    got = ac.e4m3_values(codes.astype(np.uint8))[fine] * 512
    # (the places that hold the block's largest value cost every 128th draw: those are made up for by running them elsewhere)
    y = np.full(65536, units * 2.0 ** -9, dtype=np.float32)
    y[1::128] = 448.0
    rest = ac.e4m3_values(ac.codes_of(y, EVERY, square, root)[0].astype(np.uint8))[~fine] * 512
    got, u = np.concatenate([got, rest]), float(x[1]) * 512
    step = max(2.0 ** (np.floor(np.log2(u)) - 3), 1.0)
    low = np.floor(u / step) * step
    assert set(np.unique(got)) <= {low, low + step}
    if square or (root and units < 8):
        assert abs((got ** 2).mean() - u * u) <= 2.0 ** -15 * ((low + step) ** 2 - low ** 2)
    else:
        assert abs(got.mean() - u) <= 2.0 ** -16 * step


def state_of(n):
    return ac.State(None, np.zeros(n, dtype=np.float32), np.zeros(n, dtype=np.uint8), np.zeros(n, dtype=np.uint8), np.full(n // 128, 127), np.full(n // 128, 127))


STOP, REST, STEPS = 60, 300, 420                          # gradients stop after step 60; from step 360 on nothing moves


def gradients(t):
    """Three blocks.  Every eighth element has a gradient until step 60 only: as large as its neighbours', 2^-6 and 2^-12 of those, whose gradients go on."""
    rng = np.random.default_rng(1000 + t)
    g = rng.normal(size=384) * 1e-3
    g = np.where(np.arange(384) % 8 == 3, np.abs(g) * np.exp2(-6.0 * (np.arange(384) // 128)), g)
    if t > STOP:
        g[3::8] = 0
    return ac.bf16_values(ac.bf16_bits(g.astype(np.float32)))


def assert_at_rest(m, w_then, w_now):
    """A moment is at most 448 of its block's scale when its gradient stops, 229376 steps of the smallest code, and the mean of what is left after t steps is 0.9^t of it; a scale that falls by 2^6 on
    the way (the largest of 112 averages of Gaussian gradients does not) makes that 64 times as many steps.  After 300: 2^24 0.9^300 < 3.2e-7, the most the probability can be that a code is still there
    (a whole number of steps, at least one); of 48 together 2e-5.  A moment of zero stays zero, and moves nothing."""
    assert (m[3::8] & 127 == 0).all(), "moments without a gradient: codes %s" % (m[3::8] & 127)
    assert np.array_equal(w_then[3::8], w_now[3::8])


def model_run(b2):
    s, kept = state_of(384), {}
    for t in range(1, STEPS + 1):
        s = ac.step_as_rounded(s, gradients(t), t, seed=3, **dict(HYPER, b2=b2))
        kept[t] = s
    return kept


@pytest.mark.parametrize("b2", [0.95, 0.999])
def test_weights_come_to_rest(b2):
    kept = model_run(b2)
    assert_at_rest(kept[STEPS].m, kept[STOP + REST].master, kept[STEPS].master)
    others = np.arange(384) % 8 != 3
    assert (kept[STEPS].master != kept[STOP + REST].master)[others].all()


SMALL = 2.0 ** -19                                        # of the block's largest gradient: a quarter of the smallest code, whose step is 2^-17 of a largest moment just below a power of two


def small_gradient(n):
    g = np.full(n, 2.0 ** -10 * SMALL, dtype=np.float32)
    g[::128] = 2.0 ** -10
    return g


def assert_arrived(m, m_scale):
    """Steady gradients of a quarter of the smallest code.  Each rounding is off by half a step on average at most
    (a variance of 1/4), of which 0.9^2k is left after k steps: 1.32 in all, so a standard deviation of 1.15 steps, and of 1.15 / sqrt(8128) over the 8128 elements.  Five of those; the 2^-16 of a step
    that a rounding may be off in its mean ten times; what 0.9^200 leaves is nothing."""
    unit = np.repeat(np.exp2(m_scale.astype(np.float64) - 136), 128)
    rest = np.arange(m.size) % 128 != 0
    off = ((ac.e4m3_values(m) * 512 * unit - 2.0 ** -10 * SMALL) / unit)[rest]
    assert abs(off.mean()) < 5 * 1.15 / np.sqrt(rest.sum()) + 10 * 2.0 ** -16, "m is %g steps off on average" % off.mean()


def test_small_gradients_arrive():
    s = state_of(8192)
    for t in range(1, 201):
        s = ac.step_as_rounded(s, small_gradient(8192), t, seed=5, **HYPER)
    assert_arrived(s.m, s.m_scale)


def on_gpu(n):
    from paper_2512_15306_amd import llmq
    w, g = torch.zeros(n, device="cuda:0"), torch.zeros(n, device="cuda:0")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda:0") for _ in range(2))
    ms, vs = (torch.full((n // 128,), 127, dtype=torch.uint8, device="cuda:0") for _ in range(2))
    return w, g, m, v, ms, vs, llmq.llmq_adamw_plan([llmq.AdamWTensor(None, w, g, m, v, ms, vs)])


def gpu_step(plan, t, seed, h):
    from paper_2512_15306_amd import llmq
    llmq.llmq_adamw_step(plan, llmq.llmq_adamw_hyper(t, h["lr"], h["b1"], h["b2"], h["eps"], h["wd"], seed))


def assert_same(tensors, s):
    w, g, m, v, ms, vs, _ = tensors
    for got, want in ((w, s.master), (m, s.m), (v, s.v), (ms, s.m_scale), (vs, s.v_scale)):
        got = got.cpu().numpy()
        assert np.array_equal(got, want.astype(got.dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("b2", [0.95, 0.999])
def test_weights_come_to_rest_on_the_gpu(b2):
    kept, x = model_run(b2), on_gpu(384)
    for t in range(1, STEPS + 1):
        x[1].copy_(torch.from_numpy(gradients(t)))
        gpu_step(x[-1], t, 3, dict(HYPER, b2=b2))
        if t in (1, STOP, STOP + 20, STOP + REST, STEPS):
            assert_same(x, kept[t])
        if t == STOP + REST:
            then = x[0].cpu().numpy()
    assert_at_rest(x[2].cpu().numpy(), then, x[0].cpu().numpy())


@pytest.mark.gpu
def test_small_gradients_arrive_on_the_gpu():
    x = on_gpu(8192)
    x[1].copy_(torch.from_numpy(small_gradient(8192)))
    for t in range(1, 201):
        gpu_step(x[-1], t, 5, HYPER)
    assert_arrived(x[2].cpu().numpy(), x[4].cpu().numpy())


@pytest.mark.gpu
@pytest.mark.parametrize("b2", [0.95, 0.999])
def test_codes_of_every_size_on_the_gpu(b2):
    """Gradients over 2^-30 of a block's largest: codes of all sizes, the same bits as the model."""
    n, rng = 16384, np.random.default_rng(7)
    x, s = on_gpu(n), state_of(n)
    for t in range(1, 7):
        g = (np.exp2(-30.0 * rng.random(n)) * rng.choice([-1.0, 1.0], n)).astype(np.float32)
        x[1].copy_(torch.from_numpy(g))
        gpu_step(x[-1], t, 9, dict(HYPER, b2=b2))
        s = ac.step_as_rounded(s, g, t, seed=9, **dict(HYPER, b2=b2))
        assert_same(x, s)
        if t == 1:                                        # codes below 2^-6 that are not zero: three octaves of thirty (later moments go by the largest of their gradients)
            assert ((s.m & 127 > 0) & (s.m & 127 < 8)).sum() > n // 16
