"""GPU parity of the gated products where their tiles end: rows and columns behind the outputs in every kernel and with longer contractions (formulas, inputs and tolerances: test_gpu_glu.py)."""
import pytest
import torch

from tests import test_gpu_glu as glu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def rows_behind(monkeypatch):
    """Outputs with 160 rows of rubbish behind them, more than a wave's part of any tile."""

    def empty(rows, cols):
        t = torch.full((rows + 160, cols), -7.0, device=DEV, dtype=torch.bfloat16)
        return t[:rows], t[rows:]

    monkeypatch.setattr(glu, "empty", empty)


@pytest.mark.parametrize("M,I,T", [(20, 100, 144), (33, 37, 256), (130, 333, 272), (250, 65, 128), (140, 100, 77), (257, 129, 389)])
@pytest.mark.parametrize("few", ["0", "1"])
def test_nothing_is_written_behind_the_last_row(monkeypatch, few, M, I, T):
    print("glu rows behind", few, M, I, T, flush=True)
    monkeypatch.setenv("LLMQ_GLU_FEW", few)
    glu.forward(M, I, T, 0, 3)
    glu.backward(M, I, T, 1, 4)
    glu.backward(M, I, T, 0, 5, want_h=False, in_place=True)


@pytest.mark.parametrize("kernel", ["few", "one wave", "4x4", "3x4", "4x2", "2x4", "2x2"])
@pytest.mark.parametrize("M,I,T", [(768, 512, 512), (450, 192, 1040), (520, 333, 388), (200, 101, 130), (300, 2049, 2052)])
def test_the_gradient_may_be_written_over_what_was_kept(monkeypatch, kernel, M, I, T):
    """In place: the bytes of the same call with a buffer of its own."""
    print("glu in place", kernel, M, I, T, flush=True)
    monkeypatch.setenv("LLMQ_GLU_FEW", "1" if kernel in ("few", "one wave") else "0")
    monkeypatch.setenv("LLMQ_GLU_FEW_ALONE", "1" if kernel == "one wave" else "0")
    if "x" in kernel:
        monkeypatch.setenv("LLMQ_GLU_TILE", kernel)
    for h in (True, False):
        want, got = (glu.backward(M, I, T, 1, 7, want_h=h, in_place=here) for here in (False, True))
        assert torch.equal(want[5], got[5]) and torch.equal(want[6], got[6])


@pytest.mark.parametrize("M,I,T", [(256, 256, 2048), (384, 192, 4096), (300, 320, 2048), (300, 320, 2052), (200, 96, 2060), (257, 160, 2064), (130, 100, 2064), (250, 104, 2052), (129, 333, 2048), (140, 37, 2076), (300, 64, 1924), (140, 72, 3972)])
@pytest.mark.parametrize("fmt", [0, 1])
def test_four_stages_and_four_waves(monkeypatch, M, I, T, fmt):
    """Contractions of more than 15 K steps in tiles of 128 x 128 that have their CU to themselves: against binary64, and the bytes of the form with two stages."""
    print("glu deep", M, I, T, fmt, flush=True)
    monkeypatch.setenv("LLMQ_GLU_FEW", "0")
    monkeypatch.setenv("LLMQ_GLU_TILE", "2x2")
    got = []
    for deep in ("1", "0"):
        monkeypatch.setenv("LLMQ_GEMM_DEEP", deep)
        f, b = glu.forward(M, I, T, fmt, 3), glu.backward(M, I, T, fmt, 4)
        got.append([f[4], f[5], f[6], b[5], b[6]])
    assert all(torch.equal(x, y) for x, y in zip(*got))


@pytest.mark.parametrize("tile", glu.TILES)
@pytest.mark.parametrize("M,I,T", [(450, 333, 388), (520, 2721, 1000), (300, 129, 132), (257, 260, 20), (768, 1001, 256), (64, 68, 516)])
def test_widths_of_no_whole_pieces_in_every_tile(monkeypatch, tile, M, I, T):
    """Backward tiles take any width: pieces at any address inside the matrix, element by element in its last columns."""
    print("glu tile", tile, M, I, T, flush=True)
    monkeypatch.setenv("LLMQ_GLU_FEW", "0")
    monkeypatch.setenv("LLMQ_GLU_TILE", tile)
    for fmt, want_h, in_place in ((0, True, False), (1, False, True), (1, True, True)):
        glu.backward(M, I, T, fmt, 5, want_h, in_place)


@pytest.mark.parametrize("M,I,T", glu.RAGGED + glu.WHOLE)
@pytest.mark.parametrize("fmt", [0, 1])
def test_tiles_of_problems_that_the_other_kernel_takes(monkeypatch, M, I, T, fmt):
    print("glu tiles", M, I, T, fmt, flush=True)
    monkeypatch.setenv("LLMQ_GLU_FEW", "0")
    glu.forward(M, I, T, fmt, M + I + T, keep=fmt == 0)
    glu.backward(M, I, T, fmt, M + I + T, want_h=fmt == 0, in_place=fmt == 1)
