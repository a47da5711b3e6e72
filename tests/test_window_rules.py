"""The plain forms that the GPU tests of rotated appends and windows compare with, against what they are meant to be, and refusals that need no
GPU."""
import numpy as np
import pytest
import torch

import window_ref as win


def test_turning_keeps_lengths_and_depends_on_differences():
    rng = np.random.default_rng(0)
    freq = (10000.0 ** -(np.arange(16) / 16))[None].astype(np.float32)
    q, k = rng.standard_normal((2, 1, 1, 64))
    for interleaved in (False, True):
        dots = []
        for a, b in ((5, 2), (1005, 1002), (3, 0)):
            x, _ = win.turned(q, np.array([[a]]), freq, interleaved, 1.0)
            y, _ = win.turned(k, np.array([[b]]), freq, interleaved, 1.0)
            assert abs(np.linalg.norm(x) - np.linalg.norm(q)) < 1e-12 and np.array_equal(x[..., 32:], q[..., 32:])
            dots.append((x * y).sum())
        assert np.ptp(dots) < 1e-9


def test_what_a_row_sees():
    slots = np.arange(14)
    # ten slots before, a chain of four, a window of three, two sinks
    got = [np.nonzero(win.sees(i, slots, 10, 4, None, None, 3, 2))[0].tolist() for i in range(4)]
    assert got == [[0, 1, 8, 9, 10], [0, 1, 9, 10, 11], [0, 1, 10, 11, 12], [0, 1, 11, 12, 13]]
    # a tree: nodes 1 and 2 under the root, 3 under 2
    mask = np.array([[1, 0, 0, 0], [1, 1, 0, 0], [1, 0, 1, 0], [1, 0, 1, 1]], bool)
    got = [np.nonzero(win.sees(i, slots, 10, 4, np.array([10, 11, 11, 12]), mask[i], 2, 0))[0].tolist() for i in range(4)]
    assert got == [[9, 10], [10, 11], [10, 12], [12, 13]]


def test_frequencies_of_several_axes():
    from paper_2608_20375_b200 import GraftError, Rope
    f = Rope.of(32, 100.0, device="cpu").freq
    assert f.shape == (1, 16) and torch.allclose(f[0], 100.0 ** (-torch.arange(16) / 16))
    g = Rope.of(32, 100.0, sections=[4, 6, 6], device="cpu").freq
    assert g.shape == (3, 16) and torch.equal(g.sum(0), f[0])
    assert [(g[a] != 0).nonzero().flatten().tolist() for a in range(3)] == [list(range(4)), list(range(4, 10)), list(range(10, 16))]
    h = Rope.of(32, 100.0, sections=[6, 5, 5], striped=True, device="cpu").freq
    assert [(h[a] != 0).nonzero().flatten().tolist() for a in range(3)] == [[0, 3, 6, 9, 12, 15], [1, 4, 7, 10, 13], [2, 5, 8, 11, 14]]
    for sections, striped in (([4, 4], False), ([17, -1], False), ([2, 7, 7], True)):
        with pytest.raises(GraftError):
            Rope.of(32, sections=sections, striped=striped, device="cpu")


def test_binding_refuses_positions_and_frequencies_of_other_shapes():
    from paper_2608_20375_b200 import GraftError, Rope
    r = Rope.of(32, sections=[8, 8], device="cpu")
    i32 = torch.int32
    for shape in ((3, 5), (2, 4), (2, 5, 3), (2, 5, 2, 1)):
        with pytest.raises(GraftError, match="position"):
            r._c(2, 5, torch.zeros(shape, dtype=i32), 0)
    with pytest.raises(GraftError, match="CUDA"):
        r._c(2, 5, torch.zeros((2, 5), dtype=i32), 0)
    with pytest.raises(GraftError, match="CUDA"):
        r._c(2, 5, None, 0)
    with pytest.raises(GraftError, match="axes, pairs"):
        Rope(r.freq[0])._c(2, 5, None, 0)
