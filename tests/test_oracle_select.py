"""The selection oracle against the properties it stands for."""
import numpy as np

from oracle import gemv as og
from oracle import select as osel


def test_score_bounds_every_token_of_the_block():
    rng = np.random.default_rng(0)
    k = og.bf16_to_f32(og.f32_to_bf16(rng.standard_normal((100, 2, 128)).astype(np.float32))).astype(float)
    q = og.bf16_to_f32(og.f32_to_bf16(rng.standard_normal((6, 128)).astype(np.float32))).astype(float)
    s = osel.scores(q, k)
    eq = osel.exponent(np.abs(q).max(1))
    q8 = np.rint(q / np.ldexp(1.0, eq)[:, None])
    for g in range(2):
        dots = (q8[3 * g:3 * g + 3] * np.ldexp(1.0, eq[3 * g:3 * g + 3])[:, None]) @ k[:, g].T
        for j in range(s.shape[1]):
            assert s[g, j] >= dots[:, 16 * j:16 * j + 16].max()
    assert np.array_equal(s, s.astype(np.float32))


def test_exponent_rule():
    top = np.array([0.0, 1.0, 127.0, 127.5, 2.0 ** -126, 127 * 2.0 ** -126, 3.38e38])
    e = osel.exponent(top)
    assert np.all(top <= 127 * 2.0 ** e)
    assert np.all((top > 127 * 2.0 ** (e - 1.0)) | (e == -126))


def test_selection_ties_and_ends():
    s = np.array([[1.0, 5, 5, 5, 0, 2, 9]])
    assert osel.select(s, 3, 0, 0).tolist() == [[1, 2, 6]]
    assert osel.select(s, 3, 1, 1).tolist() == [[0, 1, 6]]
    assert osel.select(s, 4, 0, 2).tolist() == [[1, 2, 5, 6]]
    assert osel.select(s, 9, 0, 0).tolist() == [[0, 1, 2, 3, 4, 5, 6, -1, -1]]
