"""The 4-bit format's oracle against hand-worked cases, and mistakes planted in it that these find (CPU)."""
import numpy as np
import pytest

from oracle import cache4 as O


def _row(*head):
    return np.array(list(head) + [0.0] * (32 - len(head)))


def test_values_of_all_codes():
    codes = np.array([[i | (i + 1) << 4 for i in range(0, 16, 2)] * 2], dtype=np.uint8)
    want = [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6]
    for e, unit in ((127, 1.0), (128, 2.0), (2, 2.0 ** -125), (252, 2.0 ** 125)):
        got = O.values(codes, np.array([[e]], dtype=np.uint8))[0]
        assert got[:16].tolist() == [w * unit for w in want] and np.signbit(got[8])
    assert np.isnan(O.values(codes, np.array([[255]], dtype=np.uint8))).all()


@pytest.mark.parametrize("largest,e", [(6.0, 0), (4.0, 0), (6.99, 0), (7.0, 1), (3.5, 0), (3.49, -1), (12.0, 1), (14.0, 2), (0.0, -125),
                                       (1e-45, -125), (float("inf"), 125), (3e38, 125), (7 * 2.0 ** -126, -125), (1.0, -2)])
def test_exponents(largest, e):
    assert O.exponents(_row(0.1 * min(largest, 1.0), -largest))[0] == e + 127


def test_rounding_and_saturation():
    x = _row(6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.99, 0.26, 0.74, 1.26, 1.74, 2.51, 3.49, 5.01, -5.0, -0.25, -0.0)
    codes, exps = O.quantised(x[None])
    assert exps[0, 0] == 127
    got = O.values(codes, exps)[0]
    assert got[:19].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 6, 0.5, 0.5, 1.5, 1.5, 3, 3, 6, -4, -0.0, -0.0]
    assert np.signbit(got[16:19]).all()
    codes, exps = O.quantised(_row(float("inf"), -float("inf"), 1.0)[None])
    assert O.values(codes, exps)[0, :3].tolist() == [6 * 2.0 ** 125, -6 * 2.0 ** 125, 0]
    codes, exps = O.quantised(_row(1.0, float("nan"))[None])
    assert exps[0, 0] == 255 and not codes.any()


def test_what_the_checks_find():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 2, 64)) * 2.0 ** rng.integers(-9, 9, (50, 2, 1))
    codes, exps = O.quantised(x)
    O.check_stored(codes, exps, x, 1e-9, "as it is")
    for wrong in (codes ^ 1, codes >> 4 | codes << 4, codes ^ 0x88, np.roll(codes, 1, -1)):
        with pytest.raises(AssertionError):
            O.check_stored(wrong, exps, x, 1e-9, "codes")
    for wrong in (exps + 1, exps - 1, exps[:, :, ::-1]):
        with pytest.raises(AssertionError):
            O.check_stored(codes, wrong, x, 1e-9, "exponents")


def test_attention_against_the_plain_one():
    from oracle import block
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal((n, 16)) for n in (9, 30, 30))
    for window in (0, 1, 5, 100):
        out, lse, size = O.attention(q, k, v, 0.25, window, 0)
        ref, ref_lse = block.attention(q, k, v, 0.25, window=window)
        assert np.allclose(out, ref, atol=1e-13) and np.allclose(lse, ref_lse, atol=1e-13)
        assert np.allclose(size, block.attention(q, k, np.abs(v), 0.25, window=window)[0], atol=1e-13)
    # first tokens: the same keys, moved next to the window
    out, lse, _ = O.attention(q[-1:], k, v, 0.25, 5, 3)
    near = list(range(3)) + list(range(25, 30))
    ref, ref_lse = block.attention(q[-1:], k[near], v[near], 0.25)
    assert np.allclose(out, ref, atol=1e-13) and np.allclose(lse, ref_lse, atol=1e-13)
    # overlapping the window, beyond the row, and all
    for sinks in (24, 27, 100):
        ref = block.attention(q, k, v, 0.25, window=0)[0]
        out = O.attention(q, k, v, 0.25, 9, sinks)[0]
        assert np.allclose(out[-1] if sinks < 100 else out, ref[-1] if sinks < 100 else ref, atol=1e-13)
    assert O.attention(q, k[:5], v[:5], 0.25, 3, 2)[0][:4].any() == False  # noqa: E712
