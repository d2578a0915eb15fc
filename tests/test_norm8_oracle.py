"""The oracle of the norm, dropout and 8-bit products against published values, differences and closed forms (CPU)."""
import numpy as np
import pytest

from oracle import norm8_oracle as O


@pytest.mark.parametrize("counter, key, want", [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
])
def test_philox_gives_the_published_vectors(counter, key, want):
    assert tuple(int(w) for w in O.philox(*counter, *key)) == want


def test_dropped_share_and_scale():
    m = O.drop_mask(400, 1000, 0.1, 12345, 7)
    n = m.size
    share, cut = (m == 0).mean(), O.drop_cut(0.1) / 65536
    assert abs(share - cut) < 5 * (cut * (1 - cut) / n) ** 0.5     # five standard deviations
    assert np.all((m == 0) | (m == 1 / (1 - cut)))
    assert (O.drop_mask(4, 64, 0.0, 1, 2) == 1).all() and O.drop_cut(0.9999999) == 65535
    assert not np.array_equal(m, O.drop_mask(400, 1000, 0.1, 12345, 8))
    assert np.array_equal(O.drop_mask(3, 1000, 0.1, 12345, 7, first_row=5), m[5:8])


def test_norm_gradient_against_differences():
    r = np.random.default_rng(0)
    h, g, dy, add = r.normal(size=(5, 24)), r.normal(size=24), r.normal(size=(5, 24)), r.normal(size=(5, 24))
    dh, dg = O.norm_bwd(dy, h, g, 1e-3, add)
    f = lambda h, g: (O.norm_fwd(h, g, 1e-3)[0] * dy).sum() + (h * add).sum()  # noqa: E731
    for _ in range(5):
        vh, vg, t = r.normal(size=h.shape), r.normal(size=24), 1e-5
        num = (f(h + t * vh, g + t * vg) - f(h - t * vh, g - t * vg)) / (2 * t)
        assert abs(num - ((dh * vh).sum() + (dg * vg).sum())) < 1e-6 * np.abs(dh * vh).sum()


def test_quantised_rows():
    v = np.array([[1, -2, 127, 0.5], [0, 0, 0, 0], [np.inf, 1, 2, 3], [1e-40, 0, 0, 0], [254, 1, 3, -5]], dtype=np.float32)
    q, s = O.quant_rows(v)
    assert q.tolist()[0] == [1, -2, 127, 0] and abs(s[0] - 1) <= 2.0 ** -23        # 127 * fl(1 / 127), ties to even
    assert not q[1].any() and s[1] > 0
    assert not q[2].any() and np.isnan(s[2])
    assert not q[3].any()                                                         # far below 2^-100 / 127
    assert q.tolist()[4] == [127, 0, 2, -2]


def test_order_of_a_weight():
    r = np.random.default_rng(1)
    c = r.integers(-127, 128, (128, 64)).astype(np.int8)
    laid = O.lay_weight(c)
    assert np.array_equal(np.sort(laid), np.sort(c.reshape(-1)))
    assert np.array_equal(laid.reshape(4, 2, 4, 16, 16), c.reshape(2, 4, 16, 4, 16).transpose(3, 0, 1, 4, 2))
