"""The 8-bit cache's plain CPU form against the format's definition, by other means."""
import numpy as np
import pytest
import torch

from oracle import q8


def test_values_are_those_of_the_format():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(q8.VALUES, t, equal_nan=True)


def test_codes_round_to_nearest_even():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(4000) * 2.0 ** rng.integers(-14, 8, 4000), (q8.VALUES[:126] + q8.VALUES[1:127]) / 2, q8.VALUES[:127],
                        [0.0, -0.0, 448.0, -448.0]])
    x = x[np.abs(x) <= 448].astype(np.float32)
    t = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(q8.codes(x, 0), t)
    assert np.array_equal(q8.codes(x.astype(np.float64) * 2.0 ** 40, 40), t)
    assert list(q8.codes(np.array([np.inf, -np.inf, np.nan, 460.0, -1e9]), 0)) == [127, 127, 127, 126, 254]


@pytest.mark.parametrize("a,e", [(1.0, -8), (1.75, -8), (1.7500001, -7), (1.99, -7), (2.0, -7), (448.0, 0), (449.0, 1), (0.0, -110),
                                 (2.0 ** -120, -110), (3.4e38, 119), (np.inf, -110), (np.nan, -110)])
def test_scale_rule(a, e):
    assert q8.exponent([0.0, -a]) == e
    if np.isfinite(a) and -110 < e < 119:
        assert 224 < abs(a) / 2.0 ** e <= 448


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("D", [64, 128])
def test_every_byte_of_a_tile_is_one_element(which, D):
    assert sorted(q8.places(which, D).ravel()) == list(range(16 * D))


@pytest.mark.parametrize("which", ["k", "v"])
def test_pack_and_unpack(which):
    x = np.random.default_rng(1).standard_normal((3, 2, 16, 64))
    tiles, scales = q8.pack(which, x)
    y = q8.unpack(which, tiles, scales, 64)
    # half a step of 2^-3, or of the smallest element 2^-9 in scales of 224 at the largest
    assert (np.abs(x - y) <= np.maximum(np.abs(x) * 2.0 ** -4, np.abs(x).max((-2, -1), keepdims=True) * 2.0 ** -10 / 224)).all()


def _cache(pages, H=1, D=64):
    return np.zeros((pages, H, 16 * D), np.uint8), np.zeros((pages, H, 16 * D), np.uint8), np.full((pages, H, 2), 17, np.uint8)


def test_append_token_by_token_grows_the_scale():
    """A page's scale is that of the largest value written since it was begun; what was
    written before is rounded to it."""
    rng = np.random.default_rng(2)
    k, v, s = _cache(3)
    bt = np.array([[2, 0]], np.int32)
    rows = rng.standard_normal((20, 1, 64)) * np.exp(2 * rng.standard_normal((20, 1, 1)))
    for t in range(20):
        k, v, s = q8.append(rows[t:t + 1], rows[t:t + 1], bt, np.array([t + 1]), k, v, s)
        begun = t // 16 * 16
        for which, pool in ((0, k), (1, v)):
            assert int(s[bt[0, t // 16], 0, which]) - 127 == q8.exponent(rows[begun:t + 1])
            got = q8.dense("kv"[which], pool, s, bt, 0, t + 1, 64)[0]
            e = q8.exponent(rows[begun:t + 1])
            # what four significant bits hold is rounded once; smaller ones by half of the
            # smallest step of each scale that the page has had, at most twice the last's
            off = np.abs(got[begun:] - rows[begun:t + 1, 0])
            assert (off <= np.abs(rows[begun:t + 1, 0]) * 2.0 ** -4 + 2 * 2.0 ** (e - 10)).all()
    assert not k[1].any() and (s[1] == 17).all()


def test_append_begins_a_page_anew():
    k, v, s = _cache(1)
    s[:] = 200
    bt = np.zeros((1, 1), np.int32)
    x = np.full((1, 1, 64), 3.0)
    _, _, s1 = q8.append(x, x, bt, np.array([1]), k, v, s)
    assert (s1 == q8.exponent(x) + 127).all()
    _, _, s2 = q8.append(x, x, bt, np.array([2]), k, v, s)  # slot 1: the page's scale stays
    assert (s2 == 200).all()


def test_read_gives_what_append_wrote():
    rng = np.random.default_rng(3)
    k, v, s = _cache(4, H=2)
    bt = np.array([[3, 1], [0, 2]], np.int32)
    ctx, qsl = np.array([20, 7]), np.array([0, 20, 27])
    kn, vn = rng.standard_normal((27, 2, 64)), rng.standard_normal((27, 2, 64))
    k, v, s = q8.append(kn, vn, bt, ctx, k, v, s, qsl)
    got = q8.read(k, v, s, bt, ctx, 64, qsl)
    for x, new in zip(got, (kn, vn)):
        assert (np.abs(x - new) <= np.maximum(np.abs(new) * 2.0 ** -4, 2.0 ** (q8.exponent(new) - 10))).all()
