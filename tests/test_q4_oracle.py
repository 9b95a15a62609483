"""The 4-bit cache's plain form (oracle/q4.py) against values worked out by
hand from the format's definition, and its properties."""
import numpy as np
import pytest

from oracle import q4


def _block(*head):
    x = np.zeros(32)
    x[:len(head)] = head
    return x


@pytest.mark.parametrize("head,byte,codes", [
    # a = 7 = 1.75 * 2^2: e = 0, and 7 is stored as 6
    ((7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0), 127, (7, 0, 2, 2, 4, 4, 6, 6)),   # ties to the even code
    # just above: e = 1, 7.5 / 2 = 3.75 -> 4
    ((7.5, -1.0, 0.49, -0.0), 128, (6, 9, 0, 8)),
    # a = 1: e = -2, 1 / 2^-2 = 4
    ((1.0, -1.0, 0.125, 0.0625), 125, (6, 14, 1, 0)),
    # zeros
    ((0.0,), 127, (0,)),
    # far below the smallest scale, and far above the largest
    ((2.0 ** -140,), 2, (0,)),
    ((3.4e38, 1.0), 252, (7, 0)),
    # a value that is not finite: the whole block
    ((1.0, np.inf, 2.0), 255, (0, 0, 0)),
    ((np.nan, 5.0), 255, (0, 0)),
])
def test_blocks_by_hand(head, byte, codes):
    c, s = q4.quantise(_block(*head))
    assert s.tolist() == [byte]
    assert c[:len(codes)].tolist() == list(codes)
    assert not (c[len(codes):] & 7).any()


def test_values_are_bf16():
    c = np.tile(np.arange(16, dtype=np.uint8), 2)
    for byte in range(2, 253):
        x = q4.values(c, np.array([byte], np.uint8)).astype(np.float32)
        assert not (x.view(np.uint32) & 0xFFFF).any()
        assert np.array_equal(x.astype(np.float64), q4.values(c, np.array([byte], np.uint8)))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("which", ["k", "v"])
def test_layout_is_a_permutation_and_round_trips(D, which):
    at = sorted([q4.byte_of(which, D, t, m) for t in range(16) for m in range(D // 2)] +
                [q4.scale_byte_of(D, t, j) for t in range(16) for j in range(D // 32)])
    assert at == list(range(q4.tile_bytes(D)))
    rng = np.random.default_rng(D)
    x = rng.standard_normal((3, 16, D)) * np.exp(rng.standard_normal((3, 16, 1)) * 4)
    tiles = q4.pack(which, x)
    y = q4.unpack(which, tiles, D)
    # stored values are their own quantisation
    assert np.array_equal(q4.pack(which, y), tiles)
    # error: half a step of the block's largest code range, 2^e
    step = np.abs(x.reshape(3, 16, -1, 32)).max(-1) / 3.5  # a > 3.5 2^e
    assert (np.abs(x - y).reshape(3, 16, -1, 32) <= step[..., None]).all()
    pool = np.zeros((2, 1, q4.tile_bytes(D)), np.uint8)
    for t in range(16):
        q4.put(which, pool, 1, 0, t, x[0, t])
    assert np.array_equal(pool[1, 0], tiles[0]) and not pool[0].any()


def test_attention_of_equal_keys_is_the_mean():
    D = 64
    k = q4.pack("k", np.ones((2, 1, 16, D)))
    v = np.arange(32.0).reshape(2, 1, 16, 1) // 8 * np.ones(D)  # 0, 1, 2, 3: all of them codes
    out, spread, mass, size, reach = q4.attention(np.ones((3, 2, D)), k, q4.pack("v", v), np.array([[1, 0]]), [20], 0.5,
                                     query_start_loc=[0, 3])
    order = np.concatenate([v[1, 0, :, 0], v[0, 0, :, 0]])
    for j in range(3):
        assert np.allclose(out[j], order[:18 + j].mean())
    assert np.allclose(spread, out) and np.allclose(size, 32.0) and np.allclose(reach, 32.0)
