"""The plain implementations the GPU tests compare with, pinned to numbers worked by hand."""
import numpy as np

import lowbit_reference as ref


def test_grid_of_four_bits_and_its_ties():
    x = np.float32([0, .25, .26, .75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, 100, -.25, -.75, -6])
    assert list(ref.round_e2m1(x)) == [0, 0, 1, 2, 2, 4, 4, 6, 6, 7, 7, 8, 10, 15]


def test_e4m3():
    x = [0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 1.0625, 1.1875, 17, 19, 447, 1000, -0.3]
    assert list(ref.round_e4m3(x)) == [0, 2.0 ** -9, 0, 2.0 ** -8, 1, 1.25, 16, 20, 448, 448, -0.3125]


def test_blocks_by_hand():
    x = np.zeros((1, 33), dtype=np.float32)
    x[0, 0], x[0, 1], x[0, 31], x[0, 32] = 13, -1, 3, 0.5
    codes, byte, d = ref.fp4_quantize(x, "mx")
    # 13: floor(log2) = 3, scale 2^1: 6.5 -> 6, -.5, 1.5; 0.5: 2^-1, scale 2^-3: 4
    assert list(byte[0]) == [128, 124] and codes[0, 0] == 7 | (9 << 4) and codes[0, 15] == 3 << 4 and codes[0, 16] == 6
    assert ref.fp4_values(codes, d, 33)[0, [0, 1, 31, 32]].tolist() == [12, -1, 3, 0.5]
    codes, byte, d = ref.fp4_quantize(x, "nv", 0.5)
    # blocks 0, 1, 2: amax 13, 3, .5; (amax / 6) / g = 4.33 -> 4.5, 1, .1667 -> .171875; d = 2.25, .5, .0859
    assert byte.shape == (1, 4) and np.allclose(d[0], [2.25, .5, .0859375, 0])
    assert codes[0, 0] == 7 | (9 << 4) and codes[0, 15] == 7 << 4 and codes[0, 16] == 7
    flat = ref.tiled_scales(np.arange(5 * 130, dtype=np.int64).reshape(130, 5).astype(np.uint8))
    assert flat.size == 4 * 512
    assert flat[16 * 3 + 4 * 2 + 1] == (67 * 5 + 1) % 256 and flat[512 + 16] == 1 * 5 + 4 and flat[1024 + 16] == 129 * 5 % 256


def test_cache_by_hand():
    rng = np.random.default_rng(0)
    c = ref.Cache("int8", 2, 1, 16, 16, np.array([[1]]), rng)
    one = np.zeros((1, 1, 16), dtype=np.float32)
    one[0, 0, :3] = 127, 2.5, -3.5
    c.append(0, one, [0, 1], [1])
    assert c.scale[0][1, 0, 0] == 1 and c.code[0][1, 0, 0, :3].tolist() == [127, 2, -4]
    c.append(0, one * 2, [0, 1], [2])                      # the scale doubles, the first token is requantised
    assert c.scale[0][1, 0, 0] == 2 and c.code[0][1, 0, :2, :3].tolist() == [[64, 1, -2], [127, 2, -4]]
    assert ref.bf16_up(np.float32([1.0, 1.0001, 0])).tolist() == [1, 1.0078125, 0]


def test_attention_by_hand():
    rng = np.random.default_rng(0)
    c = ref.Cache("int8", 1, 1, 16, 16, np.array([[0]]), rng)
    for side in range(2):
        c.scale[side][:] = 1
        c.code[side][:] = 0
    c.code[0][0, 0, 1, 0] = 1
    c.code[1][0, 0, :3, 0] = 4, 8, 100
    q = np.zeros((1, 2, 16))
    q[0, 0, 0] = np.log(3)
    out, lse, *_ = ref.attention(c, q, [0, 1], [2], 1.0, 0)
    assert np.allclose(out[0, :, 0], [(4 + 3 * 8) / 4, 6]) and np.allclose(lse[0], [np.log(4), np.log(2)])
    out, lse, *_ = ref.attention(c, q, [0, 1], [2], 1.0, 1)
    assert np.allclose(out[0, :, 0], 8) and np.allclose(lse[0], [np.log(3), 0])
