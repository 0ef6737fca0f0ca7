"""The float64 reference of blocks of 4 bits, their layout and adapters, against definitions and hand-computed values."""
import numpy as np
import pytest

from oracle import serve_oracle as so


def test_levels_are_all_sums_of_two_bits_and_a_power():
    """Exponent field of two bits, one bit behind: 0 and 0.5 below 1, then (1 + m / 2) 2^k."""
    assert list(so.LEVELS) == [0, 0.5] + [(1 + m / 2) * 2.0 ** k for k in range(3) for m in range(2)]


@pytest.mark.parametrize("top,e", [(7.0, 0), (7.0000001, 1), (3.5, -1), (1.75, -2), (6.0, 0), (4.0, 0), (3.6, 0), (7 * 2.0 ** -110, -110), (1e-40, -110), (0.0, -110),
                                   (3.3e38, 125), (7 * 2.0 ** 124, 124)])
def test_scales(top, e):
    x = np.zeros(32)
    x[5] = -top
    assert so.hold_block(x)[1] == e + 127 and so.hold(x)[1][0] == e + 127


def test_ties_go_to_the_even_code():
    x = np.zeros(32)
    x[:9] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25]
    codes, scale = so.hold_block(x)
    assert scale == 127 and list(codes[:9]) == [0, 2, 2, 4, 4, 6, 6, 7, 8]
    assert list(so.held(codes, np.array([scale]))[:9]) == [0, 1, 1, 2, 2, 4, 4, 6, 0]


@pytest.mark.parametrize("seed", range(4))
def test_both_ways_to_codes_agree_and_no_value_is_off_by_more_than_the_scale(seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((20, 32)) * 10.0 ** rng.integers(-30, 30, (20, 1))
    x[3] = 0
    x[4, 7] = np.nan
    x[5, 9] = -np.inf
    x[6] = np.round(x[6] / np.abs(x[6]).max() * 28) / 4
    codes, scales = so.hold(x)
    for i in range(20):
        c, s = so.hold_block(x[i])
        assert np.array_equal(c, codes[i]) and s == scales[i, 0]
    back = so.held(codes, scales)
    assert np.isnan(back[4:6]).all()
    good = [i for i in range(20) if i not in (4, 5)]
    step = 2.0 ** (scales[good].astype(float) - 127)
    assert (np.abs(back[good] - x[good]) <= step).all()
    top = np.abs(x[good]).max(1, keepdims=True)
    live = top[:, 0] > 0
    assert (step[live] >= top[live] / 7).all() and (step[live] < top[live] * 2 / 7).all()


@pytest.mark.parametrize("page,d", [(16, 32), (16, 64), (32, 96), (64, 128), (16, 160), (16, 256)])
@pytest.mark.parametrize("values", [False, True])
def test_every_byte_of_a_piece_has_one_place(page, d, values):
    at, at_scale = so.places(page, d, values)
    assert sorted(np.concatenate((at.ravel(), at_scale.ravel()))) == list(range(so.piece_bytes(page, d)))
    assert so.piece_bytes(page, d) == 17 * page * d // 32
    rng = np.random.default_rng(d)
    codes = rng.integers(0, 16, (2, 3, page, d)).astype(np.uint8)
    scales = rng.integers(100, 140, (2, 3, page, d // 32)).astype(np.uint8)
    assert np.array_equal(so.unpack(so.pack(codes, scales, values), page, d, values), so.held(codes, scales))


def test_a_lane_s_codes_of_four_value_rows_lie_side_by_side():
    """What the layout is for: components c d / 16 ... of rows 4 g ... 4 g + 3 are d / 8 bytes from (16 g + c) d / 8 on, their rows in order."""
    for d in (64, 96, 128, 256):
        for g in range(4):
            for c in range(16):
                got = [so.code_byte(16, d, 4 * g + r, c * d // 32 + b, True) for r in range(4) for b in range(d // 32)]
                assert got == list(range((16 * g + c) * d // 8, (16 * g + c + 1) * d // 8))


def test_adapters_by_hand():
    H, base = np.array([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0]]), np.zeros((3, 3))
    A = np.array([[[1.0, 0.0], [0.0, 1.0]]])                 # one adapter, two parts of rank 1
    B = np.array([[[10.0], [20.0], [100.0]]])
    Z, _ = so.adapt(H, base, A, B, [2.0], [0, -1, 1], [2, 3])
    assert np.array_equal(Z, [[20, 40, 400], [0, 0, 0], [0, 0, 0]])
