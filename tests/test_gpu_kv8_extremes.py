"""Attention over 8-bit cache pages at the edges of its types: values that are not finite, scales and lengths far out."""
import numpy as np
import pytest

from tests import _operators as ref
from tests.test_gpu_kv8 import PAGE, Case, _causal, torch  # noqa: F401

pytestmark = pytest.mark.gpu
MAX = 0x7F7F                                      # the largest bf16 number


def _compare(c, out, lse, floor=0.0):
    """Every row against the definition in 64 bits; NaN and infinities exactly.

    A score is a sum of D products in 32 bits and a few roundings: off by (D + 8) 2^-24 of the sum of its magnitudes, and
    a probability by twice that of itself.  It is held as two bf16 numbers: the first is off by half a step, 2^-8 of
    itself, the second by 2^-8 of that, so 2^-16 on the whole.  2^-14 of the sum of magnitudes is for what is summed in
    32 bits and for its exponent (two roundings of numbers up to 2^9, 2^-14 at most), 2^-8 of the result half a step of bf16."""
    D, G = c.D, c.nq // c.nkv
    for b in range(c.B):
        for h in range(c.nkv):
            k, v = c.keys_values(b, h)
            for j in range(c.R):
                r, n = b * c.R + j, min(int(c.vis[b, j]), c.stride * PAGE)
                for hq in range(h * G, h * G + G):
                    o, z = out[r, hq * D:(hq + 1) * D], lse[r, hq]
                    if n < 0:
                        assert (o == 77).all() and z == 55
                        continue
                    with np.errstate(invalid="ignore"):
                        want, wz, A, S, _, _ = ref.attention(ref.bf16_value(c.q[r, hq * D:(hq + 1) * D]), k, v, n, c.scale)
                        ds = (D + 8) * 2.0 ** -24 * S
                        tol = 2.0 ** -8 * np.abs(want) + A * (2.0 ** -16 + 2 * ds + 2.0 ** -14) + floor
                        ok = (np.isnan(o) & np.isnan(want)) | (o == want) | (np.isfinite(want) & (np.abs(o - want) <= tol))
                    assert ok.all(), (b, j, hq, np.flatnonzero(~ok)[:4], o[~ok][:4], want[~ok][:4])
                    assert z == wz or abs(z - wz) <= ds + 2.0 ** -20 + 2.0 ** -22 * abs(wz), (b, j, hq, z, wz)


def _check(c, err=0, floor=0.0):
    out, lse = c.run()
    assert int(c.err) == err
    _compare(c, out, lse, floor)
    return out, lse


# -- values that are not finite ----------------------------------------------------

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("R", [1, 3, 13])
def test_infinities_in_pages_that_every_row_sees(torch, D, R):  # noqa: F811
    """An infinite value in a bf16 page is infinite in every row, and NaN only against the other infinity."""
    c = Case(torch, 40 + R, 6, 2, D, [200], [0], np.full((1, R), 200, np.int32))
    for p, at, dim, bits in ((0, 3, 5, 0x7F80), (1, 60, 6, 0xFF80), (1, 7, 8, 0x7F80), (2, 9, 8, 0xFF80), (0, 1, 9, 0x7FC0),
                             (3, 2, 10, 0xFF80), (0, 2, 11, 0x7F80), (3, 1, 11, 0x7F80)):
        c.v16[c.table[0, p], 1, dim, at] = bits
    out, _ = _check(c)
    assert np.isposinf(out[:, 3 * D + 5]).all() and np.isneginf(out[:, 3 * D + 6]).all()
    # ... whatever the other rows of the pass see
    first = out[0]
    if R > 1:
        c.vis[0, 1:] = np.arange(1, R) * 13 % 150
        out, _ = _check(c)
        np.testing.assert_array_equal(out[0], first)


@pytest.mark.parametrize("n", [9 * PAGE, 9077])   # a few groups; as many as the combine takes four a wave
def test_infinities_whose_weight_vanishes(torch, n):  # noqa: F811
    """Infinite values with weights of e^-128 beside later keys, too small for the factor that joins their groups in 32
    bits: infinite all the same."""
    c = Case(torch, 44, 2, 1, 64, [n], [0], np.array([[n, 90]], np.int32))
    c.q[:] = ref.bf16(np.float32(4))
    late = np.zeros(c.n16, bool)
    late[c.table[0, 4:-(-n // PAGE)]] = True
    c.k16[:] = ref.bf16(np.where(late, 4.0, 0.0))[:, None, None, None]
    c.v16[:] = ref.bf16(np.random.default_rng(1).standard_normal(c.v16.shape))
    c.v16[c.table[0, 1], 0, 3, 30], c.v16[c.table[0, 1], 0, 4, 31] = 0x7F80, 0xFF80
    c.v16[c.table[0, 1], 0, 5, 2] = 0x7F80       # slot 66: row 1 sees it as well
    out, _ = _check(c)
    assert np.isposinf(out[0, 3]) and np.isneginf(out[0, 4]) and np.isfinite(out[1, 3:5]).all() and np.isposinf(out[:, 5]).all()


def test_the_largest_values(torch):  # noqa: F811
    """One slot of the largest numbers, and a few of them."""
    for n in (1, 2, 5):
        for packed in (0, 1):
            c = Case(torch, 45, 4, 2, 64, [n], [packed], np.array([[n]], np.int32))
            c.v16[:] = MAX
            c.v8[:], c.vs[:] = 0x6F, 2.0 ** 120   # 120 2^120
            _check(c)


def test_the_largest_values_behind_a_growing_maximum(torch):  # noqa: F811
    """A page whose scores are 2^5 times the weight of those that its wave saw before, with a value near the largest."""
    n = 72000
    c = Case(torch, 46, 1, 1, 64, [n], [0], np.array([[n]], np.int32), extra=0)
    c.k16[:], c.v16[:] = 0, 0
    c.q[:] = 0
    c.q[0, 0] = ref.bf16(np.float32(8))          # a score is its key's first element
    c.k16[c.table[0, 4], 0, 7, 0] = ref.bf16(np.float32(3.5))
    c.v16[c.table[0, 4], 0, 9, 7] = MAX
    _check(c)


# -- scales ------------------------------------------------------------------------

@pytest.mark.parametrize("far", [3, 15, 60, 110])
def test_small_scales_beside_large_ones(torch, far):  # noqa: F811
    """Pages of small values keep their digits whatever the scales of other pages of their group, seen or not: a row that
    sees a page of small values alone, most of it weighing 2^-10 to 2^-20 of one key whose value is zero, beside rows
    that see pages of large values as well."""
    c = Case(torch, 47, 6, 2, 64, [9 * PAGE], [9], np.array([[PAGE, 9 * PAGE, 2 * PAGE, 40]], np.int32))
    c.q[:] = 0
    c.q[:, ::64] = ref.bf16(np.float32(8))       # a score is its key's first element
    p = c.table[0, 0]
    c.ks[:], c.vs[:] = 1.0, 1.0
    c.k8[p, :, :, 0] = np.random.default_rng(2).integers(0x40, 0x52, (2, PAGE))   # 2 to 9
    c.k8[p, :, 11, 0] = 0x58                     # 16
    c.v8[p, :, :, 11] = 0
    c.vs[p] = 2.0 ** -far
    c.vs[c.table[0, 1]] = 2.0 ** far
    first, _ = _check(c)
    c.vis[0, 1:] = PAGE                          # the same row beside rows that see no more
    alone, _ = _check(c)
    np.testing.assert_array_equal(first[0], alone[0])


@pytest.mark.parametrize("scale", [2.0 ** -126, 1e-40, 2.0 ** -149, 1.3 * 2.0 ** 60, 2.0 ** 118])
def test_value_scales_far_out(torch, scale):  # noqa: F811
    """8-bit pages all of one scale, alone and with bf16 pages behind them."""
    for n, packed in ((5 * PAGE, 5), (5 * PAGE + 40, 4)):
        c = Case(torch, 48, 4, 2, 64, [n], [packed], _causal([n], 3))
        c.vs[:] = scale
        # results are bf16 numbers of steps of 2^-133 there, and 32-bit sums of steps of 2^-149 (held 2^8 times as coarse)
        _check(c, floor=2.0 ** -133)


def test_value_scales_of_every_magnitude(torch):  # noqa: F811
    rng = np.random.default_rng(3)
    for seed in range(3):
        n = 12 * PAGE + 7
        c = Case(torch, 49 + seed, 4, 2, 128, [n], [10], np.array([[n, 64, 200, 500, 11 * PAGE]], np.int32))
        c.vs[:] = np.exp2(rng.integers(-126, 110, c.vs.shape)).astype(np.float32) * rng.uniform(1, 2, c.vs.shape).astype(np.float32)
        _check(c, floor=2.0 ** -133)


@pytest.mark.parametrize("ks,q,scale", [(2.0 ** -126, 2e35, 128 ** -0.5), (1e-40, 2e36, 128 ** -0.5), (2.0 ** -149, 2e36, 1.0),
                                        (2.0 ** 100, 2.0 ** -117, 2.0 ** 10), (2.0 ** 112, 2.0 ** -117, 2.0 ** -2),
                                        (2.0 ** -120, 2.0 ** 10, 2.0 ** 107), (2.0 ** 126, 2.0 ** -117, 4.0)])
def test_key_scales_far_out(torch, ks, q, scale):  # noqa: F811
    for D in (64, 128):
        n = 4 * PAGE
        c = Case(torch, 52, 4, 2, D, [n], [4], _causal([n], 3))
        c.q = ref.bf16(ref.bf16_value(c.q) * q)
        c.ks[:], c.scale = ks, scale
        _check(c)


# -- lengths -----------------------------------------------------------------------

@pytest.mark.parametrize("asked", [257, 2 ** 31 - 64, 2 ** 31 - 63, 2 ** 31 - 1])
@pytest.mark.parametrize("packed", [0, 4])
def test_rows_that_ask_for_more_than_there_is(torch, asked, packed):  # noqa: F811
    """They see the table's slots, and the other rows their own."""
    c = Case(torch, 53, 4, 2, 64, [4 * PAGE], [packed], np.array([[asked, 100, 0, -1, 256]], np.int32), extra=0)
    _check(c, err=1)
