"""Passes over trees where a row could notice what it does not see, and at the ends of lengths, tables and values."""
import math

import numpy as np
import pytest

from tests import _tree as ref
from tests.test_gpu_tree import PAGE, Attn, Rows, _append, _bits, _cache, _check_append, _check_commit, _commit, _dev, _trees, torch  # noqa: F401

pytestmark = pytest.mark.gpu
NAN, INF = math.nan, math.inf

# one row tile a workgroup and two; one group of a sequence and several
SHAPES = [(4, 2, 64), (2, 1, 128), (28, 4, 128), (16, 2, 64)]
BRANCHES = [-1, 0, 0, 1, 2, 3, 4]     # two branches, rows 1 3 5 and 2 4 6


def _again(a):
    """Outputs of a call whose cache has been changed on the host."""
    a.dk, a.dv = _dev(a.torch, a.k), _dev(a.torch, a.v)
    a.cache = _cache(a.torch, a.B, a.dk, a.dv)
    return a.run()


def _same(got, want, rows):
    for x, y in zip(got, want):
        np.testing.assert_array_equal(x[rows].view(np.uint16 if x.dtype == np.uint16 else np.uint32),
                                      y[rows].view(np.uint16 if y.dtype == np.uint16 else np.uint32))


@pytest.mark.parametrize("nq,nkv,D", [(256, 256, 64), (256, 256, 128), (1280, 256, 64), (1280, 256, 128)])
@pytest.mark.parametrize("length", [300, 700])
def test_scores_of_siblings_do_not_move_a_row(torch, nq, nkv, D, length):  # noqa: F811
    """Bit for bit: a sibling's scores may be any number.  One group for each of many heads: its waves have several halves of
    pages each, of which the last holds the rows' slots."""
    rng = np.random.default_rng(31)
    p = ref.Pass([length], [7], [BRANCHES])
    a = Attn(torch, rng, p, nq, nkv, D, layers=1, layer=0)
    want = a.run()
    for j in (2, 6):
        slot = length + j
        page = a.table[0, slot // PAGE]
        others, k = [r for r in range(7) if j not in p.line(0, r)], a.k.copy()
        for factor in (30.0, -3.0, 1000.0):
            # along a query of the row: its score against itself is large
            q = ref.bf16_value(a.q[j]).reshape(nkv, nq // nkv, D)[:, 0]
            a.k[0, page, :, slot % PAGE] = ref.bf16(factor * q)
            _same(_again(a), want, others)
        a.k = k


@pytest.mark.parametrize("nq,nkv,D", SHAPES)
@pytest.mark.parametrize("length", [20, 100, 3000])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -120, 2.0 ** 100])
def test_what_siblings_hold_does_not_move_a_row(torch, nq, nkv, D, length, size):  # noqa: F811
    """Bit for bit: a sibling's slot may hold values that are not finite, and the row's own be small or large."""
    rng = np.random.default_rng(32)
    p = ref.Pass([length], [7], [BRANCHES])
    a = Attn(torch, rng, p, nq, nkv, D)
    fine = np.isfinite(ref.bf16_value(a.v))
    a.v[fine] = ref.bf16(size * ref.bf16_value(a.v))[fine]
    want = _again(a)
    for j, what in ((2, NAN), (4, INF), (6, -INF)):
        slot = length + j
        page = a.table[0, slot // PAGE]
        k, v = a.k.copy(), a.v.copy()
        a.k[1, page, :, slot % PAGE, ::7] = ref.bf16(np.array(what))
        a.v[1, page, :, ::3, slot % PAGE] = ref.bf16(np.array(what))
        _same(_again(a), want, [r for r in range(7) if j not in p.line(0, r)])
        a.k, a.v = k, v


@pytest.mark.parametrize("nq,nkv,D", SHAPES)
@pytest.mark.parametrize("length", [100, 3000])
def test_values_not_finite_in_one_dimension_leave_the_others(torch, nq, nkv, D, length):  # noqa: F811
    """Bit for bit, also of rows that see them."""
    rng = np.random.default_rng(33)
    p = ref.Pass([length], [7], [BRANCHES])
    a = Attn(torch, rng, p, nq, nkv, D)
    out, lse = a.run()
    for slot, d, what in ((3, 5, INF), (length // 2, 17, NAN), (length + 1, D - 1, -INF)):
        a.v[1, a.table[0, slot // PAGE], :, d, slot % PAGE] = ref.bf16(np.array(what))
    got, glse = _again(a)
    np.testing.assert_array_equal(glse, lse)
    keep = [d for d in range(D) if d not in (5, 17, D - 1)]
    np.testing.assert_array_equal(got.reshape(7, nq, D)[:, :, keep], out.reshape(7, nq, D)[:, :, keep])
    a.check()


def _small_bounds(out, absum, big, D, slots):
    """How far out may be off where values are small.  Relative to the sum of p |v| as in attention_bounds.  At the
    lower end of the range: a weight under 2^-126 of the largest is lost, 2^-126 of the values' size, which absum's
    2^-24 holds many times over; every product, sum and factor in 32 bits is off by 2^-150 at most, of which there are two
    products with two sums a slot, and 8 + 256 groups' shares of three operations, the sums in units of at least the result's;
    then out is rounded to bf16, half a step, 2^-134 at least."""
    e = 2 * (D + 4) * 2.0 ** -24 * big
    rel = 2 * e + 2.0 ** -22 + 2.0 ** -16 + 2 * (slots + 64) * 2.0 ** -24
    return np.maximum(2.0 ** -8 * np.abs(out), 2.0 ** -134) + 1.01 * rel * absum + (4 * slots + 3 * 264) * 2.0 ** -150


@pytest.mark.parametrize("nq,nkv,D", SHAPES)
@pytest.mark.parametrize("length", [150, 3000])
@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -118, 2.0 ** -125])
@pytest.mark.parametrize("infinite", [False, True])
def test_small_values(torch, nq, nkv, D, length, size, infinite):  # noqa: F811
    """Values down to the smallest normal ones, in bounds that outputs of zero do not pass; beside infinite ones too."""
    rng = np.random.default_rng(34)
    p = ref.Pass([length], [7], [BRANCHES])
    a = Attn(torch, rng, p, nq, nkv, D)
    fine = np.isfinite(ref.bf16_value(a.v))
    a.v[fine] = ref.bf16(size * np.where(rng.random(a.v.shape) < 0.95, 1, 0.5))[fine]
    if infinite:
        a.v[1, a.table[0, 0], :, ::8, 7] = 0x7F80
        a.v[1, a.table[0, (length + 2) // PAGE], :, 1::2, (length + 2) % PAGE] = 0xFF80
    out, _ = _again(a)
    for j in range(7):
        s = np.array(a.slots(0, j), int)
        pg, off = a.table[0, s // PAGE], s % PAGE
        for h in range(nq):
            k = ref.bf16_value(a.k[1, pg, h // (nq // nkv), off])
            v = ref.bf16_value(a.v[1, pg, h // (nq // nkv), :, off])
            w, _, absum, big = ref.attention(ref.bf16_value(a.q[j, h * D:(h + 1) * D]), k, v, a.scale)
            fin = np.isfinite(w)
            assert infinite or fin.all()
            tol = _small_bounds(w[fin], absum[fin], big, D, len(s))
            assert (tol < np.abs(w[fin]) / 8).all()
            have = ref.bf16_value(out[j, h * D:(h + 1) * D])
            np.testing.assert_array_equal(have[~fin], w[~fin])
            off_by = np.abs(have[fin] - w[fin])
            assert (off_by <= tol).all(), (j, h, float((off_by / tol).max()))


@pytest.mark.parametrize("nq,nkv", [(256, 256), (10240, 256)])
def test_large_values_of_many_slots_of_one_wave(torch, nq, nkv):  # noqa: F811
    """A wave's own sum: 12 thousand slots (24 thousand where two waves share a half) of the largest values, whose
    weights are 2^7.9 times its first slots'."""
    D, stride = 64, 1501
    pages = 2
    rng = np.random.default_rng(35)
    k = np.zeros((1, pages, nkv, PAGE, D), np.uint16)
    k[0, 1, :, :, 0] = ref.bf16(np.array(8.0 * 7.9 * math.log(2)))     # scores of the second page: 7.9 ln 2
    sign = np.where(rng.random(D) < 0.5, 1.0, -1.0)
    v = np.broadcast_to(ref.bf16(sign * 255 * 2.0 ** 120)[None, None, None, :, None], (1, pages, nkv, D, PAGE)).copy()
    q = ref.bf16(np.broadcast_to((np.arange(D) == 0) * 1.0, (1, nq, D)).reshape(1, nq * D))
    table = np.ones((1, stride), np.int32)
    table[0, :4] = 0                                                   # every wave begins with a low score
    p = ref.Pass([(stride - 1) * PAGE + 10], [1], None, stride=stride)
    a = Attn(torch, rng, p, nq, nkv, D, layers=1, layer=0, table=table, pages=pages, k=k, v=v, q=q)
    out, lse = a.run()
    np.testing.assert_array_equal(ref.bf16_value(out).reshape(nq, D), np.broadcast_to(sign * 255 * 2.0 ** 120, (nq, D)))
    z = ref.bf16_value(k[0, 1, 0, 0, 0]) / 8
    low = PAGE * int((table == 0).sum())
    want = math.log(low + (p.lens[0] + 1 - low) * math.exp(z))
    # (a wave's sum of a row's terms and the sum of waves, an exponential, a logarithm)
    assert np.abs(lse - want).max() <= (p.lens[0] / 4 + 64) * 2.0 ** -24 + 2.0 ** -21 * (1 + want)
    assert int(a.rows.err) == 0


@pytest.mark.parametrize("batch", [1, 2, 70])
def test_lengths_of_sequences_without_rows_are_not_reported(torch, batch):  # noqa: F811
    rng = np.random.default_rng(36)
    for stale in (2 * PAGE + 1, 10 ** 9, -1, 2 ** 31 - 1):
        counts = [0] * batch
        if batch > 1:
            counts[0] = 2
        p = ref.Pass([5] * batch, counts, _trees(rng, counts), 1, stride=2)
        table, pages = ref.table_of(p, rng)
        lens = [5] * (batch - 1) + [stale]
        got = _append(torch, rng, p, table, pages, 2, 1, 64, (32, 0, 0), rows=Rows(torch, p, table, lens=lens))
        _check_append(p, table, pages, 2, 1, 64, (32, 0, 0), 0, 1e4, None, 1, got)
        assert got["err"] == 0
        a = Attn(torch, rng, p, 4, 2, 64, table=table, pages=pages, rows=Rows(torch, p, table, lens=lens))
        a.check()
        assert int(a.rows.err) == 0
        tokens = [0] * p.rows
        got = _commit(torch, rng, p, tokens, tokens, table=table, pages=pages, rows=Rows(torch, p, table, lens=lens))
        assert got["err"] == 0 and got["n"][-1] == 0 and got["new"][-1] == stale
    # with rows they are
    if batch > 1:
        counts[-1] = 1
    else:
        counts = [1]
    p = ref.Pass([5] * batch, counts, _trees(rng, counts), 1, stride=2)
    a = Attn(torch, rng, p, 4, 2, 64, rows=Rows(torch, p, ref.table_of(p, rng)[0], lens=[5] * (batch - 1) + [2 * PAGE + 1]))
    a.run()
    assert int(a.rows.err) == 1


@pytest.mark.parametrize("nq,nkv,D", SHAPES)
@pytest.mark.parametrize("stride", [8, 9])
@pytest.mark.parametrize("slots", [448, 449, 511, 512, 513, 575])
def test_attention_at_the_width_of_a_table_of_one_group(torch, nq, nkv, D, stride, slots):  # noqa: F811
    """Tables of up to eight pages make one group, whose result no second kernel joins."""
    if slots > stride * PAGE:
        slots = stride * PAGE - 1
    rng = np.random.default_rng(37)
    for lens, counts in (([slots - 1], [1]), ([slots - 9], [9]), ([slots - 3, slots - 1, 5, slots - 20], [3, 1, 0, 20])):
        p = ref.Pass(lens, counts, _trees(rng, counts), 1, stride=stride)
        a = Attn(torch, rng, p, nq, nkv, D)
        a.check()
        assert int(a.rows.err) == 0


class Chains(ref.Pass):
    """Long chains, whose rows need no walk."""

    def line(self, b, j):
        return list(range(j + 1))


# heads of a workgroup, 2, 5, 8 and 4 of them, and its last share of the heads, 1, 1, 7 and 3: of passes with enough tiles of
# slots times rotated heads for several, which stream their outputs
@pytest.mark.parametrize("nq,nkv,D,lens,counts,given", [
    (28, 3, 128, [37, 0, 100], [4000, 1, 2002], True), (41, 5, 64, [130, 63], [5000, 3300], False),
    (60, 3, 64, [1, 64, 7, 500], [64, 8000, 100, 136], True), (12, 3, 128, [0], [20000], False)])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_of_many_heads_of_many_rows(torch, nq, nkv, D, lens, counts, given, in_place):  # noqa: F811
    rng = np.random.default_rng(sum(lens) + nq)
    p = Chains(lens, counts, None, 5)
    table, pages = ref.table_of(p, rng)
    pos = rng.integers(0, 5000, (3, p.rows)) if given else None
    section = (D // 8, 3 * D // 16, D // 2 - D // 8 - 3 * D // 16)
    got = _append(torch, rng, p, table, pages, nq, nkv, D, section, pos=pos, pad=8, in_place=in_place)
    assert got["err"] == 0
    _check_append(p, table, pages, nq, nkv, D, section, 0, 10000.0, pos, 1, got, in_place)


@pytest.mark.parametrize("nq,nkv,D", [(31, 4, 128), (28, 4, 128), (62, 4, 64)])
@pytest.mark.parametrize("count", [1, 2])
def test_append_of_many_sequences_of_few_rows(torch, nq, nkv, D, count):  # noqa: F811
    """79 to 160 sequences: a workgroup has several heads here too."""
    rng = np.random.default_rng(nq + count)
    batch = 160 // count
    counts = [count] * (batch - 1) + [0] * (nq == 31)
    lens = [int(x) for x in rng.integers(0, 200, len(counts))]
    p = ref.Pass(lens, counts, _trees(rng, counts), 160 - sum(counts))
    table, pages = ref.table_of(p, rng)
    got = _append(torch, rng, p, table, pages, nq, nkv, D, (D // 2, 0, 0))
    assert got["err"] == 0
    _check_append(p, table, pages, nq, nkv, D, (D // 2, 0, 0), 0, 10000.0, None, 1, got)
