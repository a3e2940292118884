"""Appending to a paged cache, tree attention over it and tree commits against 64-bit references."""
import math

import numpy as np
import pytest

from tests import _tree as ref

pytestmark = pytest.mark.gpu
PAGE = 64
NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _dev(torch, a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def _bits(t):
    return t.cpu().numpy().view(np.uint16)


class Rows:
    """A pass's description on the device."""

    def __init__(self, torch, p, table, parents="of the pass", first=None, lens=None):
        from paper_2606_31160_amd import binding as B
        i32 = lambda x: _dev(torch, np.array(x, np.int32))  # noqa: E731
        self.first, self.len, self.table = i32(first or p.first), i32(lens or p.lens), i32(table)
        flat = p.flat_parents() if p.parents is not None else None
        if not isinstance(parents, str):
            flat = np.array(parents, np.int32)
        self.parent = None if flat is None else i32(flat)
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.desc = B.rows(len(p.lens), p.rows, self.first.data_ptr(), self.len.data_ptr(), self.table.data_ptr(), table.shape[1],
                           0 if self.parent is None else self.parent.data_ptr(), self.err.data_ptr())


def _cache(torch, B, k, v):
    """k [layers, pages, nkv, 64, D], v [layers, pages, nkv, D, 64]: int16 on the device."""
    L, pages, nkv, _, D = k.shape
    return B.kv(nkv, D, pages, k.data_ptr(), v.data_ptr(), L, k.stride(0))


def _random_cache(torch, rng, L, pages, nkv, D):
    k = ref.bf16(rng.standard_normal((L, pages, nkv, PAGE, D)))
    v = ref.bf16(rng.standard_normal((L, pages, nkv, D, PAGE)))
    return k, v


# -- append ------------------------------------------------------------------------

def _append(torch, rng, p, table, pages, nq, nkv, D, section, inter=0, base=10000.0, pos=None, layer=1, pad=0, in_place=False,
            stream=None, rows=None):
    """Runs the operator on random rows; returns what it read and wrote."""
    from paper_2606_31160_amd import binding as B
    k0, v0 = _random_cache(torch, rng, 2, pages, nkv, D)
    qkv = ref.bf16(rng.standard_normal((p.rows, (nq + 2 * nkv) * D + pad)) * np.exp(rng.standard_normal((nq + 2 * nkv) * D + pad)))
    x, k, v = _dev(torch, qkv), _dev(torch, k0), _dev(torch, v0)
    q_out = torch.full((p.rows, max(nq, 1) * D + 8), 0x1234, dtype=torch.int16, device="cuda")
    rows = rows or Rows(torch, p, table)
    dpos = _dev(torch, np.array(pos, np.int32)) if pos is not None else None
    s = stream or torch.cuda.current_stream()
    s.wait_stream(torch.cuda.current_stream())
    at = x.data_ptr()
    B.spec_kv_append(_cache(torch, B, k, v), layer, rows.desc, B.rope(base, section, inter), 0 if dpos is None else dpos.data_ptr(), nq,
                     at if nq else 0, x.stride(0), at + 2 * nq * D, at + 2 * (nq + nkv) * D, x.stride(0),
                     (at if in_place else q_out.data_ptr()) if nq else 0, x.stride(0) if in_place else q_out.stride(0), s.cuda_stream)
    torch.cuda.synchronize()
    return dict(qkv=qkv, k0=k0, v0=v0, k=_bits(k), v=_bits(v), q=_bits(x if in_place else q_out), err=int(rows.err))


def _check_append(p, table, pages, nq, nkv, D, section, inter, base, pos, layer, got, in_place=False):
    """Rotations: cos and sin of an angle that 32 bits hold within pi 2^-24 of a turn's half, themselves within 2^-23, then
    two products and a sum: under 2^-21 (|x0| + |x1|); an angle in 64 bits is off by 3 and here by 5 roundings of 2^-53
    of itself (two powers, a quotient and two products); then half a step of bf16."""
    theta = base ** (-2.0 * np.arange(D // 2) / D)
    ax = ref.axes(D, section, inter)
    k1, v1, q1 = got["k0"].copy(), got["v0"].copy(), None
    x = ref.bf16_value(got["qkv"])[:, :(nq + 2 * nkv) * D].reshape(p.rows, nq + 2 * nkv, D)
    q_out = got["q"]
    touched = np.zeros(got["k0"].shape[:4], bool)
    for b in range(len(p.lens)):
        for j in range(p.counts[b]):
            r, slot = p.first[b] + j, p.lens[b] + j
            at = [p.lens[b] + len(p.line(b, j)) - 1] * 3 if pos is None else [pos[a][r] for a in range(3)]
            want = ref.rotate(x[r, :nq + nkv], theta * np.array([at[a] for a in ax], np.float64))
            mag = np.abs(x[r, :nq + nkv])
            mag = np.repeat(mag[:, 0::2] + mag[:, 1::2], 2, axis=1)
            tol = 2.0 ** -8 * np.abs(want) + 1.01 * (2.0 ** -21 + 8 * 2.0 ** -53 * max(abs(int(x)) for x in at)) * mag
            have = ref.bf16_value(q_out[r, :nq * D]).reshape(nq, D)
            assert (np.abs(have - want[:nq]) <= tol[:nq]).all(), (b, j)
            page = table[b, slot // PAGE] if slot // PAGE < table.shape[1] else -1
            if not 0 <= page < pages:
                continue
            off = slot % PAGE
            have = ref.bf16_value(got["k"][layer, page, :, off])
            assert (np.abs(have - want[nq:]) <= tol[nq:]).all(), (b, j)
            k1[layer, page, :, off] = got["k"][layer, page, :, off]
            v1[layer, page, :, :, off] = got["qkv"][r, (nq + nkv) * D:(nq + 2 * nkv) * D].reshape(nkv, D)
    np.testing.assert_array_equal(got["k"], k1)          # and nothing else
    np.testing.assert_array_equal(got["v"], v1)
    if not in_place:
        assert (q_out[p.n:] == 0x1234).all() and (q_out[:, nq * D:] == 0x1234).all()
    else:
        np.testing.assert_array_equal(q_out[:, nq * D:], got["qkv"][:, nq * D:])
        np.testing.assert_array_equal(q_out[p.n:], got["qkv"][p.n:])


HEADS = [(4, 2, 64), (7, 1, 128), (28, 4, 128), (8, 8, 64), (0, 3, 128), (5, 2, 64)]


def _section(D):
    return (D // 8, 3 * D // 16, D // 2 - D // 8 - 3 * D // 16)


@pytest.mark.parametrize("nq,nkv,D", HEADS)
@pytest.mark.parametrize("lens,counts,behind", [
    ([320], [1], 0), ([0], [1], 0), ([63], [2], 3), ([0, 64, 5, 127], [3, 0, 9, 1], 2), ([61, 130], [70, 11], 0),
    ([1] * 20, [1, 2] * 10, 1)])
def test_append_follows_the_trees(torch, nq, nkv, D, lens, counts, behind):
    rng = np.random.default_rng(sum(lens) + sum(counts) + nq)
    p = ref.Pass(lens, counts, [ref.random_tree(rng, c) if c else [] for c in counts], behind)
    table, pages = ref.table_of(p, rng)
    got = _append(torch, rng, p, table, pages, nq, nkv, D, _section(D), pad=8)
    assert got["err"] == 0
    _check_append(p, table, pages, nq, nkv, D, _section(D), 0, 10000.0, None, 1, got)


@pytest.mark.parametrize("D,section,inter,base", [
    (128, (16, 24, 24), 0, 10000.0), (128, (24, 20, 20), 1, 10000.0), (64, (32, 0, 0), 0, 1e6), (64, (0, 32, 0), 0, 10000.0),
    (128, (0, 0, 64), 0, 500.0), (64, (8, 0, 24), 0, 10000.0), (64, (8, 24, 0), 0, 1.5), (64, (32, 0, 0), 1, 10000.0)])
@pytest.mark.parametrize("far", [0, 100_000, 2 ** 31 - 1])
def test_append_rotates_by_any_positions(torch, D, section, inter, base, far):
    rng = np.random.default_rng(3)
    p = ref.Pass([7, 200], [130, 67], None, 5)
    table, pages = ref.table_of(p, rng)
    pos = rng.integers(0, 700, (3, p.rows)) if not far else far - rng.integers(0, 1000, (3, p.rows))
    pos[1] *= -1
    got = _append(torch, rng, p, table, pages, 4, 2, D, section, inter, base, pos)
    assert got["err"] == 0
    _check_append(p, table, pages, 4, 2, D, section, inter, base, pos, 1, got)


def test_append_of_a_long_chain(torch):
    rng = np.random.default_rng(4)
    p = ref.Pass([37, 0, 100], [1000, 1, 333], None, 9)
    table, pages = ref.table_of(p, rng)
    for pos in (None, rng.integers(0, 5000, (3, p.rows))):
        got = _append(torch, rng, p, table, pages, 6, 2, 128, (16, 24, 24), pos=pos)
        assert got["err"] == 0
        _check_append(p, table, pages, 6, 2, 128, (16, 24, 24), 0, 10000.0, pos, 1, got)


def test_append_in_place_and_on_another_stream(torch):
    rng = np.random.default_rng(5)
    p = ref.Pass([10, 90], [5, 80], [ref.random_tree(rng, 5), ref.random_tree(rng, 80)], 2)
    table, pages = ref.table_of(p, rng)
    got = _append(torch, rng, p, table, pages, 4, 2, 128, (16, 24, 24), in_place=True, stream=torch.cuda.Stream())
    _check_append(p, table, pages, 4, 2, 128, (16, 24, 24), 0, 10000.0, None, 1, got, in_place=True)


def test_append_of_values_that_are_not_finite_copies_them(torch):
    """Values are moved as they are; a pair's rotation is NaN only where the formula's is, and other pairs do not notice."""
    from paper_2606_31160_amd import binding as B
    p = ref.Pass([0], [2], None)
    x = np.ones((2, 3 * 64))
    x[0, 2], x[0, 64 + 5], x[0, 128 + 7], x[1, 128 + 9] = NAN, INF, NAN, -INF
    bits, rng = ref.bf16(x), np.random.default_rng(0)
    table = np.array([[0]], np.int32)
    k, v = (_dev(torch, a) for a in _random_cache(torch, rng, 1, 1, 1, 64))
    d, q = _dev(torch, bits), torch.zeros(2, 64, dtype=torch.int16, device="cuda")
    rows = Rows(torch, p, table)
    B.spec_kv_append(_cache(torch, B, k, v), 0, rows.desc, B.rope(1e4, (32, 0, 0)), 0, 1, d.data_ptr(), 192, d.data_ptr() + 128, d.data_ptr() + 256,
                     192, q.data_ptr(), 64)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(_bits(v)[0, 0, 0, :, :2].T, bits[:, 128:])
    fine = np.isfinite(ref.bf16_value(_bits(q)))
    assert not fine[0, 2:4].any() and fine[0, :2].all() and fine[0, 4:].all() and fine[1].all()
    fine = np.isfinite(ref.bf16_value(_bits(k)[0, 0, 0, :2]))
    assert not fine[0, 4:6].any() and fine[0, :4].all() and fine[0, 6:].all() and fine[1].all()


def test_append_stays_in_bounds_of_tables_and_pools(torch):
    """Pages outside the pool and slots past the table are not written, and the rest is; a broken d_first writes nothing."""
    rng = np.random.default_rng(6)
    p = ref.Pass([60, 100, 0], [10, 40, 3], None, 1, stride=2)
    table, pages = ref.table_of(ref.Pass([60, 88, 0], [10, 40, 3], None, 1), rng)
    table[0, 1], table[2, 0] = pages, -5
    got = _append(torch, rng, p, table, pages, 4, 2, 64, (32, 0, 0))
    assert got["err"] == 1
    _check_append(p, table, pages, 4, 2, 64, (32, 0, 0), 0, 10000.0, None, 1, got)
    for first, lens in (([0, 10, 5, 53], None), ([-1, 10, 50, 53], None), ([0, 10, 50, 55], None)):
        got = _append(torch, rng, p, table, pages, 4, 2, 64, (32, 0, 0), rows=Rows(torch, p, table, first=first, lens=lens))
        assert got["err"] == 1
        np.testing.assert_array_equal(got["k"], got["k0"])
        np.testing.assert_array_equal(got["v"], got["v0"])
        assert (got["q"] == 0x1234).all()
    got = _append(torch, rng, p, table, pages, 4, 2, 64, (32, 0, 0), rows=Rows(torch, p, table, lens=[-1, 100, 129]))
    assert got["err"] == 1
    q = ref.Pass([0, 100, 0], [0, 40, 0], None, 1, stride=2)
    assert (got["q"][:10] == 0x1234).all() and (got["q"][50:] == 0x1234).all() and (got["q"][10:50, :256] != 0x1234).any()
    assert (got["k"] != got["k0"]).any(axis=(0, 2, 3, 4)).sum() == 1, q    # the page of slots 100 .. 127


def test_append_takes_broken_parents_as_roots(torch):
    rng = np.random.default_rng(7)
    p = ref.Pass([5], [6], [[-1, 0, -1, 2, -1, -1]])
    table, pages = ref.table_of(p, rng)
    got = _append(torch, rng, p, table, pages, 2, 1, 64, (32, 0, 0), rows=Rows(torch, p, table, parents=[-1, 0, 7, 2, 4, -2]))
    assert got["err"] == 1
    _check_append(p, table, pages, 2, 1, 64, (32, 0, 0), 0, 10000.0, None, 1, got)


def test_append_of_many_rows_of_trees_at_given_positions(torch):
    """Positions say where rows stand, so trees may be larger than a pass that is attended."""
    rng = np.random.default_rng(8)
    counts = [200, 150]
    p = ref.Pass([30, 61], counts, [ref.random_tree(rng, c) for c in counts], 3)
    table, pages = ref.table_of(p, rng)
    pos = rng.integers(0, 9000, (3, p.rows))
    got = _append(torch, rng, p, table, pages, 6, 2, 128, (16, 24, 24), pos=pos)
    assert got["err"] == 0
    _check_append(p, table, pages, 6, 2, 128, (16, 24, 24), 0, 10000.0, pos, 1, got)


# -- attention ---------------------------------------------------------------------

class Attn:
    """Inputs of one call and its outputs, run once or more."""

    def __init__(self, torch, rng, p, nq, nkv, D, scale=None, layers=2, layer=1, q_pad=0, out_pad=0, table=None, pages=None, k=None,
                 v=None, q=None, rows=None, lse=True):
        from paper_2606_31160_amd import binding as B
        self.torch, self.B, self.p, self.nq, self.nkv, self.D, self.layer = torch, B, p, nq, nkv, D, layer
        self.scale = D ** -0.5 if scale is None else scale
        if table is None:
            table, pages = ref.table_of(p, rng)
        self.table, self.pages = table, pages
        if k is None:
            k, v = _random_cache(torch, rng, layers, pages, nkv, D)
            # nothing but the slots in use holds numbers
            used = np.zeros((pages, PAGE), bool)
            for b in range(len(p.lens)):
                for s in range(p.lens[b] + p.counts[b]):
                    if s // PAGE < table.shape[1] and 0 <= table[b, s // PAGE] < pages:
                        used[table[b, s // PAGE], s % PAGE] = True
            k[np.broadcast_to(~used[None, :, None, :, None], k.shape)] = 0x7FC0
            v[np.broadcast_to(~used[None, :, None, None, :], v.shape)] = 0xFF80
        self.k, self.v = k, v
        self.q = ref.bf16(rng.standard_normal((p.rows, nq * D + q_pad))) if q is None else q
        self.dk, self.dv, self.dq = _dev(torch, k), _dev(torch, v), _dev(torch, self.q)
        self.rows = rows or Rows(torch, p, table)
        self.out = torch.full((p.rows, nq * D + out_pad), 0x1234, dtype=torch.int16, device="cuda")
        self.lse = torch.full((p.rows, nq), -7.0, device="cuda") if lse else None
        self.cache = _cache(torch, B, self.dk, self.dv)
        n = B.spec_tree_attn_workspace_bytes(self.cache, self.rows.desc, nq)
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")

    def call(self, stream=None):
        s = stream or self.torch.cuda.current_stream()
        self.B.spec_tree_attn(self.cache, self.layer, self.rows.desc, self.nq, self.dq.data_ptr(), self.dq.stride(0), self.scale, self.out.data_ptr(),
                              self.out.stride(0), 0 if self.lse is None else self.lse.data_ptr(), self.ws.data_ptr(), self.ws.numel(), s.cuda_stream)

    def run(self):
        self.call()
        self.torch.cuda.synchronize()
        return _bits(self.out), None if self.lse is None else self.lse.cpu().numpy()

    def slots(self, b, j):
        """Slots that row j of sequence b sees, of those with a page."""
        s = list(range(self.p.lens[b])) + [self.p.lens[b] + i for i in self.p.line(b, j)]
        return [x for x in s if x // PAGE < self.table.shape[1] and 0 <= self.table[b, x // PAGE] < self.pages]

    def check(self, only=None):
        out, lse = self.run()
        p, D, G = self.p, self.D, self.nq // self.nkv
        for b in range(len(p.lens)):
            for j in range(p.counts[b]):
                if only and (b, j) not in only:
                    continue
                s = np.array(self.slots(b, j), int)
                r = p.first[b] + j
                pg, off = self.table[b, s // PAGE], s % PAGE
                for h in range(self.nq):
                    have = ref.bf16_value(out[r, h * D:(h + 1) * D])
                    if not len(s):
                        assert np.isnan(have).all() and (lse is None or lse[r, h] == -INF), (b, j, h)
                        continue
                    k = ref.bf16_value(self.k[self.layer, pg, h // G, off])
                    v = ref.bf16_value(self.v[self.layer, pg, h // G, :, off])
                    q = ref.bf16_value(self.q[r, h * D:(h + 1) * D])
                    w, l, absum, big = ref.attention(q, k, v, self.scale)
                    fine = np.isfinite(v)
                    tol, ltol = ref.attention_bounds(w, l, absum, big, D, len(s), np.abs(v[fine]).max(initial=0))
                    fin = np.isfinite(w)
                    np.testing.assert_array_equal(have[~fin], w[~fin], err_msg=str((b, j, h)))
                    off_by = np.abs(have - np.where(fin, w, 0))[fin]
                    assert (off_by <= tol[fin]).all(), (b, j, h, float((off_by / np.maximum(tol[fin], 1e-300)).max()))
                    if lse is not None and np.isfinite(l):
                        assert abs(lse[r, h] - l) <= ltol, (b, j, h, lse[r, h], l)
        assert (out[p.n:] == 0x1234).all() and (out[:, self.nq * D:] == 0x1234).all()
        assert lse is None or (lse[p.n:] == -7).all()
        return out, lse


def _trees(rng, counts, wide=3):
    return [ref.random_tree(rng, c, wide) if c else [] for c in counts]


A_HEADS = [(4, 2, 64), (7, 1, 128), (28, 4, 128), (8, 8, 64), (24, 1, 128), (2, 2, 128)]


@pytest.mark.parametrize("nq,nkv,D", A_HEADS)
@pytest.mark.parametrize("length", [0, 1, 63, 64, 65, 320, 1000])
@pytest.mark.parametrize("count", [1, 5, 40])
def test_attention_of_one_tree(torch, nq, nkv, D, length, count):
    rng = np.random.default_rng(length + count)
    p = ref.Pass([length], [count], _trees(rng, [count]))
    a = Attn(torch, rng, p, nq, nkv, D)
    a.check()
    assert int(a.rows.err) == 0


@pytest.mark.parametrize("nq,nkv,D", [(4, 2, 64), (7, 1, 128), (4, 4, 128)])
def test_attention_of_ragged_trees(torch, nq, nkv, D):
    rng = np.random.default_rng(11)
    lens, counts = [0, 500, 64, 1, 2000, 129, 63, 10], [7, 1, 0, 30, 12, 3, 2, 64]
    a = Attn(torch, rng, ref.Pass(lens, counts, _trees(rng, counts), 5), nq, nkv, D, q_pad=16, out_pad=8)
    a.check()
    assert int(a.rows.err) == 0


def test_attention_of_chains_is_causal(torch):
    rng = np.random.default_rng(12)
    Attn(torch, rng, ref.Pass([100, 0, 1], [17, 70, 9], None, 3), 4, 2, 64).check()
    Attn(torch, rng, ref.Pass([0], [160], None), 4, 2, 64, lse=False).check()


@pytest.mark.parametrize("length", [0, 40, 100])
def test_attention_of_the_largest_tree(torch, length):
    """160 rows, whose ancestors fill three words; bushy, several roots, and one row behind another."""
    rng = np.random.default_rng(13)
    for tree in (ref.random_tree(rng, 160, 40), ref.random_tree(rng, 160, roots=True), [j - 1 for j in range(160)], [-1] + [0] * 159):
        Attn(torch, rng, ref.Pass([length], [160], [tree]), 4, 2, 64).check()


def test_attention_of_many_sequences(torch):
    rng = np.random.default_rng(14)
    lens = [int(x) for x in rng.integers(0, 200, 160)]
    Attn(torch, rng, ref.Pass(lens, [1] * 160, None), 4, 2, 64).check()
    counts = [int(x) for x in rng.integers(0, 2, 150)]
    Attn(torch, rng, ref.Pass(lens[:150], counts, _trees(rng, counts), 4, stride=6), 2, 1, 128).check()


@pytest.mark.parametrize("nq,nkv,D,lens,counts", [
    (28, 4, 128, [4096], [9]), (32, 8, 128, [4117], [17]), (7, 1, 128, [20000], [6]), (28, 4, 128, [2100, 8000, 64, 5000], [9, 12, 1, 16]),
    (24, 1, 128, [9000], [3]), (8, 8, 64, [3000, 700], [64, 20]), (8, 1, 64, [30000], [33])])
def test_attention_over_long_caches(torch, nq, nkv, D, lens, counts):
    rng = np.random.default_rng(sum(lens))
    p = ref.Pass(lens, counts, _trees(rng, counts), stride=max(lens) // PAGE + 9)
    rows = [(b, j) for b in range(len(lens)) for j in sorted({0, counts[b] // 2, counts[b] - 1})]
    Attn(torch, rng, p, nq, nkv, D).check(rows)


def test_what_a_row_does_not_see_has_no_influence(torch):
    """Siblings' keys and values of NaN and infinities, and a table whose other entries lead nowhere."""
    rng = np.random.default_rng(15)
    tree = [-1, 0, 0, 1, 2, 3, 4]
    p = ref.Pass([100], [7], [tree], stride=9)
    for off, what in ((1, NAN), (3, INF), (5, -INF)):
        a = Attn(torch, rng, p, 4, 2, 128)
        slot = 100 + off
        page = a.table[0, slot // PAGE]
        a.k[1, page, :, slot % PAGE, ::7] = ref.bf16(np.array(what))
        a.v[1, page, :, ::5, slot % PAGE] = ref.bf16(np.array(what))
        a.dk, a.dv = _dev(torch, a.k), _dev(torch, a.v)
        a.cache = _cache(torch, a.B, a.dk, a.dv)
        a.check([(0, j) for j in range(7) if off not in p.line(0, j)])


@pytest.mark.parametrize("length", [150, 3000])
def test_a_key_of_nan_is_nan_for_the_rows_that_see_it(torch, length):
    rng = np.random.default_rng(23)
    p = ref.Pass([length], [5], [[-1, 0, 0, 1, 2]])
    for slots, rows in (([length + 1], [1, 3]), (range(0, length // 2), range(5))):
        a = Attn(torch, rng, p, 4, 2, 128)
        for s in slots:
            a.k[1, a.table[0, s // PAGE], 0, s % PAGE] = 0x7FC0       # of the first kv head only
        a.dk = _dev(torch, a.k)
        a.cache = _cache(torch, a.B, a.dk, a.dv)
        out, lse = a.run()
        out = ref.bf16_value(out).reshape(5, 4, 128)
        for j in range(5):
            assert np.isnan(out[j, :2]).all() == np.isnan(lse[j, :2]).all() == (j in rows)
            assert np.isfinite(out[j, 2:]).all() and np.isfinite(lse[j, 2:]).all()
        a.check([(0, j) for j in range(5) if j not in rows])


def test_a_pass_without_rows_does_nothing(torch):
    rng = np.random.default_rng(24)
    for p in (ref.Pass([10, 20], [0, 0], [[], []], 3), ref.Pass([10], [0], None, 1)):
        table, pages = ref.table_of(p, rng)
        got = _append(torch, rng, p, table, pages, 2, 1, 64, (32, 0, 0))
        _check_append(p, table, pages, 2, 1, 64, (32, 0, 0), 0, 1e4, None, 1, got)
        a = Attn(torch, rng, p, 4, 2, 64)
        a.check()
        got = _commit(torch, rng, p, [0] * p.rows, [0] * p.rows)
        _check_commit(p, [0] * p.rows, [[] for _ in p.lens], got)
        assert got["err"] == int(a.rows.err) == 0


def test_one_bad_length_among_many_sequences(torch):
    """Sequence 130 of 150 has none: it is reported and has no rows, the others have theirs."""
    rng = np.random.default_rng(25)
    lens = [int(x) for x in rng.integers(0, 100, 150)]
    p = ref.Pass(lens, [1] * 150, None, 2, stride=2)
    table, pages = ref.table_of(p, rng)
    bad = list(lens)
    bad[130] = 129
    got = _append(torch, rng, p, table, pages, 2, 1, 64, (32, 0, 0), rows=Rows(torch, p, table, lens=bad))
    assert got["err"] == 1 and (got["q"][130] == 0x1234).all()
    q = ref.bf16_value(got["q"][:, :128])
    assert np.isfinite(q[:130]).all() and (got["q"][131:150, :128] != 0x1234).any(axis=1).all()
    a = Attn(torch, rng, p, 4, 2, 64, table=table, pages=pages)
    a.rows = Rows(torch, p, table, lens=bad)
    out, lse = a.run()
    assert int(a.rows.err) == 1 and (out[130] == 0x1234).all() and (lse[130] == -7).all()
    want_out, want_lse = Attn(torch, rng, p, 4, 2, 64, table=table, pages=pages, k=a.k, v=a.v, q=a.q).run()
    others = [r for r in range(150) if r != 130]
    np.testing.assert_allclose(ref.bf16_value(out[others]), ref.bf16_value(want_out[others]), rtol=2.0 ** -7, atol=1e-6)
    got = _commit(torch, rng, p, [0] * p.rows, [0] * p.rows, table=table, pages=pages, rows=Rows(torch, p, table, lens=bad))
    assert got["err"] == 1 and got["n"] == [int(b != 130) for b in range(150)]


@pytest.mark.parametrize("nq,nkv,D", [(4, 2, 64), (14, 2, 128)])
@pytest.mark.parametrize("lens", [[150], [3000], [40, 700]])
def test_infinite_values_that_a_row_sees(torch, nq, nkv, D, lens):
    rng = np.random.default_rng(16)
    counts = [6] * len(lens)
    p = ref.Pass(lens, counts, [[-1, 0, 0, 1, 2, 3]] * len(lens), 2)
    a = Attn(torch, rng, p, nq, nkv, D)
    for b in range(len(lens)):
        # everybody's, one branch's, one row's; both signs in one dimension; NaN
        for slot, d, x in ((0, 0, INF), (lens[b] - 1, 1, -INF), (5, 2, INF), (6, 2, -INF), (lens[b] + 1, 3, INF), (lens[b] + 2, 3, -INF),
                           (lens[b] + 5, 4, -INF), (lens[b] // 2, 5, NAN), (lens[b] + 2, 6, NAN), (lens[b] - 3, 7, INF)):
            a.v[1, a.table[b, slot // PAGE], :, d, slot % PAGE] = ref.bf16(np.array(x))
    # a slot that holds an infinity has next to no weight
    a.k[1, a.table[0, 0], :, 0] = ref.bf16(-ref.bf16_value(a.q[0, :D]) * 40)
    a.dk, a.dv = _dev(torch, a.k), _dev(torch, a.v)
    a.cache = _cache(torch, a.B, a.dk, a.dv)
    a.check()


@pytest.mark.parametrize("nq,nkv,D,lens,count", [
    (28, 4, 128, [5000] + [70] * 15, 9), (16, 8, 64, [2500] + [3] * 31, 5),      # a group or two of a sequence were likely
    (28, 4, 128, [9000], 1), (7, 1, 128, [20000], 12)])                          # many groups
def test_infinite_values_in_some_of_many_groups(torch, nq, nkv, D, lens, count):
    rng = np.random.default_rng(26)
    p = ref.Pass(lens, [count] * len(lens), _trees(rng, [count] * len(lens)), stride=max(lens) // PAGE + 2)
    a = Attn(torch, rng, p, nq, nkv, D)
    n = lens[0]
    for slot, d, x in ((0, 0, INF), (n - 1, 0, INF), (n // 2, 1, -INF), (n // 3, 2, INF), (n // 4, 2, -INF), (n // 5, 3, NAN),
                       (n + count - 1, 4, INF), (n + count // 2, D - 1, -INF)):
        a.v[1, a.table[0, slot // PAGE], :, d, slot % PAGE] = ref.bf16(np.array(x))
    a.dv = _dev(torch, a.v)
    a.cache = _cache(torch, a.B, a.dk, a.dv)
    a.check([(0, j) for j in {0, count // 2, count - 1}] + [(len(lens) - 1, j) for j in {0, count - 1}])


@pytest.mark.parametrize("count", [1, 2, 4])
@pytest.mark.parametrize("nq,nkv,D", [(28, 4, 128), (6, 2, 64)])
def test_attention_of_one_long_sequence_among_many_without_rows(torch, nq, nkv, D, count):
    """Few groups were likely, and there are many: of tiles of 3 to 28 rows."""
    rng = np.random.default_rng(28)
    counts = [0] * 30 + [count] + [0] * 49
    p = ref.Pass([12000 if c else 5 for c in counts], counts, _trees(rng, counts), 20)
    a = Attn(torch, rng, p, nq, nkv, D)
    for slot, d, x in ((100, 0, INF), (11900, 0, INF), (5000, 1, -INF), (7000, 2, NAN)):
        a.v[1, a.table[30, slot // PAGE], 0, d, slot % PAGE] = ref.bf16(np.array(x))
    a.dv = _dev(torch, a.v)
    a.cache = _cache(torch, a.B, a.dk, a.dv)
    a.check()
    assert int(a.rows.err) == 0


@pytest.mark.parametrize("nq,nkv,D,lens,counts", [
    (1024, 2, 64, [700], [2]), (300, 300, 64, [40, 700], [1, 2]), (96, 48, 128, [600, 0, 130], [5, 1, 1]), (640, 1, 128, [1], [40])])
def test_attention_of_many_heads(torch, nq, nkv, D, lens, counts):
    rng = np.random.default_rng(27)
    a = Attn(torch, rng, ref.Pass(lens, counts, _trees(rng, counts), 1, stride=max(12, max(lens) // PAGE + 1)), nq, nkv, D)
    a.check([(b, j) for b, c in enumerate(counts) for j in {0, c - 1}])
    assert int(a.rows.err) == 0


@pytest.mark.parametrize("lens", [[150], [3000]])
def test_values_at_the_ends_of_their_range(torch, lens):
    """The largest bf16 values, whose sums leave the range, and the smallest normal ones."""
    rng = np.random.default_rng(17)
    p = ref.Pass(lens, [5], [[-1, 0, 0, 1, 2]])
    for x in (255 * 2.0 ** 120, 2.0 ** -100, 2.0 ** -125):
        a = Attn(torch, rng, p, 4, 2, 64)
        finite = np.isfinite(ref.bf16_value(a.v))
        a.v[finite] = ref.bf16(x * np.where(rng.random(a.v.shape) < 0.95, 1, 0.5))[finite]
        a.dv = _dev(torch, a.v)
        a.cache = _cache(torch, a.B, a.dk, a.dv)
        a.check()


@pytest.mark.parametrize("scale", [1e-30, 0.5, 40.0])
def test_scores_of_any_size(torch, scale):
    rng = np.random.default_rng(18)
    Attn(torch, rng, ref.Pass([300, 70], [9, 4], _trees(rng, [9, 4])), 4, 2, 64, scale=scale).check()


def test_scores_that_grow_and_fall_along_the_cache(torch):
    rng = np.random.default_rng(19)
    for sign in (1, -1):
        a = Attn(torch, rng, ref.Pass([2500], [4], [[-1, 0, 1, 0]]), 4, 2, 64)
        ramp = np.exp(sign * np.linspace(-3, 3, a.table.shape[1]))
        for i, f in enumerate(ramp):
            k = ref.bf16_value(a.k[1, a.table[0, i]])
            a.k[1, a.table[0, i]] = np.where(np.isnan(k), np.uint16(0x7FC0), ref.bf16(np.abs(np.nan_to_num(k)) * f * (1 if i % 2 else -1)))
        a.dk = _dev(torch, a.k)
        a.cache = _cache(torch, a.B, a.dk, a.dv)
        a.check()


def test_attention_stays_in_bounds(torch):
    rng = np.random.default_rng(20)
    # pages outside the pool; then slots past the table
    p = ref.Pass([200, 120, 0], [5, 20, 3], None, 1, stride=4)
    whole = ref.Pass([200, 108, 0], [5, 20, 3], None, 1, stride=4)
    table, pages = ref.table_of(whole, rng)
    table[0, 1], table[1, 2:], table[2, 0] = pages, -1, -9
    a = Attn(torch, rng, p, 4, 2, 64, table=table, pages=pages)
    a.check()
    assert int(a.rows.err) == 1
    p = ref.Pass([120, 64], [20, 3], _trees(rng, [20, 3]))
    table, pages = ref.table_of(ref.Pass([108, 64], [20, 3], None), rng)
    a = Attn(torch, rng, p, 4, 2, 64, table=table, pages=pages)
    a.check()
    assert int(a.rows.err) == 1 and table.shape[1] == 2
    # broken descriptions leave everything as it was
    good = ref.Pass([20, 30], [4, 4], None, 1)
    for first, lens in (([0, 9, 8], None), ([-1, 4, 8], None), ([0, 4, 10], None), (None, [-1, 200])):
        a = Attn(torch, rng, good, 4, 2, 64)
        a.rows = Rows(torch, good, a.table, first=first, lens=lens)
        out, lse = a.run()
        assert int(a.rows.err) == 1 and (out == 0x1234).all() and (lse == -7).all()
    # broken parents are roots
    good = ref.Pass([70], [6], [[-1, 0, -1, 2, -1, -1]])
    table, pages = ref.table_of(good, rng)
    a = Attn(torch, rng, good, 4, 2, 64, table=table, pages=pages, rows=Rows(torch, good, table, parents=[-1, 0, 7, 2, 4, -2]))
    a.check()
    assert int(a.rows.err) == 1


def test_attention_of_a_pool_beyond_32_bits(torch):
    """Element offsets of the last pages exceed 2^32."""
    from paper_2606_31160_amd import binding as B
    nkv, D = 4, 128
    pages = (1 << 32) // (nkv * PAGE * D) + 300
    k = torch.empty(1, pages, nkv, PAGE, D, dtype=torch.int16, device="cuda")
    v = torch.empty(1, pages, nkv, D, PAGE, dtype=torch.int16, device="cuda")
    rng = np.random.default_rng(21)
    p = ref.Pass([100], [5], [[-1, 0, 0, 1, 2]])
    small, n = _random_cache(torch, rng, 1, 2, nkv, D), 2
    at = [pages - 1, pages - 200]
    for i in range(n):
        k[0, at[i]], v[0, at[i]] = _dev(torch, small[0][0, i]), _dev(torch, small[1][0, i])
    a = Attn(torch, rng, p, 8, nkv, D, layers=1, layer=0, table=np.array([[0, 1]], np.int32), pages=2, k=small[0], v=small[1])
    want, wlse = a.check()
    far = np.array([at], np.int32)
    a.rows = Rows(torch, p, far)
    a.cache = B.kv(nkv, D, pages, k.data_ptr(), v.data_ptr())
    got, glse = a.run()
    np.testing.assert_array_equal(got, want)
    np.testing.assert_array_equal(glse, wlse)
    # ... and append and commit reach them
    x = _dev(torch, ref.bf16(rng.standard_normal((5, 2 * nkv * D))))
    near_k, near_v = _dev(torch, small[0]), _dev(torch, small[1])
    tok = torch.tensor([0, 1, 2, 3, 4], dtype=torch.int32, device="cuda")
    greedy = torch.tensor([2, 9, 4, 9, 9], dtype=torch.int32, device="cuda")
    for cache, rows in ((a.cache, a.rows), (B.kv(nkv, D, 2, near_k.data_ptr(), near_v.data_ptr()), Rows(torch, p, np.array([[0, 1]], np.int32)))):
        B.spec_kv_append(cache, 0, rows.desc, B.rope(1e4, (16, 24, 24)), 0, 0, 0, 0, x.data_ptr(), x.data_ptr() + 2 * nkv * D, x.stride(0), 0, 0)
        B.spec_tree_commit(cache, rows.desc, tok.data_ptr(), greedy.data_ptr())
        torch.cuda.synchronize()
        assert int(rows.err) == 0
    for i in range(n):
        assert torch.equal(k[0, at[i]], near_k[0, i]) and torch.equal(v[0, at[i]], near_v[0, i])
    assert not torch.equal(near_k[0, 1], _dev(torch, small[0][0, 1]))


def test_attention_repeats_itself_and_runs_on_two_streams(torch):
    rng = np.random.default_rng(22)
    counts = [9, 20, 1]
    p = ref.Pass([3000, 500, 90], counts, _trees(rng, counts))
    a, b = Attn(torch, rng, p, 28, 4, 128), Attn(torch, rng, p, 28, 4, 128)
    want = [x.run() for x in (a, b)]
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    for x in (a, b):
        x.out.fill_(0)
    torch.cuda.synchronize()
    for _ in range(5):
        a.call(s[0])
        b.call(s[1])
    torch.cuda.synchronize()
    for x, (out, lse) in zip((a, b), want):
        np.testing.assert_array_equal(_bits(x.out), out)
        np.testing.assert_array_equal(x.lse.cpu().numpy(), lse)


# -- commit ------------------------------------------------------------------------

def _commit(torch, rng, p, tokens, greedy, layers=3, nkv=2, D=64, stop=-1, budget=None, table=None, pages=None, rows=None, outs=True):
    from paper_2606_31160_amd import binding as B
    if table is None:
        table, pages = ref.table_of(p, rng)
    k0, v0 = _random_cache(torch, rng, layers, pages, nkv, D)
    k, v = _dev(torch, k0), _dev(torch, v0)
    rows = rows or Rows(torch, p, table)
    i32 = lambda x: _dev(torch, np.array(x, np.int32))  # noqa: E731
    tok, gre, bud = i32(tokens), i32(greedy), None if budget is None else i32(budget)
    path, com, n, new = (i32([-9] * m) for m in (p.rows, p.rows, len(p.lens), len(p.lens)))
    at = lambda t: t.data_ptr() if outs else 0  # noqa: E731
    B.spec_tree_commit(_cache(torch, B, k, v), rows.desc, tok.data_ptr(), gre.data_ptr(), stop, 0 if bud is None else bud.data_ptr(),
                       at(path), at(com), at(n), at(new))
    torch.cuda.synchronize()
    return dict(k0=k0, v0=v0, k=_bits(k), v=_bits(v), path=path.tolist(), committed=com.tolist(), n=n.tolist(), new=new.tolist(), err=int(rows.err),
                table=table, pages=pages)


def _check_commit(p, greedy, taken, got, outs=True):
    k, v, table = got["k0"].copy(), got["v0"].copy(), got["table"]
    path, com = [-9] * p.rows, [-9] * p.rows
    for b, rows in enumerate(taken):
        for i, j in enumerate(rows):
            path[p.first[b] + i], com[p.first[b] + i] = j, greedy[p.first[b] + j]
            src, dst = p.lens[b] + j, p.lens[b] + i
            pages = [table[b, s // PAGE] if s // PAGE < table.shape[1] else -1 for s in (src, dst)]
            if all(0 <= x < got["pages"] for x in pages):
                k[:, pages[1], :, dst % PAGE] = k[:, pages[0], :, src % PAGE]
                v[:, pages[1], :, :, dst % PAGE] = v[:, pages[0], :, :, src % PAGE]
    np.testing.assert_array_equal(got["k"], k)
    np.testing.assert_array_equal(got["v"], v)
    if outs:
        assert got["path"] == path and got["committed"] == com
        assert got["n"] == [len(t) for t in taken] and got["new"] == [l + len(t) for l, t in zip(p.lens, taken)]


def _tokens(rng, p, choices=3):
    """Few different tokens, so that siblings share some and paths go on for a while."""
    return [int(x) for x in rng.integers(0, choices, p.rows)], [int(x) for x in rng.integers(0, choices, p.rows)]


@pytest.mark.parametrize("seed", range(12))
def test_commit_of_random_trees(torch, seed):
    rng = np.random.default_rng(seed)
    counts = [int(x) for x in rng.integers(0, 30, 5)]
    lens = [int(x) for x in rng.integers(0, 200, 5)]
    p = ref.Pass(lens, counts, _trees(rng, counts, 6), int(rng.integers(0, 9)))
    tokens, greedy = _tokens(rng, p, 1 + seed % 4)
    D = (64, 128)[seed % 2]
    got = _commit(torch, rng, p, tokens, greedy, layers=1 + seed % 3, nkv=1 + seed % 4, D=D)
    assert got["err"] == 0
    _check_commit(p, greedy, ref.commit(p, tokens, greedy), got)


@pytest.mark.parametrize("length", [0, 40, 63])
def test_commit_of_long_paths(torch, length):
    """Every slot is read by one step and written by another, over page borders; and a chain, which moves nothing."""
    rng = np.random.default_rng(30)
    for tree in ([-1, 0] + [j - 1 if j % 2 else j - 2 for j in range(2, 160)], [-1, 0, 0] + [j - 1 for j in range(3, 160)], [j - 1 for j in range(160)],
                 [-1, 0, 0, 0] + [max(0, j - 1) for j in range(4, 160)]):
        p = ref.Pass([length], [160], [tree])
        deepest = max(range(160), key=lambda j: len(p.line(0, j)))
        path = p.line(0, deepest)
        tokens, greedy = [5] * 160, [9] * 160
        for i, j in zip(path, path[1:]):
            greedy[i] = tokens[j] = 100 + j
        got = _commit(torch, rng, p, tokens, greedy, D=128)
        want = ref.commit(p, tokens, greedy)
        assert want[0] == path
        _check_commit(p, greedy, want, got)


def test_commit_of_chains_and_without_outputs(torch):
    rng = np.random.default_rng(31)
    p = ref.Pass([10, 64, 0], [9, 1, 4], None, 2)
    tokens, greedy = _tokens(rng, p, 1)
    got = _commit(torch, rng, p, tokens, greedy)
    _check_commit(p, greedy, [list(range(9)), [0], list(range(4))], got)
    got = _commit(torch, rng, p, tokens, greedy, outs=False)
    _check_commit(p, greedy, [[0], [0], [0]], got, outs=False)


def test_layers_apart_and_no_word_for_errors(torch):
    """Layers with room between them, which stays as it was; and passes with faults that nobody asked to hear of."""
    from paper_2606_31160_amd import binding as B
    rng = np.random.default_rng(35)
    p = ref.Pass([60, 5], [6, 3], [[-1, 0, 0, 2, 2, 4], [-1, 0, 0]], 1)
    table, pages = ref.table_of(p, rng)
    table[1, 0] = pages + 3
    nkv, D, L, gap = 2, 64, 3, 8 * 37
    one = pages * nkv * PAGE * D
    k0, v0 = (ref.bf16(rng.standard_normal(L * (one + gap))) for _ in range(2))
    rows = Rows(torch, p, table)
    rows.desc.d_err = 0
    tokens, greedy = [0, 1, 2, 3, 4, 5, 0, 1, 2, 0], [2, 9, 4, 9, 5, 9, 2, 9, 9, 0]
    i32 = lambda x: _dev(torch, np.array(x, np.int32))  # noqa: E731
    tok, gre = i32(tokens), i32(greedy)
    q = _dev(torch, ref.bf16(rng.standard_normal((p.rows, 4 * D))))
    x = _dev(torch, ref.bf16(rng.standard_normal((p.rows, 2 * nkv * D))))
    ran = []
    for stride, a, b in ((one + gap, k0, v0), (one, *(y.reshape(L, one + gap)[:, :one] for y in (k0, v0)))):
        k, v = _dev(torch, a), _dev(torch, b)
        cache = B.kv(nkv, D, pages, k.data_ptr(), v.data_ptr(), L, stride)
        out = torch.full((p.rows, 4 * D), 0x1234, dtype=torch.int16, device="cuda")
        ws = torch.empty(B.spec_tree_attn_workspace_bytes(cache, rows.desc, 4), dtype=torch.uint8, device="cuda")
        for layer in range(L):
            B.spec_kv_append(cache, layer, rows.desc, B.rope(1e4, (32, 0, 0)), 0, 0, 0, 0, x.data_ptr(), x.data_ptr() + 2 * nkv * D, x.stride(0),
                             0, 0)
        B.spec_tree_attn(cache, 2, rows.desc, 4, q.data_ptr(), 4 * D, 0.125, out.data_ptr(), 4 * D, 0, ws.data_ptr(), ws.numel())
        B.spec_tree_commit(cache, rows.desc, tok.data_ptr(), gre.data_ptr())
        torch.cuda.synchronize()
        ran.append((_bits(k).reshape(L, stride), _bits(v).reshape(L, stride), _bits(out)))
    far, near = ran
    for i, before in ((0, k0), (1, v0)):
        np.testing.assert_array_equal(far[i][:, :one], near[i])
        np.testing.assert_array_equal(far[i][:, one:], before.reshape(L, one + gap)[:, one:])
        assert (near[i] != before.reshape(L, one + gap)[:, :one]).any(axis=1).all()
    np.testing.assert_array_equal(far[2], near[2])
    assert np.isfinite(ref.bf16_value(far[2][:6])).all() and np.isnan(ref.bf16_value(far[2][6:9])).all()


@pytest.mark.parametrize("stop", [-1, 1, 77])
def test_commit_stops_at_tokens_and_budgets(torch, stop):
    rng = np.random.default_rng(32)
    counts = [20] * 7
    p = ref.Pass([5 * b for b in range(7)], counts, _trees(rng, counts, 4))
    tokens, greedy = _tokens(rng, p, 2)
    if stop == 77:
        greedy[0] = 77
    for budget in (None, [0, 1, 2, 3, -4, 100, 2 ** 31 - 1]):
        got = _commit(torch, rng, p, tokens, greedy, stop=stop, budget=budget)
        _check_commit(p, greedy, ref.commit(p, tokens, greedy, stop, budget), got)


def test_the_first_of_equal_siblings_is_taken(torch):
    rng = np.random.default_rng(33)
    p = ref.Pass([50], [7], [[-1, 0, 0, 0, 1, 2, 2]])
    got = _commit(torch, rng, p, [0, 4, 4, 4, 6, 6, 6], [4, 0, 6, 0, 1, 2, 3])
    assert got["path"][:2] == [0, 1] and got["n"] == [2]
    got = _commit(torch, rng, p, [0, 3, 4, 4, 6, 6, 6], [4, 0, 6, 0, 1, 2, 3])
    assert got["path"][:3] == [0, 2, 5] and got["committed"][:3] == [4, 6, 2]
    _check_commit(p, [4, 0, 6, 0, 1, 2, 3], [[0, 2, 5]], got)


def test_a_further_root_is_never_taken(torch):
    rng = np.random.default_rng(34)
    p = ref.Pass([50], [4], [[-1, -1, 1, 0]])
    got = _commit(torch, rng, p, [0, 4, 4, 4], [4, 4, 4, 9])
    _check_commit(p, [4, 4, 4, 9], [[0, 3]], got)


def test_commit_stays_in_bounds(torch):
    rng = np.random.default_rng(35)
    p = ref.Pass([60, 100], [12, 40], [[-1, 0, 0] + list(range(2, 11)), [-1, 0, 0] + list(range(2, 39))], 1, stride=2)
    tokens, greedy = [1] * p.rows, [1] * p.rows
    for b in range(2):
        tokens[p.first[b] + 1] = 0
    table, pages = ref.table_of(ref.Pass([60, 88], [12, 40], None), rng)
    table[0, 1] = pages
    got = _commit(torch, rng, p, tokens, greedy, table=table, pages=pages)
    assert got["err"] == 1
    _check_commit(p, greedy, ref.commit(p, tokens, greedy), got)
    for first, lens in (([0, 53, 52], None), ([-1, 12, 52], None), ([0, 12, 54], None), (None, [-1, 200])):
        got = _commit(torch, rng, p, tokens, greedy, table=table, pages=pages, rows=Rows(torch, p, table, first=first, lens=lens))
        assert got["err"] == 1 and got["n"] == [0, 0] and got["path"] == [-9] * p.rows and got["new"] == (lens or p.lens)
        np.testing.assert_array_equal(got["k"], got["k0"])
        np.testing.assert_array_equal(got["v"], got["v0"])
    q = ref.Pass([5], [5], [[-1, 0, 1, -1, 0]])
    table, pages = ref.table_of(q, rng)
    got = _commit(torch, rng, q, [0, 1, 2, 1, 7], [1, 2, 9, 9, 9], table=table, pages=pages, rows=Rows(torch, q, table, parents=[-1, 0, 1, 3, 0]))
    assert got["err"] == 1
    _check_commit(q, [1, 2, 9, 9, 9], [[0, 1, 2]], got)


# -- together ----------------------------------------------------------------------

class Loop:
    """A stand-in for a decoder's layers: a row's q, k and v follow from its token alone."""

    def __init__(self, torch, B, batch, nq, nkv, D, layers, rng, vocab=50, most=8):
        self.torch, self.B, self.batch, self.nq, self.nkv, self.D, self.layers = torch, B, batch, nq, nkv, D, layers
        self.emb = _dev(torch, ref.bf16(rng.standard_normal((layers, vocab, (nq + 2 * nkv) * D))))
        self.pages = batch * most
        table = rng.permutation(self.pages).astype(np.int32).reshape(batch, most)
        self.k = torch.zeros(layers, self.pages, nkv, PAGE, D, dtype=torch.int16, device="cuda")
        self.v = torch.zeros(layers, self.pages, nkv, D, PAGE, dtype=torch.int16, device="cuda")
        self.table, self.cache = _dev(torch, table), _cache(torch, B, self.k, self.v)
        self.len = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.rope = B.rope(1e4, (D // 8, 3 * D // 16, 3 * D // 16))

    def begin(self, counts, behind=0):
        """Buffers of passes of these sizes."""
        t, rows = self.torch, sum(counts) + behind
        i32 = lambda n: t.zeros(n, dtype=t.int32, device="cuda")  # noqa: E731
        self.rows, self.first = rows, _dev(t, np.cumsum([0] + counts).astype(np.int32))
        self.parent, self.tok, self.greedy, self.path, self.committed = (i32(rows) for _ in range(5))
        self.n, self.new = i32(self.batch), i32(self.batch)
        self.out = t.zeros(self.layers, rows, self.nq * self.D, dtype=t.int16, device="cuda")
        self.lse = t.zeros(self.layers, rows, self.nq, device="cuda")
        self.q = t.zeros(rows, self.nq * self.D, dtype=t.int16, device="cuda")
        self.desc = self.B.rows(self.batch, rows, self.first.data_ptr(), self.len.data_ptr(), self.table.data_ptr(), self.table.shape[1],
                                self.parent.data_ptr(), self.err.data_ptr())
        self.ws = t.empty(self.B.spec_tree_attn_workspace_bytes(self.cache, self.desc, self.nq), dtype=t.uint8, device="cuda")

    def layers_pass(self):
        s, w = self.torch.cuda.current_stream().cuda_stream, 2 * self.D
        for i in range(self.layers):
            x = self.emb[i][self.tok.long()]
            at = x.data_ptr()
            self.B.spec_kv_append(self.cache, i, self.desc, self.rope, 0, self.nq, at, x.stride(0), at + self.nq * w, at + (self.nq + self.nkv) * w,
                                  x.stride(0), self.q.data_ptr(), self.q.stride(0), s)
            self.B.spec_tree_attn(self.cache, i, self.desc, self.nq, self.q.data_ptr(), self.q.stride(0), self.D ** -0.5, self.out[i].data_ptr(),
                                  self.out.stride(1), self.lse[i].data_ptr(), self.ws.data_ptr(), self.ws.numel(), s)

    def commit(self):
        s = self.torch.cuda.current_stream().cuda_stream
        self.B.spec_tree_commit(self.cache, self.desc, self.tok.data_ptr(), self.greedy.data_ptr(), -1, 0, self.path.data_ptr(), self.committed.data_ptr(),
                                self.n.data_ptr(), self.new.data_ptr(), s)

    def kv(self, b, n):
        slots = np.arange(n)
        pg, off = self.table.cpu().numpy()[b, slots // PAGE], slots % PAGE
        return _bits(self.k)[:, pg, :, off], _bits(self.v)[:, pg, :, :, off]


@pytest.mark.parametrize("captured", [False, True])
def test_rounds_of_trees_leave_the_cache_of_plain_decoding(torch, captured):
    """Trees drafted, appended, attended and committed round after round (as one captured graph, or call by call): the cache
    is bit for bit that of the committed tokens appended one after another, and the committed path's outputs are those of
    a chain over that cache."""
    from paper_2606_31160_amd import binding as B
    rng = np.random.default_rng(40)
    counts, nq, nkv, D, layers = [9, 6, 13], 4, 2, 64, 2
    loop = Loop(torch, B, 3, nq, nkv, D, layers, rng)
    loop.begin(counts, behind=2)
    lens, said, pending = [0] * 3, [[], [], []], [7, 8, 9]
    outs = [[], [], []]

    def put(t, x):
        t.copy_(torch.tensor(x, dtype=t.dtype))

    def step():
        loop.layers_pass()
        loop.commit()

    graph = None
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        put(loop.parent, [-1] * loop.rows)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for _ in range(30):
        trees = _trees(rng, counts, 4)
        p = ref.Pass(lens, counts, trees, 2)
        tok = [int(x) for x in rng.integers(0, 50, p.rows)]
        greedy = [int(x) for x in rng.integers(0, 50, p.rows)]
        for b in range(3):
            tok[p.first[b]] = pending[b]
            for i in p.line(b, int(rng.integers(0, counts[b])))[1:]:
                greedy[p.first[b] + trees[b][i]] = tok[p.first[b] + i]
        put(loop.parent, p.flat_parents().tolist())
        put(loop.tok, tok)
        put(loop.greedy, greedy)
        put(loop.len, lens)
        graph.replay() if graph else step()
        torch.cuda.synchronize()
        taken = ref.commit(p, tok, greedy)
        assert loop.n.tolist() == [len(t) for t in taken] and loop.new.tolist() == [a + len(t) for a, t in zip(lens, taken)]
        for b, path in enumerate(taken):
            assert loop.path.tolist()[p.first[b]:p.first[b] + len(path)] == path
            said[b] += [tok[p.first[b] + j] for j in path]
            pending[b] = greedy[p.first[b] + path[-1]]
            outs[b] += [_bits(loop.out)[:, p.first[b] + j] for j in path]
        lens = loop.new.tolist()
    assert int(loop.err) == 0 and PAGE < max(lens) <= 160
    plain = Loop(torch, B, 3, nq, nkv, D, layers, np.random.default_rng(40))
    for b in range(3):
        plain.begin([n if i == b else 0 for i, n in enumerate(lens)])
        plain.desc.d_parent = None
        put(plain.tok, said[b])
        plain.layers_pass()
        torch.cuda.synchronize()
        for x, y in zip(loop.kv(b, lens[b]), plain.kv(b, lens[b])):
            np.testing.assert_array_equal(x, y)
        want = ref.bf16_value(_bits(plain.out))
        have = ref.bf16_value(np.stack(outs[b], 1))
        # both are within half a step, and the sums' errors, of one value
        np.testing.assert_allclose(have, want, rtol=2 * 2.0 ** -8, atol=2.0 ** -13)


def test_two_graphs_with_workspaces_of_their_own(torch):
    """Captured calls replay side by side, several times, with eager work between."""
    rng = np.random.default_rng(41)
    counts = [8, 15]
    both = [Attn(torch, rng, ref.Pass([1500, 300], counts, _trees(rng, counts)), 14, 2, 128) for _ in range(2)]
    want = [a.run() for a in both]
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for a in both:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            a.call(torch.cuda.current_stream())
        graphs.append(g)
    for _ in range(4):
        for a in both:
            a.out.fill_(0)
            a.lse.fill_(0)
            a.ws.fill_(0xFF)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for a, (out, lse) in zip(both, want):
            np.testing.assert_array_equal(_bits(a.out), out)
            np.testing.assert_array_equal(a.lse.cpu().numpy(), lse)
