"""8-bit cache pages and attention over them against 64-bit references."""
import math

import numpy as np
import pytest

from tests import _operators as ref

pytestmark = pytest.mark.gpu
PAGE = 64


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _dev(torch, a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


# -- packing ---------------------------------------------------------------------

def _pack(torch, k, v, nkv, D, pages8, to, stride_pad=0, stream=None):
    """k, v: bf16 bits [rows][nkv*D].  Returns codes, scales and the error word."""
    from paper_2606_31160_amd import binding as B
    rows = k.shape[0]
    both = np.full((rows, 2 * nkv * D + stride_pad), 0x7FC0, np.uint16)
    both[:, :nkv * D], both[:, nkv * D:2 * nkv * D] = k, v
    kv = _dev(torch, both)
    k8 = torch.full((pages8, nkv, PAGE, D), 0xAB, dtype=torch.uint8, device="cuda")
    v8 = torch.full((pages8, nkv, D, PAGE), 0xAB, dtype=torch.uint8, device="cuda")
    ks, vs = torch.full((2, pages8, nkv), -7.0, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    t = torch.tensor(to, dtype=torch.int32, device="cuda")
    c = B.kv8(nkv, D, pages8, k8.data_ptr(), v8.data_ptr(), ks.data_ptr(), vs.data_ptr())
    s = stream or torch.cuda.current_stream()
    s.wait_stream(torch.cuda.current_stream())
    B.spec_kv8_pack(c, kv.data_ptr(), kv.data_ptr() + 2 * nkv * D, both.shape[1], rows, t.data_ptr(), err.data_ptr(),
                    s.cuda_stream)
    torch.cuda.synchronize()
    return k8.cpu().numpy(), v8.cpu().numpy(), ks.cpu().numpy(), vs.cpu().numpy(), int(err)


def _check_pages(k, v, nkv, D, to, pages8, got):
    k8, v8, ks, vs, _ = got
    rows = k.shape[0]
    touched = set()
    for i, p in enumerate(to):
        if not 0 <= p < pages8:
            continue
        touched.add(p)
        n = min(PAGE, rows - PAGE * i)
        for h in range(nkv):
            for bits, codes, scale in ((k, k8[p, h], ks[p, h]), (v, v8[p, h].T, vs[p, h])):
                x = ref.bf16_value(bits[PAGE * i:PAGE * i + n, h * D:(h + 1) * D])
                s = ref.page_scale(x)
                assert scale == s, (p, h, scale, s)
                want = ref.e4m3_round(x / s)
                have = ref.e4m3_value(codes)
                np.testing.assert_array_equal(have[:n], want)
                assert (codes[n:] == 0).all()
                fin = np.isfinite(x)
                # half a step of e4m3 relative to the value, or half the smallest step
                assert (np.abs(have[:n] * s - x)[fin] <= np.maximum(2.0 ** -4 * np.abs(x[fin]), s * 2.0 ** -10)).all()
                # what it stands for are bf16 numbers.  Not so one number of the whole range: 448 2^119 < 2^128 makes the
                # scale of the largest magnitudes 2^120, and from 248 2^120 on they round to 256 2^120 = 2^128, one
                # step beyond the largest bf16 number, 255 2^120.
                in_range = np.abs(have) * s < 2.0 ** 128
                np.testing.assert_array_equal(ref.bf16_value(ref.bf16((have * s)[in_range])), (have * s)[in_range])
                assert (np.abs(x[~in_range[:n] & fin]) >= 248 * 2.0 ** 120).all() if n == PAGE else in_range.all()
    for p in set(range(pages8)) - touched:
        assert (k8[p] == 0xAB).all() and (v8[p] == 0xAB).all() and (ks[p] == -7).all() and (vs[p] == -7).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [1, 63, 64, 65, 200])
@pytest.mark.parametrize("nkv,pad", [(1, 0), (3, 8)])
def test_pack_is_bit_exact(torch, D, rows, nkv, pad):
    rng = np.random.default_rng(rows * 7 + D + nkv)
    w = nkv * D
    k, v = (ref.bf16(rng.standard_normal((rows, w)) * np.exp(rng.standard_normal(w) * 2)) for _ in range(2))
    n = -(-rows // PAGE)
    to = list(rng.permutation(n + 2)[:n])
    got = _pack(torch, k, v, nkv, D, n + 2, to, pad)
    assert got[4] == 0
    _check_pages(k, v, nkv, D, to, n + 2, got)


def test_pack_extreme_values(torch):
    """Zeros, subnormals, the largest bf16 numbers, powers of two on a scale's border, NaN and infinities."""
    D, nkv = 64, 2
    big = 3.3895313892515355e38
    fills = [0.0, 1e-40, 9.2e-41, big, 448.0, 449.0 * 1.01, 448.0 * 2.0 ** -126, 2.0 ** -133, 1.75 * 2.0 ** -20, 1.7578125]
    k = np.zeros((PAGE * len(fills), nkv * D))
    rng = np.random.default_rng(0)
    for i, f in enumerate(fills):
        blk = rng.uniform(-1, 1, (PAGE, nkv * D)) * f
        blk[5, 3] = blk[6, D + 3] = f
        k[PAGE * i:PAGE * i + PAGE] = blk
    with np.errstate(over="ignore"):
        kb = ref.bf16(k)
    vb = kb.copy()
    vb[7, 1], vb[8, 2], vb[9, D + 2], vb[PAGE + 1, 4], vb[4 * PAGE + 2, 9] = 0x7FC0, 0x7F80, 0xFF80, 0xFFC0, 0x7F80
    vb[2 * PAGE:3 * PAGE, :D] = 0x7F80           # a head's page of infinities only
    kb[::PAGE, 0] = 0x8000                       # -0
    to = list(range(len(fills)))
    got = _pack(torch, kb, vb, nkv, D, len(fills), to)
    assert got[4] == 0
    _check_pages(kb, vb, nkv, D, to, len(fills), got)


def test_pack_skips_bad_pages(torch):
    D, nkv = 64, 1
    rng = np.random.default_rng(3)
    k, v = (ref.bf16(rng.standard_normal((5 * PAGE, D))) for _ in range(2))
    to = [2, -1, 4, 3, 2 ** 31 - 1]              # pool of 4 pages
    got = _pack(torch, k, v, nkv, D, 4, to)
    assert got[4] == 1
    _check_pages(k, v, nkv, D, to, 4, got)


def test_pack_on_another_stream(torch):
    D, nkv = 128, 2
    rng = np.random.default_rng(4)
    k, v = (ref.bf16(rng.standard_normal((100, nkv * D))) for _ in range(2))
    got = _pack(torch, k, v, nkv, D, 2, [1, 0], stream=torch.cuda.Stream())
    _check_pages(k, v, nkv, D, [1, 0], 2, got)


# -- attention -------------------------------------------------------------------

class Case:
    """A cache with its pass; lens: slots in use per sequence, packed: 8-bit pages per sequence."""

    def __init__(self, torch, seed, nq, nkv, D, lens, packed, vis, q_pad=0, out_pad=0, amp=1.0, spread=1.0, extra=2,
                 stale=0x7FC0):
        rng = np.random.default_rng(seed)
        self.torch, self.nq, self.nkv, self.D, self.B, self.R = torch, nq, nkv, D, len(lens), vis.shape[1]
        self.vis, self.packed, self.scale = vis.astype(np.int32), packed, D ** -0.5
        pages = [-(-n // PAGE) for n in lens]
        packed = [min(p, n) for p, n in zip(packed, pages)]
        n8, n16 = sum(packed) + extra, sum(pages) - sum(packed) + extra
        self.n8, self.n16 = n8, n16
        self.k8 = rng.integers(0, 256, (n8, nkv, PAGE, D), dtype=np.uint8)
        self.v8 = rng.integers(0, 256, (n8, nkv, D, PAGE), dtype=np.uint8)
        for c in (self.k8, self.v8):             # numbers only, of moderate size (at most 30)
            c[(c & 127) > 0x5F] &= 0xBF
        self.ks = np.exp2(rng.integers(-5, -2, (n8, nkv))).astype(np.float32)
        self.vs = (np.exp2(rng.uniform(-3, 3, (n8, nkv)) * spread)).astype(np.float32)   # any positive scale will do
        self.k16 = ref.bf16(rng.standard_normal((n16, nkv, PAGE, D)) * amp)
        self.v16 = ref.bf16(rng.standard_normal((n16, nkv, D, PAGE)))
        self.stride = max(max(pages), 1) + extra
        self.table = np.full((self.B, self.stride), 2 ** 30, np.int32)
        o8, o16 = iter(rng.permutation(n8)), iter(rng.permutation(n16))
        for b in range(self.B):
            for i in range(pages[b]):
                self.table[b, i] = next(o8 if i < packed[b] else o16)
            if lens[b] % PAGE:                   # slots not in use hold anything
                p, at = self.table[b, pages[b] - 1], lens[b] % PAGE
                if pages[b] - 1 < packed[b]:
                    self.k8[p, :, at:], self.v8[p, :, :, at:] = 0x7F, 0xFF
                else:
                    self.k16[p, :, at:], self.v16[p, :, :, at:] = stale, stale
        self.q = ref.bf16(rng.standard_normal((self.B * self.R, nq * D)) * amp)
        self.q_pad, self.out_pad = q_pad, out_pad

    def keys_values(self, b, h):
        ks, vs = [], []
        for i, p in enumerate(self.table[b]):
            if p >= 2 ** 30 or p < 0:
                break
            if i < self.packed[b]:
                ks.append(ref.e4m3_value(self.k8[p, h]) * float(self.ks[p, h]))
                vs.append(ref.e4m3_value(self.v8[p, h]).T * float(self.vs[p, h]))
            else:
                ks.append(ref.bf16_value(self.k16[p, h]))
                vs.append(ref.bf16_value(self.v16[p, h]).T)
        z = np.zeros((0, self.D))
        return np.concatenate(ks or [z]), np.concatenate(vs or [z])

    def upload(self):
        from paper_2606_31160_amd import binding as B
        t = self.torch
        self.d = {n: _dev(t, getattr(self, n)) for n in ("k8", "v8", "ks", "vs", "k16", "v16", "table", "vis")}
        self.d["packed"] = t.tensor(self.packed, dtype=t.int32, device="cuda")
        w = self.nq * self.D
        qp = np.full((self.B * self.R, w + self.q_pad), 0x7FC0, np.uint16)
        qp[:, :w] = self.q
        self.d["q"] = _dev(t, qp)
        self.cache = B.kv8(self.nkv, self.D, self.n8, self.d["k8"].data_ptr(), self.d["v8"].data_ptr(),
                           self.d["ks"].data_ptr(), self.d["vs"].data_ptr(), self.n16, self.d["k16"].data_ptr(),
                           self.d["v16"].data_ptr())
        self.ws_bytes = B.spec_kv8_attn_workspace_bytes(self.cache, self.B, self.R, self.nq, self.stride)
        self.ws = t.full((self.ws_bytes,), 0xFF, dtype=t.uint8, device="cuda")
        self.out = t.full((self.B * self.R, w + self.out_pad), 77.0, dtype=t.bfloat16, device="cuda")
        self.lse = t.full((self.B * self.R, self.nq), 55.0, device="cuda")
        self.err = t.zeros(1, dtype=t.int32, device="cuda")

    def call(self, stream=None, lse=True):
        from paper_2606_31160_amd import binding as B
        d = self.d
        s = stream or self.torch.cuda.current_stream()
        B.spec_kv8_attn(self.cache, self.B, self.R, self.nq, d["table"].data_ptr(), self.stride, d["packed"].data_ptr(),
                        d["vis"].data_ptr(), d["q"].data_ptr(), d["q"].stride(0), self.scale, self.out.data_ptr(),
                        self.out.stride(0), self.lse.data_ptr() if lse else 0, self.err.data_ptr(), self.ws.data_ptr(),
                        self.ws_bytes, s.cuda_stream)

    def run(self):
        self.upload()
        self.call()
        self.torch.cuda.synchronize()
        return self.out.float().cpu().numpy().astype(np.float64), self.lse.cpu().numpy().astype(np.float64)

    def check(self, err=0):
        out, lse = self.run()
        assert int(self.err) == err
        w = self.nq * self.D
        assert (out[:, w:] == 77).all()          # between the rows
        G = self.nq // self.nkv
        for b in range(self.B):
            for h in range(self.nkv):
                k, v = self.keys_values(b, h)
                for j in range(self.R):
                    r, n = b * self.R + j, int(self.vis[b, j])
                    for g in range(G):
                        hq = h * G + g
                        o, z = out[r, hq * self.D:(hq + 1) * self.D], lse[r, hq]
                        if n < 0:
                            assert (o == 77).all() and z == 55
                            continue
                        q = ref.bf16_value(self.q[r, hq * self.D:(hq + 1) * self.D])
                        want, wz, A, S, l, vm = ref.attention(q, k, v, n, self.scale)
                        # Bounds.  A score is a sum of D products in 32 bits and one rounding for its factor: off by
                        # (D + 8) 2^-24 of the sum of its magnitudes.  A probability is off by twice that (its own
                        # score, the normalisation), by half a step of fp16, 2^-11 or at most 2^-25 where it is that
                        # small, and the result by half a step of bf16, 2^-8; 2^-14 A for what is summed in 32 bits.
                        ds = (self.D + 8) * 2.0 ** -24 * S
                        tol = 2.0 ** -8 * np.abs(want) + A * (2.0 ** -11 + 2 * ds + 2.0 ** -14) + n * 2.0 ** -25 * vm / l
                        bad = ~(np.isclose(o, want, rtol=0, atol=0, equal_nan=True) | (np.abs(o - want) <= tol))
                        assert not bad.any(), (b, j, hq, np.flatnonzero(bad)[:4], o[bad][:4], want[bad][:4])
                        if math.isfinite(wz):
                            assert abs(z - wz) <= ds + 2.0 ** -20 + 2.0 ** -22 * abs(wz), (b, j, hq, z, wz)
                        else:
                            assert z == wz or (math.isnan(z) and math.isnan(wz))


def _causal(lens, R):
    return np.array([[n - R + j + 1 for j in range(R)] for n in lens], np.int32)


@pytest.mark.parametrize("nq,nkv,D", [(4, 2, 64), (7, 1, 128), (28, 4, 128), (8, 8, 64), (40, 1, 128), (1, 1, 64)])
@pytest.mark.parametrize("length,R", [(1, 1), (2, 1), (63, 1), (64, 1), (65, 2), (130, 9), (333, 17), (1500, 5)])
def test_attention_one_sequence(torch, nq, nkv, D, length, R):
    if nq * length * R > 400000:
        length = 700
    Case(torch, length + R, nq, nkv, D, [length], [max(0, (length - R) // PAGE)], _causal([length], R)).check()


@pytest.mark.parametrize("rows_per_head", [15, 16, 17, 32, 33, 48, 49, 64, 65, 80, 100, 128, 129, 160])
def test_attention_row_blocks(torch, rows_per_head):
    R = next(r for r in (17, 16, 13, 11, 10, 8, 7, 5, 3, 1) if rows_per_head % r == 0)
    G = rows_per_head // R
    Case(torch, rows_per_head, G, 1, 64, [200], [3], _causal([200], R)).check()


@pytest.mark.parametrize("packed", [0, 1, 4, 5, 9])
def test_attention_pages_of_both_kinds(torch, packed):
    """From none of the pages to all of them in 8 bits; the last one ends inside."""
    Case(torch, packed, 6, 2, 128, [8 * PAGE + 13], [packed], _causal([8 * PAGE + 13], 3)).check()


def test_attention_ragged_batch(torch):
    lens = [1, 700, 64, 65, 129, 3000, 17, 300]
    R = 4
    vis = np.array([[max(0, n - R + j + 1) for j in range(R)] for n in lens], np.int32)
    c = Case(torch, 5, 4, 2, 64, lens, [n // PAGE for n in lens], vis, q_pad=24, out_pad=8)
    c.check()


def test_attention_many_sequences(torch):
    lens = [(37 * i) % 200 + 1 for i in range(150)]
    c = Case(torch, 6, 2, 1, 64, lens, [n // PAGE for n in lens], np.array(lens, np.int32)[:, None])
    c.check()


@pytest.mark.parametrize("nq,nkv,D,R", [(2, 1, 64, 3), (7, 1, 128, 9), (4, 2, 128, 1)])
def test_attention_many_groups(torch, nq, nkv, D, R):
    """So many pages of few heads that the combine takes four groups a wave; rows of all lengths."""
    n = 9000 * nkv + 77
    vis = _causal([n], R)
    for c, v in (((R - 1) // 2, 5000), (R - 1, 0 if R > 1 else n), (0, 64 if R > 3 else n)):
        vis[0, c] = v
    if R > 5:
        vis[0, 4] = -1
    c = Case(torch, 31 + R, nq, nkv, D, [n], [n // PAGE - 3], vis)
    c.check()
    if R > 1:                                     # values that are not finite in a late page that not every row sees
        last = c.table[0, n // PAGE]
        c.v16[last, 0, 3, 5], c.v16[last, 0, 4, 6] = 0x7F80, 0x7FC0
        c.check()


def test_attention_rows_without_slots_and_without_a_row(torch):
    """Rows that see nothing, rows that are not there, whole sequences of both, rows in any order."""
    lens = [200, 0, 100, 90, 64]
    vis = np.array([[200, 0, 5, -1, 128], [0, 0, 0, 0, 0], [-1, -1, -1, -1, -1], [1, 90, 64, 65, 0], [-1, 0, 64, 63, -5]],
                   np.int32)
    Case(torch, 7, 6, 2, 64, lens, [2, 0, 1, 0, 1], vis).check()


def test_attention_nothing_to_see_at_all(torch):
    Case(torch, 8, 4, 1, 64, [0, 0], [0, 0], np.array([[0, 0], [-1, 0]], np.int32)).check()


def test_attention_values_only_some_rows_see(torch):
    """NaN and infinities in a slot reach the rows that see it and no others."""
    for D, packed in ((64, 3), (128, 0)):
        lens = [150]
        vis = np.array([[140, 141, 142, 150, 10]], np.int32)
        c = Case(torch, 9, 4, 2, D, lens, [packed], vis)
        p = c.table[0, 2]
        if packed == 3:
            c.v8[p, 0, 7, 141 - 128] = 0x7F
            c.v8[p, 1, 33, 149 - 128] = 0xFF
            c.k8[p, 1, 140 - 128, 5] = 0x7F
        else:
            c.v16[p, 0, 7, 141 - 128] = 0x7F80
            c.v16[p, 0, 100, 140 - 128] = 0xFF80
            c.v16[p, 1, 33, 149 - 128] = 0x7FC0
            c.k16[p, 1, 140 - 128, 5] = 0x7FC0
        c.check()


def test_attention_stale_infinities(torch):
    for stale in (0x7F80, 0xFF80, 0xFFFF):
        Case(torch, 10, 4, 2, 64, [70], [0], _causal([70], 2), stale=stale).check()


def test_attention_far_scales(torch):
    """Value scales of pages far apart, also beyond the range of fp16 and of one 32-bit number's exponent."""
    for spread in (4.0, 12.0, 30.0):
        Case(torch, int(spread), 4, 2, 64, [9 * PAGE], [9], _causal([9 * PAGE], 3), spread=spread).check()


def test_attention_sharp_rows(torch):
    """Scores of a wide range: most probabilities underflow."""
    Case(torch, 12, 4, 1, 128, [400], [5], _causal([400], 9), amp=6.0).check()


@pytest.mark.parametrize("D,packed", [(64, 1), (128, 1), (64, 0), (128, 0)])
def test_attention_scores_are_summed_in_32_bits(torch, D, packed):
    """Queries are whole numbers up to 255, a quarter of a key's numbers 32 to 448, the rest 2 to 7.5 in steps of 1/4
    and more: any sum of products is a whole number of 1/4 and at most 32 448 255 + 96 7.5 255 < 2^22, exact in 32
    bits in any order.  One key is visible, so lse is its score: off by the roundings of its factor, of itself, of its
    difference from itself and of the change of logarithm's base (two), half a step each, of at most its magnitude
    and 1."""
    c = Case(torch, 16, 28, 4, D, [PAGE], [packed], np.ones((1, 5), np.int32))
    rng = np.random.default_rng(17)
    c.q = ref.bf16(rng.integers(128, 256, c.q.shape) * rng.choice([-1, 1], c.q.shape))

    def codes(shape):                             # [..., D]
        large = np.arange(D) % 4 == 0
        return (np.where(large, rng.integers(0x60, 0x7F, shape), rng.integers(0x40, 0x50, shape)) |
                rng.choice([0, 0x80], shape)).astype(np.uint8)

    c.k8, c.k16 = codes(c.k8.shape), ref.bf16(ref.e4m3_value(codes(c.k16.shape)))
    c.ks[:] = 1.0
    c.scale = 2.0 ** -14
    _, lse = c.run()
    for h in range(4):
        k, _ = c.keys_values(0, h)
        for j in range(5):
            for g in range(7):
                q = ref.bf16_value(c.q[j, (7 * h + g) * D:(7 * h + g + 1) * D])
                want = float(q @ k[0]) * c.scale
                assert abs(lse[j, 7 * h + g] - want) <= 5 * 2.0 ** -24 * (abs(want) + 1), (j, h, g, lse[j, 7 * h + g], want)


def test_attention_bad_pages_and_lengths(torch):
    """Bad entries are taken as not visible and reported."""
    c = Case(torch, 13, 4, 2, 64, [5 * PAGE], [3], _causal([5 * PAGE], 2))
    good = c.table.copy()
    c.table[0, 1], c.table[0, 4] = c.n8, -3
    out, lse = c.run()
    assert int(c.err) == 1
    k = Case.keys_values
    keep = [0, 2, 3]
    c.table = good
    for h in range(2):
        kk, vv = k(c, 0, h)
        sel = np.concatenate([np.arange(PAGE * p, PAGE * p + PAGE) for p in keep])
        for j in range(2):
            for g in range(2):
                hq = 2 * h + g
                want, wz, A, S, l, vm = ref.attention(ref.bf16_value(c.q[j, hq * 64:hq * 64 + 64]), kk[sel], vv[sel], sel.size, c.scale)
                assert (np.abs(out[j, hq * 64:hq * 64 + 64] - want) <= 2.0 ** -8 * np.abs(want) + A * 2.0 ** -9).all()
    c = Case(torch, 14, 4, 2, 64, [100], [1], np.array([[100]], np.int32), extra=0)
    c.vis[0, 0] = 129                             # more than the table's 128 slots
    c.run()
    assert int(c.err) == 1
    for bad in (0.0, -1.0, math.nan, math.inf):   # scales
        c = Case(torch, 15, 4, 2, 64, [100], [1], np.array([[100]], np.int32))
        c.vs[c.table[0, 0], 1] = bad
        c.run()
        assert int(c.err) == 1


def test_attention_without_lse_and_on_another_stream(torch):
    c = Case(torch, 16, 4, 2, 64, [300], [4], _causal([300], 3))
    c.check()
    want = c.out.clone()
    c.upload()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.call(s, lse=False)
    torch.cuda.synchronize()
    assert torch.equal(c.out, want) and (c.lse == 55).all()


def test_attention_is_the_same_every_time_and_in_a_graph(torch):
    """Replays, with eager calls on the same workspace in between, and other lengths in place."""
    c = Case(torch, 17, 28, 4, 128, [1000, 333], [15, 5], _causal([1000, 333], 9))
    c.check()
    first = c.out.clone(), c.lse.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.call(s)
    vis = c.d["vis"].clone()
    for i in range(4):
        c.out.fill_(3)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, first[0]) and torch.equal(c.lse, first[1]), i
        c.d["vis"].copy_(vis - 64 * (i + 1))
        c.call()
        eager = c.out.clone()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, eager) and not torch.equal(eager, first[0])
        c.d["vis"].copy_(vis)


def test_attention_shared_pages_and_odd_page_counts(torch):
    """Sequences on the same pages, as a shared prompt's; counts of 8-bit pages past the table and below zero."""
    R = 2
    c = Case(torch, 23, 4, 2, 64, [300, 300, 300], [5, 5, 5], _causal([300, 300, 300], R))
    c.table[1] = c.table[0]
    c.packed = [5, 2 ** 31 - 1, 5]
    c.q[R:2 * R] = c.q[:R]
    out, lse = c.run()
    assert int(c.err) == 0 and (out[:R] == out[R:2 * R]).all() and (lse[:R] == lse[R:2 * R]).all()
    c = Case(torch, 24, 4, 2, 64, [130], [0], _causal([130], R))
    c.check()
    want = c.out.clone()
    c.packed = [-7]
    c.run()
    assert torch.equal(c.out, want)
    lens = [(53 * i) % 190 + 2 for i in range(80)]   # the most sequences of two rows
    Case(torch, 25, 2, 1, 64, lens, [n // PAGE for n in lens], _causal(lens, R)).check()


def test_attention_rows_that_see_refused_pages_only(torch):
    c = Case(torch, 26, 4, 2, 64, [PAGE, PAGE], [1, 1], _causal([PAGE, PAGE], 2))
    c.table[0, 0] = -1
    out, lse = c.run()
    assert int(c.err) == 1 and np.isnan(out[:2]).all() and (lse[:2] == -math.inf).all()
    assert np.isfinite(out[2:]).all() and np.isfinite(lse[2:]).all()


def test_attention_two_at_once(torch):
    """Two streams, a workspace each."""
    cs = [Case(torch, 27 + i, 28, 4, 128, [2000 + 700 * i], [30], _causal([2000 + 700 * i], 9)) for i in range(2)]
    for c in cs:
        c.check()
    want = [c.out.clone() for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    for c in cs:
        c.out.fill_(3)
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s in zip(cs, streams):
            c.call(s)
    torch.cuda.synchronize()
    assert all(torch.equal(c.out, w) for c, w in zip(cs, want))


def test_attention_pages_far_into_their_pools(torch):
    """Pages whose first byte is past 2^32 in every pool."""
    c = Case(torch, 29, 8, 4, 128, [300], [3], _causal([300], 3), extra=0)
    c.check()
    want = c.out.clone()
    for pool, far in (("k8", 2 ** 17), ("v8", 2 ** 17), ("k16", 2 ** 16), ("v16", 2 ** 16)):
        x = c.d[pool]
        big = torch.empty((far + 9,) + x.shape[1:], dtype=x.dtype, device="cuda")
        assert big[far:].data_ptr() - big.data_ptr() >= 2 ** 32
        big[far + 1:far + 1 + x.shape[0]] = x
        c.d[pool] = big
    for n in ("ks", "vs"):
        x = c.d[n]
        c.d[n] = torch.ones((2 ** 17 + 9,) + x.shape[1:], device="cuda")
        c.d[n][2 ** 17 + 1:2 ** 17 + 1 + x.shape[0]] = x
    c.d["table"][0, :3] += 2 ** 17 + 1
    c.d["table"][0, 3:] += 2 ** 16 + 1
    from paper_2606_31160_amd import binding as B
    c.cache = B.kv8(4, 128, 2 ** 17 + 9, c.d["k8"].data_ptr(), c.d["v8"].data_ptr(), c.d["ks"].data_ptr(),
                    c.d["vs"].data_ptr(), 2 ** 16 + 9, c.d["k16"].data_ptr(), c.d["v16"].data_ptr())
    c.out.fill_(3)
    c.call()
    torch.cuda.synchronize()
    assert int(c.err) == 0 and torch.equal(c.out, want)


def test_pack_rows_far_apart(torch):
    """Rows whose offset passes 2^32 bytes."""
    D, nkv, rows, stride = 64, 2, 130, 2 ** 24 + 8
    rng = np.random.default_rng(30)
    k, v = (ref.bf16(rng.standard_normal((rows, nkv * D))) for _ in range(2))
    from paper_2606_31160_amd import binding as B
    far = torch.empty((rows, stride), dtype=torch.int16, device="cuda")
    far[:, :nkv * D], far[:, nkv * D:2 * nkv * D] = _dev(torch, k), _dev(torch, v)
    k8 = torch.full((3, nkv, PAGE, D), 0xAB, dtype=torch.uint8, device="cuda")
    v8 = torch.full((3, nkv, D, PAGE), 0xAB, dtype=torch.uint8, device="cuda")
    ks, vs = torch.full((2, 3, nkv), -7.0, device="cuda")
    to = torch.tensor([1, 2, 0], dtype=torch.int32, device="cuda")
    c = B.kv8(nkv, D, 3, k8.data_ptr(), v8.data_ptr(), ks.data_ptr(), vs.data_ptr())
    B.spec_kv8_pack(c, far.data_ptr(), far.data_ptr() + 2 * nkv * D, stride, rows, to.data_ptr(), 0,
                    torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    _check_pages(k, v, nkv, D, [1, 2, 0], 3, (k8.cpu().numpy(), v8.cpu().numpy(), ks.cpu().numpy(), vs.cpu().numpy(), 0))


def test_pack_then_attention(torch):
    """A prompt's rows packed and attended to, against the rows themselves: what 8 bits cost stays within their step."""
    nq, nkv, D, n = 8, 2, 128, 5 * PAGE
    rng = np.random.default_rng(18)
    k, v = (ref.bf16(rng.standard_normal((n, nkv * D))) for _ in range(2))
    to = list(rng.permutation(7)[:5])
    k8, v8, ks, vs, _ = _pack(torch, k, v, nkv, D, 7, to)
    c = Case(torch, 19, nq, nkv, D, [n], [5], _causal([n], 4))
    assert c.n8 == 7
    c.k8, c.v8, c.ks, c.vs = k8, v8, ks, vs
    c.table[0, :5] = to
    c.check()
    out = c.out.float().cpu().numpy().astype(np.float64)
    for h in range(nkv):
        kk, vv = (ref.bf16_value(x[:, h * D:(h + 1) * D]) for x in (k, v))
        for j in range(4):
            for hq in range(4 * h, 4 * h + 4):
                q = ref.bf16_value(c.q[j, hq * D:(hq + 1) * D])
                want, _, A, S, _, _ = ref.attention(q, kk, vv, int(c.vis[0, j]), c.scale)
                # every key and value is off by 2^-4 of itself at most: scores by 2^-4 S, and at most
                # e^(2 * 2^-4 S) - 1 of the weights
                ds = 2.0 ** -4 * S
                assert (np.abs(out[j, hq * D:(hq + 1) * D] - want) <= A * (2.0 ** -4 * math.exp(2 * ds) + math.expm1(2 * ds) + 2.0 ** -7)).all()


def test_attention_queries_that_are_not_finite_or_tiny(torch):
    """NaN and infinities in a query make its own row NaN; queries of any magnitude keep their digits."""
    for D in (64, 128):
        c = Case(torch, 20, 4, 2, D, [200], [2], _causal([200], 5))
        c.q[1, 3], c.q[2, D + 7], c.q[2, 2 * D] = 0x7FC0, 0x7F80, 0xFF80
        c.check()
        for amp in (1e-38, 1e-30, 1e-3, 1e4):
            c = Case(torch, 21, 4, 2, D, [200], [2], _causal([200], 5))
            c.q = ref.bf16(ref.bf16_value(c.q) * amp)
            c.check()
        c = Case(torch, 22, 4, 2, D, [200], [2], _causal([200], 5))   # elements of one query far apart
        c.q = ref.bf16(ref.bf16_value(c.q) * np.exp2(np.random.default_rng(1).integers(-30, 4, c.q.shape)))
        c.check()
