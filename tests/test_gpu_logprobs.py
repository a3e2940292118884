"""Log probabilities, entropy and top alternatives of logits against a 64-bit reference."""
import math

import numpy as np
import pytest

from tests import _operators as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _call(torch, x, V, given, top, entropy=True, stream=None, ws=None):
    """x: device tensor [rows][>= V] of the logits' type."""
    from paper_2606_31160_amd import binding as B
    n = x.shape[0]
    dt = {torch.bfloat16: B.SPEC_BF16, torch.float16: B.SPEC_F16, torch.float32: B.SPEC_F32}[x.dtype]
    need = B.spec_logprobs_workspace_bytes(n, V, top)
    if ws is None:
        ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    out = {"lp": torch.full(given.shape, 9.0, device="cuda"), "h": torch.full((n,), 9.0, device="cuda"),
           "ti": torch.full((n, max(top, 1)), -9, dtype=torch.int32, device="cuda"),
           "tl": torch.full((n, max(top, 1)), 9.0, device="cuda")}
    s = stream or torch.cuda.current_stream()
    B.spec_logprobs(x.data_ptr(), dt, n, V, x.stride(0), given.data_ptr() if given.numel() else 0, given.shape[1], top,
                    out["lp"].data_ptr() if given.numel() else 0, out["h"].data_ptr() if entropy else 0,
                    out["ti"].data_ptr() if top else 0, out["tl"].data_ptr() if top else 0, ws.data_ptr(), ws.numel(),
                    s.cuda_stream)
    return out


def _check(torch, x, V, given, top, out):
    torch.cuda.synchronize()
    xs = x.double().cpu().numpy()[:, :V]
    lp, h, ti, tl = (out[k].double().cpu().numpy() for k in ("lp", "h", "ti", "tl"))
    gv = given.cpu().numpy()
    for r in range(xs.shape[0]):
        g, e, order, glp, (S, N, T) = ref.scores(xs[r], gv[r], top)
        assert (ti[r, :top] == order).all(), (r, ti[r, :top], order)
        if math.isnan(e):
            assert math.isnan(h[r]) and np.isnan(lp[r]).all() and np.isnan(tl[r, :top]).all()
            continue
        # Bounds.  A term e^d is off by 2^-24 (2 |d| + 3) of itself, and a sum of terms by the depth of its tree (at
        # most 64 additions one after the other) times 2^-24 more: on the whole S is off by dS, T by dT.  Terms below
        # 2^-126, the smallest normal number of 32 bits, may vanish: V of them, each times at most 150 ln 2 < 104 in T
        # (below 2^-150 nothing is left in 32 bits at all).
        u, tiny = 2.0 ** -24, V * 2.0 ** -126
        dS = u * (67 * S + 2 * abs(T)) + tiny
        d = xs[r] - xs[r].max()
        with np.errstate(invalid="ignore"):
            ed = np.exp(d)
            T2 = np.where(ed > 0, ed * np.where(ed > 0, d, 0) ** 2, 0).sum()
        dT = u * (70 * abs(T) + 2 * T2) + 104 * tiny
        dZ = dS / (N + S) + 3 * u * math.log1p(N - 1 + S)
        for have, want, idx in ([(lp[r], g, gv[r])] if gv.shape[1] else []) + [(tl[r, :top], glp, order)]:
            dd = np.array([d[i] if 0 <= i < V else math.nan for i in idx])
            with np.errstate(invalid="ignore"):
                ok = (np.abs(have - want) <= dZ + 2 * u * (np.abs(dd) + np.abs(want))) | (have == want) | (np.isnan(have) & np.isnan(want))
            assert ok.all(), (r, have[~ok], want[~ok], dZ)
        assert abs(h[r] - e) <= dZ + dT / (N + S) + abs(T) * dS / (N + S) ** 2 + 4 * u * abs(e) + 2 * u * abs(T) / (N + S), (r, h[r], e)


def _logits(torch, rng, n, V, dtype, pad=0, scale=2.5):
    x = torch.from_numpy(rng.standard_normal((n, V + pad)) * scale).cuda().to(getattr(torch, dtype))
    return x[:, :V] if pad else x


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("n,V,top,pad", [(1, 1, 1, 0), (1, 2, 2, 0), (3, 7, 3, 1), (2, 32, 32, 0), (5, 2047, 5, 0), (4, 2048, 20, 8),
                                         (4, 2049, 32, 3), (2, 8193, 1, 0), (3, 50257, 8, 7), (9, 152064, 20, 0),
                                         (2, 1 << 20, 32, 0), (130, 4099, 4, 5), (2000, 300, 3, 0), (1100, 8201, 6, 1)])
def test_scores(torch, dtype, n, V, top, pad):
    rng = np.random.default_rng(V + n)
    x = _logits(torch, rng, n, V, dtype, pad)
    given = torch.from_numpy(rng.integers(0, V, (n, 2)).astype(np.int32)).cuda()
    _check(torch, x, V, given, top, _call(torch, x, V, given, top))


@pytest.mark.parametrize("V", [5, 700, 9000, 152064])
def test_sure_tokens_keep_their_digits(torch, V):
    """Rows whose best token is all but certain: ln p is far below a step of the logits."""
    rng = np.random.default_rng(V)
    x = _logits(torch, rng, 6, V, "float32", scale=1.0)
    best = torch.from_numpy(rng.integers(0, V, (6, 1))).cuda()
    x.scatter_(1, best, torch.tensor([[8.0], [15.0], [25.0], [40.0], [90.0], [300.0]], device="cuda"))
    given = torch.cat([best, (best + 1) % V], 1).int()
    _check(torch, x, V, given, 3, _call(torch, x, V, given, 3))


@pytest.mark.parametrize("V", [64, 3000, 40000, 700001])
@pytest.mark.parametrize("kind", ["all equal", "few values", "mostly masked", "one left", "sorted up", "sorted down", "lowest", "signed zeros"])
def test_ties_masks_and_orders(torch, V, kind):
    rng = np.random.default_rng(V)
    top = 32
    if kind == "all equal":
        a = np.full((2, V), -1.5)
    elif kind == "few values":
        a = rng.integers(-2, 3, (3, V)).astype(float)
    elif kind == "mostly masked":
        a = np.where(rng.random((3, V)) < 0.999, -math.inf, rng.standard_normal((3, V)))
        a[:, V // 2] = 0.25
    elif kind == "one left":
        a = np.full((2, V), -math.inf)
        a[0, V - 1] = a[1, 0] = -3.0
    elif kind == "sorted up":
        a = np.sort(rng.standard_normal((2, V)), 1)
    elif kind == "sorted down":
        a = -np.sort(rng.standard_normal((2, V)), 1)
    elif kind == "lowest":
        a = np.where(rng.random((2, V)) < 0.9, np.finfo(np.float32).min, rng.standard_normal((2, V)))
        a[1] = np.finfo(np.float32).min
    else:
        a = np.where(rng.random((2, V)) < 0.5, -0.0, 0.0)
    for dtype in ("bfloat16", "float32"):
        b = np.maximum(a, -3.3895313892515355e38) if kind == "lowest" else a
        x = torch.from_numpy(b).cuda().to(getattr(torch, dtype))
        given = torch.tensor([[0, V - 1, V // 2]] * len(a), dtype=torch.int32, device="cuda")
        _check(torch, x, V, given, top, _call(torch, x, V, given, top))


@pytest.mark.parametrize("V", [100, 20000, 700001])
def test_rows_without_a_distribution(torch, V):
    rng = np.random.default_rng(V)
    a = rng.standard_normal((6, V)).astype(np.float32)
    a[0, V // 3] = math.nan
    a[1, 5] = math.inf
    a[2] = -math.inf
    a[3] = math.nan
    a[4, 0], a[4, V - 1] = math.inf, math.nan
    for dtype in ("bfloat16", "float16", "float32"):
        x = torch.from_numpy(a).cuda().to(getattr(torch, dtype))
        given = torch.tensor([[0, 5]] * 6, dtype=torch.int32, device="cuda")
        _check(torch, x, V, given, 6, _call(torch, x, V, given, 6))


def test_tokens_out_of_range_and_optional_outputs(torch):
    rng = np.random.default_rng(1)
    x = _logits(torch, rng, 3, 5000, "bfloat16")
    given = torch.tensor([[-1, 0, 5000], [4999, 2 ** 31 - 1, -2 ** 31], [7, 7, 7]], dtype=torch.int32, device="cuda")
    out = _call(torch, x, 5000, given, 2)
    _check(torch, x, 5000, given, 2, out)
    assert torch.isnan(out["lp"][0, 0]) and torch.isnan(out["lp"][0, 2]) and torch.isnan(out["lp"][1, 1:]).all()
    none = torch.empty(3, 0, dtype=torch.int32, device="cuda")
    o = _call(torch, x, 5000, none, 0, entropy=False)
    torch.cuda.synchronize()
    assert (o["h"] == 9).all() and (o["ti"] == -9).all() and (o["tl"] == 9).all()
    o = _call(torch, x, 5000, none, 0)
    torch.cuda.synchronize()
    assert torch.equal(o["h"], out["h"])


def test_a_row_far_into_memory(torch):
    """Rows whose offset passes 32 bits."""
    x = torch.zeros(3, 1 << 30, dtype=torch.bfloat16, device="cuda")
    x[:, :1000] = torch.randn(3, 1000, device="cuda", generator=torch.Generator("cuda").manual_seed(0)).bfloat16() * 3
    v = x[:, :1000]
    given = torch.tensor([[1], [2], [3]], dtype=torch.int32, device="cuda")
    _check(torch, v, 1000, given, 5, _call(torch, v, 1000, given, 5))


def test_the_same_every_time_on_a_stream_and_in_a_graph(torch):
    rng = np.random.default_rng(2)
    V = 30000
    x = _logits(torch, rng, 9, V, "bfloat16")
    given = torch.from_numpy(rng.integers(0, V, (9, 1)).astype(np.int32)).cuda()
    want = _call(torch, x, V, given, 20)
    _check(torch, x, V, given, 20, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    from paper_2606_31160_amd import binding as B
    with torch.cuda.stream(s):
        ws = torch.zeros(B.spec_logprobs_workspace_bytes(9, V, 20), dtype=torch.uint8, device="cuda")
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = _call(torch, x, V, given, 20, stream=s, ws=ws)
    for _ in range(4):
        for o in out.values():
            o.zero_()
        ws.fill_(0xEE)
        g.replay()
        torch.cuda.synchronize()
        again = _call(torch, x, V, given, 20, ws=ws)
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(out[k], want[k]) and torch.equal(again[k], want[k]), k
