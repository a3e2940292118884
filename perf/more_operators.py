"""Operators of a pass that verifies a tree of drafted tokens, and the cases on which they are measured.

  append  rotated queries and keys of new rows, keys and values written to their slots of a paged cache
  tree    attention of a tree's rows over such a cache: every row sees its sequence's earlier slots, its ancestors and itself
  commit  the tree's longest path that greedy decoding confirms, its keys and values moved to consecutive slots

Shapes, scene lengths and layer counts are those of the repository's workloads, or generic.
"""
import math

import torch

import workloads as W

own = False

PAGE = 64
WORKSPACE = 64 << 20   # bytes a program keeps for the calls' partial results
# q heads, kv heads, head dim, layers: the 7B-class backbone and its shard under 4-way tensor parallelism, the paper's
# backbone, the tiny workload; then plain multi-head and single-kv-head layouts
HEADS = {"7b": (28, 4, 128, 28), "tp4": (7, 1, 128, 28), "paper": (32, 8, 128, 36), "tiny": (4, 2, 64, 2),
         "mha": (8, 8, 64, 4), "mqa": (24, 1, 128, 3)}
# rotary pairs on the axes T, H, W, and whether pair d takes axis d mod 3
ROPE = {"7b": ((16, 24, 24), 0), "tp4": ((16, 24, 24), 0), "paper": ((24, 20, 20), 1), "tiny": ((8, 12, 12), 0),
        "mha": ((32, 0, 0), 0), "mqa": ((64, 0, 0), 0)}
BASE = 10000.0
SCENES_16 = " ".join(str(s.prefix_len) for s in W.get("C5").seqs)
# sixteen trees that fill a pass of 144 rows
TREES_16 = "9 12 7 9 10 8 16 1 9 5 13 9 11 6 9 10"


def _case(do, name, heads, lens, rows, tree=True, behind=0, **more):
    """lens: slots in use of each sequence; rows: its rows in this pass; tree: they form a tree, else a chain; behind: rows of
    the buffers that belong to no sequence (a program that keeps one size for every pass)."""
    c = {"do": do, "heads": heads, "lens": lens, "rows": rows, "tree": tree, "behind": behind, **more}
    return dict(c, name=name) if name else c


def listed():
    ones = " ".join(["1"] * 16)
    return [
        # the smallest call: one greedy token's keys and values behind a short prompt
        _case("append", "append greedy row", "tiny", "320", "1", tree=False, pos=False),
        # a pass over sixteen scenes, trees of different sizes; positions follow from the trees
        _case("append", "append 16 trees", "7b", SCENES_16, TREES_16, behind=16, pos=False),
        # a whole prompt of one scene with the positions of its vision blocks
        _case("append", "append prompt", "paper", "0", "4096", tree=False, pos=True),
        # pieces of five prompts of odd lengths behind what their caches hold
        _case("append", "append ragged pieces", "7b", "0 37 1000 4095 64", "2047 4099 1 6011 8191", tree=False, pos=True),
        # a small tree on a short prompt, where latency is all
        _case("tree", "tree tiny", "tiny", "320", "5"),
        # one scene, a tree as wide as single-scene serving drafts it
        _case("tree", "tree 7b", "7b", "4096", "40"),
        # the paper's backbone with a large tree
        _case("tree", "tree paper", "paper", "4117", "64"),
        # sixteen scenes, plain decoding of one row each
        _case("tree", "tree 16 scenes step", "7b", SCENES_16, ones, tree=False),
        # sixteen scenes with trees of different sizes
        _case("tree", "tree 16 trees", "7b", SCENES_16, TREES_16, behind=16),
        # one very long scene on one shard's heads
        _case("tree", "tree long scene", "tp4", "131029", "25"),
        # a small tree's accepted path, two layers
        _case("commit", "commit tiny", "tiny", "320", "5", accept=2),
        # sixteen scenes' accepted paths through every layer
        _case("commit", "commit 16 trees", "7b", SCENES_16, TREES_16, behind=16, accept=3),
    ]


def draw(rng):
    most = max(_cost(c) for c in listed())
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        do = rng.choice(["append", "append", "tree", "tree", "tree", "commit"])
        heads = rng.choice(list(HEADS))
        batch = rng.choice([1, 1, 1, 2, 3, 5, 8, 16])
        lens = [rng.choice([0, 1, 63, 64, 65]) if rng.random() < 0.1 else log(1, 65536 if batch == 1 else 8192)
                for _ in range(batch)]
        long = do == "append" and rng.random() < 0.5
        rows = [log(1, 16384 if long else min(64, 160 // batch)) for _ in range(batch)]
        if batch > 1 and rng.random() < 0.3:
            rows[rng.randrange(batch)] = 0                   # a sequence that sits this pass out
        more = {"accept": rng.randint(0, 8)} if do == "commit" else {"pos": rng.random() < 0.5} if do == "append" else {}
        c = _case(do, "", heads, " ".join(map(str, lens)), " ".join(map(str, rows)),
                  tree=not long and (do == "commit" or rng.random() < 0.8),
                  behind=rng.choice([0, 0, rng.randint(0, max(0, 160 - sum(rows)))]), **more)
        if sum(rows) and _cost(c) <= most:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 100)


def _ints(text):
    return [int(x) for x in text.split()]


def prepare(case, seed):
    import random
    seed = int(seed) % (1 << 40)
    dev, rng = "cuda", random.Random(seed)
    g = torch.Generator(dev).manual_seed(seed)
    nq, nkv, D, layers = HEADS[case["heads"]]
    do, lens, counts = case["do"], _ints(case["lens"]), _ints(case["rows"])
    B, n = len(lens), sum(counts)
    rows = n + case["behind"]
    first = [sum(counts[:b]) for b in range(B + 1)]
    parent, tokens, target = [-1] * rows, [-1] * rows, [-1] * rows
    for b in range(B):
        if not counts[b]:
            continue
        # a row continues one of the rows a little before it, as a tree written level by level does
        par = [-1] + [rng.randint(max(0, (j - 1) // 2 - 2), j - 1) if case["tree"] else j - 1 for j in range(1, counts[b])]
        parent[first[b]:first[b + 1]] = par
        if do == "commit":
            deep = [0] * counts[b]
            for j in range(1, counts[b]):
                deep[j] = deep[par[j]] + 1
            j, path = max(range(counts[b]), key=lambda i: (deep[i], i)), []
            while j >= 0:
                path.insert(0, j)
                j = par[j]
            path = path[:case["accept"] + 1]
            tok = [rng.randint(0, 150000) for _ in range(counts[b])]
            tgt = [200000 + rng.randint(0, 150000) for _ in range(counts[b])]     # what no row drafted
            for i, j in zip(path, path[1:]):
                tgt[i] = tok[j]
                for sib in range(i + 1, counts[b]):
                    if par[sib] == i and sib != j and (tok[sib] == tok[j] or sib > j and rng.random() < 0.2):
                        # a token drafted twice goes by its first row
                        tok[sib] = tok[j] if sib > j else tok[j] + 1
            tokens[first[b]:first[b + 1]], target[first[b]:first[b + 1]] = tok, tgt

    # pages: all of a sequence's where its slots are read, else those of the pass
    begin = [0 if do == "tree" else x // PAGE for x in lens]
    end = [-(-(x + c) // PAGE) for x, c in zip(lens, counts)]
    pool = sum(max(0, e - s) for s, e in zip(begin, end)) + 2
    cpu = torch.Generator().manual_seed(seed + 1)
    order, at = torch.randperm(pool, generator=cpu).int(), 0
    table = torch.full((B, max(1, max(end)) + 1), -1, dtype=torch.int32)
    for b in range(B):
        k = max(0, end[b] - begin[b])
        table[b, begin[b]:begin[b] + k] = order[at:at + k]
        at += k

    def rand(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    L = layers if do == "commit" else 1
    K, V = torch.empty(2, L, pool, nkv, PAGE * D, dtype=torch.bfloat16, device=dev)
    amp = torch.exp(0.5 * rand(nkv, 1, D))                  # channels differ
    for i in range(L):
        K[i] = (rand(pool, nkv, PAGE, D) * amp).view(pool, nkv, -1)
        V[i] = rand(pool, nkv, PAGE * D)
    s = {"do": do, "B": B, "rows": rows, "n": n, "most": max(counts), "nq": nq, "nkv": nkv, "D": D, "L": L,
         "slots": max(x + c for x, c in zip(lens, counts)), "scale": D ** -0.5, "tree": case["tree"],
         "k": K.view(L, pool, nkv, PAGE, D), "v": V.view(L, pool, nkv, D, PAGE), "table": table.to(dev),
         "first": ints(first), "len": ints(lens), "parent": ints(parent), "err": ints([0])}
    if do == "tree":
        for b in range(B):                                  # slots not yet written hold anything
            if (lens[b] + counts[b]) % PAGE:
                last, off = int(table[b, end[b] - 1]), (lens[b] + counts[b]) % PAGE
                s["k"][0, last, :, off:] = math.nan
                s["v"][0, last, :, :, off:] = math.nan
        s["q"] = rand(rows, nq, D).bfloat16()
        s["out"] = torch.zeros(rows, nq, D, dtype=torch.bfloat16, device=dev)
        s["lse"] = torch.zeros(rows, nq, device=dev)
        s["ws"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device=dev)
    elif do == "append":
        # queries, keys and values as they leave a fused projection
        s["qkv"] = (rand(rows, (nq + 2 * nkv) * D) * torch.exp(0.7 * rand((nq + 2 * nkv) * D))).bfloat16()
        s["q_out"] = torch.zeros(rows, nq, D, dtype=torch.bfloat16, device=dev)
        s["section"], s["interleaved"] = ROPE[case["heads"]]
        s["pos"] = None
        if case["pos"]:
            # rows of frames of 28 x 32 patches: three axes that go their own ways
            i = torch.arange(rows, device=dev, dtype=torch.int32)
            at = s["len"].repeat_interleave(ints(counts).long())
            at = torch.nn.functional.pad(at, (0, rows - n)) + i
            s["pos"] = torch.stack([at, at - i % 896 + i % 896 // 32, at - i % 896 + i % 32]).contiguous()
    else:
        s["tokens"], s["target"] = ints(tokens), ints(target)
        s["path"], s["committed"] = ints([-1] * rows), ints([-1] * rows)
        s["n_committed"], s["new_len"] = ints([-1] * B), ints([-1] * B)
    return s


def _places(s):
    """Of every live row: its sequence and index there, its ancestors and itself [rows, rows]; the rows' slots."""
    r = torch.arange(s["n"], device=s["len"].device)
    b = torch.searchsorted(s["first"][1:].long(), r, right=True)
    j = r - s["first"].long()[b]
    return b, j, s["len"].long()[b] + j


def _ancestors(s, b, j):
    n = s["n"]
    par = s["parent"][:n].long() if s["tree"] else j - 1
    up = torch.eye(n, device=b.device)
    has = par >= 0
    up[torch.nonzero(has)[:, 0], (s["first"].long()[b] + par)[has]] = 1
    for _ in range(8):                                      # 2^8 generations
        up = (up @ up).clamp(max=1)
    return up


def _plain_append(s):
    n, nq, nkv, D = s["n"], s["nq"], s["nkv"], s["D"]
    b, j, slot = _places(s)
    page, off = s["table"][b, slot // PAGE].long(), slot % PAGE
    if s["pos"] is None:
        deep = _ancestors(s, b, j).sum(1).long() - 1 if s["tree"] else j
        pos = (s["len"].long()[b] + deep).expand(3, n)
    else:
        pos = s["pos"][:, :n].long()
    d = torch.arange(D // 2, device=b.device)
    axis = d % 3 if s["interleaved"] else (d >= s["section"][0]).long() + (d >= s["section"][0] + s["section"][1]).long()
    angle = pos[axis].T.double() * BASE ** (-2.0 * d.double() / D)       # far positions: 32 bits would lose the turn
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    x = s["qkv"][:n].float().view(n, nq + 2 * nkv, D // 2, 2)
    even, odd = x[:, :nq + nkv, :, 0], x[:, :nq + nkv, :, 1]
    rot = torch.stack([even * cos - odd * sin, even * sin + odd * cos], -1).view(n, nq + nkv, D).bfloat16()
    s["q_out"][:n] = rot[:, :nq]
    s["k"][0, page, :, off] = rot[:, nq:]
    s["v"][0, page, :, :, off] = x[:, nq + nkv:].reshape(n, nkv, D).bfloat16()
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _plain_tree(s):
    B, n, nq, nkv, D, R = s["B"], s["n"], s["nq"], s["nkv"], s["D"], s["most"]
    b, j, slot = _places(s)
    pages = -(-s["slots"] // PAGE)
    S = pages * PAGE
    seen = torch.arange(S, device=b.device) < s["len"][b][:, None]                                  # [n, S]
    up = _ancestors(s, b, j)
    r, c = torch.nonzero(up, as_tuple=True)
    seen[r, slot[c]] = True
    table = s["table"][:, :pages].clamp(min=0).long()
    k = s["k"][0][table].float().permute(0, 2, 1, 3, 4).reshape(B, nkv, S, D)
    v = s["v"][0][table].float().permute(0, 2, 1, 4, 3).reshape(B, nkv, S, D)
    some = torch.zeros(B, R, S, dtype=torch.bool, device=b.device)
    some[b, j] = seen
    v = torch.where(some.any(1)[:, None, :, None], v, 0.0)                                          # slots that no row sees
    q = torch.zeros(B, R, nq, D, device=b.device)
    q[b, j] = s["q"][:n].float()
    q = q.view(B, R, nkv, nq // nkv, D).permute(0, 2, 1, 3, 4).reshape(B, nkv, -1, D)
    z = ((q @ k.transpose(-1, -2)) * s["scale"]).view(B, nkv, R, -1, S)
    z = torch.where(some[:, None, :, None], z, -math.inf)
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(torch.isfinite(m), m, 0.0))
    l = e.sum(-1, keepdim=True)
    o = (e.view(B, nkv, -1, S) @ v).view(B, nkv, R, -1, D) / l
    s["out"][:n] = o.permute(0, 2, 1, 3, 4).reshape(B, R, nq, D)[b, j].bfloat16()
    s["lse"][:n] = (m + torch.log(l))[..., 0].permute(0, 2, 1, 3).reshape(B, R, nq)[b, j]
    return {"out": s["out"], "lse": s["lse"]}


def _plain_commit(s):
    B, n, R = s["B"], s["n"], s["most"]
    b, j, slot = _places(s)
    dev = b.device
    par = s["parent"][:n].long() if s["tree"] else j - 1
    has = par >= 0
    up = s["first"].long()[b] + par.clamp(min=0)
    # a row is confirmed by its parent's greedy token, and taken if it is the first such child
    fits = has & (s["tokens"][:n] == s["target"][:n][up])
    lowest = torch.full((n,), n, device=dev).scatter_reduce(0, torch.where(fits, up, 0), torch.where(fits, torch.arange(n, device=dev), n), "amin")
    taken = torch.where(j == 0, True, fits & (lowest[up] == torch.arange(n, device=dev)))
    anc = _ancestors(s, b, j)
    good = (anc @ (~taken).float()) == 0                                                             # with all its ancestors
    step = (anc.sum(1).long() - 1)[good]
    gb, gj, gs = b[good], j[good], slot[good]
    to = s["first"].long()[gb] + step
    s["path"][to] = gj.int()
    s["committed"][to] = s["target"][:n][good]
    count = torch.zeros(B, dtype=torch.int32, device=dev).index_add(0, gb, torch.ones_like(gb, dtype=torch.int32))
    s["n_committed"].copy_(count)
    s["new_len"].copy_(s["len"] + count)
    dst = s["len"].long()[gb] + step
    ps, os, pd, od = s["table"][gb, gs // PAGE].long(), gs % PAGE, s["table"][gb, dst // PAGE].long(), dst % PAGE
    k, v = s["k"].transpose(0, 1), s["v"].transpose(0, 1)
    k[pd, :, :, od] = k[ps, :, :, os]
    v[pd, ..., od] = v[ps, ..., os]
    return {"k": s["k"], "v": s["v"], "path": s["path"], "committed": s["committed"], "n": s["n_committed"], "len": s["new_len"]}


def run(state):
    s = state
    if not own:
        return {"append": _plain_append, "tree": _plain_tree, "commit": _plain_commit}[s["do"]](s)
    from paper_2606_31160_amd import binding as B
    stream = torch.cuda.current_stream().cuda_stream
    k, v = s["k"], s["v"]
    cache = B.kv(s["nkv"], s["D"], k.shape[1], k.data_ptr(), v.data_ptr(), s["L"], k.stride(0))
    rows = B.rows(s["B"], s["rows"], s["first"].data_ptr(), s["len"].data_ptr(), s["table"].data_ptr(), s["table"].shape[1],
                  s["parent"].data_ptr() if s["tree"] else 0, s["err"].data_ptr())
    if s["do"] == "append":
        x, size = s["qkv"], 2 * s["D"]
        rope = B.rope(BASE, s["section"], s["interleaved"])
        at, pos = x.data_ptr(), s["pos"]
        B.spec_kv_append(cache, 0, rows, rope, 0 if pos is None else pos.data_ptr(), s["nq"], at, x.stride(0),
                         at + s["nq"] * size, at + (s["nq"] + s["nkv"]) * size, x.stride(0), s["q_out"].data_ptr(),
                         s["q_out"].stride(0), stream)
        return {"q": s["q_out"], "k": k, "v": v}
    if s["do"] == "tree":
        q, out, ws = s["q"], s["out"], s["ws"]
        B.spec_tree_attn(cache, 0, rows, s["nq"], q.data_ptr(), q.stride(0), s["scale"], out.data_ptr(), out.stride(0),
                         s["lse"].data_ptr(), ws.data_ptr(), ws.numel(), stream)
        return {"out": out, "lse": s["lse"]}
    B.spec_tree_commit(cache, rows, s["tokens"].data_ptr(), s["target"].data_ptr(), -1, 0, s["path"].data_ptr(),
                       s["committed"].data_ptr(), s["n_committed"].data_ptr(), s["new_len"].data_ptr(), stream)
    return {"k": k, "v": v, "path": s["path"], "committed": s["committed"], "n": s["n_committed"], "len": s["new_len"]}


def work(case):
    nq, nkv, D, layers = HEADS[case["heads"]]
    lens, counts = _ints(case["lens"]), _ints(case["rows"])
    n = sum(counts)
    if case["do"] == "append":
        return {"bytes": float(4 * n * (nq + 2 * nkv) * D + (12 * n if case["pos"] else 4 * n)), "flops": float(3 * n * (nq + nkv) * D)}
    if case["do"] == "tree":
        slots = sum(x + c for x, c in zip(lens, counts) if c)
        # a row's ancestors and itself, on average: half of a chain, a few of a tree
        seen = sum(c * (x + (min(c, 2 + math.log2(c)) if case["tree"] else (c + 1) / 2)) for x, c in zip(lens, counts) if c)
        return {"bytes": float(4 * slots * nkv * D + n * nq * (4 * D + 4)), "flops": float(4 * D * nq * seen)}
    # rows that a path of this length moves: all but the first, of trees that are so deep
    moved = sum(min(case["accept"], c - 1, int(2 * math.log2(c))) for c in counts if c)
    return {"bytes": float(8 * moved * nkv * D * layers + 20 * n), "flops": float(4 * n)}


def exact(case, seed):
    s = prepare(case, seed)
    nq, nkv, D, n = s["nq"], s["nkv"], s["D"], s["n"]
    first, lens, table = s["first"].tolist(), s["len"].tolist(), s["table"].tolist()
    parent = s["parent"].tolist()
    where = lambda b, slot: (table[b][slot // PAGE], slot % PAGE)  # noqa: E731

    def line(b, j):
        """Row j of sequence b and its ancestors, the eldest first."""
        if not case["tree"]:
            return list(range(j + 1))
        got = []
        while j >= 0:
            got.insert(0, j)
            j = parent[first[b] + j]
        return got

    of = [(b, j) for b in range(s["B"]) for j in range(first[b + 1] - first[b])]
    if case["do"] == "append":
        x = s["qkv"][:n].double().view(n, nq + 2 * nkv, D)
        if s["pos"] is None:
            p = torch.tensor([[lens[b] + (len(line(b, j)) - 1 if case["tree"] else j) for b, j in of]] * 3, dtype=torch.float64, device="cuda")
        else:
            p = s["pos"][:, :n].double()
        T, H, _ = s["section"]
        axes = [d % 3 if s["interleaved"] else 0 if d < T else 1 if d < T + H else 2 for d in range(D // 2)]
        angle = torch.stack([p[a] * BASE ** (-2 * d / D) for d, a in enumerate(axes)], 1)
        z = torch.view_as_complex(x[:, :nq + nkv].reshape(n, nq + nkv, D // 2, 2)) * torch.polar(torch.ones_like(angle), angle)[:, None]
        rot = torch.view_as_real(z).reshape(n, nq + nkv, D)
        q = torch.cat([rot[:, :nq], s["q_out"][n:].double()])
        k, v = s["k"].double(), s["v"].double()
        at = torch.tensor([where(b, lens[b] + j) for b, j in of], device="cuda")
        k[0, at[:, 0], :, at[:, 1]] = rot[:, nq:]
        v[0, at[:, 0], :, :, at[:, 1]] = x[:, nq + nkv:]
        return {"q": q, "k": k, "v": v}
    if case["do"] == "tree":
        out, lse = s["out"].double(), s["lse"].double()
        for b in range(s["B"]):
            c = first[b + 1] - first[b]
            if not c:
                continue
            pages = table[b][:-(-(lens[b] + c) // PAGE)]
            lines = [line(b, j) for j in range(c)]
            for h in range(nkv):
                k = s["k"][0, pages, h].double().reshape(-1, D)
                v = s["v"][0, pages, h].double().transpose(1, 2).reshape(-1, D)
                hq = slice(h * (nq // nkv), (h + 1) * (nq // nkv))
                for j in range(c):
                    see = torch.tensor(lines[j], device="cuda") + lens[b]
                    kj, vj = torch.cat([k[:lens[b]], k[see]]), torch.cat([v[:lens[b]], v[see]])
                    z = s["q"][first[b] + j, hq].double() @ kj.T * s["scale"]
                    lse[first[b] + j, hq] = torch.logsumexp(z, 1)
                    out[first[b] + j, hq] = torch.softmax(z, 1) @ vj
        return {"out": out, "lse": lse}
    tok, tgt = s["tokens"].tolist(), s["target"].tolist()
    path, committed, count = s["path"].tolist(), s["committed"].tolist(), []
    k, v = s["k"].double(), s["v"].double()
    for b in range(s["B"]):
        rows, taken = range(first[b + 1] - first[b]), []
        j = 0 if len(rows) else None
        while j is not None:
            taken.append(j)
            here = [i for i in rows if i > j and (parent[first[b] + i] if case["tree"] else i - 1) == j and tok[first[b] + i] == tgt[first[b] + j]]
            j = min(here) if here else None
        for i, j in enumerate(taken):
            path[first[b] + i], committed[first[b] + i] = j, tgt[first[b] + j]
            (ps, os), (pd, od) = where(b, lens[b] + j), where(b, lens[b] + i)
            k[:, pd, :, od] = k[:, ps, :, os]
            v[:, pd, ..., od] = v[:, ps, ..., os]
        count.append(len(taken))
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"k": k, "v": v, "path": ints(path), "committed": ints(committed), "n": ints(count), "len": ints([a + c for a, c in zip(lens, count)])}
