"""Operators around the paged boundary cache: their plain forms, their calls, and the cases they are measured on.

Four operators, in the order a rollout uses them:

  * ``rope``     per-head RMS norm of queries and keys with the rotation by multi-axis positions (time, height, width of a
                 video patch; one axis for text) in the same pass, as it runs in front of the attention passes;
  * ``rope_bwd`` its gradient, fed by the float32 dq, dk that the attention backward pass leaves;
  * ``tree``     attention of a tree of drafted tokens over [cached prefix ; ancestors in the tree] (one node = decoding);
  * ``branch``   the cache's pages at a branch point: the previous branches are freed, new ones forked from their prompts
                 (whole pages shared, the last partial page copied), and the first tokens of each branch appended;
  * ``compact``  live pages move to the low end of the pool, so that its high end can be handed back.

``own = False`` computes them with elementary torch operations in 32 bits (64 for the angles), ``own = True`` makes the
library's calls.  Head shapes are those of the 7B- and 32B-shaped benchmark configurations (28/4 and 40/8 heads of 128)
and of the small float32 one (4/2 heads of 64).
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ cases
def _rope(name, tokens, hq, hkv, d, rot, axes, dtype, far, norm=True, interleaved=False):
    return {"name": name, "op": "rope", "tokens": tokens, "hq": hq, "hkv": hkv, "d": d, "rot": rot, "axes": axes,
            "dtype": dtype, "far": far, "norm": norm, "interleaved": interleaved}


def _tree(name, batch, nodes, ctx, hq, hkv, d, ragged, unused):
    return {"name": name, "op": "tree", "batch": batch, "nodes": nodes, "ctx": ctx, "hq": hq, "hkv": hkv, "d": d,
            "ragged": ragged, "unused": unused}


def _branch(name, prompts, group, ctx, new, hkv, d):
    return {"name": name, "op": "branch", "prompts": prompts, "group": group, "ctx": ctx, "new": new, "hkv": hkv, "d": d}


def _compact(name, pages, live, rows, layers, hkv, d):
    return {"name": name, "op": "compact", "pages": pages, "live": live, "rows": rows, "layers": layers, "hkv": hkv, "d": d}


def listed():
    return [
        # one decoding step of a batch of 8: latency
        _rope("rope_decode_8", 8, 28, 4, 128, 128, 3, "bf16", 40000),
        # the prompt rows of the 7B-shaped batch (8 x 4096 tokens of video)
        _rope("rope_prompts_32768", 32768, 28, 4, 128, 128, 3, "bf16", 5000),
        # the training actor's backward over that batch's whole sequences
        {**_rope("rope_bwd_34816", 34816, 28, 4, 128, 128, 3, "bf16", 5000), "op": "rope_bwd"},
        # the small float32 configuration, partial rotation, an odd number of tokens
        {**_rope("rope_bwd_f32_289", 289, 4, 2, 64, 32, 1, "f32", 300), "op": "rope_bwd"},
        # decoding one token of one long video (32B shape)
        _tree("tree_decode_32768", 1, 1, 32768, 40, 8, 128, False, False),
        # a few drafted tokens each behind 8 prompts (7B shape)
        _tree("tree_8x8_4096", 8, 8, 4096, 28, 4, 128, False, False),
        # 32 ragged sequences with ragged trees (32B shape), some nodes unused
        _tree("tree_32x16_ragged", 32, 16, 16381, 40, 8, 128, True, True),
        # wide trees: a verification step with many candidates
        _tree("tree_wide_8x192", 8, 192, 8192, 28, 4, 128, True, False),
        # one prompt, two branches: latency
        _branch("branch_1x2", 1, 2, 777, 1, 4, 128),
        # prompt groups of 8 over 32 prompts
        _branch("branch_32x8", 32, 8, 4093, 17, 8, 128),
        # a small pool after one group has finished
        _compact("compact_600", 600, 233, 5, 1, 4, 128),
        # a pool of 24000 pages in 4 layers, half of it live
        _compact("compact_24000", 24000, 12011, 48, 4, 8, 128),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "rope_bwd", "tree", "tree", "branch", "compact"])
    limit = {}
    for c in listed():
        limit[c["op"]] = max(limit.get(c["op"], 0), _cost(c))
    while True:
        hq, hkv = rng.choice([(28, 4), (40, 8), (4, 2), (8, 8), (16, 1), (12, 4)])
        d = rng.choice([64, 128, 128])
        if op in ("rope", "rope_bwd"):
            c = _rope("", _log(rng, 1, 40000), hq, hkv, d, rng.choice([16, 32, 48, d // 2, d, d]), rng.choice([1, 2, 3, 3]),
                      rng.choice(["bf16", "bf16", "f32"]), _log(rng, 10, 2000000), rng.random() < 0.75, rng.random() < 0.4)
            c["op"] = op
        elif op == "tree":
            c = _tree("", _log(rng, 1, 48), _log(rng, 1, 256), _log(rng, 1, 40000), hq, hkv, d, rng.random() < 0.7,
                      rng.random() < 0.5)
        elif op == "branch":
            c = _branch("", _log(rng, 1, 40), rng.randint(1, 12), _log(rng, 1, 6000), rng.randint(1, 40), hkv, d)
        else:
            pages = _log(rng, 40, 30000)
            c = _compact("", pages, max(1, int(pages * rng.uniform(0.05, 0.95))), rng.randint(1, 64), rng.randint(1, 5), hkv, d)
        del c["name"]
        # the plain form of a tree keeps its scores, padded to the longest sequence: a bound on those too
        if _cost(c) <= limit[op] and (op != "tree" or c["batch"] * c["nodes"] * c["ctx"] * c["hq"] <= 4e8):
            return c


def _cost(case):
    w = work(case)
    return w["bytes"] / 6.5e12 + w["flops"] / 1.4e15


def _lens(case):
    """Cached tokens and tree sizes of the sequences of a tree case: spread over the range when ragged."""
    b, ctx, nodes = case["batch"], case["ctx"], case["nodes"]
    if not case["ragged"]:
        return [ctx] * b, [nodes] * b
    spread = [(i * 0.6180339887498949 + 0.25) % 1.0 for i in range(b)]
    return ([max(0, ctx - int(s * 0.9 * ctx)) for s in spread],
            [max(0 if b > 4 and i % 7 == 3 else 1, nodes - int(((s * 7.0) % 1.0) * nodes)) for i, s in enumerate(spread)])


def _branch_lens(case):
    return [max(1, case["ctx"] - (i * 37) % (case["ctx"] // 2 + 1)) for i in range(case["prompts"])]


def work(case):
    op, d = case["op"], case["d"]
    if op in ("rope", "rope_bwd"):
        values = case["tokens"] * (case["hq"] + case["hkv"]) * d
        size = 2 if case["dtype"] == "bf16" else 4
        per = 2 * size if op == "rope" else 2 * size + 4  # x in and out; the backward pass also reads float32 gradients
        return {"bytes": float(values * per + 4 * case["tokens"] * case["axes"]), "flops": float(values * (8 if op == "rope" else 16))}
    if op == "tree":
        lens, nodes = _lens(case)
        kv = (sum(lens) + sum(nodes)) * case["hkv"] * d * 2 * 2
        qo = sum(nodes) * case["hq"] * (2 * d * 2 + 4)
        pairs = sum(n * (p + 1) for p, n in zip(lens, nodes))
        return {"bytes": float(kv + qo + 4 * sum(-(-p // PAGE) for p in lens)), "flops": float(4 * d * case["hq"] * pairs)}
    page = case["hkv"] * PAGE * d * 2 * 2  # K and V of one page
    if op == "branch":
        lens, g, new = _branch_lens(case), case["group"], case["new"]
        held = sum(-(-(p + new) // PAGE) for p in lens) * g
        copied = sum(1 for p in lens if p % PAGE) * g
        # old rows read and cleared, new rows read and written, reference counts touched twice; copied pages; new tokens
        return {"bytes": float(held * (4 * 4 + 2 * 8) + copied * 2 * page + 2 * len(lens) * g * new * page / PAGE), "flops": 0.0}
    nb, live = case["pages"], case["live"]
    moved = live * (nb - live) / nb
    return {"bytes": float(nb * 8 + 8 * live + moved * (2 * page * case["layers"] + 8)), "flops": 0.0}


# ------------------------------------------------------------------ inputs
def _pair_axis(case):
    """Which position axis turns each rotary pair: a quarter of the pairs for time and the rest for height and width, in
    runs or taking turns."""
    n, axes = case["rot"] // 2, case["axes"]
    if axes == 1:
        return [0] * n
    sizes = [n - 2 * (3 * n // 8), 3 * n // 8, 3 * n // 8] if axes == 3 else [n - n // 2, n // 2]
    if case["interleaved"]:
        return [i % axes if i // axes < sizes[i % axes] else 0 for i in range(n)]
    return [a for a, s in enumerate(sizes) for _ in range(s)]


def _rope_inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    t, hq, hkv, d, dt = case["tokens"], case["hq"], case["hkv"], case["d"], DTYPES[case["dtype"]]
    rows = hq + 2 * hkv
    # the projection's output: q, k and v of a token side by side, so q and k are strided views of it
    scale = torch.exp(0.5 * torch.randn(t, rows, 1, device="cuda", generator=gen))
    qkv = (torch.randn(t, rows, d, device="cuda", generator=gen) * scale).to(dt)
    s = {"case": case, "q": qkv[:, :hq], "k": qkv[:, hq:hq + hkv]}
    # positions: frames of a 3-axis grid somewhere in a long context, height and width small; time first
    far, axes = case["far"], case["axes"]
    pos = torch.randint(0, 96, (axes, t), device="cuda", generator=gen, dtype=torch.int32)
    pos[0] = torch.randint(0, far, (t,), device="cuda", generator=gen, dtype=torch.int32)
    s["positions"] = pos
    n = case["rot"] // 2
    s["inv_freq"] = (1000000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float64) / n)).float()
    s["pair_axis"] = _pair_axis(case)
    s["pair_axis_dev"] = torch.tensor(s["pair_axis"], device="cuda")
    s["eps"] = 1e-6
    s["qw"] = s["kw"] = None
    if case["norm"]:
        s["qw"] = (1 + 0.2 * torch.randn(d, device="cuda", generator=gen)).to(dt)
        s["kw"] = (1 + 0.2 * torch.randn(d, device="cuda", generator=gen)).to(dt)
    if case["op"] == "rope_bwd":
        s["dq"] = torch.randn(t, hq, d, device="cuda", generator=gen)
        s["dk"] = torch.randn(t, hkv, d, device="cuda", generator=gen)
    return s


def _parents(rng, nodes, unused):
    """A drafted tree: a node hangs on one of the few before it (or on the last cached token); a tenth may be padding."""
    out = []
    for i in range(nodes):
        if unused and rng.random() < 0.1:
            out.append(-2)
            continue
        p = int(rng.integers(max(-1, i - 5), i)) if i else -1
        out.append(-1 if p >= 0 and out[p] == -2 else p)
    return out


def _tree_inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    lens, nodes = _lens(case)
    pages = [-(-p // PAGE) for p in lens]
    nb = sum(pages) + 3
    perm = rng.permutation(nb)
    table = np.full((len(lens), max(1, max(pages))), -1, np.int32)
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = perm[at:at + n]
        at += n
    total = sum(nodes)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).bfloat16()

    cu = np.zeros(len(nodes) + 1, np.int32)
    np.cumsum(nodes, out=cu[1:])
    parents = np.array(sum((_parents(rng, n, case["unused"]) for n in nodes), []), np.int32)
    return {"case": case, "q": normal(total, hq, d), "k": normal(total, hkv, d), "v": normal(total, hkv, d),
            "k_cache": normal(nb, hkv, PAGE, d), "v_cache": normal(nb, hkv, PAGE, d),
            "table": torch.from_numpy(table).cuda(), "cu": torch.from_numpy(cu).cuda(),
            "parents": torch.from_numpy(parents).cuda(), "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"),
            "max_nodes": max(nodes), "max_len": max(lens), "host": (lens, nodes, parents, table)}


def _branch_inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    n, g, new, hkv, d = case["prompts"], case["group"], case["new"], case["hkv"], case["d"]
    lens = _branch_lens(case)
    full = [-(-p // PAGE) for p in lens]
    stride = max(-(-(p + new) // PAGE) for p in lens) + 2
    extra = sum(-(-(p + new) // PAGE) - p // PAGE for p in lens) * g
    nb = sum(full) + extra + extra // 4 + 2
    perm = rng.permutation(nb)
    rows = n * (g + 1)
    table = np.full((rows, stride), -1, np.int32)
    row_lens = np.zeros(rows, np.int32)
    at = 0
    for i in range(n):
        table[i, :full[i]] = perm[at:at + full[i]]
        row_lens[i] = lens[i]
        at += full[i]
    # the branches of the step before, which this step drops: their prompt's whole pages and pages of their own
    src = np.repeat(np.arange(n), g).astype(np.int32)
    dst = np.arange(n, rows).astype(np.int32)
    for s, r in zip(src, dst):
        whole, need = lens[s] // PAGE, -(-(lens[s] + new) // PAGE)
        table[r, :whole] = table[s, :whole]
        table[r, whole:need] = perm[at:at + need - whole]
        at += need - whole
        row_lens[r] = lens[s] + new
    refs = np.bincount(table[table >= 0], minlength=nb).astype(np.int32)
    # a branch's tokens go behind what fork leaves it with: its prompt's length
    cu = np.zeros(rows + 1, np.int32)
    cu[n + 1:] = np.arange(1, n * g + 1) * new

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).bfloat16()

    def dev(a):
        return torch.from_numpy(np.ascontiguousarray(a)).cuda()

    return {"case": case, "table": dev(table), "lens": dev(row_lens), "refs": dev(refs), "src": dev(src), "dst": dev(dst),
            "k_cache": normal(nb, hkv, PAGE, d), "v_cache": normal(nb, hkv, PAGE, d), "cu": dev(cu),
            "k": normal(n * g * new, hkv, d), "v": normal(n * g * new, hkv, d), "new": new,
            "max_new": new, "host": (table, row_lens, refs, src, dst)}


def _compact_inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    nb, live, rows = case["pages"], case["live"], case["rows"]
    pages = rng.permutation(nb)[:live].astype(np.int32)
    # sequences of different lengths, the same for every seed
    parts = np.split(pages, [int(live * ((i + 1) / rows) ** 1.5) for i in range(rows - 1)])
    stride = max(1, max(len(p) for p in parts)) + 1
    table = np.full((rows, stride), -1, np.int32)
    for i, p in enumerate(parts):
        table[i, :len(p)] = p
    if rows > 1:  # the last row is a branch of the first: it shares all of its pages but its own tail
        keep = min(len(parts[0]), stride - 1)
        table[-1] = -1
        table[-1, :keep] = parts[0][:keep]
        tail = parts[-1][:stride - keep]
        table[-1, keep:keep + len(tail)] = tail
    refs = np.bincount(table[table >= 0], minlength=nb).astype(np.int32)
    hkv, d, layers = case["hkv"], case["d"], case["layers"]
    k = torch.randn(layers, nb, hkv, PAGE, d, device="cuda", generator=gen, dtype=torch.bfloat16)
    v = torch.randn(layers, nb, hkv, PAGE, d, device="cuda", generator=gen, dtype=torch.bfloat16)
    t, r = torch.from_numpy(table).cuda(), torch.from_numpy(refs).cuda()
    # the step's outputs go to buffers of their own: the pages' old places stay valid for whoever still reads them
    return {"case": case, "table": t, "refs": r, "k_cache": k, "v_cache": v, "table_out": torch.empty_like(t),
            "refs_out": torch.empty_like(r), "host": (table, refs)}


def prepare(case, seed):
    make = {"rope": _rope_inputs, "rope_bwd": _rope_inputs, "tree": _tree_inputs, "branch": _branch_inputs,
            "compact": _compact_inputs}
    return make[case["op"]](case, seed)


# ------------------------------------------------------------------ the passes
def run(state):
    op = state["case"]["op"]
    if own:
        return {"rope": _own_rope, "rope_bwd": _own_rope_bwd, "tree": _own_tree, "branch": _own_branch,
                "compact": _own_compact}[op](state)
    return {"rope": _plain_rope, "rope_bwd": _plain_rope_bwd, "tree": _plain_tree, "branch": _plain_branch,
            "compact": _plain_compact}[op](state)


def _own_rope(s):
    import paper_2608_14498_b200 as rpx

    return rpx.qk_norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], q_weight=s["qw"], k_weight=s["kw"],
                            pair_axis=s["pair_axis"], eps=s["eps"])


def _own_rope_bwd(s):
    import paper_2608_14498_b200 as rpx

    return rpx.qk_norm_rope_backward(s["q"], s["k"], s["dq"], s["dk"], s["positions"], s["inv_freq"], q_weight=s["qw"],
                                     k_weight=s["kw"], pair_axis=s["pair_axis"], eps=s["eps"])


def _own_tree(s):
    import paper_2608_14498_b200 as rpx

    return rpx.tree_attn(s["q"], s["k"], s["v"], s["cu"], s["parents"], s["lens"], s["max_nodes"], s["max_len"],
                         (s["k_cache"], s["v_cache"], s["table"]), return_lse=True)


def _own_branch(s):
    import paper_2608_14498_b200 as rpx

    rpx.pages_free(s["table"], s["lens"], s["refs"], s["dst"])
    pairs = rpx.pages_fork(s["table"], s["lens"], s["refs"], s["src"], s["dst"], s["new"])
    rpx.cache_copy_pages(s["k_cache"], s["v_cache"], *pairs)
    rpx.cache_append(s["k"], s["v"], s["cu"], s["lens"], s["max_new"], (s["k_cache"], s["v_cache"], s["table"]))
    return s["table"], s["lens"], s["refs"], pairs, s["k_cache"], s["v_cache"]


def _own_compact(s):
    import paper_2608_14498_b200 as rpx

    src, dst, n_live = rpx.pages_compact(s["table"], s["refs"], table_out=s["table_out"], ref_counts_out=s["refs_out"])
    rpx.cache_copy_pages(s["k_cache"], s["v_cache"], src, dst)
    return s["table_out"], s["refs_out"], src, dst, n_live, s["k_cache"], s["v_cache"]


# ------------------------------------------------------------------ plain forms
def _cos_sin(s):
    """cos, sin [tokens, 1, rot / 2] in 32 bits, the angles in 64."""
    pos = s["positions"].double()[s["pair_axis_dev"]]  # [rot / 2, tokens]
    angle = (pos * s["inv_freq"].double()[:, None]).t()[:, None]
    return torch.cos(angle).float(), torch.sin(angle).float()


def _turn(x, cos, sin):
    n = cos.shape[-1]
    a, b = x[..., :n], x[..., n:2 * n]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * n:]], -1)


def _plain_rope(s):
    cos, sin = _cos_sin(s)

    def one(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + s["eps"]) * w.float()
        return _turn(y, cos, sin).to(x.dtype)

    return one(s["q"], s["qw"]), one(s["k"], s["kw"])


def _plain_rope_bwd(s):
    cos, sin = _cos_sin(s)

    def one(x, dy, w):
        g = _turn(dy, cos, -sin)  # the transposed rotation
        if w is None:
            return g.to(x.dtype), None
        y = x.float()
        r = torch.rsqrt((y * y).mean(-1, keepdim=True) + s["eps"])
        u = y * r
        dw = (g * u).double().sum((0, 1)).float()
        g = g * w.float()
        return (r * (g - u * (g * u).mean(-1, keepdim=True))).to(x.dtype), dw

    (dq, dqw), (dk, dkw) = one(s["q"], s["dq"], s["qw"]), one(s["k"], s["dk"], s["kw"])
    return dq, dk, dqw, dkw


def _plain_tree(s):
    q, cu, lens = s["q"], s["cu"].long(), s["lens"].long()
    hq, d = q.shape[1:]
    hkv = s["k"].shape[1]
    n, p, dev = s["max_nodes"], s["max_len"], q.device
    b = lens.shape[0]
    counts = cu[1:] - cu[:-1]
    node = torch.arange(n, device=dev)
    there = node < counts[:, None]  # [b, n]
    at = (cu[:-1, None] + node).clamp(max=q.shape[0] - 1)
    parent = torch.where(there, s["parents"].long()[at], -2)
    used = parent > -2
    # ancestors: the inverse of (1 - A), A[i, parent of i] = 1, counts the paths from a node up to each other one: 0 or 1
    up = (parent[:, :, None] == node).float()
    eye = torch.eye(n, device=dev)
    reach = torch.linalg.solve_triangular(eye - up, eye.expand(b, n, n), upper=False) > 0.5
    own_seen = reach & used[:, :, None]
    pos = torch.arange(p, device=dev)
    page = s["table"].long()[:, pos // PAGE] if p else s["table"].long()[:, :0]
    seen = torch.cat([(pos < lens[:, None])[:, None].expand(b, n, p) & used[:, :, None], own_seen], 2)

    def keys(cache, x):
        old = cache.transpose(1, 2)[page.clamp(min=0), pos % PAGE].float()  # [b, p, hkv, d]
        both = torch.cat([old, x[at].float()], 1)
        return torch.where(seen.any(1)[:, :, None, None], both, 0.0)

    keys_k, keys_v = keys(s["k_cache"], s["k"]), keys(s["v_cache"], s["v"])
    qq = torch.where(there[:, :, None, None], q[at].float(), 0.0).view(b, n, hkv, hq // hkv, d)
    score = torch.einsum("bngid,bjgd->bgijn", qq, keys_k) / math.sqrt(d)  # [b, hkv, group, keys, n]
    hidden = ~seen.transpose(1, 2)[:, None, None]
    score = score.masked_fill(hidden, -math.inf)
    top = score.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(score - top)
    total = e.sum(3, keepdim=True)
    lse = (torch.log(total) + top)[:, :, :, 0]
    out = torch.einsum("bgijn,bjgd->bngid", e / torch.where(total > 0, total, 1.0), keys_v)
    flat = torch.nonzero(there.view(-1)).view(-1)
    out = out.reshape(b * n, hq, d)[flat].to(q.dtype)
    return out, lse.permute(0, 3, 1, 2).reshape(b * n, hq)[flat].contiguous()


def _plain_branch(s):
    table, lens, refs, new = s["table"], s["lens"], s["refs"], s["new"]
    src, dst = s["src"].long(), s["dst"].long()
    old = table[dst]
    old = old[old >= 0].long()
    refs.index_add_(0, old, torch.full_like(old, -1, dtype=torch.int32))
    table[dst] = -1
    # fork: whole pages shared, fresh pages behind them, the lowest free ones first
    have = lens[src].long()
    whole, need = have // PAGE, (have + new + PAGE - 1) // PAGE
    fresh = need - whole
    start = torch.cumsum(fresh, 0) - fresh
    free = torch.nonzero(refs == 0).view(-1)
    col = torch.arange(table.shape[1], device=table.device)
    own_col = (col >= whole[:, None]) & (col < need[:, None])
    pick = free[torch.where(own_col, start[:, None] + col - whole[:, None], 0).clamp(max=free.shape[0] - 1)].int()
    parent = table[src]
    shared = col < whole[:, None]
    rows = torch.where(shared, parent, torch.where(own_col, pick, -1))
    table[dst] = rows
    lens[dst] = have.int()
    held = rows[rows >= 0].long()
    refs.index_add_(0, held, torch.ones_like(held, dtype=torch.int32))
    part = have % PAGE != 0
    last = whole.clamp(max=table.shape[1] - 1)[:, None]
    pair_src = torch.where(part, torch.gather(parent, 1, last)[:, 0], -1)
    pair_dst = torch.where(part, torch.gather(rows, 1, last)[:, 0], -1)
    k_cache, v_cache = s["k_cache"], s["v_cache"]
    take, put = pair_src[part].long(), pair_dst[part].long()
    k_cache[put] = k_cache[take]
    v_cache[put] = v_cache[take]
    # the new tokens, one after the other behind each row's length
    cu = s["cu"].long()
    token = torch.arange(s["k"].shape[0], device=table.device)
    row = torch.searchsorted(cu, token, right=True) - 1
    pos = lens[row].long() + token - cu[row]
    page = table[row, pos // PAGE].long()
    k_cache[page, :, pos % PAGE] = s["k"]
    v_cache[page, :, pos % PAGE] = s["v"]
    return table, lens, refs, (pair_src, pair_dst), k_cache, v_cache


def _plain_compact(s):
    table, refs = s["table"], s["refs"]
    nb = refs.shape[0]
    live = refs > 0
    n_live = live.sum().int().view(1)
    page = torch.arange(nb, device=refs.device)
    high, low = torch.nonzero(live & (page >= n_live)).view(-1), torch.nonzero(~live & (page < n_live)).view(-1)
    to = page.clone()
    to[high] = low
    s["table_out"].copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), -1))
    s["refs_out"].copy_(torch.where(live, 0, refs))
    s["refs_out"][to[live]] = refs[live]
    src = torch.full((nb // 2,), -1, dtype=torch.int32, device=refs.device)
    dst = src.clone()
    src[:high.shape[0]], dst[:low.shape[0]] = high.int(), low.int()
    k_cache, v_cache = s["k_cache"], s["v_cache"]
    k_cache[:, low] = k_cache[:, high]
    v_cache[:, low] = v_cache[:, high]
    return s["table_out"], s["refs_out"], src, dst, n_live, k_cache, v_cache


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "rope_bwd": _exact_rope_bwd, "tree": _exact_tree, "branch": _exact_branch,
            "compact": _exact_compact}[case["op"]](s)


def _exact_one(s, x, w):
    """One tensor [tokens, heads, d] in 64 bits, as complex numbers turned by e^(i angle)."""
    if w is not None:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + s["eps"]) * w
    n = s["inv_freq"].shape[0]
    pos = torch.stack([s["positions"][a] for a in s["pair_axis"]], 1).double()
    z = torch.complex(x[..., :n], x[..., n:2 * n]) * torch.exp(1j * (pos * s["inv_freq"].double()))[:, None]
    return torch.cat([z.real, z.imag, x[..., 2 * n:]], -1)


def _exact_rope(s):
    return [_exact_one(s, s[n].double(), None if s[n + "w"] is None else s[n + "w"].double()) for n in ("q", "k")]


def _exact_rope_bwd(s):
    dx, dw = [], []
    for n in ("q", "k"):
        x = s[n].double().requires_grad_()
        w = None if s[n + "w"] is None else s[n + "w"].double().requires_grad_()
        got = torch.autograd.grad(_exact_one(s, x, w), [x] if w is None else [x, w], s["d" + n].double())
        dx.append(got[0])
        dw.append(got[1] if w is not None else None)
    return dx + dw


def _exact_tree(s):
    lens, nodes, parents, table = s["host"]
    hq, d = s["q"].shape[1:]
    hkv = s["k"].shape[1]
    outs, lses, at = [], [], 0
    for i, (p, n) in enumerate(zip(lens, nodes)):
        if not n:
            continue
        pages = torch.from_numpy(table[i, :-(-p // PAGE)].astype(np.int64)).cuda()

        def keys(cache, x):
            old = cache[pages].permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :p]
            return torch.cat([old, x[at:at + n].transpose(0, 1)], 1).double()

        kk, vv = keys(s["k_cache"], s["k"]), keys(s["v_cache"], s["v"])
        seen = np.zeros((n, p + n), bool)
        for j in range(n):
            up = int(parents[at + j])
            if up > -2:
                seen[j] = seen[j] if up < 0 else seen[up]
                seen[j, :p] = True
                seen[j, p + j] = True
        seen = torch.from_numpy(seen).cuda()
        for g in range(hkv):
            qq = s["q"][at:at + n, g * hq // hkv:(g + 1) * hq // hkv].transpose(0, 1).double()
            z = (qq @ kk[g].t() * d ** -0.5).masked_fill(~seen, -math.inf)
            lse = torch.logsumexp(z, -1)
            prob = torch.where(seen, torch.exp(z - lse[..., None]), 0.0)
            outs.append((at, g, (prob @ vv[g]).transpose(0, 1)))
            lses.append((at, g, lse.t()))
        at += n
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    group = hq // hkv
    for (a, g, o), (_, _, z) in zip(outs, lses):
        out[a:a + o.shape[0], g * group:(g + 1) * group] = o
        lse[a:a + o.shape[0], g * group:(g + 1) * group] = z
    return out, lse


def _exact_branch(s):
    table, lens, refs, src, dst = (a.copy() for a in s["host"])
    new = s["new"]
    for r in dst:
        for page in table[r][table[r] >= 0]:
            refs[page] -= 1
        table[r] = -1
    free = [i for i in range(refs.shape[0]) if refs[i] == 0]
    k, v = s["k_cache"].double(), s["v_cache"].double()
    pair_src, pair_dst, token = [], [], 0
    for a, r in zip(src, dst):
        whole, need = lens[a] // PAGE, -(-(lens[a] + new) // PAGE)
        table[r, :whole] = table[a, :whole]
        fresh, free = free[:need - whole], free[need - whole:]
        table[r, whole:need] = fresh
        lens[r] = lens[a]
        for page in table[r, :need]:
            refs[page] += 1
        partial = lens[a] % PAGE != 0
        pair_src.append(table[a, whole] if partial else -1)
        pair_dst.append(table[r, whole] if partial else -1)
        if partial:
            k[fresh[0]], v[fresh[0]] = k[int(table[a, whole])], v[int(table[a, whole])]
        pos = np.arange(lens[r], lens[r] + new)
        page, slot = torch.from_numpy(table[r][pos // PAGE].astype(np.int64)).cuda(), torch.from_numpy(pos % PAGE).cuda()
        k[page, :, slot], v[page, :, slot] = s["k"][token:token + new].double(), s["v"][token:token + new].double()
        token += new
    return table, lens, refs, (np.array(pair_src, np.int32), np.array(pair_dst, np.int32)), k, v


def _exact_compact(s):
    table, refs = s["host"]
    live = [i for i in range(refs.shape[0]) if refs[i] > 0]
    n = len(live)
    high = [i for i in live if i >= n]
    low = [i for i in range(n) if refs[i] == 0]
    move = dict(zip(high, low))
    new_refs = np.zeros_like(refs)
    for i in live:
        new_refs[move.get(i, i)] = refs[i]
    new_table = np.array([[move.get(int(p), int(p)) for p in row] for row in table], np.int32)
    pairs = np.full((2, refs.shape[0] // 2), -1, np.int32)
    pairs[0, :len(high)], pairs[1, :len(low)] = high, low
    k, v = s["k_cache"].clone(), s["v_cache"].clone()
    if high:
        k[:, low], v[:, low] = s["k_cache"][:, high], s["v_cache"][:, high]
    return new_table, new_refs, pairs[0], pairs[1], np.array([n], np.int32), k.double(), v.double()
