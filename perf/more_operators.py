"""Operators of a prompt group's rollout step and of the loss it is trained on: plain forms, calls, and measured cases.

Three operators, in the order in which an iteration uses them:

  * ``append`` norm and rotation of queries and keys with K and V stored into the paged cache in the same pass;
  * ``group``  attention over the paged cache for sequences in groups (the responses to one prompt) that share the pages of
               their prompt, which are read once for the whole group; one query token per sequence (decoding) or several;
  * ``policy`` the clipped policy loss with a KL term over packed response log-probs, and its gradient.

``own = False`` computes them with elementary torch operations in 32 bits (64 for angles, long sums and the borders of the
clipping), ``own = True`` makes the library's calls.  Head shapes are those of the 7B- and 32B-shaped benchmark
configurations (28/4 and 40/8 heads of 128) and of the small float32 one (4/2 heads of 64).
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ cases
def _append(name, batch, new, ctx, hq, hkv, d, rot, axes, dtype, norm, ragged):
    return {"name": name, "op": "append", "batch": batch, "new": new, "ctx": ctx, "hq": hq, "hkv": hkv, "d": d, "rot": rot,
            "axes": axes, "dtype": dtype, "norm": norm, "ragged": ragged}


def _group(name, prompts, members, new, shared, own_len, hq, hkv, d, ragged):
    return {"name": name, "op": "group", "prompts": prompts, "members": members, "new": new, "shared": shared,
            "own_len": own_len, "hq": hq, "hkv": hkv, "d": d, "ragged": ragged}


def _policy(name, batch, tokens, ratio, mean, kl, masked, per_token):
    return {"name": name, "op": "policy", "batch": batch, "tokens": tokens, "ratio": ratio, "mean": mean, "kl": kl,
            "masked": masked, "per_token": per_token}


def listed():
    return [
        # one decoding step of 256 responses (7B shape, positions on three axes): latency
        _append("append_decode_256", 256, 1, 4700, 28, 4, 128, 128, 3, "bf16", True, False),
        # prompts of the 7B-shaped batch filled into the cache (8 x 4096 tokens of video)
        _append("append_prompts_8x4096", 8, 4096, 0, 28, 4, 128, 128, 3, "bf16", True, False),
        # ragged chunks of the 32B shape behind what is cached already
        _append("append_chunks_32x509", 32, 509, 5003, 40, 8, 128, 128, 3, "bf16", True, True),
        # the small float32 configuration, partial rotation, no norm, odd lengths
        _append("append_f32_3x97", 3, 97, 61, 4, 2, 64, 32, 1, "f32", False, True),
        # 8 responses to one prompt, a decoding step: latency
        _group("group_decode_1x8", 1, 8, 1, 4096, 200, 28, 4, 128, False),
        # the ordinary step: 32 prompts of ragged length with 8 responses each (32B shape)
        _group("group_decode_32x8", 32, 8, 1, 8190, 1000, 40, 8, 128, True),
        # many samples of a few long prompts: more query rows than one tile holds
        _group("group_decode_4x64", 4, 64, 1, 16384, 500, 28, 4, 128, True),
        # several drafted tokens per response are checked at once
        _group("group_verify_8x8x5", 8, 8, 5, 6001, 300, 28, 4, 128, True),
        # one prompt's group of 8 short answers: latency
        _policy("policy_8x250", 8, 250, "token", "sequences", 3, False, False),
        # an iteration's batch: 32 prompts x 8 responses of up to 2048 tokens, some tokens masked
        _policy("policy_256x2048", 256, 2048, "token", "tokens", 3, True, False),
        # the ratio taken over whole responses
        _policy("policy_seq_512x1777", 512, 1777, "sequence", "sequences", 2, True, False),
        # a large batch with an advantage for every token
        _policy("policy_1024x4096", 1024, 4096, "token", "sequences", 3, True, True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "append", "group", "group", "group", "policy", "policy"])
    limit = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        hq, hkv = rng.choice([(28, 4), (40, 8), (28, 4), (40, 8), (4, 2), (8, 8), (16, 1), (12, 4)])
        d = rng.choice([64, 128, 128])
        if op == "append":
            c = _append("", _log(rng, 1, 300), _log(rng, 1, 5000), rng.choice([0, _log(rng, 1, 9000)]), hq, hkv, d,
                        rng.choice([16, 32, 48, d // 2, d, d]), rng.choice([1, 2, 3, 3]), rng.choice(["bf16", "bf16", "f32"]),
                        rng.random() < 0.7, rng.random() < 0.6)
        elif op == "group":
            c = _group("", _log(rng, 1, 40), _log(rng, 1, 64), rng.choice([1, 1, 1, _log(rng, 2, 16)]), _log(rng, 1, 32768),
                       _log(rng, 1, 2048), hq, hkv, d, rng.random() < 0.7)
        else:
            ratio = rng.choice(["token", "token", "sequence"])
            c = _policy("", _log(rng, 1, 4096), _log(rng, 1, 8192), ratio, rng.choice(["tokens", "sequences"]),
                        rng.choice([0, 1, 2, 3, 3]), rng.random() < 0.6, ratio == "token" and rng.random() < 0.4)
        del c["name"]
        if _cost(c) <= limit and (op != "group" or c["prompts"] * c["members"] <= 512):
            return c


def _cost(case):
    w = work(case)
    return w["bytes"] / 6.5e12 + w["flops"] / 1.4e15


def _spread(n, at=0.25):
    """Numbers spread evenly over [0, 1), the same for every seed."""
    return [(i * 0.6180339887498949 + at) % 1.0 for i in range(n)]


def _append_lens(case):
    """New tokens and cached tokens of every sequence."""
    b, new, ctx = case["batch"], case["new"], case["ctx"]
    if not case["ragged"]:
        return [new] * b, [ctx] * b
    return ([max(0 if b > 4 and i % 7 == 3 else 1, new - int(x * 0.8 * new)) for i, x in enumerate(_spread(b))],
            [ctx - int(x * 0.9 * ctx) for x in _spread(b, 0.6)])


def _group_lens(case):
    """Shared tokens of every prompt; own tokens (the query tokens among them) and query tokens of every response."""
    g, m, new = case["prompts"], case["members"], case["new"]
    if not case["ragged"]:
        return [case["shared"]] * g, [case["own_len"] + new] * (g * m), [new] * (g * m)
    news = [new - int(x * new * 0.6) for x in _spread(g * m, 0.7)]
    return ([case["shared"] - int(x * 0.8 * case["shared"]) for x in _spread(g)],
            [n + int(x * case["own_len"]) for x, n in zip(_spread(g * m, 0.4), news)], news)


def _policy_lens(case):
    return [max(0 if case["batch"] > 4 and i % 61 == 7 else 1, case["tokens"] - int(x * 0.9 * case["tokens"]))
            for i, x in enumerate(_spread(case["batch"]))]


def work(case):
    if case["op"] == "append":
        tokens, d = sum(_append_lens(case)[0]), case["d"]
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": float(tokens * d * (2 * size * case["hq"] + 2 * (size + 2) * case["hkv"]) + 4 * tokens * case["axes"]),
                "flops": float(8 * tokens * d * (case["hq"] + case["hkv"]))}
    if case["op"] == "group":
        shared, own_lens, news = _group_lens(case)
        d, hq, m = case["d"], case["hq"], case["members"]
        # the prompt's whole pages once for the group, its partial page and the response for every member
        whole = [p // PAGE * PAGE for p in shared]
        keys = sum(whole) + sum(shared[i // m] - whole[i // m] + n for i, n in enumerate(own_lens))
        pairs = sum(n * (shared[i // m] + o) - n * (n - 1) // 2 for i, (o, n) in enumerate(zip(own_lens, news)))
        return {"bytes": float(keys * case["hkv"] * d * 4 + sum(news) * hq * (4 * d + 4)), "flops": float(4 * d * hq * pairs)}
    tokens = sum(_policy_lens(case))
    per = 12 + (4 if case["kl"] else 0) + (1 if case["masked"] else 0) + (4 if case["per_token"] else 0)
    return {"bytes": float(tokens * per + 8 * case["batch"]), "flops": float(40 * tokens)}


# ------------------------------------------------------------------ inputs
def _pair_axis(case):
    """Which position axis turns each rotary pair: a quarter of the pairs for time and the rest for height and width."""
    n, axes = case["rot"] // 2, case["axes"]
    if axes == 1:
        return [0] * n
    sizes = [n - 2 * (3 * n // 8), 3 * n // 8, 3 * n // 8] if axes == 3 else [n - n // 2, n // 2]
    return [a for a, s in enumerate(sizes) for _ in range(s)]


def _cu(counts):
    cu = np.zeros(len(counts) + 1, np.int32)
    np.cumsum(counts, out=cu[1:])
    return cu


def _append_inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    hq, hkv, d, dt = case["hq"], case["hkv"], case["d"], DTYPES[case["dtype"]]
    new, ctx = _append_lens(case)
    t = sum(new)
    # the projection's output: q, k and v of a token side by side, so all three are strided views of it
    scale = torch.exp(0.5 * torch.randn(t, hq + 2 * hkv, 1, device="cuda", generator=gen))
    qkv = (torch.randn(t, hq + 2 * hkv, d, device="cuda", generator=gen) * scale).to(dt)
    pos = torch.randint(0, 96, (case["axes"], t), device="cuda", generator=gen, dtype=torch.int32)
    pos[0] = torch.from_numpy(np.concatenate([c + np.arange(n) for n, c in zip(new, ctx)]).astype(np.int32)).cuda()
    n = case["rot"] // 2
    pages = [-(-(a + c) // PAGE) for a, c in zip(new, ctx)]
    nb = sum(pages) + 3
    perm = rng.permutation(nb)
    table = np.full((len(new), max(1, max(pages))), -1, np.int32)
    at = 0
    for i, k in enumerate(pages):
        table[i, :k] = perm[at:at + k]
        at += k

    def pool():
        return torch.randn(nb, hkv, PAGE, d, device="cuda", generator=gen, dtype=torch.bfloat16)

    s = {"case": case, "q": qkv[:, :hq], "k": qkv[:, hq:hq + hkv], "v": qkv[:, hq + hkv:], "positions": pos,
         "inv_freq": (1000000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float64) / n)).float(),
         "pair_axis": _pair_axis(case), "eps": 1e-6, "qw": None, "kw": None, "cu": torch.from_numpy(_cu(new)).cuda(),
         "lens": torch.tensor(ctx, dtype=torch.int32, device="cuda"), "max_new": max(new), "k_cache": pool(),
         "v_cache": pool(), "table": torch.from_numpy(table).cuda(), "host": (new, ctx, table)}
    s["pair_axis_dev"] = torch.tensor(s["pair_axis"], device="cuda")
    if case["norm"]:
        s["qw"] = (1 + 0.2 * torch.randn(d, device="cuda", generator=gen)).to(dt)
        s["kw"] = (1 + 0.2 * torch.randn(d, device="cuda", generator=gen)).to(dt)
    return s


def _group_inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    m, hq, hkv, d = case["members"], case["hq"], case["hkv"], case["d"]
    shared, own_lens, news = _group_lens(case)
    kv = [shared[i // m] + n for i, n in enumerate(own_lens)]
    pages = [-(-n // PAGE) for n in kv]
    nb = sum(p // PAGE for p in shared) + sum(n - shared[i // m] // PAGE for i, n in enumerate(pages)) + 3
    perm = rng.permutation(nb)
    table = np.full((len(kv), max(pages)), -1, np.int32)
    at = 0
    for i, n in enumerate(pages):  # the first member brings the prompt's whole pages, the others name the same ones
        whole = shared[i // m] // PAGE
        if i % m == 0:
            prompt = perm[at:at + whole]
            at += whole
        table[i, :whole] = prompt
        table[i, whole:n] = perm[at:at + n - whole]
        at += n - whole

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen, dtype=torch.bfloat16)

    def dev(x):
        return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")

    return {"case": case, "q": normal(sum(news), hq, d), "k_cache": normal(nb, hkv, PAGE, d), "v_cache": normal(nb, hkv, PAGE, d),
            "table": dev(table), "cu": dev(_cu(news)), "kv_lens": dev(kv), "cu_groups": dev(np.arange(case["prompts"] + 1) * m),
            "shared": dev(shared), "max_new": max(news), "max_group": max(sum(news[i:i + m]) for i in range(0, len(news), m)),
            "max_kv": max(kv), "host": (kv, news)}


def _policy_inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    lens = _policy_lens(case)
    b, t = len(lens), sum(lens)

    def normal(n):
        return torch.randn(n, device="cuda", generator=gen)

    # the policy has moved a little since the responses were sampled, and further since the reference
    lp = torch.log(torch.rand(t, device="cuda", generator=gen).clamp(min=1e-6)) * 1.2
    s = {"case": case, "lp": lp, "old": lp + 0.15 * normal(t) * torch.exp(0.4 * normal(t)), "ref": None, "mask": None,
         "cu": torch.from_numpy(_cu(lens)).cuda(), "host": lens}
    if case["ratio"] == "sequence":  # whole responses move by less
        s["old"] = lp + torch.repeat_interleave(0.2 * normal(b), torch.tensor(lens, device="cuda")) + 0.15 * normal(t)
    if case["kl"]:
        s["ref"] = lp + 0.3 * normal(t)
    if case["masked"]:
        s["mask"] = torch.rand(t, device="cuda", generator=gen) < 0.9
    s["adv"] = normal(t if case["per_token"] else b)
    s["clip"] = (0.2, 0.28, 3.0)
    s["kl_coef"] = 0.02
    return s


def prepare(case, seed):
    return {"append": _append_inputs, "group": _group_inputs, "policy": _policy_inputs}[case["op"]](case, seed)


# ------------------------------------------------------------------ the passes
def run(state):
    op = state["case"]["op"]
    if own:
        return {"append": _own_append, "group": _own_group, "policy": _own_policy}[op](state)
    return {"append": _plain_append, "group": _plain_group, "policy": _plain_policy}[op](state)


def _own_append(s):
    import paper_2608_14498_b200 as rpx

    q = rpx.qk_norm_rope_append(s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], s["cu"], s["lens"], s["max_new"],
                                (s["k_cache"], s["v_cache"], s["table"]), q_weight=s["qw"], k_weight=s["kw"],
                                pair_axis=s["pair_axis"], eps=s["eps"])
    return q, s["k_cache"], s["v_cache"]


def _own_group(s):
    import paper_2608_14498_b200 as rpx

    return rpx.group_attn(s["q"], s["cu"], s["kv_lens"], s["cu_groups"], s["shared"], s["max_new"], s["max_group"], s["max_kv"],
                          (s["k_cache"], s["v_cache"], s["table"]), return_lse=True)


def _own_policy(s):
    import paper_2608_14498_b200 as rpx

    case, (low, high, dual) = s["case"], s["clip"]
    return rpx.policy_loss(s["lp"], s["old"], s["adv"], s["cu"], mask=s["mask"], ref_logprobs=s["ref"], clip_low=low,
                           clip_high=high, clip_dual=dual, kl_coef=s["kl_coef"], kl=case["kl"], ratio=case["ratio"],
                           mean=case["mean"])


# ------------------------------------------------------------------ plain forms
def _slots(s, token):
    """Page and place in it of new tokens."""
    cu = s["cu"].long()
    row = torch.searchsorted(cu, token, right=True) - 1
    pos = s["lens"].long()[row] + token - cu[row]
    return s["table"].long()[row, pos // PAGE], pos % PAGE


def _plain_append(s):
    pos = s["positions"].double()[s["pair_axis_dev"]]  # [rot / 2, tokens]
    angle = (pos * s["inv_freq"].double()[:, None]).t()[:, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    n = cos.shape[-1]

    def one(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + s["eps"]) * w.float()
        a, b = y[..., :n], y[..., n:2 * n]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., 2 * n:]], -1)

    page, place = _slots(s, torch.arange(s["k"].shape[0], device="cuda"))
    s["k_cache"][page, :, place] = one(s["k"], s["kw"]).bfloat16()
    s["v_cache"][page, :, place] = s["v"].bfloat16()
    return one(s["q"], s["qw"]).to(s["q"].dtype), s["k_cache"], s["v_cache"]


def _plain_group(s):
    kv, news = s["host"]
    hq, d = s["q"].shape[1:]
    hkv = s["k_cache"].shape[1]
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], device="cuda")
    at = 0
    for i, (length, n) in enumerate(zip(kv, news)):
        pages = s["table"][i, :-(-length // PAGE)].long()
        k, v = (c[pages].transpose(1, 2).reshape(-1, hkv, d)[:length].float() for c in (s["k_cache"], s["v_cache"]))
        q = s["q"][at:at + n].float().view(n, hkv, hq // hkv, d)
        score = torch.einsum("ngid,jgd->ngij", q, k) / math.sqrt(d)
        if n > 1:
            j = torch.arange(length, device="cuda")
            score = score.masked_fill((j > length - n + j[:n, None])[:, None, None], -math.inf)
        top = score.amax(-1, keepdim=True)
        e = torch.exp(score - top)
        total = e.sum(-1, keepdim=True)
        out[at:at + n] = torch.einsum("ngij,jgd->ngid", e / total, v).reshape(n, hq, d).to(out.dtype)
        lse[at:at + n] = (torch.log(total) + top).view(n, hq)
        at += n
    return out, lse


def _plain_policy(s):
    case, (low, high, dual) = s["case"], s["clip"]
    lp, old, cu = s["lp"], s["old"], s["cu"].long()
    b = cu.shape[0] - 1
    row = torch.repeat_interleave(torch.arange(b, device="cuda"), cu[1:] - cu[:-1])
    keep = s["mask"] if s["mask"] is not None else torch.ones_like(lp, dtype=torch.bool)
    tokens = torch.zeros(b, dtype=torch.float64, device="cuda").index_add_(0, row, keep.double())
    moved = torch.where(keep, lp.double() - old.double(), 0.0)  # 64 bits: what is next to a border falls on its own side
    if case["ratio"] == "sequence":
        total = torch.zeros(b, dtype=torch.float64, device="cuda").index_add_(0, row, moved)
        moved = (total / tokens.clamp(min=1.0))[row]
    adv = s["adv"] if case["per_token"] else s["adv"][row]
    clipped = ((adv > 0) & (moved > math.log1p(high))) | ((adv < 0) & ((moved < math.log1p(-low)) | (moved > math.log(dual))))
    ratio = torch.exp(moved.float())
    bound = torch.where(adv > 0, 1.0 + high, torch.where(moved < 0, 1.0 - low, dual))
    policy = -adv * torch.where(clipped, bound, ratio)
    grad = torch.where(clipped, 0.0, -adv * ratio)
    if case["mean"] == "tokens":
        w = keep.double() / tokens.sum().clamp(min=1.0)
    else:
        w = keep.double() / (tokens.clamp(min=1.0)[row] * (tokens > 0).sum().clamp(min=1))
    kl = torch.zeros_like(lp)
    if case["kl"]:
        x = s["ref"].double() - lp.double()  # 64 bits: the terms of the third estimator all but cancel
        kl = {1: -x, 2: 0.5 * x * x, 3: torch.expm1(x) - x}[case["kl"]].float()
        grad = grad + s["kl_coef"] * {1: torch.ones_like(x), 2: -x, 3: -torch.expm1(x)}[case["kl"]].float()

    def mean(x):
        return (w * x.double()).sum()

    p, k = mean(policy), mean(kl)
    stats = torch.stack([p + s["kl_coef"] * k, p, k, mean(clipped), mean(ratio), tokens.sum()]).float()
    return stats, (w.float() * grad)


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    return {"append": _exact_append, "group": _exact_group, "policy": _exact_policy}[case["op"]](prepare(case, seed))


def _exact_append(s):
    def one(x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + s["eps"]) * w.double()
        n = s["inv_freq"].shape[0]
        pos = torch.stack([s["positions"][a] for a in s["pair_axis"]], 1).double()
        z = torch.complex(x[..., :n], x[..., n:2 * n]) * torch.exp(1j * (pos * s["inv_freq"].double()))[:, None]
        return torch.cat([z.real, z.imag, x[..., 2 * n:]], -1)

    new, ctx, table = s["host"]
    k, v = s["k_cache"].double(), s["v_cache"].double()
    turned, at = one(s["k"], s["kw"]), 0
    for i, (n, c) in enumerate(zip(new, ctx)):
        pos = np.arange(c, c + n)
        page, place = torch.from_numpy(table[i][pos // PAGE].astype(np.int64)).cuda(), torch.from_numpy(pos % PAGE).cuda()
        k[page, :, place], v[page, :, place] = turned[at:at + n], s["v"][at:at + n].double()
        at += n
    return one(s["q"], s["qw"]), k, v


def _exact_group(s):
    kv, news = s["host"]
    t, hq, d = s["q"].shape
    hkv = s["k_cache"].shape[1]
    out = torch.zeros(t, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(t, hq, dtype=torch.float64, device="cuda")
    at, step = 0, hq // hkv
    for i, (length, n) in enumerate(zip(kv, news)):
        pages = s["table"][i, :-(-length // PAGE)].long()
        k = s["k_cache"][pages].permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :length].double()
        v = s["v_cache"][pages].permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :length].double()
        q = s["q"][at:at + n].double().permute(1, 0, 2).reshape(hkv, step * n, d)  # rows: head, then token
        z = torch.bmm(q, k.transpose(1, 2)) * d ** -0.5
        seen = torch.ones(n, length, dtype=torch.bool, device="cuda").tril(length - n).repeat(step, 1)
        z = torch.where(seen, z, -math.inf)
        total = torch.logsumexp(z, -1)
        o = torch.bmm(torch.exp(z - total[..., None]), v)
        out[at:at + n] = o.view(hq, n, d).transpose(0, 1)
        lse[at:at + n] = total.view(hq, n).t()
        at += n
    return out, lse


def _exact_policy(s):
    case, (low, high, dual) = s["case"], s["clip"]
    lens = s["host"]
    lp, old, adv = (s[n].double().cpu() for n in ("lp", "old", "adv"))
    ref = None if s["ref"] is None else s["ref"].double().cpu()
    keep = torch.ones(lp.shape, dtype=torch.bool) if s["mask"] is None else s["mask"].cpu()
    starts = _cu(lens)
    counts = [int(keep[starts[i]:starts[i + 1]].sum()) for i in range(len(lens))]
    total, seqs = sum(counts), sum(1 for n in counts if n)
    sums, grad = [0.0] * 5, torch.zeros_like(lp)
    for i, n in enumerate(counts):
        if not n:
            continue
        at = torch.nonzero(keep[starts[i]:starts[i + 1]])[:, 0] + int(starts[i])
        x = lp[at] - old[at]
        if case["ratio"] == "sequence":
            x = x.mean().expand(n)
        a = adv[at] if case["per_token"] else adv[i].expand(n)
        r = torch.exp(x)
        first, second = -a * r, -a * torch.clamp(r, 1.0 - low, 1.0 + high)
        loss = torch.maximum(first, second)
        loss = torch.where((a < 0) & (-a * dual < loss), -a * dual, loss)
        cut = loss != first
        w = 1.0 / total if case["mean"] == "tokens" else 1.0 / (n * seqs)
        g = torch.where(cut, 0.0, first)
        kl = torch.zeros(n, dtype=torch.float64)
        if case["kl"]:
            y = ref[at] - lp[at]
            kl = {1: -y, 2: y * y / 2, 3: torch.expm1(y) - y}[case["kl"]]
            g = g + s["kl_coef"] * {1: torch.ones_like(y), 2: -y, 3: 1.0 - torch.exp(y)}[case["kl"]]
        grad[at] = w * g
        for j, part in enumerate((loss + s["kl_coef"] * kl, loss, kl, cut.double(), r)):
            sums[j] += w * float(part.sum())
    return torch.tensor(sums + [float(total)], dtype=torch.float64), grad
