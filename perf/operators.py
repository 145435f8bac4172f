"""Performance cases of the sequence path: the user encoder that attends over the whole history, event by event, with a cache of
keys and values between requests.  Three operators of the public wrapper (`binding.Lime`), each a kind of case:

"rotate"   the norms of queries and keys for each head with the rotation by position, on the way into the cache
"history"  causal attention over packed histories of different lengths, grouped heads; new events behind older ones as well
"tree"     a few rows per user over the user's cached history, and over their ancestors among these rows: one new event, a list of
           candidates (all of them roots), or a tree of drafted continuations

Fields of every case: `dtype`, `Hq` query heads and `Hkv` heads of keys and values, of `dh` features each.  "rotate": `rows`, `rot`
rotated features in pairs (`inter`: of neighbours, else of halves), `far` the largest position, `cache` (keys and values go to cache rows
by slot, where `dense` also to a packed array).  "history" and "tree": `B` users with `n_min` .. `n_max` rows each, spread evenly and
dealt to the users by the seed, behind `c_min` .. `c_max` older ones.  "tree": `page` rows a cache page and `tree`, "none" (the rows are in
the cache already), "roots" or "drafts".
"""
import math

import torch

own = False

ES = {"f32": 4, "bf16": 2}
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
BASE, EPS = 10000.0, 1e-6


def rotate(dtype, Hq, Hkv, dh, rows, rot, inter=False, far=4096, cache=True, dense=True, **name):
    return dict(name, kind="rotate", dtype=dtype, Hq=Hq, Hkv=Hkv, dh=dh, rows=rows, rot=rot, inter=inter, far=far, cache=cache, dense=dense)


def history(dtype, Hq, Hkv, dh, B, n, c=(0, 0), **name):
    return dict(name, kind="history", dtype=dtype, Hq=Hq, Hkv=Hkv, dh=dh, B=B, n_min=n[0], n_max=n[1], c_min=c[0], c_max=c[1])


def tree(dtype, Hq, Hkv, dh, B, n, c, kind_of_tree, page=64, **name):
    return dict(name, kind="tree", dtype=dtype, Hq=Hq, Hkv=Hkv, dh=dh, B=B, n_min=n[0], n_max=n[1], c_min=c[0], c_max=c[1],
                tree=kind_of_tree, page=page)


def listed():
    return [
        # one new event of one user on its way into the cache: latency alone
        rotate("bf16", 4, 4, 32, 1, 32, far=1000, dense=False, name="rotate_one_event"),
        # the histories of the benchmark's batch, 256 users of 512 items, brought in for the first time
        rotate("bf16", 4, 4, 32, 256 * 512, 32, far=512, name="rotate_batch"),
        # lifelong histories of a wide model with grouped heads, an odd number of rows
        rotate("bf16", 16, 4, 128, 30011, 128, far=1_000_000, name="rotate_grouped"),
        # fp32 storage, half of the features rotated, neighbours paired, no cache
        rotate("f32", 8, 2, 64, 10007, 32, inter=True, cache=False, name="rotate_fp32"),
        # the smallest named workload: fp32 storage, a handful of short histories
        history("f32", 2, 2, 32, 4, (64, 64), name="history_tiny_fp32"),
        # ragged histories of an ordinary batch, one of them empty
        history("bf16", 4, 4, 32, 100, (0, 1000), name="history_ragged"),
        # one lifelong history of a wide model, grouped heads
        history("bf16", 16, 4, 128, 1, (16384, 16384), name="history_grouped_long"),
        # new events behind histories that are there already
        history("bf16", 8, 2, 64, 24, (1, 100), (1024, 4096), name="history_append"),
        # one user's newest event over the cached history: latency
        tree("bf16", 8, 2, 64, 1, (1, 1), (1000, 1000), "none", name="tree_one_event"),
        # one new event each of a batch of users, from new ones to those of lifelong histories
        tree("bf16", 16, 4, 128, 64, (1, 1), (16, 16384), "none", name="tree_events"),
        # candidates scored by attention: each sees the history and itself
        tree("bf16", 8, 8, 32, 32, (1000, 1000), (1024, 1024), "roots", name="tree_candidates"),
        # drafted continuations of some users, fp32 storage
        tree("f32", 8, 2, 64, 7, (5, 63), (100, 3000), "drafts", page=16, name="tree_drafts_fp32"),
    ]


def draw(rng):
    def log(a, b):
        return max(a, min(b, round(math.exp(rng.uniform(math.log(a), math.log(b + 1))))))

    kind = rng.choice(["rotate", "history", "history", "tree", "tree", "tree"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    Hkv = rng.choice([1, 2, 4, 8])
    Hq = Hkv * rng.choice([1, 1, 2, 3, 4])
    dh = rng.choice([16, 32, 40, 64, 64, 96, 128])
    if kind == "rotate":
        rows = log(1, 100_000 * 512 // ((Hq + 2 * Hkv) * dh) // (2 if dtype == "f32" else 1))
        cache = rng.random() < 0.6
        return rotate(dtype, Hq, Hkv, dh, rows, rng.choice([dh, dh, dh // 2]), inter=rng.random() < 0.3, far=log(10, 1 << 24), cache=cache,
                      dense=not cache or rng.random() < 0.5)
    if kind == "history":
        n = log(1, 8192)
        B = log(1, max(1, min(256, 600_000_000 // (Hq * n * n), 60_000 // n)))
        c = log(1, 4096) if rng.random() < 0.4 else 0
        if Hq * B * n * (n + c) > 1_000_000_000:
            c = 0
        return history(dtype, Hq, Hkv, dh, B, (rng.choice([0, 1, n // 2, n]), n), (rng.choice([0, c // 2, c]), c))
    form = rng.choice(["none", "roots", "drafts"])
    n = {"none": rng.choice([1, 1, log(1, 16)]), "roots": log(1, 1500), "drafts": log(2, 256)}[form]
    c = log(1, 20_000)
    B = log(1, max(1, min(128, 400_000_000 // (Hq * n * (n + c)), 60_000_000 // (c * Hkv * dh))))
    return tree(dtype, Hq, Hkv, dh, B, (rng.choice([1, (n + 1) // 2, n]), n), (rng.choice([0, c // 4, c]), c), form, page=rng.choice([16, 32, 64, 128]))


# ----------------------------------------------------------------------------- the sizes of a case
def spread(lo, hi, B):
    return [lo + (hi - lo) * b // max(1, B - 1) for b in range(B)] if B > 1 else [hi]


def lengths(case, rng):
    """New rows and older ones of every user: spread evenly, dealt by the seed."""
    n, c = spread(case["n_min"], case["n_max"], case["B"]), spread(case["c_min"], case["c_max"], case["B"])
    if rng is not None:
        at = torch.randperm(case["B"], generator=rng).tolist()
        n, c = [n[i] for i in at], [c[i] for i in at]
    return n, c


def work(case):
    es, Hq, Hkv, dh = ES[case["dtype"]], case["Hq"], case["Hkv"], case["dh"]
    if case["kind"] == "rotate":
        rows = case["rows"]
        moved = 2 * Hq + Hkv + Hkv * (int(case["dense"] or not case["cache"]) + (3 if case["cache"] else 0))
        return {"bytes": rows * moved * dh * es + rows * 4, "flops": rows * (Hq + Hkv) * (4 * dh + 3 * case["rot"])}
    n, c = lengths(case, None)
    rows = sum(n)
    if case["kind"] == "history":
        keys, seen = sum(n) + sum(c), sum(a * b + a * (a + 1) // 2 for a, b in zip(n, c))
    else:
        fresh = case["tree"] != "none"
        keys, seen = sum(c) + (rows if fresh else 0), sum(a * (b + (1 if fresh else 0)) for a, b in zip(n, c))
    return {"bytes": (2 * rows * Hq + 2 * keys * Hkv) * dh * es, "flops": 4 * seen * Hq * dh}


# ----------------------------------------------------------------------------- inputs
def offsets(n):
    return torch.tensor([0] + n).cumsum(0).to(torch.int32).cuda()


def prepare(case, seed):
    host = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, Hq, Hkv, dh = TYPE[case["dtype"]], case["Hq"], case["Hkv"], case["dh"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(t)

    s = dict(case=case)
    if own:
        from paper_2510_18239_b200 import binding
        s["lime"] = lime = binding.Lime(d=128, H=4, ell=32, n_layers=1, dtype=binding.LIME_F32 if case["dtype"] == "f32" else binding.LIME_BF16)
        lime.set_sequence(Hq, Hkv, dh, norm_eps=EPS, rot_dim=case.get("rot", 0), rot_interleaved=case.get("inter", False), rot_base=BASE)
    if case["kind"] == "rotate":
        rows = case["rows"]
        qkv = normal(rows, Hq + 2 * Hkv, dh)                    # what one projection leaves: queries, keys and values side by side
        s.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:])
        s.update(gq=(1 + 0.1 * torch.randn(dh, generator=gen, device="cuda")).to(t), gk=(1 + 0.1 * torch.randn(dh, generator=gen, device="cuda")).to(t))
        s["pos"] = torch.randint(0, case["far"], (rows,), generator=gen, device="cuda", dtype=torch.int32)
        if case["cache"]:
            slots = rows + rows // 8 + 64                       # the cache has rows that are not written
            s["slots"] = torch.randperm(slots, generator=gen, device="cuda")[:rows].to(torch.int32)
            pages = -(-slots // 64)
            s["cache_k"], s["cache_v"] = normal(pages, 64, Hkv, dh), normal(pages, 64, Hkv, dh)
        return s
    n, c = lengths(case, host)
    rows = sum(n)
    s["off"], s["n_most"], s["c_most"] = offsets(n), max(n), max(c)
    s["user"] = torch.repeat_interleave(torch.arange(case["B"]), torch.tensor(n)).cuda()
    s["q"] = normal(rows, Hq, dh)
    if case["kind"] == "history":
        s["kv_off"] = offsets([a + b for a, b in zip(n, c)])
        s["k"], s["v"] = normal(rows + sum(c), Hkv, dh), normal(rows + sum(c), Hkv, dh)
        return s
    page = case["page"]
    need = [-(-b // page) for b in c]
    pool = sum(need) + 3
    order = torch.randperm(pool, generator=host, dtype=torch.int32)
    table = torch.full((case["B"], max(1, max(need))), -1, dtype=torch.int32)
    first = 0
    for b, m in enumerate(need):
        table[b, :m] = order[first:first + m]
        first += m
    s["table"], s["ctx"] = table.cuda(), torch.tensor(c, dtype=torch.int32).cuda()
    s["cache_k"], s["cache_v"] = normal(pool, page, Hkv, dh), normal(pool, page, Hkv, dh)
    if case["tree"] != "none":
        s["k"], s["v"] = normal(rows, Hkv, dh), normal(rows, Hkv, dh)
    if case["tree"] == "drafts":
        place = torch.arange(rows, device="cuda") - s["off"].long()[s["user"]]
        s["parent"] = (torch.rand(rows, generator=gen, device="cuda") * place).floor().long().minimum(place - 1).to(torch.int32)
    return s


# ----------------------------------------------------------------------------- one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        lime = s["lime"]
        if kind == "rotate":
            both = s["case"]["cache"] and s["case"]["dense"]
            q, k = lime.norm_rotate(s["q"], s["k"], s["pos"], v=s["v"] if s["case"]["cache"] else None, gamma_q=s["gq"], gamma_k=s["gk"],
                                    cache_k=s.get("cache_k"), cache_v=s.get("cache_v"), slots=s.get("slots"), keep_k=both)
            return {"q": q, "k": k, "cache_k": s.get("cache_k"), "cache_v": s.get("cache_v")}
        if kind == "history":
            return lime.attend_history(s["q"], s["k"], s["v"], s["off"], kv_off=s["kv_off"])
        return lime.attend_tree(s["q"], s["cache_k"], s["cache_v"], s["table"], s["ctx"], s["off"], parent=s.get("parent"), tree_k=s.get("k"), tree_v=s.get("v"))
    return {"rotate": plain_rotate, "history": plain_history, "tree": plain_tree}[kind](s)


def plain_norm_rotate(x, gamma, cos, sin, case):
    x = x.float()
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gamma.float()
    rot = case["rot"]
    turned = x[..., :rot].reshape(x.shape[0], x.shape[1], rot // 2, 2).transpose(2, 3) if case["inter"] else x[..., :rot].reshape(x.shape[0], x.shape[1], 2, rot // 2)
    a, b = turned[:, :, 0], turned[:, :, 1]
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), 3) if case["inter"] else torch.stack((a, b), 2)
    return torch.cat((turned.reshape(x.shape[0], x.shape[1], rot), x[..., rot:]), -1)


def plain_rotate(s):
    case = s["case"]
    rot, t = case["rot"], TYPE[case["dtype"]]
    angle = s["pos"].double()[:, None, None] * BASE ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    cos, sin = angle.cos().float(), angle.sin().float()
    q, k = plain_norm_rotate(s["q"], s["gq"], cos, sin, case).to(t), plain_norm_rotate(s["k"], s["gk"], cos, sin, case).to(t)
    if not case["cache"]:
        return {"q": q, "k": k, "cache_k": None, "cache_v": None}
    at = s["slots"].long()
    s["cache_k"].view(-1, case["Hkv"], case["dh"])[at] = k
    s["cache_v"].view(-1, case["Hkv"], case["dh"])[at] = s["v"]
    return {"q": q, "k": k if case["dense"] else None, "cache_k": s["cache_k"], "cache_v": s["cache_v"]}


def plain_attention(q, k, v, visible, case):
    """q [B, n, Hq, dh], k and v [B, m, Hkv, dh], visible [B, n, m]; a row that sees nothing is zero."""
    B, n, m, Hkv, G, dh = q.shape[0], q.shape[1], k.shape[1], case["Hkv"], case["Hq"] // case["Hkv"], case["dh"]
    q = q.float().reshape(B, n, Hkv, G, dh).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, dh)
    p = torch.matmul(q, k.float().permute(0, 2, 3, 1)).mul_(1 / math.sqrt(dh)).view(B, Hkv, G, n, m)
    p.masked_fill_(~visible[:, None, None], -math.inf)
    most = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(most == -math.inf, 0.0, most)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, G * n, m), v.float().permute(0, 2, 1, 3)).view(B, Hkv, G, n, dh)
    o = o / torch.where(total == 0, 1.0, total)
    return o.permute(0, 3, 1, 2, 4).reshape(B, n, case["Hq"], dh)


def padded(x, off, most):
    """Rows of every user side by side, [B, most, ...], and which of them there are."""
    off, at = off.long(), torch.arange(most, device="cuda")
    there = at < (off[1:] - off[:-1])[:, None]
    return x[torch.where(there, off[:-1, None] + at, 0)] if x.shape[0] else x.new_zeros((len(off) - 1, most) + x.shape[1:]), there


def packed(o, s):
    return o[s["user"], torch.arange(len(s["user"]), device="cuda") - s["off"].long()[s["user"]]].to(TYPE[s["case"]["dtype"]])


def plain_history(s):
    q, new = padded(s["q"], s["off"], s["n_most"])
    k, there = padded(s["k"], s["kv_off"], s["n_most"] + s["c_most"])
    v, _ = padded(s["v"], s["kv_off"], s["n_most"] + s["c_most"])
    old = (there.sum(1) - new.sum(1))[:, None, None]
    i, j = torch.arange(q.shape[1], device="cuda")[None, :, None], torch.arange(k.shape[1], device="cuda")[None, None]
    return packed(plain_attention(q, k, v, (j <= i + old) & there[:, None] & new[:, :, None], s["case"]), s)


def plain_tree(s):
    case = s["case"]
    q, new = padded(s["q"], s["off"], s["n_most"])
    B, n = q.shape[:2]
    at = s["table"].long().clamp(min=0)
    k, v = (s[x][at].reshape(B, -1, case["Hkv"], case["dh"]) for x in ("cache_k", "cache_v"))
    visible = ((torch.arange(k.shape[1], device="cuda") < s["ctx"][:, None])[:, None] & new[:, :, None])
    if case["tree"] != "none":
        k, v = torch.cat((k, padded(s["k"], s["off"], n)[0]), 1), torch.cat((v, padded(s["v"], s["off"], n)[0]), 1)
        sees = torch.eye(n, device="cuda").expand(B, n, n)
        if case["tree"] == "drafts":
            # ancestors: with P the matrix of parents, the sum of its powers is the inverse of I - P, ones and zeros
            parent = torch.where(new, padded(s["parent"], s["off"], n)[0].long(), -1)
            step = sees - (parent[:, :, None] == torch.arange(n, device="cuda")).float()
            sees = torch.linalg.solve_triangular(step, sees, upper=False, unitriangular=True)
        visible = torch.cat((visible, (sees > 0.5) & new[:, :, None] & new[:, None]), 2)
    return packed(plain_attention(q, k, v, visible, case), s)


# ----------------------------------------------------------------------------- the definition, in 64 bits
def exact_turn(x, gamma, pos, case):
    x = x.double()
    y = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * gamma.double()
    out, rot = y.clone(), case["rot"]
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if case["inter"] else (i, i + rot // 2)
        angle = pos.double() * BASE ** (-2 * i / rot)
        out[..., a] = y[..., a] * angle.cos()[:, None] - y[..., b] * angle.sin()[:, None]
        out[..., b] = y[..., a] * angle.sin()[:, None] + y[..., b] * angle.cos()[:, None]
    return out


def exact_head(q, k, v, sees):
    """softmax over the keys a row sees, one head of keys: q [G, n, dh], k and v [m, dh], sees [n, m]."""
    score = torch.einsum("gnd,md->gnm", q.double(), k.double()) / math.sqrt(q.shape[-1])
    e = torch.where(sees, (score - torch.where(sees, score, -1e300).amax(-1, keepdim=True)).exp(), 0.0)
    return torch.einsum("gnm,md->gnd", e, v.double()) / e.sum(-1, keepdim=True).clamp(min=1e-300)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotate":
        q, k = exact_turn(s["q"], s["gq"], s["pos"], case), exact_turn(s["k"], s["gk"], s["pos"], case)
        if not case["cache"]:
            return {"q": q, "k": k, "cache_k": None, "cache_v": None}
        caches = [s[x].double().flatten(0, 1) for x in ("cache_k", "cache_v")]
        caches[0].index_copy_(0, s["slots"].long(), k)
        caches[1].index_copy_(0, s["slots"].long(), s["v"].double())
        return {"q": q, "k": k if case["dense"] else None, "cache_k": caches[0].reshape(s["cache_k"].shape), "cache_v": caches[1].reshape(s["cache_v"].shape)}
    off, G, out = s["off"].tolist(), case["Hq"] // case["Hkv"], torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        r, n = slice(off[b], off[b + 1]), off[b + 1] - off[b]
        if n == 0:
            continue
        if case["kind"] == "history":
            at = s["kv_off"].tolist()
            k, v = s["k"][at[b]:at[b + 1]], s["v"][at[b]:at[b + 1]]
            sees = torch.ones(n, len(k), dtype=torch.bool, device="cuda").tril(len(k) - n)
        else:
            c = int(s["ctx"][b])
            pages = s["table"][b, :-(-c // case["page"])].long()
            k, v = (s[x][pages].flatten(0, 1)[:c] for x in ("cache_k", "cache_v"))
            sees = torch.ones(n, c, dtype=torch.bool, device="cuda")
            if case["tree"] != "none":
                up = torch.zeros(n, n, dtype=torch.bool)
                parent = s["parent"][r].tolist() if case["tree"] == "drafts" else [-1] * n
                for i in range(n):
                    if parent[i] >= 0:
                        up[i] = up[parent[i]]
                    up[i, i] = True
                k, v, sees = torch.cat((k, s["k"][r])), torch.cat((v, s["v"][r])), torch.cat((sees, up.cuda()), 1)
        if len(k) == 0:
            continue
        for h in range(case["Hkv"]):
            out[r, h * G:(h + 1) * G] = exact_head(s["q"][r, h * G:(h + 1) * G].transpose(0, 1), k[:, h], v[:, h], sees).transpose(0, 1)
    return out
