"""Attention beside the experts, as measurable cases.

A transformer layer has attention ahead of its experts.  A prompt or a training batch goes through it as rows, packed sequence
after sequence; decoded tokens read a cache of pages.

  plan   pages for the tokens that requests bring, taken from the free ones, and where each token goes: tables, slots, positions
  store  keys and values of new tokens put into their pages, as bf16 or as 8-bit codes with a scale per token and head
  pages  attention of one new token per sequence over its pages
  rows   attention of packed sequences, causal; the queries are the last rows of their sequence; `train`: with gradients

Key j is visible to the query at position p if j <= p and, with a window, j > p - window or j < sinks.

The plain forms compute in 32 bits, whatever the inputs' type, and round at the end; `exact` does the same from the definitions
in 64 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "int8": torch.int8}
SIZE = {"bf16": 2, "fp32": 4, "int8": 1}
ROOM = 1 << 28  # elements of a plain form's largest temporary


# ---- the cases -------------------------------------------------------------------------------------------
def listed():
    return [
        # One decoding step of eight requests: a token each.
        dict(name="plan_step", kind="plan", seqs=8, longest=4000, new=1, page=16, short=False),
        # Many prompts arrive together, some requests bring nothing, and the free pages do not last for all of them.
        dict(name="plan_prompts", kind="plan", seqs=1024, longest=9000, new=700, page=32, short=True),
        # The keys and values of one decoding step.
        dict(name="store_step", kind="store", tokens=8, kv=16, dim=128, page=16, x="bf16", cache="bf16"),
        # The keys and values of a long prompt, into an 8-bit cache.
        dict(name="store_prompt_int8", kind="store", tokens=8191, kv=8, dim=128, page=64, x="bf16", cache="int8"),
        # One request, the next token: latency.
        dict(name="pages_token", kind="pages", seqs=1, longest=777, heads=16, kv=16, dim=128, page=16, cache="bf16", window=0, sinks=0),
        # A batch of requests of all lengths, groups of four heads, 8-bit cache.
        dict(name="pages_batch_int8", kind="pages", seqs=64, longest=8192, heads=32, kv=8, dim=128, page=64, cache="int8", window=0,
             sinks=0),
        # A few very long requests: their caches are split over the whole GPU.
        dict(name="pages_long", kind="pages", seqs=4, longest=131072, heads=32, kv=8, dim=128, page=32, cache="bf16", window=0, sinks=0),
        # Long requests of a model that looks back a window and at its first tokens.
        dict(name="pages_window", kind="pages", seqs=96, longest=20000, heads=32, kv=4, dim=64, page=16, cache="bf16", window=4096,
             sinks=4),
        # A short prompt of an odd length.
        dict(name="rows_prompt_odd", kind="rows", seqs=1, tokens=333, before=0, heads=16, kv=16, dim=128, window=0, sinks=0, train=False),
        # A long prompt in one piece.
        dict(name="rows_prompt_long", kind="rows", seqs=1, tokens=16384, before=0, heads=32, kv=8, dim=128, window=0, sinks=0, train=False),
        # A training batch of packed sequences, forwards and backwards.
        dict(name="rows_train", kind="rows", seqs=5, tokens=8192, before=0, heads=16, kv=16, dim=128, window=0, sinks=0, train=True),
        # The same with a window, sinks, groups of eight heads and narrow heads.
        dict(name="rows_train_window", kind="rows", seqs=9, tokens=20001, before=0, heads=16, kv=2, dim=80, window=1000, sinks=3,
             train=True),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST = {}


def _most(kind):
    """bytes and operations of the largest listed case of a kind"""
    if kind not in _MOST:
        all_ = [work(c) for c in listed() if c["kind"] == kind]
        _MOST[kind] = max(w["bytes"] for w in all_), max(w["flops"] for w in all_)
    return _MOST[kind]


def draw(rng):
    kind = rng.choice(["plan", "store", "pages", "pages", "pages", "rows", "rows", "rows", "rows"])
    while True:
        c = dict(kind=kind)
        if kind == "plan":
            c.update(seqs=_spread(rng, 1, 4096), longest=_spread(rng, 1, 20000), new=rng.choice([1, 1, _spread(rng, 1, 8000)]),
                     page=rng.choice([16, 32, 64, 128]), short=rng.random() < 0.3)
        else:
            c["kv"] = rng.choice([1, 2, 3, 4, 8, 8, 16])
            c["dim"] = rng.choice([64, 64, 128, 128, 128, 8 * rng.randint(1, 16)])
            if kind == "store":
                c.update(tokens=_spread(rng, 1, 16384), page=rng.choice([16, 32, 64, 128]), x=rng.choice(["bf16", "bf16", "fp32"]),
                         cache=rng.choice(["bf16", "int8"]))
            else:
                c["heads"] = c["kv"] * rng.choice([1, 1, 2, 4, 4, 7, 8, 16])
                c["window"] = rng.choice([0, 0, 0, _spread(rng, 1, 8192)])
                c["sinks"] = rng.choice([0, 4, _spread(rng, 1, 200)]) if c["window"] else 0
                if kind == "pages":
                    c.update(seqs=_spread(rng, 1, 512), longest=_spread(rng, 1, 131072), page=rng.choice([16, 16, 32, 64, 128]),
                             cache=rng.choice(["bf16", "bf16", "int8"]))
                else:
                    c.update(seqs=_spread(rng, 1, 40), tokens=_spread(rng, 1, 32768), train=rng.random() < 0.5)
                    c["before"] = rng.choice([0, 0, 0, _spread(rng, 1, 16384)])
        if c.get("heads", 1) > 64 or kind == "pages" and c["seqs"] * c["longest"] * c["kv"] * c["dim"] > 1 << 30:
            continue
        w, (b, f) = work(c), _most(kind)
        if w["bytes"] <= b and w["flops"] <= f:
            return c


# ---- inputs ----------------------------------------------------------------------------------------------
def _shape(c):
    """What is ragged in a case, the same for every seed.  plan: (tokens there, new tokens); pages: (lengths); rows: (rows of
    each sequence, of its earlier ones)"""
    rng = random.Random(repr(sorted((k, v) for k, v in c.items() if k != "name")))
    n = c["seqs"]
    if c["kind"] == "rows":
        if c["tokens"] <= n:
            return [1] * c["tokens"] + [0] * (n - c["tokens"]), [c["before"]] * n
        parts = [rng.uniform(0.2, 1.0) for _ in range(n)]
        each = [int(c["tokens"] * p / sum(parts)) for p in parts]
        each[0] += c["tokens"] - sum(each)
        return each, [rng.randint(0, c["before"]) for _ in range(n)]
    lengths = [c["longest"]] + [rng.randint(0, c["longest"]) if rng.random() < 0.95 else 0 for _ in range(n - 1)]
    if c["kind"] == "pages":
        return lengths
    if c["new"] == 1:
        return lengths, [1] * n
    return [v if rng.random() < 0.5 else 0 for v in lengths], [rng.randint(1, c["new"]) if rng.random() < 0.9 else 0 for _ in lengths]


def _normal(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)


def _ints(v):
    return torch.tensor(v, device=DEV, dtype=torch.int32)


def _up(a, b):
    return -(-a // b)


def _starts(each):
    at = [0]
    for v in each:
        at.append(at[-1] + v)
    return at


def _free_pages(c):
    """(pages that the new tokens need, pages on the free list)"""
    have, new = _shape(c)
    need = sum(_up(h + m, c["page"]) - _up(h, c["page"]) for h, m in zip(have, new))
    return need, max(1, need * 3 // 4 if c["short"] else need + 5)


def _codes(x):
    """8-bit codes and their scales, one for each row of the last dimension"""
    top = x.float().abs().amax(-1, keepdim=True)
    return torch.round(x.float() * (127.0 * (1.0 / top))).to(torch.int8), (top / 127.0)[..., 0].contiguous()


def _cache(c, g, pages, s):
    for name in ("k", "v"):
        x = _normal(g, pages, c["kv"], c["page"], c["dim"])
        if c["cache"] == "int8":
            s[name + "_pages"], s[name + "_scale"] = _codes(x)
        else:
            s[name + "_pages"], s[name + "_scale"] = x.to(TYPES[c["cache"]]), None


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(c=c)
    if c["kind"] == "plan":
        have, new = _shape(c)
        at = torch.randperm(c["seqs"], generator=g, device=DEV).tolist()
        have, new = [have[i] for i in at], [new[i] for i in at]
        P, W = c["page"], _up(c["longest"] + c["new"], c["page"])
        free = _free_pages(c)[1]
        there = [_up(h, P) for h in have]
        ids = torch.randperm(sum(there) + free + 3, generator=g, device=DEV).int()
        starts = _starts(there)
        s["table"] = torch.full((c["seqs"], W), -1, device=DEV, dtype=torch.int32)
        col = torch.arange(W, device=DEV)
        mine = col < _ints(there)[:, None]
        s["table"][mine] = ids[:starts[-1]]
        s["free"], s["used"] = ids[starts[-1]:], _ints([3])
        s["have"], s["more"], s["tokens"] = _ints(have), _ints(new), sum(new) + 7
    elif c["kind"] == "store":
        T, P = c["tokens"], c["page"]
        pages = _up(T, P) + 2
        _cache(c, g, pages, s)
        ids = torch.randperm(pages, generator=g, device=DEV)
        pos = torch.arange(T, device=DEV) + P // 2
        s["slots"] = (ids[pos // P] * P + pos % P).int()
        s["slots"][torch.rand(T, generator=g, device=DEV) < 0.01] = -1
        # (the keys and values lie side by side in the rows that a projection has made)
        kv = _normal(g, T, 2, c["kv"], c["dim"], dtype=TYPES[c["x"]])
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
    elif c["kind"] == "pages":
        lens = _shape(c)
        lens = [lens[i] for i in torch.randperm(len(lens), generator=g, device=DEV).tolist()]
        P, W = c["page"], _up(c["longest"], c["page"])
        there = [_up(n, P) for n in lens]
        pages = sum(there) + 2
        _cache(c, g, pages, s)
        ids = torch.randperm(pages, generator=g, device=DEV).int()
        s["table"] = torch.full((len(lens), W), -1, device=DEV, dtype=torch.int32)
        s["table"][torch.arange(W, device=DEV) < _ints(there)[:, None]] = ids[:sum(there)]
        s["lengths"] = _ints(lens)
        s["q"] = _normal(g, len(lens), c["heads"], c["dim"], std=2.0, dtype=torch.bfloat16)
    else:
        each, before = _shape(c)
        s["each"], s["keys"] = each, [a + b for a, b in zip(each, before)]
        s["offsets"] = _ints(_starts(each))
        s["k_offsets"] = _ints(_starts(s["keys"])) if c["before"] else None
        T, K, D = sum(s["each"]), sum(s["keys"]), c["dim"]
        s["q"] = _normal(g, T, c["heads"], D, std=2.0, dtype=torch.bfloat16)
        kv = _normal(g, K, 2, c["kv"], D, dtype=torch.bfloat16)
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
        if c["train"]:
            s["dy"] = _normal(g, T, c["heads"], D, dtype=torch.bfloat16)
    return s


# ---- the plain forms, in 32 bits --------------------------------------------------------------------------
def _plain_plan(s):
    P, table, free = s["c"]["page"], s["table"], s["free"].long()
    W, n, T = table.shape[1], table.shape[0], s["tokens"]
    h, m = s["have"].clamp(min=0).long(), s["more"].clamp(min=0).long()
    old, need = ((h + P - 1) // P).clamp(max=W), ((h + m + P - 1) // P).clamp(max=W)
    take = need - old
    first = s["used"].long() + take.cumsum(0) - take
    col = torch.arange(W, device=DEV)[None]
    at = first[:, None] + col - old[:, None]
    page = torch.where(at < free.numel(), free[at.clamp(0, free.numel() - 1)], -1)
    table.copy_(torch.where((col >= old[:, None]) & (col < need[:, None]), page, table.long()))
    ends = m.cumsum(0)
    r = torch.arange(T, device=DEV)
    of = (r[:, None] >= ends[None]).sum(1) if T * n <= ROOM else torch.searchsorted(ends, r, right=True)
    there = of < n
    of = of.clamp(max=n - 1)
    pos = h[of] + r - (ends - m)[of]
    p = table[of, (pos // P).clamp(0, W - 1)].long()
    slot = torch.where(there & (pos // P < W) & (p >= 0), p * P + pos % P, -1)
    return dict(table=table, offsets=torch.cat((ends.new_zeros(1), ends)).int(), slots=slot.int(), positions=torch.where(there, pos, -1).int(),
                lengths=(h + m).int(), used=(s["used"] + take.sum()).int())


def _values(s, name):
    """the cache as the values that it stands for"""
    p, scale = s[name + "_pages"], s[name + "_scale"]
    return p if scale is None else p.float() * scale[..., None]


def _plain_store(s):
    P, cache = s["c"]["page"], s["c"]["cache"]
    there = s["slots"] >= 0
    slot = s["slots"][there].long()
    for name in ("k", "v"):
        x = s[name][there]
        if cache == "int8":
            top = x.float().abs().amax(2, keepdim=True)
            s[name + "_scale"][slot // P, :, slot % P] = top[..., 0] / 127.0
            # (in 64 bits: 16-bit values are often half way between two codes)
            x = torch.round(x.double() * 127.0 / top.double())
        s[name + "_pages"][slot // P, :, slot % P] = x.to(TYPES[cache])
    return dict(k=_values(s, "k"), v=_values(s, "v"))


def _plain_pages(s):
    c = s["c"]
    P, D, kv, W = c["page"], c["dim"], c["kv"], s["table"].shape[1]
    n = s["q"].shape[0]
    # the places that can be seen: the first ones, and the last ones
    seen = W * P if c["window"] == 0 else min(W * P, c["window"] + c["sinks"])
    first = 0 if c["window"] == 0 else min(c["sinks"], seen)
    y = torch.empty_like(s["q"])
    step = max(1, ROOM // (seen * kv * D))
    i = torch.arange(seen, device=DEV)
    for a in range(0, n, step):
        length = s["lengths"][a:a + step].long()[:, None]
        back = i[None] - first + (length - c["window"] if c["window"] else 0 * length)
        pos = torch.where(i < first, i, back)
        ok = (pos < length) & ((i < first) | (pos >= first))
        pos = pos.clamp(0, W * P - 1)
        page = s["table"][a:a + step].long().gather(1, pos // P)
        ok &= page >= 0
        page = page.clamp(min=0)

        def take(name):
            x = s[name + "_pages"][page, :, pos % P].float()
            return x if s[name + "_scale"] is None else x * s[name + "_scale"][page, :, pos % P][..., None]

        q = s["q"][a:a + step].float().view(-1, kv, c["heads"] // kv, D)
        z = torch.matmul(q, take("k").permute(0, 2, 3, 1).contiguous()) * D ** -0.5
        z = torch.where(ok[:, None, None], z, -math.inf)
        e = torch.where(ok[:, None, None], torch.exp(z - z.amax(3, keepdim=True)), 0.0)
        total = e.sum(3, keepdim=True)
        out = torch.matmul(e, take("v").permute(0, 2, 1, 3).contiguous()) / torch.where(total > 0, total, 1.0)
        y[a:a + step] = out.reshape(-1, c["heads"], D).to(torch.bfloat16)
    return dict(y=y)


def _plain_rows(s):
    c = s["c"]
    H, kv, D, window, sinks = c["heads"], c["kv"], c["dim"], c["window"], c["sinks"]
    G = H // kv
    y = torch.zeros_like(s["q"])
    if c["train"]:
        dq, dk, dv = torch.zeros_like(s["q"]), torch.zeros(s["k"].shape, device=DEV), torch.zeros(s["v"].shape, device=DEV)
    tq = tk = 0
    for nq, nk in zip(s["each"], s["keys"]):
        k, v = s["k"][tk:tk + nk].float().permute(1, 0, 2), s["v"][tk:tk + nk].float().permute(1, 0, 2)
        step = max(64, ROOM // (H * max(nk, 1)))
        for a in range(0, nq, step):
            b = min(a + step, nq)
            p = torch.arange(a, b, device=DEV)[:, None] + nk - nq
            lo = max(0, a + nk - nq - window + 1) if window else 0
            j = torch.arange(lo, b + nk - nq, device=DEV)
            j = torch.cat((torch.arange(0, min(sinks, lo), device=DEV), j))
            ok = (j <= p) if window == 0 else (j <= p) & ((j > p - window) | (j < sinks))
            rows = slice(tq + a, tq + b)
            kj, vj = k[:, j], v[:, j]
            q = s["q"][rows].float().view(b - a, kv, G, D).permute(1, 2, 0, 3).reshape(kv, G * (b - a), D)
            mask = ok.repeat(G, 1)
            z = torch.where(mask, torch.matmul(q, kj.transpose(1, 2)) * D ** -0.5, -math.inf)
            e = torch.exp(z - z.amax(2, keepdim=True))
            prob = e / e.sum(2, keepdim=True)

            def back(x):
                return x.view(kv, G, b - a, D).permute(2, 0, 1, 3).reshape(b - a, H, D)

            out = torch.matmul(prob, vj)
            y[rows] = back(out).to(torch.bfloat16)
            if c["train"]:
                dy = s["dy"][rows].float().view(b - a, kv, G, D).permute(1, 2, 0, 3).reshape(kv, G * (b - a), D)
                dz = prob * (torch.matmul(dy, vj.transpose(1, 2)) - (dy * out).sum(2, keepdim=True)) * D ** -0.5
                dq[rows] = back(torch.matmul(dz, kj)).to(torch.bfloat16)
                dk[tk + j] += torch.matmul(dz.transpose(1, 2), q).permute(1, 0, 2)
                dv[tk + j] += torch.matmul(prob.transpose(1, 2), dy).permute(1, 0, 2)
        tq, tk = tq + nq, tk + nk
    return dict(y=y, dq=dq, dk=dk.to(torch.bfloat16), dv=dv.to(torch.bfloat16)) if c["train"] else dict(y=y)


def _plain(s):
    return dict(plan=_plain_plan, store=_plain_store, pages=_plain_pages, rows=_plain_rows)[s["c"]["kind"]](s)


# ---- the framework's calls --------------------------------------------------------------------------------
def _calls(s):
    import paper_2412_00099_amd as moe

    c = s["c"]
    if c["kind"] == "plan":
        p = moe.plan_pages(s["have"], s["more"], s["table"], s["free"], c["page"], s["tokens"], used=s["used"])
        return dict(table=s["table"], offsets=p.offsets, slots=p.slots, positions=p.positions, lengths=p.lengths, used=p.used)
    if c["kind"] == "store":
        moe.store_pages(s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"])
        return dict(k=_values(s, "k"), v=_values(s, "v"))
    if c["kind"] == "pages":
        return dict(y=moe.attend_pages(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["k_scale"], s["v_scale"],
                                       window=c["window"], sinks=c["sinks"]))
    kw = dict(k_offsets=s["k_offsets"], window=c["window"], sinks=c["sinks"])
    if not c["train"]:
        return dict(y=moe.attend_rows(s["q"], s["k"], s["v"], s["offsets"], **kw))
    y, lse = moe.attend_rows(s["q"], s["k"], s["v"], s["offsets"], keep=True, **kw)
    dq, dk, dv = moe.attend_rows_backward(s["q"], s["k"], s["v"], s["offsets"], y, lse, s["dy"], **kw)
    return dict(y=y, dq=dq, dk=dk, dv=dv)


def run(state):
    return _calls(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------
def _pairs(nq, nk, window, sinks):
    """how many keys the queries see, all together"""
    p = range(nk - nq, nk)
    if window == 0:
        return (p[0] + p[-1] + 2) * nq // 2 if nq else 0
    return sum(min(i + 1, window) + max(0, min(sinks, i + 1 - window)) for i in p)


def work(case):
    c = case
    if c["kind"] == "plan":
        have, new = _shape(c)
        taken = min(_free_pages(c))
        return dict(bytes=8 * len(have) + 8 * taken + 8 * sum(new) + 8 * len(have) + 4, flops=10 * len(have) + 4 * sum(new))
    if c["kind"] == "store":
        n = 2 * c["tokens"] * c["kv"]
        moved = n * c["dim"] * (SIZE[c["x"]] + SIZE[c["cache"]]) + 4 * c["tokens"]
        if c["cache"] == "int8":
            # (8-bit codes are handed back as the values that they stand for)
            moved += 4 * n + (_up(c["tokens"], c["page"]) + 2) * c["page"] * c["kv"] * 2 * (5 * c["dim"] + 4)
        return dict(bytes=moved, flops=n * c["dim"] * (3 if c["cache"] == "int8" else 1))
    if c["kind"] == "pages":
        seen = sum(n if c["window"] == 0 else min(n, c["window"]) + max(0, min(c["sinks"], n - c["window"])) for n in _shape(c))
        cache = 2 * seen * c["kv"] * (c["dim"] * SIZE[c["cache"]] + (4 if c["cache"] == "int8" else 0))
        return dict(bytes=cache + 4 * seen // c["page"] + 4 * c["seqs"] * c["heads"] * c["dim"], flops=4 * c["dim"] * c["heads"] * seen)
    each, before = _shape(c)
    keys = [a + b for a, b in zip(each, before)]
    pairs = sum(_pairs(a, b, c["window"], c["sinks"]) for a, b in zip(each, keys))
    rows, kv = 2 * sum(each) * c["heads"] * c["dim"], 2 * sum(keys) * c["kv"] * c["dim"]
    if c["train"]:
        return dict(bytes=4 * rows + 4 * kv, flops=14 * c["dim"] * c["heads"] * pairs)
    return dict(bytes=2 * rows + 2 * kv, flops=4 * c["dim"] * c["heads"] * pairs)


# ---- the same from the definitions in 64 bits -------------------------------------------------------------
def _exact_cache(c, s, name):
    x = s[name + "_pages"].double()
    return x if c["cache"] != "int8" else x * s[name + "_scale"].double()[..., None]


def _exact_attend(q, k, v, window, sinks):
    """q [nq, d], k and v [nk, d]: the queries are the last rows"""
    nq, nk = q.shape[0], k.shape[0]
    p, j = torch.arange(nk - nq, nk, device=DEV), torch.arange(nk, device=DEV)
    ago = p[:, None] - j[None, :]
    hidden = ago < 0
    if window:
        hidden = hidden | ((ago >= window) & (j >= sinks)[None, :])
    z = (q @ k.t()) / math.sqrt(q.shape[1])
    return torch.softmax(z.masked_fill(hidden, -math.inf), 1) @ v


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "plan":
        # by hand, sequence after sequence
        P, table, free = c["page"], s["table"].tolist(), s["free"].tolist()
        used, offsets, slots, positions, lengths = int(s["used"]), [0], [], [], []
        for row, h, m in zip(table, s["have"].tolist(), s["more"].tolist()):
            for page in range(_up(h, P), min(_up(h + m, P), len(row))):
                row[page] = free[used] if used < len(free) else -1
                used += 1
            for pos in range(h, h + m):
                page = row[pos // P] if pos // P < len(row) else -1
                slots.append(page * P + pos % P if page >= 0 else -1)
                positions.append(pos)
            offsets.append(offsets[-1] + m)
            lengths.append(h + m)
        none = [-1] * (s["tokens"] - len(slots))
        return dict(table=_ints(table), offsets=_ints(offsets), slots=_ints(slots + none), positions=_ints(positions + none),
                    lengths=_ints(lengths), used=_ints([used]))
    if c["kind"] == "store":
        out = {}
        place = s["slots"].tolist()
        rows = torch.tensor([i for i, p in enumerate(place) if p >= 0], device=DEV, dtype=torch.long)
        at = torch.tensor([p for p in place if p >= 0], device=DEV, dtype=torch.long)
        for name in ("k", "v"):
            x = s[name].double()[rows]
            if c["cache"] == "int8":
                top = x.abs().amax(2, keepdim=True)
                x = (127.0 * x / top).round() * (top / 127.0)
            # (pages and places ahead of the heads)
            all_ = _exact_cache(c, s, name).transpose(1, 2).reshape(-1, c["kv"], c["dim"])
            all_[at] = x
            out[name] = all_.view(-1, c["page"], c["kv"], c["dim"]).transpose(1, 2)
        return out
    G = c["heads"] // c["kv"]
    if c["kind"] == "pages":
        y = torch.zeros(s["q"].shape, device=DEV, dtype=torch.float64)
        for i, n in enumerate(s["lengths"].tolist()):
            if n == 0:
                continue
            pages = s["table"][i, :_up(n, c["page"])].long()
            part = dict(s, **{x: s[x][pages] for x in ("k_pages", "v_pages", "k_scale", "v_scale") if s[x] is not None})
            k, v = (_exact_cache(c, part, x).transpose(0, 1).reshape(c["kv"], -1, c["dim"])[:, :n] for x in ("k", "v"))
            for h in range(c["heads"]):
                y[i, h] = _exact_attend(s["q"][i, h, None].double(), k[h // G], v[h // G], c["window"], c["sinks"])[0]
        return dict(y=y)
    out = dict(y=torch.zeros(s["q"].shape, device=DEV, dtype=torch.float64))
    if c["train"]:
        out.update(dq=torch.zeros_like(out["y"]), dk=torch.zeros(s["k"].shape, device=DEV, dtype=torch.float64),
                   dv=torch.zeros(s["k"].shape, device=DEV, dtype=torch.float64))
    tq = tk = 0
    for nq, nk in zip(s["each"], s["keys"]):
        rows, keys = slice(tq, tq + nq), slice(tk, tk + nk)
        tq, tk = tq + nq, tk + nk
        if nq == 0:
            continue
        for h in range(c["heads"]):
            leaves = [s["q"][rows, h].double(), s["k"][keys, h // G].double(), s["v"][keys, h // G].double()]
            if not c["train"]:
                out["y"][rows, h] = _exact_attend(*leaves, c["window"], c["sinks"])
                continue
            leaves = [t.requires_grad_() for t in leaves]
            y = _exact_attend(*leaves, c["window"], c["sinks"])
            grads = torch.autograd.grad(y, leaves, s["dy"][rows, h].double())
            out["y"][rows, h] = y.detach()
            out["dq"][rows, h] = grads[0]
            out["dk"][keys, h // G] += grads[1]
            out["dv"][keys, h // G] += grads[2]
    return out
