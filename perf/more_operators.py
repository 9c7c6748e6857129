"""The operators of a paged cache whose speed counts: what a serving program has them do, over the sizes it meets.

Four kinds of pass, each through the public entry points of ``paper_2604_02047_b200.binding`` where ``own`` is true, and in
elementary torch operations in 32 bits where it is not:

``append``   ``append_kv_paged``: norm and rotation of a chunk's queries and keys, its K / V rows into the sequences' pages, the new rows'
             positions and weights.
``chunk``    ``chunk_attn``: attention of a chunk of new tokens, one or thousands, over the pages and over one another.
``weights``  ``kv_weights``: the attention that every cached row got from a chunk's tokens, added to what it got before.
``evict``    ``evict_kv``: a cache back to its budget, a key/value head at a time: the first rows, the latest and the heaviest stay.

Head counts and lengths are those of the repository's workloads and tests (32, 40 and 52 heads, 32 query
heads over 8 key/value heads; up to 16 384 tokens), pages are of 16 to 256 rows, in the order in which a pool hands them out.
"""
import functools
import math
import random

import numpy as np
import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
EPS = 1e-6


def append(S, H, Hkv, B, ctx, page, *, norm=True, rot=D, interleaved=False, counts=False, name=None):
    """``ctx`` = (lo, hi): the sequences' rows in the cache before the call; B new tokens each (``counts``: up to B)."""
    c = dict(op="append", S=S, H=H, Hkv=Hkv, B=B, lo=ctx[0], hi=ctx[1], page=page, norm=norm, rot=rot, interleaved=interleaved, counts=counts)
    return c if name is None else dict(c, name=name)


def chunk(S, H, Hkv, B, ctx, page, *, counts=False, name=None):
    c = dict(op="chunk", S=S, H=H, Hkv=Hkv, B=B, lo=ctx[0], hi=ctx[1], page=page, counts=counts)
    return c if name is None else dict(c, name=name)


def weights(S, H, Hkv, B, ctx, page, *, counts=False, name=None):
    c = dict(op="weights", S=S, H=H, Hkv=Hkv, B=B, lo=ctx[0], hi=ctx[1], page=page, counts=counts)
    return c if name is None else dict(c, name=name)


def evict(S, Hkv, budget, ctx, page, *, sink=4, recent=64, name=None):
    c = dict(op="evict", S=S, H=Hkv, Hkv=Hkv, B=1, budget=budget, lo=ctx[0], hi=ctx[1], page=page, sink=sink, recent=recent, counts=False)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # a token of every sequence of a serving batch: launch and a chain of dependent loads
        append(64, 32, 8, 1, (100, 4000), 16, name="append_batch"),
        # two prompts of multi-head models, half of a head rotated in neighbouring pairs
        append(2, 40, 40, 6001, (0, 100), 64, norm=False, rot=64, interleaved=True, name="append_prompt"),
        # one token of one session: latency
        chunk(1, 32, 8, 1, (511, 511), 16, name="chunk_token"),
        # a token of every sequence of a serving batch, long sessions: the caches' rows once
        chunk(64, 32, 8, 1, (500, 8192), 16, name="chunk_decode64"),
        # chains of drafts of different lengths, multi-head, one sequence gone
        chunk(16, 40, 40, 17, (33, 4000), 32, counts=True, name="chunk_drafts"),
        # a long prompt's third chunk: products
        chunk(1, 32, 8, 4096, (8192, 8192), 64, name="chunk_prompt"),
        # prompts of different lengths at once, most of them without a prefix
        chunk(5, 52, 52, 1500, (0, 700), 128, counts=True, name="chunk_prompts_ragged"),
        # what a decoding step adds to every row's weight
        weights(16, 32, 8, 1, (1000, 8192), 16, name="weights_decode"),
        # what a prompt's chunk adds
        weights(1, 32, 8, 2048, (4096, 4096), 64, name="weights_prompt"),
        # short chunks of multi-head models
        weights(6, 40, 40, 100, (10, 2000), 32, counts=True, name="weights_ragged"),
        # one session's cache back to half of what it has
        evict(1, 8, 2048, (4096, 4096), 16, name="evict_one"),
        # a serving batch's caches, some of them within the budget
        evict(16, 8, 4096, (3500, 9000), 16, recent=512, name="evict_batch"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST = {"bytes": 9e8, "flops": 3e11}       # of a drawn case: below the largest listed ones
ROWS = 1.3e6                               # heads x rows of its caches


def draw(rng):
    op = rng.choice(["append", "chunk", "chunk", "chunk", "weights", "weights", "evict"])
    H, Hkv = rng.choice([(32, 32), (40, 40), (52, 52), (32, 8), (32, 8), (32, 8), (16, 2)])
    S, page = _log(rng, 1, 64), rng.choice([16, 16, 32, 64, 128, 256])
    B = rng.choice([1, 1, 17, 60, 128, _log(rng, 2, 300), _log(rng, 100, 8192)])
    counts = S > 1 and rng.random() < 0.4

    def span(hi):
        return (hi, hi) if rng.random() < 0.3 else (int(hi * rng.uniform(0.0, 0.9)), hi)

    if op == "evict":
        budget = _log(rng, 100, 8192)
        sink, recent = rng.choice([0, 1, 4, 16]), int(budget * rng.uniform(0, 0.5))
        c = evict(S, Hkv, budget, span(int(budget * rng.uniform(1.01, 3))), page, sink=sink, recent=recent)
    elif op == "append":
        c = append(S, H, Hkv, B, span(_log(rng, 2, 4000)), page, norm=rng.random() < 0.6, rot=rng.choice([D, D, 64, 32]),
                   interleaved=rng.random() < 0.3, counts=counts)
    else:
        c = (chunk if op == "chunk" else weights)(S, H, Hkv, B, span(_log(rng, 20, 16384)), page, counts=counts)
    while any(work(c)[x] > MOST[x] for x in MOST) or c["S"] * (c["hi"] + c["B"]) * c["Hkv"] > ROWS:
        x = max(("S", "B", "hi") if op != "evict" else ("S", ), key=lambda n: {"S": 100, "B": 2, "hi": 1}[n] * (c[n] if c[n] > 1 else 0))
        c[x] = max(1, c[x] * 3 // 4)
        c["lo"], c["counts"] = min(c["lo"], c["hi"]), c["counts"] and c["S"] > 1
    return c


# ------------------------------------------------------------------------------------------------ shapes of a case
def _shapes(c):
    """Rows before the call and new tokens of the case's sequences (part of the case, not of the seed)."""
    r = random.Random("%s %d %d %d %d" % (c["op"], c["S"], c["B"], c["lo"], c["hi"]))
    lens = [r.randint(c["lo"], c["hi"]) for _ in range(c["S"])]
    new = [0 if c["op"] == "evict" else c["B"]] * c["S"]
    if c["counts"]:
        new = [r.randint((c["B"] + 2) // 3, c["B"]) for _ in range(c["S"])]
        new[r.randrange(c["S"])] = 0
    return lens, new


def work(c):
    lens, new = _shapes(c)
    H, Hkv = c["H"], c["Hkv"]
    n = sum(new)
    if c["op"] == "append":
        return {"bytes": n * (2 * (H + 2 * Hkv) * D * 2 + c["rot"] * 4 + 8 * Hkv),
                "flops": n * (H + Hkv) * (3 * c["rot"] + (4 * D if c["norm"] else 0))}
    if c["op"] == "evict":
        bytes_ = 0
        for x in lens:
            left = min(x, c["budget"])
            moved = 0
            if x > c["budget"]:                               # of rows whose weights do not know where they lie
                late = min(c["recent"], x - c["budget"])
                others = x - c["sink"] - c["recent"]
                moved = late + (x - c["budget"] - late) * (c["budget"] - c["sink"] - c["recent"]) / max(others, 1)
            bytes_ += Hkv * (8 * x + 8 * left + 8 * D * moved)
        return {"bytes": bytes_, "flops": Hkv * sum(lens)}
    rows = sum(x + k for x, k in zip(lens, new) if k)
    pairs = sum(k * x + k * (k + 1) // 2 for x, k in zip(lens, new))
    if c["op"] == "chunk":
        return {"bytes": 4 * D * Hkv * rows + (4 * D + 4) * H * n, "flops": 4 * D * H * pairs}
    return {"bytes": (2 * D + 8) * Hkv * rows + (2 * D + 4) * H * n, "flops": 2 * D * H * pairs}


# ------------------------------------------------------------------------------------------------ inputs
@functools.lru_cache(maxsize=None)
def _context():
    """The process's context: every request of a program goes through the same one."""
    from paper_2604_02047_b200 import binding
    return binding.Goose(max_S=64, max_B=128, max_H=64)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)


def _int32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _table(rot, rows):
    """cos and sin of position x frequency, worked out in 64 bits once."""
    t = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    return torch.cat([torch.cos(t), torch.sin(t)], 1).float().contiguous()


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rs = np.random.default_rng(seed)
    S, B, H, Hkv, page = c["S"], c["B"], c["H"], c["Hkv"], c["page"]
    lens, new = _shapes(c)
    st = dict(case=c, goose=_context() if own else None)
    st["n_new"] = _int32(new) if c["counts"] else None
    st["ctx_len"] = _int32(lens)
    # pages in the order in which a pool that has been in use for a while hands them out; a table's other entries are nobody's
    need = [-(-(x + k) // page) for x, k in zip(lens, new)]
    pages, width = sum(need) + 3, max(1, -(-(max(lens) + B) // page))
    order = rs.permutation(pages)
    table = np.full((S, width), -1, np.int32)
    at = 0
    for s in range(S):
        table[s, :need[s]] = order[at:at + need[s]]
        at += need[s]
    st["page_table"] = _int32(table)
    st["k_cache"] = _normal(g, pages, page, Hkv, D)
    if c["op"] != "weights":
        st["v_cache"] = _normal(g, pages, page, Hkv, D)
    room = width * page
    if c["op"] != "chunk":
        # weights as attention gives them: a few rows have most; every eighth row has had none yet
        w = torch.exp(2 * torch.randn(S, Hkv, room, generator=g, device="cuda")) * 0.01
        st["row_weight"] = w * (torch.rand(S, Hkv, room, generator=g, device="cuda") > 0.125)
    if c["op"] == "append":
        # the projection's output: a token's queries, keys and values next to one another
        qkv = _normal(g, S, B, H + 2 * Hkv, D)
        st["q"], st["k"], st["v"] = qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:]
        st["pos_off"] = _int32(rs.integers(0, 512, S))         # rows that have left the cache
        st["row_pos"] = torch.zeros(S, Hkv, room, dtype=torch.int32, device="cuda")
        st["rope"] = _table(c["rot"], 512 + c["hi"] + B)
        st["norms"] = [(1 + 0.2 * torch.randn(D, generator=g, device="cuda")).bfloat16() if c["norm"] else None for _ in range(2)]
        st["out"] = torch.zeros(S, B, H, D, dtype=torch.bfloat16, device="cuda")
    elif c["op"] == "evict":
        # positions that are left of a longer past, in order; the latest has the position in front of the next token's
        off = rs.integers(0, 2, S) * rs.integers(0, 5000, S)
        gap = torch.rand(S, Hkv, room, generator=g, device="cuda")
        st["pos_off"] = _int32(off)
        ctx, first = st["ctx_len"].long()[:, None, None], st["pos_off"].long()[:, None, None]
        at = torch.arange(room, device="cuda")
        skipped = (torch.cumsum(gap, 2) / gap.sum(2, keepdim=True) * first).long()
        skipped = torch.where(at < c["sink"], 0, torch.where(at >= ctx - c["recent"], first, skipped))
        st["row_pos"] = (at + skipped).int()
        for n in ("new_ctx_len", "new_pos_off"):
            st[n] = torch.zeros(S, dtype=torch.int32, device="cuda")
        st["new_weight"], st["new_pos"] = torch.zeros_like(st["row_weight"]), torch.zeros_like(st["row_pos"])
    else:
        st["q"] = _normal(g, S, B, H, D)
        st["lse"] = torch.zeros(S, B, H, device="cuda")
        if c["op"] == "chunk":
            st["out"] = torch.zeros(S, B, H, D, dtype=torch.bfloat16, device="cuda")
        else:                                                  # the attention has given them
            for s, n in enumerate(new):
                for hk in range(Hkv if n else 0):
                    x = _scores(st, s, hk, n)
                    m = x.amax(-1, keepdim=True)
                    st["lse"][s, :n, hk * (H // Hkv):(hk + 1) * (H // Hkv)] = (torch.log(torch.exp(x - m).sum(-1)) + m[..., 0]).T
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    c, g = st["case"], st["goose"]
    if c["op"] == "append":
        if own:
            g.append_kv_paged(st["q"], st["k"], st["v"], st["k_cache"], st["v_cache"], st["page_table"], st["ctx_len"], rope=st["rope"],
                              n_new=st["n_new"], pos_off=st["pos_off"], q_weight=st["norms"][0], k_weight=st["norms"][1], eps=EPS,
                              interleaved=c["interleaved"], row_weight=st["row_weight"], row_pos=st["row_pos"], out=st["out"])
        else:
            _plain_append(st)
        return [st["out"], st["k_cache"], st["v_cache"], st["row_weight"], st["row_pos"]]
    if c["op"] == "chunk":
        if own:
            g.chunk_attn(st["q"], st["k_cache"], st["v_cache"], st["page_table"], st["ctx_len"], SCALE, out=st["out"], lse=st["lse"],
                         n_new=st["n_new"])
        else:
            _plain_chunk(st)
        return [st["out"], st["lse"]]
    if c["op"] == "weights":
        if own:
            g.kv_weights(st["q"], st["lse"], st["k_cache"], st["page_table"], st["ctx_len"], SCALE, st["row_weight"], n_new=st["n_new"])
        else:
            _plain_weights(st)
        return st["row_weight"]
    if own:
        g.evict_kv(st["k_cache"], st["v_cache"], st["page_table"], st["ctx_len"], st["row_weight"], st["row_pos"], c["budget"], c["sink"],
                   c["recent"], st["pos_off"], new_weight=st["new_weight"], new_pos=st["new_pos"], new_ctx_len=st["new_ctx_len"],
                   new_pos_off=st["new_pos_off"])
    else:
        _plain_evict(st)
    return [st["k_cache"], st["v_cache"], st["new_weight"], st["new_pos"], st["new_ctx_len"], st["new_pos_off"]]


# ------------------------------------------------------------------------------------------------ plain forms
def _rows(st, s, first, last):
    """Rows of the caches, as one long array, that hold sequence s's rows first .. last - 1."""
    at = torch.arange(first, last, device="cuda")
    page = st["case"]["page"]
    return st["page_table"][s].long()[at // page] * page + at % page


def _scores(st, s, hk, n):
    """[H / Hkv, n, rows]: scores of the group's queries, -inf where a row is behind the token."""
    c = st["case"]
    g, ctx = c["H"] // c["Hkv"], _shapes(c)[0][s]
    K = st["k_cache"].flatten(0, 1)[_rows(st, s, 0, ctx + n), hk].float()
    x = SCALE * (st["q"][s, :n, hk * g:(hk + 1) * g].float().transpose(0, 1) @ K.T)
    at = torch.arange(ctx + n, device="cuda")
    return x.masked_fill_(at > ctx + torch.arange(n, device="cuda")[:, None], -math.inf)


def _plain_append(st):
    c = st["case"]
    lens, new = _shapes(c)
    half = c["rot"] // 2
    for s, (ctx, n) in enumerate(zip(lens, new)):
        if not n:
            continue
        pos = st["pos_off"][s] + ctx + torch.arange(n, device="cuda")
        turn = st["rope"][pos.long()][:, None]
        cos, sin = turn[..., :half], turn[..., half:]
        done = []
        for x, w in ((st["q"][s, :n], st["norms"][0]), (st["k"][s, :n], st["norms"][1])):
            x = x.float()
            if w is not None:
                x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
            a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if c["interleaved"] else (x[..., :half], x[..., half:2 * half])
            y = (a * cos - b * sin, b * cos + a * sin)
            y = torch.stack(y, -1).flatten(-2) if c["interleaved"] else torch.cat(y, -1)
            done.append(torch.cat([y, x[..., 2 * half:]], -1).bfloat16())
        rows = _rows(st, s, ctx, ctx + n)
        st["out"][s, :n] = done[0]
        st["k_cache"].flatten(0, 1)[rows] = done[1]
        st["v_cache"].flatten(0, 1)[rows] = st["v"][s, :n]
        st["row_weight"][s, :, ctx:ctx + n] = 0
        st["row_pos"][s, :, ctx:ctx + n] = pos.int()


def _plain_chunk(st):
    c = st["case"]
    lens, new = _shapes(c)
    g = c["H"] // c["Hkv"]
    for s, (ctx, n) in enumerate(zip(lens, new)):
        for hk in range(c["Hkv"] if n else 0):
            x = _scores(st, s, hk, n)
            V = st["v_cache"].flatten(0, 1)[_rows(st, s, 0, ctx + n), hk].float()
            m = x.amax(-1, keepdim=True)
            p = torch.exp(x - m)
            total = p.sum(-1, keepdim=True)
            st["out"][s, :n, hk * g:(hk + 1) * g] = (p @ V / total).bfloat16().transpose(0, 1)
            st["lse"][s, :n, hk * g:(hk + 1) * g] = (torch.log(total) + m)[..., 0].T


def _plain_weights(st):
    c = st["case"]
    lens, new = _shapes(c)
    g = c["H"] // c["Hkv"]
    for s, (ctx, n) in enumerate(zip(lens, new)):
        for hk in range(c["Hkv"] if n else 0):
            p = torch.exp(_scores(st, s, hk, n) - st["lse"][s, :n, hk * g:(hk + 1) * g].T[..., None])
            st["row_weight"][s, hk, :ctx + n] += p.sum((0, 1))


def _plain_evict(st):
    c = st["case"]
    budget = c["budget"]
    for s, ctx in enumerate(_shapes(c)[0]):
        left = min(ctx, budget)
        weight, pos = st["row_weight"][s, :, :ctx], st["row_pos"][s, :, :ctx]
        st["new_ctx_len"][s:s + 1] = left
        st["new_pos_off"][s:s + 1] = st["pos_off"][s:s + 1] + (ctx - left)
        if ctx <= budget:
            st["new_weight"][s, :, :ctx], st["new_pos"][s, :, :ctx] = weight, pos
            continue
        stays = (pos < c["sink"]) | (pos >= st["pos_off"][s] + ctx - c["recent"])
        rank = torch.sort(torch.where(stays, math.inf, weight), dim=1, descending=True, stable=True)[1]
        keep = torch.zeros_like(stays).scatter_(1, rank[:, :budget], True)
        rows = _rows(st, s, 0, ctx)
        for hk in range(c["Hkv"]):
            to, of = torch.nonzero(~keep[hk, :budget])[:, 0], budget + torch.nonzero(keep[hk, budget:])[:, 0]
            for cache in (st["k_cache"], st["v_cache"]):
                flat = cache.flatten(0, 1)
                flat[rows[to], hk] = flat[rows[of], hk]
            for old, fresh in ((weight, st["new_weight"]), (pos, st["new_pos"])):
                fresh[s, hk, :budget] = old[hk, :budget]
                fresh[s, hk, to] = old[hk, of]


# ------------------------------------------------------------------------------------------------ the same in 64 bits
def exact(c, seed):
    if c["op"] == "evict":                                     # (rows change places, nothing is computed)
        return None
    st = prepare(c, seed)
    lens, new = _shapes(c)
    H, Hkv, B, page = c["H"], c["Hkv"], c["B"], c["page"]
    table = st["page_table"].cpu().numpy().astype(np.int64)

    def place(s, j):                                           # (page, row in it) of rows j
        return torch.from_numpy(table[s, j // page]).cuda(), torch.from_numpy(j % page).cuda()

    if c["op"] == "append":
        out = [st[n].double() for n in ("out", "k_cache", "v_cache", "row_weight")] + [None]
        half = c["rot"] // 2
        i = torch.arange(half, device="cuda")
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
        for s, n in enumerate(new):
            if not n:
                continue
            angle = st["rope"].double()[int(st["pos_off"][s]) + lens[s]:][:n]
            z = torch.complex(angle[:, :half], angle[:, half:])[:, None]       # a pair as a complex number, turned by a product
            at = place(s, lens[s] + np.arange(n))
            results = []
            for x, w in ((st["q"], st["norms"][0]), (st["k"], st["norms"][1])):
                x = x[s, :n].double()
                if w is not None:
                    x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * w.double()
                y = torch.complex(x[..., a], x[..., b]) * z
                x = x.clone()
                x[..., a], x[..., b] = y.real, y.imag
                results.append(x)
            out[0][s, :n], out[1][at], out[2][at] = results[0], results[1], st["v"][s, :n].double()
            out[3][s, :, lens[s]:lens[s] + n] = 0
        return out
    first = [st["out"].double(), st["lse"].double()] if c["op"] == "chunk" else st["row_weight"].double()
    for s, n in enumerate(new):
        if not n:
            continue
        pages, slots = place(s, np.arange(lens[s] + n))
        for h in range(H):
            keys = st["k_cache"][pages, slots, h * Hkv // H].double()
            for i0 in range(0, n, 2048):
                i1 = min(n, i0 + 2048)
                x = torch.einsum("id,jd->ij", st["q"][s, i0:i1, h].double(), keys[:lens[s] + i1]) * SCALE
                x += torch.triu(torch.full_like(x, -math.inf), lens[s] + i0 + 1)
                if c["op"] == "chunk":
                    values = st["v_cache"][pages[:lens[s] + i1], slots[:lens[s] + i1], h * Hkv // H].double()
                    first[0][s, i0:i1, h] = torch.softmax(x, -1) @ values
                    first[1][s, i0:i1, h] = torch.logsumexp(x, -1)
                else:
                    first[s, h * Hkv // H, :lens[s] + i1] += torch.exp(x - st["lse"][s, i0:i1, h, None].double()).sum(0)
    return first
