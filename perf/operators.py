"""The operators around the verification step whose speed counts: what a serving program has them do, over the sizes it meets.

Four kinds of pass, each through the public entry points of ``paper_2604_02047_b200.binding`` where ``own`` is true, and in
elementary torch operations in 32 bits where it is not:

``append``   ``append_kv``: norm and rotation of the new tokens' queries and keys, their K / V rows into the cache.
``attn``     ``tree_attn_shared``: tree attention of a batch over a prefix that all its sequences share and over their own rows.
``adjust``   ``adjust_logits``: penalties over a sequence's tokens and a node's path, bias, grammar mask.
``commit``   ``append_tokens``: the accepted path's tokens behind a sequence's history.

Head counts, tree sizes, vocabularies and prefix lengths are those of the repository's workloads and tests (32, 40 and 52
heads, 32 query heads over 8 key/value heads; trees of 1 to 128 nodes; 32 000 and 128 256 vocabulary entries; up to 16 384
tokens), with odd sizes between them.
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


def append(S, H, Hkv, B, ctx, *, tree=True, norm=True, rot=D, interleaved=False, counts=False, name=None):
    """``ctx`` = (lo, hi): the sequences' rows in the cache before the call.  ``tree``: B nodes of a tree, else B tokens of a prompt."""
    c = dict(op="append", S=S, H=H, Hkv=Hkv, B=B, lo=ctx[0], hi=ctx[1], tree=tree, norm=norm, rot=rot, interleaved=interleaved, counts=counts)
    return c if name is None else dict(c, name=name)


def attn(S, H, Hkv, B, shared, ctx, *, counts=False, name=None):
    c = dict(op="attn", S=S, H=H, Hkv=Hkv, B=B, shared=shared, lo=ctx[0], hi=ctx[1], counts=counts)
    return c if name is None else dict(c, name=name)


def adjust(S, B, V, hist, *, mask=True, bias=True, counts=False, name=None):
    """``hist`` = (lo, hi): tokens of the sequences so far."""
    c = dict(op="adjust", S=S, B=B, V=V, lo=hist[0], hi=hist[1], mask=mask, bias=bias, counts=counts)
    return c if name is None else dict(c, name=name)


def commit(S, B, hist, *, counts=False, name=None):
    c = dict(op="commit", S=S, B=B, lo=hist[0], hi=hist[1], counts=counts)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one token of one session: a launch and a chain of dependent loads
        append(1, 32, 8, 1, (511, 511), name="append_token"),
        # the trees of a serving batch, of different sizes, one sequence gone
        append(16, 32, 8, 64, (100, 1000), counts=True, name="append_tree16"),
        # two prompts of multi-head models whose first half of a head is rotated, in neighbouring pairs
        append(2, 40, 40, 6001, (0, 7), tree=False, norm=False, rot=64, interleaved=True, name="append_prompt"),
        # four short chats under a short system prompt, a token each: latency
        attn(4, 32, 8, 1, 512, (1, 130), name="shared_chat"),
        # a large decoding batch under a long document: the sequences' own rows and the document's once
        attn(64, 32, 8, 1, 16384, (100, 3000), name="shared_decode64"),
        # trees of a serving batch under a long prompt: products
        attn(16, 32, 8, 64, 8192, (200, 2000), name="shared_tree16"),
        # multi-head, a prompt that ends inside a tile, trees of different sizes, one sequence gone
        attn(8, 32, 32, 60, 4001, (33, 1500), counts=True, name="shared_mha_ragged"),
        # a draft's first steps
        adjust(1, 16, 32000, (512, 512), mask=False, bias=False, name="adjust_small"),
        # a serving batch under a grammar and a bias
        adjust(16, 64, 32000, (1024, 16384), counts=True, name="adjust_tree16"),
        # a large vocabulary, a small batch
        adjust(4, 32, 128256, (4096, 16384), bias=False, name="adjust_128k"),
        # what was accepted of one tree, and of a batch
        commit(1, 16, (512, 512), name="commit_one"),
        commit(64, 128, (1024, 16384), counts=True, name="commit_batch"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST = {"bytes": 7e8, "flops": 1.5e11}     # of a drawn case: below the largest listed ones


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "adjust", "adjust", "commit"])
    S, B = _log(rng, 1, 64), rng.choice([1, 1, 16, 32, 60, 64, 80, 128, rng.randint(2, 128), rng.randint(2, 128)])
    H, Hkv = rng.choice([(32, 32), (40, 40), (52, 52), (32, 8), (32, 8), (32, 8), (16, 2)])
    counts = S > 1 and rng.random() < 0.4

    def span(hi):
        return (hi, hi) if rng.random() < 0.3 else (int(hi * rng.uniform(0.05, 0.9)), hi)

    if op == "commit":
        return commit(S, B, span(_log(rng, 30, 16384)), counts=counts)
    if op == "adjust":
        V = rng.choice([32000, 32000, 128256, 128256, rng.randint(2000, 130000)])
        c = adjust(S, B, V, span(_log(rng, 30, 16384)), mask=rng.random() < 0.6, bias=rng.random() < 0.5, counts=counts)
        small = ("S", "B")
    elif op == "append":
        tree = rng.random() < 0.6
        c = append(S, H, Hkv, B if tree else _log(rng, 1, 16384), span(_log(rng, 2, 2000)), tree=tree, norm=rng.random() < 0.6,
                   rot=rng.choice([D, D, 64, 32]), interleaved=rng.random() < 0.3, counts=counts)
        small = ("S", "hi")
    else:
        c = attn(S, H, Hkv, B, _log(rng, 100, 32768), span(_log(rng, 20, 8192)), counts=counts)
        small = ("S", "shared", "hi")
    while any(work(c)[x] > MOST[x] for x in MOST) or (op == "append" and c["S"] * (c["hi"] + c["B"]) * c["Hkv"] > 1.3e6):
        x = max(small, key=lambda n: c[n] if n != "S" else 16 * c[n])
        c[x] = max(1, c[x] * 3 // 4)
        if op == "append" and not c["tree"]:
            c["B"] = max(1, c["B"] * 3 // 4)
        c["lo"], c["counts"] = min(c["lo"], c["hi"]), c["counts"] and c["S"] > 1
    return c


# ------------------------------------------------------------------------------------------------ shapes of a case
def _shapes(c):
    """Lengths and node counts of the case's sequences (part of the case, not of the seed)."""
    r = random.Random("%s %d %d %d %d" % (c["op"], c["S"], c["B"], c["lo"], c["hi"]))
    lens = [r.randint(c["lo"], c["hi"]) for _ in range(c["S"])]
    nodes = [c["B"]] * c["S"]
    if c["counts"]:
        nodes = [r.randint((c["B"] + 2) // 3, c["B"]) for _ in range(c["S"])]
        nodes[r.randrange(c["S"])] = 0
    return lens, nodes


def work(c):
    lens, nodes = _shapes(c)
    n = sum(nodes)
    if c["op"] == "append":
        heads = c["H"] + 2 * c["Hkv"]
        return {"bytes": n * (2 * heads * D * 2 + c["rot"] * 4), "flops": n * (c["H"] + c["Hkv"]) * (3 * c["rot"] + (4 * D if c["norm"] else 0))}
    if c["op"] == "attn":
        own_keys = sum(x + k for x, k in zip(lens, nodes) if k)
        keys = sum(k * (c["shared"] + x + k) for x, k in zip(lens, nodes))
        return {"bytes": 2 * D * 2 * c["Hkv"] * (c["shared"] + own_keys) + 2 * D * 2 * c["H"] * n, "flops": 4 * D * c["H"] * keys}
    if c["op"] == "adjust":
        V = c["V"]
        return {"bytes": n * (4 * V + (V / 8 if c["mask"] else 0)) + 4 * sum(x for x, k in zip(lens, nodes) if k) + (4 * V if c["bias"] else 0),
                "flops": 4 * n * V}
    return {"bytes": 4 * (3 * n + 4 * c["S"]), "flops": n}


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


def _trees(rs, S, B):
    """Trees of a spine, a chain of a quarter of the nodes, and short branches off it; parents come before their children."""
    parent = np.empty((S, B), np.int32)
    for s in range(S):
        spine = int(rs.integers(1, max(2, B // 4) + 1))
        for i in range(B):
            parent[s, i] = i - 1 if i < spine or rs.random() < 0.5 else rs.integers(0, i)
    return parent


def _table(rot, rows):
    """cos and sin of position x frequency, worked out in 64 bits once."""
    t = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    return torch.cat([torch.cos(t), torch.sin(t)], 1).float().contiguous()


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rs = np.random.default_rng(seed)
    S, B = c["S"], c["B"]
    lens, nodes = _shapes(c)
    st = dict(case=c, goose=_context() if own else None)
    st["n_nodes"] = _int32(nodes) if c["counts"] else None
    st["parent"] = None if c["op"] == "append" and not c["tree"] else _int32(_trees(rs, S, B))
    if c["op"] in ("append", "attn"):
        H, Hkv = c["H"], c["Hkv"]
        used = np.array(lens, np.int64) + B
        first = c.get("shared", 0)
        st["row_off"] = torch.from_numpy((first + np.concatenate([[0], np.cumsum(used)[:-1]])).astype(np.int64)).cuda()
        st["ctx_len"] = _int32(lens)
        rows = first + int(used.sum())
        st["k_cache"], st["v_cache"] = _normal(g, rows, Hkv, D), _normal(g, rows, Hkv, D)
        st["out"] = torch.zeros(S, B, H, D, dtype=torch.bfloat16, device="cuda")
    if c["op"] == "append":
        # the projection's output: a token's queries, keys and values next to one another
        qkv = _normal(g, S, B, H + 2 * Hkv, D)
        st["q"], st["k"], st["v"] = qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:]
        st["pos_off"] = _int32(rs.integers(0, 512, S))         # the rows that the sequences share elsewhere in the cache
        st["rope"] = _table(c["rot"], 512 + c["hi"] + B)
        st["weights"] = [(1 + 0.2 * torch.randn(D, generator=g, device="cuda")).bfloat16() if c["norm"] else None for _ in range(2)]
    elif c["op"] == "attn":
        st["q"] = _normal(g, S, B, H, D)
    else:
        V = c.get("V", 32000)
        room = c["hi"] + 2 * B + 4
        # tokens as text has them: few that are frequent, many that are rare
        st["hist"] = _int32(np.minimum(np.exp(rs.random((S, room)) * math.log(V)) - 1, V - 1))
        st["hist_len"] = _int32(lens)
        st["tok"] = _int32(np.minimum(np.exp(rs.random((S, B)) * math.log(V)) - 1, V - 1))
    if c["op"] == "adjust":
        st["n_prompt"] = _int32(np.array(lens) * 3 // 4)
        ldl = (V + 7) // 8 * 8
        st["logits"], st["out"] = 3 * _normal(g, S * B, ldl), torch.zeros(S * B, ldl, dtype=torch.bfloat16, device="cuda")
        f = lambda lo, hi: torch.from_numpy(rs.uniform(lo, hi, S).astype(np.float32)).cuda()  # noqa: E731
        st["penalties"] = dict(repetition=f(1.0, 1.5), frequency=f(0.0, 0.5), presence=f(0.0, 0.5))
        st["bias"] = torch.randn(V, generator=g, device="cuda") * (torch.rand(V, generator=g, device="cuda") < 0.01) if c["bias"] else None
        st["mask"] = torch.randint(-2 ** 31, 2 ** 31, (S * B, (V + 31) // 32), generator=g, device="cuda", dtype=torch.int32) if c["mask"] else None
    elif c["op"] == "commit":
        accept = [int(rs.integers(0, max(n, 1))) for n in nodes]
        path = np.full((S, B), -1, np.int32)
        for s, n in enumerate(nodes):
            if n:
                path[s, :accept[s] + 1] = np.concatenate([[0], 1 + np.sort(rs.choice(n - 1, accept[s], replace=False))]) if accept[s] else 0
        st["path"], st["accept_len"] = _int32(path), _int32(accept)
        st["new_len"] = torch.zeros_like(st["hist_len"])
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    c, g = st["case"], st["goose"]
    if c["op"] == "append":
        if own:
            g.append_kv(st["q"], st["k"], st["v"], st["k_cache"], st["v_cache"], st["row_off"], st["ctx_len"], rope=st["rope"],
                        parent=st["parent"], n_nodes=st["n_nodes"], pos_off=st["pos_off"], q_weight=st["weights"][0],
                        k_weight=st["weights"][1], eps=EPS, interleaved=c["interleaved"], out=st["out"])
        else:
            _plain_append(st)
        return [st["out"], st["k_cache"], st["v_cache"]]
    if c["op"] == "attn":
        if own:
            g.tree_attn_shared(st["q"], st["k_cache"], st["v_cache"], 0, c["shared"], st["row_off"], st["ctx_len"], st["parent"],
                               SCALE, out=st["out"], n_nodes=st["n_nodes"])
        else:
            _plain_attn(st)
        return st["out"]
    if c["op"] == "adjust":
        if own:
            g.adjust_logits(st["logits"], st["hist"], st["hist_len"], st["tok"], st["parent"], V=c["V"], n_nodes=st["n_nodes"],
                            n_prompt=st["n_prompt"], bias=st["bias"], mask=st["mask"], out=st["out"], **st["penalties"])
        else:
            _plain_adjust(st)
        return st["out"]
    if own:
        g.append_tokens(st["tok"], st["path"], st["accept_len"], st["hist"], st["hist_len"], n_nodes=st["n_nodes"], new_len=st["new_len"])
    else:
        _plain_commit(st)
    return [st["hist"], st["new_len"]]


# ------------------------------------------------------------------------------------------------ plain forms
def _sees(parent):
    """[S, B, B]: node j is i or an ancestor of i."""
    S, B = parent.shape
    up = torch.where(parent < 0, torch.arange(B, device=parent.device, dtype=parent.dtype), parent).long()
    sees = torch.eye(B, dtype=torch.bool, device=parent.device).expand(S, B, B).clone()
    for _ in range(max(1, (B - 1).bit_length())):              # twice as far up each time
        sees = sees | torch.gather(sees, 1, up[:, :, None].expand(S, B, B))
        up = torch.gather(up, 1, up)
    return sees


def _live(st):
    S, B = st["case"]["S"], st["case"]["B"]
    at = torch.arange(B, device="cuda").expand(S, B)
    return at < (st["n_nodes"][:, None] if st["n_nodes"] is not None else B)


def _turn(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    if rot == 0:
        return x
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    y = (a * cos - b * sin, b * cos + a * sin)
    y = torch.stack(y, -1).flatten(-2) if interleaved else torch.cat(y, -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_append(st):
    c = st["case"]
    S, B = c["S"], c["B"]
    live = _live(st)
    depth = torch.arange(B, device="cuda").expand(S, B) if st["parent"] is None else _sees(st["parent"]).sum(2) - 1
    at = st["rope"][((st["pos_off"] + st["ctx_len"])[:, None] + depth).long()]
    cos, sin = at[:, :, None, :c["rot"] // 2], at[:, :, None, c["rot"] // 2:]
    new = []
    for x, w in ((st["q"], st["weights"][0]), (st["k"], st["weights"][1])):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
        new.append(_turn(x, cos, sin, c["interleaved"]).bfloat16())
    row = (st["row_off"] + st["ctx_len"])[:, None] + torch.arange(B, device="cuda")
    st["out"].copy_(torch.where(live[:, :, None, None], new[0], st["out"]))
    for cache, rows in ((st["k_cache"], new[1]), (st["v_cache"], st["v"])):
        keep = cache[row.view(-1)].view(rows.shape)
        cache[row.view(-1)] = torch.where(live[:, :, None, None], rows, keep).flatten(0, 1)


def _plain_attn(st):
    c = st["case"]
    lens, nodes = _shapes(c)
    H, Hkv, P = c["H"], c["Hkv"], c["shared"]
    sees = _sees(st["parent"])
    first = P
    K0, V0 = (st[n][:P].float().transpose(0, 1) for n in ("k_cache", "v_cache"))
    for s, (ctx, n) in enumerate(zip(lens, nodes)):
        if n:
            K, V = (torch.cat([z, st[name][first:first + ctx + n].float().transpose(0, 1)], 1) for z, name in ((K0, "k_cache"), (V0, "v_cache")))
            q = st["q"][s, :n].float().view(n, Hkv, H // Hkv, D).permute(1, 2, 0, 3).reshape(Hkv, -1, D)
            x = (SCALE * (q @ K.transpose(1, 2))).view(Hkv, H // Hkv, n, -1)
            x[..., P + ctx:].masked_fill_(~sees[s, :n, :n], -math.inf)
            p = torch.exp(x - x.amax(-1, keepdim=True))
            p = (p / p.sum(-1, keepdim=True)).view(Hkv, -1, p.shape[-1])
            st["out"][s, :n] = (p @ V).view(Hkv, H // Hkv, n, D).permute(2, 0, 1, 3).reshape(n, H, D).bfloat16()
        first += ctx + c["B"]


def _plain_adjust(st):
    c = st["case"]
    S, B, V = c["S"], c["B"], c["V"]
    hist, tok = st["hist"].long(), st["tok"].long()
    at = torch.arange(hist.shape[1], device="cuda")
    inside, made = at < st["hist_len"][:, None], at >= st["n_prompt"][:, None]
    sees, live = _sees(st["parent"]), _live(st)
    for s in range(S):
        seen = torch.zeros(V, device="cuda").scatter_add_(0, hist[s], inside[s].float())
        count = torch.zeros(V, device="cuda").scatter_add_(0, hist[s], (inside[s] & made[s]).float())
        path = torch.zeros(B, V, device="cuda").index_add_(1, tok[s], sees[s].float())
        x = st["logits"][s * B:(s + 1) * B, :V].float()
        rep, freq, pres = (st["penalties"][n][s] for n in ("repetition", "frequency", "presence"))
        x = torch.where(seen + path > 0, torch.where(x > 0, x / rep, x * rep), x)
        x = x - freq * (count + path) - pres * (count + path > 0)
        if st["bias"] is not None:
            x = x + st["bias"]
        if st["mask"] is not None:
            v = torch.arange(V, device="cuda")
            x = torch.where((st["mask"][s * B:(s + 1) * B, v >> 5] >> (v & 31)) & 1 == 1, x, -math.inf)
        out = st["out"][s * B:(s + 1) * B, :V]
        out.copy_(torch.where(live[s, :, None], x.bfloat16(), out))


def _plain_commit(st):
    at = torch.arange(st["path"].shape[1], device="cuda")
    alive = _live(st)[:, :1]
    taken = (at <= st["accept_len"][:, None]) & alive
    to = torch.where(taken, st["hist_len"][:, None] + at, st["hist"].shape[1] - 1).long()
    tok = torch.where(taken, torch.gather(st["tok"], 1, st["path"].clamp(min=0).long()), st["hist"][:, -1:])
    st["hist"].scatter_(1, to, tok)
    st["new_len"].copy_(torch.where(alive[:, 0], st["hist_len"] + 1 + st["accept_len"], st["hist_len"]))


# ------------------------------------------------------------------------------------------------ the same in 64 bits
def _paths(parent, n):
    """The nodes from the root to each of the first n nodes."""
    paths = []
    for i in range(n):
        paths.append((paths[parent[i]] if i else []) + [i])
    return paths


def exact(c, seed):
    st = prepare(c, seed)
    lens, nodes = _shapes(c)
    B = c["B"]
    parents = None if st["parent"] is None else st["parent"].tolist()
    if c["op"] == "commit":
        return None
    if c["op"] == "adjust":
        V = c["V"]
        out = st["out"].double()
        hist, tok = st["hist"].cpu().numpy(), st["tok"].cpu().numpy()
        for s, n in enumerate(nodes):
            if not n:
                continue
            made = int(st["n_prompt"][s])
            seen = torch.from_numpy(np.bincount(hist[s, :lens[s]], minlength=V)).cuda() > 0
            count = torch.from_numpy(np.bincount(hist[s, made:lens[s]], minlength=V)).cuda()
            rep, freq, pres = (float(st["penalties"][x][s]) for x in ("repetition", "frequency", "presence"))
            for i, path in enumerate(_paths(parents[s], n)):
                more = torch.from_numpy(np.bincount(tok[s, path], minlength=V)).cuda()
                k = (count + more).double()
                x = st["logits"][s * B + i, :V].double()
                x = torch.where(seen | (more > 0), torch.where(x > 0, x / rep, x * rep), x) - freq * k - pres * (k > 0)
                x = x if st["bias"] is None else x + st["bias"].double()
                if st["mask"] is not None:
                    bits = np.unpackbits(st["mask"][s * B + i].cpu().numpy().view(np.uint8), bitorder="little")[:V]
                    x[torch.from_numpy(bits == 0).cuda()] = -math.inf
                out[s * B + i, :V] = x
        return out
    H, Hkv = c["H"], c["Hkv"]
    out = st["out"].double()
    starts = st["row_off"].tolist()
    if c["op"] == "append":
        caches = [st["k_cache"].double(), st["v_cache"].double()]
        half = c["rot"] // 2
        for s, n in enumerate(nodes):
            if not n:
                continue
            depth = torch.arange(n) if parents is None else torch.tensor([len(p) - 1 for p in _paths(parents[s], n)])
            angle = st["rope"].double()[(int(st["pos_off"][s]) + lens[s] + depth).cuda()]
            z = torch.complex(angle[:, :half], angle[:, half:])[:, None]       # a pair as a complex number, turned by a product
            rows = slice(starts[s] + lens[s], starts[s] + lens[s] + n)
            for x, w, to in ((st["q"], st["weights"][0], out[s, :n]), (st["k"], st["weights"][1], caches[0][rows])):
                x = x[s, :n].double()
                if w is not None:
                    x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * w.double()
                to.copy_(x)
                i = torch.arange(half, device="cuda")
                a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
                y = torch.complex(x[..., a], x[..., b]) * z
                to[..., a], to[..., b] = y.real, y.imag
            caches[1][rows] = st["v"][s, :n].double()
        return [out, *caches]
    P = c["shared"]
    for s, n in enumerate(nodes):
        if not n:
            continue
        visible = torch.zeros(n, lens[s] + n, dtype=torch.bool)
        visible[:, :lens[s]] = True
        for i, path in enumerate(_paths(parents[s], n)):
            visible[i, [lens[s] + j for j in path]] = True
        visible = torch.cat([torch.ones(n, P, dtype=torch.bool), visible], 1).cuda()
        at = torch.cat([torch.arange(P), starts[s] + torch.arange(lens[s] + n)]).cuda()
        for hk in range(Hkv):
            keys, values = st["k_cache"][at, hk].double(), st["v_cache"][at, hk].double()
            heads = slice(hk * (H // Hkv), (hk + 1) * (H // Hkv))
            x = torch.einsum("nhd,kd->hnk", st["q"][s, :n, heads].double(), keys) * SCALE
            out[s, :n, heads] = torch.einsum("hnk,kd->nhd", torch.softmax(x.masked_fill(~visible, -math.inf), -1), values)
    return out
