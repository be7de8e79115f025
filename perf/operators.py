"""The cached-attention operators on real work: appending to a paged key/value cache, attention of new tokens (single
tokens, trees of drafted tokens, chunks) over it, planning an eviction by accumulated attention weight, and moving the
rows that an eviction or an accepted branch asks for.

A cache holds, per layer, pages of ``page`` tokens: k, v bf16 [layers, pages, kv heads, page, head_dim], the attention
weight that every slot has received (fp32) and its position (int32), both [layers, pages, kv heads, page].  Slot t of
sequence s is row t % page of page page_table[s, t // page]; ``used`` slots are taken, ``seen`` tokens have passed.
"""
import math
import random

import torch

own = False

THETA = 500000.0
PAST, PAD = -1, -2


# ---- the cases -------------------------------------------------------------------------------------------------
def _append(name, n_seq, lo, hi, seen, nh=20, nkv=5, hd=128, page=64, tree=False):
    return {"name": name, "op": "append", "n_seq": n_seq, "new_lo": lo, "new_hi": hi, "past_lo": seen // 2, "past_hi": seen // 2,
            "seen": seen, "nh": nh, "nkv": nkv, "hd": hd, "page": page, "tree": tree}


def _attend(name, n_seq, lo, hi, past_lo, past_hi, nh=20, nkv=5, hd=128, page=64, tree=False):
    return {"name": name, "op": "attend", "n_seq": n_seq, "new_lo": lo, "new_hi": hi, "past_lo": past_lo, "past_hi": past_hi,
            "seen": past_hi, "nh": nh, "nkv": nkv, "hd": hd, "page": page, "tree": tree}


def _plan(name, layers, n_seq, past_lo, past_hi, budget, recent, nkv=5, page=64):
    return {"name": name, "op": "plan", "layers": layers, "n_seq": n_seq, "past_lo": past_lo, "past_hi": past_hi, "budget": budget,
            "recent": recent, "sink": 4, "nkv": nkv, "page": page}


def _move(name, layers, n_seq, past, moves, shared, nkv=5, hd=128, page=64):
    return {"name": name, "op": "move", "layers": layers, "n_seq": n_seq, "past": past, "moves": moves, "shared": shared, "nkv": nkv,
            "hd": hd, "page": page}


def listed():
    """The backbone is the repository's: 30 blocks, 20 query heads on 5 key/value heads of 128, theta 500000."""
    return [
        # one agent, one token: the smallest append of a decode loop
        _append("append 1 token", 1, 1, 1, 2000),
        # 256 environments, one serialized state (15..40 tokens) each, late in their episodes
        _append("append 256 states", 256, 15, 40, 60000),
        # one agent generating one token over a 2000-token history: latency
        _attend("attend 1 token 1x2000", 1, 1, 1, 2000, 2000),
        # one agent generating one token over a very long episode
        _attend("attend 1 token 1x100k", 1, 1, 1, 100001, 100001),
        # 128 agents generating one token each, histories of every length up to 4096
        _attend("attend 1 token 128x4096", 128, 1, 1, 1, 4096),
        # 16 agents scoring a tree of candidate action texts, 24..48 drafted tokens each, over their histories
        _attend("attend tree 16x48", 16, 24, 48, 1000, 8000, tree=True),
        # 64 environments, the next state (15..40 tokens) over the episode so far
        _attend("attend states 64x40", 64, 15, 40, 200, 2000),
        # one long prompt in chunks: the second 4096 tokens
        _attend("attend chunk 4096+4100", 1, 4096, 4096, 4100, 4100),
        # one agent, one block: a state's worth over a budget of 2048
        _plan("plan 1x2083", 1, 1, 2083, 2083, 2048, 256),
        # all 30 blocks of 16 agents, prompts of up to 8192 tokens cut down to 2048
        _plan("plan 30x16x8192", 30, 16, 2000, 8192, 2048, 256),
        # acceptance of one branch (up to 12 tokens) of a drafted tree in all 30 blocks of 16 agents
        _move("move branch 30x16x12", 30, 16, 1500, 12, True),
        # the rows that an eviction moves after long prompts: up to 700 of them for each head
        _move("move evicted 30x8x700", 30, 8, 4096, 700, False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))))))


HEADS = [(20, 5, 128), (4, 2, 128), (4, 2, 64), (8, 8, 64), (12, 4, 128), (16, 1, 64), (7, 1, 128), (9, 3, 64)]


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "plan", "move"])
    nh, nkv, hd = rng.choice(HEADS)
    page = rng.choice([16, 32, 64, 128])
    if op == "append":
        n_seq = _log(rng, 1, 200)
        hi = _log(rng, 1, max(1, 7000 // n_seq))
        tree = hi <= 64 and rng.random() < 0.4
        c = _append("", n_seq, max(1, hi // 3), hi, _log(rng, 1, 200000) if n_seq * hi < 500 else _log(rng, 1, 20000), nh, nkv, hd, page, tree)
    elif op == "attend":
        kind = rng.choice(["one", "tree", "states", "chunk"])
        if kind == "one":
            n_seq = _log(rng, 1, 128)
            past = _log(rng, 1, min(60000, 250000 // n_seq))
            c = _attend("", n_seq, 1, 1, rng.choice([past, past // 3, 0]), past, nh, nkv, hd, page)
        elif kind == "tree":
            n_seq = _log(rng, 1, 16)
            hi = _log(rng, 2, 64)
            past = _log(rng, 1, 8000)
            c = _attend("", n_seq, rng.choice([0, hi // 2]), hi, past // 4, past, nh, nkv, hd, page, True)
        elif kind == "states":
            n_seq = _log(rng, 1, 64)
            hi = rng.randint(2, 60)
            past = _log(rng, 1, 2000)
            c = _attend("", n_seq, rng.choice([0, hi // 3]), hi, rng.choice([0, past // 5, past]), past, nh, nkv, hd, page)
        else:
            n_seq = rng.randint(1, 3)
            hi = _log(rng, 64, 4096 // (n_seq * n_seq))
            past = rng.choice([0, _log(rng, 1, 4000)])
            c = _attend("", n_seq, max(1, hi // 2), hi, past // 2, past, nh, nkv, hd, page)
    elif op == "plan":
        layers = rng.choice([1, 2, 8, 30])
        n_seq = _log(rng, 1, 16)
        budget = _log(rng, 16, 4000)
        past = min(8192, budget + _log(rng, 1, 4000))
        c = _plan("", layers, n_seq, rng.choice([past, past // 3]), past, budget, rng.randint(0, budget // 2), nkv, page)
    else:
        layers = rng.choice([1, 4, 30])
        n_seq = _log(rng, 1, 8)
        past = _log(rng, 32, 4096)
        shared = rng.random() < 0.4
        c = _move("", layers, n_seq, past, min(past // 4, rng.randint(1, 30)) if shared else _log(rng, 1, max(1, past // 6)), shared, nkv, hd, page)
    del c["name"]
    return c


def _lengths(n, lo, hi):
    """n lengths spread over lo..hi, the same for every seed (so that work() knows them)."""
    r = random.Random(1000003 * n + 1009 * lo + hi)
    out = [r.randint(lo, hi) for _ in range(n)]
    out[0] = hi
    return out


def _parents(c, news):
    """A drafted tree for each sequence: tokens hang on the past or on an earlier token; a few places at the end are padding."""
    r = random.Random(77 + c["n_seq"] + c["new_hi"])
    out = []
    for m in news:
        pad = r.randint(0, m // 8)
        par = []
        for i in range(m - pad):
            par.append(PAST if i == 0 or r.random() < 0.08 else i - 1 if r.random() < 0.6 else r.randint(0, i - 1))
        out.append(par + [PAD] * pad)
    return out


def _visible(c):
    """Pairs of new token and key, over all sequences (without padding)."""
    past = _lengths(c["n_seq"], c["past_lo"], c["past_hi"])
    news = _lengths(c["n_seq"], c["new_lo"], c["new_hi"])
    if not c["tree"]:
        return sum(m * p + m * (m + 1) // 2 for m, p in zip(news, past))
    total = 0
    for par, p in zip(_parents(c, news), past):
        depth = []
        for i, q in enumerate(par):
            depth.append(-1 if q == PAD else 0 if q == PAST else depth[q] + 1)
            total += 0 if q == PAD else p + depth[i] + 1
    return total


def work(c):
    if c["op"] == "append":
        T = sum(_lengths(c["n_seq"], c["new_lo"], c["new_hi"]))
        w = (c["nh"] + 2 * c["nkv"]) * c["hd"] * 2
        return {"bytes": T * (2 * w + 8 * c["nkv"]), "flops": T * (c["nh"] + c["nkv"]) * c["hd"] * 3}
    if c["op"] == "attend":
        T = sum(_lengths(c["n_seq"], c["new_lo"], c["new_hi"]))
        keys = T + sum(_lengths(c["n_seq"], c["past_lo"], c["past_hi"]))
        return {"bytes": keys * c["nkv"] * (4 * c["hd"] + 8) + 2 * T * c["nh"] * c["hd"] * 2, "flops": 4 * c["hd"] * c["nh"] * _visible(c)}
    if c["op"] == "plan":
        n = sum(_lengths(c["n_seq"], c["past_lo"], c["past_hi"])) * c["layers"] * c["nkv"]
        moves = sum(min(c["budget"], max(0, p - c["budget"])) for p in _lengths(c["n_seq"], c["past_lo"], c["past_hi"]))
        return {"bytes": n * 8 + moves * c["layers"] * c["nkv"] * 4, "flops": n}
    lists = c["layers"] * c["n_seq"] * c["nkv"]
    n = sum(_lengths(c["n_seq"], 0, c["moves"])) if c["shared"] else sum(_lengths(lists, 0, c["moves"]))
    rows = n * c["layers"] * c["nkv"] if c["shared"] else n
    return {"bytes": rows * 2 * (4 * c["hd"] + 8) + n * 8, "flops": rows}


# ---- the inputs ------------------------------------------------------------------------------------------------
def _cache(g, layers, n_seq, slots, nkv, hd, page, with_rows=True):
    """Pools with a few spare pages, pages dealt to the sequences at random; every used slot holds numbers of the size that
    normed and projected activations have, weights that earlier queries left, and rising positions."""
    max_pages = (slots + page - 1) // page
    n_pages = n_seq * max_pages + 3
    dev = "cuda"
    d = {"page_table": torch.randperm(n_pages, generator=g, device=dev)[: n_seq * max_pages].reshape(n_seq, max_pages).to(torch.int32)}
    if with_rows:
        d["k"] = torch.randn(layers, n_pages, nkv, page, hd, generator=g, device=dev, dtype=torch.bfloat16)
        d["v"] = torch.randn(layers, n_pages, nkv, page, hd, generator=g, device=dev, dtype=torch.bfloat16)
    else:  # a plan reads no rows
        d["k"] = torch.zeros(layers, n_pages, nkv, page, hd, device=dev, dtype=torch.bfloat16)
        d["v"] = torch.zeros(layers, n_pages, nkv, page, hd, device=dev, dtype=torch.bfloat16)
    d["mass"] = torch.empty(layers, n_pages, nkv, page, device=dev).exponential_(generator=g)
    d["pos"] = torch.zeros(layers, n_pages, nkv, page, device=dev, dtype=torch.int32)
    slot = torch.arange(max_pages * page, device=dev, dtype=torch.int32).reshape(1, 1, max_pages, 1, page)
    d["pos"][:, d["page_table"].long()] = slot.expand(layers, n_seq, max_pages, nkv, page)
    return d


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": c}
    if c["op"] in ("append", "attend"):
        past, news = _lengths(c["n_seq"], c["past_lo"], c["past_hi"]), _lengths(c["n_seq"], c["new_lo"], c["new_hi"])
        s |= _cache(g, 1, c["n_seq"], max(p + m for p, m in zip(past, news)), c["nkv"], c["hd"], c["page"])
        T = sum(news)
        s["used"] = _ints(past)
        s["seen"] = _ints([c["seen"] + 3 * i for i in range(c["n_seq"])])
        off = [0]
        for m in news:
            off.append(off[-1] + m)
        s["off"], s["max_new"], s["T"] = _ints(off), max(news), T
        s["parent"] = _ints([p for par in _parents(c, news) for p in par]) if c["tree"] else None
        if c["op"] == "append":
            s["qkv"] = torch.randn(T, (c["nh"] + 2 * c["nkv"]) * c["hd"], generator=g, device="cuda", dtype=torch.bfloat16)
            s["q_out"] = torch.zeros(T, c["nh"] * c["hd"], device="cuda", dtype=torch.bfloat16)
        else:
            s["q"] = 2 * torch.randn(T, c["nh"] * c["hd"], generator=g, device="cuda", dtype=torch.bfloat16)
            s["att"] = torch.zeros(T, c["nh"] * c["hd"], device="cuda", dtype=torch.bfloat16)
    elif c["op"] == "plan":
        past = _lengths(c["n_seq"], c["past_lo"], c["past_hi"])
        s |= _cache(g, c["layers"], c["n_seq"], max(past), c["nkv"], 64, c["page"], with_rows=False)
        s["used"], s["seen"] = _ints(past), _ints(past)
        room = s["page_table"].shape[1] * c["page"]
        s["moves"] = torch.full((c["layers"], c["n_seq"], c["nkv"], max(1, min(c["budget"], room - c["budget"])), 2), -1, dtype=torch.int32, device="cuda")
        s["count"] = torch.zeros(c["layers"], c["n_seq"], c["nkv"], dtype=torch.int32, device="cuda")
    else:
        s |= _cache(g, c["layers"], c["n_seq"], c["past"], c["nkv"], c["hd"], c["page"])
        s["used"] = _ints([c["past"]] * c["n_seq"])
        s["seen"] = _ints([c["past"]] * c["n_seq"])
        lists = (c["n_seq"],) if c["shared"] else (c["layers"], c["n_seq"], c["nkv"])
        n = math.prod(lists)
        if c["shared"]:  # a branch: rising places of the drafted tail go to its beginning
            tail = 4 * c["moves"]
            src = torch.rand(n, tail, generator=g, device="cuda").argsort(1)[:, : c["moves"]].sort(1).values + c["past"] - tail
            dst = torch.arange(c["moves"], device="cuda").expand(n, -1) + c["past"] - tail
        else:  # an eviction: kept slots behind the first third of the cache go to freed ones inside it
            third = c["past"] // 3
            dst = torch.rand(n, third, generator=g, device="cuda").argsort(1)[:, : c["moves"]].sort(1).values
            src = torch.rand(n, c["past"] - third, generator=g, device="cuda").argsort(1)[:, : c["moves"]].sort(1).values + third
        s["moves"] = torch.stack([src, dst], 2).to(torch.int32).reshape(*lists, c["moves"], 2).contiguous()
        s["count"] = _ints(_lengths(n, 0, c["moves"])).reshape(lists)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------
def _grid(s, c):
    """For every place (sequence, i < max_new): does it hold a token, and which row of the batch it is."""
    i = torch.arange(s["max_new"], device="cuda")
    m = (s["off"][1:] - s["off"][:-1]).long()
    live = i[None] < m[:, None]
    return live, torch.where(live, s["off"][:-1].long()[:, None] + i[None], 0)


def _ancestors(s, c):
    """[n_seq, max_new, max_new] truth values: is j the token i itself or one of its ancestors?  Padding has none."""
    live, row = _grid(s, c)
    i = torch.arange(s["max_new"], device="cuda")
    if s["parent"] is None:
        return live[:, :, None] & (i[None, None] <= i[None, :, None])
    par = torch.where(live, s["parent"][row].long(), PAD)
    edge = (par[:, :, None] == i[None, None]).double()  # row i has a one at its parent: strictly lower triangular
    eye = torch.eye(s["max_new"], device="cuda", dtype=torch.float64)
    reach = torch.linalg.solve_triangular(eye - edge, eye.expand_as(edge), upper=False)  # I + E + E^2 + ...
    return (reach > 0.5) & (par != PAD)[:, :, None]


def _slots(s, c, layer_pool):
    """A pool of one layer [pages, kv heads, page, ...] by sequence: [n_seq, kv heads, max_pages * page, ...]."""
    x = layer_pool[s["page_table"].long()]  # [n_seq, max_pages, kv heads, page, ...]
    x = x.transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], x.shape[2] * x.shape[3], *x.shape[4:])


def _plain_append(s, c):
    anc = _ancestors(s, c)
    live, row = _grid(s, c)
    live = live & anc.any(2)
    seq, i = live.nonzero(as_tuple=True)
    t = row[seq, i]
    p = s["seen"][seq].long() + anc.sum(2)[seq, i] - 1
    hd, nh, nkv = c["hd"], c["nh"], c["nkv"]
    f = torch.arange(hd // 2, device="cuda", dtype=torch.float64)
    angle = p.double()[:, None, None] * THETA ** (-2.0 * f / hd)
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    x = s["qkv"][t].float().reshape(-1, nh + 2 * nkv, hd)
    a, b = x[:, : nh + nkv, : hd // 2], x[:, : nh + nkv, hd // 2 :]
    rot = torch.cat([a * cos - b * sin, b * cos + a * sin], 2).to(torch.bfloat16)
    slot = s["used"][seq].long() + i
    page, place = s["page_table"][seq, slot // c["page"]].long(), slot % c["page"]
    s["q_out"][t] = rot[:, :nh].reshape(-1, nh * hd)
    s["k"][0, page, :, place] = rot[:, nh:]
    s["v"][0, page, :, place] = x[:, nh + nkv :].to(torch.bfloat16)
    s["pos"][0, page, :, place] = p.to(torch.int32)[:, None].expand(-1, nkv)
    s["mass"][0, page, :, place] = 0.0
    return s["q_out"], s["k"], s["v"], s["pos"], s["mass"]


def _plain_attend(s, c):
    hd, nh, nkv, rep = c["hd"], c["nh"], c["nkv"], c["nh"] // c["nkv"]
    anc = _ancestors(s, c)
    live, row = _grid(s, c)
    k, v = _slots(s, c, s["k"][0]).float(), _slots(s, c, s["v"][0]).float()
    n_seq, keys = k.shape[0], k.shape[2]
    q = s["q"][row].float().reshape(n_seq, s["max_new"], nkv, rep, hd).permute(0, 2, 3, 1, 4).reshape(n_seq, nkv, rep * s["max_new"], hd)
    at = torch.arange(keys, device="cuda")[None] - s["used"].long()[:, None]  # place among the new tokens; negative: the past
    new = torch.gather(anc, 2, at.clamp(0, s["max_new"] - 1)[:, None].expand(-1, s["max_new"], -1))
    sees = torch.where(at[:, None] < 0, anc.any(2)[:, :, None], new & (at < s["max_new"])[:, None])
    sees = sees[:, None, None].expand(n_seq, 1, rep, s["max_new"], keys).reshape(n_seq, 1, rep * s["max_new"], keys)
    score = (q @ k.transpose(2, 3)) * (1.0 / math.sqrt(hd))
    score = score.masked_fill_(~sees, -math.inf)
    top = score.amax(3, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    w = (score - top).exp_()
    w = w / w.sum(3, keepdim=True).clamp_min(1e-30)
    o = (w @ v).reshape(n_seq, nkv, rep, s["max_new"], hd).permute(0, 3, 1, 2, 4).reshape(n_seq, s["max_new"], nh * hd)
    s["att"][row[live]] = o[live].to(torch.bfloat16)
    got = w.sum(2).reshape(n_seq, nkv, -1, c["page"]).transpose(1, 2)
    pages = s["page_table"].long()
    s["mass"][0, pages] = s["mass"][0, pages] + got
    return s["att"], s["mass"]


def _plain_plan(s, c):
    B, L = c["budget"], c["layers"]
    pages = s["page_table"].long()
    mass = s["mass"][:, pages].transpose(2, 3).flatten(3)  # [L, n_seq, kv heads, slots]
    pos = s["pos"][:, pages].transpose(2, 3).flatten(3)
    n = mass.shape[3]
    slot = torch.arange(n, device="cuda")
    used = s["used"].long()[None, :, None, None]
    safe = (pos >= (s["seen"][None, :, None, None] - c["recent"])) | (pos < c["sink"])
    key = torch.where(mass.isnan(), -math.inf, mass)
    order = key.sort(dim=3, descending=True, stable=True).indices
    rank = safe.int() - 2 * (slot >= used).int()
    order = torch.gather(order, 3, torch.gather(rank, 3, order).sort(dim=3, descending=True, stable=True).indices)
    keep = torch.zeros_like(safe).scatter_(3, order[..., :B], True) & (slot < used)
    full = used > B
    src, dst = keep & (slot >= B) & full, ~keep & (slot < B) & full
    for_src, for_dst = src.nonzero(as_tuple=True), dst.nonzero(as_tuple=True)
    s["moves"][(*for_src[:3], (src.cumsum(3) - 1)[src], 0)] = for_src[3].to(torch.int32)
    s["moves"][(*for_dst[:3], (dst.cumsum(3) - 1)[dst], 1)] = for_dst[3].to(torch.int32)
    s["count"].copy_(src.sum(3))
    return s["moves"], s["count"]


def _plain_move(s, c):
    L, n_seq, nkv, page = c["layers"], c["n_seq"], c["nkv"], c["page"]
    moves, count = s["moves"].long(), s["count"]
    if c["shared"]:
        moves, count = moves[None, :, None].expand(L, n_seq, nkv, *moves.shape[1:]), count[None, :, None].expand(L, n_seq, nkv)
    has = torch.arange(moves.shape[3], device="cuda") < count[..., None]
    layer, seq, head, at = has.nonzero(as_tuple=True)
    src, dst = moves[layer, seq, head, at].unbind(1)
    fr = (layer, s["page_table"][seq, src // page].long(), head, src % page)
    to = (layer, s["page_table"][seq, dst // page].long(), head, dst % page)
    s["k"][to], s["v"][to], s["mass"][to], s["pos"][to] = s["k"][fr], s["v"][fr], s["mass"][fr], s["pos"][fr]
    return s["k"], s["v"], s["mass"], s["pos"]


def _handle(s):
    """What a user's program makes once and keeps: the cache's handle and the attention's workspace."""
    from paper_2604_24273_b200 import bitrl

    c = s["case"]
    s["cache"] = bitrl.KVCache(s["k"], s["v"], s["page_table"], s["used"], s["seen"], mass=s["mass"], pos=s["pos"])
    if c["op"] == "attend":
        n = bitrl.attention_cached_workspace_bytes(s["cache"], s["T"], s["max_new"], c["nh"])
        s["workspace"] = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    s["lib"] = bitrl
    return bitrl


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "plan": _plain_plan, "move": _plain_move}[c["op"]](s, c)
    bitrl = s.get("lib") or _handle(s)
    if c["op"] == "append":
        bitrl.kv_append(s["cache"], 0, s["qkv"], (s["off"], s["max_new"]), c["nh"], parent=s["parent"], theta=THETA, q_out=s["q_out"])
        return s["q_out"], s["k"], s["v"], s["pos"], s["mass"]
    if c["op"] == "attend":
        bitrl.attention_cached(s["cache"], 0, s["q"], (s["off"], s["max_new"]), c["nh"], parent=s["parent"], att=s["att"], workspace=s["workspace"])
        return s["att"], s["mass"]
    if c["op"] == "plan":
        bitrl.kv_evict_plan(s["cache"], c["budget"], c["recent"], sink=c["sink"], moves=s["moves"], count=s["count"])
        return s["moves"], s["count"]
    bitrl.kv_move(s["cache"], s["moves"], s["count"])
    return s["k"], s["v"], s["mass"], s["pos"]


# ---- the definition, in 64 bits ----------------------------------------------------------------------------------
def _chain(parent, i):
    """Places of token i and of those above it, from the top down."""
    out = []
    while i >= 0:
        out.append(i)
        i = parent[i]
    return out[::-1]


def exact(case, seed):
    c = case
    if c["op"] in ("plan",):
        return None
    s = prepare(c, seed)
    hd, nh, nkv, page = c["hd"], c.get("nh"), c["nkv"], c["page"]
    table, used = s["page_table"].tolist(), s["used"].tolist()
    if c["op"] == "move":  # nothing is computed: the rows themselves, in 64 bits
        k, v, mass = s["k"].clone(), s["v"].clone(), s["mass"].double()
        pt = s["page_table"].long()
        for layer in range(c["layers"]):
            for seq in range(c["n_seq"]):
                for head in range(nkv):
                    mv = s["moves"][seq] if c["shared"] else s["moves"][layer, seq, head]
                    n = int(s["count"][seq] if c["shared"] else s["count"][layer, seq, head])
                    a, b = mv[:n, 0].long(), mv[:n, 1].long()
                    k[layer, pt[seq, b // page], head, b % page] = s["k"][layer, pt[seq, a // page], head, a % page]
                    v[layer, pt[seq, b // page], head, b % page] = s["v"][layer, pt[seq, a // page], head, a % page]
                    mass[layer, pt[seq, b // page], head, b % page] = s["mass"][layer, pt[seq, a // page], head, a % page].double()
        return k.float(), v.float(), mass, None
    off = s["off"].tolist()
    parent = s["parent"].tolist() if s["parent"] is not None else None
    if c["op"] == "append":
        T = s["T"]
        place, slot_page, slot_at, rows = [], [], [], []
        for q in range(c["n_seq"]):
            seen = int(s["seen"][q])
            for i in range(off[q + 1] - off[q]):
                if parent is not None and parent[off[q] + i] == PAD:
                    continue
                depth = i if parent is None else len(_chain(parent[off[q] : off[q + 1]], i)) - 1
                rows.append(off[q] + i)
                place.append(seen + depth)
                slot_page.append(table[q][(used[q] + i) // page])
                slot_at.append((used[q] + i) % page)
        rows, place = torch.tensor(rows, device="cuda"), torch.tensor(place, device="cuda", dtype=torch.float64)
        slot_page, slot_at = torch.tensor(slot_page, device="cuda"), torch.tensor(slot_at, device="cuda")
        x = s["qkv"].double().reshape(T, nh + 2 * nkv, hd)[rows]
        z = torch.view_as_complex(torch.stack([x[:, : nh + nkv, : hd // 2], x[:, : nh + nkv, hd // 2 :]], 3))
        rate = torch.exp(-(2.0 * math.log(THETA) / hd) * torch.arange(hd // 2, device="cuda", dtype=torch.float64))
        turn = torch.polar(torch.ones_like(rate)[None].expand(len(rows), -1).contiguous(), place[:, None] * rate)
        r = torch.view_as_real(z * turn[:, None])
        r = torch.cat([r[..., 0], r[..., 1]], 2)
        q_out, k, v, mass = s["q_out"].double(), s["k"][0].double(), s["v"][0].double(), s["mass"].double()
        q_out[rows] = r[:, :nh].reshape(len(rows), nh * hd)
        k[slot_page, :, slot_at] = r[:, nh:]
        v[slot_page, :, slot_at] = x[:, nh + nkv :]
        mass[0, slot_page, :, slot_at] = 0.0
        return q_out, k[None], v[None], None, mass
    att, mass = s["att"].double(), s["mass"].double()
    rep = nh // nkv
    for q in range(c["n_seq"]):
        m, n = off[q + 1] - off[q], used[q] + off[q + 1] - off[q]
        if m == 0:
            continue
        pages = s["page_table"][q, : (n + page - 1) // page].long()
        sees = torch.zeros(m, n, dtype=torch.bool, device="cuda")
        if parent is None:
            sees = torch.ones(m, n, dtype=torch.bool, device="cuda").tril(used[q])
        else:
            rows = [[used[q] + j for j in _chain(parent[off[q] : off[q + 1]], i)] if parent[off[q] + i] != PAD else [] for i in range(m)]
            flat = [(i, j) for i, r in enumerate(rows) for j in r]
            if flat:
                a, b = torch.tensor(flat, device="cuda").unbind(1)
                sees[a, b] = True
            sees[:, : used[q]] = torch.tensor([bool(r) for r in rows], device="cuda")[:, None]
        for h in range(nkv):
            k = s["k"][0][pages][:, h].double().reshape(-1, hd)[:n]
            v = s["v"][0][pages][:, h].double().reshape(-1, hd)[:n]
            got = torch.zeros(n, dtype=torch.float64, device="cuda")
            for j in range(h * rep, h * rep + rep):
                w = s["q"][off[q] : off[q + 1], j * hd : (j + 1) * hd].double() @ k.T / math.sqrt(hd)
                w = torch.softmax(w.masked_fill(~sees, -math.inf), 1)
                w = torch.where(sees, w, 0.0)
                att[off[q] : off[q + 1], j * hd : (j + 1) * hd] = w @ v
                got += w.sum(0)
            slot = torch.arange(n, device="cuda")
            mass[0, pages[slot // page], h, slot % page] += got
    return att, mass
