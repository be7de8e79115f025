"""A plain 64-bit implementation of the operators on a paged key/value cache, and caches to run them on (CPU tensors)."""
import math

import torch

PAST, PAD = -1, -2


def gen(seed):
    return torch.Generator().manual_seed(seed)


def make(seed, used, news, nkv=2, hd=64, page=16, layers=1, room=None, junk=True, scale=1.0):
    """A cache as a dict of CPU tensors: pages dealt at random, used slots filled; the rest holds NaN and infinities."""
    g = gen(seed)
    n_seq = len(used)
    need = max(1, max(u + m for u, m in zip(used, news)))
    max_pages = -(-max(need, room or 0) // page)
    n_pages = n_seq * max_pages + 2
    c = {"used": torch.tensor(used, dtype=torch.int32), "seen": torch.tensor([u + 5 * i for i, u in enumerate(used)], dtype=torch.int32)}
    c["page_table"] = torch.randperm(n_pages, generator=g)[: n_seq * max_pages].reshape(n_seq, max_pages).to(torch.int32)
    shape = (layers, n_pages, nkv, page)
    bad = torch.tensor([math.nan, math.inf, -math.inf])
    for name in ("k", "v"):
        x = bad[torch.randint(3, (*shape, hd), generator=g)].to(torch.bfloat16) if junk else torch.zeros(*shape, hd, dtype=torch.bfloat16)
        c[name] = x
    c["mass"] = torch.zeros(shape)
    c["pos"] = torch.full(shape, -7, dtype=torch.int32)
    for s, u in enumerate(used):
        if u == 0:
            continue
        t = torch.arange(u)
        p = c["page_table"][s, t // page].long()
        for layer in range(layers):
            c["k"][layer, p, :, t % page] = (scale * torch.randn(u, nkv, hd, generator=g)).to(torch.bfloat16)
            c["v"][layer, p, :, t % page] = torch.randn(u, nkv, hd, generator=g).to(torch.bfloat16)
            c["mass"][layer, p, :, t % page] = torch.rand(u, nkv, generator=g)
            c["pos"][layer, p, :, t % page] = t.to(torch.int32)[:, None].expand(-1, nkv)
    return c


def offsets(news):
    return torch.tensor([0] + list(torch.tensor(news).cumsum(0)), dtype=torch.int32)


def tree(seed, m, pads=0):
    g = gen(seed)
    par = []
    for i in range(m - pads):
        r = float(torch.rand(1, generator=g))
        par.append(PAST if i == 0 or r < 0.15 else i - 1 if r < 0.6 else int(torch.randint(i, (1,), generator=g)))
    return par + [PAD] * pads


def above(parent, i):
    """Token i and the tokens above it (empty for padding)."""
    out = []
    if parent[i] == PAD:
        return out
    while i >= 0:
        out.append(i)
        i = parent[i]
    return out


def at(c, s, slots):
    page = c["k"].shape[3]
    slots = torch.as_tensor(slots, dtype=torch.long)
    return c["page_table"][s, slots // page].long(), slots % page


def rotated(x, p, theta):
    """x fp64 [heads, hd] at position p."""
    h = x.shape[1] // 2
    ang = p * theta ** (-2.0 * torch.arange(h, dtype=torch.float64) / x.shape[1])
    a, b = x[:, :h], x[:, h:]
    return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], 1)


def append(c, layer, qkv, off, nh, parent, theta):
    """fp64 {(row) : q [nh, hd]}, {(seq, i): (k, v, pos)} of every token that is not padding."""
    nkv, hd = c["k"].shape[2], c["k"].shape[4]
    q_out, rows = {}, {}
    for s in range(len(off) - 1):
        m = int(off[s + 1] - off[s])
        par = [i - 1 for i in range(m)] if parent is None else parent[int(off[s]) : int(off[s + 1])].tolist()
        for i in range(m):
            chain = above(par, i)
            if not chain:
                continue
            r = int(off[s]) + i
            x = qkv[r].double().reshape(nh + 2 * nkv, hd)
            p = int(c["seen"][s]) + len(chain) - 1
            q_out[r] = rotated(x[:nh], p, theta)
            rows[s, i] = (rotated(x[nh : nh + nkv], p, theta), x[nh + nkv :], p)
    return q_out, rows


def attend(c, layer, q, off, nh, parent):
    """fp64: (att [T, nh, hd], mass added like c["mass"][layer], att's tolerance, mass's tolerance, rows that are real).

    The tolerances count: a score is a sum of hd exact products in fp32 and its scaling, off by at most hd * 2^-23 of the
    sum of magnitudes (any order, truncating adds included), which moves a weight relatively by twice that (the statistics
    too) plus 2^-21 for the exponential and 2^-23 a term for the sum over keys; a weight may be rounded to bf16 (2^-8)
    before it meets the values; att is rounded once to bf16 (2^-8 of the result)."""
    nkv, hd = c["k"].shape[2], c["k"].shape[4]
    rep = nh // nkv
    T = q.shape[0]
    att, tol = torch.zeros(T, nh, hd, dtype=torch.float64), torch.zeros(T, nh, hd, dtype=torch.float64)
    add, mtol = torch.zeros(c["mass"].shape[1:], dtype=torch.float64), torch.zeros(c["mass"].shape[1:], dtype=torch.float64)
    real = torch.zeros(T, dtype=torch.bool)
    for s in range(len(off) - 1):
        t0, m, u = int(off[s]), int(off[s + 1] - off[s]), int(c["used"][s])
        if m == 0:
            continue
        real[t0 : t0 + m] = True
        par = [i - 1 for i in range(m)] if parent is None else parent[t0 : t0 + m].tolist()
        pages, places = at(c, s, range(u + m))
        sees = torch.zeros(m, u + m, dtype=torch.bool)
        for i in range(m):
            chain = above(par, i)
            if chain:
                sees[i, :u] = True
                sees[i, [u + j for j in chain]] = True
        for h in range(nkv):
            k, v = c["k"][layer][pages, h, places].double(), c["v"][layer][pages, h, places].double()
            for j in range(h * rep, (h + 1) * rep):
                x = q[t0 : t0 + m, j * hd : (j + 1) * hd].double()
                for i in range(m):
                    w = sees[i].nonzero()[:, 0]
                    if len(w) == 0:
                        continue
                    sc = k[w] @ x[i] / math.sqrt(hd)
                    d = 2 * hd * 2.0**-23 * float((k[w].abs() @ x[i].abs()).max()) / math.sqrt(hd) + 2.0**-21 + len(w) * 2.0**-23
                    p = torch.softmax(sc, 0)
                    o = p @ v[w]
                    att[t0 + i, j] = o
                    tol[t0 + i, j] = 2.0**-8 * o.abs() + (2.0**-8 + d) * (p @ v[w].abs())
                    add[pages[w], h, places[w]] += p
                    mtol[pages[w], h, places[w]] += p * (d + m * rep * 2.0**-23)
    return att, add, tol, mtol, real


def plan(c, budget, recent, sink):
    """{(layer, seq, head): [(source, destination), ...]}"""
    L, _, nkv, page = c["mass"].shape
    out = {}
    for layer in range(L):
        for s in range(len(c["used"])):
            n, seen = int(c["used"][s]), int(c["seen"][s])
            for h in range(nkv):
                out[layer, s, h] = []
                if n <= budget:
                    continue
                pages, places = at(c, s, range(n))
                w, pos = c["mass"][layer][pages, h, places].tolist(), c["pos"][layer][pages, h, places].tolist()
                rank = lambda t: (0 if pos[t] >= seen - recent or pos[t] < sink else 1,  # noqa: E731
                                  (1, 0.0) if math.isnan(w[t]) else (0, -w[t]), t)
                keep = set(sorted(range(n), key=rank)[:budget])
                out[layer, s, h] = list(zip([t for t in range(budget, n) if t in keep], [t for t in range(budget) if t not in keep]))
    return out


def move(c, lists):
    """c with the rows of {(layer, seq, head): [(source, destination)]} moved, every source read first."""
    new = {k: v.clone() for k, v in c.items()}
    for (layer, s, h), mv in lists.items():
        for a, b in mv:
            pa, ia = at(c, s, [a])
            pb, ib = at(c, s, [b])
            for name in ("k", "v", "mass", "pos"):
                new[name][layer, pb, h, ib] = c[name][layer, pa, h, ia]
    return new
