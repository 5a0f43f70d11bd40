"""Sequences that live in a pool of pages, as cases that can be timed and compared.

A pool holds N pages of P tokens for every KV head; a table names each sequence's pages, several
sequences may hold the same page, and a page is free when nobody holds it.  Kinds of case:

  attn     attention of each listed sequence's newest tokens over its pages; pages that neighbours
           in the list have in common are computed once for all of them (`attn_paged`)
  append   room for new tokens, and the gated recurrence that stores them (`page_pool_reserve`,
           `rat_append_paged`)
  fork     the forks of the last step are dropped, and the kept sequences forked again, with what is
           copied of a layer (`page_pool_free`, `page_pool_fork`, `page_pool_share`, `page_copy`,
           `rat_state_copy`)
  compact  all pages in use move to the front of the pool, with a layer's rows (`page_pool_compact`,
           `page_copy`)

Where `own` is false, all of it is done by elementary torch operations.
"""
import math

import torch

own = False
DEV = "cuda"


def _attn(name, B, Hq, Hkv, D, P, groups, shared, lo, hi, T_new=1, dtype="bf16"):
    """B sequences, in `groups` equal runs that share their first `shared` tokens, with lo .. hi tokens of their own."""
    return {"name": name, "kind": "attn", "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "P": P, "groups": groups, "shared": shared,
            "lo": lo, "hi": hi, "T_new": T_new, "dtype": dtype}


def _append(name, B, Hkv, D, P, lo, hi, T_new, dtype="bf16"):
    return {"name": name, "kind": "append", "B": B, "Hkv": Hkv, "D": D, "P": P, "lo": lo, "hi": hi, "T_new": T_new, "dtype": dtype}


def _fork(name, n, sources, Hkv, D, P, T, dtype="bf16"):
    return {"name": name, "kind": "fork", "n": n, "sources": sources, "Hkv": Hkv, "D": D, "P": P, "T": T, "dtype": dtype}


def _compact(name, S, N, Hkv, D, P, lo, hi, dtype="bf16"):
    return {"name": name, "kind": "compact", "S": S, "N": N, "Hkv": Hkv, "D": D, "P": P, "lo": lo, "hi": hi, "dtype": dtype}


def listed():
    return [
        # the smallest call: two answers to one short prompt, float32 storage
        _attn("attn_f32_600", 2, 4, 2, 64, 16, 1, 512, 30, 90, dtype="f32"),
        # a batch of unrelated requests of very different lengths, nothing in common
        _attn("attn_ragged_b24", 24, 32, 8, 128, 16, 0, 0, 40, 9000),
        # many users of one 32K document
        _attn("attn_prompt_32k_b32", 32, 32, 8, 128, 16, 1, 32768, 30, 1500),
        # 64 answers to one prompt of the paper's length, every query head with keys of its own
        _attn("attn_prompt_4k_b64", 64, 32, 32, 128, 64, 1, 4096, 20, 600),
        # three system prompts in one batch
        _attn("attn_three_prompts_b48", 48, 32, 8, 128, 32, 3, 12000, 100, 2500),
        # questions of up to 384 tokens about one 16K document, all their tokens at once
        _attn("attn_questions_b8", 8, 32, 8, 128, 16, 1, 16384, 384, 400, T_new=384),
        # a decode step's append for a large batch
        _append("append_b64", 64, 8, 128, 16, 100, 8000, 1),
        # the append of the questions
        _append("append_questions_b8", 8, 8, 128, 16, 16384, 16400, 384),
        # four samples from one short conversation
        _fork("fork_4_of_2k", 4, 1, 8, 128, 16, 2001),
        # 64 beams from 8 of 32K tokens, large pages, as many KV heads as query heads
        _fork("fork_64_of_8_32k", 64, 8, 32, 128, 64, 32700),
        # a small pool after some requests ended
        _compact("compact_1k", 12, 1024, 8, 128, 16, 200, 1500),
        # half a million tokens' pages, a bit more than half of them in use
        _compact("compact_32k", 100, 32768, 8, 128, 16, 500, 5500),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "append", "fork", "compact"])
    Hkv = rng.choice([2, 4, 8, 8, 32])
    D, P = rng.choice([64, 128, 128, 128]), rng.choice([16, 16, 32, 64])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "attn":
        G = 1 if Hkv == 32 else rng.choice([1, 2, 4, 4])
        T_new = 1 if rng.random() < 0.7 else _spread(rng, 2, 384)
        groups = rng.choice([0, 1, 1, 1, 2, 3])
        shared = _spread(rng, 100, 32768) // P * P if groups else 0
        each = 8 if T_new > 1 else 64
        B = max(1, groups) * _spread(rng, 1, each // max(1, groups))
        hi = T_new + _spread(rng, 20, 1500 if groups else 9000)
        # (no dearer than the dearest listed one)
        while (B * Hkv * (shared + hi) > 32 * 8 * 34300 or B * Hkv * G * T_new * (shared + hi) > 8 * 32 * 384 * 16784 or
               (max(1, groups) * shared + B * hi) * Hkv * D * (8 if dtype == "f32" else 4) > 1e9):
            B, shared, hi = max(1, groups, B // 2 // max(1, groups) * max(1, groups)), shared * 3 // 4 // P * P, max(T_new, hi * 3 // 4)
        c = _attn("", B, Hkv * G, Hkv, D, P, groups if shared else 0, shared, max(T_new, hi // rng.choice([2, 10, 50])), hi, T_new, dtype)
    elif kind == "append":
        T_new = 1 if rng.random() < 0.5 else _spread(rng, 2, 384)
        lo = _spread(rng, 1, 8000)
        B = _spread(rng, 1, min(64, max(1, 64 * 8 * 128 * 384 // (8 * Hkv * D * T_new))))
        c = _append("", B, Hkv, D, P, lo, lo + _spread(rng, 1, 2000), T_new, dtype)
    elif kind == "fork":
        sources = rng.choice([1, 1, 2, 4, 8])
        n = sources * _spread(rng, 1, 64 // sources)
        c = _fork("", n, sources, Hkv, D, P, _spread(rng, 1, 8 * 32700 // max(8, sources) * 8 // max(8, Hkv)), dtype)
    else:
        N = _spread(rng, 500, 32768 * 16 // P * 8 // max(8, Hkv) // (2 if dtype == "f32" else 1))
        S = _spread(rng, 3, 100)
        hi = max(2 * P, int(N * P * rng.uniform(0.5, 1.2) / S))
        c = _compact("", S, N, Hkv, D, P, max(1, hi // 10), hi, dtype)
    del c["name"]
    return c


# ---- inputs -----------------------------------------------------------------------------


def _dt(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _lengths(n, lo, hi):
    """n whole numbers between lo and hi, the largest among them, in no order."""
    return [lo + (hi - lo) * ((61 * i + 60) % 97 + 1) // 97 if i else hi for i in range(n)]


def _own_tokens(case):
    return _lengths(case["B"], case["lo"], case["hi"])


def _counts(case):
    """New tokens of every sequence."""
    T = case["T_new"]
    return [1] * case["B"] if T == 1 else _lengths(case["B"], max(1, T * 2 // 5), T)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(20260528 + 1000003 * int(seed))
    return g


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _gate(gen, *shape):
    return torch.sigmoid_(_normal(gen, *shape).mul_(0.5).add_(4.2))


def _int(x):
    return torch.tensor(x, device=DEV, dtype=torch.int32)


def _states(gen, Hkv, rows, D, dtype, dirs=None):
    """Rows as the recurrence leaves them (a gate per channel, its last 512 terms), head by head; every 1009th token answers
    to the direction that the queries look for."""
    out = torch.empty(Hkv, rows, D, device=DEV, dtype=dtype)
    for h in range(Hkv):
        x, a = _normal(gen, rows, D), _gate(gen, D)
        if dirs is not None:
            x[500::1009] = 3.0 * dirs[h] + 0.3 * x[500::1009]
        x *= 1 - a
        for k in range(9):
            if (1 << k) >= rows:
                break
            x[1 << k:] += x[:-(1 << k)] * a
            a = a * a
        out[h] = x
    return out


def _pool_tables(gen, lens, shared_pages, groups, M, N, P):
    """Table and reference counts of sequences of these lengths, in equal runs that share their first pages; which physical
    pages they hold is left to chance, as after hours of requests that came and went."""
    B = len(lens)
    pages = torch.tensor([-(-n // P) for n in lens], device=DEV)
    j = torch.arange(M, device=DEV)[None]
    of_own = (pages - shared_pages).clamp(min=0)
    first = groups * shared_pages + of_own.cumsum(0) - of_own
    run = torch.arange(B, device=DEV) * max(1, groups) // B
    number = torch.where(j < shared_pages, run[:, None] * shared_pages + j, first[:, None] + j - shared_pages)
    held = j < pages[:, None]
    perm = torch.randperm(N, generator=gen, device=DEV)
    table = torch.where(held, perm[number.clamp(0, N - 1)], -1).int()
    refs = torch.zeros(N, device=DEV, dtype=torch.int32)
    refs.scatter_add_(0, table[held].long(), torch.ones_like(table[held]))
    return table, _int(lens), refs


def _bounds(pool, N, P):
    """Smallest and largest stored key of each page, [Hkv, N, 2, D]."""
    x = pool.view(pool.shape[0], N, P, pool.shape[-1])
    return torch.stack([x.amin(2), x.amax(2)], 2)


def _inputs(case, seed):
    gen, dt, kind = _gen(seed), _dt(case), case["kind"]
    Hkv, D, P = case["Hkv"], case["D"], case["P"]
    s = dict(case)
    if kind == "attn":
        B, Hq, T, shared, groups = (case[n] for n in ("B", "Hq", "T_new", "shared", "groups"))
        lens = [shared + n for n in _own_tokens(case)]
        c = shared // P
        M = -(-(shared + case["hi"]) // P)
        N = max(1, groups) * c + B * (M - c) + 5
        dirs = _normal(gen, Hkv, D)
        dirs *= math.sqrt(D) / dirs.norm(dim=-1, keepdim=True)
        s["k_pool"], s["v_pool"] = _states(gen, Hkv, N * P, D, dt, dirs), _states(gen, Hkv, N * P, D, dt)
        s["table"], s["len"], s["refs"] = _pool_tables(gen, lens, c, groups, M, N, P)
        s["n_new"] = None if T == 1 else _int(_counts(case))
        q = _normal(gen, B, Hq, T, D)
        s["q"] = (dirs.repeat_interleave(Hq // Hkv, 0)[None, :, None] + 0.25 * q).to(dt)
        # who shares with whom: first member of the run, its members, pages in common
        size = B // max(1, groups)
        s["share"] = None if not c else _int([[b // size * size, size, c if size > 1 else 0] for b in range(B)])
        s["out"], s["lse"] = torch.zeros(B, Hq, T, D, device=DEV, dtype=dt), torch.zeros(B, Hq, T, device=DEV)
        S = B
        s["seq"] = torch.arange(B, device=DEV, dtype=torch.int32)
    elif kind == "append":
        B, T, S = case["B"], case["T_new"], case["B"] + 3
        s["steps"] = 256 if T == 1 else 12  # what the pool has room for; the loop then starts over
        lens = _own_tokens(case) + [case["lo"], 0, 1]
        M = -(-(case["hi"] + s["steps"] * T) // P)
        N = S * M
        s["k_pool"], s["v_pool"] = _states(gen, Hkv, N * P, D, dt), _states(gen, Hkv, N * P, D, dt)
        s["meta"] = _bounds(s["k_pool"], N, P)
        s["table"], s["len"], s["refs"] = _pool_tables(gen, lens, 0, 0, M, N, P)
        s["seq"] = torch.randperm(S, generator=gen, device=DEV)[:B].int()
        s["want"] = None if T == 1 else _int(_counts(case))
        s["granted"] = torch.zeros(B, device=DEV, dtype=torch.int32)
        s["k"], s["v"] = (_normal(gen, B, Hkv, T, D).to(dt) for _ in range(2))
        s["g"] = _gate(gen, B, Hkv, T, D)
        s["state_k"], s["state_v"] = (0.1 * _normal(gen, S, Hkv, D) for _ in range(2))
        s["start"] = [s[n].clone() for n in ("table", "len", "refs")]
        s["at"] = 0
    elif kind == "fork":
        n, sources = case["n"], case["sources"]
        S = sources + n
        lens = _lengths(sources, max(1, case["T"] * 7 // 8), case["T"]) + [0] * n
        M = -(-case["T"] // P) + 4
        N = sources * M + n + 3
        s["k_pool"], s["v_pool"] = _states(gen, Hkv, N * P, D, dt), _states(gen, Hkv, N * P, D, dt)
        s["meta"] = _bounds(s["k_pool"], N, P)
        s["table"], s["len"], s["refs"] = _pool_tables(gen, lens, 0, 0, M, N, P)
        s["state_k"], s["state_v"] = (0.1 * _normal(gen, S, Hkv, D) for _ in range(2))
        # beams: every source goes on as n / sources sequences, side by side in the list; which row each gets is left to chance
        s["src"] = torch.arange(sources, device=DEV, dtype=torch.int32).repeat_interleave(n // sources)
        s["dst"] = (sources + torch.randperm(n, generator=gen, device=DEV)).int()
        s["pairs"], s["carry"] = (torch.full((n, 2), -1, device=DEV, dtype=torch.int32) for _ in range(2))
        s["share"] = torch.zeros(n, 3, device=DEV, dtype=torch.int32)
        s.update(N=N, M=M)
        _fork_plain(s)  # the forks of the step before
    else:
        S, N = case["S"], case["N"]
        lens = _lengths(S, case["lo"], case["hi"])
        while sum(-(-x // P) for x in lens) > N:
            lens = [x * 3 // 4 for x in lens]
        M = -(-case["hi"] // P)
        s["k_pool"], s["v_pool"] = _states(gen, Hkv, N * P, D, dt), _states(gen, Hkv, N * P, D, dt)
        s["meta"] = _bounds(s["k_pool"], N, P)
        s["table"], s["len"], s["refs"] = _pool_tables(gen, lens, 0, 0, M, N, P)
        s["pairs"] = torch.full((N // 2, 2), -1, device=DEV, dtype=torch.int32)
        s["n_pairs"] = torch.zeros(1, device=DEV, dtype=torch.int32)
        s["start"] = [s[n].clone() for n in ("table", "refs")]
    s.update(N=N, S=S, M=M, scale=1.0 / math.sqrt(D))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2605_28640_amd import binding as rs
        s["rs"] = rs
        s["pool"] = pool = rs.make_pool(s["N"], s["S"], s["M"], s["P"])
        B = case.get("B", 1)
        s["shape"] = shape = rs.make_shape(B, case.get("Hq", case["Hkv"]), case["Hkv"], case["D"], s["N"] * s["P"], s["P"], _dt(case))
        s["ws"] = rs.Workspace(rs.attn_paged_workspace_bytes(shape, pool, case["T_new"]) if case["kind"] == "attn" else
                               rs.page_pool_workspace_bytes(pool))
    return s


# ---- one pass, by elementary operations -------------------------------------------------


def _attn_plain(s):
    B, Hq, Hkv, D, P, N, T = (s[n] for n in ("B", "Hq", "Hkv", "D", "P", "N", "T_new"))
    G, rows = Hq // Hkv, s["M"] * P
    pages = s["table"][s["seq"].long()].long().clamp(min=0)
    k, v = (s[n].view(Hkv, N, P, D)[:, pages].float().transpose(0, 1).reshape(B, Hkv, rows, D) for n in ("k_pool", "v_pool"))
    length = s["len"][s["seq"].long()].long()[:, None]
    count = s["n_new"].long()[:, None] if s["n_new"] is not None else torch.full_like(length, T)
    t = torch.arange(T, device=DEV)[None]
    at = (length - count + t)[:, None, None, :, None]  # the position of every new token
    seen = torch.arange(rows, device=DEV) <= at
    p = torch.matmul(s["q"].float().view(B, Hkv, G * T, D), k.transpose(2, 3)).view(B, Hkv, G, T, rows).mul_(s["scale"])
    p.masked_fill_(~seen, -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, G * T, rows), v).view(B, Hkv, G, T, D) / total
    lse = (top + total.log()).view(B, Hq, T)
    fresh = (t < count)[:, None]  # rows behind a sequence's new tokens stay as they were
    out = torch.where(fresh[..., None], o.view(B, Hq, T, D).to(s["out"].dtype), s["out"])
    return [out, torch.where(fresh, lse, s["lse"])]


def _reserve_plain(s):
    P, M = s["P"], s["M"]
    seq = s["seq"].long()
    want = s["want"].long() if s["want"] is not None else torch.full_like(seq, s["T_new"])
    before = s["len"][seq].long()
    held, need = -(-before // P), -(-(before + want) // P)
    j = torch.arange(M, device=DEV)[None]
    fresh = (j >= held[:, None]) & (j < need[:, None])
    free = (s["refs"] == 0).nonzero()[:, 0]
    rows = s["table"][seq]
    taken = free[:int(fresh.sum())]
    rows[fresh] = taken.int()
    s["table"][seq] = rows
    s["refs"][taken] = 1
    s["len"][seq] = (before + want).int()
    s["granted"].copy_(want)


def _append_plain(s):
    B, Hkv, D, P, N, T = (s[n] for n in ("B", "Hkv", "D", "P", "N", "T_new"))
    seq, count = s["seq"].long(), s["granted"].long()
    length = s["len"][seq].long()
    t = torch.arange(T, device=DEV)[None]
    real = t < count[:, None]
    g = torch.where(real[:, None, :, None], s["g"], torch.ones_like(s["g"]))
    at = (length - count)[:, None] + t
    page = s["table"][seq].long().gather(1, (at // P).clamp(max=s["M"] - 1))
    row = (page * P + at % P)[real]
    for x, state, pool in ((s["k"], s["state_k"], s["k_pool"]), (s["v"], s["state_v"], s["v_pool"])):
        a, y = g.clone(), (1 - g) * x.float()
        y[:, :, 0] += a[:, :, 0] * state[seq]
        for k in range((T - 1).bit_length()):  # s_t = g_t s_{t-1} + (1 - g_t) x_t, by doubling
            n = 1 << k
            y[:, :, n:] += a[:, :, n:] * y[:, :, :-n].clone()
            a[:, :, n:] *= a[:, :, :-n].clone()
        state[seq] = y[:, :, -1]
        pool.index_copy_(1, row, y.transpose(1, 2)[real].transpose(0, 1).to(pool.dtype))
    # the bounds of every page with a new row, over its rows so far
    near = torch.arange((T + P - 2) // P + 1, device=DEV)[None] + ((length - count) // P)[:, None]
    touched = (near * P < length[:, None]) & (count > 0)[:, None]
    page = s["table"][seq].long().gather(1, near.clamp(max=s["M"] - 1))[touched]
    rows = s["k_pool"].view(Hkv, N, P, D)[:, page].float()
    stored = ((near * P)[..., None] + torch.arange(P, device=DEV) < length[:, None, None])[touched][None, ..., None]
    s["meta"][:, page, 0] = rows.masked_fill(~stored, math.inf).amin(2).to(s["meta"].dtype)
    s["meta"][:, page, 1] = rows.masked_fill(~stored, -math.inf).amax(2).to(s["meta"].dtype)


def _free_plain(s):
    rows = s["table"][s["dst"].long()]
    s["refs"].scatter_add_(0, rows[rows >= 0].long(), torch.full_like(rows[rows >= 0], -1))
    s["table"][s["dst"].long()] = -1
    s["len"][s["dst"].long()] = 0


def _copy_plain(s, src, dst):
    for n in ("k_pool", "v_pool", "meta"):
        x = s[n].view(s["Hkv"], s["N"], -1)
        x[:, dst] = x[:, src]


def _fork_plain(s):
    P, M = s["P"], s["M"]
    src, dst = s["src"].long(), s["dst"].long()
    length = s["len"][src].long()
    j = torch.arange(M, device=DEV)[None]
    rows = torch.where(j < (length // P)[:, None], s["table"][src], -1)
    s["refs"].scatter_add_(0, rows[rows >= 0].long(), torch.ones_like(rows[rows >= 0]))
    part = length % P > 0
    last = j == (length // P)[:, None]
    old = s["table"][src][last & part[:, None]]
    new = (s["refs"] == 0).nonzero()[:old.numel(), 0]
    rows[last & part[:, None]] = new.int()
    s["refs"][new] = 1
    s["table"][dst] = rows
    s["len"][dst] = length.int()
    s["pairs"].fill_(-1)
    s["pairs"][part] = torch.stack([old, new.int()], 1)
    s["carry"].copy_(torch.stack([src, dst], 1))
    # a layer's part: the partial pages and the carries
    _copy_plain(s, old.long(), new)
    for n in ("state_k", "state_v"):
        s[n][dst] = s[n][src]
    # who shares with whom: runs of the list with at least one full page in common
    full = (j < (length // P)[:, None])
    both = (rows[1:] == rows[:-1]) & full[1:] & full[:-1]
    common = both.int().cumprod(1).sum(1)
    begins = torch.cat([torch.ones(1, device=DEV, dtype=torch.bool), common < 1])
    run = begins.long().cumsum(0) - 1
    size = torch.bincount(run, minlength=run.numel())
    pages = torch.full_like(size, M)
    pages.scatter_reduce_(0, run[1:][~begins[1:]], common[~begins[1:]], "amin")
    first = torch.arange(run.numel(), device=DEV)[begins][run]
    s["share"].copy_(torch.stack([first, size[run], torch.where(size[run] > 1, pages[run], 0)], 1))


def _compact_plain(s):
    N, refs = s["N"], s["refs"]
    live = refs > 0
    L = int(live.sum())
    holes, movers = (~live[:L]).nonzero()[:, 0], live[L:].nonzero()[:, 0] + L
    to = torch.arange(N, device=DEV)
    to[movers] = holes
    s["table"].copy_(torch.where(s["table"] >= 0, to[s["table"].long().clamp(min=0)].int(), -1))
    refs[holes] = refs[movers]
    refs[movers] = 0
    s["pairs"].fill_(-1)
    s["pairs"][:holes.numel()] = torch.stack([movers, holes], 1).int()
    s["n_pairs"].fill_(holes.numel())
    _copy_plain(s, movers, holes)


# ---- one pass ---------------------------------------------------------------------------


def run(s):
    kind = s["kind"]
    if own:
        rs = s["rs"]
    if kind == "attn":
        if not own:
            return _attn_plain(s)
        rs.attn_paged(s["shape"], s["pool"], s["q"], s["k_pool"], s["v_pool"], s["table"], s["len"], s["seq"], s["n_new"], s["T_new"],
                      s["share"], s["scale"], s["out"], s["lse"], s["ws"])
        return [s["out"], s["lse"]]
    if kind == "append":
        if s["at"] == s["steps"]:  # the pool is full: the next requests of these lengths
            s["at"] = 0
            s["table"].copy_(s["start"][0])
            s["len"].copy_(s["start"][1])
            s["refs"].copy_(s["start"][2])
        s["at"] += 1
        if own:
            rs.page_pool_reserve(s["pool"], s["table"], s["len"], s["refs"], s["seq"], s["want"], s["T_new"], s["granted"], s["ws"])
            rs.rat_append_paged(s["shape"], s["pool"], s["k"], s["v"], s["g"], s["state_k"], s["state_v"], s["k_pool"], s["v_pool"],
                                s["meta"], s["table"], s["len"], s["seq"], s["granted"], s["T_new"])
        else:
            _reserve_plain(s)
            _append_plain(s)
        return [s[n] for n in ("state_k", "state_v", "k_pool", "v_pool", "meta", "table", "len", "refs", "granted")]
    if kind == "fork":
        if own:
            rs.page_pool_free(s["pool"], s["table"], s["len"], s["refs"], s["dst"], s["ws"])
            rs.page_pool_fork(s["pool"], s["table"], s["len"], s["refs"], s["src"], s["dst"], s["pairs"], s["carry"], s["ws"])
            rs.page_pool_share(s["pool"], s["table"], s["len"], s["dst"], 1, s["share"])
            rs.page_copy(s["shape"], s["k_pool"], s["v_pool"], s["meta"], s["shape"], s["k_pool"], s["v_pool"], s["meta"], s["pairs"], None)
            rs.rat_state_copy(s["shape"], s["state_k"], s["state_v"], s["carry"])
        else:
            _free_plain(s)
            _fork_plain(s)
        return [s[n] for n in ("k_pool", "v_pool", "meta", "state_k", "state_v", "table", "len", "refs", "pairs", "carry", "share")]
    s["table"].copy_(s["start"][0])  # the pool as the requests that ended leave it
    s["refs"].copy_(s["start"][1])
    if own:
        rs.page_pool_compact(s["pool"], s["table"], s["len"], s["refs"], s["pairs"], s["n_pairs"], s["ws"])
        rs.page_copy(s["shape"], s["k_pool"], s["v_pool"], s["meta"], s["shape"], s["k_pool"], s["v_pool"], s["meta"], s["pairs"],
                     s["n_pairs"])
    else:
        _compact_plain(s)
    return [s[n] for n in ("k_pool", "v_pool", "meta", "table", "refs", "pairs", "n_pairs")]


# ---- what a pass cannot do without ------------------------------------------------------


def work(case):
    kind, e = case["kind"], 4 if case["dtype"] == "f32" else 2
    Hkv, D, P = case["Hkv"], case["D"], case["P"]
    page = 2 * Hkv * (P + 1) * D * e  # a page's keys, values and bounds
    if kind == "attn":  # every page once, the queries and the outputs
        Hq, shared, lens, counts = case["Hq"], case["shared"], _own_tokens(case), _counts(case)
        keys = case["groups"] * shared + sum(lens)
        seen = sum(n * (shared + x - n) + n * (n + 1) // 2 for x, n in zip(lens, counts))
        return {"bytes": 2 * keys * Hkv * D * e + sum(counts) * Hq * (2 * D * e + 4), "flops": 4 * D * Hq * seen}
    if kind == "append":  # keys, values and gates in, rows and page bounds out, carries both ways, the counts of references
        n = sum(_counts(case))
        pages = sum(-(-x // P) for x in _counts(case))
        return {"bytes": Hkv * D * (n * (4 * e + 4) + 16 * case["B"] + 4 * e * pages), "flops": 8 * n * Hkv * D}
    if kind == "fork":  # the tables' rows both ways, counts of references, partial pages and carries both ways
        n, lens = case["n"], _lengths(case["sources"], max(1, case["T"] * 7 // 8), case["T"])
        each = n // case["sources"]
        held = sum(-(-x // P) for x in lens)
        part = sum(1 for x in lens if x % P) * each
        return {"bytes": 2 * part * page + 16 * n * Hkv * D + 4 * held * (3 + each), "flops": 0}
    lens, N = _lengths(case["S"], case["lo"], case["hi"]), case["N"]
    live = min(N, sum(-(-x // P) for x in lens))
    moves = live * (N - live) // N  # pages in use that chance has put behind the others' number
    return {"bytes": 2 * moves * page + 8 * (N + live), "flops": 0}


# ---- the same in 64 bits ----------------------------------------------------------------


def _exact_attn(case, s):
    B, Hq, Hkv, D, P, T = (case[n] for n in ("B", "Hq", "Hkv", "D", "P", "T_new"))
    out, lse = torch.zeros(B, Hq, T, D, device=DEV, dtype=torch.float64), torch.zeros(B, Hq, T, device=DEV, dtype=torch.float64)
    lens, counts, table = s["len"].tolist(), _counts(case), s["table"].tolist()
    for b in range(B):
        L, n = lens[b], counts[b]
        rows = torch.tensor([table[b][i // P] * P + i % P for i in range(L)], device=DEV)
        hidden = torch.arange(L, device=DEV)[None] > torch.arange(L - n, L, device=DEV)[:, None]
        for h in range(Hkv):
            k, v = s["k_pool"][h, rows].double(), s["v_pool"][h, rows].double()
            for q in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                p = (s["q"][b, q, :n].double() @ k.T / math.sqrt(D)).masked_fill_(hidden, -math.inf)
                z = torch.logsumexp(p, 1)
                lse[b, q, :n] = z
                out[b, q, :n] = torch.exp(p - z[:, None]) @ v
    return [out, lse]


def _exact_append(case, s):
    Hkv, D, P, N = case["Hkv"], case["D"], case["P"], s["N"]
    table, lens, free = s["table"].tolist(), s["len"].tolist(), [i for i, n in enumerate(s["refs"].tolist()) if n == 0]
    states = [s[n].double() for n in ("state_k", "state_v")]
    pools = [s[n].double() for n in ("k_pool", "v_pool")]
    meta = s["meta"].double()
    for b, (q, n) in enumerate(zip(s["seq"].tolist(), _counts(case))):
        rows = []
        for i in range(lens[q], lens[q] + n):
            if i % P == 0:
                table[q][i // P] = free.pop(0)
            rows.append(table[q][i // P] * P + i % P)
        where = torch.tensor(rows, device=DEV)
        for x, state, pool in zip((s["k"], s["v"]), states, pools):
            y, every = state[q].clone(), []
            for t in range(n):
                g = s["g"][b, :, t].double()
                y = g * y + (1 - g) * x[b, :, t].double()
                every.append(y)
            state[q] = y
            pool[:, where] = torch.stack(every, 1)
        for i in range(lens[q] // P, (lens[q] + n - 1) // P + 1):
            at = table[q][i] * P
            kept = pools[0][:, at:at + min(P, lens[q] + n - i * P)]
            meta[:, table[q][i], 0], meta[:, table[q][i], 1] = kept.amin(1), kept.amax(1)
    return states + pools + [meta, None, None, None, None]


def _exact_fork(case, s):
    P, M = case["P"], s["M"]
    table, lens, refs = s["table"].tolist(), s["len"].tolist(), s["refs"].tolist()
    src, dst = s["src"].tolist(), s["dst"].tolist()
    for d in dst:
        for i in table[d]:
            if i >= 0:
                refs[i] -= 1
    free = [i for i, n in enumerate(refs) if n == 0]
    k, v, meta, sk, sv = (s[n].double() for n in ("k_pool", "v_pool", "meta", "state_k", "state_v"))
    for a, d in zip(src, dst):
        if lens[a] % P:
            old, new = table[a][lens[a] // P], free.pop(0)
            for x in (k, v):
                x[:, new * P:(new + 1) * P] = x[:, old * P:(old + 1) * P]
            meta[:, new] = meta[:, old]
        sk[d], sv[d] = sk[a], sv[a]
    return [k, v, meta, sk, sv] + [None] * 6


def _exact_compact(case, s):
    P, refs = case["P"], s["refs"].tolist()
    live = sum(n > 0 for n in refs)
    k, v, meta = (s[n].double() for n in ("k_pool", "v_pool", "meta"))
    old = torch.tensor([i for i in range(live, len(refs)) if refs[i] > 0], device=DEV, dtype=torch.long)
    new = torch.tensor([i for i in range(live) if refs[i] == 0], device=DEV, dtype=torch.long)
    within = torch.arange(P, device=DEV)
    for x in (k, v):
        x[:, (new[:, None] * P + within).flatten()] = x[:, (old[:, None] * P + within).flatten()]
    meta[:, new] = meta[:, old]
    return [k, v, meta] + [None] * 4


def exact(case, seed):
    s = _inputs(case, seed)
    return {"attn": _exact_attn, "append": _exact_append, "fork": _exact_fork, "compact": _exact_compact}[case["kind"]](case, s)
