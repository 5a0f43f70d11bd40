"""Caches that live long, as cases that can be timed and compared.

A 4-bit cache holds a row of D channels as D / 2 bytes of codes (two channels a byte, the lower one in the low half) and a scale byte
for each 32 channels: a channel is +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} times 2 ** (byte - 127).  Kinds of case:

  append   new rows go into a 4-bit cache with their pages' bounds, and are read back as the values that they stand for
           (`kv4_append`, `kv4_fetch`)
  attn     one token's attention over a 4-bit cache, whole or listed pages, with or without the tally of how much weight every
           row has had so far (`kv4_attn_decode`)
  tally    the same with the tally over a float32 or bfloat16 cache (`attn_decode_tally`)
  evict    sequences that have outgrown their budget keep the rows that have had most weight (`cache_evict`)
  evict4   the same in a 4-bit cache, whose kept rows are read back (`kv4_evict`, `kv4_fetch`)

Where `own` is false, all of it is done by elementary torch operations.
"""
import math

import torch

own = False
DEV = "cuda"
GROUP = 32  # channels that share a scale


def _append(name, B, Hkv, D, P, lo, hi, T_new, dtype="bf16"):
    """B sequences of lo .. hi tokens, the last T_new (from 2/5 of that on, if more than one) of which are new."""
    return {"name": name, "kind": "append", "B": B, "Hkv": Hkv, "D": D, "P": P, "lo": lo, "hi": hi, "T_new": T_new, "dtype": dtype}


def _attn(name, B, Hq, Hkv, D, lo, hi, tally, pages=0, P=16, shared=False, dtype="bf16"):
    """pages: how many each list holds, of a query head or (shared) of a KV head; 0: no lists."""
    return {"name": name, "kind": "attn", "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "P": P, "lo": lo, "hi": hi, "tally": tally, "pages": pages,
            "shared": shared, "dtype": dtype}


def _tally(name, B, Hq, Hkv, D, lo, hi, dtype="bf16"):
    return {"name": name, "kind": "tally", "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "P": 16, "lo": lo, "hi": hi, "dtype": dtype}


def _evict(name, B, Hkv, D, lo, hi, keep, first, recent, four=False, dtype="bf16"):
    """Sequences of lo .. hi tokens; lo = hi = keep: each decodes one token a pass and gives up one row."""
    return {"name": name, "kind": "evict4" if four else "evict", "B": B, "Hkv": Hkv, "D": D, "P": 16, "lo": lo, "hi": hi, "keep": keep,
            "first": first, "recent": recent, "dtype": dtype}


def listed():
    return [
        # a serving step's new tokens, grouped heads
        _append("append_token_b64", 64, 8, 128, 16, 150, 8000, 1),
        # a long prompt of no round size goes into the cache
        _append("append_prompt_32k", 1, 32, 128, 16, 32001, 32001, 32001),
        # the smallest call: two short sequences, float32 queries
        _attn("attn4_f32_600", 2, 4, 2, 64, 37, 600, False, dtype="f32"),
        # a step of two dozen unrelated requests of very different lengths that keep a tally
        _attn("attn4_ragged_b24", 24, 32, 8, 128, 40, 9000, True),
        # the benchmark's layer, all of its 64K tokens
        _attn("attn4_64k_b4", 4, 32, 32, 128, 65536, 65536, False),
        # the same by its lists: 1/16 of the pages
        _attn("attn4_pages_64k_b4", 4, 32, 32, 128, 65536, 65536, False, pages=256),
        # a small model in float32, five requests of 3 to 3001 tokens
        _tally("tally_f32_3k", 5, 8, 4, 64, 3, 3001, dtype="f32"),
        # a batch of requests at a budget of 4096 rows
        _tally("tally_4k_b32", 32, 32, 8, 128, 4097, 4097),
        # the step after that: each gives up one row
        _evict("evict_token_b32", 32, 8, 128, 4096, 4096, 4096, 4, 64),
        # long conversations go down to a budget of 16384 rows
        _evict("evict_half_32k", 2, 8, 128, 30000, 32768, 16384, 4, 256),
        # the same for many shorter ones, in 4 bits, some of them within their budget
        _evict("evict4_half_8k", 8, 8, 128, 1000, 8191, 4096, 4, 64, four=True),
        # a prompt of 16K tokens is brought down to 1/8
        _evict("evict4_prompt_16k", 4, 8, 128, 16384, 16384, 2048, 16, 128, four=True),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attn", "attn", "attn", "tally", "tally", "evict", "evict4"])
    Hkv, D = rng.choice([2, 4, 8, 8, 32]), rng.choice([64, 128, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    e = 4 if dtype == "f32" else 2
    if kind == "append":
        T = 1 if rng.random() < 0.5 else _spread(rng, 2, 32001)
        B = _spread(rng, 1, max(1, min(64, 32 * 128 * 32001 * 2 // (Hkv * D * e * T))))
        hi = T + (_spread(rng, 1, 8000) if T < 8000 else 0)
        hi = max(T, min(hi, 4 * 32 * 65536 * 128 // (B * Hkv * D)))
        c = _append("", B, Hkv, D, rng.choice([16, 16, 32, 64]), max(T, hi // rng.choice([2, 10, 50])), hi, T, dtype)
    elif kind in ("attn", "tally"):
        G = 1 if Hkv == 32 else rng.choice([1, 2, 4, 4, 7])
        hi = _spread(rng, 1, 65536)
        row = D * 17 / 32 if kind == "attn" else D * e
        room = 4 * 32 * 65536 * 68 if kind == "attn" else 32 * 8 * 4097 * 256
        B = _spread(rng, 1, max(1, min(64, int(room / (Hkv * hi * row)))))
        hi = min(hi, max(1, int(room / (B * Hkv * row))))
        lo = max(1, hi // rng.choice([1, 3, 200]))
        P = rng.choice([16, 16, 32, 64])
        if kind == "tally":
            c = _tally("", B, Hkv * G, Hkv, D, lo, hi, dtype)
        elif rng.random() < 0.3 and -(-lo // P) >= 4:
            pages = max(2, int(-(-lo // P) * rng.choice([1 / 2, 1 / 4, 1 / 16])))
            c = _attn("", B, Hkv * G, Hkv, D, lo, hi, False, pages, P, rng.random() < 0.5, dtype)
        else:
            c = _attn("", B, Hkv * G, Hkv, D, lo, hi, rng.random() < 0.5, dtype=dtype)
    else:
        keep = _spread(rng, 20, 16384)
        most = 2 * 8 * 32768 * 128 * 2 if kind == "evict" else 8 * 8 * 16384 * 128 * 2  # bytes as bfloat16
        hi = keep if kind == "evict" and rng.random() < 0.4 else keep + _spread(rng, 1, min(16384, 7 * keep))
        hi = min(hi, max(keep, most // (Hkv * D * e)))
        B = _spread(rng, 1, max(1, min(64, most // (Hkv * D * e * hi))))
        lo = keep if hi == keep else max(1, hi // rng.choice([1, 2, 20]))
        first = min(4, keep // 4)
        c = _evict("", B, Hkv, D, lo, hi, keep, first, _spread(rng, 1, keep - first), kind == "evict4", dtype)
    del c["name"]
    return c


# ---- inputs -----------------------------------------------------------------------------


def _dt(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _lengths(n, lo, hi):
    """n whole numbers between lo and hi, the largest among them, in no order."""
    return [lo + (hi - lo) * ((61 * i + 60) % 97 + 1) // 97 if i else hi for i in range(n)]


def _lens(case):
    return _lengths(case["B"], case["lo"], case["hi"])


def _counts(case):
    """New tokens of every sequence of an append."""
    T = case["T_new"]
    return [T] * case["B"] if T == 1 or case["B"] == 1 else [min(a, b) for a, b in zip(_lengths(case["B"], max(1, T * 2 // 5), T), _lens(case))]


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(20260528 + 1000003 * int(seed))
    return g


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _int(x):
    return torch.tensor(x, device=DEV, dtype=torch.int32)


def _states(gen, B, H, T, D, dtype, dirs=None):
    """Rows as the recurrence leaves them (a gate per channel, its last 128 terms); every 1009th token answers to the direction
    that the queries look for."""
    out = torch.empty(B, H, T, D, device=DEV, dtype=dtype)
    for b in range(B):
        x, a = _normal(gen, H, T, D), torch.sigmoid_(_normal(gen, H, 1, D).mul_(0.5).add_(4.2))
        if dirs is not None:
            x[:, 500::1009] = 3.0 * dirs[:, None] + 0.3 * x[:, 500::1009]
        x *= 1 - a
        for k in range(7):
            if (1 << k) >= T:
                break
            x[:, 1 << k:] += x[:, :-(1 << k)] * a
            a = a * a
        out[b] = x
    return out


def _cap(case):
    """Rows that the cache has room for."""
    return -(-(case["hi"] + 1) // 64) * 64


def _inputs(case, seed):
    gen, dt, kind = _gen(seed), _dt(case), case["kind"]
    B, Hkv, D, P, cap = case["B"], case["Hkv"], case["D"], case["P"], _cap(case)
    Hq = case.get("Hq", Hkv)
    s = dict(case, Hq=Hq, cap=cap)
    dirs = _normal(gen, Hkv, D)
    dirs *= math.sqrt(D) / dirs.norm(dim=-1, keepdim=True)
    s["k_cache"], s["v_cache"] = _states(gen, B, Hkv, cap, D, dt, dirs), _states(gen, B, Hkv, cap, D, dt)
    s["len"] = _int(_lens(case))
    if kind in ("append", "attn", "evict4"):
        k, v = s.pop("k_cache"), s.pop("v_cache")
        s["k4"], s["k4_scale"] = _pack(k)
        s["v4"], s["v4_scale"] = _pack(v)
        del k, v
    if kind == "append":
        T = case["T_new"]
        s["n_new"] = None if T == 1 or B == 1 else _int(_counts(case))
        s["k"], s["v"] = _states(gen, B, Hkv, T, D, dt, dirs), _states(gen, B, Hkv, T, D, dt)
        s["meta"] = torch.zeros(B, Hkv, cap // P, 2, D, device=DEV, dtype=dt)
        s["k_out"], s["v_out"] = (torch.zeros(B, Hkv, T, D, device=DEV, dtype=dt) for _ in range(2))
    if kind in ("attn", "tally"):
        s["q"] = (dirs.repeat_interleave(Hq // Hkv, 0) + 0.25 * _normal(gen, B, Hq, D)).to(dt)
        s["out"], s["lse"] = torch.zeros(B, Hq, D, device=DEV, dtype=dt), torch.zeros(B, Hq, device=DEV)
        s["scale"] = 1.0 / math.sqrt(D)
    if kind == "attn" and case["pages"]:
        # the first page, the last, and some between them, as a selection leaves them
        H, K = Hkv if case["shared"] else Hq, case["pages"]
        pages = -(-s["len"][:, None, None].long() // P)
        j = torch.arange(cap // P, device=DEV)
        rank = torch.rand(B, H, cap // P, generator=gen, device=DEV)
        rank = rank.masked_fill((j == 0) | (j == pages - 1), 2.0).masked_fill(j >= pages, -1.0)
        s["idx"] = rank.topk(K, -1).indices.sort(-1).values.int()
    if kind == "tally" or kind.startswith("evict") or case.get("tally"):
        # weight so far: a few rows have had nearly all of it, many nothing at all
        x = _normal(gen, B, Hkv, cap).mul_(2).exp_().mul_(1e-3)
        s["sum"] = x * (torch.rand(x.shape, generator=gen, device=DEV) < 0.9)
    if kind.startswith("evict"):
        s["start"] = [s[n].clone() for n in ("len", "sum")]
        s["pos"] = torch.zeros(B, Hkv, cap, device=DEV, dtype=torch.int32)
        s["mark"] = torch.zeros(B, 2, device=DEV, dtype=torch.int32)
    if kind == "evict4":
        s["k_out"], s["v_out"] = (torch.zeros(B, Hkv, case["keep"], D, device=DEV, dtype=dt) for _ in range(2))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2605_28640_amd import binding as rs
        s["rs"] = rs
        for n in ("k4", "v4"):  # a cache of bytes, which the calls ask for
            if n in s:
                s[n] = s[n].to(torch.uint8)
        s["shape"] = shape = rs.make_shape(s["B"], s["Hq"], s["Hkv"], s["D"], s["cap"], s["P"], _dt(case))
        if case["kind"] == "attn":
            lists = s["idx"].shape[1:] if case["pages"] else (0, 0)
            s["ws"] = rs.Workspace(rs.kv4_attn_decode_workspace_bytes(shape, *lists, case["tally"]))
        elif case["kind"] == "tally":
            s["ws"] = rs.Workspace(rs.attn_decode_tally_workspace_bytes(shape))
        elif case["kind"] != "append":
            s["ws"] = rs.Workspace(rs.cache_evict_workspace_bytes(shape, case["keep"]))
    return s


# ---- one pass, by elementary operations -------------------------------------------------


def _two(e):
    """2 ** e for whole e from -126 to 127, by its bits: a power function may miss it by one."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _pack(x):
    """Codes and scale bytes of rows [..., D]."""
    x = x.float().unflatten(-1, (-1, GROUP))
    top = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)  # top = m 2^e, 1/2 <= m < 1; at most 7 units of the scale
    e = torch.where(m <= 0.875, e - 3, e - 2).clamp(-125, 125)
    y = x.abs() * _two(-e)
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    y = (torch.round(y / step) * step).clamp(max=6.0)
    code = torch.where(y < 2, 2 * y, torch.where(y < 4, y + 2, y / 2 + 4)).to(torch.uint8)
    code = (code + 8 * (x < 0)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)[..., 0]


def _values(codes, scales):
    """What they stand for, in 32 bits."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEV)
    table = torch.cat([table, -table])
    x = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).flatten(-2)
    return (x.unflatten(-1, (-1, GROUP)) * _two(scales.int() - 127)[..., None]).flatten(-2)


def _append_plain(s):
    B, Hkv, D, P, T, cap = (s[n] for n in ("B", "Hkv", "D", "P", "T_new", "cap"))
    length = s["len"].long()[:, None]
    count = s["n_new"].long()[:, None] if s["n_new"] is not None else torch.full_like(length, T)
    t = torch.arange(T, device=DEV)[None]
    b, i = (t < count).nonzero(as_tuple=True)
    at = (length - count)[b, 0] + i
    for x in "kv":
        codes, scales = _pack(s[x])
        s[x + "4"][b, :, at] = codes[b, :, i]
        s[x + "4_scale"][b, :, at] = scales[b, :, i]
    # the bounds of every page with a new row
    near = torch.arange((T + P - 2) // P + 1, device=DEV)[None] + (length - count) // P
    b, i = (near * P < length).nonzero(as_tuple=True)
    page = near[b, i]
    rows = _values(*(s[n].unflatten(2, (-1, P))[b, :, page] for n in ("k4", "k4_scale")))
    stored = (page[:, None] * P + torch.arange(P, device=DEV) < length[b])[:, None, :, None]
    s["meta"][b, :, page, 0] = rows.masked_fill(~stored, math.inf).amin(2).to(s["meta"].dtype)
    s["meta"][b, :, page, 1] = rows.masked_fill(~stored, -math.inf).amax(2).to(s["meta"].dtype)
    _fetch_plain(s, length - T + t)
    return [s["k_out"], s["v_out"], s["meta"]]


def _fetch_plain(s, token):
    """Rows of these tokens [B, T] to k_out and v_out; those that a sequence does not have stay as they are."""
    real = ((token >= 0) & (token < s["len"].long()[:, None]))[:, None, :, None]
    b = torch.arange(s["B"], device=DEV)[:, None]
    for x in "kv":
        rows = (s[n][b, :, token.clamp(min=0)].transpose(1, 2) for n in (x + "4", x + "4_scale"))
        s[x + "_out"].copy_(torch.where(real, _values(*rows).to(s[x + "_out"].dtype), s[x + "_out"]))


def _attend(s, k, v, seen):
    """Outputs, log-sum-exps and weights of the queries over rows k, v of their KV heads, [B, Hkv or Hq, rows, D]."""
    B, Hq, D, H = s["B"], s["Hq"], s["D"], k.shape[1]
    p = torch.matmul(s["q"].float().view(B, H, Hq // H, D), k.transpose(2, 3)).mul_(s["scale"])
    p.masked_fill_(~seen, -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p /= total
    return torch.matmul(p, v).view(B, Hq, D).to(s["out"].dtype), (top + total.log()).view(B, Hq), p


def _attn_plain(s):
    B, Hq, Hkv, P, cap = (s[n] for n in ("B", "Hq", "Hkv", "P", "cap"))
    length = s["len"].long()[:, None, None, None]
    if "idx" in s:
        H, idx = s["idx"].shape[1], s["idx"].long()
        b, h = torch.arange(B, device=DEV)[:, None, None], torch.arange(H, device=DEV)[None, :, None] * Hkv // H
        k, v = (_values(*(s[n].unflatten(2, (-1, P))[b, h, idx].flatten(2, 3) for n in (x + "4", x + "4_scale"))) for x in "kv")
        t = (idx[..., None] * P + torch.arange(P, device=DEV)).flatten(2)[:, :, None]
        return list(_attend(s, k, v, t < length)[:2])
    if s["kind"] == "tally":
        k, v = s["k_cache"].float(), s["v_cache"].float()
    else:
        k, v = _values(s["k4"], s["k4_scale"]), _values(s["v4"], s["v4_scale"])
    t = torch.arange(cap, device=DEV)
    seen = t < length
    out, lse, p = _attend(s, k, v, seen)
    if "sum" not in s:
        return [out, lse]
    before = torch.where(t == length[:, 0] - 1, 0, s["sum"])  # the newest row has had none
    s["sum"].copy_(torch.where(seen[:, 0], before + p.sum(2), s["sum"]))
    return [out, lse, s["sum"]]


def _evict_plain(s):
    B, Hkv, cap, keep = (s[n] for n in ("B", "Hkv", "cap", "keep"))
    length, (known, before) = s["len"].long()[:, None, None], s["mark"].long().t()[:, :, None, None]
    t = torch.arange(cap, device=DEV)
    total = before + length - known
    pos = torch.where(t < known, s["pos"].long(), before + t - known)
    over = length > keep
    safe = (pos < s["first"]) | (pos >= total - s["recent"])
    rank = torch.where(safe, math.inf, s["sum"]).masked_fill(t >= length, -1.0)  # (a tally is not below 0)
    order = rank.argsort(dim=-1, descending=True, stable=True)
    kept = torch.zeros_like(rank, dtype=torch.bool).scatter_(-1, order[..., :keep], True)
    holes, movers = ~kept & (t < keep), kept & (t >= keep)
    to = torch.where(holes, t, cap).sort(-1).values[..., :min(keep, cap - keep)]
    src = torch.where(movers, t, cap).sort(-1).values[..., :min(keep, cap - keep)]
    real = (to < cap) & (src < cap) & over
    b, h, i = real.nonzero(as_tuple=True)
    src, to = src[b, h, i], to[b, h, i]
    for n in ("k4", "k4_scale", "v4", "v4_scale") if s["kind"] == "evict4" else ("k_cache", "v_cache"):
        s[n][b, h, to] = s[n][b, h, src]
    s["sum"][b, h, to] = s["sum"][b, h, src]
    pos[b, h, to] = pos[b, h, src]
    s["pos"].copy_(torch.where(over & (t < keep), pos, s["pos"].long()))
    s["mark"].copy_(torch.where(over[:, 0], torch.stack([torch.full_like(total, keep), total], -1)[:, 0, 0], s["mark"].long()))
    s["len"].clamp_(max=keep)


# ---- one pass ---------------------------------------------------------------------------


def run(s):
    kind = s["kind"]
    if own:
        rs, shape = s["rs"], s["shape"]
        four = [s[n] for n in ("k4", "k4_scale", "v4", "v4_scale")] if "k4" in s else []
    if kind == "append":
        if not own:
            return _append_plain(s)
        rs.kv4_append(shape, s["k"], s["v"], 0, s["len"], s["n_new"], s["T_new"], *four, s["meta"])
        rs.kv4_fetch(shape, *four, s["len"], -s["T_new"], s["T_new"], s["k_out"], s["v_out"])
        return [s["k_out"], s["v_out"], s["meta"]]
    if kind in ("attn", "tally"):
        if not own:
            return _attn_plain(s)
        if kind == "attn":
            rs.kv4_attn_decode(shape, s["q"], *four, s["len"], s["scale"], s.get("idx"), s.get("sum"), 1, s["out"], s["lse"], s["ws"])
        else:
            rs.attn_decode_tally(shape, s["q"], s["k_cache"], s["v_cache"], s["len"], s["scale"], s["sum"], 1, s["out"], s["lse"], s["ws"])
        return [s[n] for n in ("out", "lse", "sum") if n in s]
    if s["hi"] == s["keep"]:
        s["len"].add_(1)  # the next token's row is there
    else:  # the sequences have grown again
        s["len"].copy_(s["start"][0])
        s["sum"].copy_(s["start"][1])
    if own:
        more = (s["sum"], s["pos"], s["mark"], s["len"], s["keep"], s["first"], s["recent"], 0, s["ws"])
        if kind == "evict4":
            rs.kv4_evict(shape, *four, *more)
            rs.kv4_fetch(shape, *four, s["len"], 0, s["keep"], s["k_out"], s["v_out"])
        else:
            rs.cache_evict(shape, s["k_cache"], s["v_cache"], *more)
    else:
        _evict_plain(s)
        if kind == "evict4":
            _fetch_plain(s, torch.arange(s["keep"], device=DEV).expand(s["B"], -1))
    rows = ("k_out", "v_out") if kind == "evict4" else ("k_cache", "v_cache")
    return [s[n] for n in rows + ("sum", "pos", "mark", "len")]


# ---- what a pass cannot do without ------------------------------------------------------


def work(case):
    kind, e = case["kind"], 4 if case["dtype"] == "f32" else 2
    B, Hkv, D, P = case["B"], case["Hkv"], case["D"], case["P"]
    four = D // 2 + D // GROUP
    if kind == "append":  # rows in, codes out, bounds out; codes in, values out
        n = sum(_counts(case))
        pages = sum(-(-x // P) for x in _counts(case))
        return {"bytes": 2 * Hkv * (n * (2 * D * e + 2 * four) + pages * D * e), "flops": 4 * n * Hkv * D}
    if kind in ("attn", "tally"):
        Hq, lens, row = case["Hq"], _lens(case), 2 * (four if kind == "attn" else D * e)
        keys, seen = Hkv * sum(lens), Hq * sum(lens)
        if case.get("pages"):
            each = Hkv if case["shared"] else Hq
            seen = sum(min(case["pages"] * P, n) for n in lens) * Hq
            keys = sum(min(case["pages"] * P * (each // Hkv), n) for n in lens) * Hkv
        elif kind == "tally" or case["tally"]:
            row += 8
        return {"bytes": keys * row + B * Hq * (2 * D * e + 4), "flops": 4 * D * seen}
    keep, lens = case["keep"], _lens(case)
    out = [max(0, n - keep) for n in lens] if case["hi"] > keep else [1] * B
    move = Hkv * sum(x * keep // (x + keep) if case["hi"] > keep else 1 for x in out)  # where chance has put the kept ones
    read = 8 * Hkv * sum(keep + x for x in out if x)
    back = Hkv * sum(min(n, keep) for n in lens) * 2 * (four + D * e) if kind == "evict4" else 0
    return {"bytes": read + move * 2 * (2 * (four if kind == "evict4" else D * e) + 8) + back, "flops": 0}


# ---- the same in 64 bits ----------------------------------------------------------------

_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_two(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_values(codes, scales):
    n = codes.long()
    n = torch.stack([n % 16, n // 16], -1).reshape(*codes.shape[:-1], -1)
    grid = torch.tensor(_GRID, device=DEV, dtype=torch.float64)
    x = grid[n % 8] * (1 - 2 * (n // 8)).double()
    return x * _exact_two(scales.long() - 127).repeat_interleave(GROUP, -1)


def _exact_rounded(x):
    """Values that rows [..., D] have in 4 bits: the nearest of the grid, of two equally near ones that with the even code."""
    x = x.double().unflatten(-1, (-1, GROUP))
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 7)).clamp(-125, 125)
    e = torch.where((top > 7 * _exact_two(e)) & (e < 125), e + 1, e)
    e = torch.where((top <= 7 * _exact_two(e - 1)) & (e > -125), e - 1, e)
    y = x.abs() / _exact_two(e)
    best = torch.zeros_like(y)
    for i in range(1, 8):
        middle = (_GRID[i - 1] + _GRID[i]) / 2
        best = torch.where((y > middle) | ((y == middle) & (i % 2 == 0)), _GRID[i], best)
    return (best * torch.sign(x) * _exact_two(e)).flatten(-2)


def _exact_append(case, s):
    P, T = case["P"], case["T_new"]
    k, v = _exact_values(s["k4"], s["k4_scale"]), _exact_values(s["v4"], s["v4_scale"])
    meta, k_out, v_out = (s[n].double() for n in ("meta", "k_out", "v_out"))
    for b, (n, new) in enumerate(zip(_lens(case), _counts(case))):
        k[b, :, n - new:n], v[b, :, n - new:n] = _exact_rounded(s["k"][b, :, :new]), _exact_rounded(s["v"][b, :, :new])
        back = min(n, T)
        k_out[b, :, T - back:], v_out[b, :, T - back:] = k[b, :, n - back:n], v[b, :, n - back:n]
        for p in range((n - new) // P, (n - 1) // P + 1):
            meta[b, :, p, 0], meta[b, :, p, 1] = k[b, :, p * P:min(n, p * P + P)].amin(1), k[b, :, p * P:min(n, p * P + P)].amax(1)
    return [k_out, v_out, meta]


def _exact_attn(case, s):
    B, Hq, Hkv, P = case["B"], s["Hq"], case["Hkv"], case["P"]
    out, lse = s["out"].double(), s["lse"].double()
    total = s["sum"].double() if "sum" in s else None
    for b, n in enumerate(_lens(case)):
        for h in range(Hkv):
            if case["kind"] == "tally":
                k, v = s["k_cache"][b, h, :n].double(), s["v_cache"][b, h, :n].double()
            else:
                k, v = _exact_values(s["k4"][b, h, :n], s["k4_scale"][b, h, :n]), _exact_values(s["v4"][b, h, :n], s["v4_scale"][b, h, :n])
            weight = torch.zeros(n, device=DEV, dtype=torch.float64)
            for q in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                rows = slice(None)
                if "idx" in s:
                    page = s["idx"][b, h if case["shared"] else q].long()
                    rows = (page[:, None] * P + torch.arange(P, device=DEV)).flatten()
                    rows = rows[rows < n]
                z = k[rows] @ s["q"][b, q].double() / math.sqrt(case["D"])
                lse[b, q] = torch.logsumexp(z, 0)
                p = torch.exp(z - lse[b, q])
                out[b, q] = p @ v[rows]
                if total is not None:
                    weight += p
            if total is not None:
                total[b, h, n - 1] = 0
                total[b, h, :n] += weight
    return [out, lse] if total is None else [out, lse, total]


def _exact_evict(case, s):
    keep, four = case["keep"], case["kind"] == "evict4"
    k, v = (_exact_values(s[x + "4"], s[x + "4_scale"]) if four else s[x + "_cache"].double() for x in "kv")
    total = s["sum"].double()
    for b, n in enumerate([case["hi"] + 1] * case["B"] if case["hi"] == keep else _lens(case)):
        if n <= keep:
            continue
        for h in range(case["Hkv"]):
            free = total[b, h, case["first"]:n - case["recent"]]  # (at the first pass a row's place is its position)
            gone = torch.sort(free.flip(0), stable=True).indices[:n - keep]  # the smallest; of equal ones the later
            gone = n - case["recent"] - 1 - gone
            stays = torch.ones(n, device=DEV, dtype=torch.bool)
            stays[gone] = False
            to, src = (~stays[:keep]).nonzero()[:, 0], stays[keep:].nonzero()[:, 0] + keep
            for x in (k, v, total):
                x[b, h, to] = x[b, h, src]
    if four:
        full = torch.zeros(case["B"], case["Hkv"], keep, case["D"], device=DEV, dtype=torch.float64)
        real = torch.arange(keep, device=DEV)[None, None, :, None] < s["len"].long()[:, None, None, None]
        k, v = (torch.where(real, x[:, :, :keep], full) for x in (k, v))
    return [k, v, total, None, None, None]


def exact(case, seed):
    s = _inputs(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "tally": _exact_attn, "evict": _exact_evict, "evict4": _exact_evict}[case["kind"]](case, s)
