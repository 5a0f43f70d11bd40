"""One token's attention over caches in 4 bits, bfloat16 and float32 with a tally of the rows' weights, against a computation in 64 bits.

What is allowed: a score's rounding makes a weight off by M.rounding (relative); bfloat16 results take weights rounded to bfloat16 (2^-8 relative each, against
weights that sum up to 1: 2^-8 sum p |v|) and are rounded once more (2^-8 of the result)."""
import numpy as np
import pytest
import torch

import kv4_model as M
from gpu_util import say, tdtype
from test_gpu_kv4 import Cache

pytestmark = pytest.mark.gpu

KINDS = [("four", "bf16"), ("four", "f32"), ("rows", "bf16"), ("rows", "f32")]


class Decode:
    """Caches, queries and a tally; rows from a sequence's length on hold NaN and infinities."""

    def __init__(self, rs, kind, dtype, B, Hq, Hkv, D, Tcap, lens, P=16, seed=0, big=1.0):
        self.rs, self.kind, self.lens, self.D, self.scale = rs, kind, list(lens), D, 1 / np.sqrt(D)
        r = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.s = rs.make_shape(B, Hq, Hkv, D, Tcap, P, tdtype(dtype))
        dt = tdtype(dtype)
        rand = lambda *n: torch.randn(*n, device="cuda", generator=g)
        k, v = rand(B, Hkv, Tcap, D), rand(B, Hkv, Tcap, D)
        if kind == "four":
            full = [x.to(dt) for x in (k, v)]
            self.c = Cache(rs, B, Hkv, D, Tcap, P, dtype, [Tcap] * B, seed=seed)
            self.c.byte = [np.full_like(x, 127) for x in self.c.byte]
            rs.kv4_append(self.c.s, *full, 0, self.c.len, None, Tcap, *self.c.dev, None)
            self.cache = self.c.dev
            got = [x.cpu().numpy() for x in self.cache]
            self.k, self.v = (M.values(M.from_bytes(c), f) for c, f in zip(got[0::2], got[1::2]))
            for x in self.cache[1::2]:  # from the length on: NaN
                for b, L in enumerate(lens):
                    x[b, :, min(max(L, 0), Tcap):] = 255
        else:
            self.cache = [x.to(dt) for x in (k, v)]
            self.k, self.v = (x.double().cpu().numpy() for x in self.cache)
            for x, bad in zip(self.cache, (np.nan, np.inf)):
                for b, L in enumerate(lens):
                    x[b, :, min(max(L, 0), Tcap):] = bad
        self.len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.q = (rand(B, Hq, D) * big).to(dt)
        self.out, self.lse = torch.full((B, Hq, D), 5.0, device="cuda", dtype=dt), torch.full((B, Hq), 5.0, device="cuda")
        self.tally = rand(B, Hkv, Tcap).abs()

    def run(self, tally=True, fresh=1, idx=None, ws=None):
        rs, s = self.rs, self.s
        if self.kind == "four":
            lists = idx.shape[1:] if idx is not None else (0, 0)
            ws = ws or rs.Workspace(rs.kv4_attn_decode_workspace_bytes(s, *lists, tally))
            rs.kv4_attn_decode(s, self.q, *self.cache, self.len, self.scale, idx, self.tally if tally else None, fresh, self.out, self.lse, ws)
        else:
            ws = ws or rs.Workspace(rs.attn_decode_tally_workspace_bytes(s))
            rs.attn_decode_tally(s, self.q, *self.cache, self.len, self.scale, self.tally, fresh, self.out, self.lse, ws)
        self.ws = ws
        torch.cuda.synchronize()

    def check(self, before=None, fresh=1, idx=None):
        """before: the tally before the call (None: no tally)."""
        s, D, G = self.s, self.D, self.s.Hq // self.s.Hkv
        q, out, lse = (x.double().cpu().numpy() for x in (self.q, self.out, self.lse))
        bf = self.out.dtype == torch.bfloat16
        if before is not None:
            before, after = (x.double().cpu().numpy() for x in (before, self.tally))
        worst = 0.0
        for b, L in enumerate(self.lens):
            L = min(max(L, 0), s.Tcap)
            for h in range(s.Hkv):
                heads = slice(h * G, h * G + G)
                if idx is None:
                    rows = [np.arange(L)] * G
                else:
                    per = idx.shape[1] // s.Hkv
                    rows = []
                    for g in range(G):
                        pages = idx[b, h * per + (g if per > 1 else 0)].cpu().numpy()
                        pages = pages[(pages >= 0) & (pages < s.Tcap // s.P)]
                        t = (pages[:, None] * s.P + np.arange(s.P)).ravel()
                        rows.append(t[t < L])
                weight = np.zeros(s.Tcap)
                slack = np.zeros(s.Tcap)
                for g in range(G):
                    t = rows[g]
                    o, z, p, a, most = M.attention(q[b, heads][g:g + 1], self.k[b, h, t], self.v[b, h, t], self.scale)
                    e = M.rounding(most[0], len(t), D)
                    tol = (e + (2.0 ** -8 if bf else 0)) * a[0] + (2.0 ** -8 if bf else 2.0 ** -24) * np.abs(o[0]) + 1e-30
                    err = np.abs(out[b, h * G + g] - o[0])
                    assert np.all(err <= tol), (b, h, g, L, float((err / tol).max()))
                    worst = max(worst, float((err / tol).max()) if L else 0.0)
                    if len(t) == 0:
                        assert lse[b, h * G + g] == -np.inf
                        continue
                    assert abs(lse[b, h * G + g] - z[0]) <= e + 2.0 ** -22 * abs(z[0]), (b, h, g, lse[b, h * G + g], z[0])
                    weight[t] += p[0]
                    slack[t] += e * p[0]
                if before is not None:
                    base = before[b, h].copy()
                    base[max(0, L - fresh):L] = 0
                    want = base + weight
                    err = np.abs(after[b, h] - want)
                    assert np.all(err <= slack + 2.0 ** -22 * np.abs(want)), (b, h, L, int(np.argmax(err)))
                    assert np.array_equal(after[b, h, L:], before[b, h, L:])
        say("   worst of what is allowed: %.2f" % worst)


SHAPES = [  # B, Hq, Hkv, D, Tcap, lengths
    (1, 2, 2, 64, 64, [1]),
    (3, 4, 2, 64, 208, [1, 0, 205]),
    (2, 8, 2, 128, 1000, [1000, 63]),
    (4, 14, 2, 128, 333, [64, 65, 128, 400]),
    (6, 3, 1, 64, 700, [700, 3, 129, -2, 16, 17]),
    (2, 40, 2, 128, 300, [299, 31]),   # 20 queries to a head: two tiles
    (1, 64, 1, 64, 150, [150]),
    (1, 4, 4, 128, 5000, [4999]),      # cut over many workgroups
    (70, 2, 2, 64, 320, [(37 * i) % 321 for i in range(70)]),
    (70, 2, 1, 64, 2200, [(371 * i) % 2201 for i in range(70)]),  # more sequences than lanes, tiles of many steps
    (3, 8, 8, 64, 1500, [1500, 0, 1]),
    (1, 300, 1, 64, 1300, [1234]),     # 300 queries to a head
    (2, 34, 2, 128, 2500, [2500, 1111]),
]


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention_and_tally(rs, kind, dtype, shape):
    B, Hq, Hkv, D, Tcap, lens = SHAPES[shape]
    say("decode", kind, dtype, SHAPES[shape][:5])
    d = Decode(rs, kind, dtype, B, Hq, Hkv, D, Tcap, lens, seed=shape)
    for fresh in (1, 0, 70):
        before = d.tally.clone()
        d.run(fresh=fresh)
        d.check(before, fresh)
    out, lse = d.out.clone(), d.lse.clone()
    d.run(fresh=0, ws=d.ws)
    assert torch.equal(out, d.out) and torch.equal(lse, d.lse)
    if kind == "four":  # without a tally: the same results
        kept = d.tally.clone()
        d.run(tally=False)
        assert torch.equal(out, d.out) and torch.equal(lse, d.lse) and torch.equal(kept, d.tally)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(2, 4, 4, 64, 256, 16, 4, [256, 100]), (2, 8, 2, 128, 512, 32, 5, [512, 77]), (3, 4, 2, 128, 1024, 128, 3, [1000, 0, 130]),
                                   (1, 4, 2, 64, 1024, 512, 2, [600]), (2, 32, 8, 128, 2048, 16, 40, [2047, 1999]),
                                   (2, 40, 2, 128, 4096, 16, 200, [4096, 3001]), (3, 6, 3, 64, 2048, 64, 30, [2048, 0, 1333])])
@pytest.mark.parametrize("shared", [False, True])
def test_listed_pages(rs, dtype, shape, shared):
    B, Hq, Hkv, D, Tcap, P, K, lens = shape
    say("listed", dtype, shape, shared)
    d = Decode(rs, "four", dtype, B, Hq, Hkv, D, Tcap, lens, P=P, seed=K)
    H = Hkv if shared else Hq
    r = np.random.default_rng(K)
    idx = np.stack([[r.permutation(Tcap // P)[:K] for _ in range(H)] for _ in range(B)]).astype(np.int32)
    idx[:, ::2] = np.sort(idx[:, ::2])
    idx[0, 0, 1::2] = -1                 # entries that name no page
    idx[-1, -1, 0] = Tcap // P + 3
    if H > 1:
        idx[0, 1] = -5                   # a list of nothing
    idx = torch.from_numpy(idx).cuda()
    d.run(tally=False, idx=idx)
    d.check(idx=idx)


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_large_scores(rs, kind, dtype):
    """Scores of hundreds: one row takes nearly all of the weight, and the reference point moves."""
    d = Decode(rs, kind, dtype, 2, 8, 2, 128, 700, [700, 333], seed=11, big=40.0)
    before = d.tally.clone()
    d.run()
    d.check(before)


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_values_that_are_not_finite(rs, kind, dtype):
    """NaN in a row that is attended shows in its head's results; sequences and heads beside it are as ever."""
    d = Decode(rs, kind, dtype, 2, 4, 2, 64, 200, [200, 150], seed=12)
    d.run()
    out = d.out.clone()
    x = d.cache[1 if kind == "four" else 0]
    x[1, 0, 140] = 255 if kind == "four" else float("nan")
    d.run()
    assert d.out[1, :2].isnan().all() and d.lse[1, :2].isnan().all() and d.tally[1, 0, :150].isnan().all()
    assert torch.equal(d.out[0], out[0]) and torch.equal(d.out[1, 2:], out[1, 2:]) and not d.tally[1, 1].isnan().any() and not d.tally[0].isnan().any()
    assert not d.tally[1, 0, 150:].isnan().any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_scores(rs, dtype):
    """Rows whose score is -inf have no weight; where all are, the row sees nothing; +inf is NaN, as the formula has it."""
    d = Decode(rs, "rows", dtype, 3, 2, 2, 64, 300, [300, 300, 300], seed=13)
    d.q.fill_(1.0)
    k = d.cache[0]
    k[0, 0, :290, 5] = -float("inf")
    k[1, 0, :, 7] = -float("inf")
    k[2, 0, 40, 9] = float("inf")
    d.tally.zero_()
    d.run(fresh=0)
    assert d.out[0].isfinite().all() and (d.tally[0, 0, :290] == 0).all() and abs(float(d.tally[0, 0].sum()) - 1) < 1e-5
    assert (d.out[1, 0] == 0).all() and d.lse[1, 0] == -float("inf") and (d.tally[1, 0] == 0).all()
    assert d.out[2, 0].isnan().all()
    assert d.out[:, 1].isfinite().all()


@pytest.mark.parametrize("kind,dtype", [("four", "bf16"), ("rows", "bf16"), ("rows", "f32")])
def test_two_streams_and_a_shared_workspace_in_graphs(rs, kind, dtype):
    """Two graphs and eager calls of another shape share a workspace; a call on another stream than the current one's tensors."""
    a = Decode(rs, kind, dtype, 3, 8, 2, 128, 900, [900, 5, 500], seed=21)
    b = Decode(rs, kind, dtype, 2, 4, 4, 128, 400, [123, 400], seed=22)
    for d in (a, b):
        d.run(fresh=0)
        d.want, d.before = (d.out.clone(), d.lse.clone()), d.tally.clone()
    ws = a.ws if a.ws.nbytes >= b.ws.nbytes else b.ws
    graphs = []
    for d in (a, b):
        d.tally.copy_(d.before)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            args = (d.s, d.q, *d.cache, d.len, d.scale) + ((None,) if kind == "four" else ()) + (d.tally, 0, d.out, d.lse, ws)
            (rs.kv4_attn_decode if kind == "four" else rs.attn_decode_tally)(*args)
        graphs.append(g)
    step = {}
    for turn in range(4):
        for d, g in zip((a, b), graphs):
            d.out.fill_(9)
            before = d.tally.clone()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(d.out, d.want[0]) and torch.equal(d.lse, d.want[1])
            step.setdefault(id(d), d.tally - before)
            if turn == 1:  # eager work between the replays, a longer cache
                kept = d.tally.clone()
                d.run(fresh=0, ws=ws)
                d.tally.copy_(kept)
    # the lengths live on the device: a replay follows them
    a.len.copy_(torch.tensor([17, 900, 0], dtype=torch.int32))
    a.lens = [17, 900, 0]
    if kind == "rows":
        fresh = Decode(rs, kind, dtype, 3, 8, 2, 128, 900, [900, 900, 900], seed=21)
        for x, y in zip(a.cache, fresh.cache):
            x.copy_(y)
    else:
        fresh = Decode(rs, kind, dtype, 3, 8, 2, 128, 900, [900, 900, 900], seed=21)
        for x, y in zip(a.cache, fresh.cache):
            x.copy_(y)
    before = a.tally.clone()
    graphs[0].replay()
    torch.cuda.synchronize()
    a.check(before, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.run(fresh=0)
    side.synchronize()
    assert torch.equal(b.out, b.want[0])


@pytest.mark.parametrize("kind", ["four", "rows"])
def test_a_long_cache(rs, kind):
    """Offsets past 2^32 bytes within a head: 20 million rows (4 bits: 80 million) of 128 channels, of which few count for anything: all others are zeros with
    queries that see them at a score of 0."""
    Tcap, D = (80_000_000, 128) if kind == "four" else (20_000_000, 128)
    dt = torch.bfloat16
    s = rs.make_shape(1, 1, 1, D, Tcap, 16, dt)
    q = torch.ones(1, 1, D, device="cuda", dtype=dt)
    last = torch.full((1, 1, 1, D), 4.0, device="cuda", dtype=dt)
    length = torch.tensor([Tcap - 3], dtype=torch.int32, device="cuda")
    tally = torch.zeros(1, 1, Tcap, device="cuda")
    out, lse = torch.zeros(1, 1, D, device="cuda", dtype=dt), torch.zeros(1, 1, device="cuda")
    if kind == "four":
        cache = [torch.zeros(1, 1, Tcap, n, dtype=torch.uint8, device="cuda") for n in (64, 4, 64, 4)]
        rs.kv4_append(s, last, last, 0, length, None, 1, *cache, None)
        rs.kv4_attn_decode(s, q, *cache, length, 1.0, None, tally, 0, out, lse, rs.Workspace(rs.kv4_attn_decode_workspace_bytes(s, 0, 0, True)))
    else:
        cache = [torch.zeros(1, 1, Tcap, D, dtype=dt, device="cuda") for _ in "kv"]
        for x in cache:
            x[:, :, Tcap - 4] = last[:, :, 0]
        rs.attn_decode_tally(s, q, *cache, length, 1.0, tally, 0, out, lse, rs.Workspace(rs.attn_decode_tally_workspace_bytes(s)))
    torch.cuda.synchronize()
    assert abs(float(lse) - 512) < 1e-3 and (out == 4).all()  # e^512 against 80 million e^0
    assert float(tally[0, 0, Tcap - 4]) == 1 and float(tally.sum()) == 1


def _values(codes, byte):
    """A 4-bit cache's values on the device, in 64 bits."""
    grid = torch.tensor(np.concatenate([M.GRID, -M.GRID]), device="cuda")
    x = torch.stack([grid[(codes & 15).int()], grid[(codes >> 4).int()]], -1).flatten(-2)
    return x * ((byte.long() + 896) << 52).view(torch.float64).repeat_interleave(32, -1)


@pytest.mark.parametrize("B,Hq,Hkv,lens", [(4, 16, 8, [20000, 19001, 17, 20016]), (130, 4, 4, None), (1024, 2, 1, None)])
@pytest.mark.parametrize("tally", [False, True])
def test_many_units_a_wave(rs, B, Hq, Hkv, lens, tally):
    """More work than the line's shares are alike for (three workgroups a CU), and as many sequences as are taken."""
    D, G = 128, Hq // Hkv
    lens = lens or [(7919 * i) % 2600 for i in range(B)]
    Tcap = max(lens) + 3
    g = torch.Generator(device="cuda").manual_seed(B)
    s = rs.make_shape(B, Hq, Hkv, D, Tcap, 16, torch.bfloat16)
    dev = [torch.randint(lo, hi, (B, Hkv, Tcap, n), dtype=torch.uint8, device="cuda", generator=g) for lo, hi, n in
           ((0, 256, 64), (121, 126, 4), (0, 256, 64), (121, 126, 4))]
    q = torch.randn(B, Hq, D, device="cuda", generator=g).bfloat16()
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    before = torch.rand(B, Hkv, Tcap, device="cuda", generator=g)
    got = before.clone()
    out, lse = torch.zeros_like(q), torch.zeros(B, Hq, device="cuda")
    ws = rs.Workspace(rs.kv4_attn_decode_workspace_bytes(s, 0, 0, tally))
    rs.kv4_attn_decode(s, q, *dev, ln, 0.09, None, got if tally else None, 1, out, lse, ws)
    first = out.clone()
    rs.kv4_attn_decode(s, q, *dev, ln, 0.09, None, got.clone() if tally else None, 1, out, lse, ws)
    torch.cuda.synchronize()
    assert torch.equal(first, out)
    for b in range(B):
        L = lens[b]
        if L == 0:
            assert (out[b] == 0).all() and (lse[b] == -float("inf")).all()
            continue
        k, v = _values(dev[0][b, :, :L], dev[1][b, :, :L]), _values(dev[2][b, :, :L], dev[3][b, :, :L])
        qq = q[b].double().view(Hkv, G, D)
        z = torch.matmul(qq, k.transpose(1, 2).contiguous()) * 0.09
        want = torch.logsumexp(z, -1)
        p = torch.exp(z - want[..., None])
        o, a = torch.matmul(p, v).view(Hq, D), torch.matmul(p, v.abs()).view(Hq, D)
        e = M.rounding(float((torch.matmul(qq.abs(), k.abs().transpose(1, 2).contiguous()) * 0.09).max()), L, D)
        assert ((out[b].double() - o).abs() <= (e + 2.0 ** -8) * a + 2.0 ** -8 * o.abs()).all(), b
        assert ((lse[b].double() - want.view(Hq)).abs() <= e + 2.0 ** -22 * want.view(Hq).abs()).all(), b
        if tally:
            base = before[b].double()
            base[:, L - 1] = 0
            w = base[:, :L] + p.sum(1)
            assert ((got[b, :, :L].double() - w).abs() <= e * p.sum(1) + 2.0 ** -22 * w).all(), b
            assert torch.equal(got[b, :, L:], before[b, :, L:])


def test_quest_over_a_4_bit_cache(rs):
    """Recurrence, append with bounds, page selection, attention of the listed pages, eviction and the bounds anew: together, as a decode loop has them."""
    B, Hq, Hkv, D, P, Tcap, T0, steps, K = 2, 8, 4, 128, 16, 512, 333, 20, 9
    dt = torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(9)
    rand = lambda *n: torch.randn(*n, device="cuda", generator=g)
    s, s1 = rs.make_shape(B, Hq, Hkv, D, Tcap, P, dt), rs.make_shape(B, Hq, Hkv, D, 16, 16, dt)
    four = [torch.zeros(B, Hkv, Tcap, n, dtype=torch.uint8, device="cuda") for n in (64, 4, 64, 4)]
    meta = torch.zeros(B, Hkv, Tcap // P, 2, D, device="cuda", dtype=dt)
    sk, sv = torch.zeros(B, Hkv, D, device="cuda"), torch.zeros(B, Hkv, D, device="cuda")
    full = [torch.zeros(B, Hkv, Tcap, D, device="cuda", dtype=dt) for _ in "kv"]
    ws = rs.Workspace(max(rs.rat_scan_workspace_bytes(s, T0), rs.quest_select_decode_workspace_bytes(s, Tcap), rs.kv4_attn_decode_workspace_bytes(s, Hq, K, False),
                          rs.kv4_attn_decode_workspace_bytes(s, 0, 0, True), rs.cache_evict_workspace_bytes(s, 200)))
    rs.rat_scan(s, rand(B, Hkv, T0, D).to(dt), rand(B, Hkv, T0, D).to(dt), torch.sigmoid(rand(B, Hkv, T0, D) * 0.5 + 3), sk, sv, *full, 0, T0, ws)
    length = torch.full((B,), T0, dtype=torch.int32, device="cuda")
    rs.kv4_append(s, *full, 0, length, None, T0, *four, meta)
    stage = [torch.zeros(B, Hkv, 16, D, device="cuda", dtype=dt) for _ in "kv"]
    out, lse, idx = torch.zeros(B, Hq, D, device="cuda", dtype=dt), torch.zeros(B, Hq, device="cuda"), torch.zeros(B, Hq, K, device="cuda", dtype=torch.int32)
    for i in range(steps):
        T = T0 + i + 1
        rs.rat_scan(s1, rand(B, Hkv, 1, D).to(dt), rand(B, Hkv, 1, D).to(dt), torch.sigmoid(rand(B, Hkv, 1, D) * 0.5 + 3), sk, sv, *stage, 0, 1)
        length.add_(1)
        rs.kv4_append(s, *stage, 0, length, None, 1, *four, meta)
        q = (2 * rand(B, Hq, D)).to(dt)
        rs.quest_select_decode(s, q, meta, T, K, 1, 1, idx, None, ws)
        rs.kv4_attn_decode(s, q, *four, length, D ** -0.5, idx, None, 1, out, lse, ws)
        torch.cuda.synchronize()
        k, v = _values(*four[:2])[:, :, :T], _values(*four[2:])[:, :, :T]
        pages = -(-T // P)
        for p in range(pages):  # the bounds hold the values themselves
            rows = k[:, :, p * P:p * P + P]
            assert torch.equal(meta[:, :, p].double(), torch.stack([rows.amin(2), rows.amax(2)], 2))
        for b in range(B):
            for h in range(Hq):
                t = (idx[b, h].cpu().numpy()[:, None] * P + np.arange(P)).ravel()
                t = t[t < T]
                assert len(set(t)) == len(t) and {0, T - 1} <= set(t)
                o, z, _, a, most = M.attention(q[b, h:h + 1].double().cpu().numpy(), k[b, h // 2, t].cpu().numpy(), v[b, h // 2, t].cpu().numpy(), D ** -0.5)
                e = M.rounding(most[0], len(t), D)
                assert np.all(np.abs(out[b, h].double().cpu().numpy() - o[0]) <= (e + 2.0 ** -8) * a[0] + 2.0 ** -8 * np.abs(o[0]))
    tally, pos = torch.zeros(B, Hkv, Tcap, device="cuda"), torch.zeros(B, Hkv, Tcap, device="cuda", dtype=torch.int32)
    mark = torch.zeros(B, 2, device="cuda", dtype=torch.int32)
    rs.kv4_attn_decode(s, q, *four, length, D ** -0.5, None, tally, 1, out, lse, ws)
    rs.kv4_evict(s, *four, tally, pos, mark, length, 200, 4, 32, 0, ws)
    rs.kv4_page_meta(s, *four[:2], length, length, Tcap, meta)
    torch.cuda.synchronize()
    assert length.tolist() == [200] * B
    k2 = _values(*four[:2])[:, :, :200]
    assert torch.equal(k2, k.gather(2, pos[:, :, :200, None].long().expand(-1, -1, -1, D)))  # a row is its position's token
    for p in range(13):
        rows = k2[:, :, p * P:min(200, p * P + P)]
        assert torch.equal(meta[:, :, p].double(), torch.stack([rows.amin(2), rows.amax(2)], 2))


def test_a_list_of_no_pages_is_refused(rs):
    s = rs.make_shape(1, 2, 2, 64, 64, 16, torch.bfloat16)
    four = [torch.zeros(1, 2, 64, n, dtype=torch.uint8, device="cuda") for n in (32, 2, 32, 2)]
    length, q = torch.full((1,), 64, dtype=torch.int32, device="cuda"), torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7)
    ws = rs.Workspace(rs.kv4_attn_decode_workspace_bytes(s, 0, 0, False))
    with pytest.raises(rs.RatsparseError, match="no pages"):
        rs.kv4_attn_decode(s, q, *four, length, 0.1, torch.zeros(1, 2, 0, dtype=torch.int32, device="cuda"), None, 0, out, None, ws)
    torch.cuda.synchronize()
    assert bool((out == 7).all())
