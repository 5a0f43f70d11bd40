"""A cache in 4 bits: rows in, page bounds, rows out; against the format's definition in 64 bits, bit for bit."""
import numpy as np
import pytest
import torch

import kv4_model as M
from gpu_util import say, tdtype

pytestmark = pytest.mark.gpu


class Cache:
    """A 4-bit cache whose unused rows hold other bytes, NaN groups among them."""

    def __init__(self, rs, B, Hkv, D, Tcap, P, dtype, lens, seed=0):
        r = np.random.default_rng(seed)
        self.s = rs.make_shape(B, 2 * Hkv, Hkv, D, Tcap, P, tdtype(dtype))
        self.dt, self.lens = tdtype(dtype), list(lens)
        self.code = [r.integers(0, 256, (B, Hkv, Tcap, D // 2), dtype=np.uint8) for _ in "kv"]
        self.byte = [r.choice(np.array([2, 100, 120, 127, 130, 252, 255], dtype=np.uint8), (B, Hkv, Tcap, D // 32)) for _ in "kv"]
        self.dev = [torch.from_numpy(x.copy()).cuda() for pair in zip(self.code, self.byte) for x in pair]
        self.len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.meta = torch.full((B, Hkv, Tcap // P, 2, D), 3.0, device="cuda", dtype=self.dt)

    def rows(self, b, t0, t1):
        """Values of K and V rows, [Hkv, t, D]."""
        return [M.values(M.from_bytes(c[b, :, t0:t1]), f[b, :, t0:t1]) for c, f in zip(self.code, self.byte)]

    def check(self):
        got = [x.cpu().numpy() for x in self.dev]
        for name, x, y in zip(("k4", "k4_scale", "v4", "v4_scale"), got, (self.code[0], self.byte[0], self.code[1], self.byte[1])):
            assert np.array_equal(x, y), (name, np.argwhere(x != y)[:5])


def source(r, shape, dtype, wild=False):
    """Rows of every size of number; wild: also the ends of the range, infinities and NaN."""
    x = r.standard_normal(shape) * 2.0 ** r.integers(-20, 12, shape[:-1] + (1,))
    x = x * 2.0 ** np.repeat(r.integers(-3, 4, shape[:-1] + (shape[-1] // 32,)), 32, -1)
    ties = r.integers(-28, 29, shape) * 0.25  # ties of every kind, 7 and 5 among them
    x = np.where(r.random(shape[:-1] + (1,)) < 0.3, ties, x)
    x = np.where(r.random(shape) < 0.05, 0.0, x)
    x[r.random(shape[:-1]) < 0.05] = 0.0
    if wild:
        some = r.choice([3e38, -3.3e38, 2.6e38, 1e-37, 2e-38, -1.2e-38, 9e-39, -4e-39, 1e-40], shape)
        x = np.where(r.random(shape[:-1] + (1,)) < 0.4, some, x)
        odd = r.choice([np.inf, -np.inf, np.nan], shape)
        x = np.where(r.random(shape) < 0.003, odd, x)
    with np.errstate(over="ignore"):
        t = torch.from_numpy(x.astype(np.float32))
    return t.to(tdtype(dtype))


def bounds_of(k, dt):
    """Smallest and largest value of each channel, [Hkv, 2, D]; NaN passed over."""
    lo, hi = np.where(np.isnan(k), np.inf, k).min(1), np.where(np.isnan(k), -np.inf, k).max(1)
    return torch.from_numpy(np.stack([lo, hi], 1)).to(torch.float32).to(dt)


def touched(P, L, n):
    return range((L - n) // P, (L - 1) // P + 1) if n else range(0)


CASES = [  # B, Hkv, D, Tcap, P, dtype, lengths, new, T_new, rows of the source, first of them
    (3, 2, 64, 64, 16, "bf16", [1, 17, 64], None, 1, 1, 0),
    (3, 2, 128, 64, 16, "f32", [1, 0, 64], None, 1, 16, 5),
    (4, 1, 128, 512, 512, "bf16", [512, 511, 3, 200], [1, 0, 3, 7], 7, 7, 0),
    (2, 3, 64, 1024, 64, "f32", [1000, 777], [333, 40], 333, 400, 60),
    (5, 2, 128, 320, 32, "bf16", [320, 40, 5, 400, -3], [100, 41, -2, 500, 1], 100, 100, 0),
    (1, 2, 128, 2048, 16, "bf16", [2003], None, 2003, 2048, 0),
    (2, 5, 64, 96, 16, "bf16", [77, 96], [77, 5], 96, 96, 0),
    # calls long enough to go as a stream
    (8, 32, 64, 320, 16, "bf16", [320, 319, 300, 17, 0, 1, 100, 257], [299, 16, 300, 17, 5, 1, 77, 30], 300, 300, 0),
    (4, 24, 128, 768, 32, "f32", [768, 700, 33, 500], None, 700, 768, 40),
    (4, 32, 128, 640, 32, "bf16", [640, 639, 555, 64], [640, 1, 33, 64], 640, 640, 0),
    (64, 40, 64, 64, 64, "f32", [(5 * i) % 65 for i in range(64)], [(7 * i) % 41 for i in range(64)], 40, 40, 0),
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("meta", [True, False])
@pytest.mark.parametrize("wild", [False, True])
def test_append(rs, case, meta, wild):
    B, Hkv, D, Tcap, P, dtype, lens, new, T, T_src, t_src = CASES[case]
    say("kv4 append", case, meta, wild)
    r = np.random.default_rng(100 * case + wild)
    c = Cache(rs, B, Hkv, D, Tcap, P, dtype, lens, seed=case)
    k, v = (source(r, (B, Hkv, T_src, D), dtype, wild) for _ in "kv")
    n_new = torch.tensor(new, dtype=torch.int32, device="cuda") if new else None
    want_meta = c.meta.clone().cpu()
    for b in range(B):
        L = min(max(lens[b], 0), Tcap)
        n = min(max(new[b] if new else T, 0), T)
        n = n if n <= L else 0
        for i, x in enumerate((k, v)):
            code, byte = M.pack(x[b, :, t_src:t_src + n].double().numpy())
            c.code[i][b, :, L - n:L], c.byte[i][b, :, L - n:L] = M.to_bytes(code), byte
        for p in touched(P, L, n) if meta else ():
            want_meta[b, :, p] = bounds_of(c.rows(b, p * P, min(L, p * P + P))[0], c.dt)
    for _ in range(2):  # twice the same: the same bytes
        rs.kv4_append(c.s, k.cuda(), v.cuda(), t_src, c.len, n_new, T, *c.dev, c.meta if meta else None)
    torch.cuda.synchronize()
    c.check()
    assert torch.equal(c.meta.cpu(), want_meta)
    if meta:  # the bounds by themselves
        c.meta.fill_(3.0)
        rs.kv4_page_meta(c.s, c.dev[0], c.dev[1], c.len, n_new, T, c.meta)
        torch.cuda.synchronize()
        assert torch.equal(c.meta.cpu(), want_meta)


def test_bounds_of_all_pages(rs):
    c = Cache(rs, 3, 2, 128, 256, 32, "bf16", [200, 0, 256], seed=9)
    rs.kv4_page_meta(c.s, c.dev[0], c.dev[1], c.len, c.len, 256, c.meta)
    want = torch.full_like(c.meta, 3.0).cpu()
    for b, L in enumerate(c.lens):
        for p in touched(32, L, L):
            want[b, :, p] = bounds_of(c.rows(b, p * 32, min(L, p * 32 + 32))[0], c.dt)
    assert torch.equal(c.meta.cpu(), want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t0,T", [(0, 1), (0, 200), (5, 33), (-1, 1), (-33, 33), (-190, 7), (150, 60)])
def test_fetch(rs, D, dtype, t0, T):
    lens = [1, 37, 0, 192, 500]
    c = Cache(rs, 5, 3, D, 192, 16, dtype, lens, seed=D + T)
    k, v = (torch.full((5, 3, T, D), 7.0, device="cuda", dtype=c.dt) for _ in "kv")
    rs.kv4_fetch(c.s, *c.dev, c.len, t0, T, k, v)
    for b in range(5):
        L = min(lens[b], 192)
        rows = c.rows(b, 0, L)
        for got, x in zip((k, v), rows):
            want = np.full((3, T, D), 7.0)
            for i in range(T):
                t = (L + t0 if t0 < 0 else t0) + i
                if 0 <= t < L:
                    want[:, i] = x[:, t]
            np.testing.assert_array_equal(got[b].double().cpu().numpy(), torch.from_numpy(want).to(c.dt).double().numpy())


def test_append_of_a_scan_and_captured(rs):
    """Tokens go through the recurrence into a staging buffer and from there into the 4-bit cache, step by step in a replayed graph; the same calls by hand
    give the same bytes, bounds included, and the rows are the rounded states."""
    B, Hkv, D, P, Tcap, T0, steps = 3, 2, 128, 16, 128, 21, 40
    g = torch.Generator(device="cuda").manual_seed(5)
    s1 = rs.make_shape(B, Hkv, Hkv, D, 16, 16, torch.bfloat16)  # the staging buffer's
    rand = lambda *n: torch.randn(*n, device="cuda", generator=g)
    k0, v0 = (rand(B, Hkv, T0, D).bfloat16() for _ in "kv")
    g0 = torch.sigmoid(rand(B, Hkv, T0, D) * 0.5 + 3)
    toks = [[rand(B, Hkv, 1, D).bfloat16(), rand(B, Hkv, 1, D).bfloat16(), torch.sigmoid(rand(B, Hkv, 1, D) * 0.5 + 3)] for _ in range(steps)]

    class Run:
        def __init__(self):
            self.c = Cache(rs, B, Hkv, D, Tcap, P, "bf16", [T0] * B, seed=1)
            self.sk, self.sv = (torch.zeros(B, Hkv, D, device="cuda") for _ in "kv")
            full = [torch.zeros(B, Hkv, 32, D, device="cuda", dtype=torch.bfloat16) for _ in "kv"]
            s0 = rs.make_shape(B, Hkv, Hkv, D, 32, 16, torch.bfloat16)
            rs.rat_scan(s0, k0, v0, g0, self.sk, self.sv, *full, 0, T0, rs.Workspace(rs.rat_scan_workspace_bytes(s0, T0)))
            rs.kv4_append(self.c.s, *full, 0, self.c.len, None, T0, *self.c.dev, self.c.meta)
            self.stage = [torch.zeros(B, Hkv, 16, D, device="cuda", dtype=torch.bfloat16) for _ in "kv"]
            self.full = [[x[:, :, :T0].clone()] for x in full]
            self.tok = [x.clone() for x in toks[0]]

        def scan(self, i):
            for a, b in zip(self.tok, toks[i]):
                a.copy_(b)
            rs.rat_scan(s1, *self.tok, self.sk, self.sv, *self.stage, 0, 1)
            for f, x in zip(self.full, self.stage):
                f.append(x[:, :, :1].clone())

        def append(self):
            self.c.len.add_(1)
            rs.kv4_append(self.c.s, *self.stage, 0, self.c.len, None, 1, *self.c.dev, self.c.meta)

    a, b = Run(), Run()
    for i in range(steps):
        a.scan(i)
        a.append()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.append()
    for i in range(steps):
        b.scan(i)
        graph.replay()
        torch.cuda.synchronize()
    for x, y in zip(a.c.dev + [a.c.meta, a.c.len], b.c.dev + [b.c.meta, b.c.len]):
        assert torch.equal(x, y)
    for i in range(2):
        rows = torch.cat(a.full[i], 2).double().cpu().numpy()
        code, byte = M.pack(rows)
        n = T0 + steps
        a.c.code[i][:, :, :n], a.c.byte[i][:, :, :n] = M.to_bytes(code), byte
    a.c.check()


def test_rows_far_into_a_long_cache(rs):
    """Offsets past 2^32 bytes: two heads of 70 million rows of 128 channels, 9 GB of codes a tensor."""
    Tcap, D = 70_000_000, 128  # 4.5 GB of codes a head
    s = rs.make_shape(1, 2, 2, D, Tcap // 16 * 16, 16, torch.float32)
    Tcap = s.Tcap
    dev = [torch.zeros(1, 2, Tcap, n, dtype=torch.uint8, device="cuda") for n in (D // 2, D // 32, D // 2, D // 32)]
    L, T = Tcap - 5, 19
    length = torch.tensor([L], dtype=torch.int32, device="cuda")
    r = np.random.default_rng(3)
    k, v = (source(r, (1, 2, T, D), "f32") for _ in "kv")
    rs.kv4_append(s, k.cuda(), v.cuda(), 0, length, None, T, *dev, None)
    out = [torch.zeros(1, 2, T, D, device="cuda") for _ in "kv"]
    rs.kv4_fetch(s, *dev, length, -T, T, *out)
    for x, y, codes, byte in zip((k, v), out, dev[0::2], dev[1::2]):
        want = M.values(*M.pack(x.double().numpy()))
        np.testing.assert_array_equal(y.double().cpu().numpy(), want)
        assert int(codes[:, :, L:].max()) == 0 and int(byte[:, :, L:].max()) == 0 and int(byte[:, :, L - T - 64:L - T].max()) == 0


@pytest.mark.parametrize("D,P,dtype", [(64, 16, "bf16"), (128, 16, "f32"), (64, 64, "f32")])
def test_a_stream_of_many_pages_a_wave(rs, D, P, dtype):
    """A call so long that a wave takes several pages in turn stores what many short calls store, bounds included."""
    B, Hkv, Tcap, T, T0 = 16, 64, 1280, 1117, 7
    lens = [T0 + T - (5 * b) % 40 for b in range(B)]
    new = [min(n, T) - (3 * b) % 50 for b, n in enumerate(lens)]
    g = torch.Generator(device="cuda").manual_seed(D)
    k, v = (torch.randn(B, Hkv, T, D, device="cuda", generator=g).to(tdtype(dtype)) for _ in "kv")
    a, b = (Cache(rs, B, Hkv, D, Tcap, P, dtype, lens, seed=1) for _ in "ab")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    rs.kv4_append(a.s, k, v, 0, a.len, ints(new), T, *a.dev, a.meta)
    for i in range(0, T, 32):
        n = min(32, T - i)
        some = [max(0, min(n, m - i)) for m in new]
        ln = ints([x - m + i + s for x, m, s in zip(lens, new, some)])
        rs.kv4_append(b.s, k, v, i, ln, ints(some), n, *b.dev, b.meta)
    torch.cuda.synchronize()
    for x, y in zip(a.dev + [a.meta], b.dev + [b.meta]):
        assert torch.equal(x, y)
    a.meta.fill_(3.0)
    rs.kv4_page_meta(a.s, a.dev[0], a.dev[1], a.len, ints(new), T, a.meta)
    assert torch.equal(a.meta, b.meta)


def test_bounds_of_no_pages_are_refused(rs):
    s = rs.make_shape(1, 2, 2, 64, 32, 64, torch.bfloat16)  # a page is longer than the cache
    four = [torch.full((1, 2, 32, n), 7, dtype=torch.uint8, device="cuda") for n in (32, 2, 32, 2)]
    rows, length = torch.ones(1, 2, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.full((1,), 4, dtype=torch.int32, device="cuda")
    with pytest.raises(rs.RatsparseError, match="no pages"):
        rs.kv4_append(s, rows, rows, 0, length, None, 4, *four, torch.zeros(1, 2, 0, 2, 64, dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
    assert all(bool((x == 7).all()) for x in four)
    rs.kv4_append(s, rows, rows, 0, length, None, 4, *four, None)
    torch.cuda.synchronize()
    assert bool((four[0][:, :, :4] != 7).all())
