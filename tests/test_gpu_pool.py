"""Pages of a pool: who holds which, against a model in plain Python (every number equal); the copies that follow; the append
through the table against the recurrence in 64 bits."""
import random

import numpy as np
import pytest
import torch

from gpu_util import say, tdtype
from pool_model import Pool, recurrence

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Device:
    """A pool on the device beside its model."""

    def __init__(self, rs, N, S, M, P):
        self.rs, self.m, self.p = rs, Pool(N, S, M, P), rs.make_pool(N, S, M, P)
        self.table = torch.full((S, M), -1, dtype=torch.int32, device="cuda")
        self.len, self.refs = ints([0] * S), ints([0] * N)
        self.ws = rs.Workspace(rs.page_pool_workspace_bytes(self.p))

    def state(self):
        return self.p, self.table, self.len, self.refs

    def check(self, what, taken=True):
        torch.cuda.synchronize()
        if taken:
            self.ws.async_status()
        else:
            with pytest.raises(self.rs.RatsparseError, match="status 7"):
                self.ws.async_status()
            self.ws.async_status()  # reported once
        assert self.table.tolist() == self.m.table, what
        assert self.len.tolist() == self.m.len, what
        assert self.refs.tolist() == self.m.refs, what

    def reserve(self, seq, want):
        granted = ints([7] * len(seq))
        self.rs.page_pool_reserve(*self.state(), ints(seq), ints(want), 5, granted, self.ws)
        taken = self.m.reserve(seq, want)
        self.check(("reserve", seq, want), taken)
        assert granted.tolist() == (want if taken else [0] * len(seq))
        return taken

    def fork(self, src, dst):
        pairs, carry = ints([[5, 5]] * len(src)), ints([[5, 5]] * len(src))
        self.rs.page_pool_fork(*self.state(), ints(src), ints(dst), pairs, carry, self.ws)
        taken, mp, mc = self.m.fork(src, dst)
        self.check(("fork", src, dst), taken)
        assert pairs.tolist() == mp and carry.tolist() == mc
        return taken

    def free(self, seq):
        self.rs.page_pool_free(*self.state(), ints(seq), self.ws)
        taken = self.m.free(seq)
        self.check(("free", seq), taken)
        return taken

    def compact(self):
        pairs, n = ints([[5, 5]] * max(1, self.m.N // 2)), ints([9])
        self.rs.page_pool_compact(*self.state(), pairs, n, self.ws)
        moves = self.m.compact()
        self.check("compact")
        assert n.tolist() == [len(moves)]
        if self.m.N > 1:
            assert pairs.tolist() == moves + [[-1, -1]] * (self.m.N // 2 - len(moves))
        return moves

    def share(self, seq, least):
        out = ints([[5, 5, 5]] * len(seq))
        self.rs.page_pool_share(self.p, self.table, self.len, ints(seq), least, out)
        assert out.tolist() == self.m.share(seq, least)


@pytest.mark.parametrize("N,S,M,P,seed", [(1, 1, 1, 16, 0), (37, 5, 9, 16, 1), (400, 40, 30, 32, 2), (16400, 9, 8000, 16, 3),
                                          (40003, 3000, 17, 512, 4)])
def test_a_pool_s_life(rs, N, S, M, P, seed):
    """Calls of every kind in no order, some of which cannot be taken."""
    say("pool", N, S, M, P)
    d, r = Device(rs, N, S, M, P), random.Random(seed)
    seen = {}
    for _ in range(60 if N < 1000 else 25):
        kind = r.choice(["reserve", "reserve", "fork", "free", "compact", "share"])
        some = r.sample(range(S), r.randint(1, min(S, r.choice([3, S]))))
        if kind == "reserve":
            top = r.choice([1, P, M * P // 4 + 1, M * P])
            taken = d.reserve(some, [r.choice([0, 1, r.randint(0, top)]) for _ in some])
        elif kind == "fork":
            empty = [s for s in some if d.m.len[s] == 0] or some
            taken = d.fork([r.randrange(S) for _ in empty], empty)
        elif kind == "free":
            taken = d.free(some[:max(1, len(some) // 2)])
        elif kind == "compact":
            taken = len(d.compact()) > 0
        else:
            taken = d.share([r.choice(some) for _ in range(r.randint(1, 40))], r.randint(1, 3))
        seen[kind, bool(taken)] = seen.get((kind, bool(taken)), 0) + 1
    say("  ", seen)


def test_refused_as_a_whole(rs):
    d = Device(rs, 10, 4, 6, 16)
    assert d.reserve([2, 0], [40, 17])
    for seq, want in (([1, 1], [1, 1]), ([-1], [1]), ([4], [1]), ([1], [-1]), ([0], [80]), ([1, 3], [1, 80]), ([2 ** 31 - 1], [1]),
                      ([1], [2 ** 31 - 1])):
        assert not d.reserve(seq, want), (seq, want)
    for src, dst in (([2], [0]), ([2, 2], [1, 1]), ([2], [2]), ([9], [1]), ([2], [4]), ([1], [1]), ([2, 3], [3, 1])):
        assert not d.fork(src, dst), (src, dst)
    for seq in ([0, 0], [0, 4], [-1]):
        assert not d.free(seq), seq
    assert d.reserve([1], [80])  # the pool is full: no page for a fork's partial one
    assert not d.fork([0], [3]) and d.free([1, 3])
    assert d.fork([3], [1]) and d.m.len[1] == 0  # an empty one
    assert d.reserve([0, 1], [0, 0])


@pytest.mark.parametrize("n,M", [(3, 700), (200, 5), (128, 64), (60, 300), (17, 257)])
def test_long_lists_and_wide_tables(rs, n, M):
    d, r = Device(rs, n * 3 + M + 9, 2 * n + 1, M, 16), random.Random(n)
    assert d.reserve([0], [16 * M - 20])
    assert d.fork([0] * n, list(range(1, n + 1)))
    assert d.reserve(list(range(1, n + 1)), [r.randint(0, 20) for _ in range(n)])
    d.share(list(range(n + 1)), 1)
    some = r.sample(range(n + 1), n)
    assert d.fork(some, list(range(n + 1, 2 * n + 1)))
    d.share([s for i in range(n) for s in (some[i], n + 1 + i)], 2)
    assert d.free(r.sample(range(2 * n + 1), n))
    d.compact()


def test_share(rs):
    d = Device(rs, 300, 12, 250, 16)
    assert d.reserve([0, 1, 2], [3213, 16 * 5, 7])
    assert d.fork([0, 0, 0, 1, 1, 2], [3, 4, 5, 6, 7, 8])
    assert d.reserve([4, 5, 6], [30, 1, 17])
    for seq in ([0], [0, 3, 4, 5], [3, 6, 7, 1, 4, 5], [2, 8], [6, 7, 3, 4], [0, 0, 3], [-1, 0, 3, 12], [10, 11, 0, 4] * 100):
        for least in (1, 6, 200, 201):
            d.share(seq, least)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,P,Hkv", [(64, 16, 3), (128, 64, 2), (128, 512, 1)])
def test_page_copy(rs, dtype, D, P, Hkv):
    """Between two pools of different size, with bounds and without; pairs to pass over; a count on the device."""
    dt, gen = tdtype(dtype), torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *n: torch.randn(*n, device="cuda", generator=gen).to(dt)
    N, M = 9, 23
    s, o = rs.make_shape(1, Hkv, Hkv, D, N * P, P, dt), rs.make_shape(5, Hkv, Hkv, D, M * P, P, dt)
    src = [rnd(Hkv, N * P, D), rnd(Hkv, N * P, D), rnd(Hkv, N, 2, D)]
    pairs = [[3, 20], [-1, 2], [8, 0], [1, -1], [9, 4], [0, 23], [2, 22], [7, 7], [2 ** 31 - 1, 1], [5, 11]]
    for count in (None, 0, 3, 10, 99, -4):
        for bounds in (True, False):
            dst = [rnd(Hkv, M * P, D), rnd(Hkv, M * P, D), rnd(Hkv, M, 2, D)]
            want = [x.clone() for x in dst]
            for a, b in pairs[:len(pairs) if count is None else max(0, count)]:
                if 0 <= a < N and 0 <= b < M:
                    for w, x, n in zip(want, src, (P, P, 2)) if bounds else list(zip(want, src, (P, P, 2)))[:2]:
                        w.view(Hkv, M, n, D)[:, b] = x.view(Hkv, N, n, D)[:, a]
            rs.page_copy(s, *(src if bounds else src[:2] + [None]), o, *(dst if bounds else dst[:2] + [None]), ints(pairs),
                         None if count is None else ints([count]))
            assert all(torch.equal(x, y) for x, y in zip(dst, want)), (count, bounds)


def test_more_pages_than_workgroups(rs):
    """Within one pool, every other page to the page after it."""
    dt, N, P, D, Hkv = torch.bfloat16, 3000, 16, 64, 4
    s = rs.make_shape(1, Hkv, Hkv, D, N * P, P, dt)
    k, v = (torch.randn(Hkv, N * P, D, device="cuda").to(dt) for _ in range(2))
    wk, wv = k.clone(), v.clone()
    for x in (wk, wv):
        y = x.view(Hkv, N, P, D)
        y[:, 1::2] = y[:, ::2]
    rs.page_copy(s, k, v, None, s, k, v, None, ints([[2 * i, 2 * i + 1] for i in range(N // 2)]), None)
    assert torch.equal(k, wk) and torch.equal(v, wv)


@pytest.mark.parametrize("Hkv,D", [(1, 64), (5, 128), (40, 128)])
def test_state_copy(rs, Hkv, D):
    s = rs.make_shape(1, Hkv, Hkv, D, 16, 16, torch.float32)
    a, b = torch.randn(6, Hkv, D, device="cuda"), torch.randn(6, Hkv, D, device="cuda")
    wa, wb = a.clone(), b.clone()
    for w in (wa, wb):
        w[4], w[0] = w[1], w[5]
    rs.rat_state_copy(s, a, b, ints([[1, 4], [-1, -1], [5, 0], [6, 2], [2, 6]]))
    assert torch.equal(a, wa) and torch.equal(b, wb)


APPEND = [
    # B, Hkv, D, P, T_new, lengths before, counts (None: T_new for all)
    (1, 1, 64, 16, 1, [0], None),
    (3, 2, 128, 16, 1, [15, 16, 17], None),
    (4, 3, 64, 32, 7, [0, 31, 40, 5], [7, 0, 1, 3]),
    (2, 2, 128, 16, 100, [3, 160], [100, 99]),
    (2, 1, 64, 512, 700, [100, 0], None),
    (5, 2, 128, 64, 33, [64, 63, 1, 130, 0], [33, 2, 33, 9, 40]),  # (counts above T_new are cut)
    (8, 32, 128, 32, 40, list(range(10, 18)), None),               # many heads
    (16, 32, 128, 64, 70, list(range(50, 66)), [70 - i for i in range(16)]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append(rs, case, dtype):
    B, Hkv, D, P, T, before, counts = APPEND[case]
    say("append", case, dtype)
    dt, S, r = tdtype(dtype), B + 2, np.random.default_rng(case)
    M = -(-(max(before) + T) // P) + 1
    d = Device(rs, S * M, S, M, P)
    seq = r.permutation(S)[:B].tolist()
    for i in r.permutation(B):  # (pages in no order)
        assert d.reserve([seq[i]], [before[i]])
    s = rs.make_shape(B, Hkv, Hkv, D, S * M * P, P, dt)
    rnd = lambda *n: torch.from_numpy(r.standard_normal(n).astype(np.float32)).cuda()
    k, v = rnd(B, Hkv, T, D).to(dt), rnd(B, Hkv, T, D).to(dt)
    g = torch.sigmoid(rnd(B, Hkv, T, D) + 2.5)
    cut = [min(T, c) for c in counts] if counts else [T] * B
    for i in range(B):  # what lies past the counts is not read
        for x in (k, v, g):
            x[i, :, cut[i]:] = float("nan")
    sk, sv = rnd(S, Hkv, D), rnd(S, Hkv, D)
    kp, vp = rnd(Hkv, S * M * P, D).to(dt), rnd(Hkv, S * M * P, D).to(dt)
    meta = rnd(Hkv, S * M, 2, D).to(dt)
    olds = [x.clone() for x in (sk, sv, kp, vp, meta)]
    assert d.reserve(seq, cut)
    rs.rat_append_paged(s, d.p, k, v, g, sk, sv, kp, vp, meta, d.table, d.len, ints(seq), ints(counts) if counts else None, T)
    torch.cuda.synchronize()
    eps = 2.0 ** -24
    touched = {}
    for x, state, pool, old_state, old_pool in ((k, sk, kp, olds[0], olds[2]), (v, sv, vp, olds[1], olds[3])):
        want_pool = old_pool.clone()
        for i in range(B):
            if cut[i] == 0:
                continue
            hx, hg = (y[i, :, :cut[i]].float().cpu().numpy().swapaxes(0, 1) for y in (x, g))
            every = recurrence(old_state[seq[i]].cpu().numpy(), hx, hg)  # [T, Hkv, D]
            # three roundings of at most half a step a token, of values no larger than what went in; later gates shrink them
            tol = 3 * cut[i] * eps * max(np.abs(hx).max(), float(old_state[seq[i]].abs().max()))
            assert np.abs(state[seq[i]].double().cpu().numpy() - every[-1]).max() <= tol
            rows = d.m.rows(seq[i])[-cut[i]:]
            stored = pool[:, rows].double().cpu().numpy().swapaxes(0, 1)
            half = 2.0 ** -8 if dtype == "bf16" else 0.0
            assert (np.abs(stored - every) <= half * (np.abs(every) + tol) + tol).all()
            want_pool[:, rows] = pool[:, rows]
            touched[i] = rows
        assert torch.equal(pool, want_pool)  # nothing else is written
        others = [i for i in range(S) if i not in seq or cut[seq.index(i)] == 0]
        assert torch.equal(state[others], old_state[others])
    want_meta = olds[4].clone()
    for i in touched:
        L, row = d.m.len[seq[i]], d.m.table[seq[i]]
        for j in range((L - cut[i]) // P, (L - 1) // P + 1):
            rows = kp[:, row[j] * P:row[j] * P + min(P, L - j * P)]
            want_meta[:, row[j], 0], want_meta[:, row[j], 1] = rows.amin(1), rows.amax(1)
    assert torch.equal(meta, want_meta)
    # the same without bounds; the carries as bits
    again = [x.clone() for x in olds[:4]]
    rs.rat_append_paged(s, d.p, k, v, g, *again, None, d.table, d.len, ints(seq), ints(cut), T)
    assert all(torch.equal(x, y) for x, y in zip(again, (sk, sv, kp, vp)))


def test_append_passes_over_what_it_cannot_take(rs):
    """A sequence out of range, listed twice, too short; a table entry that names no page."""
    dt, P, S, M, N, Hkv, D, T = torch.float32, 16, 4, 3, 12, 2, 64, 4
    d = Device(rs, N, S, M, P)
    assert d.reserve([0, 1, 2], [20, 18, 3])
    d.table[1, 1] = N  # no such page
    seq = [0, 7, 0, -1, 2, 1]
    s = rs.make_shape(len(seq), Hkv, Hkv, D, N * P, P, dt)
    k, v, g = torch.ones(6, Hkv, T, D, device="cuda"), torch.ones(6, Hkv, T, D, device="cuda"), torch.full((6, Hkv, T, D), 0.5, device="cuda")
    sk, sv = torch.zeros(S, Hkv, D, device="cuda"), torch.zeros(S, Hkv, D, device="cuda")
    kp, vp, meta = (torch.zeros(*n, device="cuda") for n in ((Hkv, N * P, D), (Hkv, N * P, D), (Hkv, N, 2, D)))
    rs.rat_append_paged(s, d.p, k, v, g, sk, sv, kp, vp, meta, d.table, d.len, ints(seq), None, T)
    want = torch.tensor([0.5, 0.75, 0.875, 0.9375], device="cuda")
    assert sk[0].eq(0.9375).all() and sk[1].eq(0.9375).all() and not sk[2:].any()
    assert torch.equal(kp[0, d.m.rows(0)[-4:], 5], want)
    assert torch.equal(kp[0, d.m.rows(1, 16)[-2:], 5], want[:2])  # positions 14, 15; 16 and 17 have no page
    written = set(d.m.rows(0)[-4:].tolist()) | set(d.m.rows(1, 16)[-2:].tolist())
    assert set(kp[1, :, 0].nonzero()[:, 0].tolist()) == written and set(vp[1, :, 0].nonzero()[:, 0].tolist()) == written


def test_as_the_contiguous_append_does_it(rs):
    """The same tokens into a contiguous cache by rat_scan, one by one: equal bits."""
    dt, P, Hkv, D, T0, steps, B = torch.bfloat16, 16, 2, 128, 30, 5, 2
    M = 4
    d = Device(rs, B * M, B, M, P)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *n: torch.randn(*n, device="cuda", generator=gen)
    s = rs.make_shape(B, Hkv, Hkv, D, M * P, P, dt)
    kc, vc, meta = torch.zeros(B, Hkv, M * P, D, device="cuda", dtype=dt), torch.zeros(B, Hkv, M * P, D, device="cuda", dtype=dt), \
        torch.zeros(B, Hkv, M, 2, D, device="cuda", dtype=dt)
    sk, sv = torch.zeros(B, Hkv, D, device="cuda"), torch.zeros(B, Hkv, D, device="cuda")
    ws = rs.Workspace(rs.rat_scan_workspace_bytes(s, T0))
    rs.rat_scan(s, rnd(B, Hkv, T0, D).to(dt), rnd(B, Hkv, T0, D).to(dt), torch.sigmoid(rnd(B, Hkv, T0, D) + 4), sk, sv, kc, vc, 0, T0, ws, meta)
    # the prompts' rows into pages
    o = rs.make_shape(B, Hkv, Hkv, D, B * M * P, P, dt)
    kp, vp, pm = torch.zeros(Hkv, B * M * P, D, device="cuda", dtype=dt), torch.zeros(Hkv, B * M * P, D, device="cuda", dtype=dt), \
        torch.zeros(Hkv, B * M, 2, D, device="cuda", dtype=dt)
    assert d.reserve([1, 0], [T0, T0])
    for b in range(B):
        rs.page_copy(s, kc[b], vc[b], meta[b], o, kp, vp, pm, ints([[j, d.m.table[b][j]] for j in range(2)]), None)
    pk, pv = sk.clone(), sv.clone()
    for t in range(steps):
        k, v, g = rnd(B, Hkv, 1, D).to(dt), rnd(B, Hkv, 1, D).to(dt), torch.sigmoid(rnd(B, Hkv, 1, D) + 4)
        rs.rat_scan(s, k, v, g, sk, sv, kc, vc, T0 + t, 1, ws, meta)
        assert d.reserve([0, 1], [1, 1])
        rs.rat_append_paged(o, d.p, k, v, g, pk, pv, kp, vp, pm, d.table, d.len, ints([0, 1]), None, 1)
    assert torch.equal(pk, sk) and torch.equal(pv, sv)
    for b in range(B):
        rows = torch.from_numpy(d.m.rows(b)).cuda()
        assert torch.equal(kp[:, rows], kc[b, :, :T0 + steps]) and torch.equal(vp[:, rows], vc[b, :, :T0 + steps])
        assert torch.equal(pm[:, d.m.table[b][:3]], meta[b, :, :3])


def test_plain_and_other_arguments_make_the_same_call(rs):
    """Through native.cpp, and (a subclass of torch.Tensor is not of the plain type) through ctypes."""
    class Other(torch.Tensor):
        pass
    for kind in (lambda x: x, lambda x: x.as_subclass(Other)):
        d = Device(rs, 20, 4, 5, 16)
        granted = ints([9, 9])
        rs.page_pool_reserve(d.p, kind(d.table), d.len, d.refs, ints([3, 1]), None, 20, granted, d.ws)
        assert d.m.reserve([3, 1], [20, 20]) and granted.tolist() == [20, 20]
        d.check("reserve")
        pairs, carry, share = ints([[0, 0]]), ints([[0, 0]]), ints([[9] * 3] * 2)
        rs.page_pool_fork(d.p, d.table, kind(d.len), d.refs, ints([3]), ints([0]), pairs, carry, d.ws)
        d.m.fork([3], [0])
        d.check("fork")
        rs.page_pool_share(d.p, d.table, d.len, kind(ints([3, 0])), 1, share)
        assert share.tolist() == d.m.share([3, 0], 1) == [[0, 2, 1]] * 2
        rs.page_pool_free(d.p, d.table, d.len, d.refs, kind(ints([3])), d.ws)
        d.m.free([3])
        d.check("free")
        moves, n = ints([[0, 0]] * 10), ints([0])
        rs.page_pool_compact(d.p, d.table, d.len, kind(d.refs), moves, n, d.ws)
        assert moves[:n.item()].tolist() == d.m.compact()
        d.check("compact")
        s = rs.make_shape(1, 1, 1, 64, 320, 16, torch.float32)
        k, v, sk = torch.randn(1, 320, 64, device="cuda"), torch.randn(1, 320, 64, device="cuda"), torch.randn(4, 1, 64, device="cuda")
        want, ws = k.clone(), sk.clone()
        want[:, 32:48], ws[2] = k[:, 16:32], sk[1]
        rs.page_copy(s, k, kind(v), None, s, k, v, None, ints([[1, 2]]), None)
        rs.rat_state_copy(s, kind(sk), sk.clone(), ints([[1, 2]]))
        assert torch.equal(k, want) and torch.equal(sk, ws)
        x = torch.ones(1, 1, 1, 64, device="cuda")
        rs.rat_append_paged(s, d.p, kind(x), x, torch.zeros_like(x), sk, sk.clone(), k, v, None, d.table, d.len, ints([1]), None, 1)
        assert k[0, d.m.rows(1)[-1]].eq(1).all() and sk[1].eq(1).all()
        out, lse = torch.zeros(1, 1, 1, 64, device="cuda"), torch.zeros(1, 1, 1, device="cuda")
        rs.attn_paged(s, d.p, kind(x), k, v, d.table, d.len, ints([1]), None, 1, None, 0.0, out, lse, rs.Workspace(rs.attn_paged_workspace_bytes(s, d.p, 1)))
        assert (out[0, 0, 0] - v[0, d.m.rows(1)].mean(0)).abs().max() < 1e-5
        for bad in (lambda: rs.page_pool_free(d.p, d.table[:2], d.len, d.refs, ints([1]), d.ws),
                    lambda: rs.page_pool_free(d.p, d.table.long(), d.len, d.refs, ints([1]), d.ws),
                    lambda: rs.attn_paged(s, d.p, x.to(torch.bfloat16), k, v, d.table, d.len, ints([1]), None, 1, None, 0.0, out, lse, d.ws)):
            with pytest.raises(rs.RatsparseError):
                bad()


@pytest.mark.parametrize("N", [(1 << 21) - 2, (1 << 21) - 1, 1 << 22])
@pytest.mark.parametrize("S,M,n,want", [(128, 1 << 24, 128, 16 << 24),                # 2^31 pages together: negative as 32 bits
                                        (256, 1 << 24, 256, 16 << 24),                # 2^32: nothing
                                        (1024, (1 << 22) + 1, 1024, 16 * ((1 << 22) + 1)),  # 2^32 + 1024: few
                                        (1024, 1 << 21, 1024, 16 << 21),              # each no more than there may be pages
                                        (1100, 1 << 22, 1100, (16 << 22) - 15)])      # over two turns of a workgroup's threads
def test_more_pages_asked_for_than_32_bits_count(rs, N, S, M, n, want):
    """Refused as a whole, like any call that asks for more than there is.  (The table is not looked at: it may hold anything.)"""
    p = rs.make_pool(N, S, M, 16)
    table = torch.empty(S, M, dtype=torch.int32, device="cuda")
    length, refs = ints([0] * S), torch.zeros(N, dtype=torch.int32, device="cuda")
    ws = rs.Workspace(rs.page_pool_workspace_bytes(p))
    granted, seq = ints([7] * n), torch.arange(n, dtype=torch.int32, device="cuda")
    for each in (None, torch.full((n,), want, dtype=torch.int32, device="cuda")):
        rs.page_pool_reserve(p, table, length, refs, seq, each, want, granted, ws)
        with pytest.raises(rs.RatsparseError, match="status 7"):
            ws.async_status()
        assert not length.any() and not refs.any() and not granted.any()
        granted.fill_(7)
    del table  # (up to 18 GB)
    torch.cuda.empty_cache()


def test_all_pages_at_once(rs):
    """The most that can be given, over more than one turn of the threads."""
    N, S = 5000, 1030
    d = Device(rs, N, S, 5, 16)
    want = [80] * 900 + [0] * 30 + [60, 64] * 50
    assert sum(-(-w // 16) for w in want) == 4900
    assert d.reserve(list(range(S)), want)
    assert not d.reserve(list(range(900, 921)), [80] * 20 + [1])
    assert d.reserve(list(range(900, 920)), [80] * 20) and d.m.free_pages() == []


def test_room_in_a_pool_of_many_pages(rs):
    """Sums formed in two halves, of needs on both sides of 2^16: every sequence gets the next pages in order."""
    N, S, M = (1 << 21) + 77, 40, 70000
    p = rs.make_pool(N, S, M, 16)
    table, length, refs = torch.full((S, M), -1, dtype=torch.int32, device="cuda"), ints([0] * S), torch.zeros(N, dtype=torch.int32, device="cuda")
    ws = rs.Workspace(rs.page_pool_workspace_bytes(p))
    need = [65535, 65536, 65537, 1, 0, 69999] + [50001 + 17 * i for i in range(34)]
    want = [max(0, 16 * n - 3) for n in need]
    granted, seq = ints([0] * S), list(reversed(range(S)))
    rs.page_pool_reserve(p, table, length, refs, ints(seq), ints(want), 1, granted, ws)
    ws.async_status()
    at = 0
    for s, n, w in zip(seq, need, want):
        assert torch.equal(table[s, :n], torch.arange(at, at + n, dtype=torch.int32, device="cuda")) and table[s, n:].eq(-1).all()
        at += n
    assert refs[:at].eq(1).all() and not refs[at:].any() and granted.tolist() == want and length.tolist() == want[::-1]
    assert at + 69998 <= N < at + 2 * 69998
    rs.page_pool_reserve(p, table, length, refs, ints([35, 36]), ints([16 * 69998] * 2), 1, None, ws)  # (one of them could be taken)
    with pytest.raises(rs.RatsparseError, match="status 7"):
        ws.async_status()
    assert not refs[at:].any()


def test_a_refusal_leaves_an_expired_wait_on_record(rs):
    """One workspace for a scan, whose wait expired (1 in the first word), and a call on the pool that is refused after it."""
    d = Device(rs, 10, 4, 6, 16)
    word = d.ws.buf[:4].view(torch.int32)
    calls = (lambda: rs.page_pool_reserve(*d.state(), ints([9]), None, 1, None, d.ws),
             lambda: rs.page_pool_fork(*d.state(), ints([9]), ints([1]), ints([[5, 5]]), None, d.ws),
             lambda: rs.page_pool_free(*d.state(), ints([9]), d.ws))
    for call in calls:
        word.fill_(1)
        call()
        with pytest.raises(rs.RatsparseError, match="status 5"):
            d.ws.async_status()
        d.ws.async_status()
        call(), call()
        with pytest.raises(rs.RatsparseError, match="status 7"):
            d.ws.async_status()
        d.ws.async_status()


def test_more_listed_heads_than_the_contiguous_calls_take(rs):
    """B Hq is limited where a head has control words of a workspace; these calls have none.  rat_append_paged, page_copy, rat_state_copy."""
    B, Hq, Hkv, D, P, dt = 700, 16, 2, 64, 16, torch.float32
    d = Device(rs, B, B, 2, P)
    assert d.reserve(list(range(B)), [1] * B)
    s = rs.make_shape(B, Hq, Hkv, D, B * P, P, dt)
    k, v = torch.randn(B, Hkv, 1, D, device="cuda"), torch.randn(B, Hkv, 1, D, device="cuda")
    sk, sv = torch.zeros(B, Hkv, D, device="cuda"), torch.zeros(B, Hkv, D, device="cuda")
    kp, vp = torch.zeros(Hkv, B * P, D, device="cuda"), torch.zeros(Hkv, B * P, D, device="cuda")
    rs.rat_append_paged(s, d.p, k, v, torch.zeros_like(k), sk, sv, kp, vp, None, d.table, d.len, ints(list(range(B))), None, 1)
    assert torch.equal(sk, k[:, :, 0]) and torch.equal(kp[:, ::P], k[:, :, 0].transpose(0, 1)) and torch.equal(vp[:, ::P], v[:, :, 0].transpose(0, 1))
    rs.page_copy(s, kp, vp, None, s, kp, vp, None, ints([[3, 699]]), None)
    assert torch.equal(kp[:, 699 * P:], kp[:, 3 * P:4 * P])
    rs.rat_state_copy(s, sk, sv, ints([[3, 699]]))
    assert torch.equal(sk[699], sk[3])


def test_compaction_of_a_pool_of_one_page(rs):
    """Nothing can move: the list's one entry says so, for a copy that goes without the number of pairs."""
    d = Device(rs, 1, 1, 1, 16)
    for room in (0, 3):
        assert d.reserve([0], [room])
        pairs, n = ints([[0, 0]]), ints([9])
        rs.page_pool_compact(*d.state(), pairs, n, d.ws)
        assert d.m.compact() == [] and n.item() == 0 and pairs.tolist() == [[-1, -1]]
        d.check("compact")


def test_a_workspace_that_is_not_on_the_device(rs):
    """Refused before anything is enqueued, by every call over a pool that takes one."""
    d, one, pairs = Device(rs, 10, 4, 6, 16), ints([0]), ints([[0, 0]] * 5)
    d.ws.buf = d.ws.buf.cpu()
    s = rs.make_shape(1, 1, 1, 64, 160, 16, torch.float32)
    x, rows = torch.zeros(1, 1, 1, 64, device="cuda"), torch.zeros(1, 160, 64, device="cuda")
    for call in (lambda: rs.page_pool_reserve(*d.state(), one, None, 1, None, d.ws),
                 lambda: rs.page_pool_fork(*d.state(), one, one, pairs[:1], None, d.ws),
                 lambda: rs.page_pool_free(*d.state(), one, d.ws),
                 lambda: rs.page_pool_compact(*d.state(), pairs, one.clone(), d.ws),
                 lambda: rs.attn_paged(s, d.p, x, rows, rows, d.table, d.len, one, None, 1, None, 0.1, x.clone(), None, d.ws)):
        with pytest.raises(AssertionError):
            call()
    assert not d.len.any() and not d.refs.any()
