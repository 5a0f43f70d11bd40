"""Attention over pages, shared ones once for all, against a softmax in 64 bits over the rows that each sequence's table names."""
import math

import numpy as np
import pytest
import torch

from gpu_util import say, tdtype
from pool_model import Pool, attention

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Batch:
    """Sequences over a pool: runs of them share their first pages; physical pages in no order; rows that nobody sees hold NaN."""

    def __init__(self, rs, Hq, Hkv, D, P, lens, runs=(), shared=0, T=1, counts=None, dtype="bf16", seed=0, scale=None, big=1.0):
        self.rs, self.dt, self.P, self.T, self.D, self.Hq, self.Hkv = rs, tdtype(dtype), P, T, D, Hq, Hkv
        r = self.r = np.random.default_rng(seed)
        B, c = len(lens), shared // P
        M = max(-(-max(lens) // P), 1) + 1
        N = B * M + 3
        m = self.m = Pool(N, B, M, P)
        pages = r.permutation(N).tolist()
        run_of, self.share = {}, [[b, 1, 0] for b in range(B)]
        at = 0
        for n in runs:
            first = [pages.pop() for _ in range(c)]
            for b in range(at, at + n):
                run_of[b] = first
                self.share[b] = [at, n, c if n > 1 else 0]
            at += n
        for b in range(B):
            m.len[b] = lens[b]
            row = (run_of.get(b, []) + [pages.pop() for _ in range(max(0, -(-lens[b] // P) - (c if b in run_of else 0)))])
            m.table[b][:len(row)] = row
        self.p, self.s = rs.make_pool(N, B, M, P), rs.make_shape(B, Hq, Hkv, D, N * P, P, self.dt)
        self.counts = counts
        rnd = lambda *n: torch.from_numpy(r.standard_normal(n).astype(np.float32)).cuda()
        self.k, self.v = (big * rnd(Hkv, N * P, D)).to(self.dt), rnd(Hkv, N * P, D).to(self.dt)
        used = np.zeros(N * P, bool)
        for b in range(B):
            used[m.rows(b)] = True
        self.k[:, ~torch.from_numpy(used)] = float("nan")
        self.v[:, ~torch.from_numpy(used)] = float("inf")
        self.q = rnd(B, Hq, T, D).to(self.dt)
        for b in range(B if counts else 0):  # not read
            self.q[b, :, min(max(counts[b], 0), T):] = float("nan")
        self.scale = 1 / math.sqrt(D) if scale is None else scale
        self.table, self.len, self.seq = ints(m.table), ints(m.len), ints(list(range(B)))
        self.ws = rs.Workspace(rs.attn_paged_workspace_bytes(self.s, self.p, T))

    def run(self, share=True, out=None, lse=None):
        B = len(self.m.len)
        out = torch.full((B, self.Hq, self.T, self.D), 7.0, device="cuda", dtype=self.dt) if out is None else out
        lse = torch.full((B, self.Hq, self.T), 7.0, device="cuda") if lse is None else lse
        self.rs.attn_paged(self.s, self.p, self.q, self.k, self.v, self.table, self.len, self.seq,
                           ints(self.counts) if self.counts else None, self.T, ints(self.share) if share else None, self.scale, out, lse, self.ws)
        torch.cuda.synchronize()
        self.ws.async_status()
        return out, lse

    def check(self, out, lse, heads=None):
        """Against the formula.  A weight is off by at most e^(2 delta) where a score is by delta: D terms of a product and their
        sum in float32, the scale, and 2^x with its argument's rounding; sums over n keys in float32; bfloat16 weights (half a step
        of 2^-8 each, of the weighted magnitudes) and the rounding of the result."""
        k, v, q, o, z = (x.float().cpu().numpy() for x in (self.k, self.v, self.q, out, lse))
        bf, G, e = self.dt == torch.bfloat16, self.Hq // self.Hkv, 2.0 ** -24
        worst = 0.0
        for b in range(len(self.m.len)):
            rows, L = self.m.rows(b), self.m.len[b]
            n = min(max(self.counts[b], 0), self.T) if self.counts else self.T
            assert np.all(o[b, :, n:] == 7.0) and np.all(z[b, :, n:] == 7.0)  # left as they were
            for h in range(self.Hq) if heads is None else heads:
                kk, vv = k[h // G][rows], v[h // G][rows]
                want, lw, mag, big = attention(q[b, h, :n], kk, vv, [L - n + i for i in range(n)], self.scale)
                delta = 2 * ((self.D + 4) * e * big + 4 * e * (1 + np.where(np.isfinite(lw), np.abs(lw), 0)))
                tol = mag * (2 * delta[:, None] + (L + 16) * e + (2.0 ** -8 if bf else 0)) * 1.01
                tol = tol + (2.0 ** -8 * (np.abs(want) + tol) if bf else 0) + 1e-30
                err = np.abs(o[b, h, :n] - want)
                assert np.all(err <= tol), (b, h, float((err / tol).max()))
                worst = max(worst, float((err / tol).max()) if n else 0.0)
                seen = np.isfinite(lw)
                assert np.all(z[b, h, :n][~seen] == -np.inf) and np.all(o[b, h, :n][~seen] == 0)
                assert np.all(np.abs(z[b, h, :n][seen] - lw[seen]) <= (delta + (L + 16) * e)[seen] + 2 * e * np.abs(lw[seen])), (b, h)
        say("  of the tolerance: %.3f" % worst)


CASES = [
    # Hq, Hkv, D, P, lens, runs, shared, T, counts
    (1, 1, 64, 16, [1], (), 0, 1, None),                                    # one token
    (2, 2, 128, 16, [16, 17, 15, 0, 1], (), 0, 1, None),                    # page ends, an empty sequence
    (4, 2, 64, 16, [130, 140, 129], (3,), 128, 1, None),                    # all share eight pages
    (8, 2, 128, 32, [700, 641, 1300, 33, 700], (3,), 640, 1, None),         # three of five share
    (6, 2, 128, 16, [100, 97, 99, 2000, 300, 310], (2, 1, 3), 96, 1, None),  # runs of two, one and three
    (32, 1, 64, 64, [65, 300], (2,), 64, 1, None),                          # more heads to a KV head than a small tile's rows
    (40, 1, 128, 16, [40, 41, 600], (3,), 32, 1, None),                     # ... than a large one's
    (4, 4, 128, 512, [513, 1025, 600], (3,), 512, 1, None),                 # large pages
    (4, 2, 128, 16, [50, 60, 33], (3,), 32, 5, None),                       # several tokens, with pages in common
    (4, 2, 128, 16, [50, 60, 33, 40], (4,), 32, 7, [7, 1, 0, 3]),           # a different number of each
    (4, 1, 64, 16, [200, 77, 350], (), 0, 70, [70, 1, 33]),                 # more rows than a tile
    (2, 2, 128, 16, [90], (), 0, 90, None),                                 # a whole prompt
    (8, 2, 128, 32, [400, 390], (2,), 320, 60, [60, 50]),                   # rows of one sequence fill tiles: nothing is put together
    (2, 1, 64, 16, [3, 20, 0], (), 0, 6, [6, 6, 2]),                        # fewer tokens than new ones
    (2, 2, 64, 16, [96, 96, 80], (3,), 80, 4, None),                        # new tokens inside the pages in common
    (1, 1, 128, 16, [9000], (), 0, 1, None),                                # one sequence over all workgroups
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_formula(rs, case, dtype):
    Hq, Hkv, D, P, lens, runs, shared, T, counts = CASES[case]
    say("paged", case, dtype)
    b = Batch(rs, Hq, Hkv, D, P, lens, runs, shared, T, counts, dtype, seed=case)
    got = b.run()
    b.check(*got)
    b.check(*b.run(share=False))  # the same sequences, nothing put together
    again = b.run()
    assert all(torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences(rs, dtype):
    """More places of the list than threads of a workgroup, tiles of shared rows that end anywhere."""
    r = np.random.default_rng(5)
    runs = [1, 150, 3, 2, 77, 40]
    B = sum(runs) + 30
    lens = [(64 if b < sum(runs) else 0) + int(x) for b, x in enumerate(r.integers(1, 60, B))]
    b = Batch(rs, 4, 2, 64, 16, lens, runs, 64, 1, None, dtype, seed=7)
    b.check(*b.run(), heads=[0, 3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_of_many_tiles(rs, dtype):
    """More row tiles to a sequence than a wave has lanes; one of them, and none, for the others."""
    b = Batch(rs, 4, 1, 64, 16, [2600, 2100, 0, 30], (), 0, 2600, [2600, 900, 0, 1], dtype, seed=13)
    b.check(*b.run(), heads=[0, 3])


MANY = [
    # Hq, Hkv, D, P, lens, runs, shared, T, counts: every sequence has more rows than a small tile
    (8, 2, 128, 16, [100, 97, 130, 60], (3,), 64, 12, [12, 5, 12, 0]),          # with room for others' in a large one
    (6, 2, 64, 32, [200, 230, 225, 700, 300], (2, 2), 192, 11, None),           # two runs
    (40, 1, 128, 16, [40, 41, 600], (2,), 32, 3, [3, 1, 2]),
    (4, 2, 64, 16, [20 + b % 45 for b in range(150)], (100,), 16, 17, None),    # a long list
    (2, 2, 128, 16, [33, 129, 4000], (), 0, 33, [33, 33, 20]),                  # one row past a small tile; one step past a turn of the ring
]


@pytest.mark.parametrize("case", range(len(MANY)))
def test_many_rows_a_sequence(rs, case):
    Hq, Hkv, D, P, lens, runs, shared, T, counts = MANY[case]
    say("many", case)
    b = Batch(rs, Hq, Hkv, D, P, lens, runs, shared, T, counts, "bf16", seed=40 + case)
    got = b.run()
    b.check(*got, heads=[0, Hq - 1])
    b.check(*b.run(share=False), heads=[0, Hq - 1])
    assert all(torch.equal(x, y) for x, y in zip(got, b.run()))


def test_listed_in_another_order_and_twice(rs):
    b = Batch(rs, 4, 2, 64, 16, [40, 35, 70, 90], (), 0, 1)
    out, lse = b.run()
    order = [2, 0, 0, 3]
    b.seq = ints(order)
    q = b.q
    b.q = q[order].contiguous()
    o2, l2 = b.run()
    assert torch.equal(o2, out[order]) and torch.equal(l2, lse[order])


def test_no_lse(rs):
    b = Batch(rs, 4, 2, 64, 16, [40, 35], (2,), 32, 1)
    out, _ = b.run()
    o2 = torch.zeros_like(out)
    rs.attn_paged(b.s, b.p, b.q, b.k, b.v, b.table, b.len, b.seq, None, 1, ints(b.share), b.scale, o2, None, b.ws)
    assert torch.equal(o2, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores_and_other_scales(rs, dtype):
    """Scores far beyond what e^x holds; a negative scale; zero."""
    for scale, big in ((4.0, 3.0), (-0.3, 1.0), (0.0, 1.0)):
        b = Batch(rs, 4, 2, 64, 16, [300, 250], (2,), 160, 1, None, dtype, seed=3, scale=scale, big=big)
        b.check(*b.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_values_that_a_row_does_not_see(rs, dtype, bad):
    """The last new token holds no number: the rows before it are what they would be without it."""
    b = Batch(rs, 4, 2, 128, 16, [45, 200], (), 0, 40, [40, 21], dtype, seed=11)
    clean, lse = b.run()
    for i in range(2):
        row = int(b.m.rows(i)[-1])
        b.k[0, row, 3] = bad
        b.v[:, row, ::5] = bad
    out, l2 = b.run()
    for i, n in ((0, 40), (1, 21)):
        # (these steps are taken key by key, with the weights in float32: another rounding)
        err = (out[i, :, :n - 1].float() - clean[i, :, :n - 1].float()).abs()
        assert torch.isfinite(out[i, :, :n - 1]).all() and torch.isfinite(l2[i, :, :n - 1]).all()
        assert err.max() <= 4 * 2.0 ** -8 * b.v[:, b.m.rows(i)[:-1]].float().abs().max()
        # both within what Batch.check allows of the formula; a score's terms sum to no more than the norms' product
        big = b.scale * float(b.q[i, :, :n].float().norm(dim=-1).max() * b.k[:, b.m.rows(i)[:-1]].float().norm(dim=-1).max())
        near = 2 * (2 * (132 * big + 4 * (1 + 10)) + 216 + 2 * 10) * 2.0 ** -24  # (the log-sum-exp is below 10)
        assert (l2[i, :, :n - 1] - lse[i, :, :n - 1]).abs().max() <= near and lse[i, :, :n - 1].abs().max() < 10
        assert not torch.isfinite(out[i, :, n - 1, ::5]).any()


def test_table_entries_that_name_no_page_hide_their_tokens(rs):
    b = Batch(rs, 2, 1, 64, 16, [64, 64, 40], (), 0, 1, None, "f32")
    b.table[0, 1], b.table[1, 3], b.table[2, 0] = -1, b.m.N, -2 ** 31
    b.table[1, 2] = 2 ** 31 - 1
    out, lse = b.run()
    k, v, q = (x.double().cpu().numpy() for x in (b.k, b.v, b.q))
    for i, hidden in enumerate((range(16, 32), range(32, 64), range(0, 16))):
        rows = np.array([x for t, x in enumerate(b.m.rows(i)) if t not in hidden])
        want, lw, _, _ = attention(q[i, :, 0], k[0][rows], v[0][rows], [len(rows) - 1] * 2, b.scale)
        assert np.abs(out[i, :, 0].double().cpu().numpy() - want).max() < 1e-5
        assert np.abs(lse[i, :, 0].double().cpu().numpy() - lw).max() < 1e-5
    b.table[:] = -1
    out, lse = b.run()
    assert not out.any() and torch.isneginf(lse).all()


def test_sequences_and_shares_that_are_out_of_range(rs):
    b = Batch(rs, 4, 2, 64, 16, [64, 70, 40], (), 0, 1, None, "f32")
    want, lw = b.run(share=False)
    b.seq = ints([0, 3, -1])
    out, lse = b.run(share=False)
    assert torch.equal(out[0], want[0]) and not out[1:].any() and torch.isneginf(lse[1:]).all()
    b.seq = ints([0, 1, 2])
    for share in ([[0, 4, 2]] * 3, [[-1, 2, 2]] * 3, [[2, 1, 9], [5, 5, 5], [2, 2, 1]], [[0, 1, 4], [0, 2, 2], [2, -1, 3]],
                  [[0, 2, -3]] * 3, [[0, 2 ** 31 - 1, 1]] * 3):  # none of these describes a run: each by itself
        b.share = share
        b.check(*b.run())  # (joined in another order than without the argument)


def test_shares_whose_runs_overlap(rs):
    """No page_pool_share gives these: an entry belongs to the run that it names, and to none if that does not reach it."""
    b = Batch(rs, 4, 2, 64, 16, [64, 70, 90], (3,), 48, 1, None, "f32")
    for share in ([[0, 3, 3], [1, 2, 2], [1, 2, 2]], [[0, 3, 3], [1, 2, 3], [0, 3, 1]], [[0, 2, 3], [0, 2, 3], [0, 2, 3]]):
        b.share = share
        first = b.run()
        b.check(*first)
        assert all(torch.equal(x, y) for x, y in zip(first, b.run()))


def test_a_longer_workspace_and_what_it_held_before(rs):
    b = Batch(rs, 8, 2, 64, 16, [300, 310, 900], (2,), 288, 1)
    out, lse = b.run()
    b.ws = rs.Workspace(b.ws.nbytes + 4096)
    b.ws.buf[rs.RS_WS_CTRL_BYTES:].fill_(255)  # NaN
    o2, l2 = b.run()
    assert torch.equal(out, o2) and torch.equal(lse, l2)


def test_far_rows_of_a_large_pool(rs):
    """Rows whose offsets pass 32 bits: 2^31 bytes into a KV head's rows and beyond."""
    P, D, N, dt = 16, 128, 1 << 20, torch.bfloat16
    k, v = (torch.zeros(1, N * P, D, device="cuda", dtype=dt) for _ in range(2))
    m = Pool(N, 2, 8, P)
    m.table[0][:5], m.table[1][:5] = [N - 1, 3, N - 2, 700000, 600000], [N - 1, 3, 524288, 524287, 0]
    m.len = [75, 70]
    gen = torch.Generator(device="cuda").manual_seed(2)
    for s in range(2):
        rows = torch.from_numpy(m.rows(s)).cuda()
        k[0, rows], v[0, rows] = (torch.randn(len(rows), D, device="cuda", generator=gen).to(dt) for _ in range(2))
    s, p = rs.make_shape(2, 2, 1, D, N * P, P, dt), rs.make_pool(N, 2, 8, P)
    q = torch.randn(2, 2, 1, D, device="cuda", generator=gen).to(dt)
    out, lse = torch.zeros(2, 2, 1, D, device="cuda", dtype=dt), torch.zeros(2, 2, 1, device="cuda")
    ws = rs.Workspace(rs.attn_paged_workspace_bytes(s, p, 1))
    rs.attn_paged(s, p, q, k, v, ints(m.table), ints(m.len), ints([0, 1]), None, 1, ints([[0, 2, 2]] * 2), 0.1, out, lse, ws)
    for b in range(2):
        rows = torch.from_numpy(m.rows(b)).cuda()
        want, lw, mag, _ = attention(q[b, :, 0].float().cpu().numpy(), k[0, rows].float().cpu().numpy(), v[0, rows].float().cpu().numpy(),
                                     [m.len[b] - 1] * 2, 0.1)
        assert np.all(np.abs(out[b, :, 0].float().cpu().numpy() - want) <= 2.0 ** -8 * (2.1 * mag))
        assert np.abs(lse[b, :, 0].cpu().numpy() - lw).max() < 1e-4
    # and the pages' copies
    rs.page_copy(s, k, v, None, s, k, v, None, ints([[N - 1, 900000]]), None)
    assert torch.equal(k[:, 900000 * P:900001 * P], k[:, (N - 1) * P:])


def test_on_another_stream(rs):
    b = Batch(rs, 8, 2, 128, 16, [300, 310, 900], (2,), 288, 1)
    want, lw = b.run()
    side = torch.cuda.Stream()
    out, lse = torch.zeros_like(want), torch.zeros_like(lw)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rs.attn_paged(b.s, b.p, b.q, b.k, b.v, b.table, b.len, b.seq, None, 1, ints(b.share), b.scale, out, lse, b.ws)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, lw)


def _serve(rs, dtype, graph):
    """A prompt scanned as contiguous rows and copied into pages; four users of it with questions of their own; tokens one by one; two
    users leave, the pool is compacted, and two forks of one that stays go on.  Yields what every attention gave."""
    dt, P, Hq, Hkv, D, T0, S = tdtype(dtype), 16, 4, 2, 64, 75, 8
    N, M = 64, 12
    m, p = Pool(N, S, M, P), rs.make_pool(N, S, M, P)
    gen = torch.Generator(device="cuda").manual_seed(31)
    rnd = lambda *n: torch.randn(*n, device="cuda", generator=gen)
    gates = lambda *n: torch.sigmoid(rnd(*n) * 0.5 + 2)
    pool = dict(k=torch.zeros(Hkv, N * P, D, device="cuda", dtype=dt), v=torch.zeros(Hkv, N * P, D, device="cuda", dtype=dt),
                meta=torch.zeros(Hkv, N, 2, D, device="cuda", dtype=dt), sk=torch.zeros(S, Hkv, D, device="cuda"), sv=torch.zeros(S, Hkv, D, device="cuda"))
    table, length, refs = torch.full((S, M), -1, dtype=torch.int32, device="cuda"), ints([0] * S), ints([0] * N)
    ws = rs.Workspace(max(rs.page_pool_workspace_bytes(p), *(rs.attn_paged_workspace_bytes(rs.make_shape(4, Hq, Hkv, D, N * P, P, dt), p, t) for t in (1, 9))))
    shape = lambda B: rs.make_shape(B, Hq, Hkv, D, N * P, P, dt)
    scale = 1 / math.sqrt(D)

    # the prompt
    cs = rs.make_shape(1, Hq, Hkv, D, 80, P, dt)
    kc, vc, mc = (torch.zeros(*n, D, device="cuda", dtype=dt) for n in ((1, Hkv, 80), (1, Hkv, 80), (1, Hkv, 5, 2)))
    k0, v0, g0 = rnd(1, Hkv, T0, D).to(dt), rnd(1, Hkv, T0, D).to(dt), gates(1, Hkv, T0, D)
    sk, sv = torch.zeros(1, Hkv, D, device="cuda"), torch.zeros(1, Hkv, D, device="cuda")
    rs.rat_scan(cs, k0, v0, g0, sk, sv, kc, vc, 0, T0, rs.Workspace(rs.rat_scan_workspace_bytes(cs, T0)), mc)
    rs.page_pool_reserve(p, table, length, refs, ints([5]), None, T0, None, ws)
    m.reserve([5], [T0])
    rs.page_copy(cs, kc[0], vc[0], mc[0], shape(1), pool["k"], pool["v"], pool["meta"],
                 torch.stack([torch.arange(5, device="cuda", dtype=torch.int32), table[5, :5]], 1).contiguous(), None)
    pool["sk"][5], pool["sv"][5] = sk[0], sv[0]

    def fork(src, dst):
        pairs, carry = ints([[0, 0]] * len(src)), ints([[0, 0]] * len(src))
        rs.page_pool_fork(p, table, length, refs, ints(src), ints(dst), pairs, carry, ws)
        rs.page_copy(shape(1), pool["k"], pool["v"], pool["meta"], shape(1), pool["k"], pool["v"], pool["meta"], pairs, None)
        rs.rat_state_copy(shape(1), pool["sk"], pool["sv"], carry)
        m.fork(src, dst)

    def layer(B, T, x, seq, share, granted, out, lse):
        rs.rat_append_paged(shape(B), p, x["k"], x["v"], x["g"], pool["sk"], pool["sv"], pool["k"], pool["v"], pool["meta"], table, length, seq,
                            granted, T)
        rs.attn_paged(shape(B), p, x["q"], pool["k"], pool["v"], table, length, seq, granted, T, share, scale, out, lse, ws)

    def inputs(B, T):
        return dict(k=rnd(B, Hkv, T, D).to(dt), v=rnd(B, Hkv, T, D).to(dt), g=gates(B, Hkv, T, D), q=rnd(B, Hq, T, D).to(dt))

    def checked(seq, want, x, out, lse, before):
        b = Batch.__new__(Batch)  # (its check looks at these)
        b.k, b.v, b.q, b.dt, b.Hq, b.Hkv, b.D, b.T, b.scale, b.counts = pool["k"], pool["v"], x["q"], dt, Hq, Hkv, D, x["q"].shape[2], scale, want
        b.m = Pool(N, len(seq), M, P)
        b.m.table, b.m.len = [m.table[s] for s in seq], [m.len[s] for s in seq]
        b.check(out, lse)
        assert table.tolist() == m.table and length.tolist() == m.len and refs.tolist() == m.refs

    users, share = [1, 7, 0, 2], ints([[0, 0, 0]] * 4)
    fork([5] * 4, users)
    rs.page_pool_share(p, table, length, ints(users), 1, share)
    assert share.tolist() == [[0, 4, 4]] * 4
    want, granted = [9, 4, 1, 6], ints([0] * 4)
    rs.page_pool_reserve(p, table, length, refs, ints(users), ints(want), 9, granted, ws)
    m.reserve(users, want)
    x, out, lse = inputs(4, 9), torch.full((4, Hq, 9, D), 7.0, device="cuda", dtype=dt), torch.full((4, Hq, 9), 7.0, device="cuda")
    layer(4, 9, x, ints(users), share, granted, out, lse)
    checked(users, want, x, out, lse, None)
    yield out, lse

    def steps(seq, share, n):
        B, seq_d, granted = len(seq), ints(seq), ints([0] * len(seq))
        x, out, lse = inputs(B, 1), torch.full((B, Hq, 1, D), 7.0, device="cuda", dtype=dt), torch.full((B, Hq, 1), 7.0, device="cuda")

        def step():
            rs.page_pool_reserve(p, table, length, refs, seq_d, None, 1, granted, ws)
            layer(B, 1, x, seq_d, share, granted, out, lse)
        g = None
        if graph:
            g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
            torch.cuda.synchronize()
            with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
                step()
            torch.cuda.synchronize()
        for _ in range(n):
            for name, y in inputs(B, 1).items():
                x[name].copy_(y)
            out.fill_(7.0), lse.fill_(7.0)
            if graph:
                g.replay()
            else:
                step()
            torch.cuda.synchronize()
            m.reserve(seq, [1] * B)
            checked(seq, [1] * B, x, out, lse, None)
            yield out.clone(), lse.clone()

    yield from steps(users, share, 20)
    rs.page_pool_free(p, table, length, refs, ints([7, 5]), ws)
    m.free([7, 5])
    pairs, n_pairs = ints([[0, 0]] * (N // 2)), ints([0])
    rs.page_pool_compact(p, table, length, refs, pairs, n_pairs, ws)
    rs.page_copy(shape(1), pool["k"], pool["v"], pool["meta"], shape(1), pool["k"], pool["v"], pool["meta"], pairs, n_pairs)
    assert m.compact() and max(max(r) for r in m.table) < sum(n > 0 for n in m.refs)
    fork([2, 2], [4, 6])
    seq = [0, 2, 4, 6]
    share = ints([[0, 0, 0]] * 4)
    rs.page_pool_share(p, table, length, ints(seq), 1, share)
    yield from steps(seq, share, 18)
    ws.async_status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_serving_eagerly_and_from_a_graph(rs, dtype):
    say("serve", dtype)
    eager = [(o.clone(), l.clone()) for o, l in _serve(rs, dtype, False)]
    replayed = [(o.clone(), l.clone()) for o, l in _serve(rs, dtype, True)]
    assert len(eager) == len(replayed) == 39
    for (o, l), (o2, l2) in zip(eager, replayed):
        assert torch.equal(o, o2) and torch.equal(l, l2)


def test_the_longest_list(rs):
    r = np.random.default_rng(8)
    lens = [int(x) for x in r.integers(0, 40, 1024)]
    for i in range(500, 700):
        lens[i] = 16 + int(r.integers(1, 20))
    b = Batch(rs, 2, 1, 128, 16, lens, [1] * 500 + [200], 16, 1, None, "bf16", seed=9)
    b.check(*b.run())


def test_nothing_new(rs):
    b = Batch(rs, 2, 2, 64, 16, [40, 35], (2,), 32, 3, [0, -5])
    out, lse = b.run()
    assert out.eq(7.0).all() and lse.eq(7.0).all()


def test_two_calls_at_once(rs):
    """On two streams, each with a workspace of its own."""
    one, two = Batch(rs, 8, 2, 128, 16, [3000, 3010, 5000], (2,), 2992, 1, seed=1), Batch(rs, 4, 4, 64, 32, [900, 700], (), 0, 9, seed=2)
    want = one.run(), two.run()
    side = [torch.cuda.Stream() for _ in range(2)]
    got = [(torch.full_like(o, 7.0), torch.full_like(l, 7.0)) for o, l in want]
    shares = [ints(b.share) for b in (one, two)]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, st, (o, l), sh in zip((one, two), side, got, shares):
            with torch.cuda.stream(st):
                rs.attn_paged(b.s, b.p, b.q, b.k, b.v, b.table, b.len, b.seq, None, b.T, sh, b.scale, o, l, b.ws)
    torch.cuda.synchronize()
    for (o, l), (wo, wl) in zip(got, want):
        assert torch.equal(o, wo) and torch.equal(l, wl)


@pytest.mark.parametrize("case", [3, 4, 9, 10])
def test_a_workspace_used_for_other_calls_in_between(rs, case):
    """Two captured graphs and eager calls of another shape share one workspace."""
    Hq, Hkv, D, P, lens, runs, shared, T, counts = CASES[case]
    one, two = Batch(rs, Hq, Hkv, D, P, lens, runs, shared, T, counts, seed=case), Batch(rs, 4, 2, 64, 16, [130, 140, 129], (3,), 128, 1, seed=2)
    ws = rs.Workspace(max(one.ws.nbytes, two.ws.nbytes))
    one.ws = two.ws = ws
    want = one.run(), two.run()
    outs = [(torch.full_like(o, 7.0), torch.full_like(l, 7.0)) for o, l in want]
    graphs, extra = [], [(ints(b.counts) if b.counts else None, ints(b.share)) for b in (one, two)]
    for b, (o, l), (n_new, share) in zip((one, two), outs, extra):
        g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
            rs.attn_paged(b.s, b.p, b.q, b.k, b.v, b.table, b.len, b.seq, n_new, b.T, share, b.scale, o, l, ws)
        graphs.append(g)
    for rep in range(3):
        for o, l in outs:
            o.fill_(7.0), l.fill_(7.0)
        graphs[0].replay()
        two.run()
        graphs[1].replay()
        one.run(share=False)
        torch.cuda.synchronize()
        for (o, l), (wo, wl) in zip(outs, want):
            assert torch.equal(o, wo) and torch.equal(l, wl), rep


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,T", [(4, 1, 1), (8, 1, 1), (2, 2, 1), (20, 1, 1), (40, 1, 1), (4, 1, 3)])
def test_values_that_every_row_sees(rs, Hq, Hkv, T, dtype):
    """Rows of V without a number that all of a tile's rows see: their channels are not numbers, and nothing else changes by a bit (no
    row is taken key by key for them).  Rows of a tile that do not exist are not rows that see less."""
    say("visible", Hq, Hkv, T, dtype)
    for bad in (float("nan"), float("inf")):
        b = Batch(rs, Hq, Hkv, 128, 16, [45, 200, 64, 1500], (), 0, T, None, dtype, seed=17)
        clean, lse = b.run()
        for i, at in ((0, [3, 45 - T]), (1, [0, 100, 200 - T]), (2, [64 - T]), (3, [640, 1500 - T])):
            if T > 1:  # far from the new tokens, whose steps some rows do not see to their end
                at = [x for x in at if x < b.m.len[i] - 64]
            b.v[:, b.m.rows(i)[at], 5::32] = bad
        out, l2 = b.run()
        assert torch.equal(l2, lse)
        odd = torch.zeros(128, dtype=torch.bool, device="cuda")
        odd[5::32] = True
        assert torch.equal(out[..., ~odd], clean[..., ~odd])
        for i in range(4):
            if T == 1 or i in (1, 3):
                assert torch.isnan(out[i][..., odd]).all() if math.isnan(bad) else torch.isposinf(out[i][..., odd]).all()


def places(dtype, G, Hkv, P, lens, T, counts, run, shared):
    """How a call's work is divided, counted on the host: for each kind of tile (few rows, many rows) the places of its line over all KV
    heads, and the shares it is cut into where it is long.  One run of `run` sequences from the first on, `shared` tokens."""
    bf = dtype == "bf16"
    counts = [T] * len(lens) if counts is None else counts
    rows, unit, before = {False: 32, True: 128}, {False: 32 if bf else 16, True: 128}, {False: 3, True: 2}
    line = {False: 0, True: 0}
    own_many, together = bf and T * G > 32, T * G < (128 if bf else 32)
    shared = shared // P * P if together and run > 1 else 0
    for b, (L, n) in enumerate(zip(lens, counts)):
        k0 = shared if b < run else 0
        for t0 in range(0, n * G, rows[own_many]):
            keys = L - n + min(n - 1, (t0 + rows[own_many] - 1) // G) + 1 - k0
            line[own_many] += -(-keys // unit[own_many]) + before[own_many] if keys > 0 else 0
    if shared:
        many = bf and run * T * G > 32
        line[many] += -(-run * T * G // rows[many]) * (-(-shared // unit[many]) + before[many])
    groups = 768 if own_many and len(lens) <= 112 else 512
    if line[False] and line[True]:
        part = 5.25 * line[True] / (5.25 * line[True] + line[False])
        taken = 8 * max(1, min(63, 2 * int(part * 32 + 0.5)))
    else:
        taken = groups if line[True] else 0
    return (line[False] * Hkv, (groups - taken) * 4), (line[True] * Hkv, taken)


LONG = [
    # Hq, Hkv, D, P, lens, run, shared, T, counts, keys of a share at least (few rows, many rows; 0: no such line)
    (16, 8, 64, 16, [9000, 17000, 7001, 300, 9500], 2, 7000, 1, None, (64, 0)),         # one token each, a run whose rows are few
    (16, 8, 64, 16, [24016 + 40 * b for b in range(24)], 24, 24000, 1, None, (64, 512)),  # a long prompt's rows are many, the rest few
    (4, 4, 64, 512, [600000], 0, 0, 1, None, (1100, 0)),                                # more entries of the table to a share than a wave lists at once
    (32, 32, 64, 16, [20000, 3000], 0, 0, 300, [300, 120], (0, 1100)),                  # several tiles of 128 rows; three workgroups a CU
    (16, 16, 64, 16, [24010 + 190 * b for b in range(8)], 8, 24000, 40, None, (0, 512)),  # more new tokens than a small tile's rows, over a shared prompt
    (4, 4, 64, 16, [420 + b for b in range(120)], 0, 0, 33, None, (0, 512)),            # a list for which two workgroups fit a CU
    (16, 8, 64, 16, [60001 + b % 7 for b in range(24)], 24, 60000, 1, None, (300, 512)),  # nearly all CUs for the rows that are many
    (16, 8, 64, 16, [5000 + 200 * b for b in range(24)], 24, 256, 1, None, (512, 512)),   # nearly none
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(LONG)))
def test_lines_cut_into_long_shares(rs, case, dtype):
    """Four places of a line and more to a share: shares are weighted by which workgroup came first.  Rows at the ends of tiles, of the first and
    the last KV head, of every sequence."""
    Hq, Hkv, D, P, lens, run, shared, T, counts, least = LONG[case]
    say("long", case, dtype)
    dt, G, B = tdtype(dtype), Hq // Hkv, len(lens)
    lines = places(dtype, G, Hkv, P, lens, T, counts, run, shared)
    summed = 0  # terms that a sum takes one after the other: the keys of a share (twice the mean is more than the weights give), then the shares
    for (all_places, shares), keys, unit in zip(lines, least, (32 if dtype == "bf16" else 16, 128)):
        if dtype == "bf16":
            assert (all_places > 0) == (keys > 0)
        if all_places:
            assert all_places >= 4 * shares and all_places * unit >= (keys if dtype == "bf16" else 0) * shares
            summed += 2 * all_places * unit // shares + -(-shares // Hkv)
    M = -(-max(lens) // P)
    m = Pool(sum(-(-x // P) for x in lens) - max(0, run - 1) * (shared // P) + 5, B, M, P)
    r, gen = np.random.default_rng(case), torch.Generator(device="cuda").manual_seed(case)
    pages = r.permutation(m.N).tolist()
    first = [pages.pop() for _ in range(shared // P)]
    for b in range(B):
        m.len[b] = lens[b]
        row = first[:] if b < run else []
        row += [pages.pop() for _ in range(-(-lens[b] // P) - len(row))]
        m.table[b][:len(row)] = row
    k, v = (torch.randn(Hkv, m.N * P, D, device="cuda", generator=gen).to(dt) for _ in range(2))
    q = torch.randn(B, Hq, T, D, device="cuda", generator=gen).to(dt)
    share = [[0, run, shared // P] if b < run else [b, 1, 0] for b in range(B)]
    s, p = rs.make_shape(B, Hq, Hkv, D, m.N * P, P, dt), rs.make_pool(m.N, B, M, P)
    ws = rs.Workspace(rs.attn_paged_workspace_bytes(s, p, T))
    args = (s, p, q, k, v, ints(m.table), ints(m.len), ints(list(range(B))), ints(counts) if counts else None, T, ints(share), 1 / math.sqrt(D))
    got = []
    for _ in range(2):
        out, lse = torch.full((B, Hq, T, D), 7.0, device="cuda", dtype=dt), torch.full((B, Hq, T), 7.0, device="cuda")
        rs.attn_paged(*args, out, lse, ws)
        torch.cuda.synchronize()
        got.append((out, lse))
    assert all(torch.equal(x, y) for x, y in zip(*got))
    bf, e, worst = dtype == "bf16", 2.0 ** -24, 0.0
    for b in range(B):
        rows, L, n = m.rows(b), lens[b], counts[b] if counts else T
        terms = min(L, summed) + 16
        some = sorted({t for x in (0, 31, 32, 127, 128, 255, 256, n * G - 1) for t in (x // G,) if t < n})
        assert out[b, :, n:].eq(7.0).all() and lse[b, :, n:].eq(7.0).all()
        for h in sorted({0, G - 1, Hq - 1}):
            kk, vv = (x[h // G, torch.from_numpy(rows).cuda()].float().cpu().numpy() for x in (k, v))
            o, z = (x[b, h, some].float().cpu().numpy() for x in (out, lse))
            want, lw, mag, big = attention(q[b, h, some].float().cpu().numpy(), kk, vv, [L - n + t for t in some], args[-1])
            # as in Batch.check, but for the sums
            delta = 2 * ((D + 4) * e * big + 4 * e * (1 + np.abs(lw)))
            tol = mag * (2 * delta[:, None] + terms * e + (2.0 ** -8 if bf else 0)) * 1.01
            tol = tol + (2.0 ** -8 * (np.abs(want) + tol) if bf else 0) + 1e-30
            assert np.all(np.abs(o - want) <= tol), (b, h, float((np.abs(o - want) / tol).max()))
            assert np.all(np.abs(z - lw) <= delta + terms * e + 2 * e * np.abs(lw)), (b, h)
            worst = max(worst, float((np.abs(o - want) / tol).max()))
    say("  of the tolerance: %.3f" % worst)


def test_more_listed_heads_than_the_contiguous_calls_take(rs):
    """B Hq past 8160, which limits calls whose heads have control words of a workspace."""
    r = np.random.default_rng(4)
    lens = [33 + int(x) for x in r.integers(0, 40, 300)]
    b = Batch(rs, 32, 8, 64, 16, lens, (5, 200), 32, 1, None, "bf16", seed=21)
    b.check(*b.run(), heads=[0, 31])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_without_a_number_where_a_tile_goes_key_by_key(rs, dtype):
    """Keys of infinities that rows see, in a tile whose last value no other row may look at: rows get what they get without that value."""
    b = Batch(rs, 4, 2, 64, 16, [45, 60, 50], (), 0, 20, None, dtype, seed=23)
    b.q[..., 0] = b.q[..., 0].abs() + 0.5
    b.k[:, b.m.rows(0)[30], 0] = float("inf")   # seen by the rows from position 30 on, of 25 to 44: no numbers
    b.k[:, b.m.rows(1)[50], 0] = float("-inf")  # counts for nothing
    b.k[:, b.m.rows(2)[:45], 0] = float("-inf")  # rows of positions 30 to 44 see nothing else
    plain, lse = b.run()
    for i in range(3):
        b.v[:, int(b.m.rows(i)[-1]), 3] = float("nan")
    out, l2 = b.run()
    for o, z in ((plain, lse), (out, l2)):
        assert torch.isfinite(o[0, :, :5]).all() and torch.isnan(o[0, :, 5:-1]).all() and torch.isnan(z[0, :, 5:-1]).all()
        assert torch.isfinite(o[1, :, :-1]).all() and torch.isfinite(z[1, :, :-1]).all()
        assert o[2, :, :15].eq(0).all() and torch.isneginf(z[2, :, :15]).all() and torch.isfinite(o[2, :, 15:-1]).all()
    # as in test_values_that_a_row_does_not_see
    for i, rows in ((0, slice(0, 5)), (1, slice(0, 19)), (2, slice(15, 19))):
        assert (out[i, :, rows].float() - plain[i, :, rows].float()).abs().max() <= 4 * 2.0 ** -8 * b.v[:, b.m.rows(i)[:-1]].float().abs().max()
