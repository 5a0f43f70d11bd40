"""Eviction by tally against a plain model: which rows stay, where they go, what is left as it was."""
import numpy as np
import pytest
import torch

import kv4_model as M
from gpu_util import say, tdtype

pytestmark = pytest.mark.gpu


class State:
    """A cache of bytes or numbers, its tally, positions and lengths, and the model's copies."""

    def __init__(self, rs, four, dtype, B, Hkv, D, Tcap, lens, seed=0, tally="spread"):
        self.rs, self.four, self.lens = rs, four, list(lens)
        self.s = rs.make_shape(B, Hkv, Hkv, D, Tcap, 16, tdtype(dtype))
        r = np.random.default_rng(seed)
        if four:
            self.rows = [torch.from_numpy(r.integers(0, 256, (B, Hkv, Tcap, n), dtype=np.uint8)).cuda() for n in (D // 2, D // 32, D // 2, D // 32)]
        else:
            self.rows = [torch.from_numpy(r.standard_normal((B, Hkv, Tcap, D)).astype(np.float32)).to(tdtype(dtype)).cuda() for _ in "kv"]
        t = np.exp(2 * r.standard_normal((B, Hkv, Tcap))).astype(np.float32)
        if tally == "ties":
            t = r.integers(0, 4, t.shape).astype(np.float32)
        elif tally == "same":
            t[:] = 0.25
        elif tally == "odd":
            t = r.choice(np.array([np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, -2.0, 1e-40, 3e38], dtype=np.float32), t.shape)
        elif tally == "close":  # neighbours in the last bits
            t = (np.float32(1) + r.integers(0, 1000, t.shape) * np.float32(2.0 ** -23)).astype(np.float32)
        self.tally = torch.from_numpy(t).cuda()
        self.pos = torch.full((B, Hkv, Tcap), -7, dtype=torch.int32, device="cuda")
        self.mark = torch.zeros(B, 2, dtype=torch.int32, device="cuda")
        self.len = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def copies(self):
        return [x.clone().cpu() for x in self.rows + [self.tally, self.pos, self.mark, self.len]]

    def call(self, keep, first, recent, slack, ws=None):
        rs = self.rs
        ws = ws or rs.Workspace(rs.cache_evict_workspace_bytes(self.s, keep))
        (rs.kv4_evict if self.four else rs.cache_evict)(self.s, *self.rows, self.tally, self.pos, self.mark, self.len, keep, first, recent, slack, ws)

    def expect(self, before, keep, first, recent, slack):
        rows, (tally, pos, mark, length) = before[:len(self.rows)], before[len(self.rows):]
        n_moved = 0
        for b in range(self.s.B):
            L = min(max(int(length[b]), 0), self.s.Tcap)
            known, had = int(mark[b, 0]), int(mark[b, 1])
            for h in range(self.s.Hkv):
                got = M.evict(tally[b, h].numpy(), pos[b, h].numpy(), known, had, L, keep, first, recent, slack)
                if got is None:
                    continue
                pairs, at = got
                n_moved += len(pairs)
                pos[b, h, :keep] = torch.tensor(at, dtype=torch.int32)
                if pairs:
                    src, to = (torch.tensor(x) for x in zip(*pairs))
                    for x in rows + [tally]:
                        x[b, h, to] = x[b, h, src].clone()
            if L > keep + slack:
                length[b], mark[b, 0], mark[b, 1] = keep, keep, had + L - known
        return rows + [tally, pos, mark, length], n_moved

    def check(self, want):
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(self.rows + [self.tally, self.pos, self.mark, self.len], want)):
            x = x.cpu()
            if x.is_floating_point():  # by their bits: NaN among them
                x, y = (t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32) for t in (x, y))
            assert torch.equal(x, y), (i, (x != y).nonzero()[:5])


CASES = [  # B, Hkv, D, Tcap, lengths, keep, first, recent, slack
    (1, 1, 64, 16, [2], 1, 0, 0, 0),
    (1, 2, 64, 64, [5], 3, 0, 1, 0),
    (3, 2, 128, 100, [100, 40, 41], 40, 4, 9, 0),
    (3, 2, 128, 100, [100, 60, 51], 40, 0, 40, 10),
    (4, 3, 64, 700, [700, 0, 650, 900], 600, 600, 0, 0),
    (2, 2, 128, 3000, [2999, 1500], 100, 3, 20, 0),
    (2, 1, 64, 5000, [4097, 5000], 4096, 4, 64, 0),
    (1, 2, 64, 20000, [19999], 9000, 10, 100, 0),
    (2, 2, 64, 256, [-3, 256], 255, 1, 254, 0),
    (1, 1, 128, 300, [300], 300, 0, 0, 0),
    (1, 1, 64, 70000, [69999], 30011, 7, 1000, 0),
    (1, 2, 64, 12000, [11999], 700, 0, 3, 0),
    (5, 1, 64, 2000, [1999, 1995, 1991, 1992, 2000], 1991, 5, 1986, 0),   # up to nine rows go, of hardly more that may
    (2, 2, 64, 34816, [34816, 34815], 34808, 0, 0, 0),
    (9, 30, 64, 130, [130, 0, 66, 65, 64, 73, 74, 129, 1], 65, 3, 7, 0),   # more heads than compute units
    (2, 131, 64, 2304, [2304, 2301], 1030, 3, 70, 0),
    (3, 90, 64, 2305, [2305, 1025, 2049], 1024, 0, 1, 0),
]


@pytest.mark.parametrize("four,dtype", [(True, "bf16"), (False, "bf16"), (False, "f32")])
@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("tally", ["spread", "ties", "same", "odd", "close"])
def test_evict(rs, four, dtype, case, tally):
    B, Hkv, D, Tcap, lens, keep, first, recent, slack = CASES[case]
    say("evict", four, dtype, CASES[case], tally)
    x = State(rs, four, dtype, B, Hkv, D, Tcap, lens, seed=case, tally=tally)
    for _ in range(2):  # (the second call finds every sequence within its budget)
        want, moved = x.expect(x.copies(), keep, first, recent, slack)
        x.call(keep, first, recent, slack)
        x.check(want)
    assert moved == 0


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("B,Hkv,Tcap,L,keep", [(2, 2, 300, 300, 293), (2, 2, 300, 300, 40), (2, 2, 300, 299, 150), (1, 1, 35000, 34999, 900), (9, 30, 200, 193, 20),
                                               (9, 30, 200, 200, 192)])
@pytest.mark.parametrize("share", [1.0, 0.7])
def test_positions_that_repeat(rs, four, B, Hkv, Tcap, L, keep, share):
    """Positions cleared by mistake, so that more rows than n_keep have to stay: the first of them do, and nothing else is written."""
    say("repeat", four, B, Hkv, Tcap, L, keep, share)
    x = State(rs, four, "bf16", B, Hkv, 64, Tcap, [L] * B, seed=1)
    r = np.random.default_rng(2)
    x.pos.copy_(torch.from_numpy(np.where(r.random((B, Hkv, Tcap)) < share, 0, 20).astype(np.int32)))
    x.mark[:] = L
    want, _ = x.expect(x.copies(), keep, 1, 0, 0)
    x.call(keep, 1, 0, 0)
    x.check(want)


@pytest.mark.parametrize("four", [True, False])
def test_again_and_again(rs, four):
    """Sequences that grow by different numbers and give up rows as they go, positions and budgets that change among it, in a replayed graph too."""
    B, Hkv, D, Tcap = 3, 2, 64, 200
    x = State(rs, four, "bf16", B, Hkv, D, Tcap, [90, 10, 0], seed=5, tally="ties")
    r = np.random.default_rng(6)
    ws = rs.Workspace(rs.cache_evict_workspace_bytes(x.s, 80))
    graph = None
    for i in range(30):
        grown = torch.from_numpy(r.integers(0, 12, B).astype(np.int32)).cuda()
        x.len.copy_(torch.minimum(x.len + grown, torch.full_like(x.len, Tcap)))
        x.tally += torch.from_numpy(r.integers(0, 3, x.tally.shape).astype(np.float32)).cuda()
        args = (80, 4, 16, 0 if i % 3 else 7)
        want, _ = x.expect(x.copies(), *args)
        if i < 6 or i % 3 == 0:
            x.call(*args, ws)
        else:
            if graph is None:
                side = torch.cuda.Stream()
                side.wait_stream(torch.cuda.current_stream())
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    x.call(*args, ws)
            graph.replay()
        x.check(want)
    assert int(x.mark[:, 1].max()) > 90
    # a sequence ends and another begins in its row: only its mark is cleared
    x.mark[0] = 0
    x.len[0] = 95
    want, _ = x.expect(x.copies(), 80, 4, 16, 0)
    x.call(80, 4, 16, 0, ws)
    x.check(want)


@pytest.mark.parametrize("four", [True, False])
def test_a_cache_within_its_budget_is_decoded(rs, four):
    """Append, attend with the tally, evict, step by step, against the same in 64 bits: the sets of positions agree wherever the tallies that
    decide are apart by more than their rounding, and results throughout (the model takes the library's set)."""
    B, Hq, Hkv, D, keep, first, recent, steps, T0 = 2, 4, 2, 64, 48, 2, 8, 60, 40
    Tcap = 64
    dt = torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *n: torch.randn(*n, device="cuda", generator=g)
    s = rs.make_shape(B, Hq, Hkv, D, Tcap, 16, dt)
    every = [rand(B, Hkv, T0 + steps, D).to(dt) for _ in "kv"]
    queries = rand(steps, B, Hq, D).to(dt)
    tally, pos = torch.zeros(B, Hkv, Tcap, device="cuda"), torch.zeros(B, Hkv, Tcap, device="cuda", dtype=torch.int32)
    mark, length = torch.zeros(B, 2, device="cuda", dtype=torch.int32), torch.full((B,), T0, device="cuda", dtype=torch.int32)
    out, lse = torch.zeros(B, Hq, D, device="cuda", dtype=dt), torch.zeros(B, Hq, device="cuda")
    if four:
        cache = [torch.zeros(B, Hkv, Tcap, n, dtype=torch.uint8, device="cuda") for n in (D // 2, D // 32, D // 2, D // 32)]
        rs.kv4_append(s, *every, 0, length, None, T0, *cache, None)
        ws = rs.Workspace(max(rs.kv4_attn_decode_workspace_bytes(s, 0, 0, True), rs.cache_evict_workspace_bytes(s, keep)))
        k, v = (M.values(*M.pack(x.double().cpu().numpy())) for x in every)
    else:
        cache = [torch.zeros(B, Hkv, Tcap, D, dtype=dt, device="cuda") for _ in "kv"]
        for x, y in zip(cache, every):
            x[:, :, :T0] = y[:, :, :T0]
        ws = rs.Workspace(max(rs.attn_decode_tally_workspace_bytes(s), rs.cache_evict_workspace_bytes(s, keep)))
        k, v = (x.double().cpu().numpy() for x in every)
    at = np.tile(np.arange(T0), (B, Hkv, 1))   # positions of the rows
    had = np.zeros((B, Hkv, T0 + steps))       # tally by position, in 64 bits
    for i in range(steps):
        n, t = at.shape[2] + 1, T0 + i
        length.add_(1)
        if four:
            rs.kv4_append(s, *every, t, length, None, 1, *cache, None)
            rs.kv4_attn_decode(s, queries[i].contiguous(), *cache, length, D ** -0.5, None, tally, 1, out, lse, ws)
        else:
            for x, y in zip(cache, every):
                x[:, :, n - 1] = y[:, :, t]
            rs.attn_decode_tally(s, queries[i].contiguous(), *cache, length, D ** -0.5, tally, 1, out, lse, ws)
        (rs.kv4_evict if four else rs.cache_evict)(s, *cache, tally, pos, mark, length, keep, first, recent, 0, ws)
        torch.cuda.synchronize()
        at = np.concatenate([at, np.full((B, Hkv, 1), t)], 2)
        now = []
        for b in range(B):
            for h in range(Hkv):
                q = queries[i][b, h * 2:h * 2 + 2].double().cpu().numpy()
                rows = at[b, h]
                o, z, p, a, most = M.attention(q, k[b, h, rows], v[b, h, rows], D ** -0.5)
                e = M.rounding(most[:, None], n, D)
                err = np.abs(out[b, h * 2:h * 2 + 2].double().cpu().numpy() - o)
                assert np.all(err <= (e + 2.0 ** -8) * a + 2.0 ** -8 * np.abs(o))
                had[b, h, rows] += p.sum(0)
                if n <= keep:
                    continue
                got = pos[b, h, :keep].cpu().numpy()
                gone = sorted(set(rows) - set(got))
                assert len(gone) == 1 and len(set(got)) == keep
                free = [x for x in rows if first <= x < t + 1 - recent]
                assert gone[0] in free and had[b, h, gone[0]] <= min(had[b, h, free]) * (1 + (i + 1) * float(e.max())) + 1e-12
                tallies = tally[b, h, :keep].double().cpu().numpy()
                assert np.allclose(tallies, had[b, h, got], rtol=(i + 1) * (float(e.max()) + 2.0 ** -23), atol=0)
                now.append(got)
        if n > keep:
            at = np.stack(now).reshape(B, Hkv, keep)
            assert length.tolist() == [keep] * B and mark.tolist() == [[keep, t + 1]] * B


def test_rows_far_into_a_long_cache(rs):
    """Offsets past 2^32 bytes: 20 million float32 rows of 64 channels."""
    Tcap, D, keep = 20_000_000, 64, 19_999_990
    s = rs.make_shape(1, 1, 1, D, Tcap, 16, torch.float32)
    k, v = (torch.zeros(1, 1, Tcap, D, device="cuda") for _ in "kv")
    k[0, 0, keep:] = torch.arange(10.0, device="cuda")[:, None] + 1
    v[0, 0, keep:] = torch.arange(10.0, device="cuda")[:, None] + 21
    tally = torch.ones(1, 1, Tcap, device="cuda")
    gone = torch.tensor([3, 17_000_000, 17_000_001, 18_000_000, 18_500_000, 19_000_000, 19_999_000, 19_999_988, 19_999_989, 0], device="cuda").sort().values
    tally[0, 0, gone] = 0.5
    pos, mark = torch.zeros(1, 1, Tcap, dtype=torch.int32, device="cuda"), torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    length = torch.tensor([Tcap], dtype=torch.int32, device="cuda")
    rs.cache_evict(s, k, v, tally, pos, mark, length, keep, 0, 10, 0, rs.Workspace(rs.cache_evict_workspace_bytes(s, keep)))
    torch.cuda.synchronize()
    assert torch.equal(k[0, 0, gone, 5], torch.arange(10.0, device="cuda") + 1) and torch.equal(v[0, 0, gone, 63], torch.arange(10.0, device="cuda") + 21)
    assert torch.equal(pos[0, 0, gone], torch.arange(keep, Tcap, device="cuda", dtype=torch.int32)) and int(length) == keep
    assert int((k[0, 0, :keep, 0] != 0).sum()) == 10 and mark.tolist() == [[keep, Tcap]]
