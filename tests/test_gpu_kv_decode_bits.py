"""One token's attention over caches in 4 bits, bfloat16 and float32: weights keep all of their bits, very large and
infinite queries, lines whose shares are not alike, rows that are not finite in tiles that are cut, tallies of replays.  Against a computation in 64 bits.

What is allowed: a score's rounding makes a weight off by M.rounding (relative to it, so the result by that times sum p |v|); a bfloat16 result is
rounded once (2^-8 of it)."""
import numpy as np
import pytest
import torch

import kv4_model as M
from gpu_util import say, tdtype
from test_gpu_kv_decode import KINDS, Decode, _values

pytestmark = pytest.mark.gpu


def last_rounding(out):
    return 2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -24


def check(d, idx=None):
    """Decode.check without a rounding of the weights."""
    s, G = d.s, d.s.Hq // d.s.Hkv
    q, out, lse = (x.double().cpu().numpy() for x in (d.q, d.out, d.lse))
    for b, L in enumerate(d.lens):
        for h in range(s.Hq):
            t = np.arange(L)
            if idx is not None:
                pages = idx[b, h * idx.shape[1] // s.Hq].cpu().numpy()
                t = (pages[:, None] * s.P + np.arange(s.P)).ravel()
                t = t[t < L]
            o, z, _, a, most = M.attention(q[b, h:h + 1], d.k[b, h // G, t], d.v[b, h // G, t], d.scale)
            e = M.rounding(most[0], len(t), d.D)
            assert np.all(np.abs(out[b, h] - o[0]) <= e * a[0] + last_rounding(d.out) * np.abs(o[0]) + 1e-30), (b, h, L)
            assert z[0] == lse[b, h] or abs(lse[b, h] - z[0]) <= e + 2.0 ** -22 * abs(z[0]), (b, h, L)


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("shape", [(2, 4, 2, 64, 256, [200, 3]), (1, 8, 1, 128, 128, [127]), (2, 4, 4, 128, 5000, [5000, 700]), (2, 6, 2, 64, 3000, [2999, 1]),
                                   (2, 40, 2, 128, 1500, [1500, 33])])
def test_weights_keep_their_bits(rs, kind, dtype, shape):
    """Rows of nearly equal weight, whose values nearly cancel: a weight of fewer bits than 24 shows in the result."""
    B, Hq, Hkv, D, Tcap, lens = shape
    say("bits", kind, dtype, shape)
    d = Decode(rs, kind, dtype, B, Hq, Hkv, D, Tcap, lens, seed=31, big=0.05)
    d.run()
    check(d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("K", [5, 90])
def test_weights_of_listed_pages_keep_their_bits(rs, dtype, shared, K):
    say("bits, listed", dtype, shared, K)
    d = Decode(rs, "four", dtype, 2, 8, 2, 128, 2048, [2048, 1999], seed=32, big=0.05)
    r = np.random.default_rng(K)
    idx = np.stack([[r.permutation(128)[:K] for _ in range(2 if shared else 8)] for _ in range(2)]).astype(np.int32)
    idx = torch.from_numpy(idx).cuda()
    d.run(tally=False, idx=idx)
    check(d, idx)

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Tcap,L", [(300, 300), (5000, 4999)])  # one launch, two
@pytest.mark.parametrize("listed", [False, True])
def test_very_large_and_infinite_queries_of_a_4_bit_cache(rs, dtype, Tcap, L, listed):
    """A finite query channel next to the end of its type's range counts as it is (rows have nothing there); one of -inf against positive values: the row sees nothing;
    one of +inf: NaN, as the formula has it."""
    say("large queries", dtype, Tcap, listed)
    Tcap = -(-Tcap // 16) * 16
    d = Decode(rs, "four", dtype, 3, 2, 2, 64, Tcap, [L] * 3, seed=13)
    codes = d.cache[0]
    codes[:, :, :, 5 // 2] = codes[:, :, :, 5 // 2] & 0x0F        # channel 5: 0
    codes[:, :, :, 7 // 2] = codes[:, :, :, 7 // 2] & 0x0F | 0x20  # channel 7: 1 times the scale
    four = [x.cpu().numpy() for x in d.cache]
    d.k, d.v = (M.values(M.from_bytes(c), f) for c, f in zip(four[0::2], four[1::2]))
    d.q[0, :, 5] = torch.finfo(d.q.dtype).max
    d.q[0, 1, 5] *= -1
    d.q[1, 0, 7] = -float("inf")
    d.q[2, 0, 7] = float("inf")
    d.tally.zero_()
    idx = torch.arange(L // 16, dtype=torch.int32, device="cuda").repeat(3, 2, 1) if listed else None
    d.run(tally=not listed, fresh=0, idx=idx)
    assert (d.out[1, 0] == 0).all() and d.lse[1, 0] == -float("inf") and (d.tally[1, 0] == 0).all()
    assert d.out[2, 0].isnan().all() and d.lse[2, 0].isnan()
    for b, h in ((0, 0), (0, 1), (1, 1), (2, 1)):
        n = L // 16 * 16 if listed else L
        q = d.q[b, h:h + 1].double().cpu().numpy()
        o, z, p, a, most = M.attention(q, d.k[b, h, :n], d.v[b, h, :n], d.scale)
        e = M.rounding(most[0], n, 64)
        assert np.all(np.abs(d.out[b, h].double().cpu().numpy() - o[0]) <= e * a[0] + last_rounding(d.out) * np.abs(o[0])), (b, h)
        assert abs(float(d.lse[b, h]) - z[0]) <= e + 2.0 ** -22 * abs(z[0]), (b, h)
        if not listed:
            assert np.all(np.abs(d.tally[b, h, :n].double().cpu().numpy() - p[0]) <= e * p[0] + 2.0 ** -22 * p[0]), (b, h)


def check_on_device(q, dev, scale, idx, P, lens, out, lse):
    """A 4-bit cache's outputs against 64 bits on the device, and the weights that a sequence's tally gets [Hkv, L] (no lists)."""
    B, Hq, D = q.shape
    Hkv = dev[0].shape[1]
    H = idx.shape[1] if idx is not None else Hkv
    weights = []
    for b in range(B):
        k, v = (_values(dev[i][b, :, :lens[b]], dev[i + 1][b, :, :lens[b]]) for i in (0, 2))
        per = []
        for h in range(H):
            kk, vv = k[h * Hkv // H], v[h * Hkv // H]
            if idx is not None:
                pages = idx[b, h][idx[b, h] >= 0].long()
                t = (pages[:, None] * P + torch.arange(P, device="cuda")).flatten()
                t = t[t < lens[b]]
                kk, vv = kk[t], vv[t]
            g = slice(h * Hq // H, (h + 1) * Hq // H)
            qq = q[b, g].double()
            z = (qq @ kk.t().contiguous()) * scale
            want = torch.logsumexp(z, -1)
            p = torch.exp(z - want[:, None])
            o, a = p @ vv, p @ vv.abs()
            e = M.rounding(float(((qq.abs() @ kk.abs().t().contiguous()) * scale).max()), kk.shape[0], D)
            assert ((out[b, g].double() - o).abs() <= e * a + last_rounding(out) * o.abs()).all(), (b, h)
            assert ((lse[b, g].double() - want).abs() <= e + 2.0 ** -22 * want.abs()).all(), (b, h)
            per.append((p.sum(0), e))
        weights.append(per)
    return weights


def random_cache(B, Hkv, Tcap, D, g):
    return [torch.randint(lo, hi, (B, Hkv, Tcap, n), dtype=torch.uint8, device="cuda", generator=g) for lo, hi, n in
            ((0, 256, D // 2), (121, 126, D // 32), (0, 256, D // 2), (121, 126, D // 32))]


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("K", [252, 256, 260])  # 128 lists of 63, 64, 65 units of 64 tokens: below, at and above what the shares are weighted from
def test_lists_of_many_units(rs, dtype, D, shared, K):
    say("lists of many units", dtype, shared, K)
    B, H, Tcap, P, lens = 4, 32, 8192, 16, [8192, 8000, 4163, 8191]
    dt = tdtype(dtype)
    g = torch.Generator(device="cuda").manual_seed(K)
    s = rs.make_shape(B, 64 if shared else 32, H, D, Tcap, P, dt)
    dev = random_cache(B, H, Tcap, D, g)
    q = torch.randn(B, s.Hq, D, device="cuda", generator=g).to(dt)
    idx = torch.rand(B, H, Tcap // P, device="cuda", generator=g).topk(K, -1).indices.int()
    idx[1, :, 3::7] = -1
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(B, s.Hq, device="cuda")
    ws = rs.Workspace(rs.kv4_attn_decode_workspace_bytes(s, H, K, False))
    for _ in range(2):  # (its records from the call before are there the second time)
        rs.kv4_attn_decode(s, q, *dev, ln, 0.09, idx, None, 0, out, lse, ws)
        check_on_device(q, dev, 0.09, idx, P, lens, out, lse)


@pytest.mark.parametrize("tally", [False, True])
def test_many_units_a_wave_float32(rs, tally):
    """64 channels in float32: three workgroups a CU too."""
    B, Hq, Hkv, D, lens = 4, 32, 16, 64, [9000, 8191, 8999, 8200]
    Tcap = 9008
    g = torch.Generator(device="cuda").manual_seed(5)
    s = rs.make_shape(B, Hq, Hkv, D, Tcap, 16, torch.float32)
    dev = random_cache(B, Hkv, Tcap, D, g)
    q = torch.randn(B, Hq, D, device="cuda", generator=g)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    before = torch.rand(B, Hkv, Tcap, device="cuda", generator=g)
    got = before.clone()
    out, lse = torch.zeros_like(q), torch.zeros(B, Hq, device="cuda")
    rs.kv4_attn_decode(s, q, *dev, ln, 0.12, None, got if tally else None, 1, out, lse, rs.Workspace(rs.kv4_attn_decode_workspace_bytes(s, 0, 0, tally)))
    weights = check_on_device(q, dev, 0.12, None, 16, lens, out, lse)
    for b, L in enumerate(lens) if tally else ():
        for h, (p, e) in enumerate(weights[b]):
            want = before[b, h, :L].double()
            want[L - 1] = 0
            want += p
            assert ((got[b, h, :L].double() - want).abs() <= e * p + 2.0 ** -22 * want).all() and torch.equal(got[b, h, L:], before[b, h, L:])


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("t", [0, 2500, 4998])
def test_values_that_are_not_finite_in_a_tile_that_is_cut(rs, kind, dtype, t):
    """NaN in one row of K or V, where the row's share is one of many: it shows in its head's results, and nowhere else."""
    d = Decode(rs, kind, dtype, 2, 4, 2, 64, 5000, [5000, 4999], seed=14)
    d.run()
    out, lse, tally = d.out.clone(), d.lse.clone(), d.tally.clone()
    for i in (0, 1):  # K, V
        x = d.cache[2 * i + 1 if kind == "four" else i]
        kept = x[1, 0, t].clone()
        x[1, 0, t] = 255 if kind == "four" else float("nan")
        d.tally.zero_()
        d.run(fresh=0)
        x[1, 0, t] = kept
        assert d.out[1, :2].isnan().all() and torch.equal(d.out[0], out[0]) and torch.equal(d.out[1, 2:], out[1, 2:])
        assert torch.equal(d.lse[0], lse[0]) and torch.equal(d.lse[1, 2:], lse[1, 2:])
        assert not d.tally[0].isnan().any() and not d.tally[1, 1].isnan().any() and (d.tally[1, 0, 4999:] == 0).all()
        if i == 0:
            assert d.lse[1, :2].isnan().all() and d.tally[1, 0, :4999].isnan().all()
        else:
            assert torch.equal(d.lse, lse) and not d.tally.isnan().any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_scores_in_tiles_that_are_cut(rs, dtype):
    """Shares of rows that all have a score of -inf add nothing; where all rows have one, the row sees nothing; +inf is NaN, as the formula has it."""
    d = Decode(rs, "rows", dtype, 3, 2, 2, 64, 5000, [5000, 4999, 5000], seed=15)
    d.q.fill_(1.0)
    k = d.cache[0]
    k[0, 0, :4990, 5] = -float("inf")
    k[0, 1, 10:, 5] = -float("inf")
    k[1, 0, :, 7] = -float("inf")
    k[2, 0, 2000, 9] = float("inf")
    d.tally.zero_()
    d.run(fresh=0)
    assert d.out[0].isfinite().all() and (d.tally[0, 0, :4990] == 0).all() and (d.tally[0, 1, 10:] == 0).all()
    assert ((d.tally[0].sum(-1) - 1).abs() < 1e-5).all()
    assert (d.out[1, 0] == 0).all() and d.lse[1, 0] == -float("inf") and (d.tally[1, 0] == 0).all()
    assert d.out[2, 0].isnan().all() and d.out[1:, 1].isfinite().all()


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_tallies_of_two_graphs_that_share_a_workspace(rs, kind, dtype):
    """Every replay adds the weights of its own scores, whatever the other graph or an eager call left in the workspace."""
    a = Decode(rs, kind, dtype, 3, 8, 2, 128, 1900, [1900, 5, 500], seed=23)
    b = Decode(rs, kind, dtype, 2, 4, 4, 128, 1400, [123, 1400], seed=24)
    need = []
    for d in (a, b):
        d.run(fresh=0)
        need.append(d.ws.nbytes)
    ws = (a, b)[need[1] > need[0]].ws
    graphs = []
    for d in (a, b):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            (rs.kv4_attn_decode if kind == "four" else rs.attn_decode_tally)(
                d.s, d.q, *d.cache, d.len, d.scale, *((None,) if kind == "four" else ()), d.tally, 0, d.out, d.lse, ws)
        graphs.append(g)
    for turn in range(3):
        for d, other, g in zip((a, b), (b, a), graphs):
            before = d.tally.clone()
            d.out.fill_(9)
            d.lse.fill_(9)
            g.replay()
            torch.cuda.synchronize()
            d.check(before, 0)
            if turn == 1:
                other.run(fresh=0, ws=ws)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Tcap,L", [(64, 1), (300, 300), (5000, 4999)])
@pytest.mark.parametrize("big", [0.0, 1.0])
def test_infinite_values(rs, dtype, Tcap, L, big):
    """An infinite value with a weight, also one of few bits (rows of equal scores), is an infinite result, as the formula has it; of both signs: NaN."""
    say("infinite values", dtype, Tcap, L, big)
    d = Decode(rs, "rows", dtype, 2, 4, 2, 64, Tcap, [L, L], seed=16, big=big)
    t = L // 2
    for h in (0, 1):
        d.cache[1][0, h, t, 3] = float("inf")
        d.cache[1][0, h, L - 1, 60] = -float("inf")
        d.v[0, h, t, 3] = d.v[0, h, L - 1, 60] = 0
    if L > 1:
        d.cache[1][0, 1, t + 1, 3] = -float("inf")
        d.v[0, 1, t + 1, 3] = 0
    before = d.tally.clone()
    d.run()
    a, b = d.out[0, :2].clone(), d.out[0, 2:].clone()
    assert (a[:, 3] == float("inf")).all() and (a[:, 60] == -float("inf")).all() and (b[:, 60] == -float("inf")).all()
    assert (b[:, 3].isnan() if L > 1 else b[:, 3] == float("inf")).all()
    # the other channels, and all else, as ever
    for c in (3, 60):
        d.out[0, :, c] = 0
        d.v[0, :, :, c] = 0
    check(d)
    assert d.lse.isfinite().all() and not d.tally.isnan().any() and torch.equal(d.tally[:, :, L:], before[:, :, L:])
