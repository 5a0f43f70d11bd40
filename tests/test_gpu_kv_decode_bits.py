"""One token's attention over caches in 4 bits, bfloat16 and float32: weights keep all of their bits, very large and
infinite queries.  Against a computation in 64 bits.

What is allowed: a score's rounding makes a weight off by M.rounding (relative to it, so the result by that times sum p |v|); a bfloat16 result is
rounded once (2^-8 of it)."""
import numpy as np
import pytest
import torch

import kv4_model as M
from gpu_util import say
from test_gpu_kv_decode import KINDS, Decode

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
