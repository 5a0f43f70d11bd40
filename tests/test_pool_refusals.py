"""What the page pool's entry points refuse before anything is enqueued, and the model that their GPU tests go by."""
import ctypes

import pytest
import torch

from paper_2605_28640_amd import binding as rs
from pool_model import Pool

A = 1 << 20  # an aligned made-up address
BIG = 1 << 30
BF = rs.RS_BF16


def _pool(N=16, S=4, M=8, P=16):
    return ctypes.byref(rs.make_pool(N, S, M, P))


@pytest.mark.parametrize("bad,status", [((0, 4, 8, 16), 1), ((16, 0, 8, 16), 1), ((16, 4, -1, 16), 1), ((16, 4, 8, 24), 2),
                                        ((16, 32769, 8, 16), 2), ((1 << 28, 4, 8, 16), 2), ((16, 4, 1 << 28, 16), 2)])
def test_pools(bad, status):
    lib, p = rs.load(), _pool(*bad)
    s = ctypes.byref(rs.make_shape(2, 4, 2, 64, 256, 16, BF))
    assert lib.page_pool_workspace_bytes(p) == 0 and lib.attn_paged_workspace_bytes(s, p, 1) == 0
    assert lib.page_pool_reserve(p, A, A, A, A, 1, None, 1, None, A, BIG, None) == status
    assert lib.page_pool_fork(p, A, A, A, A, A, 1, A, None, A, BIG, None) == status
    assert lib.page_pool_free(p, A, A, A, A, 1, A, BIG, None) == status
    assert lib.page_pool_compact(p, A, A, A, A, A, A, BIG, None) == status
    assert lib.page_pool_share(p, A, A, A, 1, 1, A, None) == status
    assert lib.rat_append_paged(s, p, A, A, A, A, A, A, A, None, A, A, A, None, 1, None) == status
    assert lib.attn_paged(s, p, A, A, A, A, A, A, None, 1, None, 0.1, A, None, A, BIG, None) == status


def test_pool_calls():
    lib, p = rs.load(), _pool()
    need = lib.page_pool_workspace_bytes(p)
    assert need > rs.RS_WS_CTRL_BYTES

    def reserve(table=A, len=A, refs=A, seq=A, n=1, want=None, T=1, granted=None, ws=A, nb=need):
        return lib.page_pool_reserve(p, table, len, refs, seq, n, want, T, granted, ws, nb, None)
    for bad in (dict(table=None), dict(len=None), dict(refs=None), dict(seq=None), dict(n=0), dict(n=5), dict(want=A + 4),
                dict(T=-1), dict(granted=A + 8), dict(refs=A + 4), dict(seq=A + 4)):
        assert reserve(**bad) == 1, bad
    assert reserve(nb=need - 1) == 3 and reserve(ws=None) == 3

    def fork(src=A, dst=A, n=1, pairs=A, carry=A, ws=A, nb=need):
        return lib.page_pool_fork(p, A, A, A, src, dst, n, pairs, carry, ws, nb, None)
    for bad in (dict(src=None), dict(dst=None), dict(pairs=None), dict(pairs=A + 4), dict(carry=A + 8), dict(n=0), dict(n=5)):
        assert fork(**bad) == 1, bad
    assert fork(nb=need - 1) == 3
    assert lib.page_pool_free(p, A, A, A, None, 1, A, need, None) == 1
    assert lib.page_pool_free(p, A, A, A, A, 5, A, need, None) == 1
    assert lib.page_pool_free(p, A, A, A, A, 1, A, need - 1, None) == 3
    assert lib.page_pool_compact(p, A, A, A, None, A, A, need, None) == 1
    assert lib.page_pool_compact(p, A, A, A, A, None, A, need, None) == 1
    assert lib.page_pool_compact(p, A, A, A, A, A, A, need - 1, None) == 3
    assert lib.page_pool_share(p, A, A, A, 1, 0, A, None) == 1
    assert lib.page_pool_share(p, A, A, A, 0, 1, A, None) == 1
    assert lib.page_pool_share(p, A, A, A, 1025, 1, A, None) == 2
    assert lib.page_pool_share(p, A, A, A, 1, 1, None, None) == 1


def test_copies():
    lib = rs.load()
    s = rs.make_shape(1, 2, 2, 64, 256, 16, BF)

    def copy(other=s, ks=A, vs=A, ms=A, kd=A, vd=A, md=A, pairs=A, n=1, count=None):
        return lib.page_copy(ctypes.byref(s), ks, vs, ms, ctypes.byref(other), kd, vd, md, pairs, n, count, None)
    for bad in (dict(ks=None), dict(vs=None), dict(kd=None), dict(vd=None), dict(ms=None), dict(md=None), dict(pairs=None),
                dict(pairs=A + 4), dict(count=A + 4), dict(n=0), dict(ks=A + 8)):
        assert copy(**bad) == 1, bad
    for other in ((1, 4, 4, 64, 256, 16, BF), (1, 2, 2, 128, 256, 16, BF), (1, 2, 2, 64, 256, 32, BF), (1, 2, 2, 64, 256, 16, rs.RS_F32),
                  (1, 2, 2, 64, 250, 16, BF)):
        assert copy(other=rs.make_shape(*other)) == 1, other
    assert copy(other=rs.make_shape(1, 2, 2, 96, 256, 16, BF)) == 2
    assert lib.rat_state_copy(ctypes.byref(s), None, A, 4, A, 1, None) == 1
    assert lib.rat_state_copy(ctypes.byref(s), A, A, 0, A, 1, None) == 1
    assert lib.rat_state_copy(ctypes.byref(s), A, A, 4, A, 0, None) == 1
    assert lib.rat_state_copy(ctypes.byref(s), A, A, 4, A + 4, 1, None) == 1


def test_append_and_attention():
    lib, p = rs.load(), _pool()
    s = ctypes.byref(rs.make_shape(2, 4, 2, 64, 256, 16, BF))
    args = dict(k=A, v=A, g=A, sk=A, sv=A, kp=A, vp=A, meta=A, table=A, len=A, seq=A, n_new=A, T=1)
    for bad in [{n: None} for n in ("k", "v", "g", "sk", "sv", "kp", "vp", "table", "len", "seq")] + [{n: A + 4} for n in args if n != "T"] + \
            [dict(T=0), dict(T=-3)]:
        assert lib.rat_append_paged(s, p, *{**args, **bad}.values(), None) == 1, bad
    args = dict(q=A, kp=A, vp=A, table=A, len=A, seq=A, n_new=A, T=1, share=A, scale=0.1, out=A, lse=A)
    need = lib.attn_paged_workspace_bytes(s, p, 1)
    for bad in [{n: None} for n in ("q", "kp", "vp", "table", "len", "seq", "out")] + \
            [{n: A + 4} for n in args if n not in ("T", "scale")] + [dict(T=0)]:
        assert lib.attn_paged(s, p, *{**args, **bad}.values(), A, need, None) == 1, bad
    assert lib.attn_paged(s, p, *args.values(), A, need - 1, None) == 3
    assert lib.attn_paged(s, p, *args.values(), None, need, None) == 3
    # a pool of another size than the shape's, and of another page size
    for other in ((15, 4, 8, 16), (8, 4, 8, 32)):
        q = _pool(*other)
        assert lib.attn_paged(s, q, *args.values(), A, BIG, None) == 1
        assert lib.rat_append_paged(s, q, A, A, A, A, A, A, A, A, A, A, A, A, 1, None) == 1
    many = ctypes.byref(rs.make_shape(1025, 2, 2, 64, 256, 16, BF))
    assert lib.attn_paged(many, p, *args.values(), A, 1 << 40, None) == 2 and lib.attn_paged_workspace_bytes(many, p, 1) == 0
    # more units of work than are counted in 32 bits
    huge, wide = ctypes.byref(rs.make_shape(1000, 8, 1, 64, 1 << 24, 512, BF)), _pool(1 << 15, 4, 1 << 21, 512)
    assert lib.attn_paged(huge, wide, *{**args, "T": 20000}.values(), A, 1 << 40, None) == 2
    # (rows of one sequence that fill a tile need no records of their own: the workspace grows no further)
    assert lib.attn_paged_workspace_bytes(s, p, 64) == lib.attn_paged_workspace_bytes(s, p, 6400)


def test_binding_looks_at_types_and_shapes():
    p, s = rs.make_pool(4, 2, 3, 16), rs.make_shape(1, 2, 2, 64, 64, 16, torch.bfloat16)
    i = lambda *n: torch.zeros(*n, dtype=torch.int32)
    ws = rs.Workspace.__new__(rs.Workspace)
    for t in (torch.zeros(2, 3), i(3, 2), torch.zeros(2, 3, dtype=torch.int64)):
        with pytest.raises(rs.RatsparseError):
            rs.page_pool_free(p, t, i(2), i(4), i(1), ws)
    with pytest.raises(AssertionError):  # not on a device
        rs.page_pool_free(p, i(2, 3), i(2), i(4), i(1), ws)
    with pytest.raises(rs.RatsparseError):
        rs.attn_paged(s, p, torch.zeros(1, 2, 1, 64), None, None, i(2, 3), i(2), i(1), None, 1, None, 0.1, None, None, ws)
    with pytest.raises(rs.RatsparseError):
        rs.rat_append_paged(s, p, torch.zeros(1, 2, 1, 64), *[None] * 7, i(2, 3), i(2), i(1), None, 1)


def test_statuses():
    assert b"pool" in rs.load().ratsparse_status_string(7)


def test_the_model():
    p = Pool(8, 4, 4, 16)
    assert p.reserve([0], [33]) and p.table[0] == [0, 1, 2, -1] and p.len[0] == 33
    taken, pairs, carry = p.fork([0, 0], [2, 1])
    assert taken and pairs == [[2, 3], [2, 4]] and carry == [[0, 2], [0, 1]] and p.refs == [3, 3, 1, 1, 1, 0, 0, 0]
    assert p.share([2, 1, 3], 1) == [[0, 2, 2], [0, 2, 2], [2, 1, 0]]
    assert not p.reserve([0, 0], [1, 1]) and not p.reserve([3], [65]) and not p.reserve([3, 1], [50, 16])
    assert p.free([0]) and p.refs == [2, 2, 0, 1, 1, 0, 0, 0]
    assert p.compact() == [[4, 2]] and p.table[1] == [0, 1, 2, -1] and p.refs == [2, 2, 1, 1, 0, 0, 0, 0]
    assert p.reserve([1], [15]) and p.len[1] == 48 and p.table[1] == [0, 1, 2, -1]


@pytest.mark.parametrize("name,names", [
    ("page_pool_reserve", "p table len refs seq want T_new granted ws"),
    ("page_pool_fork", "p table len refs src dst pairs_out carry_out ws"),
    ("page_pool_free", "p table len refs seq ws"),
    ("page_pool_compact", "p table len refs pairs_out n_pairs_out ws"),
    ("page_pool_share", "p table len seq min_pages share_out"),
    ("page_copy", "s_src k_src v_src meta_src s_dst k_dst v_dst meta_dst pairs n_pairs"),
    ("rat_state_copy", "s state_k state_v pairs"),
    ("rat_append_paged", "s p k v g state_k state_v k_pool v_pool meta table len seq n_new T_new"),
    ("attn_paged", "s p q k_pool v_pool table len seq n_new T_new share scale out lse_out ws"),
])
def test_signatures(name, names):
    """And the calls as native.cpp takes them: the same number of arguments; what is not of its plain type is left unmade."""
    import inspect
    assert list(inspect.signature(getattr(rs, name)).parameters) == names.split()
    fast, n = getattr(rs._calls(), name), len(names.split())
    assert fast(*[0.5] * n) is False
    for wrong in (n - 1, n + 1):
        with pytest.raises(TypeError):
            fast(*[None] * wrong)


def test_listed_heads_are_not_limited_by_control_words():
    """A list of 1024 sequences is taken whatever the heads; a contiguous call's B Hq is limited."""
    lib, p = rs.load(), _pool()
    s = ctypes.byref(rs.make_shape(1024, 64, 8, 64, 256, 16, BF))
    assert lib.attn_paged_workspace_bytes(s, p, 1) > 0 and lib.sparse_attn_decode_workspace_bytes(s, 256, 4) == 0
    need = lib.attn_paged_workspace_bytes(s, p, 1)
    assert lib.attn_paged(s, p, A, A, A, A, A, A, None, 1, None, 0.1, A, None, A, need - 1, None) == 3
    assert lib.page_copy(s, A, A, None, s, A, A, None, A, 0, None, None) == 1 and lib.rat_state_copy(s, A, A, 4, A, 0, None) == 1
    assert lib.rat_append_paged(s, p, A, A, A, A, A, A, A, None, A, A, A, None, 0, None) == 1
    # more heads than a sequence may have
    wide = ctypes.byref(rs.make_shape(1, 8161, 8161, 128, 256, 16, BF))
    assert lib.rat_append_paged(wide, p, A, A, A, A, A, A, A, None, A, A, A, None, 1, None) == 2
    assert lib.attn_paged_workspace_bytes(wide, p, 1) == 0 and lib.page_copy(wide, A, A, None, wide, A, A, None, A, 1, None, None) == 2
    assert lib.rat_state_copy(wide, A, A, 4, A, 1, None) == 2
    longer = ctypes.byref(rs.make_shape(32769, 2, 2, 64, 256, 16, BF))
    assert lib.rat_append_paged(longer, p, A, A, A, A, A, A, A, None, A, A, A, None, 1, None) == 2


def test_a_workspace_that_is_not_on_the_device():
    ws = rs.Workspace.__new__(rs.Workspace)
    ws.buf = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(AssertionError):
        rs._scratch(ws)
