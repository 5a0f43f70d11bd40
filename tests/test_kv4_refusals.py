"""What the calls of a 4-bit cache, of the tally and of eviction refuse before anything is enqueued, and the model that their GPU tests go by."""
import ctypes
import inspect

import numpy as np
import pytest
import torch

import kv4_model as M
from paper_2605_28640_amd import binding as rs

A = 1 << 20  # an aligned made-up address
BIG = 1 << 40
BF = rs.RS_BF16


def _shape(B=2, Hq=4, Hkv=2, D=64, Tcap=256, P=16, dtype=BF):
    return ctypes.byref(rs.make_shape(B, Hq, Hkv, D, Tcap, P, dtype))


CALLS = {  # arguments between the shape and the stream
    "kv4_append": dict(k=A, v=A, T_src=20, t_src=3, len=A, n_new=A, T_new=17, k4=A, k4_scale=A, v4=A, v4_scale=A, meta=A),
    "kv4_page_meta": dict(k4=A, k4_scale=A, len=A, n_new=A, T_new=17, meta=A),
    "kv4_fetch": dict(k4=A, k4_scale=A, v4=A, v4_scale=A, len=A, t0=0, T=9, k_out=A, v_out=A),
    "kv4_attn_decode": dict(q=A, k4=A, k4_scale=A, v4=A, v4_scale=A, len=A, scale=0.1, idx=None, H_idx=0, K=0, tally=A, n_fresh=1, out=A, lse=A, ws=A,
                            nb=BIG),
    "attn_decode_tally": dict(q=A, k=A, v=A, len=A, scale=0.1, tally=A, n_fresh=1, out=A, lse=A, ws=A, nb=BIG),
    "cache_evict": dict(k=A, v=A, tally=A, pos=A, mark=A, len=A, n_keep=40, n_first=4, n_recent=8, n_slack=0, ws=A, nb=BIG),
    "kv4_evict": dict(k4=A, k4_scale=A, v4=A, v4_scale=A, tally=A, pos=A, mark=A, len=A, n_keep=40, n_first=4, n_recent=8, n_slack=0, ws=A, nb=BIG),
}
MAY_BE_NULL = {"n_new", "lse", "idx"}
NULL_TOO = {"kv4_append": {"meta"}, "kv4_attn_decode": {"tally"}}
NUMBERS = {"T_src", "t_src", "T_new", "t0", "T", "scale", "H_idx", "K", "n_fresh", "nb", "n_keep", "n_first", "n_recent", "n_slack"}


def call(name, shape=None, **other):
    args = dict(CALLS[name], **other)
    return getattr(rs.load(), name)(shape or _shape(), *args.values(), None)


@pytest.mark.parametrize("name", CALLS)
def test_pointers(name):
    for arg in CALLS[name]:
        if arg in NUMBERS:
            continue
        bad = 3 if arg == "ws" else 1
        assert call(name, **{arg: A + 4}) == bad, arg
        if arg not in MAY_BE_NULL | NULL_TOO.get(name, set()):
            assert call(name, **{arg: None}) == bad, arg


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("bad,status", [(dict(D=96), 2), (dict(dtype=2), 2), (dict(B=0), 1), (dict(Hq=3), 1), (dict(Tcap=0), 1), (dict(Hq=8162, Hkv=2), 2),
                                        (dict(Tcap=(1 << 30) + 512), 2)])
def test_shapes(name, bad, status):
    assert call(name, _shape(**bad)) == status


def test_numbers():
    for bad in (dict(T_new=0), dict(T_new=257, T_src=300), dict(T_src=19), dict(t_src=-1), dict(t_src=4), dict(T_src=0)):
        assert call("kv4_append", **bad) == 1, bad
    for bad in (dict(T_new=0), dict(T_new=257)):
        assert call("kv4_page_meta", **bad) == 1, bad
    for bad in (dict(T=0), dict(t0=256), dict(t0=-257)):
        assert call("kv4_fetch", **bad) == 1, bad
    lists = dict(idx=A, tally=None, H_idx=4, K=5)
    for bad in (dict(lists, H_idx=3), dict(lists, K=0), dict(lists, K=17), dict(lists, H_idx=0), dict(lists, K=-1), dict(lists, tally=A), dict(lists, idx=A + 4),
                dict(n_fresh=-1)):
        assert call("kv4_attn_decode", **bad) == 1, bad
    assert call("attn_decode_tally", n_fresh=-1) == 1
    for name in ("cache_evict", "kv4_evict"):
        for bad in (dict(n_keep=0), dict(n_keep=257), dict(n_first=-1), dict(n_recent=-1), dict(n_slack=-1), dict(n_first=33), dict(n_recent=37),
                    dict(n_first=2 ** 31 - 1, n_recent=2 ** 31 - 1)):
            assert call(name, **bad) == 1, (name, bad)
    # pages
    for name in ("kv4_append", "kv4_page_meta"):
        assert call(name, _shape(P=24, Tcap=240)) == 2 and call(name, _shape(Tcap=250)) == 1
    assert call("kv4_attn_decode", _shape(P=24, Tcap=240), **lists) == 2
    # more (sequence, head) pairs, or sequences, than the grids take
    for name in ("kv4_append", "kv4_page_meta", "kv4_fetch", "cache_evict", "kv4_evict"):
        assert call(name, _shape(B=32768, Hq=2, Hkv=2)) == 2, name
    for name in ("kv4_attn_decode", "attn_decode_tally"):
        assert call(name, _shape(B=1025, Hq=2, Hkv=2)) == 2, name
        assert call(name, _shape(B=1024, Hq=64, Hkv=64, Tcap=1 << 30)) == 2, name


def test_workspaces():
    lib = rs.load()
    s = _shape()
    for name, need in (("kv4_attn_decode", lib.kv4_attn_decode_workspace_bytes(s, 0, 0, 1)), ("attn_decode_tally", lib.attn_decode_tally_workspace_bytes(s)),
                       ("cache_evict", lib.cache_evict_workspace_bytes(s, 40)), ("kv4_evict", lib.cache_evict_workspace_bytes(s, 40))):
        assert need > rs.RS_WS_CTRL_BYTES and call(name, nb=need - 1) == 3 and call(name, nb=0) == 3, name
    # lists and no tally need no scores
    assert lib.kv4_attn_decode_workspace_bytes(s, 4, 16, 0) == lib.kv4_attn_decode_workspace_bytes(s, 0, 0, 0) < lib.kv4_attn_decode_workspace_bytes(s, 0, 0, 1)
    bad = _shape(D=96)
    assert lib.kv4_attn_decode_workspace_bytes(bad, 0, 0, 0) == lib.attn_decode_tally_workspace_bytes(bad) == lib.cache_evict_workspace_bytes(bad, 40) == 0
    assert lib.cache_evict_workspace_bytes(s, 0) == lib.cache_evict_workspace_bytes(s, 257) == lib.kv4_attn_decode_workspace_bytes(s, 3, 4, 0) == 0


@pytest.mark.parametrize("name,names", [
    ("kv4_append", "s k v t_src len n_new T_new k4 k4_scale v4 v4_scale meta"),
    ("kv4_page_meta", "s k4 k4_scale len n_new T_new meta"),
    ("kv4_fetch", "s k4 k4_scale v4 v4_scale len t0 T k_out v_out"),
    ("kv4_attn_decode_workspace_bytes", "s H_idx K with_tally"),
    ("kv4_attn_decode", "s q k4 k4_scale v4 v4_scale len scale idx tally n_fresh out lse_out ws"),
    ("attn_decode_tally_workspace_bytes", "s"),
    ("attn_decode_tally", "s q k_cache v_cache len scale tally n_fresh out lse_out ws"),
    ("cache_evict_workspace_bytes", "s n_keep"),
    ("cache_evict", "s k_cache v_cache tally pos mark len n_keep n_first n_recent n_slack ws"),
    ("kv4_evict", "s k4 k4_scale v4 v4_scale tally pos mark len n_keep n_first n_recent n_slack ws"),
])
def test_signatures(name, names):
    assert list(inspect.signature(getattr(rs, name)).parameters) == names.split()
    if name.endswith("_bytes"):
        return
    # as native.cpp takes it: the same number of arguments; what is not of its plain type is left unmade
    fast, n = getattr(rs._calls(), name), len(names.split())
    assert fast(*[0.5] * n) is False
    for wrong in (n - 1, n + 1):
        with pytest.raises(TypeError):
            fast(*[None] * wrong)


def test_binding_looks_at_types_and_shapes():
    s = rs.make_shape(2, 4, 2, 64, 32, 16, torch.bfloat16)
    z, i32, u8, bf = torch.zeros, torch.int32, torch.uint8, torch.bfloat16
    four = [z(2, 2, 32, n, dtype=u8) for n in (32, 2, 32, 2)]
    ln, ws = z(2, dtype=i32), rs.Workspace.__new__(rs.Workspace)
    wrong = rs.RatsparseError
    with pytest.raises(wrong):  # float32 rows in a bfloat16 shape
        rs.kv4_append(s, z(2, 2, 4, 64), z(2, 2, 4, 64), 0, ln, None, 4, *four, None)
    with pytest.raises(wrong):
        rs.kv4_page_meta(s, z(2, 2, 32, 64, dtype=u8), four[1], ln, None, 1, None)
    with pytest.raises(wrong):
        rs.kv4_fetch(s, z(2, 2, 32, 32, dtype=torch.int8), *four[1:], ln, 0, 4, None, None)
    with pytest.raises(wrong):
        rs.kv4_attn_decode(s, z(2, 4, 1, 64, dtype=bf), *four, ln, 0.1, None, None, 1, None, None, ws)
    with pytest.raises(wrong):
        rs.attn_decode_tally(s, z(2, 4, 64), None, None, ln, 0.1, None, 1, None, None, ws)
    with pytest.raises(wrong):
        rs.cache_evict(s, z(2, 2, 32, 32, dtype=bf), None, None, None, None, ln, 4, 0, 0, 0, ws)
    with pytest.raises(wrong):
        rs.kv4_evict(s, four[1], *four[1:], None, None, None, ln, 4, 0, 0, 0, ws)
    for shape in ((2, 2, 0), (2, 0, 4)):  # a list of no pages is not the same as none
        with pytest.raises(wrong, match="no pages"):
            rs.kv4_attn_decode(s, z(2, 4, 64, dtype=bf), *four, ln, 0.1, z(*shape, dtype=i32), None, 1, z(2, 4, 64, dtype=bf), None, ws)
    with pytest.raises(AssertionError):  # not on a device
        rs.kv4_page_meta(s, four[0], four[1], ln, None, 1, None)


def test_the_model():
    x = np.array([[0.0, 0.25, 0.26, 0.75, 1.25, 2.5, 3.5, 5.0, 5.01, 7.0, -0.1, -7.0] + [0.0] * 20])
    code, byte = M.pack(x)
    assert byte.tolist() == [[127]] and M.values(code, byte)[0, :12].tolist() == [0, 0, 0.5, 1, 1, 2, 4, 4, 6, 6, 0, -6]
    assert M.from_bytes(M.to_bytes(code)).tolist() == code.tolist()
    assert M.pack(np.full((1, 32), 7.01))[1].tolist() == [[128]] and M.pack(np.zeros((1, 32)))[1].tolist() == [[2]]
    code, byte = M.pack(np.array([[np.inf] + [1.0] * 31, [3.4e38] * 32, [2.0 ** -126] * 32]))
    assert byte[:, 0].tolist() == [255, 252, 2] and np.isnan(M.values(code, byte)[0]).all() and (M.values(code, byte)[2] == 2.0 ** -126).all()
    pairs, at = M.evict([5, 1, 1, 0, 9, 1], [0] * 6, 0, 0, 6, 3, 0, 0, 0)  # 9, 5 and the first 1
    assert pairs == [(4, 2)] and at == [0, 1, 4]
    pairs, at = M.evict([0, 1, np.nan, 7], [3, 0, 9, 0], 3, 10, 4, 2, 1, 1, 0)  # positions 3, 0, 9, 10: the first and the newest
    assert pairs == [(3, 0)] and at == [10, 0]
    assert M.evict([1.0] * 5, [0] * 5, 0, 0, 5, 4, 0, 0, 1) is None


def test_bounds_of_no_pages_are_not_the_same_as_none():
    s = rs.make_shape(2, 4, 2, 64, 32, 64, torch.bfloat16)  # a page is longer than the cache
    z, bf = torch.zeros, torch.bfloat16
    four = [z(2, 2, 32, n, dtype=torch.uint8) for n in (32, 2, 32, 2)]
    with pytest.raises(rs.RatsparseError, match="no pages"):
        rs.kv4_append(s, z(2, 2, 4, 64, dtype=bf), z(2, 2, 4, 64, dtype=bf), 0, z(2, dtype=torch.int32), None, 4, *four, z(2, 2, 0, 2, 64, dtype=bf))


def test_limits():
    lib = rs.load()
    # an eviction's sequences: a control word each
    for name in ("cache_evict", "kv4_evict"):
        assert call(name, _shape(B=16320, Hq=1, Hkv=1), nb=0) == 3 and call(name, _shape(B=16321, Hq=1, Hkv=1)) == 2, name
    assert lib.cache_evict_workspace_bytes(_shape(B=16320, Hq=1, Hkv=1), 40) > 0 == lib.cache_evict_workspace_bytes(_shape(B=16321, Hq=1, Hkv=1), 40)
    # the attention's second launch: a workgroup a query, and 1024 rows of a KV head
    for need in (lib.attn_decode_tally_workspace_bytes, lambda s: lib.kv4_attn_decode_workspace_bytes(s, 0, 0, 1)):
        assert need(_shape(B=1, Hq=1600, Hkv=1600, Tcap=10 << 20)) > 0 == need(_shape(B=1, Hq=1700, Hkv=1700, Tcap=10 << 20))
