"""How the causal and the shared-prefix attention cut their launches: the planners are host functions of libjf
(paper_2512_14681_amd/csrc/jf_internal.h), called here by their C++ names, without a GPU."""
import ctypes
import os

import pytest

from paper_2512_14681_amd import jf

I, P, SZ = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t


def _fields(text):
    kinds = {"i": I, "p": P, "z": SZ, "l": ctypes.c_int64}
    return [(n, kinds[k]) for k, names in (part.split(":") for part in text.split()) for n in names.split(",")]


class CausalArgs(ctypes.Structure):
    _fields_ = _fields("i:n_seqs,n_rows,H,G,hd p:row_start,flags,q,k,v z:ld_q,ld_k,ld_v i:vec p:out z:ld_out i:vec_out "
                       "p:lse i:f32,groups,blocks")


class CausalGradArgs(ctypes.Structure):
    _fields_ = [("f", CausalArgs)] + _fields("p:g_out z:ld_g_out i:vec_dot p:g_q,g_k,g_v z:ld_g_q,ld_g_k,ld_g_v i:vec_q,vec_kv "
                                             "p:dots,kv_part i:parts")


class BatchArgs(ctypes.Structure):
    _fields_ = _fields("i:n_seqs,n_rows,max_rows,max_ctx,n_pages,stride p:row_start,ctx,table,flags")


class SharedArgs(ctypes.Structure):
    _fields_ = [("b", BatchArgs)] + _fields(
        "i:n_groups,max_group_rows,max_pages p:seq_start,pages i:H,G,hd p:q z:q_plane p:kv,vis,out z:out_plane p:o_part,ml_part "
        "i:shared_few,own_few,shared_groups,own_groups,shared_splits,own_splits,parts l:shared_jobs64,own_jobs64 i:shared_jobs")


# Calls for both forms of the shared-prefix attention on either side, {(shared pages: four tiles of 32 queries a workgroup,
# the sequences' own: the same): (groups of (shared pages, [(own tokens, rows)]), (own tokens, rows) of sequences of no
# group, query heads, KV heads)}.
SHARED_TILES = {(True, True): ([(5, [(30, 140), (5, 2)]), (2, [(100, 7)])], [(64, 3)], 16, 2),
                (True, False): ([(4, [(70, 12)] * 7 + [(3, 60)]), (1, [(0, 1)])], [(200, 2)], 16, 2),
                (False, True): ([(3, [(9, 3)] * 4)], [(130, 150)], 16, 2),
                (False, False): ([(5, [(30, 40), (5, 2)]), (2, [(100, 7)])], [(64, 3)], 16, 2)}


# Calls for every kernel of the causal attention and its gradient, {(type, head_dim, rows of a block / 32): (rows of the
# sequences, query heads, KV heads)}: sequences of several blocks, with steps before the masked ones, and of a few rows.
NARROW, MIDDLE, WIDE = [400, 1, 130, 70], [400, 1, 130, 70], [400, 1, 130, 0] + [5] * 30
CAUSAL_BLOCKS = {(name, hd, n): call
                 for name in ("f32", "bf16") for hd in (32, 64, 128)
                 for n, call in ((1, (NARROW, 6, 2)), (2, (MIDDLE, 28, 4)), (4, (WIDE, 28, 4))) if n > 1 or hd < 128}


# Calls whose gradient sums a group's heads in so many shares: (type, rows of the sequences, query heads, KV heads, head_dim).
CAUSAL_SHARES = {1: ("bf16", [5] * 150 + [300], 28, 4, 64),     # one workgroup goes over all heads
                 4: ("bf16", [5] * 75 + [300], 28, 4, 128),     # 7 heads: shares of 2, 2, 2 and 1
                 8: ("f32", [5] * 35 + [300], 64, 4, 32)}       # 16 heads in pairs


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(jf.LIB_PATH):
        pytest.skip("libjf.so not built (python -m paper_2512_14681_amd.build)")
    return ctypes.CDLL(jf.LIB_PATH)


def causal_plan(L, n_seqs, n_rows, H, G, hd, f32):
    a = CausalArgs()
    a.n_seqs, a.n_rows, a.H, a.G, a.hd, a.f32 = n_seqs, n_rows, H, G, hd, f32
    f = L._ZN2jf11causal_planERNS_10CausalArgsE
    f.restype, f.argtypes = None, [ctypes.POINTER(CausalArgs)]
    f(ctypes.byref(a))
    return a


def grad_plan(L, n_seqs, n_rows, H, G, hd, f32):
    a = CausalGradArgs()
    a.f.n_seqs, a.f.n_rows, a.f.H, a.f.G, a.f.hd, a.f.f32 = n_seqs, n_rows, H, G, hd, f32
    f = L._ZN2jf16causal_grad_planERNS_14CausalGradArgsE
    f.restype, f.argtypes = None, [ctypes.POINTER(CausalGradArgs)]
    f(ctypes.byref(a))
    return a


ROWS = [*range(1, 40), *range(40, 2000, 61), *range(2000, 20000, 509), 40000, 100000]
SEQS = [1, 2, 3, 9, 33, 64, 65, 100, 1000]


@pytest.mark.parametrize("H,G,hd", [(28, 4, 128), (16, 2, 64), (4, 4, 32), (8, 1, 128), (64, 1, 64), (6, 2, 64)])
def test_a_larger_calls_gradient_workspace_holds_smaller_calls(L, H, G, hd):
    """Every call's need (two floats a row and head; the shares' gradients) is within what the size query gives for that
    call, and for any with more rows or sequences."""
    size = jf.lib().jf_attention_causal_grad_ws_bytes
    most = [0] * len(SEQS)
    for n in ROWS:
        for i, s in enumerate(SEQS):
            got = size(s, n, H, G, hd)
            for f32 in (0, 1):
                parts = grad_plan(L, s, n, H, G, hd, f32).parts
                assert 1 <= parts <= H // G
                assert got >= n * H * 8 + (2 * parts * n * G * hd * 4 if parts > 1 else 0)
            # all smaller counts are at or before this place of the lists
            assert got >= max(most[:i + 1]), (s, n)
            most[i] = max(most[:i + 1] + [got])


@pytest.mark.parametrize("name,hd,n", CAUSAL_BLOCKS, ids=lambda x: str(x))
def test_every_block_height_has_a_case(L, name, hd, n):
    """Which calls of CAUSAL_BLOCKS run on blocks of which height, forward and gradient; there are no others."""
    lens, H, G = CAUSAL_BLOCKS[name, hd, n]
    f32 = int(name == "f32")
    fwd, grad = causal_plan(L, len(lens), sum(lens), H, G, hd, f32), grad_plan(L, len(lens), sum(lens), H, G, hd, f32)
    assert (fwd.groups, grad.f.groups) == (n, n)
    assert grad.parts == H // G     # a join of several shares as well


def test_no_other_block_heights(L):
    for f32 in (0, 1):
        for hd in (32, 64, 128):
            seen = set()
            for H in (1, 4, 28, 64):
                for rows in (1, 60, 500, 3000, 20000):
                    for seqs in (1, 4, 80):
                        seen.add(causal_plan(L, seqs, rows, H, 1, hd, f32).groups)
                        seen.add(grad_plan(L, seqs, rows, H, 1, hd, f32).f.groups)
            assert seen == {n for t, d, n in CAUSAL_BLOCKS if (t, d) == (("bf16", "f32")[f32], hd)}


@pytest.mark.parametrize("parts", CAUSAL_SHARES)
def test_every_kind_of_share_has_a_case(L, parts):
    name, lens, H, G, hd = CAUSAL_SHARES[parts]
    assert grad_plan(L, len(lens), sum(lens), H, G, hd, int(name == "f32")).parts == parts


@pytest.mark.parametrize("wide", SHARED_TILES, ids=str)
def test_every_form_of_shared_prefixes_has_a_case(L, wide):
    """Which form the calls of SHARED_TILES take on either side."""
    groups, loners, H, G = SHARED_TILES[wide]
    members = [(p, c, r) for p, seqs in groups for c, r in seqs] + [(0, c, r) for c, r in loners]
    a = SharedArgs()
    a.b.n_seqs, a.b.n_rows = len(members), sum(r for _, _, r in members)
    a.b.max_rows, a.b.max_ctx = max(r for _, _, r in members), max(64 * p + c + r for p, c, r in members)
    a.n_groups, a.H, a.G, a.hd = len(groups), H, G, 64
    a.max_group_rows = max(sum(r for _, r in seqs) for p, seqs in groups)
    a.max_pages = max(p for p, _ in groups)
    f = L._ZN2jf11shared_planERNS_10SharedArgsE
    f.restype, f.argtypes = None, [ctypes.POINTER(SharedArgs)]
    f(ctypes.byref(a))
    assert (not a.shared_few, not a.own_few) == wide
    assert a.parts == a.shared_splits + a.own_splits > 1
