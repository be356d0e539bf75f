"""The 4-bit cache's format and the page tables: the oracle against brute force, and what the entry points refuse on the host."""
import ctypes as C

import numpy as np
import pytest

from oracle import ref
from paper_2608_04962_b200 import binding as S
from paper_2608_04962_b200 import build as B


def test_scales_cover_32_binades_in_order():
    steps = ref.KV4_STEPS
    assert steps[0] == 2.0 ** -20 and steps[255] == 15 * 2.0 ** 8 and (np.diff(steps) > 0).all()
    bits = (np.arange(256, dtype=np.uint32) << 4) + (107 << 7)                 # as bf16: the byte four bits up
    assert np.array_equal((bits << 16).view(np.float32).astype(np.float64), steps)


def test_quantised_values_are_the_nearest():
    g = np.random.default_rng(1)
    x = g.standard_normal((200, 64)) * np.exp2(g.integers(-12, 8, (200, 1)))
    x[0] = 0
    q, c = ref.kv4_quantise(x)
    s = np.repeat(ref.KV4_STEPS[c], 32, -1)
    assert (np.abs(x - q * s) <= s / 2 * (1 + 1e-12)).all()
    top = np.abs(x).reshape(200, 2, 32).max(-1)
    best = np.abs(ref.KV4_STEPS[None, None] - top[..., None] / 7).min(-1)
    assert np.allclose(np.abs(ref.KV4_STEPS[c] - top / 7), best, rtol=1e-12, atol=0)
    v = ref.kv4_values(q, c)
    assert (v.astype(np.float32) == v).all() and not (v.astype(np.float32).view(np.uint32) & 0xffff).any()     # exact in bf16


def test_halves_and_what_is_not_finite():
    x = np.zeros(32)
    x[:8] = [7, 0.5, -0.5, 1.5, -2.5, 3.25, np.nan, -6.5]                      # scale 1
    q, c = ref.kv4_quantise(x)
    assert ref.KV4_STEPS[c[0]] == 1 and list(q[:8]) == [7, 1, -1, 2, -3, 3, 0, -7]
    x[1:3] = [np.inf, -np.inf]
    q, c = ref.kv4_quantise(x)
    assert c[0] == 255 and list(q[:4]) == [0, 7, -8, 0]
    assert np.array_equal(ref.kv4_quantise(np.full(32, np.nan))[0], np.zeros(32))


@pytest.mark.parametrize("D", [64, 128])
def test_packing_is_undone_by_unpacking(D):
    g = np.random.default_rng(2)
    q, c = g.integers(-8, 8, (3, 2, 128, D)).astype(np.int8), g.integers(0, 256, (3, 2, 128, D // 32)).astype(np.uint8)
    tile = ref.kv4_pack(q, c)
    assert tile.shape == (3, 2, 128 * (D // 2 + D // 32)) and tile.shape[-1] == S.kv4_tile_bytes(D)
    q2, c2 = ref.kv4_unpack(tile, D)
    assert np.array_equal(q, q2) and np.array_equal(c, c2)
    one = np.zeros((128, D), np.int8) - 8
    one[3, 8 + 5] = -7                                                         # element 5 of the second word of token 3
    assert list(ref.kv4_pack(one, np.zeros((128, D // 32)))[3 * D // 2 + 4:][:4]) == [0, 0, 0, 1]


def test_page_plan_by_hand():
    r = ref.page_plan([100, 0, 300, 128], [30, 129, -1, 0], [7, 1, 2, 3, 4], [0, 1, 1, 4, 5], [9, 8, 6, 5, 0], 4, 8, 160)
    assert list(r["page_table"]) == [7, 9, 8, 6, 4, -1, -1, -1] and list(r["page_indptr"]) == [0, 2, 4, 4, 5]
    assert list(r["tok_indptr"]) == [0, 30, 159, 159, 159] and not r["short"]
    assert r["slot_map"][0] == 7 * 128 + 100 and r["slot_map"][28] == 9 * 128 and r["slot_map"][30] == 8 * 128
    assert r["slot_map"][158] == 6 * 128 and r["slot_map"][159] == -1
    assert list(r["free_list"]) == [5, 1, 2, 3, -1] and r["n_free"] == 4


def _null_calls():
    null = C.c_void_p(0)
    some = np.zeros(64, np.int64).ctypes.data_as(C.c_void_p)                   # (refused on the host: never read)
    return S.lib(), null, some


def test_page_plan_refuses_on_the_host():
    L, null, some = _null_calls()
    i32, i64 = C.c_int32, C.c_int64

    def call(B=2, n_table=4, free_cap=4, table_cap=4, slot_cap=4, inp=some, out=some, slots=some):
        return L.specroll_page_plan(i32(B), inp, inp, inp, i32(n_table), inp, inp, i32(free_cap), inp, i32(table_cap), i64(slot_cap),
                                    out, out, out, slots, out, out, null, null)
    B.build()
    assert call(B=-1) == 1 and call(slot_cap=-1) == 1 and call(free_cap=(1 << 24) + 1) == 1
    assert call(B=4097) == 6
    assert call(inp=null) == 1 and call(out=null) == 1
    assert call() == 1                                                          # outputs on top of inputs
    base = np.zeros(64, np.int64).ctypes.data
    assert call(slots=C.c_void_p(base + 8 if base % 16 == 0 else base)) == 2    # alignment


def test_the_cache_calls_refuse_on_the_host():
    L, null, some = _null_calls()
    i32, i64 = C.c_int32, C.c_int64
    base = np.zeros(64, np.int64).ctypes.data // 16 * 16 + 16
    ok, odd = C.c_void_p(base), C.c_void_p(base + 8)

    def store(T=4, H=2, D=64, K=ok, slots=ok, pool=ok, pages=1, f=L.specroll_kv4_store):
        return f(i64(T), i32(H), i32(D), K, K, slots, pool, i64(pages), null, null)
    for f in (L.specroll_kv4_store,):
        assert store(T=-1, f=f) == 1 and store(D=96, f=f) == 1 and store(H=0, f=f) == 1 and store(pages=(1 << 24) + 1, f=f) == 1
        assert store(K=null, f=f) == 1 and store(slots=null, f=f) == 1 and store(pool=null, f=f) == 1
        assert store(K=odd, f=f) == 2 and store(pool=odd, f=f) == 2
        assert store(T=0, K=null, slots=null, pool=null, pages=0, f=f) == 0
    assert L.specroll_kv4_load(i64(4), i32(2), i32(80), ok, i64(1), ok, ok, ok, null, null) == 1
    assert L.specroll_kv4_load(i64(4), i32(2), i32(64), odd, i64(1), ok, ok, ok, null, null) == 2
    assert L.specroll_kv4_load(i64(0), i32(2), i32(64), null, i64(0), null, null, null, null, null) == 0
    assert S.kv4_tile_bytes(64) == 4352 and S.kv4_tile_bytes(128) == 8704 and S.kv4_tile_bytes(96) == 0

    def commit(B=2, N=8, K=3, H=2, D=64, Kt=ok, pool=ok):
        return L.specroll_commit_path_kv4(i32(B), i32(N), i32(K), i32(H), i32(D), Kt, Kt, ok, ok, pool, i64(1), ok, ok, ok, null, null,
                                          null)
    assert commit(N=65) == 1 and commit(K=9) == 1 and commit(D=32) == 1 and commit(Kt=null) == 1 and commit(pool=odd) == 2
    assert commit(B=0) == 0


def test_the_attention_refuses_on_the_host():
    L, null, some = _null_calls()
    parent = np.array([-1, 0, 0, 1], np.int32)
    lens = np.array([100, 200], np.int32)
    base = np.zeros(64, np.int64).ctypes.data // 16 * 16 + 16
    ok, odd = C.c_void_p(base), C.c_void_p(base + 8)

    def call(B=2, N=4, Hq=4, Hkv=2, D=64, scale=0.125, flags=0, pool=ok, Q=ok, lens=lens, parent=parent, ws=null, n=0, table=ok, pages=4):
        d = S.AttnDesc(B, N, Hq, Hkv, D, scale, flags)
        return L.specroll_tree_attn_kv4(C.byref(d), Q, pool, C.c_int64(pages), table, ok, ok, lens.ctypes.data_as(C.c_void_p), ok, ok,
                                        parent.ctypes.data_as(C.c_void_p), ok, null, ws, C.c_size_t(n), null)
    assert call(Hq=5) == 1 and call(D=96) == 1 and call(scale=0.0) == 1 and call(flags=64) == 1 and call(Q=null) == 1
    assert call(pool=null) == 1 and call(table=null) == 1 and call(pages=-1) == 1
    assert call(lens=np.array([100, -1], np.int32)) == 1
    assert call(parent=np.array([-1, 2, 0, 1], np.int32)) == 1
    assert call(pool=odd) == 2 and call(Q=odd) == 2
    assert call(flags=S.ATTN_LEGACY_MMA) == 6                                   # only the bf16 cache has that kernel
    assert call() == 3                                                          # no workspace
    assert call(B=0) == 0
    assert S.tree_attn_kv4_workspace_bytes(2, 4, 4, 2, 64, lens) > 0
    assert S.tree_attn_kv4_workspace_bytes(2, 4, 4, 2, 96, lens) == 0


@pytest.mark.parametrize("N,Hq,Hkv", [(1, 1, 1), (1, 12, 2), (8, 2, 1), (48, 10, 2)])
def test_lengths_that_round_up_past_31_bits_are_refused(N, Hq, Hkv):
    """The plan rounds lengths up to whole pages: the longest that still has a rounding is planned, one more is refused on the host."""
    most = 2 ** 31 - 128
    for f in (S.tree_attn_kv4_workspace_bytes, S.tree_attn_paged_workspace_bytes):
        for lens in ([most], [100, most]):
            assert f(len(lens), N, Hq, Hkv, 128, np.array(lens, np.int32)) > 0
        for lens in ([most + 1], [2 ** 31 - 1], [0, 2 ** 31 - 50]):
            assert f(len(lens), N, Hq, Hkv, 128, np.array(lens, np.int32)) == 0
    parent, lens = np.arange(-1, N - 1, dtype=np.int32), np.array([2 ** 31 - 1], np.int32)
    ok = C.c_void_p(np.zeros(64, np.int64).ctypes.data // 16 * 16 + 16)
    d = S.AttnDesc(1, N, Hq, Hkv, 128, 0.1, 0)
    L = S.lib()
    assert L.specroll_tree_attn_kv4(C.byref(d), ok, ok, C.c_int64(4), ok, ok, ok, lens.ctypes.data_as(C.c_void_p), ok, ok,
                                    parent.ctypes.data_as(C.c_void_p), ok, C.c_void_p(0), C.c_void_p(0), C.c_size_t(0), C.c_void_p(0)) == 1


def test_an_empty_page_table_is_taken_where_no_tokens_are_cached():
    L, null, _ = _null_calls()
    ok = C.c_void_p(np.zeros(64, np.int64).ctypes.data // 16 * 16 + 16)

    def call(lens, B=2, indptr=ok):
        lens, d = np.array(lens, np.int32), S.AttnDesc(B, 1, 4, 2, 64, 0.125, 0)
        return L.specroll_tree_attn_kv4(C.byref(d), ok, null, C.c_int64(0), null, indptr, ok, lens.ctypes.data_as(C.c_void_p), ok, ok,
                                        np.array([-1], np.int32).ctypes.data_as(C.c_void_p), ok, null, null, C.c_size_t(0), null)
    assert call([0, 0]) == 3                                                   # as far as the workspace, which is missing here
    assert call([0, 1]) == 1 and call([0, 0], indptr=null) == 1 and call([], B=0, indptr=null) == 0


def test_loading_k_and_v_to_one_place_is_refused():
    L, null, _ = _null_calls()
    base, i32, i64 = np.zeros(64, np.int64).ctypes.data // 16 * 16 + 16, C.c_int32, C.c_int64
    at = lambda off: C.c_void_p(base + off)  # noqa: E731
    for off in (0, 16, 4 * 2 * 64 * 2 - 16, -16, 16 - 4 * 2 * 64 * 2):         # (never read or written: refused on the host)
        assert L.specroll_kv4_load(i64(4), i32(2), i32(64), at(0), i64(1), at(0), at(0), at(off), null, null) == 1
