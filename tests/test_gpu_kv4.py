"""The 4-bit paged cache on the GPU: page tables and the written bytes exactly, attention within its roundings of float64.

Attention's tolerance: probabilities are rounded to bf16 (half a step is 2^-8 of each, so 2^-8 of the sum of p |v|), the result once
more (2^-8 of itself); a score of D products in fp32 is off by at most D 2^-23 of the sum of |q k| scale, which goes into p as a
relative error, and the exponential and the sums add less than 2^-18."""
import numpy as np
import pytest
import torch

from oracle import ref
from paper_2608_04962_b200 import binding as S
from paper_2608_04962_b200 import inputs as I
from tests.util import dev, dev_bf16, host

pytestmark = pytest.mark.gpu


def _bits(g, *shape, std=1.0):
    return I.f32_to_bf16_bits((g.standard_normal(shape) * std).astype(np.float32))


def _f64(bits):
    return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


# ------------------------------------------------------------------ page tables

def _plan_args(g, B, longest, most_add, finished, spare):
    kv_len = g.integers(0, longest + 1, B).astype(np.int32)
    add = g.integers(0, most_add + 1, B).astype(np.int32)
    add[g.random(B) < finished] = -1
    own = (kv_len + 127) // 128 + (g.random(B) < 0.3)
    indptr = np.concatenate([[0], np.cumsum(own)]).astype(np.int32)
    need = int((np.maximum(0, (kv_len + add + 127) // 128 - own) * (add >= 0)).sum())
    pages = g.permutation(int(indptr[-1]) + need + spare).astype(np.int32)
    free = np.concatenate([pages[indptr[-1]:], np.zeros(indptr[-1], np.int32)])
    return kv_len, add, pages[:indptr[-1]], indptr, free, np.array([need + spare], np.int32)


def _check_plan(args, table_cap, slot_cap, want_status=0):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = S.page_plan(*[dev(a) for a in args], table_cap, slot_cap, status=status)
    want = ref.page_plan(*args[:5], int(args[5][0]), table_cap, slot_cap)
    for k in ("page_table", "page_indptr", "tok_indptr", "slot_map", "free_list"):
        assert np.array_equal(host(got[k]), want[k]), k
    assert int(got["n_free"]) == want["n_free"] and int(status) == (6 if want["short"] else 0) == want_status


@pytest.mark.parametrize("B,longest,most_add,finished,spare", [(1, 0, 1, 0, 0), (1, 500, 300, 0, 3), (7, 300, 5, 0.3, 2), (33, 1000, 1000, 0.2, 1),
                                                               (256, 3000, 5, 0, 40), (513, 600, 700, 0.5, 0), (4096, 200, 130, 0.1, 9)])
def test_page_plan(B, longest, most_add, finished, spare):
    args = _plan_args(np.random.default_rng(B), B, longest, most_add, finished, spare)
    want = ref.page_plan(*args[:5], int(args[5][0]), 0, 0)
    _check_plan(args, int(want["page_indptr"][-1]) + 5, int(want["tok_indptr"][-1]))
    _check_plan(args, int(want["page_indptr"][-1]), int(want["tok_indptr"][-1]) + 3)


def test_page_plan_when_something_runs_out():
    args = list(_plan_args(np.random.default_rng(5), 40, 900, 400, 0.2, 0))
    want = ref.page_plan(*args[:5], int(args[5][0]), 0, 0)
    cap, slots = int(want["page_indptr"][-1]), int(want["tok_indptr"][-1])
    _check_plan(args, cap - 7, slots, 6)
    _check_plan(args, cap, slots - 9, 6)
    _check_plan(args, 0, 0, 6)
    args[5] = args[5] - 11                                                    # the free list is too short
    _check_plan(args, cap, slots, 6)


def test_page_plan_of_nothing():
    e, one = np.zeros(0, np.int32), np.zeros(1, np.int32)
    _check_plan((e, e, e, one, np.array([4, 2, 0], np.int32), np.array([2], np.int32)), 3, 2)
    _check_plan((np.array([-5], np.int32), np.array([3], np.int32), e, np.zeros(2, np.int32), np.array([4], np.int32), np.array([1], np.int32)), 1, 3)


def test_page_plan_into_the_callers_arrays_and_its_refusals():
    args = [dev(a) for a in _plan_args(np.random.default_rng(6), 9, 900, 400, 0.2, 2)]
    a = S.page_plan(*args, 100, 4000)
    b = {k: torch.full_like(v, 77) for k, v in a.items()}
    assert S.page_plan(*args, 100, 4000, out=b) is b and all(torch.equal(a[k], b[k]) for k in a)
    with pytest.raises(S.SpecrollError):
        S.page_plan(*args, 101, 4000, out=b)
    with pytest.raises(S.SpecrollError):
        S.page_plan(args[0], args[1][:-1].contiguous(), *args[2:], 100, 4000)
    with pytest.raises(S.SpecrollError):
        S.page_plan(args[0].long(), *args[1:], 100, 4000)
    with pytest.raises(S.SpecrollError):
        S.page_plan(*args, 100, 4000, out=dict(b, free_list=args[4]))


def test_page_plan_refuses_arrays_that_overlap():
    args = [dev(a) for a in _plan_args(np.random.default_rng(6), 9, 900, 400, 0.2, 2)]
    out = S.page_plan(*args, 100, 4000)
    words = out["slot_map"].view(torch.int32)
    for bad in (dict(tok_indptr=out["page_indptr"]), dict(page_table=words[8:108]), dict(n_free=out["tok_indptr"][3:4]), dict(n_free=args[0][:1]),
                dict(tok_indptr=args[3]), dict(page_indptr=args[4][:10])):
        with pytest.raises(S.SpecrollError):
            S.page_plan(*args, 100, 4000, out=dict(out, **bad))
    with pytest.raises(S.SpecrollError):
        S.page_plan(*args, 100, 4000, status=out["n_free"], out=out)
    S.page_plan(*args, 100, 4000, status=torch.zeros(1, dtype=torch.int32, device="cuda"), out=dict(out, page_table=words[:100], slot_map=torch.empty_like(out["slot_map"])))


# ------------------------------------------------------------------ writing and reading

def _blocks(g, T, H, D):
    """Values that go to the borders: halves, powers of two, zeros, blocks of one magnitude, tiny and large ones."""
    x = g.standard_normal((T, H, D)) * np.exp2(g.integers(-14, 10, (T, H, 1)))
    x = I.f32_to_bf16_bits(x.astype(np.float32))
    f = _f64(x)
    if T > 6:
        f[0] = 0
        f[1] = np.round(g.standard_normal((H, D)) * 3.5) / 2 * 0.25          # many halves of the scale
        f[1, :, ::32] = 7 * 0.25
        f[2] = g.choice([-1.0, 1.0], (H, D)) * 2.0 ** -5
        f[3] = g.standard_normal((H, D)) * 1e-7
        f[4] = g.standard_normal((H, D)) * 1e5
        f[5, :, ::32] = 119 * 2.0 ** -6                                      # a seventh of it lies between two scales
    return I.f32_to_bf16_bits(f.astype(np.float32))


@pytest.mark.parametrize("T,H,D", [(1, 1, 64), (1, 1, 128), (37, 2, 64), (130, 3, 128), (300, 8, 128), (257, 5, 64)])
def test_store_writes_the_oracles_bytes_and_load_gives_their_values(T, H, D):
    g = np.random.default_rng(T)
    K, V = _blocks(g, T, H, D), _blocks(g, T, H, D)
    pages = T // 128 + 2
    pool = g.integers(0, 256, (pages, H, 2, S.kv4_tile_bytes(D))).astype(np.uint8)
    slots = g.permutation(pages * 128)[:T].astype(np.int64)
    if T > 9:
        slots[7], slots[9] = -1, -128
    dpool, status = dev(pool), torch.zeros(1, dtype=torch.int32, device="cuda")
    S.kv4_store(dev_bf16(K), dev_bf16(V), dev(slots), dpool, status=status)
    want = ref.kv4_store(_f64(K), _f64(V), slots, pool)
    assert np.array_equal(host(dpool), want) and int(status) == 0            # (and no byte of another slot has changed)
    k, v = S.kv4_load(dpool, dev(slots), status=status)
    wk, wv = ref.kv4_pool_values(want, D)
    for got, w in ((k, wk), (v, wv)):
        rows = np.where((slots >= 0)[:, None, None], w.reshape(-1, H, D)[np.maximum(slots, 0)], 0.0)
        assert np.array_equal(host(got.double()), rows)
    assert int(status) == 0


def test_store_of_what_is_not_finite():
    x = np.zeros((2, 1, 64), np.uint16)
    x[0, 0, :6] = [0x7FC0, 0x3F80, 0xBF80, 0x7F80, 0xFF80, 0xFFC1]           # NaN 1 -1 inf -inf -NaN
    x[1, 0, :4] = [0x7FC0, 0x40E0, 0xBF00, 0x3F00]                           # NaN 7 -0.5 0.5
    x[1, 0, 32:] = 0x7FC0
    pool = torch.zeros(1, 1, 2, S.kv4_tile_bytes(64), dtype=torch.uint8, device="cuda")
    S.kv4_store(dev_bf16(x), dev_bf16(x), torch.tensor([0, 5], device="cuda"), pool)
    want = ref.kv4_store(_f64(x), _f64(x), [0, 5], np.zeros(pool.shape, np.uint8))
    assert np.array_equal(host(pool), want)
    k, _ = S.kv4_load(pool, torch.tensor([0, 5, 0], device="cuda"))
    assert bool(torch.isfinite(k).all()) and torch.equal(k[0], k[2])
    assert host(k[1, 0, :4].float()).tolist() == [0.0, 7.0, -1.0, 1.0] and float(k[0, 0, 3]) == 7 * 15 * 2.0 ** 8


def test_slots_beyond_the_pool_are_reported_and_nothing_is_written():
    g = np.random.default_rng(3)
    K = dev_bf16(_bits(g, 4, 2, 64))
    pool = torch.full((2, 2, 2, S.kv4_tile_bytes(64)), 9, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    slots = torch.tensor([256, 1 << 40, -1, (1 << 62)], device="cuda")
    S.kv4_store(K, K, slots, pool, status=status)
    assert int(status) == 6 and bool((pool == 9).all())
    status.zero_()
    k, v = S.kv4_load(pool, slots, status=status)
    assert int(status) == 6 and not k.any() and not v.any()
    S.kv4_store(K, K, slots, pool)                                           # without a status word
    e = torch.empty(0, dtype=torch.int64, device="cuda")
    S.kv4_store(K[:0], K[:0], e, pool)
    assert S.kv4_load(pool, e)[0].shape == (0, 2, 64)


def test_the_cache_calls_check_their_tensors():
    g = np.random.default_rng(4)
    K = dev_bf16(_bits(g, 4, 2, 64))
    pool = torch.zeros(2, 2, 2, S.kv4_tile_bytes(64), dtype=torch.uint8, device="cuda")
    slots = torch.arange(4, device="cuda")
    for bad in (lambda: S.kv4_store(K, K[:3], slots, pool), lambda: S.kv4_store(K, K, slots[:3], pool), lambda: S.kv4_store(K, K, slots.int(), pool),
                lambda: S.kv4_store(K.float(), K.float(), slots, pool), lambda: S.kv4_store(K, K, slots, pool[..., :-1].contiguous()),
                lambda: S.kv4_store(K.transpose(0, 1), K.transpose(0, 1), slots[:2], pool), lambda: S.kv4_store(K[:, :1].contiguous(), K[:, :1].contiguous(), slots, pool),
                lambda: S.kv4_load(pool.cpu(), slots), lambda: S.kv4_load(pool, slots, out=(K, K[:3])), lambda: S.kv4_store(K, K, slots.cpu(), pool)):
        with pytest.raises(S.SpecrollError):
            bad()
    out = (torch.empty_like(K), torch.empty_like(K))
    assert S.kv4_load(pool, slots, out=out)[0].data_ptr() == out[0].data_ptr()


# ------------------------------------------------------------------ attention

def _case(B, N, Hq, Hkv, D, lengths, seed, spare=0, std=1.0):
    g = np.random.default_rng(seed)
    lengths = np.asarray(lengths, np.int32)
    own = (lengths + spare + 127) // 128
    indptr = np.concatenate([[0], np.cumsum(own)]).astype(np.int32)
    pages = int(indptr[-1]) + 3
    table = g.permutation(pages)[:indptr[-1]].astype(np.int32)
    K, V = (g.standard_normal((pages, Hkv, 128, D)) * std for _ in range(2))
    pool = np.stack([ref.kv4_pack(*ref.kv4_quantise(K)), ref.kv4_pack(*ref.kv4_quantise(V))], 2)
    for b in range(B):                                                       # rows beyond the length: the largest values there are
        if lengths[b] % 128 and own[b]:
            page, at = table[indptr[b] + lengths[b] // 128], lengths[b] % 128
            pool[page, :, :, at * D // 2:64 * D] = 0xFF
            pool[page, :, :, 64 * D + at * D // 32:] = 0xFF
    wk, wv = ref.kv4_pool_values(pool, D)
    cat = lambda w: [w[table[indptr[b]:indptr[b + 1]]].reshape(-1, Hkv, D)[:lengths[b]] for b in range(B)]  # noqa: E731
    parent = np.array([-1] + [int(g.integers(max(0, n - 6), n)) for n in range(1, N)], np.int32)
    return dict(Q=_bits(g, B, N, Hq, D, std=std), Kt=_bits(g, B, N, Hkv, D), Vt=_bits(g, B, N, Hkv, D), pool=pool, table=table, indptr=indptr,
                len=lengths, parent=parent, K=cat(wk), V=cat(wv))


def _run(x, flags=0, **kw):
    return S.tree_attn_kv4(dev_bf16(x["Q"]), dev(x["pool"]), dev(x["table"]), dev(x["indptr"]), dev(x["len"]), x["len"], dev_bf16(x["Kt"]),
                           dev_bf16(x["Vt"]), x["parent"], flags=flags, **kw)


def _check(x, scale=None, **kw):
    D = x["Q"].shape[-1]
    O, lse = _run(x, want_lse=True, check_status=True, scale=scale, **kw)
    want, wl, A, dot = ref.tree_attn64(_f64(x["Q"]), x["K"], x["V"], x["len"], _f64(x["Kt"]), _f64(x["Vt"]), x["parent"],
                                       scale if scale is not None else D ** -0.5)
    score = D * 2.0 ** -23 * dot + 2.0 ** -18
    off = np.abs(host(O.double()) - want)
    tol = 2.0 ** -8 * (A + np.abs(want)) + 2 * score * A + 1e-30
    assert (off <= tol).all(), (off / tol).max()
    assert np.abs(host(lse.double()) - wl).max() <= score + 2.0 ** -23 * np.abs(wl).max()
    return O


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,Hq,Hkv", [(1, 1, 1), (1, 4, 2), (1, 12, 2), (1, 28, 4), (1, 16, 1), (2, 8, 8), (3, 10, 2), (8, 4, 2), (17, 6, 2)])
def test_attention_matches_float64(N, Hq, Hkv, D):
    _check(_case(6, N, Hq, Hkv, D, [0, 1, 127, 128, 129, 700], seed=N * 100 + Hq + D))


@pytest.mark.parametrize("N,Hq,Hkv,D", [(16, 12, 2, 128), (32, 14, 2, 128), (48, 10, 2, 128), (64, 7, 1, 128), (33, 7, 1, 64), (64, 16, 2, 64),
                                        (64, 32, 1, 128), (5, 64, 1, 64), (2, 128, 1, 128)])
def test_attention_of_trees(N, Hq, Hkv, D):
    _check(_case(4, N, Hq, Hkv, D, [0, 333, 64, 900], seed=N + Hq))


@pytest.mark.parametrize("N,Hq,Hkv,D,lengths", [(1, 7, 1, 128, [9000]), (1, 4, 4, 64, [5000, 3, 2500]), (8, 7, 1, 128, [6000, 130]),
                                                (16, 6, 1, 128, [7000, 0, 129]), (40, 5, 1, 64, [4000])])
def test_attention_of_long_sequences_in_chunks(N, Hq, Hkv, D, lengths):
    _check(_case(len(lengths), N, Hq, Hkv, D, lengths, seed=7, spare=200))


@pytest.mark.parametrize("N,Hq,Hkv,lengths", [(1, 2, 1, [60 + 37 * (b % 9) for b in range(40)]), (5, 6, 2, [(b * 53) % 400 for b in range(130)])])
def test_attention_of_many_sequences(N, Hq, Hkv, lengths):
    _check(_case(len(lengths), N, Hq, Hkv, 64, lengths, seed=8))


@pytest.mark.parametrize("std,scale", [(30.0, None), (1.0, 3.0), (1e-3, 1.0)])
@pytest.mark.parametrize("N,Hq", [(1, 4), (24, 12)])
def test_attention_where_the_reference_moves(N, Hq, std, scale):
    """Scores that span hundreds of powers of two, and scores that hardly differ."""
    x = _case(3, N, Hq, 2, 128, [1000, 200, 1], seed=9, std=std)
    _check(x, scale=scale)


@pytest.mark.parametrize("N,Hq", [(1, 8), (20, 14)])
def test_pages_outside_the_pool_read_as_zeros(N, Hq):
    x = _case(3, N, Hq, 2, 128, [500, 300, 256], seed=10)
    x["table"][1], x["table"][x["indptr"][2]] = -1, x["pool"].shape[0]
    for w in (x["K"], x["V"]):
        w[0][128:256] = 0
        w[2][:128] = 0
    _check(x)


@pytest.mark.parametrize("N,Hq", [(1, 14), (16, 12), (48, 10)])
def test_a_kept_plan_and_a_settled_cache(N, Hq):
    x = _case(5, N, Hq, 2, 128, [700, 64, 1500, 333, 2900], seed=11)
    ws = S.alloc(S.tree_attn_kv4_workspace_bytes(5, N, Hq, 2, 128, x["len"]), dtype=torch.uint8, device="cuda")
    a = _run(x, workspace=ws)
    outs = [_run(x, workspace=ws, flags=f) for f in (S.ATTN_REUSE_PLAN, S.ATTN_REUSE_PLAN | S.ATTN_CACHE_SETTLED, S.ATTN_NO_PDL,
                                                     S.ATTN_REUSE_PLAN | S.ATTN_NO_PDL)]
    assert S.workspace_status(ws) == 0 and all(torch.equal(a, o) for o in outs)


@pytest.mark.parametrize("N,Hq", [(1, 14), (48, 10)])
def test_a_captured_call_follows_its_inputs(N, Hq):
    x, y = (_case(3, N, Hq, 2, 128, [700, 64, 1500], seed=s) for s in (12, 13))
    t = {k: (dev_bf16 if k in ("Q", "Kt", "Vt") else dev)(x[k]) for k in ("Q", "pool", "table", "indptr", "len", "Kt", "Vt")}
    ws = [S.alloc(S.tree_attn_kv4_workspace_bytes(3, N, Hq, 2, 128, x["len"]), dtype=torch.uint8, device="cuda") for _ in range(2)]
    out = [torch.empty_like(t["Q"]) for _ in range(2)]

    def call(i, parent):
        S.tree_attn_kv4(t["Q"], t["pool"], t["table"], t["indptr"], t["len"], x["len"], t["Kt"], t["Vt"], parent, workspace=ws[i], out=out[i])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(0, x["parent"])
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(0, x["parent"])
        call(1, x["parent"])
    for k in t:
        t[k].copy_((dev_bf16 if k in ("Q", "Kt", "Vt") else dev)(y[k]))
    for o in out:
        o.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    want = _run({**y, "parent": x["parent"]})
    assert all(torch.equal(o, want) for o in out) and S.workspace_status(ws[0]) == 0


def test_the_attention_checks_its_tensors():
    x = _case(2, 4, 4, 2, 64, [100, 30], seed=14)
    for bad in ({"pool": x["pool"][..., :-16]}, {"pool": x["pool"][:, :1]}, {"Q": x["Q"][:1]}, {"len": x["len"][:1]}, {"Kt": x["Kt"][:, :3]},
                {"len": np.array([-1, 3], np.int32)}, {"parent": x["parent"][:2]}):
        with pytest.raises(S.SpecrollError):
            _run({**x, **bad})
    with pytest.raises(S.SpecrollError):
        _run(x, flags=S.ATTN_LEGACY_MMA)
    with pytest.raises(S.SpecrollError):
        _run(x, out=torch.empty(2, 4, 4, 32, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(S.SpecrollError):
        _run(x, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))


# ------------------------------------------------------------------ as a rollout uses them

@pytest.mark.parametrize("N,Hq,Hkv,D,K", [(1, 4, 2, 64, 1), (8, 12, 2, 128, 3), (40, 14, 2, 128, 4)])
def test_a_rollout_over_the_cache(N, Hq, Hkv, D, K):
    """Pages for the prompts, the prompts stored, rounds of attention and commit with pages planned in between, a sequence that
    finishes; against the same cache kept as lists of rows."""
    g, B, layers = np.random.default_rng(15), 5, 2
    prompt = np.array([200, 1, 128, 37, 255], np.int32)
    n_pages = 24
    pools = [torch.zeros(n_pages, Hkv, 2, S.kv4_tile_bytes(D), dtype=torch.uint8, device="cuda") for _ in range(layers)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    state = dict(page_table=torch.empty(0, dtype=torch.int32, device="cuda"), page_indptr=torch.zeros(B + 1, dtype=torch.int32, device="cuda"),
                 free_list=dev(g.permutation(n_pages).astype(np.int32)), n_free=torch.tensor([n_pages], dtype=torch.int32, device="cuda"))

    def plan(lens, add):
        return S.page_plan(lens, dev(add.astype(np.int32)), state["page_table"], state["page_indptr"], state["free_list"], state["n_free"],
                           n_pages, int(np.maximum(add, 0).sum()), status=status)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    state = plan(lens, prompt)
    rows = [[[], []] for _ in range(layers)]                                 # per layer: K, V as lists per sequence
    for l in range(layers):
        kv = [_bits(g, int(prompt.sum()), Hkv, D) for _ in range(2)]
        S.kv4_store(dev_bf16(kv[0]), dev_bf16(kv[1]), state["slot_map"], pools[l], status=status)
        for i in range(2):
            rows[l][i] = np.split(ref.kv4_values(*ref.kv4_quantise(_f64(kv[i]))), np.cumsum(prompt)[:-1])
    lens = dev(prompt)
    parent = np.array([-1] + [int(g.integers(max(0, n - 3), n)) for n in range(1, N)], np.int32)
    for step in range(3):
        host_len = host(lens)
        done = step == 2
        add = np.full(B, K + 1)
        if done:
            add[1] = -1                                                      # finished: its pages go back
        state = plan(lens, add)
        assert host(state["page_indptr"])[2] - host(state["page_indptr"])[1] == 0 if done else True
        if done:
            lens[1] = 0
            host_len = host(lens)
            for l in range(layers):
                for i in range(2):
                    rows[l][i][1] = rows[l][i][1][:0]
        n_acc = g.integers(0, min(K, N - 1) + 1, B).astype(np.int32)
        path = np.where(np.arange(K + 1) <= n_acc[:, None], np.minimum(np.arange(K + 1), N - 1), -1).astype(np.int32)
        if done:
            n_acc[1] = -1                                                    # nothing is committed for it
        Kt, Vt = ([_bits(g, B, N, Hkv, D) for _ in range(layers)] for _ in range(2))
        for l in range(layers):
            Q = _bits(g, B, N, Hq, D)
            x = dict(Q=Q, Kt=Kt[l], Vt=Vt[l], pool=host(pools[l]), table=host(state["page_table"]), indptr=host(state["page_indptr"]),
                     len=host_len, parent=parent, K=rows[l][0], V=rows[l][1])
            _check(x)
        new = torch.empty_like(lens)
        S.commit_path_kv4_layers([dev_bf16(k) for k in Kt], [dev_bf16(v) for v in Vt], dev(path), dev(n_acc), pools, state["page_table"],
                                 state["page_indptr"], lens, kv_len_out=new, status=status)
        for l in range(layers):
            for i, t in enumerate((Kt[l], Vt[l])):
                for b in range(B):
                    take = _f64(t[b][path[b, :n_acc[b] + 1]])
                    if n_acc[b] >= 0:
                        rows[l][i][b] = np.concatenate([rows[l][i][b], ref.kv4_values(*ref.kv4_quantise(take))])
        lens = new
    assert int(status) == 0
    assert host(lens).tolist() == [len(r) for r in rows[0][0]]


def test_commit_of_one_layer_in_place_and_without_room():
    g = np.random.default_rng(16)
    B, N, K, Hkv, D = 3, 16, 4, 2, 128
    kv_len = np.array([126, 64, 250], np.int32)
    table, indptr = np.array([2, 0, 3, 1], np.int32), np.array([0, 1, 2, 4], np.int32)
    Kt, Vt = _bits(g, B, N, Hkv, D), _bits(g, B, N, Hkv, D)
    path = np.tile(np.array([0, 1, 4, 7, 9], np.int32), (B, 1))
    n_acc = np.array([4, 2, 4], np.int32)
    pool = g.integers(0, 256, (5, Hkv, 2, S.kv4_tile_bytes(D))).astype(np.uint8)
    want = pool
    for b in range(B):
        for i in range(n_acc[b] + 1):
            pos = kv_len[b] + i
            if pos // 128 < indptr[b + 1] - indptr[b]:
                slot = table[indptr[b] + pos // 128] * 128 + pos % 128
                want = ref.kv4_store(_f64(Kt[b, path[b, i]])[None], _f64(Vt[b, path[b, i]])[None], [slot], want)
    status, dpool, dl = torch.zeros(1, dtype=torch.int32, device="cuda"), dev(pool), dev(kv_len)
    S.commit_path_kv4(dev_bf16(Kt), dev_bf16(Vt), dev(path), dev(n_acc), dpool, dev(table), dev(indptr), dl, kv_len_out=dl, status=status)
    assert np.array_equal(host(dpool), want) and int(status) == 6            # the first sequence's last tokens had no page
    assert np.array_equal(host(dl), kv_len + n_acc + 1)
    with pytest.raises(S.SpecrollError):
        S.commit_path_kv4(dev_bf16(Kt), dev_bf16(Vt), dev(path), dev(n_acc)[:2], dpool, dev(table), dev(indptr), dl)
    with pytest.raises(S.SpecrollError):
        S.commit_path_kv4(dev_bf16(Kt), dev_bf16(Vt), dev(path), dev(n_acc), dpool[:, :1].contiguous(), dev(table), dev(indptr), dl)
    with pytest.raises(S.SpecrollError):
        S.commit_path_kv4_layers([], [], dev(path), dev(n_acc), [], dev(table), dev(indptr), dl)


def test_two_streams_with_workspaces_of_their_own():
    xs = [_case(4, 1 + 15 * i, 14, 2, 128, [900, 5, 0, 2000], seed=20 + i) for i in range(2)]
    want = [_run(x) for x in xs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(_run(xs[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in got[i])


@pytest.mark.parametrize("N,Hq", [(1, 8), (24, 12)])
def test_places_beyond_four_gigabytes(N, Hq):
    """A pool of 5 GB of which a few pages near its end and its beginning are used."""
    g = np.random.default_rng(17)
    Hkv, D, lens = 2, 128, np.array([300, 129], np.int32)
    n_pages = 5 * (1 << 30) // (Hkv * 2 * S.kv4_tile_bytes(D))
    pool = torch.empty(n_pages, Hkv, 2, S.kv4_tile_bytes(D), dtype=torch.uint8, device="cuda")
    table, indptr = np.array([n_pages - 1, 0, n_pages - 2, n_pages // 2, n_pages - 7], np.int32), np.array([0, 3, 5], np.int32)
    slots = np.concatenate([table[indptr[b] + np.arange(lens[b]) // 128].astype(np.int64) * 128 + np.arange(lens[b]) % 128 for b in range(2)])
    K, V = _bits(g, len(slots), Hkv, D), _bits(g, len(slots), Hkv, D)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    S.kv4_store(dev_bf16(K), dev_bf16(V), dev(slots), pool, status=status)
    vals = [ref.kv4_values(*ref.kv4_quantise(_f64(x))) for x in (K, V)]
    for got, want in zip(S.kv4_load(pool, dev(slots), status=status), vals):
        assert np.array_equal(host(got.double()), want)
    parent = np.array([-1] + [int(g.integers(0, n)) for n in range(1, N)], np.int32)
    Q, Kt, Vt = _bits(g, 2, N, Hq, D), _bits(g, 2, N, Hkv, D), _bits(g, 2, N, Hkv, D)
    want, wl, A, dot = ref.tree_attn64(_f64(Q), *[np.split(x, [300]) for x in vals], lens, _f64(Kt), _f64(Vt), parent, D ** -0.5)
    O = S.tree_attn_kv4(dev_bf16(Q), pool, dev(table), dev(indptr), dev(lens), lens, dev_bf16(Kt), dev_bf16(Vt), parent, check_status=True)
    assert (np.abs(host(O.double()) - want) <= 2.0 ** -8 * (A + np.abs(want)) + 2 * (D * 2.0 ** -23 * dot + 2.0 ** -18) * A).all()
    path, n_acc = np.zeros((2, 2), np.int32), np.zeros(2, np.int32)          # the first node's rows behind the last token
    S.commit_path_kv4(dev_bf16(Kt), dev_bf16(Vt), dev(path), dev(n_acc), pool, dev(table), dev(indptr), dev(lens), status=status)
    at = np.array([table[2] * 128 + 300 % 128, table[4] * 128 + 129 % 128], np.int64)
    k, _ = S.kv4_load(pool, dev(at))
    assert np.array_equal(host(k.double()), ref.kv4_values(*ref.kv4_quantise(_f64(Kt[:, 0])))) and int(status) == 0


@pytest.mark.parametrize("N,Hq", [(1, 8), (24, 12)])
def test_a_round_in_one_graph(N, Hq):
    """Pages, attention and commit captured together and replayed on other lengths' caches of the same plan."""
    x, y = (_case(4, N, Hq, 2, 128, [300, 130, 128, 1], seed=s, spare=5) for s in (18, 19))
    bf = ("Q", "Kt", "Vt")
    t = {k: (dev_bf16 if k in bf else dev)(x[k]) for k in ("Q", "pool", "table", "indptr", "len", "Kt", "Vt")}
    n_pages = x["pool"].shape[0]
    free = np.setdiff1d(np.arange(n_pages), x["table"]).astype(np.int32)
    t |= {"free": dev(np.concatenate([free, np.zeros(n_pages - len(free), np.int32)])), "n_free": dev(np.array([len(free)], np.int32)),
          "add": torch.full((4,), 2, dtype=torch.int32, device="cuda"), "path": dev(np.tile(np.array([0, N - 1], np.int32), (4, 1))),
          "n_acc": dev(np.array([1, 0, 1, 0], np.int32))}
    out = {}

    def round_():
        out["plan"] = S.page_plan(t["len"], t["add"], t["table"], t["indptr"], t["free"], t["n_free"], n_pages, 8)
        out["O"] = S.tree_attn_kv4(t["Q"], t["pool"], out["plan"]["page_table"], out["plan"]["page_indptr"], t["len"], x["len"], t["Kt"], t["Vt"],
                                   x["parent"])
        out["len"] = torch.empty_like(t["len"])
        S.commit_path_kv4(t["Kt"], t["Vt"], t["path"], t["n_acc"], t["pool"], out["plan"]["page_table"], out["plan"]["page_indptr"], t["len"],
                          kv_len_out=out["len"])
        out["KV"] = S.kv4_load(t["pool"], out["plan"]["slot_map"])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        round_()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        round_()
    for k in ("Q", "pool", "Kt", "Vt", "table"):
        t[k].copy_((dev_bf16 if k in bf else dev)(y[k]))
    free = np.setdiff1d(np.arange(n_pages), y["table"]).astype(np.int32)
    t["free"][:len(free)] = dev(free)
    graph.replay()
    torch.cuda.synchronize()
    want = _run({**y, "parent": x["parent"]})
    assert torch.equal(out["O"], want) and host(out["len"]).tolist() == [302, 131, 130, 2]
    rows = ref.kv4_values(*ref.kv4_quantise(np.stack([_f64(y["Kt"])[:, 0], _f64(y["Kt"])[:, N - 1]], 1)))
    got = host(out["KV"][0].double()).reshape(4, 2, 2, 128)
    for b, n in enumerate((2, 1, 2, 1)):
        assert np.array_equal(got[b, :n], rows[b, :n])


def test_a_settled_cache_written_two_kernels_ago():
    """Commit into layer B's pool, attention of layer A, attention of layer B, which may fetch its pages while A's is finishing."""
    x = _case(8, 16, 12, 2, 128, [700, 64, 1500, 333, 129, 2900, 256, 77], seed=21, spare=8)
    t = {k: (dev_bf16 if k in ("Q", "Kt", "Vt") else dev)(x[k]) for k in ("Q", "pool", "table", "indptr", "len", "Kt", "Vt")}
    path, n_acc, first = torch.arange(5, dtype=torch.int32, device="cuda").repeat(8, 1), torch.full((8,), 4, dtype=torch.int32, device="cuda"), torch.zeros_like(t["len"])
    A, B = t["pool"], t["pool"].clone()
    others = [torch.zeros_like(B) for _ in range(12)]
    ws = S.alloc(S.tree_attn_kv4_workspace_bytes(8, 16, 12, 2, 128, x["len"]), dtype=torch.uint8, device="cuda")

    def attn(pool, flags):
        return S.tree_attn_kv4(t["Q"], pool, t["table"], t["indptr"], t["len"], x["len"], t["Kt"], t["Vt"], x["parent"], workspace=ws, flags=flags)

    def commit(pools):
        S.commit_path_kv4_layers([t["Kt"]] * len(pools), [t["Vt"]] * len(pools), path, n_acc, pools, t["table"], t["indptr"], first)
    commit([B])
    want_a, want_b = attn(A, 0), attn(B, 0)
    assert not torch.equal(want_a, want_b)
    for _ in range(20):
        B.copy_(A)
        torch.cuda.synchronize()
        commit(others + [B])
        flags = S.ATTN_REUSE_PLAN | S.ATTN_CACHE_SETTLED
        got_a, got_b = attn(A, flags), attn(B, flags)
        torch.cuda.synchronize()
        assert torch.equal(got_a, want_a) and torch.equal(got_b, want_b)
    assert S.workspace_status(ws) == 0


@pytest.mark.parametrize("N,Hq", [(1, 3), (6, 3)])
def test_4096_sequences_and_no_more(N, Hq):
    B, D = 4096, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    lens = np.random.default_rng(1).integers(0, 130, B).astype(np.int32)
    pages = 64
    pool = torch.randint(0, 255, (pages, 1, 2, S.kv4_tile_bytes(D)), dtype=torch.uint8, device="cuda", generator=g)
    pool[..., 64 * D:] = 8 * 20                                              # (scales of one)
    table = torch.randint(0, pages, (2 * B,), dtype=torch.int32, device="cuda", generator=g)
    indptr = torch.arange(0, 2 * B + 1, 2, dtype=torch.int32, device="cuda")
    Q, Kt, Vt = (torch.randn(B, N, h, D, device="cuda", generator=g).bfloat16() for h in (Hq, 1, 1))
    parent = np.arange(-1, N - 1, dtype=np.int32)

    def call(n):
        return S.tree_attn_kv4(Q[:n].contiguous(), pool, table, indptr[:n + 1].contiguous(), dev(lens[:n]), lens[:n], Kt[:n].contiguous(),
                               Vt[:n].contiguous(), parent)
    O = call(B)
    for b in (0, 1, 777, 2048, 4095):                                        # (each like the call of it alone)
        one = S.tree_attn_kv4(Q[b:b + 1].contiguous(), pool, table[2 * b:2 * b + 2].contiguous(), indptr[:2].contiguous(), dev(lens[b:b + 1]),
                              lens[b:b + 1], Kt[b:b + 1].contiguous(), Vt[b:b + 1].contiguous(), parent)
        assert (O[b].float() - one[0].float()).abs().max() <= 2.0 ** -6 * one.float().abs().max()
    Q, Kt, Vt, lens = (torch.cat([v, v[:1]]) for v in (Q, Kt, Vt)), 0, 0, np.append(lens, 5).astype(np.int32)
    Q, Kt, Vt = list(Q)
    table, indptr = torch.cat([table, table[:2]]), torch.arange(0, 2 * B + 3, 2, dtype=torch.int32, device="cuda")
    with pytest.raises(S.SpecrollError):
        call(B + 1)


def test_more_than_128_query_heads_a_cache_head_are_refused():
    x = _case(1, 1, 129, 1, 64, [10], seed=22)
    with pytest.raises(S.SpecrollError):
        _run(x, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))


def test_outputs_from_the_ordinary_allocator():
    """Arrays that share an allocation: sizes, types, alignment, and none on top of another."""
    from paper_2608_04962_b200 import binding
    args = _plan_args(np.random.default_rng(7), 37, 900, 400, 0.2, 2)
    want = ref.page_plan(*args[:5], int(args[5][0]), 333, 4001)
    binding.set_allocator(None)
    p = S.page_plan(*[dev(a) for a in args], 333, 4001)
    for k in ("page_table", "page_indptr", "tok_indptr", "slot_map", "free_list"):
        assert np.array_equal(host(p[k]), want[k]) and p[k].data_ptr() % 256 == 0 and p[k].is_contiguous(), k
    spans = sorted((v.data_ptr(), v.data_ptr() + v.numel() * v.element_size()) for v in p.values())
    assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:])) and p["slot_map"].dtype == torch.int64
    pool = torch.full((2, 3, 2, S.kv4_tile_bytes(64)), 0x99, dtype=torch.uint8, device="cuda")
    k, v = S.kv4_load(pool, torch.tensor([3, -1, 200], device="cuda"))
    k.zero_()
    assert v.shape == (3, 3, 64) and bool((v[0] != 0).all()) and not v[1].any() and bool((v[2] != 0).all())
    assert v.clone().data_ptr() != v.data_ptr() and (v + 0).shape == v.shape  # (an ordinary tensor to torch)


@pytest.mark.parametrize("N,Hq", [(1, 4), (24, 12)])
@pytest.mark.parametrize("B", [3, 40])
def test_a_negative_length_on_the_device_counts_as_none(B, N, Hq):
    x = _case(B, N, Hq, 2, 64, [0 if b % 3 == 1 else 130 + b for b in range(B)], seed=21)
    want = _run(x)
    t = [dev_bf16(x["Q"]), dev(x["pool"]), dev(x["table"]), dev(x["indptr"]), dev(np.where(x["len"] > 0, x["len"], -1000).astype(np.int32)),
         x["len"], dev_bf16(x["Kt"]), dev_bf16(x["Vt"])]
    assert torch.equal(S.tree_attn_kv4(*t, x["parent"], check_status=True), want)


@pytest.mark.parametrize("N,Hq,lengths", [(1, 4, [128, 100, 1, 0]), (1, 4, [9000, 0, 6900, 1]), (8, 4, [5000, 129, 0, 9100]), (1, 32, [1, 2, 3, 4])])
def test_lengths_below_the_hosts(N, Hq, lengths):
    """A call planned for the longest that the sequences get, as one that was captured, follows the lengths on the device; and what reads its
    outputs next waits for them, also where nothing is cut any more and the merge has no work."""
    x = _case(4, N, Hq, 2, 128, [9000, 8000, 7000, 9100], seed=22)
    y = dict(x, len=np.array(lengths, np.int32), K=[k[:n] for k, n in zip(x["K"], lengths)], V=[v[:n] for v, n in zip(x["V"], lengths)])
    want, _, A, dot = ref.tree_attn64(_f64(y["Q"]), y["K"], y["V"], y["len"], _f64(y["Kt"]), _f64(y["Vt"]), y["parent"], 128 ** -0.5)
    tol = 2.0 ** -8 * (A + np.abs(want)) + 2 * (128 * 2.0 ** -23 * dot + 2.0 ** -18) * A + 1e-30   # as in _check
    t = [dev_bf16(x["Q"]), dev(x["pool"]), dev(x["table"]), dev(x["indptr"]), dev(y["len"]), x["len"], dev_bf16(x["Kt"]), dev_bf16(x["Vt"])]
    out = torch.zeros_like(t[0])
    rows, slots = out.view(4 * N, Hq, 128), torch.arange(4 * N, device="cuda")
    pools = [torch.zeros((1, Hq, 2, S.kv4_tile_bytes(128)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    for _ in range(20):
        out.zero_()
        S.tree_attn_kv4(*t, x["parent"], out=out)
        S.kv4_store(rows, rows, slots, pools[0])
        torch.cuda.synchronize()
        S.kv4_store(rows, rows, slots, pools[1])
        assert torch.equal(*pools)
        assert (np.abs(host(out.double()) - want) <= tol).all()
