"""The 4-bit paged cache where its kernels take other ways than small calls do: stages used again, many tokens, many layers, plans of many
units.  Tables, bytes and copies exactly; attention with the tolerance of test_gpu_kv4.py."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import ref
from paper_2608_04962_b200 import binding as S
from tests.test_gpu_kv4 import _bits, _case, _check, _f64, _run
from tests.util import dev, dev_bf16, host

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("N,Hq,D", [(1, 4, 64), (1, 16, 128), (8, 4, 128)])
@pytest.mark.parametrize("missing", [2, 3, 7])
def test_pages_that_are_missing_in_turn_with_pages_that_are_there(N, Hq, D, missing):
    """Few rows: a stage is filled by plain stores for a page that does not exist and by copies for the next one, many times over, and a
    cut plan's search has used the first stage before either."""
    x = _case(4, N, Hq, 2, D, [9000, 700, 0, 5000], seed=30 + missing)
    for b in range(4):
        for i in range(x["indptr"][b], x["indptr"][b + 1]):
            if (i - x["indptr"][b]) % missing == b % missing:
                x["table"][i] = -1 if i % 2 else x["pool"].shape[0] + i
                at = (i - x["indptr"][b]) * 128
                for w in (x["K"], x["V"]):
                    w[b][at:at + 128] = 0
    O = _check(x)
    assert all(torch.equal(O, _run(x)) for _ in range(10))


SETTLED = r"""
import sys
sys.path.insert(0, %r)
import numpy as np, torch
from paper_2608_04962_b200 import binding as S
from tests.test_gpu_kv4 import _case, _run
from tests.util import dev, dev_bf16
assert S.check_status()[0] == 0, "not a build with index checks"
g = torch.Generator(device="cuda").manual_seed(1)


def long_call(Hkv, pages=900000, D=128):
    pool = torch.randint(0, 255, (8, Hkv, 2, S.kv4_tile_bytes(D)), dtype=torch.uint8, device="cuda", generator=g)
    table = torch.randint(0, 8, (pages,), dtype=torch.int32, device="cuda", generator=g)
    lens = np.array([128 * pages - 5], np.int32)
    Q, Kt, Vt = (torch.randn(1, 1, Hkv, D, device="cuda", generator=g).bfloat16() for _ in range(3))
    ws = torch.zeros(S.tree_attn_kv4_workspace_bytes(1, 1, Hkv, Hkv, D, lens), dtype=torch.uint8, device="cuda")
    indptr, on_gpu, out = torch.tensor([0, pages], dtype=torch.int32, device="cuda"), dev(lens), torch.empty_like(Q)
    return lambda: S.tree_attn_kv4(Q, pool, table, indptr, on_gpu, lens, Kt, Vt, [-1], workspace=ws, out=out)


def ms(f):
    t = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    t[0].record()
    f()
    t[1].record()
    torch.cuda.synchronize()
    return t[0].elapsed_time(t[1])


x = _case(4, 17, 4, 2, 128, [1000, 700, 1500, 384], seed=40)
t = [dev_bf16(x["Q"]), dev(x["pool"]), dev(x["table"]), dev(x["indptr"]), dev(x["len"]), x["len"], dev_bf16(x["Kt"]), dev_bf16(x["Vt"]), x["parent"]]
ws, out = torch.zeros(S.tree_attn_kv4_workspace_bytes(4, 17, 4, 2, 128, x["len"]), dtype=torch.uint8, device="cuda"), torch.zeros_like(t[0])
want = S.tree_attn_kv4(*t, workspace=ws).clone()
even, uneven = long_call(98), long_call(100)
even(), uneven()
torch.cuda.synchronize()
print("ms of 588 and of 600 units:", ms(even), ms(uneven))
for _ in range(2):
    out.zero_()
    uneven()
    S.tree_attn_kv4(*t, workspace=ws, out=out, flags=S.ATTN_REUSE_PLAN | S.ATTN_CACHE_SETTLED)
    torch.cuda.synchronize()
    assert S.workspace_status(ws) == 0 and torch.equal(out, want)
print("settled ok")
"""


def test_a_settled_cache_behind_a_long_kernel():
    """600 units where 592 run side by side: for tens of milliseconds few SMs are busy, and the next call's CTAs are there and fetch their
    first pages.  The debug build's waits give up after 20 ms; none may be running by then."""
    from paper_2608_04962_b200 import build as B
    p = subprocess.run([sys.executable, "-c", SETTLED % ROOT], env=dict(os.environ, SPECROLL_LIB=B.build(check=True)), capture_output=True,
                       text=True, timeout=600)
    print(p.stdout)
    assert p.returncode == 0 and "settled ok" in p.stdout, p.stdout + p.stderr


@pytest.mark.parametrize("N,Hq,host_lens", [(1, 4, [3000, 200, 100, 2000]), (8, 4, [2000, 200, 2500, 100]), (1, 32, [4000, 0, 0, 0])])
@pytest.mark.parametrize("D", [64, 128])
def test_lengths_above_the_hosts_are_reported_and_nothing_is_written(N, Hq, host_lens, D):
    """A cut plan of few rows, replayed on lengths that make more chunks than it has: the status word says so, and outputs stay as they were,
    whatever an earlier call has left in the workspace."""
    x = _case(4, N, Hq, 2, D, [9000, 8000, 7000, 9100], seed=50)
    host_lens = np.array(host_lens, np.int32)
    ws = S.alloc(S.tree_attn_kv4_workspace_bytes(4, N, Hq, 2, D, host_lens), dtype=torch.uint8, device="cuda")
    t = [dev_bf16(x["Q"]), dev(x["pool"]), dev(x["table"]), dev(x["indptr"]), dev(host_lens), host_lens, dev_bf16(x["Kt"]), dev_bf16(x["Vt"])]
    out = [torch.empty_like(t[0]), torch.empty(t[0].shape[:3], device="cuda")]

    def call():
        S.tree_attn_kv4(*t, x["parent"], workspace=ws, out=out[0], lse=out[1])
        return [o.clone() for o in out]
    want = call()
    assert S.workspace_status(ws) == 0
    short = {**x, "len": host_lens, "K": [k[:n] for k, n in zip(x["K"], host_lens)], "V": [v[:n] for v, n in zip(x["V"], host_lens)]}
    assert torch.equal(want[0], _check(short))
    for lens in (x["len"], np.where(np.arange(4) == 3, x["len"], host_lens), np.where(np.arange(4) == 1, x["len"], host_lens),
                 host_lens + [300, 9000, 0, 0], np.where(np.arange(4) == 2, 2 ** 31 - 1, host_lens), np.full(4, 2 ** 31 - 20)):
        t[4].copy_(dev((lens if lens.max() > 2 ** 30 else np.minimum(lens, x["len"])).astype(np.int32)))   # (nothing is read of the longest)
        for o in out:
            o.fill_(-7.0)
        assert all(bool((o == -7.0).all()) for o in call()) and S.workspace_status(ws) == 6
        with pytest.raises(S.SpecrollError):
            S.tree_attn_kv4(*t, x["parent"], workspace=ws, out=out[0], lse=out[1], check_status=True)
        t[4].copy_(dev(host_lens))
        assert all(torch.equal(o, w) for o, w in zip(call(), want)) and S.workspace_status(ws) == 0


def test_a_few_tokens_above_the_hosts_lengths():
    """More tokens, but no more chunks than the host's lengths make, or nothing cut at all: the lengths on the device are followed."""
    for lens, above in (([9000, 300], [9001, 330]), ([100, 120, 64], [129, 600, 0])):
        x = _case(len(lens), 1, 4, 2, 128, above, seed=51)
        t = [dev_bf16(x["Q"]), dev(x["pool"]), dev(x["table"]), dev(x["indptr"]), dev(x["len"]), np.array(lens, np.int32), dev_bf16(x["Kt"]), dev_bf16(x["Vt"])]
        got, want = S.tree_attn_kv4(*t, x["parent"], check_status=True), _check(x)
        assert (got.float() - want.float()).abs().max() <= 2.0 ** -6 * want.float().abs().max()


@pytest.mark.parametrize("kv_len,add", [(2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 126), (2 ** 31 - 130, 5), (0, 2 ** 31 - 1), (2 ** 31 - 1, 0)])
def test_a_page_plan_of_the_longest_lengths(kv_len, add):
    """The pages that a length near 2^31 needs, also where it and the tokens to come round up past 2^32."""
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = ([kv_len, 100], [add, 100], [7, 8, 9], [0, 2, 3], [4, 2, 5, 0], [3])
    p = S.page_plan(*[dev(np.array(a, np.int32)) for a in args], 8, 6, status=status)
    need = -(-(kv_len + add) // 128)
    assert host(p["page_indptr"]).tolist() == [0, need, need + 2]
    assert host(p["tok_indptr"]).tolist() == [0, add, min(add + 100, 2 ** 31 - 1)]
    assert host(p["page_table"]).tolist() == [7, 8, 4, 2, 5, -1, -1, -1]     # (all there are; the second sequence's places are far beyond)
    assert int(p["n_free"]) == 0 and host(p["free_list"]).tolist() == [-1] * 4 and int(status) == 6


@pytest.mark.parametrize("indptr,status_is", [([0, 2, 3, 5], 0), ([1, 2, 2, 5], 0), ([0, 2, 3, 6], 6), ([0, 2, 7, 9], 6), ([-1, 2, 3, 5], 6),
                                              ([0, 3, 2, 5], 6), ([0, 0, 0, 0], 0), ([9, 9, 9, 9], 0), ([-2 ** 31, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1], 6)])
@pytest.mark.parametrize("add", [(1, 1, 1), (1, -1, 1), (-1, -1, -1)])
def test_a_page_plan_of_places_outside_the_table(indptr, status_is, add):
    """A sequence whose places are not all in the table is reported, live or finished; what lies inside is what it was."""
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    table = np.array([10, 11, 12, 13, 14], np.int32)
    args = [np.array(a, np.int32) for a in ([0, 0, 0], add, table, indptr, [4, 2, 5, 3] + [0] * 12, [4])]
    p = S.page_plan(*[dev(a) for a in args], 16, 3, status=status)
    assert int(status) == status_is
    if status_is == 0:
        want = ref.page_plan(*args[:5], 4, 16, 3)
        for k in ("page_table", "page_indptr", "tok_indptr", "slot_map", "free_list"):
            assert np.array_equal(host(p[k]), want[k]), k
    elif indptr[0] >= -1:
        own = [[int(table[i]) if 0 <= i < 5 else -1 for i in range(indptr[b], indptr[b + 1])] for b in range(3)]
        free, tables = [4, 2, 5, 3], []
        for b in range(3):
            tables.append([] if add[b] < 0 else own[b] or [free.pop(0)])
        for b in range(3):
            free += own[b] if add[b] < 0 else []
        flat = sum(tables, [])
        assert host(p["page_table"]).tolist() == flat + [-1] * (16 - len(flat))
        assert host(p["free_list"]).tolist() == free + [-1] * (16 - len(free)) and int(p["n_free"]) == len(free)


# ------------------------------------------------------------------ writers and reader of many tokens and layers

def _stored(pool, slots, K, V, D):
    """The pool after K, V [T, Hkv, D] (float64) have gone to slots that differ (negative ones: nowhere), all tokens at once."""
    q, c = (x.copy() for x in ref.kv4_unpack(pool, D))                       # [page, Hkv, K or V, 128, ..]
    on = slots >= 0
    page, at = np.divmod(slots[on], 128)
    for i, x in enumerate((K, V)):
        xq, xc = ref.kv4_quantise(x[on])
        q[page, :, i, at], c[page, :, i, at] = xq, xc
    return ref.kv4_pack(q, c)


def test_the_oracle_for_many_tokens_is_the_oracle():
    g = np.random.default_rng(1)
    pool = g.integers(0, 256, (3, 2, 2, S.kv4_tile_bytes(64))).astype(np.uint8)
    slots, K, V = g.permutation(384)[:50].astype(np.int64), *(_f64(_bits(g, 50, 2, 64)) for _ in range(2))
    slots[3] = -1
    assert np.array_equal(_stored(pool, slots, K, V, 64), ref.kv4_store(K, V, slots, pool))


@pytest.mark.parametrize("T,H,D", [(1301, 8, 128), (9601, 2, 64), (6403, 3, 64), (803, 12, 128), (37, 12, 128), (130, 33, 64), (18949, 1, 64),
                                   (1185, 8, 128), (1184, 8, 128)])
def test_store_and_load_of_many_tokens_and_of_many_heads(T, H, D):
    """Four tokens a thread and a remainder (more than 303104 words of eight elements in all), tokens side by side in a block or a token in
    several blocks, and the largest call with one token a thread."""
    g = np.random.default_rng(T)
    K, V = _bits(g, T, H, D), _bits(g, T, H, D)
    pages = T // 128 + 2
    pool = g.integers(0, 256, (pages, H, 2, S.kv4_tile_bytes(D))).astype(np.uint8)
    slots = g.permutation(pages * 128)[:T].astype(np.int64)
    slots[g.permutation(T)[:5]] = -1
    dpool, status = dev(pool), torch.zeros(1, dtype=torch.int32, device="cuda")
    S.kv4_store(dev_bf16(K), dev_bf16(V), dev(slots), dpool, status=status)
    assert np.array_equal(host(dpool), _stored(pool, slots, _f64(K), _f64(V), D))
    for got, x in zip(S.kv4_load(dpool, dev(slots), status=status), (K, V)):
        want = np.where((slots >= 0)[:, None, None], ref.kv4_values(*ref.kv4_quantise(_f64(x))), 0.0)
        assert np.array_equal(host(got.double()), want)
    assert int(status) == 0
    far = slots.copy()
    far[T - 1] = pages * 128                                                 # the last token's slot is beyond the pool: only that is told
    S.kv4_store(dev_bf16(K), dev_bf16(V), dev(far), dpool, status=status)
    assert int(status) == 6


@pytest.mark.parametrize("B,layers,H,D,N,K", [(48, 28, 2, 64, 16, 4), (200, 27, 1, 64, 8, 5), (20, 65, 2, 128, 9, 8), (150, 9, 12, 128, 6, 2), (3, 130, 1, 64, 4, 1),
                                              (70, 17, 3, 128, 30, 7), (301, 8, 8, 128, 5, 3)])
@pytest.mark.parametrize("in_place", [False, True])
def test_commit_of_many_layers(B, layers, H, D, N, K, in_place):
    """Up to eight layers to a block with a remainder, rows of more than 256 words, and more layers than one launch takes."""
    g = np.random.default_rng(B + layers)
    kv_len = g.integers(0, 300, B).astype(np.int32)
    own = (kv_len + K + 1 + 127) // 128
    indptr = np.concatenate([[0], np.cumsum(own)]).astype(np.int32)
    table = g.permutation(indptr[-1] + 2)[:indptr[-1]].astype(np.int32)
    n_acc = g.integers(-1, min(K, N - 1) + 1, B).astype(np.int32)
    path = np.sort(np.argsort(g.random((B, max(N, K + 1))), 1)[:, :K + 1], 1).astype(np.int32) % N
    pos = kv_len[:, None] + np.arange(K + 1)
    slots = table[indptr[:-1, None] + pos // 128].astype(np.int64) * 128 + pos % 128
    slots[np.arange(K + 1) > n_acc[:, None]] = -1
    gt = torch.Generator(device="cuda").manual_seed(B)
    Kt, Vt = (torch.randn(layers, B, N, H, D, device="cuda", generator=gt).bfloat16() for _ in range(2))
    pools = torch.randint(0, 256, (layers, int(indptr[-1]) + 2, H, 2, S.kv4_tile_bytes(D)), dtype=torch.uint8, device="cuda", generator=gt)
    before = pools.clone()
    status, lens = torch.zeros(1, dtype=torch.int32, device="cuda"), dev(kv_len)
    out = lens if in_place else torch.full_like(lens, -9)
    S.commit_path_kv4_layers(list(Kt), list(Vt), dev(path), dev(n_acc), list(pools), dev(table), dev(indptr), lens, kv_len_out=out, status=status)
    assert int(status) == 0 and np.array_equal(host(out), kv_len + n_acc + 1)
    seq = torch.arange(B, device="cuda")[:, None]
    for l in range(layers):                                                  # (every layer against the writer by slot, some against the oracle)
        rows = [x[l][seq, dev(path).long()].flatten(0, 1).contiguous() for x in (Kt, Vt)]
        want = before[l].clone()
        S.kv4_store(*rows, dev(slots.reshape(-1)), want)
        assert torch.equal(pools[l], want), l
    for l in {0, layers // 2, layers - 1}:
        rows = [host(x[l][seq, dev(path).long()].flatten(0, 1).double()) for x in (Kt, Vt)]
        assert np.array_equal(host(pools[l]), _stored(host(before[l]), slots.reshape(-1), *rows, D)), l


# ------------------------------------------------------------------ plans of many units

def _cut(x):
    """Whether the plan cuts a sequence (its workspace is then larger than that of as many sequences of one token)."""
    B, N, Hq, D = x["Q"].shape
    f = S.tree_attn_kv4_workspace_bytes
    return f(B, N, Hq, x["Kt"].shape[2], D, x["len"]) > f(B, N, Hq, x["Kt"].shape[2], D, np.ones(B, np.int32))


@pytest.mark.parametrize("N,Hq,Hkv,D,lengths,merged_inside", [
    (17, 4, 4, 128, [2100] + [300 + 7 * b for b in range(39)], True), (24, 14, 2, 128, [2000, 1900] + [b * 53 % 700 for b in range(100)], True),
    (48, 10, 2, 128, [1500, 1400] + [b * 11 % 700 for b in range(60)], True), (33, 4, 4, 64, [1500, 1400] + [b * 53 % 700 for b in range(60)], True),
    (20, 6, 2, 128, [(b * 53) % 400 for b in range(180)], False), (18, 1, 1, 64, [(b * 31) % 300 for b in range(700)], False)])
def test_trees_in_more_units_than_ctas(N, Hq, Hkv, D, lengths, merged_inside):
    """Persistent CTAs that take several units each, with sequences in two to four chunks that the attention kernel merges itself, or whole."""
    x = _case(len(lengths), N, Hq, Hkv, D, lengths, seed=N)
    indptr = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    assert _cut(x) == merged_inside and S.tree_attn_launches(len(lengths), N, Hq, Hkv, D, indptr) == 2   # (plan and attention: no kernel merges)
    O = _check(x)
    assert all(torch.equal(O, _run(x)) for _ in range(10))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,Hq,Hkv,lengths", [(2, 8, 1, [9000]), (1, 8, 1, [9000, 0, 1]), (1, 16, 1, [700, 9001, 130]), (16, 1, 1, [5000, 4999])])
def test_few_rows_in_many_chunks(N, Hq, Hkv, lengths, D):
    """More than eight chunks of a sequence: the merge with several blocks a sequence and head, for both numbers of rows and both widths."""
    x = _case(len(lengths), N, Hq, Hkv, D, lengths, seed=60)
    assert _cut(x)
    O = _check(x)
    assert all(torch.equal(O, _run(x)) for _ in range(10))


@pytest.mark.parametrize("N,Hq", [(1, 4), (3, 4)])
def test_few_rows_of_many_sequences_of_which_some_are_cut(N, Hq):
    """The search for a unit where a thread has more sequences than it keeps pages of."""
    lengths = [(b * 13) % 90 for b in range(700)]
    for b in (0, 3, 5, 411, 699):
        lengths[b] = 20000 + b
    x = _case(700, N, Hq, 1, 64, lengths, seed=61)
    assert _cut(x)
    O = _check(x)
    assert all(torch.equal(O, _run(x)) for _ in range(10))


@pytest.mark.parametrize("N,Hq", [(1, 4), (8, 4), (30, 12)])
def test_attention_with_nothing_cached(N, Hq):
    """No sequence has tokens yet: an empty page table, and a pool of no pages."""
    x = _case(3, N, Hq, 2, 64, [0, 0, 0], seed=70)
    assert len(x["table"]) == 0
    O = _check(x)
    assert torch.equal(O, _run({**x, "pool": x["pool"][:0]})) and torch.equal(O, _run({**x, "table": np.array([2], np.int32)}))
