// Page tables, slot maps and the free list of a paged cache from the lengths of its sequences: one launch, nothing read back.
//
// Everything an output entry needs is in four running sums over the sequences (pages owned afterwards, new tokens, pages taken
// from the free list, pages given back), so no block waits for another: each makes the sums for itself in shared memory (a few
// loads and shuffles a sequence) and writes its share of the entries, finding an entry's sequence by bisection.  A decode
// step's call is bound by these latencies; many prompts' by writing eight bytes a slot.
#include <algorithm>

#include "common.cuh"

namespace specroll {

constexpr int PLAN_MAX_B = 4096, PLAN_THREADS = 256;
constexpr int PLAN_PER = 4;  // neighbouring slots a thread writes at a time (two 16-byte stores)
constexpr uint32_t PLAN_SAT = 0x7fffffffu;

struct PagePlanArgs {
    const int32_t *kv_len, *add, *table, *indptr, *free_list, *n_free;
    int32_t *table_out, *indptr_out, *tok_indptr, *free_out, *n_free_out, *status;
    long long *slots;
    int32_t B, n_table, free_cap, table_cap;
    long long slot_cap;
};

// The largest b in [0, B) with sum[b] <= at (sum[0] = 0, at < sum[B]).
__device__ __forceinline__ int plan_seq_of(const int32_t *sum, int B, int at) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sum[mid] <= at) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Sums stop at 2^31 - 1: what is beyond is beyond every capacity too, and reported.
__device__ __forceinline__ uint32_t plan_add(uint32_t x, uint32_t y) { return min(x + y, PLAN_SAT); }

__global__ void __launch_bounds__(PLAN_THREADS)
page_plan_kernel(const PagePlanArgs a) {
    extern __shared__ int32_t sums[];  // [4][B + 1] running sums, then of every sequence its first old page's place, its old pages, its length
    __shared__ uint32_t warp_tot[4][PLAN_THREADS / 32];
    pdl_wait();
    pdl_launch_dependents();
    const int B = a.B, t = threadIdx.x, lane = t & 31, warp = t >> 5;
    int32_t *const owns = sums, *const toks = sums + (B + 1), *const takes = toks + (B + 1), *const gives = takes + (B + 1);
    int32_t *const old_at = gives + (B + 1), *const hads = old_at + B, *const lens = hads + B;
    const int nf_given = __ldg(a.n_free);

    // ---- per sequence: pages it owns afterwards, new tokens, pages it takes, pages it gives back; then the running sums
    const int per = (B + PLAN_THREADS - 1) / PLAN_THREADS, b0 = min(B, t * per), b1 = min(B, b0 + per);
    auto of_seq = [&](int b, int add, uint32_t (&v)[4]) {
        const uint32_t had = (uint32_t)hads[b], more = add < 0 ? 0u : (uint32_t)add;
        // (in 64 bits: both are below 2^31, but their sum rounded up to pages may pass 2^32)
        const uint32_t need = (uint32_t)(((unsigned long long)(uint32_t)lens[b] + more + (SPECROLL_PAGE_TOKENS - 1)) / SPECROLL_PAGE_TOKENS);
        v[1] = more;
        v[2] = add < 0 || need < had ? 0u : need - had;
        v[0] = add < 0 ? 0u : had + v[2];
        v[3] = add < 0 ? had : 0u;
    };
    uint32_t run[4] = {0u, 0u, 0u, 0u}, tot[4], one[4];
    bool astray = false;  // a sequence whose pages are not all in the table: those outside count as -1, and the caller is told
    for (int b = b0; b < b1; ++b) {
        const int at = a.indptr[b], end = a.indptr[b + 1], add = a.add[b], len = a.kv_len[b];
        old_at[b] = at;
        hads[b] = end > at ? (int)min((long long)end - at, (long long)PLAN_SAT) : 0;
        astray |= end < at || (end > at && (at < 0 || end > a.n_table));
        lens[b] = max(len, 0);
        of_seq(b, add, one);
#pragma unroll
        for (int q = 0; q < 4; ++q) run[q] = plan_add(run[q], one[q]);
    }
    if (astray && blockIdx.x == 0 && a.status) atomicExch(a.status, SPECROLL_ELIMIT);
    uint32_t before[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t incl = run[q];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl = plan_add(incl, x);
        }
        if (lane == 31) warp_tot[q][warp] = incl;
        before[q] = __shfl_up_sync(0xffffffffu, incl, 1);  // exclusive within the warp
        if (lane == 0) before[q] = 0u;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t ahead = 0u, all = 0u;
#pragma unroll
        for (int w = 0; w < PLAN_THREADS / 32; ++w) {
            const uint32_t x = warp_tot[q][w];
            ahead = w < warp ? plan_add(ahead, x) : ahead;
            all = plan_add(all, x);
        }
        run[q] = plan_add(before[q], ahead);
        tot[q] = all;
    }
    for (int b = b0; b < b1; ++b) {
        if (per > 1) of_seq(b, a.add[b], one);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            sums[q * (B + 1) + b] = (int32_t)run[q];
            run[q] = plan_add(run[q], one[q]);
        }
    }
    if (t < 4) sums[t * (B + 1) + B] = (int32_t)(t == 0 ? tot[0] : t == 1 ? tot[1] : t == 2 ? tot[2] : tot[3]);
    __syncthreads();

    const int nf = min(max(nf_given, 0), a.free_cap);
    const long long left = max((long long)nf - tot[2], 0LL), free_after = left + tot[3];
    if (blockIdx.x == 0 && t == 0) {
        *a.n_free_out = (int32_t)min(free_after, (long long)a.free_cap);
        if (a.status && (tot[2] > (uint32_t)nf || tot[0] > (uint32_t)a.table_cap || tot[1] > min(a.slot_cap, (long long)PLAN_SAT - 1) || free_after > a.free_cap))
            atomicExch(a.status, SPECROLL_ELIMIT);
    }

    // the pages as they were, and those of the free list, by place; -1 where there is none
    auto old_page = [&](int b, int i) -> int {
        const long long at = (long long)old_at[b] + i;
        return at >= 0 && at < a.n_table ? __ldg(a.table + at) : -1;
    };
    auto new_page = [&](long long j) -> int { return j < nf ? __ldg(a.free_list + j) : -1; };
    auto page_of = [&](int b, int i, int had) -> int { return i < had ? old_page(b, i) : new_page((long long)takes[b] + i - had); };

    // one index for all entries (index rows, the table, the free list, groups of slots), so that a thread has one chain of latencies
    const long long n_slots = min((long long)tot[1], min(a.slot_cap, (long long)PLAN_SAT));
    const long long to_table = B + 1, to_free = to_table + a.table_cap, to_slots = to_free + a.free_cap;
    const long long end_of_all = to_slots + (a.slot_cap + PLAN_PER - 1) / PLAN_PER;
    for (long long e = (long long)blockIdx.x * PLAN_THREADS + t; e < end_of_all; e += (long long)gridDim.x * PLAN_THREADS) {
        if (e < to_table) {
            a.indptr_out[e] = owns[e];
            a.tok_indptr[e] = toks[e];
            continue;
        }
        if (e < to_free) {
            const long long i = e - to_table;
            int page = -1;
            if (i < tot[0]) {
                const int b = plan_seq_of(owns, B, (int)i);
                page = page_of(b, (int)i - owns[b], hads[b]);
            }
            a.table_out[i] = page;
            continue;
        }
        if (e < to_slots) {
            const long long i = e - to_free;
            int page = -1;
            if (i < left) page = new_page((long long)tot[2] + i);
            else if (i < free_after) {
                const int at = (int)(i - left), b = plan_seq_of(gives, B, at);
                page = old_page(b, at - gives[b]);
            }
            a.free_out[i] = page;
            continue;
        }
        const long long i0 = (e - to_slots) * PLAN_PER;
        long long out[PLAN_PER];
        int b = -1, had = 0, end = -1, page = -1;
        long long first = 0, in_page = -1;  // the sequence's first new position less its first new token; the page held
#pragma unroll
        for (int q = 0; q < PLAN_PER; ++q) {
            const long long i = i0 + q;
            out[q] = -1;
            if (i >= n_slots) continue;
            if (i >= end) {
                b = plan_seq_of(toks, B, (int)i);
                end = toks[b + 1];
                had = hads[b];
                first = (long long)lens[b] - toks[b];
                in_page = -1;
            }
            const long long pos = first + i, p = pos / SPECROLL_PAGE_TOKENS;
            if (p != in_page) {
                page = page_of(b, (int)p, had);
                in_page = p;
            }
            if (page >= 0) out[q] = (long long)page * SPECROLL_PAGE_TOKENS + pos % SPECROLL_PAGE_TOKENS;
        }
        if (i0 + PLAN_PER <= a.slot_cap) {
#pragma unroll
            for (int q = 0; q < PLAN_PER; q += 2) *reinterpret_cast<longlong2 *>(a.slots + i0 + q) = make_longlong2(out[q], out[q + 1]);
        } else {
#pragma unroll
            for (int q = 0; q < PLAN_PER; ++q)
                if (i0 + q < a.slot_cap) a.slots[i0 + q] = out[q];
        }
    }
}

}  // namespace specroll

using namespace specroll;

static size_t plan_smem(int B) { return (size_t)(7 * B + 4) * sizeof(int32_t); }

extern "C" int specroll_page_plan(int32_t B, const int32_t *kv_len, const int32_t *add, const int32_t *page_table, int32_t n_table,
                                  const int32_t *page_indptr, const int32_t *free_list, int32_t free_cap, const int32_t *n_free,
                                  int32_t table_cap, int64_t slot_cap, int32_t *page_table_out, int32_t *page_indptr_out,
                                  int32_t *tok_indptr, int64_t *slot_map, int32_t *free_list_out, int32_t *n_free_out, int32_t *status,
                                  void *cuda_stream) {
    if (B < 0 || n_table < 0 || free_cap < 0 || table_cap < 0 || slot_cap < 0 || free_cap > (1 << 24)) return SPECROLL_EINVAL;
    if (B > PLAN_MAX_B) return SPECROLL_ELIMIT;
    if (!page_indptr_out || !tok_indptr || !n_free || !n_free_out || (table_cap && !page_table_out) || (slot_cap && !slot_map) ||
        (free_cap && (!free_list || !free_list_out)) || (n_table && !page_table) || (B && (!kv_len || !add || !page_indptr)))
        return SPECROLL_EINVAL;
    if (!aligned16(slot_map)) return SPECROLL_EALIGN;
    // blocks read the old state while others write the new one: no output meets an input or another output
    struct Span {
        uintptr_t at, bytes;
    };
    const auto span = [](const void *x, long long n, size_t size) { return Span{reinterpret_cast<uintptr_t>(x), x ? (uintptr_t)n * size : 0}; };
    const Span spans[] = {span(page_table_out, table_cap, 4), span(page_indptr_out, B + 1LL, 4), span(tok_indptr, B + 1LL, 4), span(slot_map, slot_cap, 8),
                          span(free_list_out, free_cap, 4), span(n_free_out, 1, 4), span(status, 1, 4), span(kv_len, B, 4), span(add, B, 4),
                          span(page_table, n_table, 4), span(page_indptr, B ? B + 1LL : 0, 4), span(free_list, free_cap, 4), span(n_free, 1, 4)};
    constexpr int OUTS = 7, SPANS = sizeof(spans) / sizeof(spans[0]);
    for (int i = 0; i < OUTS; ++i)
        for (int j = i + 1; j < SPANS; ++j)
            if (spans[i].bytes && spans[j].bytes && spans[i].at < spans[j].at + spans[j].bytes && spans[j].at < spans[i].at + spans[i].bytes) return SPECROLL_EINVAL;
    const size_t smem = plan_smem(B);
    int n_sm = 0;
    const int rc = device_setup(reinterpret_cast<const void *>(page_plan_kernel), (int)plan_smem(PLAN_MAX_B), &n_sm);
    if (rc != SPECROLL_OK) return rc;
    const PagePlanArgs a = {kv_len, add, page_table, page_indptr, free_list, n_free, page_table_out, page_indptr_out, tok_indptr,
                            free_list_out, n_free_out, status, reinterpret_cast<long long *>(slot_map), B, n_table, free_cap, table_cap,
                            slot_cap};
    // as many blocks as give every thread an entry or four neighbouring slots, up to two a multiprocessor: every block makes the sums for
    // itself (1021 sequences, 10^6 slots: 11.2 us with 256 threads twice a multiprocessor, 14 with 512 twice, 15 with 256 once)
    const long long all = (long long)B + 1 + table_cap + free_cap + (slot_cap + PLAN_PER - 1) / PLAN_PER;
    const long long want = std::min<long long>((all + PLAN_THREADS - 1) / PLAN_THREADS, 2LL * n_sm);
    SR_CUDA_TRY(launch_dependent(true, page_plan_kernel, dim3((unsigned)std::max<long long>(want, 1)), dim3(PLAN_THREADS), smem,
                                 static_cast<cudaStream_t>(cuda_stream), a));
    return SPECROLL_OK;
}
