// Page tables, slot maps and the free list of a paged cache from the lengths of its sequences: one launch, nothing read back.
//
// Everything an output entry needs is in four running sums over the sequences (pages owned afterwards, new tokens, pages taken
// from the free list, pages given back), so no block waits for another: each makes the sums for itself in shared memory (a few
// loads and shuffles a sequence) and writes its share of the entries, finding an entry's sequence by bisection.  A decode
// step's call is bound by these latencies; many prompts' by writing eight bytes a slot.
#include <algorithm>

#include "common.cuh"

namespace specroll {

constexpr int PLAN_MAX_B = 4096, PLAN_THREADS = 512;
constexpr int PLAN_PER = 4;  // neighbouring slots a thread writes at a time (two 16-byte stores)
constexpr long long PLAN_SAT = 0x7fffffffLL;

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

__global__ void __launch_bounds__(PLAN_THREADS)
page_plan_kernel(const PagePlanArgs a) {
    extern __shared__ int32_t sums[];  // [4][B + 1]
    __shared__ long long warp_tot[4][PLAN_THREADS / 32];
    pdl_wait();
    pdl_launch_dependents();
    const int B = a.B, t = threadIdx.x, lane = t & 31, warp = t >> 5;
    int32_t *const owns = sums, *const toks = sums + (B + 1), *const takes = toks + (B + 1), *const gives = takes + (B + 1);
    const int nf = min(max(*a.n_free, 0), a.free_cap);

    // ---- per sequence: pages it had, takes, owns afterwards, gives back, and its new tokens; then the running sums.  They are
    // made in 64 bits and kept to 31: what is beyond is beyond every capacity too, and reported.
    const int per = (B + PLAN_THREADS - 1) / PLAN_THREADS, b0 = t * per, b1 = min(B, b0 + per);
    auto of_seq = [&](int b, long long (&v)[4]) {
        const int add = a.add[b];
        const long long len = max(a.kv_len[b], 0);
        const int had = max(a.indptr[b + 1] - a.indptr[b], 0);
        const long long need = (len + max(add, 0) + SPECROLL_PAGE_TOKENS - 1) / SPECROLL_PAGE_TOKENS;
        v[2] = add < 0 ? 0 : max(need - had, 0LL);
        v[0] = add < 0 ? 0 : had + v[2];
        v[1] = max(add, 0);
        v[3] = add < 0 ? had : 0;
    };
    long long run[4] = {0, 0, 0, 0}, tot[4];
    for (int b = b0; b < b1; ++b) {
        long long v[4];
        of_seq(b, v);
#pragma unroll
        for (int q = 0; q < 4; ++q) run[q] += v[q];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const long long mine = run[q];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, run[q], o);
            if (lane >= o) run[q] += x;
        }
        if (lane == 31) warp_tot[q][warp] = run[q];
        run[q] -= mine;  // exclusive within the warp
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        long long before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < PLAN_THREADS / 32; ++w) {
            const long long x = warp_tot[q][w];
            before += w < warp ? x : 0;
            all += x;
        }
        run[q] += before;
        tot[q] = all;
    }
    for (int b = b0; b < b1; ++b) {
        long long v[4];
        of_seq(b, v);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            sums[q * (B + 1) + b] = (int32_t)min(run[q], PLAN_SAT);
            run[q] += v[q];
        }
    }
    if (t < 4) sums[t * (B + 1) + B] = (int32_t)min(t == 0 ? tot[0] : t == 1 ? tot[1] : t == 2 ? tot[2] : tot[3], PLAN_SAT);
    __syncthreads();

    const long long left = max((long long)nf - tot[2], 0LL), free_after = left + tot[3];
    if (blockIdx.x == 0 && t == 0) {
        *a.n_free_out = (int32_t)min(free_after, (long long)a.free_cap);
        if (a.status && (tot[2] > nf || tot[0] > a.table_cap || tot[1] > min(a.slot_cap, PLAN_SAT) || free_after > a.free_cap))
            atomicExch(a.status, SPECROLL_ELIMIT);
    }

    // the pages as they were, and those of the free list, by place; -1 where there is none
    auto old_page = [&](int b, int i) -> int {
        const long long at = (long long)a.indptr[b] + i;
        return at >= 0 && at < a.n_table ? __ldg(a.table + at) : -1;
    };
    auto new_page = [&](long long j) -> int { return j < nf ? __ldg(a.free_list + j) : -1; };
    auto page_of = [&](int b, int i, int had) -> int { return i < had ? old_page(b, i) : new_page((long long)takes[b] + i - had); };

    const long long stride = (long long)gridDim.x * PLAN_THREADS, me = (long long)blockIdx.x * PLAN_THREADS + t;
    for (long long i = me; i <= B; i += stride) {
        a.indptr_out[i] = owns[i];
        a.tok_indptr[i] = toks[i];
    }
    for (long long i = me; i < a.table_cap; i += stride) {
        int page = -1;
        if (i < tot[0]) {
            const int b = plan_seq_of(owns, B, (int)i);
            page = page_of(b, (int)i - owns[b], max(a.indptr[b + 1] - a.indptr[b], 0));
        }
        a.table_out[i] = page;
    }
    for (long long i = me; i < a.free_cap; i += stride) {
        int page = -1;
        if (i < left) page = new_page(tot[2] + i);
        else if (i < free_after) {
            const int at = (int)(i - left), b = plan_seq_of(gives, B, at);
            page = old_page(b, at - gives[b]);
        }
        a.free_out[i] = page;
    }
    const long long n_slots = min(a.slot_cap, PLAN_SAT);
    for (long long i0 = me * PLAN_PER; i0 < a.slot_cap; i0 += stride * PLAN_PER) {
        long long out[PLAN_PER];
        int b = -1, had = 0, end = -1, page = -1;
        long long first = 0, in_page = -1;  // the sequence's first new position less its first new token; the page held
#pragma unroll
        for (int q = 0; q < PLAN_PER; ++q) {
            const long long i = i0 + q;
            out[q] = -1;
            if (i >= min(tot[1], n_slots)) continue;
            if (i >= end) {
                b = plan_seq_of(toks, B, (int)i);
                end = toks[b + 1];
                had = max(a.indptr[b + 1] - a.indptr[b], 0);
                first = (long long)max(a.kv_len[b], 0) - toks[b];
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
    // blocks read the old state while others write the new one
    const auto meet = [](const int32_t *x, long long nx, const int32_t *y, long long ny) { return x && y && x < y + ny && y < x + nx; };
    if (meet(page_table, n_table, page_table_out, table_cap) || meet(free_list, free_cap, free_list_out, free_cap) || meet(n_free, 1, n_free_out, 1) ||
        meet(page_indptr, (long long)B + 1, page_indptr_out, (long long)B + 1))
        return SPECROLL_EINVAL;
    const size_t smem = (size_t)4 * (B + 1) * sizeof(int32_t);
    int n_sm = 0;
    const int rc = device_setup(reinterpret_cast<const void *>(page_plan_kernel), 4 * (PLAN_MAX_B + 1) * (int)sizeof(int32_t), &n_sm);
    if (rc != SPECROLL_OK) return rc;
    const PagePlanArgs a = {kv_len, add, page_table, page_indptr, free_list, n_free, page_table_out, page_indptr_out, tok_indptr,
                            free_list_out, n_free_out, status, reinterpret_cast<long long *>(slot_map), B, n_table, free_cap, table_cap,
                            slot_cap};
    // as many blocks as give every thread an entry or four neighbouring slots, up to two a multiprocessor
    const long long most = std::max<long long>({(long long)B + 1, table_cap, free_cap, (slot_cap + PLAN_PER - 1) / PLAN_PER});
    const long long want = std::min<long long>((most + PLAN_THREADS - 1) / PLAN_THREADS, 2LL * n_sm);
    SR_CUDA_TRY(launch_dependent(true, page_plan_kernel, dim3((unsigned)std::max<long long>(want, 1)), dim3(PLAN_THREADS), smem,
                                 static_cast<cudaStream_t>(cuda_stream), a));
    return SPECROLL_OK;
}
