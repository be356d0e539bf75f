// Writing and reading the 4-bit paged cache: tokens by slot (prompts), the committed path of a round, and back to bf16.
//
// A block of 32 elements has one scale, the largest magnitude over 7 to four significant bits, and codes to the nearest
// multiple of it.  All three are bound by HBM: a token's head is 2 D bytes of bf16 against 17 D / 32 bytes of codes and scales.
// A thread has eight elements (16 bytes of bf16, one 32-bit word of codes), four threads a block, so that both sides are
// contiguous over a warp.  The arithmetic is kept to about four instructions an element, because the writer is otherwise
// bound by it: a multiple of the reciprocal is added to a constant whose last four bits then are the code.  98304 tokens of eight
// heads of 128 (510 MB): store 103 us, with 80 % of the issue slots taken, load 94 us; the copy rate of HBM would have 78 each.
#include <algorithm>

#include "kv4.cuh"

namespace specroll {

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Codes of eight elements, and the block's scale byte, from the four threads that share the block.
__device__ __forceinline__ uint32_t kv4_encode(const uint4 &x, uint32_t &scale) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    // magnitudes as integers: 0x7f80 is infinity, above it NaN
    uint32_t m2 = w[0] & 0x7fff7fffu;
#pragma unroll
    for (int i = 1; i < 4; ++i) m2 = max_u16x2(m2, w[i] & 0x7fff7fffu);
    m2 = max_u16x2(m2, __shfl_xor_sync(0xffffffffu, m2, 1));
    m2 = max_u16x2(m2, __shfl_xor_sync(0xffffffffu, m2, 2));
    uint32_t top = max(m2 & 0xffffu, m2 >> 16);
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    bool clip = false;
    if (top > 0x7f80u) {  // some NaN in the block: it counts as 0
        float mx = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = v[i] == v[i] ? v[i] : 0.f;
            mx = fmaxf(mx, fabsf(v[i]));
        }
        // (the four threads of a block take this branch together)
        const uint32_t four = 0xfu << (threadIdx.x & 28u);
        mx = fmaxf(mx, __shfl_xor_sync(four, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(four, mx, 2));
        top = __float_as_uint(mx) >> 16;
    }
    // (128 + M) 2^(E - 134) over 7 to four significant bits, halves up: (128 + M) / 14 or, from 224 on, / 28, rounded
    const int M = (int)(top & 127u), r = M < 96 ? ((135 + M) * 4682 >> 16) - 8 : (142 + M) * 2341 >> 16;
    int c = 8 * ((int)(top >> 7) - 110) + r;
    if (c > 255) {
        c = 255;
        clip = true;
    }
    if (c < 0) c = 0;
    const float s = __uint_as_float(kv4_scale_bits((uint32_t)c) << 16);
    if (clip) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fminf(fmaxf(v[i], -8.0f * s), 7.0f * s);
    }
    // The reciprocal (good to 2^-23) is taken a little too large, so that halves, which are exact quotients, go away from zero; every
    // other quotient of an 8-bit and a 4-bit significand is further than 2^-12 from a half.  1.5 2^23 + 8 leaves code = q + 8.
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    inv *= 1.0f + 0x1p-21f;
    uint32_t y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __float_as_uint(fmaf(v[i], inv, 12582920.0f));
    const uint32_t even = y[0] + (y[2] << 4) + (y[4] << 8) + (y[6] << 12), odd = y[1] + (y[3] << 4) + (y[5] << 8) + (y[7] << 12);
    scale = (uint32_t)c;
    return __byte_perm(even, odd, 0x5410);
}

constexpr int KV4_THREADS = 256, KV4_EACH = 4;  // words of 16 bytes of bf16 that a thread takes side by side

// What the two kernels by slot share out.  A thread has one word of K or of V of its tokens for good (a token has `columns` = 2 Hkv D / 8
// words; 256 threads are 256 / columns tokens side by side, or a part of one, by blockIdx.y) and goes through tokens, so that everything
// but the slot is found once, in 32 bits (with places in 64 bits found for every word the kernels took 160 instructions a word and were
// bound by them).  A warp reads and writes contiguous memory on the bf16 side.
struct Kv4Tokens {
    const long long *slots;
    unsigned long long n_slots;  // slots of the pool
    uint32_t T, columns, side, each, page_bytes;  // tokens; words of a token; tokens side by side; tokens of a thread; bytes of a page
};

template <int D>
struct Kv4Column {
    uint32_t tok, word, v;  // first token, word of K or V
    uint32_t at, sat;       // places of the word's codes and scale in row 0 of the head's tile, from the page's first byte
    bool on;
    __device__ __forceinline__ explicit Kv4Column(const Kv4Tokens &a) {
        const uint32_t l = a.columns < KV4_THREADS ? threadIdx.x / a.columns : 0u;
        const uint32_t col = threadIdx.x - l * a.columns + blockIdx.y * KV4_THREADS, words = a.columns / 2;
        on = l < a.side && col < a.columns;
        v = col >= words;
        word = v ? col - words : col;
        tok = blockIdx.x * a.side * a.each + l;
        const uint32_t tile = (word / (D / 8) * 2 + v) * Kv4<D>::TILE, of_head = word % (D / 8);
        at = tile + of_head * 4;
        sat = tile + Kv4<D>::CODES + of_head / 4;
    }
    __device__ __forceinline__ bool has(const Kv4Tokens &a, uint32_t q) const { return on && q < a.each && tok + q * a.side < a.T; }
    __device__ __forceinline__ unsigned long long slot(const Kv4Tokens &a, uint32_t q) const {
        return has(a, q) ? (unsigned long long)__ldg(a.slots + tok + q * a.side) : ~0ull;
    }
};
static_assert(SPECROLL_PAGE_TOKENS == 128, "slot >> 7");

template <int D>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_store_kernel(const uint4 *__restrict__ K, const uint4 *__restrict__ V, const Kv4Tokens a, uint8_t *__restrict__ pool,
                 int32_t *__restrict__ status) {
    pdl_wait();
    pdl_launch_dependents();
    const Kv4Column<D> c(a);
    const uint4 *const src = (c.v ? V : K) + c.word;
    unsigned long long slot[KV4_EACH];
    uint4 x[KV4_EACH];
#pragma unroll
    for (uint32_t q = 0; q < KV4_EACH; ++q) slot[q] = c.slot(a, q);
#pragma unroll
    for (uint32_t q = 0; q < KV4_EACH; ++q)
        x[q] = slot[q] < a.n_slots ? ld_nc_v4(src + (unsigned long long)(c.tok + q * a.side) * (a.columns / 2)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (uint32_t q = 0; q < KV4_EACH; ++q) {
        uint32_t scale;
        const uint32_t codes = kv4_encode(x[q], scale);  // (four threads a block of 32, all in it together)
        if (slot[q] < a.n_slots) {
            uint8_t *const page = pool + (unsigned long long)(uint32_t)(slot[q] >> 7) * a.page_bytes;
            const uint32_t row = (uint32_t)slot[q] & 127u;
            *reinterpret_cast<uint32_t *>(page + (c.at + row * Kv4<D>::ROW)) = codes;
            if ((c.word & 3) == 0) page[c.sat + row * Kv4<D>::SROW] = (uint8_t)scale;
        } else if ((long long)slot[q] >= 0 && status && c.word == 0) {
            atomicExch(status, SPECROLL_ELIMIT);
        }
    }
}

template <int D>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_load_kernel(const uint8_t *__restrict__ pool, const Kv4Tokens a, uint4 *__restrict__ K, uint4 *__restrict__ V, int32_t *__restrict__ status) {
    pdl_wait();
    pdl_launch_dependents();
    const Kv4Column<D> c(a);
    uint4 *const dst = (c.v ? V : K) + c.word;
    unsigned long long slot[KV4_EACH];
    uint32_t codes[KV4_EACH], scale[KV4_EACH];
#pragma unroll
    for (uint32_t q = 0; q < KV4_EACH; ++q) slot[q] = c.slot(a, q);
#pragma unroll
    for (uint32_t q = 0; q < KV4_EACH; ++q) {
        codes[q] = 0x88888888u;  // (zeros)
        scale[q] = 0u;
        if (slot[q] < a.n_slots) {
            const uint8_t *const page = pool + (unsigned long long)(uint32_t)(slot[q] >> 7) * a.page_bytes;
            const uint32_t row = (uint32_t)slot[q] & 127u;
            codes[q] = __ldg(reinterpret_cast<const uint32_t *>(page + (c.at + row * Kv4<D>::ROW)));
            scale[q] = __ldg(page + (c.sat + row * Kv4<D>::SROW));
        } else if ((long long)slot[q] >= 0 && status && c.word == 0) {
            atomicExch(status, SPECROLL_ELIMIT);
        }
    }
#pragma unroll
    for (uint32_t q = 0; q < KV4_EACH; ++q) {
        uint32_t r[4];
        kv4_word(codes[q], kv4_scale_of(scale[q]), r);
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = hmul2_bf16(r[i], KV4_UP_PAIR);
        if (c.has(a, q)) __stcs(dst + (unsigned long long)(c.tok + q * a.side) * (a.columns / 2), make_uint4(r[0], r[1], r[2], r[3]));
    }
}

constexpr int KV4_COMMIT_LAYERS = 64;  // layers one launch can serve (their pointers travel as kernel arguments)

struct Kv4Layers {
    const uint4 *Kt[KV4_COMMIT_LAYERS], *Vt[KV4_COMMIT_LAYERS];
    uint8_t *pool[KV4_COMMIT_LAYERS];
};

// grid = (B, groups of `each` layers): the committed rows of sequence b go to cache positions kv_len[b] + i of those layers' pools, as
// commit_path_kernel has it for a bf16 cache.  The first warp finds the rows' places, once for K, V and all layers of the group (a block
// for every row and layer spent its time on that chain of loads); a thread then has one column, as above, and takes four words at a time.
template <int D>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_commit_kernel(const __grid_constant__ Kv4Layers lay, const int32_t *__restrict__ path_node, const int32_t *__restrict__ n_acc,
                  long long n_pages, const int32_t *__restrict__ page_table, const int32_t *__restrict__ page_indptr,
                  const int32_t *__restrict__ kv_len, int N, int K, int Hkv, int n_layers, int each, int32_t *__restrict__ status,
                  int32_t *__restrict__ kv_len_out) {
    constexpr int W = D / 8;
    __shared__ long long sh_src[SPECROLL_MAX_HEADS + 1], sh_page[SPECROLL_MAX_HEADS + 1];  // first word of the tree row; first byte of the page
    __shared__ uint32_t sh_row[SPECROLL_MAX_HEADS + 1];
    __shared__ int sh_rows;
    pdl_wait();
    pdl_launch_dependents();
    const int b = blockIdx.x;
    if (threadIdx.x < 32) {
        const int i = threadIdx.x, na = n_acc[b], len = kv_len[b], first = page_indptr[b], own = page_indptr[b + 1] - first;
        const bool committed = na >= 0 && na <= K;
        const bool mine = committed && i <= na;
        const int node = mine ? path_node[(size_t)b * (K + 1) + i] : -1;
        const long long pos = (long long)len + i, at = pos / SPECROLL_PAGE_TOKENS;
        int page = -1;
        if (node >= 0 && node < N && len >= 0 && at < own) page = page_table[first + at];
        const bool ok = page >= 0 && page < n_pages;
        // no room (or a bad table): nothing is written for this token, and the caller is told
        if (mine && !ok && status && blockIdx.y == 0) atomicExch(status, SPECROLL_ELIMIT);
        const uint32_t have = __ballot_sync(0xffffffffu, ok);
        if (ok) {
            const int r = __popc(have & ((1u << i) - 1u));
            sh_src[r] = ((long long)b * N + node) * Hkv * W;
            sh_page[r] = (long long)page * Hkv * (2 * Kv4<D>::TILE);
            sh_row[r] = (uint32_t)(pos % SPECROLL_PAGE_TOKENS);
        }
        if (i == 0) {
            sh_rows = __popc(have);
            if (kv_len_out && blockIdx.y == 0) kv_len_out[b] = len + (committed ? na + 1 : 0);
        }
    }
    __syncthreads();
    // a thread has one word of K or V (or several, KV4_THREADS apart) of `side` (layer, row) pairs side by side and goes through the pairs
    const uint32_t words = (uint32_t)(Hkv * W), columns = 2 * words, rows = (uint32_t)sh_rows, l0 = blockIdx.y * each;
    const uint32_t pairs = rows * (uint32_t)min(each, n_layers - (int)l0), side = max(1u, KV4_THREADS / columns);
    const uint32_t first = columns < KV4_THREADS ? threadIdx.x / columns : 0u;
    const uint32_t per_row = rows ? 65536u / rows + 1u : 0u;  // (pair * per_row >> 16 is pair / rows: pairs are below 2^8)
    for (uint32_t c0 = 0; c0 < columns; c0 += KV4_THREADS) {
        const uint32_t col = threadIdx.x - first * columns + c0, v = col >= words, word = v ? col - words : col;
        const bool on = first < side && col < columns;
        const uint32_t tile = (word / W * 2 + v) * Kv4<D>::TILE, at = tile + word % W * 4, sat = tile + Kv4<D>::CODES + word % W / 4;
        for (uint32_t p0 = 0; p0 < pairs; p0 += side * KV4_EACH) {
            uint4 x[KV4_EACH];
            uint32_t lr[KV4_EACH];  // layer and row of the pair
#pragma unroll
            for (uint32_t q = 0; q < KV4_EACH; ++q) {
                const uint32_t p = p0 + first + q * side, l = p * per_row >> 16, r = p - l * rows;
                const bool has = on && p < pairs;
                lr[q] = has ? l << 8 | r : ~0u;
                x[q] = has ? ld_nc_v4((v ? lay.Vt[l0 + l] : lay.Kt[l0 + l]) + sh_src[r] + word) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (uint32_t q = 0; q < KV4_EACH; ++q) {
                uint32_t scale;
                const uint32_t codes = kv4_encode(x[q], scale);  // (four threads a block of 32, all in it together)
                if (lr[q] == ~0u) continue;
                uint8_t *const page = lay.pool[l0 + (lr[q] >> 8)] + sh_page[lr[q] & 255u];
                const uint32_t row = sh_row[lr[q] & 255u];
                *reinterpret_cast<uint32_t *>(page + (at + row * Kv4<D>::ROW)) = codes;
                if ((word & 3) == 0) page[sat + row * Kv4<D>::SROW] = (uint8_t)scale;
            }
        }
    }
}

__global__ void kv4_len_kernel(const int32_t *kv_len, const int32_t *__restrict__ n_acc, int B, int K, int32_t *kv_len_out) {
    pdl_wait();
    pdl_launch_dependents();
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= B) return;
    const int na = n_acc[b];
    kv_len_out[b] = kv_len[b] + ((na < 0 || na > K) ? 0 : na + 1);
}

}  // namespace specroll

using namespace specroll;

extern "C" size_t specroll_kv4_tile_bytes(int32_t D) {
    return D == 64 ? Kv4<64>::TILE : D == 128 ? Kv4<128>::TILE : 0;
}

// What the two calls by slot share: the checks, and how the tokens are shared out (grid.x = 0: nothing to do).
static int by_slot(int64_t T, int32_t Hkv, int32_t D, const void *K, const void *V, const int64_t *slots, const void *pool, int64_t n_pages,
                   Kv4Tokens *a, dim3 *grid) {
    grid->x = 0;
    if (T < 0 || T > (1LL << 30) || Hkv < 1 || Hkv > 4096 || (D != 64 && D != 128) || n_pages < 0 || n_pages > (1LL << 24)) return SPECROLL_EINVAL;
    if (T == 0) return SPECROLL_OK;  // (no tokens have empty arrays: their pointers may be NULL)
    if (!K || !V || !slots || (n_pages > 0 && !pool)) return SPECROLL_EINVAL;
    if (!aligned16(K) || !aligned16(V) || !aligned16(pool)) return SPECROLL_EALIGN;
    a->slots = reinterpret_cast<const long long *>(slots);
    a->n_slots = (unsigned long long)n_pages * SPECROLL_PAGE_TOKENS;
    a->T = (uint32_t)T;
    a->columns = (uint32_t)(2 * Hkv * (D / 8));
    a->page_bytes = (uint32_t)(Hkv * 2 * specroll_kv4_tile_bytes(D));
    a->side = std::max(1u, KV4_THREADS / a->columns);
    // one word a thread while that is less than a wave of blocks: few tokens are a chain of latencies (store and load, us: 37 tokens 3.4, with
    // four words 3.9; 98304 tokens 500 and 197; eight or sixteen, four at a time: 197)
    a->each = T * a->columns > 148LL * 8 * KV4_THREADS ? KV4_EACH : 1;
    grid->x = (unsigned)((T + a->side * a->each - 1) / (a->side * a->each));
    grid->y = (a->columns + KV4_THREADS - 1) / KV4_THREADS;
    return SPECROLL_OK;
}

extern "C" int specroll_kv4_store(int64_t T, int32_t Hkv, int32_t D, const void *K, const void *V, const int64_t *slot_map, void *pool,
                                  int64_t n_pages, int32_t *status, void *cuda_stream) {
    Kv4Tokens a;
    dim3 grid;
    const int rc = by_slot(T, Hkv, D, K, V, slot_map, pool, n_pages, &a, &grid);
    if (rc != SPECROLL_OK || grid.x == 0) return rc;
    SR_CUDA_TRY(launch_dependent(true, D == 128 ? kv4_store_kernel<128> : kv4_store_kernel<64>, grid, dim3(KV4_THREADS), 0,
                                 static_cast<cudaStream_t>(cuda_stream), static_cast<const uint4 *>(K), static_cast<const uint4 *>(V), a,
                                 static_cast<uint8_t *>(pool), status));
    return SPECROLL_OK;
}

extern "C" int specroll_kv4_load(int64_t T, int32_t Hkv, int32_t D, const void *pool, int64_t n_pages, const int64_t *slot_map, void *K,
                                 void *V, int32_t *status, void *cuda_stream) {
    Kv4Tokens a;
    dim3 grid;
    const int rc = by_slot(T, Hkv, D, K, V, slot_map, pool, n_pages, &a, &grid);
    if (rc != SPECROLL_OK || grid.x == 0) return rc;
    // (two threads would write one place: which value stays would be a matter of luck)
    const uintptr_t k = reinterpret_cast<uintptr_t>(K), v = reinterpret_cast<uintptr_t>(V), bytes = (uintptr_t)T * a.columns * 8;
    if (k < v + bytes && v < k + bytes) return SPECROLL_EINVAL;
    SR_CUDA_TRY(launch_dependent(true, D == 128 ? kv4_load_kernel<128> : kv4_load_kernel<64>, grid, dim3(KV4_THREADS), 0,
                                 static_cast<cudaStream_t>(cuda_stream), static_cast<const uint8_t *>(pool), a, static_cast<uint4 *>(K),
                                 static_cast<uint4 *>(V), status));
    return SPECROLL_OK;
}

extern "C" int specroll_commit_path_kv4_layers(int32_t B, int32_t N, int32_t K, int32_t Hkv, int32_t D, int32_t n_layers,
                                               const void *const *Kt, const void *const *Vt, const int32_t *path_node, const int32_t *n_acc,
                                               void *const *pool, int64_t n_pages, const int32_t *page_table, const int32_t *page_indptr,
                                               const int32_t *kv_len, int32_t *kv_len_out, int32_t *status, void *cuda_stream) {
    if (B < 0 || N < 1 || N > SPECROLL_MAX_NODES || K < 1 || K > SPECROLL_MAX_HEADS || Hkv < 1 || Hkv > 4096 || (D != 64 && D != 128) ||
        n_pages < 0 || n_pages > (1LL << 24) || n_layers < 1)
        return SPECROLL_EINVAL;
    if (B == 0) return SPECROLL_OK;  // (an empty batch has empty arrays: their pointers may be NULL)
    if (!Kt || !Vt || !path_node || !n_acc || !pool || !page_table || !page_indptr || !kv_len) return SPECROLL_EINVAL;
    for (int l = 0; l < n_layers; ++l) {
        if (!Kt[l] || !Vt[l] || !pool[l]) return SPECROLL_EINVAL;
        if (!aligned16(Kt[l]) || !aligned16(Vt[l]) || !aligned16(pool[l])) return SPECROLL_EALIGN;
    }
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int n_sm = 0;
    const int rc = device_setup(nullptr, 0, &n_sm);
    if (rc != SPECROLL_OK) return rc;
    const bool apart = kv_len_out && (kv_len_out >= kv_len + B || kv_len_out + B <= kv_len);
    for (int l0 = 0; l0 < n_layers; l0 += KV4_COMMIT_LAYERS) {
        const int nl = n_layers - l0 < KV4_COMMIT_LAYERS ? n_layers - l0 : KV4_COMMIT_LAYERS;
        Kv4Layers lay;
        for (int l = 0; l < nl; ++l) {
            lay.Kt[l] = static_cast<const uint4 *>(Kt[l0 + l]);
            lay.Vt[l] = static_cast<const uint4 *>(Vt[l0 + l]);
            lay.pool[l] = static_cast<uint8_t *>(pool[l0 + l]);
        }
        // layers to a block: as many as leave four blocks to every SM, up to 8 (256 sequences, 28 layers of two heads, with all rows read back, us: 27.4 with two
        // layers, 22.4 with four, 20.3 with eight, 21.1 with twelve, 28.5 with all)
        const int each = (int)std::min<long long>(std::max<long long>((long long)B * nl / (4LL * n_sm), 1), 8);
        SR_CUDA_TRY(launch_dependent(true, D == 128 ? kv4_commit_kernel<128> : kv4_commit_kernel<64>,
                                     dim3((unsigned)B, (unsigned)((nl + each - 1) / each)), dim3(KV4_THREADS), 0, st, lay, path_node, n_acc,
                                     (long long)n_pages, page_table, page_indptr, kv_len, N, K, Hkv, nl, each, status,
                                     apart && l0 == 0 ? kv_len_out : nullptr));
    }
    // in place: after the copies in stream order
    if (kv_len_out && !apart)
        SR_CUDA_TRY(launch_dependent(true, kv4_len_kernel, dim3((unsigned)(B + 255) / 256), dim3(256), 0, st, kv_len, n_acc, B, K, kv_len_out));
    return SPECROLL_OK;
}

extern "C" int specroll_commit_path_kv4(int32_t B, int32_t N, int32_t K, int32_t Hkv, int32_t D, const void *Kt, const void *Vt,
                                        const int32_t *path_node, const int32_t *n_acc, void *pool, int64_t n_pages,
                                        const int32_t *page_table, const int32_t *page_indptr, const int32_t *kv_len, int32_t *kv_len_out,
                                        int32_t *status, void *cuda_stream) {
    return specroll_commit_path_kv4_layers(B, N, K, Hkv, D, 1, &Kt, &Vt, path_node, n_acc, &pool, n_pages, page_table, page_indptr, kv_len,
                                           kv_len_out, status, cuda_stream);
}
