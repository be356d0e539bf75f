// Writing and reading the 4-bit paged cache: tokens by slot (prompts), the committed path of a round, and back to bf16.
//
// A block of 32 elements has one scale, the largest magnitude over 7 to four significant bits, and codes to the nearest
// multiple of it.  All three are bound by HBM: a token's head is 2 D bytes of bf16 against 17 D / 32 bytes of codes and scales.
// A thread has eight elements (16 bytes of bf16, one 32-bit word of codes), four threads a block, so that both sides are
// contiguous over a warp.  The arithmetic is kept to about four instructions an element, because the writer is otherwise
// bound by it: a multiple of the reciprocal is added to a constant whose last four bits then are the code.
#include "kv4.cuh"

namespace specroll {

// Codes of eight elements, and the block's scale byte, from the four threads that share the block.
__device__ __forceinline__ uint32_t kv4_encode(const uint4 &x, uint32_t &scale) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    // magnitudes as integers: 0x7f80 is infinity, above it NaN
    uint32_t m2 = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) m2 = __vmaxu2(m2, w[i] & 0x7fff7fffu);
    uint32_t top = max(m2 & 0xffffu, m2 >> 16);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
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
    const float t = __fdiv_rn(__uint_as_float(top << 16), 7.0f);
    int c = (int)((__float_as_uint(t) + (1u << 19)) >> 20) - (int)(KV4_EXP0 >> 4);
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
    // The reciprocal is taken a little too large, so that halves, which are exact quotients, go away from zero; every other
    // quotient of an 8-bit and a 4-bit significand is further than 2^-12 from a half.  1.5 2^23 + 8 leaves code = q + 8.
    const float inv = __fdiv_rn(1.0f + 0x1p-21f, s);
    uint32_t y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __float_as_uint(fmaf(v[i], inv, 12582920.0f));
    const uint32_t even = y[0] + (y[2] << 4) + (y[4] << 8) + (y[6] << 12), odd = y[1] + (y[3] << 4) + (y[5] << 8) + (y[7] << 12);
    scale = (uint32_t)c;
    return __byte_perm(even, odd, 0x5410);
}

// Codes and scale of eight elements to their places: word `at` of row `row` of a tile.
template <int D>
__device__ __forceinline__ void kv4_put(uint8_t *tile, int row, int at, uint32_t codes, uint32_t scale) {
    *reinterpret_cast<uint32_t *>(tile + row * Kv4<D>::ROW + at * 4) = codes;
    if ((at & 3) == 0) tile[Kv4<D>::CODES + row * Kv4<D>::SROW + (at >> 2)] = (uint8_t)scale;
}

constexpr int KV4_THREADS = 256;

// Thread i has word i mod D/8 of row i / (D/8); rows are (token, K or V, head), so that a warp reads contiguous memory.
template <int D>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_store_kernel(const uint4 *__restrict__ K, const uint4 *__restrict__ V, const long long *__restrict__ slots, long long n_words, int Hkv,
                 uint8_t *__restrict__ pool, long long n_slots, int32_t *__restrict__ status) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int W = D / 8;
    const long long i = (long long)blockIdx.x * KV4_THREADS + threadIdx.x;
    const bool in = i < n_words;  // (whole blocks of 32 elements at a time: n_words is a multiple of W)
    const int at = (int)(i % W), heads = Hkv * W;
    const long long line = i / heads;  // token and K or V
    const int head = (int)((i - line * heads) / W), v = (int)(line & 1);
    const long long tok = line >> 1;
    const long long slot = in ? __ldg(slots + tok) : -1;
    const bool ok = slot >= 0 && slot < n_slots;
    const uint4 x = ok ? __ldg((v ? V : K) + tok * heads + head * W + at) : make_uint4(0u, 0u, 0u, 0u);
    uint32_t scale;
    const uint32_t codes = kv4_encode(x, scale);
    if (ok) {
        uint8_t *tile = pool + ((slot / SPECROLL_PAGE_TOKENS * Hkv + head) * 2 + v) * (long long)Kv4<D>::TILE;
        kv4_put<D>(tile, (int)(slot % SPECROLL_PAGE_TOKENS), at, codes, scale);
    } else if (in && slot >= n_slots && status && at == 0 && head == 0) {
        atomicExch(status, SPECROLL_ELIMIT);
    }
}

template <int D>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_load_kernel(const uint8_t *__restrict__ pool, const long long *__restrict__ slots, long long n_words, int Hkv, long long n_slots,
                uint4 *__restrict__ K, uint4 *__restrict__ V, int32_t *__restrict__ status) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int W = D / 8;
    const long long i = (long long)blockIdx.x * KV4_THREADS + threadIdx.x;
    if (i >= n_words) return;
    const int at = (int)(i % W), heads = Hkv * W;
    const long long line = i / heads;
    const int head = (int)((i - line * heads) / W), v = (int)(line & 1);
    const long long tok = line >> 1, slot = __ldg(slots + tok);
    uint32_t r[4] = {0u, 0u, 0u, 0u};
    if (slot >= 0 && slot < n_slots) {
        const uint8_t *tile = pool + ((slot / SPECROLL_PAGE_TOKENS * Hkv + head) * 2 + v) * (long long)Kv4<D>::TILE;
        const int row = (int)(slot % SPECROLL_PAGE_TOKENS);
        const uint32_t w = __ldg(reinterpret_cast<const uint32_t *>(tile + row * Kv4<D>::ROW) + at);
        const uint32_t s = kv4_scale_bits(__ldg(tile + Kv4<D>::CODES + row * Kv4<D>::SROW + (at >> 2))) * 0x10001u;
        kv4_word(w, s, kv4_offset(s), r);
    } else if (slot >= n_slots && status && at == 0 && head == 0) {
        atomicExch(status, SPECROLL_ELIMIT);
    }
    (v ? V : K)[tok * heads + head * W + at] = make_uint4(r[0], r[1], r[2], r[3]);
}

constexpr int KV4_COMMIT_LAYERS = 64;  // layers one launch can serve (their pointers travel as kernel arguments)

struct Kv4Layers {
    const uint4 *Kt[KV4_COMMIT_LAYERS], *Vt[KV4_COMMIT_LAYERS];
    uint8_t *pool[KV4_COMMIT_LAYERS];
};

// grid = (B, K + 1, layers): block (b, i, l) writes tree row path_node[b, i] of layer l at cache position kv_len[b] + i, as
// commit_path_kernel does for a bf16 cache.
template <int D>
__global__ void __launch_bounds__(128)
kv4_commit_kernel(const __grid_constant__ Kv4Layers lay, const int32_t *__restrict__ path_node, const int32_t *__restrict__ n_acc,
                  long long n_pages, const int32_t *__restrict__ page_table, const int32_t *__restrict__ page_indptr,
                  const int32_t *__restrict__ kv_len, int N, int K, int Hkv, int32_t *__restrict__ status, int32_t *__restrict__ kv_len_out) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int W = D / 8;
    const int b = blockIdx.x, i = blockIdx.y;
    const int na = n_acc[b], len = kv_len[b];
    if (kv_len_out && i == 0 && blockIdx.z == 0 && threadIdx.x == 0) kv_len_out[b] = len + ((na < 0 || na > K) ? 0 : na + 1);
    if (i > na || na < 0 || na > K) return;
    const int node = path_node[(size_t)b * (K + 1) + i];
    const long long pos = (long long)len + i, slot = pos / SPECROLL_PAGE_TOKENS;
    const int first = page_indptr[b], own = page_indptr[b + 1] - first;
    int page = -1;
    if (node >= 0 && node < N && len >= 0 && slot < own) page = page_table[first + slot];
    if (page < 0 || page >= n_pages) {
        // no room (or a bad table): nothing is written for this token, and the caller is told
        if (threadIdx.x == 0 && status) atomicExch(status, SPECROLL_ELIMIT);
        return;
    }
    const int heads = Hkv * W, row = (int)(pos % SPECROLL_PAGE_TOKENS);
    const uint4 *const Kt = lay.Kt[blockIdx.z], *const Vt = lay.Vt[blockIdx.z];
    uint8_t *const tiles = lay.pool[blockIdx.z] + (size_t)page * Hkv * 2 * Kv4<D>::TILE;
    const size_t src = ((size_t)b * N + node) * heads;
    for (int w0 = 0; w0 < 2 * heads; w0 += 128) {  // (whole warps: the four threads of a block meet in the encoder)
        const int w = w0 + (int)threadIdx.x;
        const bool in = w < 2 * heads;
        const int v = w >= heads, word = v ? w - heads : w;
        const uint4 x = in ? __ldg((v ? Vt : Kt) + src + word) : make_uint4(0u, 0u, 0u, 0u);
        uint32_t scale;
        const uint32_t codes = kv4_encode(x, scale);
        if (in) kv4_put<D>(tiles + (size_t)(word / W * 2 + v) * Kv4<D>::TILE, row, word % W, codes, scale);
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

// What the two calls by slot share.  *n_words: 16-byte words of bf16 over both K and V.
static int by_slot_check(int64_t T, int32_t Hkv, int32_t D, const void *K, const void *V, const int64_t *slots, const void *pool,
                         int64_t n_pages, long long *n_words) {
    if (T < 0 || T > (1LL << 31) || Hkv < 1 || Hkv > 4096 || (D != 64 && D != 128) || n_pages < 0 || n_pages > (1LL << 24)) return SPECROLL_EINVAL;
    *n_words = 2LL * T * Hkv * (D / 8);
    if ((*n_words + KV4_THREADS - 1) / KV4_THREADS > 0x7fffffffLL) return SPECROLL_EINVAL;
    if (T == 0) return SPECROLL_OK;  // (no tokens have empty arrays: their pointers may be NULL)
    if (!K || !V || !slots || (n_pages > 0 && !pool)) return SPECROLL_EINVAL;
    if (!aligned16(K) || !aligned16(V) || !aligned16(pool)) return SPECROLL_EALIGN;
    return SPECROLL_OK;
}

extern "C" int specroll_kv4_store(int64_t T, int32_t Hkv, int32_t D, const void *K, const void *V, const int64_t *slot_map, void *pool,
                                  int64_t n_pages, int32_t *status, void *cuda_stream) {
    long long n = 0;
    const int rc = by_slot_check(T, Hkv, D, K, V, slot_map, pool, n_pages, &n);
    if (rc != SPECROLL_OK || T == 0) return rc;
    SR_CUDA_TRY(launch_dependent(true, D == 128 ? kv4_store_kernel<128> : kv4_store_kernel<64>, dim3((unsigned)((n + KV4_THREADS - 1) / KV4_THREADS)),
                                 dim3(KV4_THREADS), 0, static_cast<cudaStream_t>(cuda_stream), static_cast<const uint4 *>(K),
                                 static_cast<const uint4 *>(V), reinterpret_cast<const long long *>(slot_map), n, Hkv, static_cast<uint8_t *>(pool),
                                 (long long)n_pages * SPECROLL_PAGE_TOKENS, status));
    return SPECROLL_OK;
}

extern "C" int specroll_kv4_load(int64_t T, int32_t Hkv, int32_t D, const void *pool, int64_t n_pages, const int64_t *slot_map, void *K,
                                 void *V, int32_t *status, void *cuda_stream) {
    long long n = 0;
    const int rc = by_slot_check(T, Hkv, D, K, V, slot_map, pool, n_pages, &n);
    if (rc != SPECROLL_OK || T == 0) return rc;
    SR_CUDA_TRY(launch_dependent(true, D == 128 ? kv4_load_kernel<128> : kv4_load_kernel<64>, dim3((unsigned)((n + KV4_THREADS - 1) / KV4_THREADS)),
                                 dim3(KV4_THREADS), 0, static_cast<cudaStream_t>(cuda_stream), static_cast<const uint8_t *>(pool),
                                 reinterpret_cast<const long long *>(slot_map), n, Hkv, (long long)n_pages * SPECROLL_PAGE_TOKENS,
                                 static_cast<uint4 *>(K), static_cast<uint4 *>(V), status));
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
    const bool apart = kv_len_out && (kv_len_out >= kv_len + B || kv_len_out + B <= kv_len);
    for (int l0 = 0; l0 < n_layers; l0 += KV4_COMMIT_LAYERS) {
        const int nl = n_layers - l0 < KV4_COMMIT_LAYERS ? n_layers - l0 : KV4_COMMIT_LAYERS;
        Kv4Layers lay;
        for (int l = 0; l < nl; ++l) {
            lay.Kt[l] = static_cast<const uint4 *>(Kt[l0 + l]);
            lay.Vt[l] = static_cast<const uint4 *>(Vt[l0 + l]);
            lay.pool[l] = static_cast<uint8_t *>(pool[l0 + l]);
        }
        SR_CUDA_TRY(launch_dependent(true, D == 128 ? kv4_commit_kernel<128> : kv4_commit_kernel<64>,
                                     dim3((unsigned)B, (unsigned)(K + 1), (unsigned)nl), dim3(128), 0, st, lay, path_node, n_acc,
                                     (long long)n_pages, page_table, page_indptr, kv_len, N, K, Hkv, status,
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
