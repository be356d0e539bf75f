// Tree attention over the 4-bit paged cache, for few query rows per KV head: single tokens and small trees.
//
// A CTA takes one chunk of a sequence's pages for one KV head and all its query rows, at most 8 R8 (nodes x query heads of the KV head).
// Its four warps go through slices of 32 tokens, each for itself: a warp's first thread fetches its slices (K and V codes and scales)
// with untiled bulk copies into three stages of its own, so that no warp waits for another before the end.  Codes are decoded
// straight into mma.sync fragments: a cached element passes through shared memory once, as four bits, and is decoded once for all rows:
//   S^T (16 tokens x 8 rows)  = K (A operand, from codes) x Q^T (B operand, in registers for the whole unit)
//   O^T (D x 8 rows)         += V^T (A operand, from codes) x P^T (B operand: P transposed by movmatrix)
// What an index of a fragment stands for is free as long as both operands agree, and is chosen so that a thread's codes are
// contiguous: for K a thread has 1/4 of a token's elements (one scale block where D = 128), for V 1/8 of four tokens' elements,
// paired by byte permutes before decoding.  Tokens of a pair change places in every other pair, which halves the bank conflicts
// of V's reads.
// Every warp has a softmax of its own (reference maximum per row, which stays until a score is 2^8 above it); the four meet in
// shared memory at the end.  The tree's bf16 rows (sixteen nodes at most) are done by the first warp before its slices.
// What bounds it: long sequences take an SM 0.50 us a page and head (17 KB, 0.39 at HBM's rate: 79 %; without decoding 0.42).  Decoding
// is some 80 integer and 64 packed floating operations a thread for 16 tokens, which the tensor operations and the rest do not quite hide;
// more warps on an SM (five CTAs at 96 registers; there are 128, with 28 bytes of spill where D = 128) changed nothing, nor did whole pages by one copy each into stages that the four
// warps share.  A unit takes 12 us beyond its pages: lengths, page table, pages, then the warps' meeting, each a round trip, of which
// the other three CTAs of the SM hide a part.
#include <math.h>

#include "kv4.cuh"
#include "tc05.cuh"
#include "tree_attn.cuh"

namespace specroll {

namespace akv4 {
constexpr int WARPS = 4, THREADS = 32 * WARPS;
constexpr int SLICE = 32;  // tokens a warp fetches and takes at a time
constexpr int STAGES = 3;

template <int D, int R8>
struct Cfg {
    // a slice: K codes, K scales, V codes, V scales
    static constexpr int CODES = SLICE * Kv4<D>::ROW, SCALES = SLICE * Kv4<D>::SROW, HALF = CODES + SCALES, BYTES = 2 * HALF;
    static constexpr int RING = WARPS * STAGES * BYTES;
    static constexpr int RUN = D / 4, STEPS = D / 16;  // a thread's elements of a K row; contraction steps of S
    static constexpr int VRUN = D / 8, MB = D / 16;    // a thread's elements of a V row; row blocks of O^T
    static constexpr int ROWS = 8 * R8;
    // at the end: per warp the rows' references and sums, and O
    static constexpr int O_FLOATS = D * ROWS;
    static constexpr int JOIN = WARPS * (O_FLOATS + 2 * ROWS) * 4;
    static constexpr int BODY = (RING > JOIN ? RING : JOIN);
    static constexpr int FOUND = BODY + 8 * WARPS * STAGES + 16;  // the unit's search
    static constexpr int SMEM = FOUND + 4 * (8 + WARPS);
    static constexpr int CTAS = R8 == 1 ? KV4_CTAS_8 : KV4_CTAS_16;
    static_assert(SCALES % 16 == 0 && CTAS * (SMEM + 1024) <= 233472, "bulk copies; shared memory of an SM");
};

__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
}  // namespace akv4

template <int D, int R8>
__global__ void __launch_bounds__(akv4::THREADS, (akv4::Cfg<D, R8>::CTAS))
tree_attn_kv4_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ TopoMask mask, int32_t *__restrict__ status) {
    using namespace akv4;
    using C = Cfg<D, R8>;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, c = lane & 3;
    unsigned char *const mine = smem + warp * STAGES * C::BYTES;  // this warp's stages
    const uint32_t bars = smem_u32(smem) + C::BODY + 8 * STAGES * warp;
    volatile int *const abort_flag = reinterpret_cast<volatile int *>(smem + C::BODY + 8 * WARPS * STAGES);
    if (lane == 0)
        for (int s = 0; s < STAGES; ++s) mbar_init(bars + 8 * s, 1);
    if (threadIdx.x == 0) *abort_flag = 0;
    if (lane == 0) fence_mbar_init();
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();

    // ---- the unit: (chunk, KV head).  Chunks are counted in the order of the sequences; every CTA finds its own from the
    // lengths (a plan made by a kernel in front took ten microseconds for 256 sequences).
    if (blockIdx.x == 0 && threadIdx.x == 0) *status = 0;  // (seconds ahead of any wait that could run out)
    const int hkv = (int)blockIdx.x % a.Hkv, item = (int)blockIdx.x / a.Hkv;
    int b = item, split = 0, n_splits = 1, L, slot0;
    if (a.items == a.B) {  // (nothing is cut)
        L = max(__ldg(a.kv_len + b), 0);
        slot0 = __ldg(a.page_indptr + b);
    } else {
        // [0..4]: the unit, [8 ..]: chunks of the warps' sequences.  (Not in the ring: copies go there next, which would take a fence
        // and a barrier.)
        volatile int *const found = reinterpret_cast<volatile int *>(smem + C::FOUND);
        const int per = (a.B + THREADS - 1) / THREADS, b0 = min(a.B, (int)threadIdx.x * per), b1 = min(a.B, b0 + per);
        auto chunks = [&](int len) {  // (the rounding without a sign: the longest lengths pass 31 bits by it)
            return max(1, ((int)(((unsigned)len + (SPECROLL_PAGE_TOKENS - 1)) / SPECROLL_PAGE_TOKENS) + a.chunk_tiles - 1) / a.chunk_tiles);
        };
        // (lengths four at a time, so that their loads are under way together; the first four sequences' pages as well)
        int own = 0, pages[4];
        for (int i = b0; i < b1; i += 4) {
            int len[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) len[q] = i + q < b1 ? __ldg(a.kv_len + i + q) : 0;
            if (i == b0) {
#pragma unroll
                for (int q = 0; q < 4; ++q) pages[q] = i + q < b1 ? __ldg(a.page_indptr + i + q) : 0;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) own += i + q < b1 ? chunks(max(len[q], 0)) : 0;
            own = min(own, a.items + 1);  // (what is beyond the host's chunks is too much, however far; those are some thousands at most)
        }
        int sum = own;
#pragma unroll
        for (int o_ = 1; o_ < 32; o_ <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, sum, o_);
            if (lane >= o_) sum += x;
        }
        if (lane == 31) found[8 + warp] = sum;
        if (threadIdx.x == 0) found[0] = -1;
        __syncthreads();
        int at = sum - own, total = 0;
#pragma unroll
        for (int q = 0; q < WARPS; ++q) {
            at += q < warp ? found[8 + q] : 0;
            total += found[8 + q];
        }
        if (total > a.items) {  // lengths that make more chunks than the host's, which have no CTA and no place: nothing is written
            if (blockIdx.x == 0) {
                for (int i = b0; i < b1; ++i) a.item_start[i] = a.items;  // (the merge sees by it that its sequence has no chunks)
                if (threadIdx.x == 0) atomicExch(status, SPECROLL_ELIMIT);
            }
            return;
        }
        if (item >= at && item < at + own) {
            for (int i = b0; i < b1; ++i) {
                const int len = max(__ldg(a.kv_len + i), 0), ns = chunks(len);
                if (item < at + ns) {
                    found[0] = i;
                    found[1] = item - at;
                    found[2] = ns;
                    found[3] = len;
                    found[4] = i - b0 == 0 ? pages[0] : i - b0 == 1 ? pages[1] : i - b0 == 2 ? pages[2] : i - b0 == 3 ? pages[3] : __ldg(a.page_indptr + i);
                    if (item == at && hkv == 0) a.item_start[i] = at;  // (for the merge)
                    break;
                }
                at += ns;
            }
        }
        __syncthreads();
        b = found[0];
        split = found[1];
        n_splits = found[2];
        L = found[3];
        slot0 = found[4];
        if (b < 0) return;  // (lengths that make fewer chunks than the host's)
    }
    const int tiles_b = (L + SPECROLL_PAGE_TOKENS - 1) / SPECROLL_PAGE_TOKENS;
    const int tps = (tiles_b + n_splits - 1) / n_splits;
    const int t_lo = min(tiles_b, split * tps), n_t = min(tiles_b, t_lo + tps) - t_lo;
    const bool has_tree = split == n_splits - 1;
    const int N = a.N, G = a.G;
    // this warp's slices: slice i is the 32 tokens of the sequence from first + STRIDE i on, a quarter of a page
    constexpr int STRIDE = WARPS * SLICE;
    const int first = t_lo * SPECROLL_PAGE_TOKENS + warp * SLICE, end = min(L, (t_lo + n_t) * SPECROLL_PAGE_TOKENS);
    const int n_i = end > first ? (end - first + STRIDE - 1) / STRIDE : 0;
    auto page_at = [&](int i) { return (warp * SLICE + STRIDE * i) / SPECROLL_PAGE_TOKENS; };

    float o[R8][C::MB][4];
    float m[R8][2], ref[R8][2], l[R8][2];  // reference maxima (ref: the same, but 0 where there is none yet) and sums
#pragma unroll
    for (int r = 0; r < R8; ++r) {
        m[r][0] = m[r][1] = -INFINITY;
        l[r][0] = l[r][1] = ref[r][0] = ref[r][1] = 0.f;
#pragma unroll
        for (int i = 0; i < C::MB; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[r][i][e] = 0.f;
    }

    // ---- loads: slice i into stage i mod STAGES, by the warp's first thread.  A page that does not exist is not fetched: the warp writes
    // codes that stand for zero (whatever the scale) in its place.
    const int32_t *const pt = a.page_table + slot0 + t_lo;
    auto load = [&](int i, int page) {
        const int s = i % STAGES;
        const uint32_t bar = bars + 8 * s;
        if (page >= 0 && page < a.n_pages) {
            if (lane == 0) {
                const uint32_t dst = smem_u32(mine) + s * C::BYTES;
                const int part = (warp + WARPS * i) % (SPECROLL_PAGE_TOKENS / SLICE);
                const uint8_t *k = a.pool + ((size_t)page * a.Hkv + hkv) * (2 * Kv4<D>::TILE) + part * C::CODES;
                const uint8_t *ks = k + Kv4<D>::CODES - part * (C::CODES - C::SCALES);
                mbar_arrive_expect_tx(bar, C::BYTES);
                bulk_load(dst, k, C::CODES, bar);
                bulk_load(dst + C::CODES, ks, C::SCALES, bar);
                bulk_load(dst + C::HALF, k + Kv4<D>::TILE, C::CODES, bar);
                bulk_load(dst + C::HALF + C::CODES, ks + Kv4<D>::TILE, C::SCALES, bar);
            }
        } else {
            for (int j = lane; j < C::BYTES / 4; j += 32) reinterpret_cast<uint32_t *>(mine + s * C::BYTES)[j] = 0x88888888u;
            fence_proxy_async();  // (a later slice's copies go over them)
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        }
    };
    int page[STAGES + 1];
#pragma unroll
    for (int i = 0; i <= STAGES; ++i) page[i] = i < n_i ? __ldg(pt + page_at(i)) : -1;

    {
        // ------------------------------------------------------------------ attention
        // Q: rows g of every block of eight, the elements of this thread's run
        uint32_t qf[R8][2 * C::STEPS];
#pragma unroll
        for (int r = 0; r < R8; ++r) {
            const int gr = 8 * r + g;
            const bool ok = gr < a.rows;
            const int n = ok ? gr / G : 0, gq = ok ? gr % G : 0;
            const uint4 *src = reinterpret_cast<const uint4 *>(a.Q + (((size_t)b * N + n) * a.Hq + hkv * G + gq) * D + C::RUN * c);
#pragma unroll
            for (int i = 0; i < C::STEPS / 2; ++i) {
                const uint4 x = ok ? __ldg(src + i) : make_uint4(0u, 0u, 0u, 0u);
                qf[r][4 * i] = x.x;
                qf[r][4 * i + 1] = x.y;
                qf[r][4 * i + 2] = x.z;
                qf[r][4 * i + 3] = x.w;
            }
        }
        // the tree's rows, bf16: K rows and V rows as the codes of the cache are divided among the threads
        const bool tree = has_tree && warp == 0;  // (rows of one KV head: sixteen nodes at most)
        uint4 kx[2][C::RUN / 8], vx[4][C::VRUN / 8];
        // the tokens (of 16) that a thread's indexes stand for: index 2 j + e is token 2 j + (e ^ (j & 1))
        const int k_tok = g ^ ((g >> 1) & 1);               // K rows g and g + 8: tokens k_tok and k_tok + 8
        const int v_a = 2 * c + (c & 1), v_b = v_a ^ 1;     // V pairs: tokens (v_a, v_b) and those + 8
        const float sc = a.scale_log2 * KV4_UP;  // (K decodes to 2^-KV4_DOWN of itself; V too, and the tree's probabilities follow it)
        if (tree) {
            const size_t rows_of_b = (size_t)b * N;
            const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = k_tok + 8 * h;
                const uint4 *src = reinterpret_cast<const uint4 *>(a.Kt + ((rows_of_b + n) * a.Hkv + hkv) * D + C::RUN * c);
#pragma unroll
                for (int i = 0; i < C::RUN / 8; ++i) kx[h][i] = n < N ? __ldg(src + i) : zero;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = ((q & 1) ? v_b : v_a) + 8 * (q >> 1);
                const uint4 *src = reinterpret_cast<const uint4 *>(a.Vt + ((rows_of_b + n) * a.Hkv + hkv) * D + C::VRUN * g);
#pragma unroll
                for (int i = 0; i < C::VRUN / 8; ++i) vx[q][i] = n < N ? __ldg(src + i) : zero;
            }
        }
        // (the page numbers are there by now; the first pages arrive while the tree is worked on)
#pragma unroll
        for (int i = 0; i < STAGES; ++i)
            if (i < n_i) load(i, page[i]);
        int next_page = page[STAGES];

        // Scores (products) of GP groups of 16 tokens to probabilities, in fragments for the product with V.  admits(p, r, e): whether the
        // token of score e (k_tok of group p, + 8 from e = 2 on) counts for row 2 c + (e & 1) of block r; `whole`: they all do.
        // The exponentials are taken against the references as they stand, and a row's sum is the alarm for one that has to move: a
        // score 2^8 above it makes the sum exceed 2^8.  sc: the scores' factor; down: that of the fragments.
        auto softmax = [&](auto &s, float sc, float down, bool start, bool whole, auto admits, auto &pf) {
            constexpr int GP = sizeof(s) / sizeof(s[0]);
            float q[GP][R8][4], sum[R8][2];
            auto exps = [&]() {
#pragma unroll
                for (int p = 0; p < GP; ++p)
#pragma unroll
                    for (int r = 0; r < R8; ++r)
#pragma unroll
                        for (int e = 0; e < 4; ++e) q[p][r][e] = ex2_approx(fmaf(s[p][r][e], sc, -ref[r][e & 1]));
                if (!whole) {
#pragma unroll
                    for (int p = 0; p < GP; ++p)
#pragma unroll
                        for (int r = 0; r < R8; ++r)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (!admits(p, r, e)) q[p][r][e] = 0.f;
                }
#pragma unroll
                for (int r = 0; r < R8; ++r)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        sum[r][e] = q[0][r][e] + q[0][r][e + 2];
#pragma unroll
                        for (int p = 1; p < GP; ++p) sum[r][e] += q[p][r][e] + q[p][r][e + 2];
                    }
            };
            bool move = start;
            if (!start) {
                exps();
#pragma unroll
                for (int r = 0; r < R8; ++r) move |= !(fmaxf(sum[r][0], sum[r][1]) <= 256.0f) || !(sum[r][0] + sum[r][1] <= 512.0f);
            }
            if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                for (int r = 0; r < R8; ++r)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = -INFINITY;
#pragma unroll
                        for (int p = 0; p < GP; ++p)
#pragma unroll
                            for (int h = 0; h < 4; h += 2)
                                if (admits(p, r, e + h)) mx = fmaxf(mx, s[p][r][e + h] * sc);
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                        if (mx > m[r][e]) {  // (also where there was none)
                            const float f = ex2_approx(m[r][e] - mx);
                            m[r][e] = ref[r][e] = mx;
                            l[r][e] *= f;
#pragma unroll
                            for (int i = 0; i < C::MB; ++i) {
                                o[r][i][e] *= f;
                                o[r][i][e + 2] *= f;
                            }
                        }
                    }
                exps();
            }
#pragma unroll
            for (int r = 0; r < R8; ++r) {
                l[r][0] += sum[r][0];
                l[r][1] += sum[r][1];
#pragma unroll
                for (int p = 0; p < GP; ++p) {
                    // (bf16, the type of V in the product: half a step is 2^-8 of each, outputs are 2.3e-3 from 64 bits, of which their own
                    // rounding is 1.7e-3; the sums above are of the probabilities in fp32)
                    pf[p][r][0] = movmatrix(pack_bf16x2(q[p][r][0] * down, q[p][r][1] * down));
                    pf[p][r][1] = movmatrix(pack_bf16x2(q[p][r][2] * down, q[p][r][3] * down));
                }
            }
        };

        if (tree) {
            float s[1][R8][4];
#pragma unroll
            for (int r = 0; r < R8; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[0][r][e] = 0.f;
#pragma unroll
            for (int i = 0; i < C::RUN / 8; ++i) {
                const uint32_t lo[4] = {kx[0][i].x, kx[0][i].y, kx[0][i].z, kx[0][i].w};
                const uint32_t hi[4] = {kx[1][i].x, kx[1][i].y, kx[1][i].z, kx[1][i].w};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t af[4] = {lo[2 * h], hi[2 * h], lo[2 * h + 1], hi[2 * h + 1]};
#pragma unroll
                    for (int r = 0; r < R8; ++r) mma_bf16_16816(s[0][r], af, qf[r][4 * i + 2 * h], qf[r][4 * i + 2 * h + 1]);
                }
            }
            uint32_t pf[1][R8][2];
            softmax(s, a.scale_log2, 1.0f / KV4_UP, true, false, [&](int, int r, int e) {
                const int gr = 8 * r + 2 * c + (e & 1);
                return gr < a.rows && ((mask.anc[gr / G] >> (k_tok + (e & 2 ? 8 : 0))) & 1ull);
            }, pf);
#pragma unroll
            for (int i = 0; i < C::VRUN / 8; ++i) {
                const uint32_t x[4][4] = {{vx[0][i].x, vx[0][i].y, vx[0][i].z, vx[0][i].w}, {vx[1][i].x, vx[1][i].y, vx[1][i].z, vx[1][i].w},
                                          {vx[2][i].x, vx[2][i].y, vx[2][i].z, vx[2][i].w}, {vx[3][i].x, vx[3][i].y, vx[3][i].z, vx[3][i].w}};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t af[4] = {__byte_perm(x[0][j], x[1][j], 0x5410), __byte_perm(x[0][j], x[1][j], 0x7632),
                                            __byte_perm(x[2][j], x[3][j], 0x5410), __byte_perm(x[2][j], x[3][j], 0x7632)};
#pragma unroll
                    for (int r = 0; r < R8; ++r) mma_bf16_16816(o[r][4 * i + j], af, pf[0][r][0], pf[0][r][1]);
                }
            }
        }

        bool ok = true;
        for (int i = 0; i < n_i; ++i) {
            const int st = i % STAGES;
            ok = mbar_wait(bars + 8 * st, (i / STAGES) & 1u, abort_flag);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const unsigned char *tile = mine + st * C::BYTES;
            // ---- S^T = K Q^T
            float s[2][R8][4];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
#pragma unroll
                for (int r = 0; r < R8; ++r)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[p][r][e] = 0.f;
                const int t0 = 16 * p + k_tok;
                uint32_t kw[2][C::RUN / 8];
                Kv4Scale sk[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const unsigned char *row = tile + (t0 + 8 * h) * Kv4<D>::ROW + (C::RUN / 2) * c;
                    if constexpr (D == 128) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(row);
                        kw[h][0] = x.x, kw[h][1] = x.y, kw[h][2] = x.z, kw[h][3] = x.w;
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2 *>(row);
                        kw[h][0] = x.x, kw[h][1] = x.y;
                    }
                    const uint32_t sb = tile[C::CODES + (t0 + 8 * h) * Kv4<D>::SROW + (D == 128 ? c : c >> 1)];
                    sk[h] = kv4_scale_of(sb);
                }
#pragma unroll
                for (int j = 0; j < C::RUN / 8; ++j) {
                    uint32_t lo[4], hi[4];
                    kv4_word(kw[0][j], sk[0], lo);
                    kv4_word(kw[1][j], sk[1], hi);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t af[4] = {lo[2 * h], hi[2 * h], lo[2 * h + 1], hi[2 * h + 1]};
#pragma unroll
                        for (int r = 0; r < R8; ++r) mma_bf16_16816(s[p][r], af, qf[r][4 * j + 2 * h], qf[r][4 * j + 2 * h + 1]);
                    }
                }
            }
            // ---- softmax
            uint32_t pf[2][R8][2];
            const int left = L - (first + i * STRIDE) - k_tok;  // > 0: token k_tok is in the sequence
            softmax(s, sc, 1.0f, i == 0, left + k_tok >= SLICE, [&](int p, int, int e) { return left > 16 * p + (e & 2 ? 8 : 0); }, pf);
            // ---- O^T += V^T P^T
            const unsigned char *vt = tile + C::HALF;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                uint32_t vw[4][C::VRUN / 8], sb[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int tok = 16 * p + ((q & 1) ? v_b : v_a) + 8 * (q >> 1);
                    const unsigned char *row = vt + tok * Kv4<D>::ROW + (C::VRUN / 2) * g;
                    if constexpr (D == 128) {
                        const uint2 x = *reinterpret_cast<const uint2 *>(row);
                        vw[q][0] = x.x, vw[q][1] = x.y;
                    } else {
                        vw[q][0] = *reinterpret_cast<const uint32_t *>(row);
                    }
                    sb[q] = vt[C::CODES + tok * Kv4<D>::SROW + (g * C::VRUN) / 32];
                }
                const Kv4Scale s0 = kv4_scale_of(sb[0], sb[1]), s1 = kv4_scale_of(sb[2], sb[3]);
#pragma unroll
                for (int j = 0; j < C::VRUN / 8; ++j) {
                    // lower halves: elements 0 2 4 6 of the word, upper halves: 1 3 5 7, of two tokens each
                    uint32_t e0_[4], e1_[4], d0_[4], d1_[4];
                    kv4_word(__byte_perm(vw[0][j], vw[1][j], 0x5410), s0, e0_);
                    kv4_word(__byte_perm(vw[0][j], vw[1][j], 0x7632), s0, d0_);
                    kv4_word(__byte_perm(vw[2][j], vw[3][j], 0x5410), s1, e1_);
                    kv4_word(__byte_perm(vw[2][j], vw[3][j], 0x7632), s1, d1_);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t af[4] = {e0_[q], d0_[q], e1_[q], d1_[q]};
#pragma unroll
                        for (int r = 0; r < R8; ++r) mma_bf16_16816(o[r][4 * j + q], af, pf[p][r][0], pf[p][r][1]);
                    }
                }
            }
            __syncwarp();
            if (i + STAGES < n_i) {
                load(i + STAGES, next_page);
                next_page = i + STAGES + 1 < n_i ? __ldg(pt + page_at(i + STAGES + 1)) : 0;
            }
        }
#pragma unroll
        for (int r = 0; r < R8; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                l[r][e] += __shfl_xor_sync(0xffffffffu, l[r][e], 4);
                l[r][e] += __shfl_xor_sync(0xffffffffu, l[r][e], 8);
                l[r][e] += __shfl_xor_sync(0xffffffffu, l[r][e], 16);
            }
    }

    // ------------------------------------------------------------------ the warps' shares together, in the ring's place
    __syncthreads();  // (every copy has been waited for, unless the CTA is aborting)
    if (*abort_flag) {
        if (threadIdx.x == 0) {
            atomicExch(status, SPECROLL_ETIMEOUT);
            // copies in flight get time to land before the CTA goes away
            const unsigned long long t0 = globaltimer_ns();
            while (globaltimer_ns() - t0 < 20000000ull) {
            }
        }
        return;
    }
    float *const jo = reinterpret_cast<float *>(smem);                   // [warp][row][D]
    float *const jm = jo + WARPS * C::O_FLOATS, *const jl = jm + WARPS * C::ROWS;  // [warp][row]
    {
#pragma unroll
        for (int r = 0; r < R8; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = 8 * r + 2 * c + e;
                if (g == 0) {
                    jm[warp * C::ROWS + row] = m[r][e];
                    jl[warp * C::ROWS + row] = l[r][e];
                }
                // O^T block 4 i + j: index g is element 8 i + 2 j of this thread's run, g + 8 the one after it
                float *dst = jo + ((size_t)warp * C::ROWS + row) * D + C::VRUN * g;
#pragma unroll
                for (int i = 0; i < C::MB; ++i)
                    *reinterpret_cast<float2 *>(dst + 2 * i) = make_float2(o[r][i][e], o[r][i][e + 2]);
            }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < C::ROWS * (D / 4); i += THREADS) {
        const int row = i % C::ROWS, d4 = i / C::ROWS;
        if (row >= a.rows) continue;
        float M = -INFINITY;
#pragma unroll
        for (int q = 0; q < WARPS; ++q) M = fmaxf(M, jm[q * C::ROWS + row]);
        float sum = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int q = 0; q < WARPS; ++q) {
            const float mq = jm[q * C::ROWS + row], f = mq == -INFINITY ? 0.f : ex2_approx(mq - M);
            const float4 x = *reinterpret_cast<const float4 *>(jo + ((size_t)q * C::ROWS + row) * D + 4 * d4);
            sum += f * jl[q * C::ROWS + row];
            acc.x += f * x.x;
            acc.y += f * x.y;
            acc.z += f * x.z;
            acc.w += f * x.w;
        }
        acc = make_float4(acc.x * KV4_UP, acc.y * KV4_UP, acc.z * KV4_UP, acc.w * KV4_UP);
        const int n = row / G, gq = row % G;
        if (n_splits == 1) {
            const float inv = sum > 0.f ? 1.0f / sum : 0.f;
            const size_t at = ((size_t)b * N + n) * a.Hq + hkv * G + gq;
            *reinterpret_cast<uint2 *>(a.O + at * D + 4 * d4) =
                make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
            if (a.lse && d4 == 0) a.lse[at] = (M + log2f(sum)) * 0.6931471805599453f;
        } else {
            const size_t unit = (size_t)item * a.Hkv + hkv;
            reinterpret_cast<float4 *>(a.part_o)[(unit * (D / 4) + d4) * a.rows_pad + row] = acc;
            if (d4 == 0) reinterpret_cast<float2 *>(a.part_ml)[unit * a.rows_pad + row] = make_float2(M, sum);
        }
    }
}

template <int D, int R8>
static int launch_kv4(const AttnArgs &a, const TopoMask &mask, int32_t *status, cudaStream_t st) {
    using C = akv4::Cfg<D, R8>;
    const auto kern = tree_attn_kv4_kernel<D, R8>;
    const int rc = device_setup(reinterpret_cast<const void *>(kern), C::SMEM, nullptr);
    if (rc != SPECROLL_OK) return rc;
    SR_CUDA_TRY(launch_dependent(!a.no_pdl, kern, dim3((unsigned)a.total_work), dim3(akv4::THREADS), C::SMEM, st, a, mask, status));
    return SPECROLL_OK;
}

// Sums the chunks of every split sequence.  grid = (B, Hkv, Z): a block has a Z-th of D of all rows of one (sequence, KV head), four floats
// a thread, and as many parts of the chunks as 256 threads have room for; a part's chunks are taken eight at a time with all their loads
// in flight.  Z = 4 where some sequence has more than 8 chunks, else the fewest blocks (attention and merge, us: 8 sequences of 20000
// tokens, 32 chunks, 31.3 with Z = 4 and 35.2 with 1; 256 of 1500, 8 chunks at most, 52.2 and 47.8).  Launched as a programmatic dependent
// of the attention kernel, which lets it start only behind its own wait: the lengths can be read ahead of the wait for the partials.
template <int D, int ROWS, int Z>
__global__ void __launch_bounds__(256) attn_merge_kv4_kernel(AttnArgs a) {
    constexpr int COLS = D / 4 / Z, ITEMS = ROWS * COLS, PARTS = 256 / ITEMS, STEP = 8;
    static_assert(PARTS >= 1 && PARTS * ITEMS == 256, "whole blocks");
    __shared__ float2 sh_ml[256];
    __shared__ float4 sh_acc[256];
    pdl_launch_dependents();
    const int b = blockIdx.x, hkv = blockIdx.y, part = threadIdx.x / ITEMS, row = threadIdx.x % ROWS, d4 = blockIdx.z * COLS + threadIdx.x % ITEMS / ROWS;
    const int len = max(__ldg(a.kv_len + b), 0);
    const int n_splits = ((len + SPECROLL_PAGE_TOKENS - 1) / SPECROLL_PAGE_TOKENS + a.chunk_tiles - 1) / a.chunk_tiles;
    // (blocks with nothing to do leave their places to those that have, but for one: where no block waited, the kernel after this one would
    // not wait for the attention kernel)
    if (n_splits < 2 && (blockIdx.x | blockIdx.y | blockIdx.z) != 0) return;
    pdl_wait();
    if (n_splits < 2) return;
    const int item0 = __ldcg(a.item_start + b);
    if (item0 + n_splits > a.items) return;  // (lengths that make more chunks than the host's: the attention kernel has said so)
    const size_t unit = (size_t)item0 * a.Hkv + hkv;
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + unit * a.rows_pad + row;
    const float4 *po = reinterpret_cast<const float4 *>(a.part_o) + (unit * (D / 4) + d4) * a.rows_pad + row;
    const size_t step_ml = (size_t)a.Hkv * a.rows_pad, step_o = step_ml * (D / 4);
    float M = -INFINITY, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int i0 = part; i0 < n_splits; i0 += STEP * PARTS) {
        float2 v[STEP];
        float4 x[STEP];
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
            const size_t s = (size_t)min(i0 + i * PARTS, n_splits - 1);  // (a chunk beyond the last: weight zero below)
            v[i] = __ldcg(ml + s * step_ml);
            x[i] = __ldcg(po + s * step_o);
        }
        float top = M;
#pragma unroll
        for (int i = 0; i < STEP; ++i) top = fmaxf(top, v[i].x);
        const float f = M == -INFINITY ? 0.f : ex2_approx(M - top);
        M = top;
        sum *= f;
        acc = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
            const float w = (i0 + i * PARTS >= n_splits || v[i].x == -INFINITY) ? 0.f : ex2_approx(v[i].x - M);
            sum += w * v[i].y;
            acc.x += w * x[i].x;
            acc.y += w * x[i].y;
            acc.z += w * x[i].z;
            acc.w += w * x[i].w;
        }
    }
    sh_ml[threadIdx.x] = make_float2(M, sum);
    sh_acc[threadIdx.x] = acc;
    __syncthreads();
    if (part == 0 && row < a.rows) {
#pragma unroll
        for (int q = 1; q < PARTS; ++q) M = fmaxf(M, sh_ml[q * ITEMS + threadIdx.x].x);
        sum = 0.f;
        acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
            const float2 e = sh_ml[q * ITEMS + threadIdx.x];
            const float4 y = sh_acc[q * ITEMS + threadIdx.x];
            const float w = e.x == -INFINITY ? 0.f : ex2_approx(e.x - M);
            sum += w * e.y;
            acc.x += w * y.x;
            acc.y += w * y.y;
            acc.z += w * y.z;
            acc.w += w * y.w;
        }
        const float inv = sum > 0.f ? 1.0f / sum : 0.f;
        const size_t at = ((size_t)b * a.N + row / a.G) * a.Hq + hkv * a.G + row % a.G;
        *reinterpret_cast<uint2 *>(a.O + at * D + 4 * d4) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
        if (a.lse && d4 == 0) a.lse[at] = (M + log2f(sum)) * 0.6931471805599453f;
    }
}

template <int D, int ROWS, int Z>
static int launch_merge(const AttnArgs &a, cudaStream_t st) {
    SR_CUDA_TRY(launch_dependent(!a.no_pdl, attn_merge_kv4_kernel<D, ROWS, Z>, dim3((unsigned)a.B, (unsigned)a.Hkv, Z), dim3(256), 0, st, a));
    return SPECROLL_OK;
}

int launch_attn_merge_kv4(const AttnArgs &a, int D, int max_splits, cudaStream_t st) {
    const bool one = a.rows_per_block == 8, few = max_splits <= 8;
    if (D == 128 && one) return few ? launch_merge<128, 8, 1>(a, st) : launch_merge<128, 8, 4>(a, st);
    if (D == 128) return few ? launch_merge<128, 16, 2>(a, st) : launch_merge<128, 16, 4>(a, st);
    if (one) return few ? launch_merge<64, 8, 1>(a, st) : launch_merge<64, 8, 4>(a, st);
    return few ? launch_merge<64, 16, 1>(a, st) : launch_merge<64, 16, 4>(a, st);
}

int launch_attn_kv4(const AttnArgs &a, const TopoMask &mask, int D, int32_t *status, cudaStream_t st) {
    const bool one = a.rows_per_block == 8;
    if (D == 128) return one ? launch_kv4<128, 1>(a, mask, status, st) : launch_kv4<128, 2>(a, mask, status, st);
    return one ? launch_kv4<64, 1>(a, mask, status, st) : launch_kv4<64, 2>(a, mask, status, st);
}

}  // namespace specroll
