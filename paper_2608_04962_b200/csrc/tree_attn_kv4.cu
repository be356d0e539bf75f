// Tree attention over the 4-bit paged cache, for few query rows per KV head: single tokens and small trees.
//
// A CTA takes one chunk of a sequence's pages for one KV head and up to 8 R8 query rows (rows = nodes x query heads of the KV head).
// Whole pages (K and V codes and scales of the head are one run of 136 D bytes) go into a ring with untiled bulk copies, which the first
// warp issues on the side; each of the eight warps has 16 of a page's tokens and decodes them straight into mma.sync fragments, so that a cached
// element passes through shared memory once, as four bits, and is decoded once for all rows:
//   S^T (16 tokens x 8 rows)  = K (A operand, from codes) x Q^T (B operand, in registers for the whole unit)
//   O^T (D x 8 rows)         += V^T (A operand, from codes) x P^T (B operand: P transposed by movmatrix)
// What an index of a fragment stands for is free as long as both operands agree, and is chosen so that a thread's codes are
// contiguous: for K a thread has 1/4 of a token's elements (one scale block where D = 128), for V 1/8 of four tokens' elements,
// paired by byte permutes before decoding.  Tokens of a pair change places in every other pair, which halves the bank conflicts
// of V's reads.
// Every warp has a softmax of its own (reference maximum per row, moved only when a score exceeds it by 2^8); the eight meet in
// shared memory at the end.  The tree's bf16 rows are done by the first warps after the cache.
// What bounds it: 17 KB of a page in 0.4 us at the HBM rate of one SM, against about 450 issue slots a scheduler for decoding it.
#include <math.h>

#include "kv4.cuh"
#include "tc05.cuh"
#include "tree_attn.cuh"

namespace specroll {

namespace akv4 {
constexpr int WARPS = 8, THREADS = 32 * WARPS;
constexpr int STAGES = 6, LAG = 2;  // a stage is loaded anew LAG tiles after its last use began, when every warp is done with it
constexpr float RESCALE_LOG2 = 8.0f;

template <int D, int R8>
struct Cfg {
    static constexpr int PAIR = 2 * Kv4<D>::TILE;  // K and V of a page and head
    static constexpr int RING = STAGES * PAIR;
    static constexpr int RUN = D / 4, STEPS = D / 16;  // a thread's elements of a K row; contraction steps of S
    static constexpr int VRUN = D / 8, MB = D / 16;    // a thread's elements of a V row; row blocks of O^T
    static constexpr int ROWS = 8 * R8;
    // at the end: per warp the rows' references and sums, and O
    static constexpr int O_FLOATS = D * ROWS;
    static constexpr int JOIN = WARPS * (O_FLOATS + 2 * ROWS) * 4;
    static constexpr int BODY = (RING > JOIN ? RING : JOIN);
    static constexpr int SMEM = BODY + 16 * STAGES + 4 * STAGES + 16;
};

__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
}  // namespace akv4

template <int D, int R8>
__global__ void __launch_bounds__(akv4::THREADS, R8 == 1 ? 2 : 1)
tree_attn_kv4_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ TopoMask mask, int32_t *__restrict__ status) {
    using namespace akv4;
    using C = Cfg<D, R8>;
    extern __shared__ __align__(128) unsigned char smem[];
    const uint32_t ring_s = smem_u32(smem), bars = ring_s + C::BODY;
    auto full = [&](int s) { return bars + 8u * (uint32_t)s; };
    auto empty = [&](int s) { return bars + 8u * (uint32_t)(STAGES + s); };
    volatile int *const gone = reinterpret_cast<volatile int *>(smem + C::BODY + 16 * STAGES);  // [STAGES]: no such page
    volatile int *const abort_flag = gone + STAGES;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, c = lane & 3;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), WARPS);
        }
        *abort_flag = 0;
        fence_mbar_init();
    }
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();

    // ---- the unit: (chunk in work order, KV head, row block)
    int w = blockIdx.x;
    const int rb = w % a.n_rb;
    w /= a.n_rb;
    const int hkv = w % a.Hkv, si = w / a.Hkv;
    const int4 e0 = __ldg(reinterpret_cast<const int4 *>(a.unit_tab) + 2 * (size_t)si);
    const int4 e1 = __ldg(reinterpret_cast<const int4 *>(a.unit_tab) + 2 * (size_t)si + 1);
    const int b = e0.x, split = e0.y, n_splits = e0.z, item = e0.w + split, slot0 = e1.x, L = e1.y;
    const int tiles_b = (L + SPECROLL_PAGE_TOKENS - 1) / SPECROLL_PAGE_TOKENS;
    const int tps = (tiles_b + n_splits - 1) / n_splits;
    const int t_lo = min(tiles_b, split * tps), n_t = min(tiles_b, t_lo + tps) - t_lo;
    const bool has_tree = split == n_splits - 1;
    const int N = a.N, G = a.G, row0 = rb * C::ROWS;

    float o[R8][C::MB][4];
    float m[R8][2], l[R8][2];
#pragma unroll
    for (int r = 0; r < R8; ++r) {
        m[r][0] = m[r][1] = -INFINITY;
        l[r][0] = l[r][1] = 0.f;
#pragma unroll
        for (int i = 0; i < C::MB; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[r][i][e] = 0.f;
    }

    // ---- loads: tile t into stage t mod STAGES, by one thread (false: a wait ran out)
    const int32_t *const pt = a.page_table + slot0 + t_lo;
    int next_page = n_t > 0 && threadIdx.x == 0 ? __ldg(pt) : 0;
    auto load = [&](int t) -> bool {
        const int s = t % STAGES, page = next_page;
        next_page = t + 1 < n_t ? __ldg(pt + t + 1) : 0;
        if (t >= STAGES && !mbar_wait(empty(s), (t / STAGES - 1) & 1u, abort_flag)) return false;
        const bool there = page >= 0 && page < a.n_pages;
        gone[s] = !there;
        if (there) {
            mbar_arrive_expect_tx(full(s), C::PAIR);
            bulk_load(ring_s + s * C::PAIR, a.pool + ((size_t)page * a.Hkv + hkv) * C::PAIR, C::PAIR, full(s));
        } else {
            mbar_arrive(full(s));  // (read as zeros)
        }
        return true;
    };
    if (threadIdx.x == 0)
        for (int t = 0; t < min(n_t, STAGES); ++t) load(t);
    __syncwarp();

    {
        // ------------------------------------------------------------------ attention
        // Q: rows g of every block of eight, the elements of this thread's run
        uint32_t qf[R8][2 * C::STEPS];
#pragma unroll
        for (int r = 0; r < R8; ++r) {
            const int gr = row0 + 8 * r + g;
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
        // the tokens (of 16) that a thread's indexes stand for: index 2 j + e is token 2 j + (e ^ (j & 1))
        const int k_tok = g ^ ((g >> 1) & 1);               // K rows g and g + 8: tokens k_tok and k_tok + 8
        const int v_a = 2 * c + (c & 1), v_b = v_a ^ 1;     // V pairs: tokens (v_a, v_b) and those + 8
        const float sc = a.scale_log2;

        // Scores (already products) to probabilities: ok0 / ok1 are bit masks over r and e for tokens k_tok and k_tok + 8.
        auto softmax = [&](float(&s)[R8][4], auto admits, uint32_t(&pf)[R8][2]) {
            bool move = false;
#pragma unroll
            for (int r = 0; r < R8; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[r][e] = admits(r, e) ? s[r][e] * sc : -INFINITY;
                    move |= s[r][e] > m[r][e & 1] + RESCALE_LOG2;
                }
            if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                for (int r = 0; r < R8; ++r)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(s[r][e], s[r][e + 2]);
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                        if (mx > m[r][e] + RESCALE_LOG2) {
                            const float f = ex2_approx(m[r][e] - mx);
                            m[r][e] = mx;
                            l[r][e] *= f;
#pragma unroll
                            for (int i = 0; i < C::MB; ++i) {
                                o[r][i][e] *= f;
                                o[r][i][e + 2] *= f;
                            }
                        }
                    }
            }
#pragma unroll
            for (int r = 0; r < R8; ++r) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = ex2_approx(s[r][e] - (m[r][e & 1] == -INFINITY ? 0.f : m[r][e & 1]));
                l[r][0] += p[0] + p[2];
                l[r][1] += p[1] + p[3];
                pf[r][0] = movmatrix(pack_bf16x2(p[0], p[1]));
                pf[r][1] = movmatrix(pack_bf16x2(p[2], p[3]));
            }
        };

        bool ok = true;
        for (int t = 0; t < n_t; ++t) {
            const int st = t % STAGES;
            if (threadIdx.x == 0 && t >= LAG && t + STAGES - LAG < n_t) load(t + STAGES - LAG);
            __syncwarp();
            ok = mbar_wait(full(st), (t / STAGES) & 1u, abort_flag);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const unsigned char *tile = smem + st * C::PAIR;
            const uint32_t keep = gone[st] ? 0u : 0xffffffffu;
            // ---- S^T = K Q^T
            float s[R8][4];
#pragma unroll
            for (int r = 0; r < R8; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[r][e] = 0.f;
            {
                const int t0 = 16 * warp + k_tok;
                uint32_t kw[2][C::RUN / 8], s2[2], o2[2];
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
                    const uint32_t sb = tile[Kv4<D>::CODES + (t0 + 8 * h) * Kv4<D>::SROW + (D == 128 ? c : c >> 1)];
                    s2[h] = kv4_scale_pair(sb, sb) & keep;
                    o2[h] = kv4_offset(s2[h]);
                }
#pragma unroll
                for (int i = 0; i < C::RUN / 8; ++i) {
                    uint32_t lo[4], hi[4];
                    kv4_word(kw[0][i], s2[0], o2[0], lo);
                    kv4_word(kw[1][i], s2[1], o2[1], hi);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t af[4] = {lo[2 * h], hi[2 * h], lo[2 * h + 1], hi[2 * h + 1]};
#pragma unroll
                        for (int r = 0; r < R8; ++r) mma_bf16_16816(s[r], af, qf[r][4 * i + 2 * h], qf[r][4 * i + 2 * h + 1]);
                    }
                }
            }
            // ---- softmax
            uint32_t pf[R8][2];
            const int left = L - (t_lo + t) * SPECROLL_PAGE_TOKENS - 16 * warp - k_tok;  // > 0: token k_tok is in the sequence
            softmax(s, [&](int, int e) { return left > (e & 2 ? 8 : 0); }, pf);
            // ---- O^T += V^T P^T
            {
                const unsigned char *vt = tile + Kv4<D>::TILE;
                uint32_t vw[4][C::VRUN / 8], sb[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int tok = 16 * warp + ((q & 1) ? v_b : v_a) + 8 * (q >> 1);
                    const unsigned char *row = vt + tok * Kv4<D>::ROW + (C::VRUN / 2) * g;
                    if constexpr (D == 128) {
                        const uint2 x = *reinterpret_cast<const uint2 *>(row);
                        vw[q][0] = x.x, vw[q][1] = x.y;
                    } else {
                        vw[q][0] = *reinterpret_cast<const uint32_t *>(row);
                    }
                    sb[q] = vt[Kv4<D>::CODES + tok * Kv4<D>::SROW + (g * C::VRUN) / 32];
                }
                const uint32_t s0 = kv4_scale_pair(sb[0], sb[1]) & keep, s1 = kv4_scale_pair(sb[2], sb[3]) & keep;
                const uint32_t f0 = kv4_offset(s0), f1 = kv4_offset(s1);
#pragma unroll
                for (int i = 0; i < C::VRUN / 8; ++i) {
                    // lower halves: elements 0 2 4 6 of the word, upper halves: 1 3 5 7, of two tokens each
                    uint32_t e0_[4], e1_[4], d0_[4], d1_[4];
                    kv4_word(__byte_perm(vw[0][i], vw[1][i], 0x5410), s0, f0, e0_);
                    kv4_word(__byte_perm(vw[0][i], vw[1][i], 0x7632), s0, f0, d0_);
                    kv4_word(__byte_perm(vw[2][i], vw[3][i], 0x5410), s1, f1, e1_);
                    kv4_word(__byte_perm(vw[2][i], vw[3][i], 0x7632), s1, f1, d1_);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t af[4] = {e0_[j], d0_[j], e1_[j], d1_[j]};
#pragma unroll
                        for (int r = 0; r < R8; ++r) mma_bf16_16816(o[r][4 * i + j], af, pf[r][0], pf[r][1]);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty(st));
        }
        if (ok && has_tree && 16 * warp < N) {
            // ---- the tree's rows, bf16 from global memory, sixteen nodes a warp
            float s[R8][4];
#pragma unroll
            for (int r = 0; r < R8; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[r][e] = 0.f;
            const size_t rows_of_b = (size_t)b * N;
            const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
            uint4 kx[2][C::RUN / 8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = 16 * warp + k_tok + 8 * h;
                const uint4 *src = reinterpret_cast<const uint4 *>(a.Kt + ((rows_of_b + n) * a.Hkv + hkv) * D + C::RUN * c);
#pragma unroll
                for (int i = 0; i < C::RUN / 8; ++i) kx[h][i] = n < N ? __ldg(src + i) : zero;
            }
#pragma unroll
            for (int i = 0; i < C::RUN / 8; ++i) {
                const uint32_t lo[4] = {kx[0][i].x, kx[0][i].y, kx[0][i].z, kx[0][i].w};
                const uint32_t hi[4] = {kx[1][i].x, kx[1][i].y, kx[1][i].z, kx[1][i].w};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t af[4] = {lo[2 * h], hi[2 * h], lo[2 * h + 1], hi[2 * h + 1]};
#pragma unroll
                    for (int r = 0; r < R8; ++r) mma_bf16_16816(s[r], af, qf[r][4 * i + 2 * h], qf[r][4 * i + 2 * h + 1]);
                }
            }
            uint32_t pf[R8][2];
            const int n0 = 16 * warp + k_tok;
            softmax(s, [&](int r, int e) {
                const int gr = row0 + 8 * r + 2 * c + (e & 1);
                return gr < a.rows && ((mask.anc[gr / G] >> (n0 + (e & 2 ? 8 : 0))) & 1ull);
            }, pf);
            uint4 vx[4][C::VRUN / 8];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = 16 * warp + ((q & 1) ? v_b : v_a) + 8 * (q >> 1);
                const uint4 *src = reinterpret_cast<const uint4 *>(a.Vt + ((rows_of_b + n) * a.Hkv + hkv) * D + C::VRUN * g);
#pragma unroll
                for (int i = 0; i < C::VRUN / 8; ++i) vx[q][i] = n < N ? __ldg(src + i) : zero;
            }
#pragma unroll
            for (int i = 0; i < C::VRUN / 8; ++i) {
                const uint32_t x[4][4] = {{vx[0][i].x, vx[0][i].y, vx[0][i].z, vx[0][i].w}, {vx[1][i].x, vx[1][i].y, vx[1][i].z, vx[1][i].w},
                                          {vx[2][i].x, vx[2][i].y, vx[2][i].z, vx[2][i].w}, {vx[3][i].x, vx[3][i].y, vx[3][i].z, vx[3][i].w}};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t af[4] = {__byte_perm(x[0][j], x[1][j], 0x5410), __byte_perm(x[0][j], x[1][j], 0x7632),
                                            __byte_perm(x[2][j], x[3][j], 0x5410), __byte_perm(x[2][j], x[3][j], 0x7632)};
#pragma unroll
                    for (int r = 0; r < R8; ++r) mma_bf16_16816(o[r][4 * i + j], af, pf[r][0], pf[r][1]);
                }
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
        const int row = i % C::ROWS, d4 = i / C::ROWS, gr = row0 + row;
        if (gr >= a.rows) continue;
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
        const int n = gr / G, gq = gr % G;
        if (n_splits == 1) {
            const float inv = sum > 0.f ? 1.0f / sum : 0.f;
            const size_t at = ((size_t)b * N + n) * a.Hq + hkv * G + gq;
            *reinterpret_cast<uint2 *>(a.O + at * D + 4 * d4) =
                make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
            if (a.lse && d4 == 0) a.lse[at] = (M + log2f(sum)) * 0.6931471805599453f;
        } else {
            const size_t unit = (size_t)item * a.Hkv + hkv;
            reinterpret_cast<float4 *>(a.part_o)[(unit * (D / 4) + d4) * a.rows_pad + gr] = acc;
            if (d4 == 0) reinterpret_cast<float2 *>(a.part_ml)[unit * a.rows_pad + gr] = make_float2(M, sum);
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

int launch_attn_kv4(const AttnArgs &a, const TopoMask &mask, int D, int32_t *status, cudaStream_t st) {
    const bool one = a.rows_per_block == 8;
    if (D == 128) return one ? launch_kv4<128, 1>(a, mask, status, st) : launch_kv4<128, 2>(a, mask, status, st);
    return one ? launch_kv4<64, 1>(a, mask, status, st) : launch_kv4<64, 2>(a, mask, status, st);
}

}  // namespace specroll
