// The matrix product of the operators on a caller's own activations and weights: 16-bit operands, fp32 sums, tcgen05.
//
// One persistent kernel.  A warp fetches blocks of 64 along the summed axis of both operands by TMA into a ring, a warp issues the products,
// eight warps work on finished tiles out of tensor memory while the products of the next one run (two accumulators).  Operands may lie either
// way: rows along the summed axis (boxes of 64 rows of 64 elements, "MN-major") or across it ("K-major"); nothing is transposed in memory.
#include "xsm_product.cuh"

#include <limits.h>
#include <string.h>

#include <atomic>
#include <type_traits>

namespace xsm {

constexpr int kEpiWarps = 8;
constexpr int kProductThreads = 64 + 32 * kEpiWarps;
constexpr int kABytes = 128 * 128;              // of a stage and a CTA: 128 rows of A, 64 elements of the summed axis
constexpr int kRingBytes = 192 * 1024;

template <int CG, int BN> struct Cut {
    static constexpr int stage = kABytes + BN / CG * 128, stages = kRingBytes / stage, tm = 128 * CG;
};

// ------------------------------------------------------------------------------------------- instructions

// Descriptor of an operand tile with the 128-byte swizzle.  K-major: rows of 64 elements, groups of 8 rows 1024 bytes apart.  MN-major: rows of
// 64 elements across the summed axis, groups of 8 steps of it 1024 bytes apart, the next 64 elements a box (8 KB) further.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool mn) {
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)(mn ? 8192 >> 4 : 1) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
template <typename T> __device__ __forceinline__ uint32_t product_idesc(int m, int n, bool a_mn, bool b_mn) {
    const uint32_t f = std::is_same<T, bf16>::value ? 1u : 0u;
    return (1u << 4) | (f << 7) | (f << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
template <int CG> __device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// an arrival at the barrier (of both CTAs of a pair) when the products issued so far have completed
template <int CG> __device__ __forceinline__ void commit(uint32_t bar) {
    if constexpr (CG == 1)
        umma_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" :: "r"(bar), "h"((uint16_t)3) : "memory");
}
template <int CG> __device__ __forceinline__ void tma_2d(uint32_t dst, const void *map, int x, int y, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                     :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// the same at this CTA's barrier alone
template <int CG> __device__ __forceinline__ void commit_here(uint32_t bar) {
    if constexpr (CG == 1) umma_commit(bar);
    else asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(bar) : "memory");
}
template <int N> __device__ __forceinline__ void tmem_ld(uint32_t (&v)[N], uint32_t addr) {
    if constexpr (N == 16) {
        tmem_ld16(v, addr);
    } else {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,"
                     "%28,%29,%30,%31}, [%32];"
                     : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
                       "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]),
                       "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]),
                       "=r"(v[31]) : "r"(addr) : "memory");
    }
}

// ------------------------------------------------------------------------------------------------- numbers

// act(g) and its derivative
__device__ __forceinline__ void activate(int kind, float g, float &a, float &da) {
    if (kind == ACT_SILU) {
        const float s = __fdividef(1.f, 1.f + ex2(-g * kLog2e));
        a = g * s;
        da = s * (1.f + g * (1.f - s));
    } else {
        const float c = 0.5f * erfcf(-0.70710678f * g);
        a = g * c;
        da = c + g * 0.39894228f * ex2(-0.5f * kLog2e * g * g);
    }
}

// Power of two that takes the largest of kAmaxBlocks numbers to [2^to, 2^(to + 1)); 1 where there is none.
__device__ __forceinline__ float scale_of(const float *amax, int to) {
    if (amax == nullptr) return 1.f;
    float m = 0.f;
    for (int i = threadIdx.x & 31; i < kAmaxBlocks; i += 32) m = fmaxf(m, amax[i]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (!(m > 0.f)) return 1.f;
    int e = (int)(__float_as_uint(m) >> 23) - 127;
    e = max(-100, min(100, to - e));
    return __uint_as_float((unsigned)(e + 127) << 23);
}

template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b) {
    T p[2] = {rounded<T>(a), rounded<T>(b)};
    uint32_t r;
    memcpy(&r, p, 4);
    return r;
}
// N numbers to a row's columns from `col` on, of `n`; whole: 16-byte pieces fit
template <typename T, int N> __device__ __forceinline__ void store_row(T *row, int col, int n, bool whole, const float (&x)[N]) {
    if (whole && col + N <= n) {
#pragma unroll
        for (int i = 0; i < N; i += 8)
            *reinterpret_cast<uint4 *>(row + col + i) = make_uint4(pack2<T>(x[i], x[i + 1]), pack2<T>(x[i + 2], x[i + 3]), pack2<T>(x[i + 4], x[i + 5]), pack2<T>(x[i + 6], x[i + 7]));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (col + i < n) row[col + i] = rounded<T>(x[i]);
    }
}

// -------------------------------------------------------------------------------------------------- kernel

struct Tile { int m, n, split, job, k0, k1; };
__device__ __forceinline__ Tile tile_of(const ProductArgs &A, int t) {
    Tile r;
    r.m = t % A.tiles_m;
    t /= A.tiles_m;
    r.n = t % A.tiles_n;
    t /= A.tiles_n;
    r.split = t % A.splits;
    r.job = t / A.splits;
    r.k0 = (int)((long long)A.kb * r.split / A.splits);
    r.k1 = (int)((long long)A.kb * (r.split + 1) / A.splits);
    return r;
}

template <int CG, int BN, int EPI, typename T>
__global__ void __launch_bounds__(kProductThreads, 1) product_kernel(const __grid_constant__ ProductMaps M, const __grid_constant__ ProductArgs A) {
    using C = Cut<CG, BN>;
    constexpr int S = C::stages;
    extern __shared__ char smem_raw[];
    __shared__ __align__(8) uint64_t full[S], empty[S], sums_full[2], sums_empty[2], last;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int dead;           // a wait of this CTA has run out
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0, first = blockIdx.x / CG, step = gridDim.x / CG;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    chain_go();
    if (tid == 0) {
        for (int i = 0; i < S; ++i) { mbar_init(smem_u32(&full[i]), 1u); mbar_init(smem_u32(&empty[i]), 1u); }
        for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&sums_full[i]), 1u); mbar_init(smem_u32(&sums_empty[i]), kEpiWarps * CG); }
        mbar_init(smem_u32(&last), 1u);
        dead = 0;
        mbar_init_fence();
    }
    if (warp == 1) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&tmem_slot)), "n"(2 * BN) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&tmem_slot)), "n"(2 * BN) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    tcgen05_before_sync();
    __syncthreads();
    if constexpr (CG == 2) { cluster_arrive(); cluster_wait(); }
    tcgen05_after_sync();
    const uint32_t tmem = tmem_slot;
    chain_wait();

    // false: the limit ran out, here or elsewhere in the CTA; the results are void
    auto wait = [&](uint64_t &b, uint32_t parity) {
        const uint32_t bar = smem_u32(&b);
        for (unsigned i = 0; i <= A.tries; ++i) {
            if (mbar_try_wait(bar, parity)) return true;
            if ((i & 63u) == 63u && dead) return false;
        }
        dead = 1;
        atomicExch(A.status, XSM_STATUS_TIMEOUT);
        return false;
    };

    auto wait_warp = [&](uint64_t &b, uint32_t parity) { return __all_sync(0xffffffffu, wait(b, parity)) != 0; };        // (all lanes or none)

    if (warp == 0) {
        if (elect_one()) {
            int fills = 0;        // stages asked for
            bool ok = true;
            int s = 0;
            uint32_t par = 1u;
            for (int t = first; ok && t < A.tiles; t += step) {
                const Tile w = tile_of(A, t);
                const int m0 = w.m * C::tm + rank * 128, n0 = EPI == PR_GATED || EPI == PR_GATED_GRAD ? w.n * (BN / 2) : w.n * BN + rank * (BN / CG);
                for (int k = w.k0; k < w.k1; ++k) {
                    if (!(ok = wait(empty[s], par))) break;
                    if (!A.starve) {
                        const uint32_t f = CG == 2 ? map_rank(smem_u32(&full[s]), 0) : smem_u32(&full[s]);
                        if (rank == 0) mbar_arrive_expect_tx(smem_u32(&full[s]), A.stage_tx);
                        const uint32_t sa = ring + (uint32_t)(s * C::stage), sb = sa + kABytes;
                        const int pair = k >= A.kb0, at = (k - (pair ? A.kb0 : 0)) * 64;
                        const void *ma = &M.a[pair + w.job], *mb = &M.b[pair];
                        if (A.a_mn) {
                            tma_2d<CG>(sa, ma, m0, at, f);
                            tma_2d<CG>(sa + 8192, ma, m0 + 64, at, f);
                        } else {
                            tma_2d<CG>(sa, ma, at, m0, f);
                        }
                        if constexpr (EPI == PR_GATED || EPI == PR_GATED_GRAD) {
                            if constexpr (CG == 2) {
                                tma_2d<CG>(sb, &M.b[rank], at, n0, f);
                            } else {
                                tma_2d<CG>(sb, &M.b[0], at, n0, f);
                                tma_2d<CG>(sb + BN / 2 * 128, &M.b[1], at, n0, f);
                            }
                        } else if (A.b_mn) {
#pragma unroll
                            for (int i = 0; i < BN / CG / 64; ++i) tma_2d<CG>(sb + i * 8192, mb, n0 + 64 * i, at, f);
                        } else {
                            tma_2d<CG>(sb, mb, at, n0, f);
                        }
                        ++fills;
                    }
                    if (++s == S) { s = 0; par ^= 1u; }
                }
            }
            // What was asked for lands before the CTA ends, also where nobody waits for it any more.  (Both CTAs' copies count on this one's barriers.)
            if (rank == 0)
                for (int i = max(0, fills - S); i < fills; ++i)
                    for (unsigned n = 0; n < A.tries && !mbar_try_wait(smem_u32(&full[i % S]), (uint32_t)(i / S) & 1u); ++n);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            const bool leader = elect_one();
            const uint32_t idesc = product_idesc<T>(128 * CG, BN, A.a_mn, A.b_mn);
            const uint64_t da = operand_desc(ring, A.a_mn), db = operand_desc(ring + kABytes, A.b_mn);
            const uint32_t a_step = A.a_mn ? 2048 >> 4 : 32 >> 4, b_step = A.b_mn ? 2048 >> 4 : 32 >> 4;
            bool ok = true;
            int s = 0, acc = 0;
            uint32_t par = 0u, acc_par = 1u;
            for (int t = first; ok && t < A.tiles; t += step) {
                const Tile w = tile_of(A, t);
                if (!(ok = wait_warp(sums_empty[acc], acc_par))) break;
                tcgen05_after_sync();
                const uint32_t d = tmem + (uint32_t)(acc * BN);
                for (int k = w.k0; k < w.k1; ++k) {
                    if (!(ok = wait_warp(full[s], par))) break;
                    tcgen05_after_sync();
                    if (leader) {
                        const uint64_t a = da + (uint64_t)(uint32_t)(s * (C::stage >> 4)), b = db + (uint64_t)(uint32_t)(s * (C::stage >> 4));
#pragma unroll
                        for (int i = 0; i < 4; ++i) mma_f16<CG>(d, a + i * a_step, b + i * b_step, idesc, (k > w.k0 || i > 0) ? 1u : 0u);
                        commit<CG>(smem_u32(&empty[s]));
                    }
                    __syncwarp();
                    if (++s == S) { s = 0; par ^= 1u; }
                }
                if (!ok) break;
                if (leader) commit<CG>(smem_u32(&sums_full[acc]));
                __syncwarp();
                if (++acc == 2) { acc = 0; acc_par ^= 1u; }
            }
            // products under way end before the tensor memory goes back, also where nobody waits for them any more
            if (leader) commit_here<CG>(smem_u32(&last));
            __syncwarp();
            for (unsigned n = 0; n < A.tries && !mbar_try_wait(smem_u32(&last), 0u); ++n);
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        const float scale = scale_of(A.amax, A.amax_to);
        int acc = 0;
        uint32_t acc_par = 0u;
        for (int t = first; t < A.tiles; t += step) {
            const Tile w = tile_of(A, t);
            const int row = w.m * C::tm + rank * 128 + quarter * 32 + lane;
            const bool live = row < A.m;
            if (!wait_warp(sums_full[acc], acc_par)) break;
            tcgen05_after_sync();
            const uint32_t sums = lanes + (uint32_t)(acc * BN);
            if constexpr (EPI == PR_GATED || EPI == PR_GATED_GRAD) {
                constexpr int N = BN / 4 < 32 ? BN / 4 : 32;
                const int col0 = w.n * (BN / 2) + half * (BN / 4);
                const bool whole = (A.out_ld & 7) == 0;
#pragma unroll 1
                for (int c = 0; c < BN / 4; c += N) {
                    uint32_t vg[N], vu[N];
                    tmem_ld(vg, sums + (uint32_t)(half * (BN / 4) + c));
                    tmem_ld(vu, sums + (uint32_t)(BN / 2 + half * (BN / 4) + c));
                    const int col = col0 + c;
                    float x[N];
                    if constexpr (EPI == PR_GATED_GRAD) {
                        const T *gy = reinterpret_cast<const T *>(A.g_y) + (long long)row * A.g_y_ld;
                        if (live && col + N <= A.n && (A.g_y_ld & 7) == 0 && ((uintptr_t)A.g_y & 15) == 0) {
#pragma unroll
                            for (int i = 0; i < N; i += 8) {
                                const uint4 u = *reinterpret_cast<const uint4 *>(gy + col + i);
                                T e[8];
                                memcpy(e, &u, 16);
#pragma unroll
                                for (int j = 0; j < 8; ++j) x[i + j] = to_f(e[j]) * scale;
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < N; ++i) x[i] = live && col + i < A.n ? to_f(gy[col + i]) * scale : 0.f;
                        }
                    }
                    tmem_wait_ld();
                    if constexpr (EPI == PR_GATED) {
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            float a, da;
                            activate(A.activation, __uint_as_float(vg[i]), a, da);
                            x[i] = a * __uint_as_float(vu[i]);
                        }
                        if (live) store_row(reinterpret_cast<T *>(A.out[0]) + (long long)row * A.out_ld, col, A.n, whole && ((uintptr_t)A.out[0] & 15) == 0, x);
                    } else {
                        float y[N];
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            float a, da;
                            activate(A.activation, __uint_as_float(vg[i]), a, da);
                            y[i] = x[i] * a;
                            x[i] = x[i] * __uint_as_float(vu[i]) * da;
                        }
                        if (live) {        // (workspace rows of a multiple of eight elements: what lies behind the last column is nobody's)
                            const int n8 = (int)A.out_ld;
                            store_row(reinterpret_cast<T *>(A.out[0]) + (long long)row * A.out_ld, col, n8, true, x);
                            store_row(reinterpret_cast<T *>(A.out[1]) + (long long)row * A.out_ld, col, n8, true, y);
                        }
                    }
                }
            } else {
                constexpr int N = 32;
                const int col0 = w.n * BN + half * (BN / 2);
                long long token = -1;
                float mx = -INFINITY, sum = 0.f, g = 0.f, gp = 0.f, lse2 = 0.f;
                if (EPI == PR_STATS || EPI == PR_DLOGITS) {
                    if (live) {
                        token = A.token_bytes == 8 ? reinterpret_cast<const long long *>(A.tokens)[row * A.token_ld] : (long long)reinterpret_cast<const int *>(A.tokens)[row * A.token_ld];
                        token -= A.vocab0;
                        if constexpr (EPI == PR_DLOGITS) {
                            const bool there = token + A.vocab0 >= 0 && token + A.vocab0 < A.vocab;
                            const float lse = A.lse[row];
                            g = A.g && there ? A.g[row * A.g_ld] : 0.f;
                            gp = g - (A.g_lse ? A.g_lse[row * A.g_lse_ld] : 0.f);
                            g *= A.inv_t * scale;
                            gp *= A.inv_t * scale;
                            lse2 = lse * kLog2e;
                            if (lse == -INFINITY) g = gp = lse2 = 0.f;
                        }
                    }
                }
#pragma unroll 1
                for (int c = 0; c < BN / 2; c += N) {
                    uint32_t v[N];
                    tmem_ld(v, sums + (uint32_t)(half * (BN / 2) + c));
                    const int col = col0 + c;
                    tmem_wait_ld();
                    float x[N];
                    if constexpr (EPI == PR_STATS) {
                        const int n = A.n - col;
                        float top = -INFINITY;
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            x[i] = i < n ? __uint_as_float(v[i]) * A.c : -INFINITY;
                            top = fmaxf(top, x[i]);
                        }
                        if (token >= col && token < col + N) {
#pragma unroll
                            for (int i = 0; i < N; ++i)
                                if (token == col + i && i < n) A.token_z[row] = __uint_as_float(v[i]) * A.inv_t;
                        }
                        const float was = mx;
                        mx = fmaxf(mx, top);
                        const float base = mx == -INFINITY ? 0.f : mx;
                        sum *= ex2(was - base);
#pragma unroll
                        for (int i = 0; i < N; ++i) sum += ex2(x[i] - base);
                    } else if constexpr (EPI == PR_DLOGITS) {
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            x[i] = -gp * ex2(fmaf(__uint_as_float(v[i]), A.c, -lse2));
                            if (token == col + i) x[i] += g;
                        }
                        if (live) store_row(reinterpret_cast<T *>(A.out[0]) + (long long)row * A.out_ld, col, (int)A.out_ld, true, x);
                    } else {
                        if (A.partial) {
                            float *p = A.partial + (((long long)w.job * A.splits + w.split) * A.m + row) * A.n + col;
                            if (live)
#pragma unroll
                                for (int i = 0; i < N; i += 4)
                                    if (col + i < A.n) {
                                        float4 o = make_float4(__uint_as_float(v[i]), __uint_as_float(v[i + 1]), __uint_as_float(v[i + 2]), __uint_as_float(v[i + 3]));
                                        if (A.add) {
                                            const float4 q = *reinterpret_cast<const float4 *>(p + i);
                                            o.x += q.x; o.y += q.y; o.z += q.z; o.w += q.w;
                                        }
                                        *reinterpret_cast<float4 *>(p + i) = o;
                                    }
                        } else if (live) {
                            const float back = 1.f / scale;
#pragma unroll
                            for (int i = 0; i < N; ++i) x[i] = __uint_as_float(v[i]) * back;
                            store_row(reinterpret_cast<T *>(A.out[w.job]) + (long long)row * A.out_ld, col, A.n, true, x);
                        }
                    }
                }
                if constexpr (EPI == PR_STATS) {
                    if (live) A.parts[(long long)(2 * w.n + half) * A.m + row] = make_float2(mx, sum);
                }
            }
            tcgen05_before_sync();
            __syncwarp();
            if (lane == 0) {
                if constexpr (CG == 2) arrive_cluster(map_rank(smem_u32(&sums_empty[acc]), 0));
                else mbar_arrive(smem_u32(&sums_empty[acc]));
            }
            if (++acc == 2) { acc = 0; acc_par ^= 1u; }
        }
        __syncwarp();
    }
    tcgen05_before_sync();
    __syncthreads();
    if constexpr (CG == 2) { cluster_arrive(); cluster_wait(); }        // (nobody leaves while the other CTA's barriers and memory are still in use)
    if (warp == 1) {
        tcgen05_after_sync();
        if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(2 * BN) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(2 * BN) : "memory");
    }
}

// -------------------------------------------------------------------------------------------- small kernels

// the largest |x| of 16-bit elements, infinities and NaN apart, a number for each block
template <typename T>
__global__ void __launch_bounds__(256) amax_rows_kernel(const T *x, long long rows, int cols, long long ld, float *amax) {
    chain_go();
    chain_wait();
    __shared__ float s[8];
    float m = 0.f;
    auto take = [&](float v) { v = fabsf(v); if (v < INFINITY) m = fmaxf(m, v); };
    const bool whole = ((uintptr_t)x & 15) == 0 && (ld & 7) == 0;
    const int pieces = whole ? cols / 8 : 0;
    for (long long r = blockIdx.x; r < rows; r += kAmaxBlocks) {
        const T *row = x + r * ld;
#pragma unroll 4
        for (int i = threadIdx.x; i < pieces; i += 256) {
            const uint4 u = reinterpret_cast<const uint4 *>(row)[i];
            T e[8];
            memcpy(e, &u, 16);
#pragma unroll
            for (int j = 0; j < 8; ++j) take(to_f(e[j]));
        }
        for (int i = pieces * 8 + threadIdx.x; i < cols; i += 256) take(to_f(row[i]));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) m = fmaxf(m, s[i]);
        amax[blockIdx.x] = m;
    }
}

__global__ void __launch_bounds__(32) amax_pairs_kernel(const float *g, long long g_ld, const float *h, long long h_ld, int rows, float by, float *amax) {
    chain_go();
    chain_wait();
    float m = 0.f;
    for (int r = blockIdx.x * 32 + threadIdx.x; r < rows; r += kAmaxBlocks * 32) {
        const float v = (2.f * (g ? fabsf(g[r * g_ld]) : 0.f) + (h ? fabsf(h[r * h_ld]) : 0.f)) * by;
        if (v < INFINITY) m = fmaxf(m, v);
        if (r > INT_MAX - kAmaxBlocks * 32) break;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (threadIdx.x == 0) amax[blockIdx.x] = m;
}

struct JoinArgs {
    const float *partial, *amax;
    void *out[2];
    long long out_ld, all;          // all: quads of a job
    int m, n, splits, amax_to;
};
template <typename T> __global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ JoinArgs A) {
    chain_go();
    chain_wait();
    const float back = 1.f / scale_of(A.amax, A.amax_to);
    const int quads = A.n / 4, job = blockIdx.y;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < A.all; i += gridDim.x * 256ll) {
        const long long r = i / quads;
        const int c = (int)(i - r * quads) * 4;
        const float *p = A.partial + ((long long)job * A.splits * A.m + r) * A.n + c;
        float4 s = *reinterpret_cast<const float4 *>(p);
#pragma unroll 4
        for (int k = 1; k < A.splits; ++k) {
            const float4 q = *reinterpret_cast<const float4 *>(p + (long long)k * A.m * A.n);
            s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
        }
        T *o = reinterpret_cast<T *>(A.out[job]) + r * A.out_ld + c;
        *reinterpret_cast<uint2 *>(o) = make_uint2(pack2<T>(s.x * back, s.y * back), pack2<T>(s.z * back, s.w * back));
    }
}

// ------------------------------------------------------------------------------------------------------ host

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static std::atomic<EncodeTiledFn> g_encode{nullptr};
static cudaError_t encoder(EncodeTiledFn *fn) {
    *fn = g_encode.load(std::memory_order_acquire);
    if (*fn) return cudaSuccess;
    void *p = nullptr;
    cudaDriverEntryPointQueryResult q;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q);
    if (e != cudaSuccess) return e;
    if (q != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
    *fn = (EncodeTiledFn)p;
    g_encode.store(*fn, std::memory_order_release);
    return cudaSuccess;
}

static bool operand_map(EncodeTiledFn encode, CUtensorMap *out, const Operand &o, int dtype, int box_rows) {
    cuuint64_t dims[2] = {(cuuint64_t)o.row, (cuuint64_t)o.rows}, strides[1] = {(cuuint64_t)o.ld * 2};
    cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, one[2] = {1, 1};
    return encode(out, dtype == XSM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(o.p), dims, strides, box, one,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int product_sms() {
    static std::atomic<int> known[kMaxDevices];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0;
    n = known[dev].load(std::memory_order_relaxed);
    if (n == 0 && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

static std::atomic<unsigned> g_tries{kMbarSpinLimit};
static std::atomic<int> g_starve{0};
void product_waits(unsigned *tries, int *starve) {
    *tries = g_tries.load(std::memory_order_relaxed);
    *starve = g_starve.load(std::memory_order_relaxed);
}

int product_splits(long long tiles, int kb, bool wide) {
    const int slots = wide ? product_sms() / 2 : product_sms();
    const long long s = tiles > 0 ? slots / tiles : 1;
    return (int)(s < 1 ? 1 : s > kb / 8 ? (kb / 8 < 1 ? 1 : kb / 8) : s);
}

template <int CG, int BN, int EPI, typename T> static cudaError_t start(const ProductMaps &M, const ProductArgs &A, cudaStream_t st) {
    using C = Cut<CG, BN>;
    const int smem = C::stage * C::stages + 1024;
    const void *fn = (const void *)product_kernel<CG, BN, EPI, T>;
    cudaError_t e = open_kernel(fn, smem, false);
    if (e != cudaSuccess) return e;
    const int slots = product_sms() / CG;
    if (slots < 1) return cudaErrorInvalidDevice;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((A.tiles < slots ? A.tiles : slots) * CG));
    cfg.blockDim = dim3(kProductThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim = {CG, 1, 1};
    cfg.attrs = at;
    cfg.numAttrs = CG == 2 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, product_kernel<CG, BN, EPI, T>, M, A);
}
template <int CG, int BN, typename T> static cudaError_t start_epi(ProductEpi epi, const ProductMaps &M, const ProductArgs &A, cudaStream_t st) {
    switch (epi) {
        case PR_STATS: return start<CG, BN, PR_STATS, T>(M, A, st);
        case PR_DLOGITS: return start<CG, BN, PR_DLOGITS, T>(M, A, st);
        case PR_GATED: return start<CG, BN, PR_GATED, T>(M, A, st);
        case PR_GATED_GRAD: return start<CG, BN, PR_GATED_GRAD, T>(M, A, st);
        default: return start<CG, BN, PR_OUT, T>(M, A, st);
    }
}

cudaError_t launch_product(ProductEpi epi, int dtype, bool wide, ProductArgs A, const Operand (&a)[2], const Operand (&b)[2], int pairs, cudaStream_t st) {
    EncodeTiledFn encode;
    cudaError_t e = encoder(&encode);
    if (e != cudaSuccess) return e;
    const bool gated = epi == PR_GATED || epi == PR_GATED_GRAD;
    const ProductCut cut = product_cut(wide);
    const int tm = 128 * cut.group, tn = gated ? cut.bn / 2 : cut.bn;
    A.tiles_m = (A.m + tm - 1) / tm;
    A.tiles_n = (A.n + tn - 1) / tn;
    const long long summed = A.a_mn ? a[0].rows : a[0].row;
    A.kb0 = (int)((summed + 63) / 64);
    A.kb = A.kb0 * pairs;
    const long long tiles = (long long)A.tiles_m * A.tiles_n * A.jobs * A.splits;
    if (tiles > 0x3fffffff) return cudaErrorInvalidValue;
    A.tiles = (int)tiles;
    A.a_rows = A.m >= 128 ? 128 : (A.m + 7) / 8 * 8;
    const int b_box = gated ? (wide ? 128 : cut.bn / 2) : cut.bn / cut.group;
    A.stage_tx = (uint32_t)(cut.group * ((A.a_mn ? kABytes : A.a_rows * 128) + cut.bn / cut.group * 128));
    product_waits(&A.tries, &A.starve);
    ProductMaps M;
    memset(&M, 0, sizeof M);
    const int na = pairs > A.jobs ? pairs : A.jobs, nb = gated ? 2 : pairs;
    for (int i = 0; i < na; ++i)
        if (!operand_map(encode, &M.a[i], a[i], dtype, A.a_mn ? 64 : A.a_rows)) return cudaErrorInvalidValue;
    for (int i = 0; i < nb; ++i)
        if (!operand_map(encode, &M.b[i], b[i], dtype, A.b_mn ? 64 : b_box)) return cudaErrorInvalidValue;
    const bool bf = dtype == XSM_BF16;
    if (wide) return bf ? start_epi<2, 256, bf16>(epi, M, A, st) : start_epi<2, 256, __half>(epi, M, A, st);
    return bf ? start_epi<1, 64, bf16>(epi, M, A, st) : start_epi<1, 64, __half>(epi, M, A, st);
}

cudaError_t launch_amax_rows(const void *x, int dtype, long long rows, long long cols, long long ld, float *amax, cudaStream_t st) {
    if (dtype == XSM_BF16) return launch_early(amax_rows_kernel<bf16>, dim3(kAmaxBlocks), dim3(256), 0, st, (const bf16 *)x, rows, (int)cols, ld, amax);
    return launch_early(amax_rows_kernel<__half>, dim3(kAmaxBlocks), dim3(256), 0, st, (const __half *)x, rows, (int)cols, ld, amax);
}
cudaError_t launch_amax_pairs(const float *g, long long g_ld, const float *h, long long h_ld, int rows, float by, float *amax, cudaStream_t st) {
    return launch_early(amax_pairs_kernel, dim3(kAmaxBlocks), dim3(32), 0, st, g, g_ld, h, h_ld, rows, by, amax);
}

cudaError_t launch_join(const ProductArgs &A, int dtype, cudaStream_t st) {
    JoinArgs J;
    J.partial = A.partial; J.amax = A.amax;
    J.out[0] = A.out[0]; J.out[1] = A.out[1];
    J.out_ld = A.out_ld; J.all = (long long)A.m * (A.n / 4);
    J.m = A.m; J.n = A.n; J.splits = A.splits; J.amax_to = A.amax_to;
    const long long blocks = (J.all + 255) / 256, most = (long long)product_sms() * 8;
    const dim3 grid((unsigned)(blocks < most ? blocks : most), (unsigned)A.jobs);
    if (dtype == XSM_BF16) return launch_early(join_kernel<bf16>, grid, dim3(256), 0, st, J);
    return launch_early(join_kernel<__half>, grid, dim3(256), 0, st, J);
}

}  // namespace xsm

xsm_status xsm_debug_product_waits(uint32_t tries, int starve) {
    xsm::g_tries.store(tries ? tries : xsm::kMbarSpinLimit, std::memory_order_relaxed);
    xsm::g_starve.store(starve != 0, std::memory_order_relaxed);
    return XSM_OK;
}
