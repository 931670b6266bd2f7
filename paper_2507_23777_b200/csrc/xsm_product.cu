// The matrix product of the operators on a caller's own activations and weights: 16-bit operands, fp32 sums, tcgen05.
//
// One persistent kernel.  A warp fetches blocks of 64 along the summed axis of both operands by TMA into a ring, a warp issues the products,
// eight warps work on finished tiles out of tensor memory while the products of the next one run (two accumulators).  Operands may lie either
// way: rows along the summed axis (boxes of 64 rows of 64 elements, "MN-major") or across it ("K-major"); nothing is transposed in memory.
//
// What bounds it.  Many rows, two CTAs a tile of 256 x 256: the tensor cores.  8192 x 32003 x 2048 takes 983,000 cycles of 901,000 that the products alone take in their
// 55 rounds of 74 tiles, 660 us at the 1.49 GHz that the power limit leaves: 1.63 PFLOP/s.  Summed axes below some 800 would be bound by what is done with a tile
// (4,000 cycles; act(gate) up 2,650) where these are not the products' 4 cycles a step.  A launch's first products come 3,400 cycles after its beginning, its end 6,000
// after its last products.  Few rows: the bytes of the weights (96 x 131071 x 1024: 49 us, 41 at the copy rate), very few a chain (5 x 4096 x 1024: 7.5 us: 2,000 cycles
// to the first copy, 3,700 for the bytes, 1,600 for the tile, then the last CTA's sums).
#include "xsm_product.cuh"

#include <string.h>

#include <atomic>
#include <type_traits>

namespace xsm {

constexpr int kEpiWarps = 8;
constexpr int kProductThreads = 64 + 32 * kEpiWarps;
constexpr int kABytes = 128 * 128;              // of a stage and a CTA: 128 rows of A, 64 elements of the summed axis
constexpr int kRingBytes = 192 * 1024;
constexpr int kMaxStages = 24;

// ------------------------------------------------------------------------------------------- instructions

// Descriptor of an operand tile with the 128-byte swizzle.  K-major: rows of 64 elements, groups of 8 rows 1024 bytes apart.  MN-major: rows of
// 64 elements across the summed axis, groups of 8 steps of it 1024 bytes apart, the next 64 elements `next` bytes (a box of 8 KB, or two) further.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool mn, uint32_t next = 8192) {
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)(mn ? next >> 4 : 1) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
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
template <int CG> __device__ __forceinline__ void tma_3d(uint32_t dst, const void *map, int x, int y, int z, uint32_t bar) {
    if constexpr (CG == 1)
        tma_box(dst, map, x, y, z, bar);
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];"
                     :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
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

__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// act(g) and its derivative.  gelu: g Phi(g), Phi by the rational approximation 7.1.26 of Abramowitz and Stegun (erfc(x) = t p(t) exp(-x^2), t = 1 / (1 + 0.3275911 x); off by
// 1.5e-7 at most, and by less where the exponential is small), whose exponential is the derivative's too.
template <int KIND> __device__ __forceinline__ void activate(float g, float &a, float &da) {
    if constexpr (KIND == ACT_SILU) {
        const float s = rcp(1.f + ex2(-g * kLog2e));
        a = g * s;
        da = fmaf(a, 1.f - s, s);
    } else {
        const float e = ex2(-0.5f * kLog2e * g * g), t = rcp(fmaf(0.3275911f * 0.70710678f, fabsf(g), 1.f));
        const float q = 0.5f * e * t * fmaf(fmaf(fmaf(fmaf(1.061405429f, t, -1.453152027f), t, 1.421413741f), t, -0.284496736f), t, 0.254829592f);
        const float c = g < 0.f ? q : 1.f - q;
        a = g * c;
        da = fmaf(0.39894228f * g, e, c);
    }
}

// Power of two that takes `most` to [2^to, 2^(to + 1)); 1 where there is nothing.
__device__ __forceinline__ float scale_for(float most, int to) {
    if (!(most > 0.f)) return 1.f;
    int e = (int)(__float_as_uint(most) >> 23) - 127;
    e = max(-100, min(100, to - e));
    return __uint_as_float((unsigned)(e + 127) << 23);
}

// the largest of kAmaxBlocks numbers
__device__ __forceinline__ float most_of(const float *amax) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < kAmaxBlocks; i += 32) m = fmaxf(m, amax[i + (threadIdx.x & 31)]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}
constexpr int kScaleTo = 13;        // the largest gradient that may be is taken to [2^13, 2^14)

// What the gradients by a row's logits may be: 2|g| + |g_lse| over T, g where there is a token, both where there is an lse; infinities and NaN: nothing.
__device__ __forceinline__ float row_bound(const ProductArgs &A, long long r) {
    const long long t = A.token_bytes == 8 ? reinterpret_cast<const long long *>(A.tokens)[r * A.token_ld] : (long long)reinterpret_cast<const int *>(A.tokens)[r * A.token_ld];
    const float lse = A.lse[r], g = A.g ? A.g[r * A.g_ld] : 0.f, h = A.g_lse ? A.g_lse[r * A.g_lse_ld] : 0.f;
    const float v = (2.f * (t >= 0 && t < A.vocab ? fabsf(g) : 0.f) + fabsf(h)) * A.inv_t;
    return lse > -INFINITY && v < INFINITY ? v : 0.f;
}
// ... of all rows at most, looked for by the warps of finished tiles while their first products run
__device__ __forceinline__ float most_of_rows(const ProductArgs &A, int w, int lane) {
    __shared__ float most[kEpiWarps];
    float m = 0.f;
    const int rows = A.part[0].m;
#pragma unroll 4
    for (long long r = w * 32 + lane; r < rows; r += 32 * kEpiWarps) m = fmaxf(m, row_bound(A, r));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) most[w] = m;
    bar_sync<32 * kEpiWarps>(1);
#pragma unroll
    for (int i = 0; i < kEpiWarps; ++i) m = fmaxf(m, most[i]);
    return m;
}
// A row's own power of two.  Rows down to 2^-12 of the largest have the one for all: fp16's smallest number is off by 2^-26 of their bound at most.  Smaller ones, which would lose bits to
// it, are taken to 2^-12 of the largest too, by up to 2^14; the row of the weights' gradients' other operand is as much smaller, and its elements off by up to 2^-11 (of rows below 2^-26
// of the largest).  Larger powers would cost these sums what they give the others.
__device__ __forceinline__ float row_scale(float bound, float all) { return bound > 0.f ? fminf(fmaxf(scale_for(bound, kScaleTo) * 0x1p-12f, all), all * 0x1p14f) : all; }
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b) {
    T p[2] = {rounded<T>(a), rounded<T>(b)};
    uint32_t r;
    memcpy(&r, p, 4);
    return r;
}
// A.h's rows, scaled by the power of all over their own (own(row)), to A.h_out: by the same warps
template <typename T, typename F> __device__ __forceinline__ void scale_rows(const ProductArgs &A, float all, F own, int w, int lane) {
    for (long long r = (long long)blockIdx.x * kEpiWarps + w; r < A.part[0].m; r += (long long)gridDim.x * kEpiWarps) {
        const float f = all / own(r);
        const uint4 *from = reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(A.h) + r * A.h_ld);
        uint4 *to = reinterpret_cast<uint4 *>(reinterpret_cast<T *>(A.h_out) + r * A.h_out_ld);
#pragma unroll 4
        for (int i = lane; i < A.d / 8; i += 32) {
            const uint4 u = from[i];
            T e[8];
            memcpy(e, &u, 16);
            to[i] = make_uint4(pack2<T>(to_f(e[0]) * f, to_f(e[1]) * f), pack2<T>(to_f(e[2]) * f, to_f(e[3]) * f), pack2<T>(to_f(e[4]) * f, to_f(e[5]) * f), pack2<T>(to_f(e[6]) * f, to_f(e[7]) * f));
        }
    }
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

// The same twice: numbers rounded to T, and, `low` elements further (0: not), what the rounding left.
template <typename T, int N> __device__ __forceinline__ void store_both(T *row, long long low, int col, int n, const float (&x)[N]) {
    store_row(row, col, n, true, x);
    if (low == 0) return;
    float rest[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float r = x[i] - to_f(rounded<T>(x[i]));
        rest[i] = fabsf(r) < INFINITY ? r : 0.f;
    }
    store_row(row + low, col, n, true, rest);
}

// ----------------------------------------------------------------------------------------------------- tiles

// Tiles in groups of `group_m` tiles of rows; in a group the rows first, then the columns: the tiles that run at a time then share both operands'
// panels (63 x 8 tiles of 8192 steps rows first: every column of tiles fetched all of A again from memory).
struct Tile { int m, n, split, job, k0, k1, at; };        // at: number of the tile of its job's and split's kind
__device__ __forceinline__ Tile tile_of(const ProductPart &P, unsigned t) {
    Tile r;
    t -= (unsigned)P.first;
    const unsigned z = P.by_plane.of(t);
    t -= z * P.by_plane.d;
    r.job = (int)P.by_splits.of(z);
    r.split = (int)(z - (unsigned)r.job * P.by_splits.d);
    r.at = (int)(t + (unsigned)r.job * P.by_plane.d);
    const unsigned g = P.by_group.of(t);
    t -= g * P.by_group.d;
    const bool last = (int)(g + 1) * P.group_m > P.tiles_m;
    r.n = (int)(last ? P.by_last_rows.of(t) : P.by_rows.of(t));
    r.m = (int)(g * (unsigned)P.group_m + t - (unsigned)r.n * (last ? P.by_last_rows.d : P.by_rows.d));
    r.k0 = r.split * P.kb_each + min(r.split, P.kb_more);
    r.k1 = r.k0 + P.kb_each + (r.split < P.kb_more);
    return r;
}

// ---------------------------------------------------------------------------------------- rows in shared memory

// A warp's 32 rows of 128 bytes (16-byte pieces permuted as TMA's 128-byte swizzle does) on their way between a thread's own row and memory.
__device__ __forceinline__ uint32_t piece_at(uint32_t buf, int row, int piece) { return buf + (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4)); }
__device__ __forceinline__ void sts128(uint32_t addr, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
// the buffer's last store has been read
__device__ __forceinline__ void rows_free(int lane) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
}
__device__ __forceinline__ void rows_store(const void *map, uint32_t buf, int x, int y, int z, bool some, int lane) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (some && lane == 0) {
        asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" :: "l"(map), "r"(x), "r"(y), "r"(z), "r"(buf) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}
// the same by the warp itself, for rows that are not aligned: elements [col, n) of rows [row0, m)
template <typename T> __device__ __forceinline__ void rows_copy_out(T *out, long long ld, int row0, int m, int col, int n, uint32_t buf, int lane) {
    __syncwarp();
    const bool has0 = col + 2 * lane < n, has1 = col + 2 * lane + 1 < n;
#pragma unroll 4
    for (int r = 0; r < 32; ++r) {
        if (row0 + r >= m) break;
        uint32_t v;
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(piece_at(buf, r, lane >> 2) + (uint32_t)(lane & 3) * 4) : "memory");
        T e[2];
        memcpy(e, &v, 4);
        T *p = out + (row0 + r) * ld + col + 2 * lane;
        if (has0) p[0] = e[0];
        if (has1) p[1] = e[1];
    }
    __syncwarp();
}
// rows [row0, m), elements [col, n) of a matrix into the buffer, zeros elsewhere; to be waited for with rows_landed
template <typename T> __device__ __forceinline__ void rows_fetch(const T *x, long long ld, int row0, int m, int col, int n, bool aligned, uint32_t buf, int lane) {
    if (aligned) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = i * 4 + (lane >> 3), c = lane & 7, left = (n - col - c * 8) * 2, bytes = row0 + r < m ? max(0, min(16, left)) : 0;
            const T *p = bytes ? x + (row0 + r) * ld + col + c * 8 : x;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(piece_at(buf, r, c)), "l"(p), "r"(bytes) : "memory");
        }
    } else {
        const bool has0 = col + 2 * lane < n, has1 = col + 2 * lane + 1 < n;
#pragma unroll 8
        for (int r = 0; r < 32; ++r) {
            T e[2] = {rounded<T>(0.f), rounded<T>(0.f)};
            const T *p = x + (row0 + r) * ld + col + 2 * lane;
            if (row0 + r < m && has0) e[0] = p[0];
            if (row0 + r < m && has1) e[1] = p[1];
            uint32_t v;
            memcpy(&v, e, 4);
            asm volatile("st.shared.b32 [%0], %1;" :: "r"(piece_at(buf, r, lane >> 2) + (uint32_t)(lane & 3) * 4), "r"(v) : "memory");
        }
    }
}
__device__ __forceinline__ void rows_landed() {
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
}
// thirty-two numbers rounded to T, or sixteen bytes' worth of fp32 each, into a row: pieces from `first` on
template <typename T> __device__ __forceinline__ void put_row(uint32_t buf, int row, int first, const float (&x)[32]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        sts128(piece_at(buf, row, first + i), make_uint4(pack2<T>(x[8 * i], x[8 * i + 1]), pack2<T>(x[8 * i + 2], x[8 * i + 3]), pack2<T>(x[8 * i + 4], x[8 * i + 5]), pack2<T>(x[8 * i + 6], x[8 * i + 7])));
}

// -------------------------------------------------------------------------------------------------- kernel

template <int CG, int BN, int EPI, typename T>
__global__ void __launch_bounds__(kProductThreads, 1) product_kernel(const __grid_constant__ ProductMaps M, const __grid_constant__ ProductArgs A) {
    constexpr int TM = 128 * CG;
    constexpr bool kGated = EPI == PR_GATED || EPI == PR_GATED_GRAD, kOut = EPI == PR_OUT, kRounds = (EPI == PR_STATS || EPI == PR_DLOGITS) && CG == 1;
    extern __shared__ char smem_raw[];
    __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages], sums_full[2], sums_empty[2], last;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int dead;           // a wait of this CTA has run out
    __shared__ int fills;                   // stages that were asked for
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0, first = blockIdx.x / CG, step = gridDim.x / CG;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    chain_go();
    if (warp == 1) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&tmem_slot)), "n"(2 * BN) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&tmem_slot)), "n"(2 * BN) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    } else if (warp == 0) {        // (a barrier each: one thread takes 30 cycles for each of them)
        if (lane < A.stages) { mbar_init(smem_u32(&full[lane]), 1u); mbar_init(smem_u32(&empty[lane]), 1u); }
        if (lane < 2) { mbar_init(smem_u32(&sums_full[lane]), 1u); mbar_init(smem_u32(&sums_empty[lane]), kEpiWarps * CG); }
        if (lane == 2) mbar_init(smem_u32(&last), 1u);
        if (lane == 3) { dead = 0; fills = 0; }
        mbar_init_fence();
    }
    tcgen05_before_sync();
    __syncthreads();
    if constexpr (CG == 2) { cluster_arrive(); cluster_wait(); }
    tcgen05_after_sync();
    const uint32_t tmem = tmem_slot;
    // (what the first tile needs is worked out, and the operands' descriptions are on their way, before what other kernels write is waited for)
    if (warp != 0) chain_wait();

    // false: the limit ran out, here or elsewhere in the CTA; the results are void
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (mbar_try_wait(bar, parity)) return true;
        for (unsigned i = 0; i < A.tries; ++i) {
            if (mbar_try_wait(bar, parity)) return true;
            if ((i & 63u) == 63u && dead) return false;
        }
        dead = 1;
        atomicExch(A.status, XSM_STATUS_TIMEOUT);
        return false;
    };
    auto wait_warp = [&](uint32_t bar, uint32_t parity) {        // (all lanes or none)
        return __all_sync(0xffffffffu, mbar_try_wait(bar, parity)) || __all_sync(0xffffffffu, wait(bar, parity));
    };
    auto part_of = [&](int t) -> const ProductPart & { return A.part[kOut && t >= A.part[1].first]; };
    const uint32_t full0 = smem_u32(full), empty0 = smem_u32(empty), sums_full0 = smem_u32(sums_full), sums_empty0 = smem_u32(sums_empty);

    // The two loops below run once for 64 steps of the summed axis, 512 cycles of the tensor cores: what does not change stands outside, and nothing
    // branches that need not.  (With divisions, an operand's orientation and the barriers' addresses worked out within, 550 cycles a turn.)
    if (warp == 0) {
        if (elect_one() && !A.starve) {
            const uint32_t full_at = CG == 2 ? map_rank(full0, 0) : full0;
            int n = 0, s = 0;
            uint32_t par = 1u, sa = ring;
            const uint32_t a_next = kOut && A.low ? 16384 : 8192;        // (A's rows and what their rounding left come by one copy, one behind the other)
            bool ok = true;
            for (int t = first; ok && t < A.tiles; t += step) {
                const ProductPart &P = part_of(t);
                const Tile w = tile_of(P, (unsigned)t);
                const int m0 = w.m * TM + rank * 128, n0 = kGated ? w.n * (BN / 2) : w.n * BN + rank * (BN / CG);
                const int second = kOut && w.k0 >= P.kb0, rows_a = kOut && P.rows_a;
                const uint32_t tx = P.stage_tx;
                const CUtensorMap *ma = &M.a[kOut ? P.map_a + second + w.job : 0], *mb = &M.b[kOut ? P.map_b + second : kGated && CG == 2 ? rank : 0];
                // a stage of one block: columns `at`; of several: blocks of 64 columns from z on, what is left of the rows in a stage of its own
                const bool many = !kOut && CG == 1 && A.chunks > 1;
                int at = (w.k0 - (second ? P.kb0 : 0)) * 64, z = 0;
                if (t == first) {
                    asm volatile("prefetch.tensormap [%0];" :: "l"(ma) : "memory");
                    asm volatile("prefetch.tensormap [%0];" :: "l"(mb) : "memory");
                    chain_wait();
                }
                if (many) at = 0;
                for (int k = w.k0; k < w.k1; ++k) {
                    if (!(ok = wait(empty0 + 8u * (uint32_t)s, par))) break;
                    if (many && A.tail && k + 1 == w.k1) { ++ma; mb += 2; z = 0; }
                    const uint32_t f = full_at + 8u * (uint32_t)s, sb = sa + A.stage_b;
                    if (CG == 1 || rank == 0) mbar_arrive_expect_tx(full0 + 8u * (uint32_t)s, tx);
                    if (rows_a) {
                        tma_3d<CG>(sa, ma, m0, at, 0, f);
                        tma_3d<CG>(sa + a_next, ma, m0 + 64, at, 0, f);
                    } else {
                        tma_3d<CG>(sa, ma, at, m0, z, f);
                    }
                    if constexpr (kOut) {
#pragma unroll
                        for (int i = 0; i < BN / CG / 64; ++i) tma_3d<CG>(sb + i * 8192, mb, n0 + 64 * i, at, 0, f);
                    } else {
                        tma_3d<CG>(sb, mb, at, n0, z, f);
                        if constexpr (kGated && CG == 1) tma_3d<CG>(sb + (uint32_t)A.chunks * (BN / 2 * 128), mb + 1, at, n0, z, f);
                    }
                    ++n;
                    if (many) z += A.chunks;
                    else at += 64;
                    if (kOut && k + 1 == P.kb0) { at = 0; ++ma; ++mb; }
                    sa += A.stage;
                    if (++s == A.stages) { s = 0; par ^= 1u; sa = ring; }
                }
            }
            fills = n;
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            const bool leader = elect_one();
            constexpr uint32_t b_step = kOut ? 2048 >> 4 : 32 >> 4;
            const uint64_t db = operand_desc(ring + A.stage_b, kOut);
            const uint32_t stage = A.stage >> 4;
            const bool low = kOut && A.low != 0;
            bool ok = true;
            int s = 0, acc = 0;
            uint32_t par = 0u, acc_par = 1u, at = 0u;
            for (int t = first; ok && t < A.tiles; t += step) {
                const ProductPart &P = part_of(t);
                const Tile w = tile_of(P, (unsigned)t);
                const bool rows_a = kOut && P.rows_a;
                const uint32_t idesc = product_idesc<T>(128 * CG, kGated && CG == 1 ? BN / 2 : BN, rows_a, kOut), a_step = rows_a ? 2048 >> 4 : 32 >> 4, a_chunk = (uint32_t)P.a_rows * 128 >> 4;
                const uint64_t da = operand_desc(ring, rows_a, low ? 16384 : 8192);
                const uint32_t a_low = (rows_a ? 8192u : (uint32_t)P.a_rows * 128u) >> 4;
                if (!(ok = wait_warp(sums_empty0 + 8u * (uint32_t)acc, acc_par))) break;
                tcgen05_after_sync();
                uint32_t d = tmem + (uint32_t)(acc * BN), add = 0u;
                int left = kRounds ? A.round : 0;
                for (int k = w.k0; k < w.k1; ++k) {
                    if (!(ok = wait_warp(full0 + 8u * (uint32_t)s, par))) break;
                    tcgen05_after_sync();
                    if (leader) {
                        uint64_t a = da + at, b = db + at;
                        for (int c = 0;; ++c) {
                            if constexpr (kGated && CG == 1) {        // gate's columns and up's lie in boxes of their own
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    mma_f16<CG>(d, a + i * a_step, b + i * b_step, idesc, i > 0 ? 1u : add);
                                    mma_f16<CG>(d + BN / 2, a + i * a_step, b + (uint32_t)A.chunks * (BN / 2 * 128 >> 4) + i * b_step, idesc, i > 0 ? 1u : add);
                                }
                            } else {
#pragma unroll
                                for (int i = 0; i < 4; ++i) mma_f16<CG>(d, a + i * a_step, b + i * b_step, idesc, i > 0 ? 1u : add);
                                if (low) {
#pragma unroll
                                    for (int i = 0; i < 4; ++i) mma_f16<CG>(d, a + a_low + i * a_step, b + i * b_step, idesc, 1u);
                                }
                            }
                            if (CG == 2 || kOut || c + 1 == A.chunks) break;
                            a += a_chunk;
                            b += (kGated ? BN / 2 : BN) * 128 >> 4;
                            add = 1u;
                        }
                        commit<CG>(empty0 + 8u * (uint32_t)s);
                    }
                    __syncwarp();
                    add = 1u;
                    at += stage;
                    if (++s == A.stages) { s = 0; par ^= 1u; at = 0u; }
                    if constexpr (kRounds) {
                        if (--left == 0 && k + 1 < w.k1) {
                            if (leader) commit<CG>(sums_full0 + 8u * (uint32_t)acc);
                            __syncwarp();
                            if (++acc == 2) { acc = 0; acc_par ^= 1u; }
                            if (!(ok = wait_warp(sums_empty0 + 8u * (uint32_t)acc, acc_par))) break;
                            tcgen05_after_sync();
                            d = tmem + (uint32_t)(acc * BN);
                            add = 0u;
                            left = A.round;
                        }
                    }
                }
                if (!ok) break;
                if (leader) commit<CG>(sums_full0 + 8u * (uint32_t)acc);
                __syncwarp();
                if (++acc == 2) { acc = 0; acc_par ^= 1u; }
            }
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16), buf = ring + (uint32_t)(kRingBytes + (warp - 2) * 4096);
        constexpr bool kScaled = std::is_same<T, __half>::value && (EPI == PR_DLOGITS || EPI == PR_GATED_GRAD || kOut);
        float all = 1.f;
        [[maybe_unused]] float factor = 1.f;        // of the rows' bounds
        if constexpr (kScaled && kOut) all = *A.all_scale;
        if constexpr (kScaled && !kOut) {
            if constexpr (EPI == PR_GATED_GRAD) factor = most_of(A.amax + kAmaxBlocks);
            if constexpr (EPI == PR_DLOGITS) all = scale_for(A.look ? most_of_rows(A, warp - 2, lane) : most_of(A.amax), kScaleTo);
            else all = scale_for(most_of(A.amax) * factor, kScaleTo);
            if (blockIdx.x == 0 && tid == 64) *A.all_scale = all;
        }
        [[maybe_unused]] auto own_scale = [&](long long r) {
            if constexpr (EPI == PR_DLOGITS) return row_scale(row_bound(A, r), all);
            else return row_scale(A.bounds[r] * factor, all);
        };
        if constexpr (kScaled && !kOut) {
            if (A.h_out) scale_rows<T>(A, all, own_scale, warp - 2, lane);
        }
        float scale = 1.f;
        const float back = 1.f / all;
        int acc = 0;
        uint32_t acc_par = 0u;
        float mx = -INFINITY, sum = 0.f;        // PR_STATS
        auto release = [&] {        // the products may have the accumulator again
            tcgen05_before_sync();
            __syncwarp();
            if (lane == 0) {
                if constexpr (CG == 2) arrive_cluster(map_rank(smem_u32(&sums_empty[acc]), 0));
                else mbar_arrive(smem_u32(&sums_empty[acc]));
            }
            if (++acc == 2) { acc = 0; acc_par ^= 1u; }
        };
        for (int t = first; t < A.tiles; t += step) {
            const ProductPart &P = part_of(t);
            const Tile w = tile_of(P, (unsigned)t);
            const int row0 = w.m * TM + rank * 128 + quarter * 32, row = row0 + lane;
            const bool live = row < P.m;
            if constexpr (kScaled && EPI == PR_GATED_GRAD) {
                scale = live ? own_scale(row) : 0.f;
                if (live && w.n == 0 && half == 0) A.row_scale[row] = scale;
            }
            if constexpr (EPI == PR_GATED_GRAD && CG == 2) {
                rows_free(lane);
                rows_fetch(reinterpret_cast<const T *>(A.g_y), A.g_y_ld, row0, P.m, w.n * (BN / 2) + half * (BN / 4), P.n, (A.g_y_ld & 7) == 0 && ((uintptr_t)A.g_y & 15) == 0, buf, lane);
            }
            if (!wait_warp(sums_full0 + 8u * (uint32_t)acc, acc_par)) break;
            tcgen05_after_sync();
            const uint32_t sums = lanes + (uint32_t)(acc * BN);
            if constexpr (EPI == PR_GATED || EPI == PR_GATED_GRAD) {
                constexpr int N = BN / 4 < 32 ? BN / 4 : 32;
                const int col0 = w.n * (BN / 2) + half * (BN / 4);
                [[maybe_unused]] const bool whole = EPI == PR_GATED_GRAD && (A.g_y_ld & 7) == 0 && ((uintptr_t)A.g_y & 15) == 0;
                if constexpr (CG == 2 && EPI == PR_GATED) rows_free(lane);
                if constexpr (CG == 2 && EPI == PR_GATED_GRAD) rows_landed();
                uint32_t held[CG == 2 && EPI == PR_GATED_GRAD ? BN / 8 : 1];        // up's gradients, packed, until the buffer is free again
                auto columns = [&](auto kind) {
#pragma unroll
                    for (int c = 0; c < BN / 4; c += N) {
                        uint32_t vg[N], vu[N];
                        tmem_ld(vg, sums + (uint32_t)(half * (BN / 4) + c));
                        tmem_ld(vu, sums + (uint32_t)(BN / 2 + half * (BN / 4) + c));
                        [[maybe_unused]] const int col = col0 + c;
                        float x[N];
                        if constexpr (EPI == PR_GATED_GRAD) {
                            if constexpr (CG == 2) {
#pragma unroll
                                for (int i = 0; i < N; i += 8) {
                                    const uint4 u = lds128(piece_at(buf, lane, (c + i) / 8));
                                    T e[8];
                                    memcpy(e, &u, 16);
#pragma unroll
                                    for (int j = 0; j < 8; ++j) x[i + j] = to_f(e[j]) * scale;
                                }
                            } else {
                                const T *gy = reinterpret_cast<const T *>(A.g_y) + (long long)row * A.g_y_ld;
                                if (live && whole && col + N <= P.n) {
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
                                    for (int i = 0; i < N; ++i) x[i] = live && col + i < P.n ? to_f(gy[col + i]) * scale : 0.f;
                                }
                            }
                        }
                        tmem_wait_ld();
                        if constexpr (EPI == PR_GATED) {
#pragma unroll
                            for (int i = 0; i < N; ++i) {
                                float a, da;
                                activate<decltype(kind)::value>(__uint_as_float(vg[i]), a, da);
                                x[i] = a * __uint_as_float(vu[i]);
                            }
                            if constexpr (CG == 2) put_row<T>(buf, lane, c / 8, x);
                            else if (live) store_row(reinterpret_cast<T *>(A.out[0]) + (long long)row * A.out_ld, col, P.n, (A.out_ld & 7) == 0 && ((uintptr_t)A.out[0] & 15) == 0, x);
                        } else {
                            float y[N];
#pragma unroll
                            for (int i = 0; i < N; ++i) {
                                float a, da;
                                activate<decltype(kind)::value>(__uint_as_float(vg[i]), a, da);
                                y[i] = x[i] * a;
                                x[i] = x[i] * __uint_as_float(vu[i]) * da;
                            }
                            if constexpr (CG == 2) {
                                put_row<T>(buf, lane, c / 8, x);
#pragma unroll
                                for (int i = 0; i < N; i += 2) held[(c + i) / 2] = pack2<T>(y[i], y[i + 1]);
                            } else if (live) {        // (workspace rows of a multiple of eight elements: what lies behind the last column is nobody's)
                                const int n8 = (int)A.out_ld;
                                store_both(reinterpret_cast<T *>(A.out[0]) + (long long)row * A.out_ld, A.low, col, n8, x);
                                store_both(reinterpret_cast<T *>(A.out[1]) + (long long)row * A.out_ld, A.low, col, n8, y);
                            }
                        }
                    }
                };
                if (A.activation == ACT_SILU) columns(std::integral_constant<int, ACT_SILU>());
                else columns(std::integral_constant<int, ACT_GELU>());
                if constexpr (CG == 2) {
                    if (A.tma_out) rows_store(&M.out[0], buf, col0, row0, 0, row0 < P.m && col0 < P.n, lane);
                    else rows_copy_out(reinterpret_cast<T *>(A.out[0]), A.out_ld, row0, P.m, col0, P.n, buf, lane);
                    if constexpr (EPI == PR_GATED_GRAD) {
                        rows_free(lane);
#pragma unroll
                        for (int i = 0; i < BN / 32; ++i) sts128(piece_at(buf, lane, i), make_uint4(held[4 * i], held[4 * i + 1], held[4 * i + 2], held[4 * i + 3]));
                        rows_store(&M.out[1], buf, col0, row0, 0, row0 < P.m && col0 < P.n, lane);
                    }
                }
            } else {
                constexpr int N = BN / 2 < 32 ? BN / 2 : 32;
                const int col0 = w.n * BN + half * (BN / 2);
                long long token = -1;
                float g = 0.f, gp = 0.f, gl = 0.f, lse2 = 0.f;
                if (EPI == PR_STATS || EPI == PR_DLOGITS) {
                    if (live) {
                        token = A.token_bytes == 8 ? reinterpret_cast<const long long *>(A.tokens)[row * A.token_ld] : (long long)reinterpret_cast<const int *>(A.tokens)[row * A.token_ld];
                        const bool there = token >= 0 && token < A.vocab;
                        token = there ? token - A.vocab0 : -1;
                        if constexpr (EPI == PR_DLOGITS) {
                            const float lse = A.lse[row];
                            if constexpr (kScaled) {
                                scale = own_scale(row);
                                if (w.n == 0 && half == 0) A.row_scale[row] = scale;
                            }
                            g = A.g && there ? A.g[row * A.g_ld] : 0.f;
                            gl = A.g_lse ? A.g_lse[row * A.g_lse_ld] : 0.f;
                            gp = g - gl;
                            g *= A.inv_t * scale;
                            gl *= A.inv_t * scale;
                            gp *= A.inv_t * scale;
                            lse2 = lse * kLog2e;
                            if (lse == -INFINITY) g = gl = gp = lse2 = 0.f;
                        }
                    }
                }
                if constexpr (kOut) {
                    constexpr int kPieces = BN / 64, kTile = CG * kEpiWarps * kPieces * 1024;        // of 32 columns a warp; fp32 sums of a tile
                    // Sums in memory lie as the threads hold them: piece by piece, four columns of the 32 rows side by side.
                    auto place = [&](float *p, long long tile) { return p + tile * kTile + ((rank * kEpiWarps + warp - 2) * kPieces) * 1024 + lane * 4; };
                    const int pieces = min(kPieces, (P.n - col0 + 31) / 32);        // (that have columns)
                    bool mine = row0 < P.m;
                    if (P.splits > 1 && mine) {
                        // Every split leaves its sums; whoever comes last of a tile's and a warp's adds them up, in the order of the splits.
                        float *p = place(P.partial, (long long)w.at * P.splits + w.split);
#pragma unroll 1
                        for (int c = 0; c < pieces; ++c) {
                            uint32_t v[32];
                            tmem_ld(v, sums + (uint32_t)(half * (BN / 2) + c * 32));
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                __stcg(reinterpret_cast<uint4 *>(p + c * 1024 + i * 128), make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]));
                        }
                        if (P.apart) {
                            mine = false;
                        } else {
                            __threadfence();
                            __syncwarp();
                            unsigned before = 0;
                            if (lane == 0) before = atomicInc(A.counter + P.counters + (unsigned)((w.at * CG + rank) * kEpiWarps + warp - 2), (unsigned)P.splits - 1u);
                            mine = __shfl_sync(0xffffffffu, before, 0) == (unsigned)P.splits - 1u;
                            __threadfence();
                        }
                    }
                    if (mine) {
#pragma unroll 1
                        for (int c = 0; c < pieces; ++c) {
                            const int col = col0 + c * 32;
                            float x[32];
                            if (P.splits > 1) {
                                const float *p = place(P.partial, (long long)w.at * P.splits) + c * 1024;
#pragma unroll
                                for (int i = 0; i < 32; ++i) x[i] = 0.f;
                                // (two splits' on their way at a time: their latency is most of this)
#pragma unroll 1
                                for (int s = 0; s < P.splits; s += 2, p += 2 * kTile) {
                                    const bool two = s + 1 < P.splits;
                                    float4 q[8], r[8];
#pragma unroll
                                    for (int i = 0; i < 8; ++i) {
                                        q[i] = __ldcg(reinterpret_cast<const float4 *>(p + i * 128));
                                        r[i] = two ? __ldcg(reinterpret_cast<const float4 *>(p + kTile + i * 128)) : make_float4(0.f, 0.f, 0.f, 0.f);
                                    }
#pragma unroll
                                    for (int i = 0; i < 8; ++i) {
                                        x[4 * i] = x[4 * i] + q[i].x + r[i].x;
                                        x[4 * i + 1] = x[4 * i + 1] + q[i].y + r[i].y;
                                        x[4 * i + 2] = x[4 * i + 2] + q[i].z + r[i].z;
                                        x[4 * i + 3] = x[4 * i + 3] + q[i].w + r[i].w;
                                    }
                                }
                            } else {
                                uint32_t v[32];
                                tmem_ld(v, sums + (uint32_t)(half * (BN / 2) + c * 32));
                                tmem_wait_ld();
#pragma unroll
                                for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(v[i]);
                            }
                            if (P.sums) {
                                float *p = place(P.sums, w.at) + c * 1024;
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    float4 *q = reinterpret_cast<float4 *>(p + i * 128);
                                    if (P.go_on) {
                                        const float4 o = *q;
                                        x[4 * i] += o.x; x[4 * i + 1] += o.y; x[4 * i + 2] += o.z; x[4 * i + 3] += o.w;
                                    }
                                    if (!P.end) *q = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                                }
                                if (!P.end) continue;
                            }
                            float by = back;
                            if constexpr (kScaled) {
                                if (!P.rows_a) by = live ? 1.f / A.row_scale[row] : 0.f;
                            }
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[i] *= by;
                            if ((c & 1) == 0) rows_free(lane);
                            put_row<T>(buf, lane, (c & 1) * 4, x);
                            if ((c & 1) || c + 1 == pieces) rows_store(&M.out[P.map_out + w.job], buf, col - (c & 1) * 32, row0, 0, true, lane);
                        }
                    }
                } else {
                    // The tensor core cuts its sums off where they are added to: of few rows, where there is time for it, no more than 512 steps are added up there, and these here.
                    // (13 x 24000 x 1824: lse off by 1.2e-6 of itself otherwise; and the gradient's probabilities are those of the same sums.)
                    [[maybe_unused]] float z[kRounds ? BN / 2 : 1];
                    const bool more_z = kRounds && w.k1 - w.k0 > A.round;
                    if constexpr (kRounds) {
                        bool ok = true;
                        for (int k = w.k0, left = w.k1 - w.k0; left > A.round; k += A.round, left -= A.round) {
#pragma unroll
                            for (int c = 0; c < BN / 2; c += N) {
                                uint32_t v[N];
                                tmem_ld(v, lanes + (uint32_t)(acc * BN + half * (BN / 2) + c));
                                tmem_wait_ld();
#pragma unroll
                                for (int i = 0; i < N; ++i) z[c + i] = (k > w.k0 ? z[c + i] : 0.f) + __uint_as_float(v[i]);
                            }
                            release();
                            if (!(ok = wait_warp(sums_full0 + 8u * (uint32_t)acc, acc_par))) break;
                            tcgen05_after_sync();
                        }
                        if (!ok) break;
                    }
#pragma unroll(kRounds ? BN / 2 / N : 1)
                    for (int c = 0; c < BN / 2; c += N) {
                        uint32_t v[N];
                        tmem_ld(v, lanes + (uint32_t)(acc * BN + half * (BN / 2) + c));
                        const int col = col0 + c;
                        if (CG == 2 && EPI == PR_DLOGITS && (c & 32) == 0) rows_free(lane);
                        tmem_wait_ld();
                        if constexpr (kRounds) {
                            if (more_z) {
#pragma unroll
                                for (int i = 0; i < N; ++i) v[i] = __float_as_uint(z[c + i] + __uint_as_float(v[i]));
                            }
                        }
                        if constexpr (EPI == PR_STATS) {
                            if (col + N > P.n) {
#pragma unroll
                                for (int i = 0; i < N; ++i)
                                    if (col + i >= P.n) v[i] = 0xff800000u;        // -infinity
                            }
                            float top = __uint_as_float(v[0]);
#pragma unroll
                            for (int i = 1; i < N; ++i) top = fmaxf(top, __uint_as_float(v[i]));
                            if (token >= col && token < col + N) {
#pragma unroll
                                for (int i = 0; i < N; ++i)
                                    if (token == col + i) A.token_z[row] = __uint_as_float(v[i]);
                            }
                            const float was = mx;
                            mx = fmaxf(mx, top * A.c);
                            const float base = mx == -INFINITY ? 0.f : mx;
                            float more[2] = {0.f, 0.f};
#pragma unroll
                            for (int i = 0; i < N; ++i) more[i & 1] += ex2(fmaf(__uint_as_float(v[i]), A.c, -base));
                            sum = fmaf(sum, ex2(was - base), more[0] + more[1]);
                        } else {
                            float x[N];
#pragma unroll
                            for (int i = 0; i < N; ++i) x[i] = -gp * ex2(fmaf(__uint_as_float(v[i]), A.c, -lse2));
                            if (token >= col && token < col + N) {
                                // g (1 - p) + g_lse p; 1 - p from the log probability: next to 1, z - lse has none of it left
                                const float lp = A.given ? A.given[row] : 0.f, own = fmaf(gl, expf(lp), -g * expm1f(lp));
#pragma unroll
                                for (int i = 0; i < N; ++i)
                                    if (token == col + i) x[i] = A.given ? own : x[i] + g;
                            }
                            if constexpr (CG == 2) {
                                put_row<T>(buf, lane, (c & 32) / 8, x);
                                if (c & 32) rows_store(&M.out[0], buf, col - 32, row0, 0, row0 < P.m && col - 32 < P.n, lane);
                            } else if (live) {
                                store_both(reinterpret_cast<T *>(A.out[0]) + (long long)row * A.out_ld, A.low, col, (int)A.out_ld, x);
                            }
                        }
                    }
                }
                if constexpr (EPI == PR_STATS) {
                    if (!A.carry) {
                        if (live) A.parts[(long long)(2 * w.n + half) * P.m + row] = make_float2(mx, sum);
                        mx = -INFINITY;
                        sum = 0.f;
                    } else if (t + step >= A.tiles && live) {
                        if (A.counter) A.parts[(long long)row * 2 * gridDim.x + 2 * first + half] = make_float2(mx, sum);
                        else A.parts[(long long)(2 * first + half) * P.m + row] = make_float2(mx, sum);
                    }
                }
            }
            release();
        }
        if ((CG == 2 || kOut) && EPI != PR_STATS && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
    }
    tcgen05_before_sync();
    __syncthreads();
    if (dead) {
        // What was asked for lands before the CTA ends, and products under way end before the tensor memory goes back, also where nobody waits for them any more.
        // (Both CTAs' copies count on this one's barriers; the other's last wait has run out long after its last copy.)
        if (tid == 0 && rank == 0)
            for (int i = max(0, fills - A.stages); i < fills; ++i)
                for (unsigned n = 0; n < A.tries && !mbar_try_wait(smem_u32(&full[i % A.stages]), (uint32_t)(i / A.stages) & 1u); ++n);
        if (warp == 1 && rank == 0) {
            if (elect_one()) commit_here<CG>(smem_u32(&last));
            __syncwarp();
            for (unsigned n = 0; n < A.tries && !mbar_try_wait(smem_u32(&last), 0u); ++n);
        }
        __syncthreads();
    }
    if constexpr (EPI == PR_STATS && CG == 1) {
        if (A.counter) {
            __shared__ int last_of_all;
            if (tid == 0) {
                __threadfence();
                last_of_all = atomicInc(A.counter, gridDim.x - 1) == gridDim.x - 1;        // (back to zero with the last)
                __threadfence();
            }
            __syncthreads();
            if (last_of_all)
                for (int row = warp; row < A.part[0].m; row += kProductThreads / 32) {
                    RowSums r;
#pragma unroll 4
                    for (int i = lane; i < 2 * (int)gridDim.x; i += 32) r.take(__ldcg(&A.parts[(long long)row * 2 * gridDim.x + i]));
                    r.across_lanes();
                    if (lane == 0) r.finish(A.tokens, A.token_ld, A.token_bytes, A.vocab, row, A.token_z, A.c, A.to_lse, A.logprob, A.lse_out, A.kept);
                }
        }
    }
    if constexpr (CG == 2) { cluster_arrive(); cluster_wait(); }        // (nobody leaves while the other CTA's barriers and memory are still in use)
    if (warp == 1) {
        tcgen05_after_sync();
        if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(2 * BN) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(2 * BN) : "memory");
    }
}

// -------------------------------------------------------------------------------------------- small kernels

// The largest of n elements, or the sum of their squares (kSquares), by a warp, each lane's own.  Elements up to the first 16-byte boundary and behind the last one by one; eight loads of a
// lane on their way, which the compiler would put beside their uses otherwise (64 rows, 8192 of 2048: 38 us, 19 so; 2047 x 2051 of 768 12.5 and 8.8).
template <bool kSquares, bool kFinite> __device__ __forceinline__ float row_size_of(const __half *p, long long n, int lane) {
    float m = 0.f;
    auto take = [&](float v) {
        if (kFinite && !(fabsf(v) < INFINITY)) v = 0.f;
        m = kSquares ? fmaf(v, v, m) : fmaxf(m, fabsf(v));
    };
    const long long before = min(n, (long long)((16 - ((uintptr_t)p & 15)) / 2 & 7)), pieces = (n - before) / 8, behind = before + pieces * 8;
    const float first = lane < before ? to_f(p[lane]) : 0.f, last = lane < n - behind ? to_f(p[behind + lane]) : 0.f;
    const uint4 *body = reinterpret_cast<const uint4 *>(p + before);
    for (long long i = lane; i < pieces; i += 256) {
        uint4 u[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u[k].x), "=r"(u[k].y), "=r"(u[k].z), "=r"(u[k].w) : "l"(body + (i + 32 * k < pieces ? i + 32 * k : i)));
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (i + 32 * k >= pieces) u[k] = make_uint4(0u, 0u, 0u, 0u);
            __half2 e[4];
            memcpy(e, &u[k], 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = __half22float2(e[j]);
                take(f.x);
                take(f.y);
            }
        }
    }
    take(first);
    take(last);
    return m;
}
// ... infinities and NaN apart
template <bool kSquares> __device__ __forceinline__ float row_size(const __half *p, long long n, int lane) {
    auto all = [](float m) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = kSquares ? m + __shfl_xor_sync(0xffffffffu, m, o) : fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        return m;
    };
    const float m = all(row_size_of<kSquares, false>(p, n, lane));
    return m < INFINITY ? m : all(row_size_of<kSquares, true>(p, n, lane));
}
// GatedSizes: a warp a row, x's with g's, then the weights'.  The weights' bytes bound it where rows are few: 64 rows, 8192 of 2048 61 -> 78 us with it, 2047 x 2051 of 768 53 -> 57.
constexpr int kSizeThreads = 512;
__global__ void __launch_bounds__(kSizeThreads, 2) gated_sizes_kernel(const __grid_constant__ GatedSizes A) {
    chain_go();
    chain_wait();
    __shared__ float most[2][kSizeThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long rows = A.x.rows, ff = A.w[0].rows;
    float bounds = 0.f, factors = 0.f;
    for (long long t = (long long)blockIdx.x * (kSizeThreads / 32) + warp; t < rows + 2 * ff; t += kAmaxBlocks * (kSizeThreads / 32)) {
        const long long f = t - rows;
        const Operand &O = f < 0 ? A.x : A.w[f >= ff];
        float bound = sqrtf(row_size<true>(reinterpret_cast<const __half *>(O.p) + (f < 0 ? t : f >= ff ? f - ff : f) * O.ld, O.row, lane));
        if (f < 0) bound *= row_size<false>(reinterpret_cast<const __half *>(A.g.p) + t * A.g.ld, A.g.row, lane);
        else if (f >= ff) bound *= 1.13f;
        if (f < 0) {
            bounds = fmaxf(bounds, bound);
            if (lane == 0) A.bounds[t] = bound;
        } else {
            factors = fmaxf(factors, bound);
        }
    }
    if (lane == 0) { most[0][warp] = bounds; most[1][warp] = factors; }
    __syncthreads();
    if (warp < 2) {
        float m = lane < kSizeThreads / 32 ? most[warp][lane] : 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (lane == 0) A.amax[warp * kAmaxBlocks + blockIdx.x] = m;
    }
}

__global__ void __launch_bounds__(32) amax_losses_kernel(const __grid_constant__ ProductArgs A, int rows, float *amax) {
    chain_go();
    chain_wait();
    float m = 0.f;
#pragma unroll 4
    for (long long r = blockIdx.x * 32 + threadIdx.x; r < rows; r += kAmaxBlocks * 32) m = fmaxf(m, row_bound(A, r));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (threadIdx.x == 0) amax[blockIdx.x] = m;
}

// Adds up the sums of many splits, which lie as the threads of product_kernel left them: four columns of 32 rows a block, of which every warp takes each eighth split, then the first
// the warps' sums.  (Where the last split adds them up itself, one CTA of a tile reads them all: 24 splits of a tile of 256 x 256 take it 20 us.  A thread that adds up all splits waits for
// one batch of them after the other: 40 of them 11 us, so 5.)
template <int CG, int BN, typename T>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ ProductPart P, const __grid_constant__ ProductArgs A) {
    constexpr int kPieces = BN / 64, kTile = CG * kEpiWarps * kPieces * 1024;
    __shared__ float4 sums[7][32];
    chain_go();
    chain_wait();
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const float back = A.all_scale ? 1.f / *A.all_scale : 1.f;
    const int groups = (int)(P.by_plane.d * (unsigned)P.jobs) * (kTile / 128);
    for (int i = blockIdx.x; i < groups; i += gridDim.x) {
        const int at = i / (kTile / 128), q = i - at * (kTile / 128), four = q & 7, piece = (q >> 3) % kPieces, w = (q >> 3) / kPieces % kEpiWarps, rank = (q >> 3) / (kPieces * kEpiWarps),
                  job = at / (int)P.by_plane.d;
        const Tile t = tile_of(P, (unsigned)P.first + (unsigned)(at - job * (int)P.by_plane.d));
        const int row = t.m * 128 * CG + rank * 128 + ((w + 2) & 3) * 32 + lane, col = t.n * BN + (w >> 2) * (BN / 2) + piece * 32 + four * 4;
        if (row - lane >= P.m || col >= P.n) continue;        // (the whole block)
        const float4 *p = reinterpret_cast<const float4 *>(P.partial) + (long long)at * P.splits * (kTile / 4) + q * 32 + lane;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = slice; k < P.splits; k += 8) {
            const float4 x = __ldcg(p + (long long)k * (kTile / 4));
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        if (slice) sums[slice - 1][lane] = s;
        __syncthreads();
        if (slice == 0) {
#pragma unroll
            for (int k = 0; k < 7; ++k) {
                const float4 x = sums[k][lane];
                s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
            }
            if (row < P.m) {
                const float by = A.row_scale && !P.rows_a ? 1.f / A.row_scale[row] : back;
                *reinterpret_cast<uint2 *>(reinterpret_cast<T *>(P.out[job]) + (long long)row * P.out_ld + col) = make_uint2(pack2<T>(s.x * by, s.y * by), pack2<T>(s.z * by, s.w * by));
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------------ host

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static std::atomic<EncodeTiledFn> g_encode{nullptr};
static cudaError_t encoder(EncodeTiledFn *fn) {
    const cudaError_t bound = bind_device();
    if (bound != cudaSuccess) return bound;
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

// Boxes of 64 elements of `box_rows` rows; of `chunks` > 1 neighbouring runs of 64 elements of each row, one behind the other: of the whole runs, or (rest) of the one that is left, as if
// there were more.
// low: the boxes of a second matrix, so many elements further, come behind the first's.
static bool operand_map(EncodeTiledFn encode, CUtensorMap *out, Operand o, int dtype, int box_rows, int chunks, long long low = 0, bool rest = false) {
    cuuint64_t dims[3] = {(cuuint64_t)(rest ? o.row % 64 : chunks > 1 ? 64 : o.row), (cuuint64_t)o.rows, (cuuint64_t)(rest ? 1 : chunks > 1 ? o.row / 64 : low ? 2 : 1)};
    if (rest) o.p = (const char *)o.p + o.row / 64 * 128;
    cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, chunks > 1 ? 128 : low ? (cuuint64_t)low * 2 : (cuuint64_t)o.ld * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)box_rows, low ? 2 : (cuuint32_t)chunks}, one[3] = {1, 1, 1};
    return encode(out, dtype == XSM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(o.p), dims, strides, box, one,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Results as a warp stores them: 32 rows of 64 elements.
static bool result_map(EncodeTiledFn encode, CUtensorMap *out, void *p, int m, int n, long long ld, int dtype) {
    cuuint64_t dims[3] = {(cuuint64_t)n, (cuuint64_t)m, 1}, strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * 2 * m};
    cuuint32_t box[3] = {64, 32, 1}, one[3] = {1, 1, 1};
    return encode(out, dtype == XSM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, p, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int product_sms() {
    static std::atomic<int> known[kMaxDevices];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0;
    n = known[dev].load(std::memory_order_relaxed);
    if (n == 0 && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

int product_ctas(long long tiles, bool wide) {
    const int slots = wide ? product_sms() / 2 : product_sms();
    return (int)(tiles < slots ? tiles : slots) * (wide ? 2 : 1);
}

static std::atomic<unsigned> g_tries{kMbarSpinLimit};
static std::atomic<int> g_starve{0};
void product_waits(unsigned *tries, int *starve) {
    *tries = g_tries.load(std::memory_order_relaxed);
    *starve = g_starve.load(std::memory_order_relaxed);
}

template <int CG, int BN, int EPI, typename T> static cudaError_t start(const ProductMaps &M, const ProductArgs &A, cudaStream_t st) {
    const int smem = kRingBytes + (CG == 2 || EPI == PR_OUT ? kEpiWarps * 4096 : kABytes) + 1024;        // (few rows: the tensor cores read 128 rows of A whatever the box brought)
    const void *fn = (const void *)product_kernel<CG, BN, EPI, T>;
    cudaError_t e = open_for(fn, smem);
    if (e != cudaSuccess) return e;
    if (product_sms() < 2) return cudaErrorInvalidDevice;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)product_ctas(A.tiles, CG == 2));
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
bool product_few(ProductEpi epi, long long m, long long n) { return m <= 128 || n <= (epi == PR_GATED || epi == PR_GATED_GRAD ? 32 : 64); }

// Few rows or columns: what a CTA fetches decides, its tiles times the rows of both operands; of the widths that fetch least, the widest.  (96 rows x 131071 tokens: 64 columns 83 us,
// 128 49; 5 rows x 4096: 64 columns 10.6, 32 9.8, before stages of several blocks.)  Otherwise two CTAs a tile, but where there are too few such tiles for all of them: of what the rounds of
// tiles take, in cycles, the least: a block of 64 is 512 of the tensor cores, or what its operands' bytes are from the L2 (64 a cycle and CTA), a tile has its last products and what is done
// with its sums on top, more where outputs of odd length leave number by number.  (us, forward + gradient: loss 195 x 684 of 344 10.8 + 16.0 -> 7.3 + 12.0, 161 x 131 of 1472 14.0 + 18.5 ->
// 9.3 + 12.4, 1697 x 332 of 1952 17.1 + 28.9 -> 12.2 + 22.9; gated 486 x 532 of 1080 12.9 + 26.8 -> 12.4 + 23.4; 665 x 111 of 392 8.4 + 16.7 -> 9.3 + 14.0, whose forward stays wide.)
ProductCut product_cut(ProductEpi epi, long long m, long long n, long long d) {
    const bool gated = epi == PR_GATED || epi == PR_GATED_GRAD, few = product_few(epi, m, n);
    const long long sms = product_sms() < 2 ? 2 : product_sms(), blocks = (d + 63) / 64;
    const int odd = epi == PR_GATED && n % 8 ? 6144 : 0;
    ProductCut best = {!few, few ? 128 : 256};
    double least = few ? 1e300 : (double)((best.tiles(m, n, gated) + sms / 2 - 1) / (sms / 2)) * (double)(blocks * 512 + 4096);
    for (int bn = 128; bn >= (gated ? 64 : 32); bn /= 2) {
        const ProductCut c = {false, bn};
        const double rounds = (double)((c.tiles(m, n, gated) + sms - 1) / sms);
        const double cost = few ? rounds * (double)((m < 128 ? m : 128) + bn) : rounds * (double)(blocks * (256 + 2 * bn) + 1024 + 16 * bn + odd);
        if (cost < least) { least = cost; best = c; }
    }
    return best;
}

// Tiles, splits and their divisors; false: too many
static bool fill_part(ProductPart &P, const ProductCut &cut, bool gated, int m, int n, long long stages, int pairs, int jobs, int splits, long long first) {
    P.m = m; P.n = n; P.jobs = jobs; P.splits = splits;
    P.tiles_m = (m + cut.tm() - 1) / cut.tm();
    const long long tiles_n = (n + cut.tn(gated) - 1) / cut.tn(gated), tiles = P.tiles_m * tiles_n * jobs * splits;
    if (first + tiles > 0x3fffffff || stages * pairs > 0x3fffffff) return false;
    P.first = (int)first;
    P.tiles = (int)tiles;
    P.kb0 = (int)stages;
    P.kb = P.kb0 * pairs;
    P.group_m = P.tiles_m < 8 ? P.tiles_m : 8;
    const int last_rows = P.tiles_m % P.group_m;
    P.by_plane = Divisor((unsigned)(P.tiles_m * tiles_n));
    P.by_group = Divisor((unsigned)(P.group_m * tiles_n));
    P.by_rows = Divisor((unsigned)P.group_m);
    P.by_last_rows = Divisor((unsigned)(last_rows ? last_rows : P.group_m));
    P.by_splits = Divisor((unsigned)splits);
    P.kb_each = P.kb / splits;
    P.kb_more = P.kb % splits;
    return true;
}

template <int EPI> static cudaError_t start_cut(const ProductCut &cut, int dtype, const ProductMaps &M, const ProductArgs &A, cudaStream_t st) {
    const bool bf = dtype == XSM_BF16;
    auto go = [&](auto cg, auto bn) {
        constexpr int CG = decltype(cg)::value, BN = decltype(bn)::value;
        return bf ? start<CG, BN, EPI, bf16>(M, A, st) : start<CG, BN, EPI, __half>(M, A, st);
    };
    using std::integral_constant;
    if (cut.wide) return go(integral_constant<int, 2>(), integral_constant<int, 256>());
    if constexpr (EPI != PR_OUT) {
        if (cut.bn == 64) return go(integral_constant<int, 1>(), integral_constant<int, 64>());
    }
    if constexpr (EPI == PR_STATS || EPI == PR_DLOGITS) {
        if (cut.bn == 32) return go(integral_constant<int, 1>(), integral_constant<int, 32>());
    }
    return go(integral_constant<int, 1>(), integral_constant<int, 128>());
}

cudaError_t launch_product(ProductEpi epi, int dtype, ProductCut cut, ProductArgs A, int m, int n, const Operand &a, const Operand (&b)[2], cudaStream_t st) {
    EncodeTiledFn encode;
    cudaError_t e = encoder(&encode);
    if (e != cudaSuccess) return e;
    const bool gated = epi == PR_GATED || epi == PR_GATED_GRAD, wide = cut.wide;
    const int group = wide ? 2 : 1, a_rows = m >= 128 ? 128 : (m + 7) / 8 * 8;
    // Few rows: a stage of several blocks, each operand's by one copy, as long as three stages fit; a copy costs the TMA unit some 200 cycles whatever it brings (5 rows x 4096
    // tokens 9.8 -> 7.8 us).  What is left of rows that are no whole blocks has a stage of its own, which long rows are worth (us: 3 x 11421 of 1552 26.5 -> 21.1, 2 x 1056 of
    // 1848 13.4 -> 11.4; 8 x 139 of 1312 8.9 -> 7.8; but 3 x 1607 of 840 7.3 -> 7.8, 43 x 5344 of 328 8.4 -> 9.2).
    A.chunks = 1;
    if (!wide && (a.row % 64 == 0 || a.row >= 1024))
        while (A.chunks < 4 && 2 * A.chunks <= a.row / 64 && 2 * A.chunks * (a_rows + cut.bn) * 128 * 3 <= kRingBytes) A.chunks *= 2;
    A.tail = A.chunks > 1 && a.row % 64 != 0;
    ProductPart &P = A.part[0];
    const long long stages = A.chunks > 1 ? (a.row / 64 + A.chunks - 1) / A.chunks + A.tail : (a.row + 63) / 64;
    if (!fill_part(P, cut, gated, m, n, stages, 1, 1, 1, 0)) return cudaErrorInvalidValue;
    A.tiles = P.tiles;
    P.a_rows = a_rows;
    A.stage_b = (uint32_t)(a_rows * 128 * A.chunks);
    A.stage = A.stage_b + (uint32_t)(cut.bn / group * 128 * A.chunks);
    P.stage_tx = group * A.stage;
    A.stages = kRingBytes / (int)A.stage < kMaxStages ? kRingBytes / (int)A.stage : kMaxStages;
    A.round = 8 / A.chunks;
    product_waits(&A.tries, &A.starve);
    ProductMaps M;
    memset(&M, 0, sizeof M);
    const int b_box = gated ? (wide ? 128 : cut.bn / 2) : cut.bn / group;
    bool ok = operand_map(encode, &M.a[0], a, dtype, a_rows, A.chunks);
    for (int i = 0; i < (gated ? 2 : 1); ++i) ok = ok && operand_map(encode, &M.b[i], b[i], dtype, b_box, A.chunks);
    if (A.tail) {
        ok = ok && operand_map(encode, &M.a[1], a, dtype, a_rows, A.chunks, 0, true);
        for (int i = 0; i < (gated ? 2 : 1); ++i) ok = ok && operand_map(encode, &M.b[2 + i], b[i], dtype, b_box, A.chunks, 0, true);
    }
    if (wide && epi != PR_STATS) {
        A.tma_out = A.out_ld % 8 == 0 && (uintptr_t)A.out[0] % 16 == 0;
        for (int i = 0; i < (epi == PR_GATED_GRAD ? 2 : 1) && A.tma_out; ++i) ok = ok && result_map(encode, &M.out[i], A.out[i], m, n, A.out_ld, dtype);
    }
    if (!ok) return cudaErrorInvalidValue;
    switch (epi) {
        case PR_STATS: return start_cut<PR_STATS>(cut, dtype, M, A, st);
        case PR_DLOGITS: return start_cut<PR_DLOGITS>(cut, dtype, M, A, st);
        case PR_GATED: return start_cut<PR_GATED>(cut, dtype, M, A, st);
        case PR_GATED_GRAD: return start_cut<PR_GATED_GRAD>(cut, dtype, M, A, st);
        default: return cudaErrorInvalidValue;
    }
}

static size_t tile_bytes(const ProductCut &cut) { return (size_t)cut.tm() * cut.bn * 4; }
size_t sums_bytes(const ProductCut &cut, long long rows, long long d) { return (size_t)cut.tiles(rows, d, false) * tile_bytes(cut); }

// Splits that the last of them adds up itself; more are added up by a kernel of its own.
constexpr int kJoinedHere = 6;

// Both products' tiles are dealt out in one row, x's first; where a CTA would have too much to do the summed axes are cut.  Of both widths of tiles and of the splits, those that
// leave the CTAs with most to do least, in cycles: a block of 64 of the summed axis is 512 of the tensor cores in tiles of 256 x 256 (256 in those of 128 x 128, whose operands
// take longer to come), twice that in two parts; a tile has its last products and what is done with its sums on top, more where it is cut, and for each split that is added up (a piece
// of 32 columns at a time), or a launch for all.
static SumsPlan cut_sums(ProductCut cut, long long rows, long long cols, long long d, int pairs, bool x, bool y, bool once, bool low, double *least) {
    SumsPlan p = {};
    p.cut = cut;
    p.splits_x = p.splits_y = 1;
    const long long slots = product_sms() < 2 ? 1 : cut.wide ? product_sms() / 2 : product_sms(), kx = (cols + 63) / 64 * pairs, ky = (rows + 63) / 64;
    const long long tx = x ? cut.tiles(rows, d, false) : 0, ty = y ? cut.tiles(cols, d, false) * pairs : 0, per = (cut.wide ? 2 : 1) * 8;
    static const int tries[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64, 96, 128};
    const double stage = (cut.wide ? 512 : 400) * (low ? cut.wide ? 2 : 1.5 : 1), tile = cut.wide ? 4096 : 2048, each = d <= 32 ? 512 : d <= 64 || !cut.wide ? 1024 : 1536;
    auto cost = [&](long long k, int s) { return (double)((k + s - 1) / s) * stage + (s == 1 ? tile : s <= kJoinedHere ? 2 * tile + each * s : 2 * tile); };
    *least = 1e300;
    for (int sx : tries) {
        if (sx > 1 && (!x || sx * 4 > kx || tx * (sx - 1) > 2 * slots || (!once && sx > kJoinedHere))) break;
        for (int sy : tries) {
            if (sy > 1 && (!y || sy * 4 > ky || ty * (sy - 1) > 2 * slots)) break;
            if ((sx > 1 && sx <= kJoinedHere ? tx : 0) * per + (sy > 1 && sy <= kJoinedHere ? ty : 0) * per > kSumCounters) continue;
            const long long nx = tx * sx, all = nx + ty * sy;
            const double cx = cost(kx, sx), cy = cost(ky, sy);
            double most = 0;
            auto of = [&](long long c) {        // what CTA (pair) c has to do: tiles c, c + slots, ...
                if (c < 0 || c >= slots || c >= all) return;
                const long long mine = (all - 1 - c) / slots + 1, of_x = c < nx ? (nx - 1 - c) / slots + 1 : 0;
                const double t = of_x * cx + (mine - of_x) * cy;
                if (t > most) most = t;
            };
            of(0); of(nx % slots - 1); of(nx % slots); of(all % slots - 1); of(all % slots);
            most += (sx > kJoinedHere ? 10240 : 0) + (sy > kJoinedHere ? 10240 : 0);
            if (most < *least - 1e-9) { *least = most; p.splits_x = sx; p.splits_y = sy; }
        }
    }
    p.partial_x = 0;
    p.partial_y = p.splits_x > 1 ? (size_t)tx * p.splits_x * tile_bytes(cut) : 0;
    p.bytes = p.partial_y + (p.splits_y > 1 ? (size_t)ty * p.splits_y * tile_bytes(cut) : 0);
    return p;
}

// (us, in tiles of 256 and of 128: gradients of a loss over 96 rows of 131071 tokens, 1024 wide, 245 and 214; 5 x 11436 x 80 18 and 16; gated, 1125 x 2259 x 1296 62 and 72; 1162 x 2899 x 600
// 49 and 61; of 43 drawn cases the rule takes the slower one in 2, by 1 and 3 %.  300 or 550 cycles a narrow block: 1.8 and 0.4 % slower over 50.)
SumsPlan plan_sums(long long rows, long long cols, long long d, int pairs, bool x, bool y, bool once, bool low) {
    double wide, narrow;
    const SumsPlan p = cut_sums({true, 256}, rows, cols, d, pairs, x, y, once, low, &wide), q = cut_sums({false, 128}, rows, cols, d, pairs, x, y, once, low, &narrow);
    return wide <= narrow ? p : q;
}

static cudaError_t launch_join(const ProductCut &cut, int dtype, const ProductPart &P, const ProductArgs &A, cudaStream_t st) {
    const long long blocks = (long long)P.by_plane.d * P.jobs * (long long)(tile_bytes(cut) / 512), most = (long long)product_sms() * 8;
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    if (cut.wide)
        return dtype == XSM_BF16 ? launch_early(join_kernel<2, 256, bf16>, grid, dim3(256), 0, st, P, A) : launch_early(join_kernel<2, 256, __half>, grid, dim3(256), 0, st, P, A);
    return dtype == XSM_BF16 ? launch_early(join_kernel<1, 128, bf16>, grid, dim3(256), 0, st, P, A) : launch_early(join_kernel<1, 128, __half>, grid, dim3(256), 0, st, P, A);
}

cudaError_t launch_sums(int dtype, const SumsPlan &p, const Sums &s, cudaStream_t st) {
    EncodeTiledFn encode;
    cudaError_t e = encoder(&encode);
    if (e != cudaSuccess) return e;
    const int group = p.cut.wide ? 2 : 1;
    const int rows = (int)s.g[0].rows, cols = (int)s.g[0].row, d = (int)s.h.row;
    ProductArgs A = {};
    A.status = s.status;
    A.counter = s.counters;
    A.row_scale = s.row_scale;
    A.all_scale = s.all_scale;
    A.chunks = 1;
    A.low = s.low;
    const int parts = s.low ? 2 : 1;
    A.stage_b = (uint32_t)(kABytes * parts);
    A.stage = A.stage_b + (uint32_t)(p.cut.bn / group * 128);
    A.stages = kRingBytes / (int)A.stage < kMaxStages ? kRingBytes / (int)A.stage : kMaxStages;
    product_waits(&A.tries, &A.starve);
    ProductMaps M;
    memset(&M, 0, sizeof M);
    ProductPart &X = A.part[0], &Y = A.part[1];
    bool ok = true;
    const bool y = s.y[0] != nullptr;
    if (s.x) {
        const int splits = p.splits_x <= (cols + 63) / 64 * s.pairs ? p.splits_x : (cols + 63) / 64 * s.pairs;        // (the last piece of a vocabulary may be short)
        if (!fill_part(X, p.cut, false, rows, d, (cols + 63) / 64, s.pairs, 1, splits, 0)) return cudaErrorInvalidValue;
        X.a_rows = rows >= 128 ? 128 : (rows + 7) / 8 * 8;
        X.stage_tx = (uint32_t)(group * (X.a_rows * 128 * parts + p.cut.bn / group * 128));
        X.partial = (float *)(s.partial + p.partial_x);
        X.apart = X.splits > kJoinedHere;
        X.sums = s.x_sums; X.go_on = s.go_on; X.end = s.end;
        X.out[0] = s.x; X.out_ld = s.x_ld;
        for (int i = 0; i < s.pairs; ++i) {
            ok = ok && operand_map(encode, &M.a[i], s.g[i], dtype, X.a_rows, 1, s.low) && operand_map(encode, &M.b[i], s.w[i], dtype, 64, 1);
        }
        ok = ok && result_map(encode, &M.out[0], s.x, rows, d, s.x_ld, dtype);
    }
    A.tiles = X.tiles;
    Y.first = 0x7fffffff;
    if (y) {
        if (!fill_part(Y, p.cut, false, cols, d, (rows + 63) / 64, 1, s.pairs, p.splits_y, A.tiles)) return cudaErrorInvalidValue;
        Y.rows_a = 1;
        Y.a_rows = 128;
        Y.stage_tx = group * A.stage;
        Y.map_a = 2; Y.map_b = 2; Y.map_out = 1;
        Y.partial = (float *)(s.partial + p.partial_y);
        Y.apart = Y.splits > kJoinedHere;
        Y.counters = X.splits > 1 && !X.apart ? (unsigned)(X.by_plane.d * group * 8) : 0;
        for (int i = 0; i < s.pairs; ++i) {
            ok = ok && operand_map(encode, &M.a[2 + i], s.g[i], dtype, 64, 1, s.low);
            Y.out[i] = s.y[i];
            ok = ok && result_map(encode, &M.out[1 + i], s.y[i], cols, d, s.y_ld, dtype);
        }
        Y.out_ld = s.y_ld;
        ok = ok && operand_map(encode, &M.b[2], s.h, dtype, 64, 1);
        A.tiles += Y.tiles;
    }
    if (!ok) return cudaErrorInvalidValue;
    if (A.tiles) e = start_cut<PR_OUT>(p.cut, dtype, M, A, st);
    for (const ProductPart &P : A.part)
        if (e == cudaSuccess && P.tiles && P.apart) e = launch_join(p.cut, dtype, P, A, st);
    return e;
}

cudaError_t launch_gated_sizes(const GatedSizes &s, cudaStream_t st) { return launch_early(gated_sizes_kernel, dim3(kAmaxBlocks), dim3(kSizeThreads), 0, st, s); }
cudaError_t launch_amax_losses(const ProductArgs &A, int rows, float *amax, cudaStream_t st) { return launch_early(amax_losses_kernel, dim3(kAmaxBlocks), dim3(32), 0, st, A, rows, amax); }

}  // namespace xsm

xsm_status xsm_debug_product_waits(uint32_t tries, int starve) {
    xsm::g_tries.store(tries ? tries : xsm::kMbarSpinLimit, std::memory_order_relaxed);
    xsm::g_starve.store(starve != 0, std::memory_order_relaxed);
    return XSM_OK;
}
