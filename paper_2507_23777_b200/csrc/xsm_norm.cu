// Norms of queries and keys for each head with the rotation of the positions in the same pass: whole sequences for training, with the gradients, and new
// tokens on their way to the pages of a cache.
//
// y = R(position) (gain x r), r = (mean x^2 + eps)^(-1/2) over a head.  Gradient: u = R^-1 dy, d_gain = sum over rows of u x r, dx = r (w - x r^2 mean(w x)), w = gain u.
// A head is 2 to 32 neighbouring lanes, which hold two runs of 16 bytes each, the two halves of their pairs, so that norm and rotation need nothing but
// the lanes' own registers and a sum over them.  A group of lanes takes some heads of a token one behind the other, what the token's angles and the gains have to do with an
// element in registers; the heads to come are on their way to slots of shared memory that each lane has for itself, so that neither registers nor barriers limit
// how many.  d_gain is added up in registers over all rows of a group, then over a block, then over blocks in a fixed order: no result hangs on who
// comes first.
//
// What bounds it.  8192 tokens of 32 + 8 heads of 128 in bf16: forward 33 us where its bytes take 26 at the copy rate, gradient 54 and a kernel of 5 where they take 39: memory at 77 and
// 66 %, half of the issue slots (two numbers an instruction), four warps a scheduler, which the registers allow (three blocks an SM instead of two: 33 -> 43 us).  Four rows
// on their way are enough (six, eight: no faster).  A window of five tokens into the pages: 3.2 us, two latencies behind a launch.
#include "xsm_ops.h"
#include "xsm_chain.cuh"

#include <limits.h>
#include <string.h>

#include <type_traits>

namespace xsm {

enum NormMode { NM_FORWARD, NM_APPEND, NM_GRAD };
constexpr int kNormThreads = 256;
constexpr int kNormBlocks = 2;        // of an SM

struct NormTensor {
    const void *x, *g;              // rows, gradients of the result
    void *out;                      // result, or gradient by x
    const void *gain;
    float *part;                    // NM_GRAD: [block][d]
    void *d_gain;
    long long xs[3], gs[3], os[3];  // strides of sequence, token, head
    int heads, blocks;              // heads, blocks that work on the tensor
    Divisor by_chunks;              // units of a token
};
struct NormArgs {
    NormTensor t[3];                // queries, keys, values
    const int *starts, *counts, *positions;
    const float2 *rope;
    unsigned tokens, m;
    Divisor by_m;
    int d, rope_n, rot, hp, gain_dtype;      // hp: heads of a unit
    float eps, inv_d;
    unsigned *counter;              // NM_GRAD: of blocks that have ended
};

__device__ __forceinline__ float gain_at(const void *p, int dtype, int i) {
    return dtype == XSM_F32 ? reinterpret_cast<const float *>(p)[i] : dtype == XSM_BF16 ? to_f(reinterpret_cast<const bf16 *>(p)[i]) : to_f(reinterpret_cast<const __half *>(p)[i]);
}

// two fp32 numbers that are worked on together
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair(float a, float b) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 both(Pair p) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
    return r;
}
__device__ __forceinline__ Pair swapped(Pair p) { const float2 v = both(p); return pair(v.y, v.x); }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Where a token is, and whether there is something to be done for it.
struct Token {
    bool live;                  // it has a position that the rope has: otherwise its rows are zero
    long long pos, place;       // place: NM_APPEND, of its row in head 0 of the pools, in elements; -1: none
};
template <int MODE> __device__ __forceinline__ int first_of(const NormArgs &A, int b, int j) {        // what its position comes from
    return MODE == NM_APPEND ? A.starts[b] : A.positions ? A.positions[(long long)b * A.m + j] : j;
}
template <int MODE> __device__ __forceinline__ Token token_at(const NormArgs &A, const Pages &P, int b, int j, int from) {
    Token t = {true, 0, -1};
    if (MODE == NM_APPEND) {
        t.live = A.counts == nullptr || j < A.counts[b];
        t.pos = (long long)from + j;
    } else if (A.rope != nullptr) {
        t.pos = from;
    }
    t.live = t.live && (A.rope == nullptr || (t.pos >= 0 && t.pos < A.rope_n));
    if (MODE == NM_APPEND && t.live && t.pos >= 0 && t.pos <= INT_MAX) {
        const int at = (int)t.pos / P.size;
        const int page = at < P.max_pages ? P.table[b * P.table_ld + at] : -1;
        if (page >= 0 && page < P.n_pages) t.place = page * P.page + ((int)t.pos - at * P.size) * P.row;
    }
    return t;
}

// 16-byte pieces of a head and a lane, heads on their way, bytes of a block's slots
template <int MODE> struct NormSlots { static constexpr int pieces = MODE == NM_GRAD ? 4 : 2, ahead = 4, bytes = ahead * pieces * 16 * kNormThreads; };

// 2H numbers rounded to T (kPool: as elements of a pool)
template <bool kPool, typename T, int H> __device__ __forceinline__ void store_run(T *p, const Pair (&x)[H]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < H / 2; ++i) {
            const float2 a = both(x[2 * i]), b = both(x[2 * i + 1]);
            reinterpret_cast<float4 *>(p)[i] = make_float4(a.x, a.y, b.x, b.y);
        }
    } else {
        uint32_t w[H];
#pragma unroll
        for (int i = 0; i < H; ++i) {
            const float2 v = both(x[i]);
            if constexpr (std::is_same<T, bf16>::value) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
                memcpy(&w[i], &h, 4);
            } else {
                T h[2] = {kPool ? to_stored<T>(v.x) : rounded<T>(v.x), kPool ? to_stored<T>(v.y) : rounded<T>(v.y)};
                memcpy(&w[i], h, 4);
            }
        }
        if constexpr (H == 4) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
    }
}

// Adds up the d_gain of a few blocks where the last of them ends: 8 to 32 threads a quad of elements, each every so-many-th block, then these; nothing hangs on which is the last.
__device__ __forceinline__ void finish_gains(const NormArgs &A) {
    __shared__ int last;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicInc(A.counter, gridDim.x - 1) == gridDim.x - 1;
        __threadfence();
    }
    __syncthreads();
    if (!last) return;
    const int quads = A.d / 4, parts = quads <= 8 ? 32 : quads <= 16 ? 16 : 8, part = (int)threadIdx.x % parts;
    for (int t = 0; t < 2; ++t) {
        const NormTensor &T = A.t[t];
        if (!T.heads) continue;
        for (int q0 = 0; q0 < quads; q0 += kNormThreads / parts) {
            const int q = q0 + (int)threadIdx.x / parts;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (q < quads) {
                const float *from = T.part + 4 * q;
#pragma unroll 4
                for (int b = part; b < T.blocks; b += parts) {
                    const float4 x = __ldcg(reinterpret_cast<const float4 *>(from + (long long)b * A.d));
                    v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
                }
            }
            for (int o = parts / 2; o > 0; o >>= 1) {
                v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
                v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
                v.z += __shfl_xor_sync(0xffffffffu, v.z, o);
                v.w += __shfl_xor_sync(0xffffffffu, v.w, o);
            }
            if (q < quads && part < 4) {
                const float f = part == 0 ? v.x : part == 1 ? v.y : part == 2 ? v.z : v.w;
                const int e = 4 * q + part;
                if (A.gain_dtype == XSM_F32) reinterpret_cast<float *>(T.d_gain)[e] = f;
                else if (A.gain_dtype == XSM_BF16) reinterpret_cast<bf16 *>(T.d_gain)[e] = rounded<bf16>(f);
                else reinterpret_cast<__half *>(T.d_gain)[e] = rounded<__half>(f);
            }
        }
    }
}

// Rows and angles in 16-byte pieces.  L lanes a head; the lanes' first runs lie side by side, and so do the second ones, half of the turned (of the other) part of the head
// further: with half-split pairs a lane then has both elements of each, with neighbouring ones (kNear) anyway.  (Two runs of a lane side by side made accesses of half
// sectors: 20 us instead of 13 for 3003 tokens of 32 heads of 64 in fp32.)
// kFinish: the block that ends last adds up the blocks' d_gain (a kernel of its own: the code for it costs the loop 3 us of 20).
template <typename TI, typename TC, int L, bool kNear, int MODE, bool kFinish>
__global__ void __launch_bounds__(kNormThreads, kNormBlocks) norm_kernel(const __grid_constant__ NormArgs A, const __grid_constant__ Pages P) {
    constexpr int G = kNormThreads / L, N = 16 / (int)sizeof(TI), H = N / 2;        // N elements a run
    using Slots = NormSlots<MODE>;
    extern __shared__ __align__(16) char smem[];
    chain_go();
    chain_wait();
    int blk = (int)blockIdx.x, job = 0;
    while (job < 2 && blk >= A.t[job].blocks) blk -= A.t[job++].blocks;
    const NormTensor &T = A.t[job];
    const bool norm = job < 2;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const unsigned mask = L == 32 ? 0xffffffffu : ((1u << L) - 1u) << ((threadIdx.x & 31) & ~(L - 1));
    const int turned = norm ? A.rot / (2 * N) : 0;
    const bool have = lane < A.d / (2 * N), turn = lane < turned;
    const int e0 = turn ? lane * N : turned * 2 * N + (lane - turned) * N, e1 = e0 + (turn ? turned : A.d / (2 * N) - turned) * N;
    Pair g0[H], g1[H], a0[H], a1[H];
#pragma unroll
    for (int k = 0; k < H; ++k) {
        const bool g = norm && have;
        g0[k] = pair(g ? gain_at(T.gain, A.gain_dtype, e0 + 2 * k) : 1.f, g ? gain_at(T.gain, A.gain_dtype, e0 + 2 * k + 1) : 1.f);
        g1[k] = pair(g ? gain_at(T.gain, A.gain_dtype, e1 + 2 * k) : 1.f, g ? gain_at(T.gain, A.gain_dtype, e1 + 2 * k + 1) : 1.f);
        a0[k] = a1[k] = pair(0.f, 0.f);
    }
    const unsigned units = A.tokens * T.by_chunks.d, stride = (unsigned)T.blocks * G;

    // The head that is asked for, `ahead` heads before it is worked on.
    struct Place {
        unsigned u;
        int h, h1;
        const TI *x, *dy;
    };
    auto open = [&](Place &c, unsigned u) {
        c.u = u;
        if (u >= units) return;
        const unsigned token = T.by_chunks.of(u), b = A.by_m.of(token), j = token - b * A.m;
        c.h = (int)(u - token * T.by_chunks.d) * A.hp;
        c.h1 = min(c.h + A.hp, T.heads);
        c.x = reinterpret_cast<const TI *>(T.x) + b * T.xs[0] + j * T.xs[1] + c.h * T.xs[2];
        if (MODE == NM_GRAD) c.dy = reinterpret_cast<const TI *>(T.g) + b * T.gs[0] + j * T.gs[1] + c.h * T.gs[2];
    };
    const uint32_t slots = smem_u32(smem) + threadIdx.x * 16u;
    constexpr uint32_t kPiece = 16u * kNormThreads, kSlot = Slots::pieces * kPiece;
    Place ask = {};
    uint32_t ask_slot = slots, slot = slots;
    auto fetch = [&]() {
        if (ask.u < units) {
            if (have) {
                auto run = [&](const TI *p, int which) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(ask_slot + (uint32_t)which * kPiece), "l"(p) : "memory"); };
                run(ask.x + e0, 0);
                run(ask.x + e1, 1);
                if (MODE == NM_GRAD) {
                    run(ask.dy + e0, 2);
                    run(ask.dy + e1, 3);
                }
            }
            if (++ask.h == ask.h1) {
                open(ask, ask.u + stride);
            } else {
                ask.x += T.xs[2];
                if (MODE == NM_GRAD) ask.dy += T.gs[2];
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        ask_slot = ask_slot == slots + (Slots::ahead - 1) * kSlot ? slots : ask_slot + kSlot;
    };
    // run `which` of the present head
    auto take = [&](int which, Pair (&v)[H]) {
        uint32_t w[4];
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(slot + (uint32_t)which * kPiece) : "memory");
#pragma unroll
        for (int q = 0; q < H; ++q) {
            if constexpr (sizeof(TI) == 4) {
                v[q] = pair(__uint_as_float(w[2 * q]), __uint_as_float(w[2 * q + 1]));
            } else if constexpr (std::is_same<TI, bf16>::value) {
                v[q] = pair(__uint_as_float(w[q] << 16), __uint_as_float(w[q] & 0xffff0000u));
            } else {
                __half2 h;
                memcpy(&h, &w[q], 4);
                const float2 f = __half22float2(h);
                v[q] = pair(f.x, f.y);
            }
        }
    };

    open(ask, (unsigned)blk * G + group);
#pragma unroll
    for (int f = 0; f < Slots::ahead; ++f) fetch();
    // (the next unit's position is read while this one is worked on, and its angles are brought to the L1: two latencies a unit otherwise)
    auto ahead = [&](unsigned u) {
        if (u >= units) return 0;
        const unsigned token = T.by_chunks.of(u), b = A.by_m.of(token);
        return first_of<MODE>(A, (int)b, (int)(token - b * A.m));
    };
    int from = ahead((unsigned)blk * G + group);
    for (unsigned u = (unsigned)blk * G + group; u < units; u += stride) {
        const unsigned token = T.by_chunks.of(u);
        const int b = (int)A.by_m.of(token), j = (int)(token - (unsigned)b * A.m), h0 = (int)(u - token * T.by_chunks.d) * A.hp, h1 = min(h0 + A.hp, T.heads);
        const Token at = token_at<MODE>(A, P, b, j, from);
        from = ahead(u + stride);
        // What the angles have to do with two elements x at a time.  kNear, x = (a, b) a pair: R x = x (c, c) + (b, a) (-s, s).  Otherwise x of the first run, y of the second,
        // two pairs: (x c - y s, x s + y c).  Forward with the gains in it, backward by the angles' negatives.
        Pair c0[H], c1[H], s0[H], s1[H];
#pragma unroll
        for (int k = 0; k < H; ++k) c0[k] = c1[k] = s0[k] = s1[k] = pair(0.f, 0.f);
        if (turn && at.live) {
            const float2 *angles = A.rope + at.pos * (A.rot / 2);
            if constexpr (!kNear) {
#pragma unroll
                for (int k = 0; k < H; ++k) {        // two pairs
                    const float4 t = reinterpret_cast<const float4 *>(angles + lane * N)[k];
                    const Pair c = pair(t.x, t.z), s = pair(t.y, t.w), minus = pair(-t.y, -t.w);
                    c0[k] = MODE == NM_GRAD ? c : mul2(c, g0[k]);
                    if (MODE != NM_GRAD) c1[k] = mul2(c, g1[k]);
                    s0[k] = MODE == NM_GRAD ? s : mul2(minus, g1[k]);
                    s1[k] = MODE == NM_GRAD ? minus : mul2(s, g0[k]);
                }
            } else {
                auto near = [&](float2 t, Pair g, Pair &c, Pair &s) {
                    c = MODE == NM_GRAD ? pair(t.x, t.x) : mul2(pair(t.x, t.x), g);
                    s = MODE == NM_GRAD ? pair(t.y, -t.y) : mul2(pair(-t.y, t.y), swapped(g));
                };
#pragma unroll
                for (int k = 0; k < H; k += 2) {
                    const float4 t = reinterpret_cast<const float4 *>(angles + lane * H)[k / 2], v = reinterpret_cast<const float4 *>(angles + A.rot / 4 + lane * H)[k / 2];
                    near(make_float2(t.x, t.y), g0[k], c0[k], s0[k]);
                    near(make_float2(t.z, t.w), g0[k + 1], c0[k + 1], s0[k + 1]);
                    near(make_float2(v.x, v.y), g1[k], c1[k], s1[k]);
                    near(make_float2(v.z, v.w), g1[k + 1], c1[k + 1], s1[k + 1]);
                }
            }
        }
        TI *dst = reinterpret_cast<TI *>(T.out) + b * T.os[0] + j * T.os[1] + h0 * T.os[2];
        TC *row = MODE == NM_APPEND && job > 0 ? reinterpret_cast<TC *>(job == 1 ? P.k : P.v) + at.place + h0 * P.head : nullptr;
        for (int h = h0; h < h1; ++h) {
            asm volatile("cp.async.wait_group %0;" :: "n"(Slots::ahead - 1) : "memory");
            Pair p[H], q[H], up[H], uq[H];
            if (have) {
                take(0, p);
                take(1, q);
                if (MODE == NM_GRAD) {
                    take(2, up);
                    take(3, uq);
                }
            } else {
#pragma unroll
                for (int k = 0; k < H; ++k) p[k] = q[k] = up[k] = uq[k] = pair(0.f, 0.f);
            }
            fetch();        // (into the slot that has just been read)
            slot = slot == slots + (Slots::ahead - 1) * kSlot ? slots : slot + kSlot;
            float r = 1.f;
            if (norm) {
                Pair sums = pair(0.f, 0.f), more = sums;
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    sums = fma2(p[k], p[k], sums);
                    more = fma2(q[k], q[k], more);
                }
                const float2 x = both(sums), y = both(more);
                float ss = (x.x + x.y) + (y.x + y.y);
#pragma unroll
                for (int o = L / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(mask, ss, o);
                r = rsqrtf(fmaf(ss, A.inv_d, A.eps));
            }
            const Pair rr = pair(r, r);
            if (!at.live) {
#pragma unroll
                for (int k = 0; k < H; ++k) p[k] = q[k] = pair(0.f, 0.f);
            } else if (MODE == NM_GRAD) {
                Pair dots = pair(0.f, 0.f);
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    if (turn) {
                        if constexpr (kNear) {
                            up[k] = fma2(up[k], c0[k], mul2(swapped(up[k]), s0[k]));
                            uq[k] = fma2(uq[k], c1[k], mul2(swapped(uq[k]), s1[k]));
                        } else {
                            const Pair first = fma2(up[k], c0[k], mul2(uq[k], s0[k]));
                            uq[k] = fma2(uq[k], c0[k], mul2(up[k], s1[k]));
                            up[k] = first;
                        }
                    }
                    a0[k] = fma2(up[k], mul2(p[k], rr), a0[k]);
                    a1[k] = fma2(uq[k], mul2(q[k], rr), a1[k]);
                    up[k] = mul2(up[k], g0[k]);
                    uq[k] = mul2(uq[k], g1[k]);
                    dots = fma2(up[k], p[k], dots);
                    dots = fma2(uq[k], q[k], dots);
                }
                const float2 x = both(dots);
                float dot = x.x + x.y;
#pragma unroll
                for (int o = L / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(mask, dot, o);
                const float f = -r * r * dot * A.inv_d;
                const Pair ff = pair(f, f);
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    p[k] = mul2(rr, fma2(p[k], ff, up[k]));
                    q[k] = mul2(rr, fma2(q[k], ff, uq[k]));
                }
            } else if (turn) {
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    if constexpr (kNear) {
                        p[k] = mul2(rr, fma2(p[k], c0[k], mul2(swapped(p[k]), s0[k])));
                        q[k] = mul2(rr, fma2(q[k], c1[k], mul2(swapped(q[k]), s1[k])));
                    } else {
                        const Pair first = mul2(rr, fma2(p[k], c0[k], mul2(q[k], s0[k])));
                        q[k] = mul2(rr, fma2(q[k], c1[k], mul2(p[k], s1[k])));
                        p[k] = first;
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    p[k] = mul2(mul2(p[k], rr), g0[k]);
                    q[k] = mul2(mul2(q[k], rr), g1[k]);
                }
            }
            if (MODE == NM_APPEND && job > 0) {
                if (have && at.place >= 0) {
                    store_run<true>(row + e0, p);
                    store_run<true>(row + e1, q);
                }
                row += P.head;
            } else {
                if (have) {
                    store_run<false>(dst + e0, p);
                    store_run<false>(dst + e1, q);
                }
                dst += T.os[2];
            }
            if (MODE != NM_APPEND && h == h0 && turn && (unsigned)from < (unsigned)A.rope_n)
                asm volatile("prefetch.global.L1 [%0];" :: "l"(A.rope + (long long)from * (A.rot / 2) + lane * N));
        }
    }
    if constexpr (MODE == NM_GRAD) {
        constexpr int W = 2 * N * L + 1;
        float *s = reinterpret_cast<float *>(smem);
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        if (have)
#pragma unroll
            for (int k = 0; k < H; ++k) {
                const float2 x = both(a0[k]), y = both(a1[k]);
                s[group * W + e0 + 2 * k] = x.x; s[group * W + e0 + 2 * k + 1] = x.y;
                s[group * W + e1 + 2 * k] = y.x; s[group * W + e1 + 2 * k + 1] = y.y;
            }
        __syncthreads();
        for (int e = threadIdx.x; e < A.d; e += kNormThreads) {
            float v = 0.f;
            for (int g = 0; g < G; ++g) v += s[g * W + e];
            T.part[(long long)blk * A.d + e] = v;
        }
        if constexpr (kFinish) finish_gains(A);
    }
}

// The same for rows or angles of any alignment: a warp a head, up to four pairs of elements a lane.
template <typename TI, typename TC, bool kNear, int MODE, bool kFinish>
__global__ void __launch_bounds__(kNormThreads) norm_any_kernel(const __grid_constant__ NormArgs A, const __grid_constant__ Pages P) {
    constexpr int I = 4, G = kNormThreads / 32;
    __shared__ float s[MODE == NM_GRAD ? G : 1][257];
    chain_go();
    chain_wait();
    int blk = (int)blockIdx.x, job = 0;
    while (job < 2 && blk >= A.t[job].blocks) blk -= A.t[job++].blocks;
    const NormTensor &T = A.t[job];
    const bool norm = job < 2;
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    int e0[I], e1[I];
    bool have[I], turn[I];
    float g0[I], g1[I], a0[I], a1[I];
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int c = lane + 32 * i;
        have[i] = c < A.d / 2;
        turn[i] = norm && c < A.rot / 2;
        e0[i] = turn[i] && !kNear ? c : 2 * c;
        e1[i] = turn[i] && !kNear ? c + A.rot / 2 : 2 * c + 1;
        g0[i] = norm && have[i] ? gain_at(T.gain, A.gain_dtype, e0[i]) : 1.f;
        g1[i] = norm && have[i] ? gain_at(T.gain, A.gain_dtype, e1[i]) : 1.f;
        a0[i] = a1[i] = 0.f;
    }
    const unsigned units = A.tokens * T.by_chunks.d;
    for (unsigned u = (unsigned)blk * G + group; u < units; u += (unsigned)T.blocks * G) {
        const unsigned token = T.by_chunks.of(u);
        const int b = (int)A.by_m.of(token), j = (int)(token - (unsigned)b * A.m), h0 = (int)(u - token * T.by_chunks.d) * A.hp, h1 = min(h0 + A.hp, T.heads);
        const Token at = token_at<MODE>(A, P, b, j, first_of<MODE>(A, b, j));
        if (MODE == NM_APPEND && job > 0 && at.place < 0) continue;
        for (int h = h0; h < h1; ++h) {
            const TI *x = reinterpret_cast<const TI *>(T.x) + b * T.xs[0] + j * T.xs[1] + h * T.xs[2];
            const TI *dy = MODE == NM_GRAD ? reinterpret_cast<const TI *>(T.g) + b * T.gs[0] + j * T.gs[1] + h * T.gs[2] : nullptr;
            float p[I], q[I], up[I], uq[I], ss = 0.f, r = 1.f;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                p[i] = have[i] ? to_f(x[e0[i]]) : 0.f;
                q[i] = have[i] ? to_f(x[e1[i]]) : 0.f;
                up[i] = MODE == NM_GRAD && have[i] ? to_f(dy[e0[i]]) : 0.f;
                uq[i] = MODE == NM_GRAD && have[i] ? to_f(dy[e1[i]]) : 0.f;
                ss = fmaf(p[i], p[i], fmaf(q[i], q[i], ss));
            }
            if (norm) r = rsqrtf(fmaf(warp_sum(ss), A.inv_d, A.eps));
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const float2 cs = turn[i] && at.live ? A.rope[at.pos * (A.rot / 2) + lane + 32 * i] : make_float2(1.f, 0.f);
                if (MODE == NM_GRAD) {
                    if (turn[i]) {
                        const float f = up[i] * cs.x + uq[i] * cs.y;
                        uq[i] = uq[i] * cs.x - up[i] * cs.y;
                        up[i] = f;
                    }
                    if (at.live) {
                        a0[i] = fmaf(up[i], p[i] * r, a0[i]);
                        a1[i] = fmaf(uq[i], q[i] * r, a1[i]);
                    }
                    up[i] *= g0[i];
                    uq[i] *= g1[i];
                    dot = fmaf(up[i], p[i], fmaf(uq[i], q[i], dot));
                } else {
                    p[i] = p[i] * r * g0[i];
                    q[i] = q[i] * r * g1[i];
                    if (turn[i]) {
                        const float f = p[i] * cs.x - q[i] * cs.y;
                        q[i] = p[i] * cs.y + q[i] * cs.x;
                        p[i] = f;
                    }
                }
            }
            if (MODE == NM_GRAD) {
                const float f = -r * r * warp_sum(dot) * A.inv_d;
#pragma unroll
                for (int i = 0; i < I; ++i) {
                    p[i] = r * fmaf(p[i], f, up[i]);
                    q[i] = r * fmaf(q[i], f, uq[i]);
                }
            }
            TI *dst = reinterpret_cast<TI *>(T.out) + b * T.os[0] + j * T.os[1] + h * T.os[2];
            TC *row = MODE == NM_APPEND && job > 0 ? reinterpret_cast<TC *>(job == 1 ? P.k : P.v) + at.place + h * P.head : nullptr;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                if (!have[i]) continue;
                if (MODE == NM_APPEND && job > 0) {
                    row[e0[i]] = to_stored<TC>(p[i]);
                    row[e1[i]] = to_stored<TC>(q[i]);
                } else {
                    dst[e0[i]] = rounded<TI>(at.live ? p[i] : 0.f);
                    dst[e1[i]] = rounded<TI>(at.live ? q[i] : 0.f);
                }
            }
        }
    }
    if constexpr (MODE == NM_GRAD) {
#pragma unroll
        for (int i = 0; i < I; ++i)
            if (have[i]) { s[group][e0[i]] = a0[i]; s[group][e1[i]] = a1[i]; }
        __syncthreads();
        for (int e = threadIdx.x; e < A.d; e += kNormThreads) {
            float v = 0.f;
            for (int g = 0; g < G; ++g) v += s[g][e];
            T.part[(long long)blk * A.d + e] = v;
        }
        if constexpr (kFinish) finish_gains(A);
    }
}

struct GainArgs {
    const float *part[2];
    void *out[2];
    int blocks[2], d, dtype;
};
// d_gain: 32 elements a block, 32 threads an element
__global__ void __launch_bounds__(1024) gain_kernel(const __grid_constant__ GainArgs A) {
    chain_go();
    chain_wait();
    __shared__ float s[32][33];
    const int which = blockIdx.y, x = threadIdx.x & 31, y = threadIdx.x >> 5;
    if (A.out[which] == nullptr) return;
    float v = 0.f;
#pragma unroll 4
    for (int b = y; b < A.blocks[which]; b += 32) v += A.part[which][(long long)b * A.d + blockIdx.x * 32 + x];
    s[y][x] = v;
    __syncthreads();
    v = s[x][y];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (x) return;
    const int e = blockIdx.x * 32 + y;
    if (A.dtype == XSM_F32) reinterpret_cast<float *>(A.out[which])[e] = v;
    else if (A.dtype == XSM_BF16) reinterpret_cast<bf16 *>(A.out[which])[e] = rounded<bf16>(v);
    else reinterpret_cast<__half *>(A.out[which])[e] = rounded<__half>(v);
}

// ------------------------------------------------------------------------------------------------------ host

static int norm_sms() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 1;
    return n;
}
static int lanes_of(int d, int es, bool wide) { return !wide ? 32 : d == 96 ? 128 * es / 32 : d * es / 32; }

// Heads of a unit and blocks of each tensor.  No more blocks than run at a time (one more: 41 us instead of 33 for 8192 tokens of 32 + 8 heads of 128), shared out by the tensors' heads; of 8, 4, 2 and 1 heads a
// unit those with which the groups that have most to do have least: a unit costs a group as much as one and a half heads before the first of them.
static int cut_norm(NormArgs &A, int lanes) {
    const int groups = kNormThreads / lanes, most = norm_sms() * kNormBlocks;
    long long heads = 0;
    int all = 0;
    double least = 1e300;
    for (const NormTensor &t : A.t) heads += t.heads;
    for (int hp = 8; hp >= 1; hp /= 2) {
        long long units = 0;
        for (const NormTensor &t : A.t) units += (long long)A.tokens * ((t.heads + hp - 1) / hp);
        const double cost = (double)((units + (long long)most * groups - 1) / ((long long)most * groups)) * (hp + 1.5);
        if (cost < least) { least = cost; A.hp = hp; }
    }
    for (NormTensor &t : A.t) {
        const int chunks = (t.heads + A.hp - 1) / A.hp;
        t.by_chunks = Divisor((unsigned)(chunks ? chunks : 1));
        const long long need = ((long long)A.tokens * chunks + groups - 1) / groups, share = most * t.heads / heads < 1 ? 1 : most * t.heads / heads;
        t.blocks = (int)(need < share ? need : share);
        all += t.blocks;
    }
    return all;
}

template <typename TI, typename TC, int MODE>
static cudaError_t launch_norm(const NormArgs &A, const Pages &P, int blocks, bool wide, bool near, cudaStream_t st) {
    auto start = [&](auto fn, int smem) {
        const cudaError_t e = smem > 48 * 1024 ? open_for((const void *)fn, smem) : cudaSuccess;
        return e != cudaSuccess ? e : launch_early(fn, dim3(blocks), dim3(kNormThreads), smem, st, A, P);
    };
    auto finish = [&](auto f) {        // f(whether the last block adds up)
        if constexpr (MODE == NM_GRAD) return A.counter ? f(std::true_type()) : f(std::false_type());
        else return f(std::false_type());
    };
    if (!wide)
        return finish([&](auto fin) {
            return near ? start(norm_any_kernel<TI, TC, true, MODE, decltype(fin)::value>, 0) : start(norm_any_kernel<TI, TC, false, MODE, decltype(fin)::value>, 0);
        });
    auto go = [&](auto l) {
        constexpr int L = decltype(l)::value, slots = NormSlots<MODE>::bytes, sums = MODE == NM_GRAD ? kNormThreads / L * (32 / (int)sizeof(TI) * L + 1) * 4 : 0, smem = slots > sums ? slots : sums;
        return finish([&](auto fin) {
            return near ? start(norm_kernel<TI, TC, L, true, MODE, decltype(fin)::value>, smem) : start(norm_kernel<TI, TC, L, false, MODE, decltype(fin)::value>, smem);
        });
    };
    using std::integral_constant;
    const int lanes = lanes_of(A.d, (int)sizeof(TI), true);
    if constexpr (sizeof(TI) == 2) {
        if (lanes == 2) return go(integral_constant<int, 2>());
    } else {
        if (lanes == 32) return go(integral_constant<int, 32>());
    }
    switch (lanes) {
        case 4: return go(integral_constant<int, 4>());
        case 8: return go(integral_constant<int, 8>());
        default: return go(integral_constant<int, 16>());
    }
}

static bool aligned(const void *p, const int64_t *s, int es) {
    return ((uintptr_t)p | (uintptr_t)(s[0] * es) | (uintptr_t)(s[1] * es) | (uintptr_t)(s[2] * es)) % 16 == 0;
}
static const char *wrong_norm(int dtype, int gain_dtype, float eps, const void *rope, int rope_positions, int rope_dims, int d) {
    if (!is_dtype(dtype) || !is_dtype(gain_dtype)) return "types must be 0 (fp32), 1 (bf16) or 2 (fp16)";
    if (d != 32 && d != 64 && d != 96 && d != 128 && d != 256) return "d_head must be 32, 64, 96, 128 or 256";
    if (!(eps >= 0.f) || !(eps < INFINITY)) return "eps must be finite and not negative";
    if (rope && (rope_dims < 2 || rope_dims % 2 || rope_dims > d || rope_positions < 1)) return "rope_dims must be even and in [2, d_head], rope_positions positive";
    if ((uintptr_t)rope % 8) return "rope must be 8-byte aligned";
    return nullptr;
}

// What norm_rotate and its gradient have in common.
struct NormSizes {
    int batch, m, n_heads, n_kv_heads, d_head, dtype, gain_dtype, rope_positions, rope_dims;
    float eps;
};
static const char *wrong_sizes(const NormSizes &s, const void *rope) {
    if (const char *w = wrong_norm(s.dtype, s.gain_dtype, s.eps, rope, s.rope_positions, s.rope_dims, s.d_head)) return w;
    if (s.batch < 0 || s.m < 0 || s.n_heads < 0 || s.n_kv_heads < 0 || s.n_heads > 4096 || s.n_kv_heads > 4096) return "batch and m must not be negative, n_heads and n_kv_heads in [0, 4096]";
    if ((long long)s.batch * s.m * (s.n_heads > s.n_kv_heads ? s.n_heads : s.n_kv_heads) > INT_MAX) return "more than 2^31 - 1 heads of tokens";
    return nullptr;
}
static NormArgs norm_args(const NormSizes &s, const int32_t *positions, const float *rope) {
    NormArgs A = {};
    A.positions = positions;
    A.rope = reinterpret_cast<const float2 *>(rope);
    A.tokens = (unsigned)s.batch * (unsigned)s.m;
    A.m = (unsigned)s.m;
    A.by_m = Divisor(A.m);
    A.d = s.d_head; A.rope_n = s.rope_positions; A.rot = rope ? s.rope_dims : 0;
    A.gain_dtype = s.gain_dtype; A.eps = s.eps; A.inv_d = 1.f / (float)s.d_head;
    A.t[0].heads = s.n_heads;
    A.t[1].heads = s.n_kv_heads;
    return A;
}

static size_t up(size_t n) { return (n + 255) & ~(size_t)255; }
static size_t gain_parts(int d) { return up((size_t)(norm_sms() * kNormBlocks + 3) * d * 4); }

}  // namespace xsm

using namespace xsm;

xsm_status xsm_norm_rotate(const xsm_norm_rotate_args *a, void *cuda_stream) {
    if (!a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    const NormSizes s = {a->batch, a->m, a->n_heads, a->n_kv_heads, a->d_head, a->dtype, a->gain_dtype, a->rope_positions, a->rope_dims, a->eps};
    if (const char *w = wrong_sizes(s, a->rope)) return op_failed(XSM_ERR_INVALID_ARG, w);
    if (a->batch == 0 || a->m == 0 || a->n_heads + a->n_kv_heads == 0) return XSM_OK;
    if ((a->n_heads && (!a->q || !a->q_out || !a->q_gain)) || (a->n_kv_heads && (!a->k || !a->k_out || !a->k_gain))) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    NormArgs A = norm_args(s, a->positions, a->rope);
    const void *x[2] = {a->q, a->k}, *gain[2] = {a->q_gain, a->k_gain};
    void *out[2] = {a->q_out, a->k_out};
    const int64_t *xs[2] = {a->q_stride, a->k_stride}, *os[2] = {a->q_out_stride, a->k_out_stride};
    const int es = element_size(a->dtype);
    bool wide = A.rot % (32 / es) == 0 && (uintptr_t)a->rope % 16 == 0;
    for (int i = 0; i < 2; ++i) {
        NormTensor &t = A.t[i];
        if (!t.heads) continue;
        t.x = x[i]; t.out = out[i]; t.gain = gain[i];
        for (int k = 0; k < 3; ++k) { t.xs[k] = xs[i][k]; t.os[k] = os[i][k]; }
        if (((uintptr_t)t.x | (uintptr_t)t.out) % es || (uintptr_t)t.gain % element_size(a->gain_dtype)) return op_failed(XSM_ERR_INVALID_ARG, "tensors must be aligned to their elements");
        wide = wide && aligned(t.x, xs[i], es) && aligned(t.out, os[i], es);
    }
    const int blocks = cut_norm(A, lanes_of(A.d, es, wide));
    const Pages P = {};
    cudaError_t e = cudaSuccess;
    with_dtype(a->dtype, [&](auto in) { e = launch_norm<decltype(in), decltype(in), NM_FORWARD>(A, P, blocks, wide, a->interleaved != 0, (cudaStream_t)cuda_stream); });
    return launched(e);
}

size_t xsm_norm_rotate_grad_workspace(int d_head) { return d_head < 1 || d_head > 256 ? 0 : gain_parts(d_head); }

xsm_status xsm_norm_rotate_grad(const xsm_norm_rotate_grad_args *a, void *cuda_stream) {
    if (!a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    const NormSizes s = {a->batch, a->m, a->n_heads, a->n_kv_heads, a->d_head, a->dtype, a->gain_dtype, a->rope_positions, a->rope_dims, a->eps};
    if (const char *w = wrong_sizes(s, a->rope)) return op_failed(XSM_ERR_INVALID_ARG, w);
    if (a->n_heads + a->n_kv_heads == 0) return XSM_OK;
    if ((a->n_heads && (!a->q_gain || !a->d_q_gain)) || (a->n_kv_heads && (!a->k_gain || !a->d_k_gain))) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    const int gs = element_size(a->gain_dtype);
    if ((uintptr_t)(a->n_heads ? a->d_q_gain : nullptr) % gs || (uintptr_t)(a->n_kv_heads ? a->d_k_gain : nullptr) % gs) return op_failed(XSM_ERR_INVALID_ARG, "tensors must be aligned to their elements");
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    if (a->batch == 0 || a->m == 0) {
        cudaError_t e = a->n_heads ? cudaMemsetAsync(a->d_q_gain, 0, (size_t)a->d_head * gs, st) : cudaSuccess;
        if (e == cudaSuccess && a->n_kv_heads) e = cudaMemsetAsync(a->d_k_gain, 0, (size_t)a->d_head * gs, st);
        return launched(e);
    }
    if ((a->n_heads && (!a->q || !a->g_q || !a->d_q)) || (a->n_kv_heads && (!a->k || !a->g_k || !a->d_k)) || !a->workspace || !a->counters) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if ((uintptr_t)a->workspace % 16 || (uintptr_t)a->counters % 4) return op_failed(XSM_ERR_INVALID_ARG, "workspace must be 16-byte aligned, counters to their elements");
    if (a->workspace_bytes < (int64_t)gain_parts(a->d_head)) return op_failed(XSM_ERR_CAPACITY, "the workspace is too small");
    NormArgs A = norm_args(s, a->positions, a->rope);
    const void *x[2] = {a->q, a->k}, *g[2] = {a->g_q, a->g_k}, *gain[2] = {a->q_gain, a->k_gain};
    void *out[2] = {a->d_q, a->d_k}, *d_gain[2] = {a->d_q_gain, a->d_k_gain};
    const int64_t *xs[2] = {a->q_stride, a->k_stride}, *ys[2] = {a->g_q_stride, a->g_k_stride}, *os[2] = {a->d_q_stride, a->d_k_stride};
    const int es = element_size(a->dtype);
    bool wide = A.rot % (32 / es) == 0 && (uintptr_t)a->rope % 16 == 0;
    for (int i = 0; i < 2; ++i) {
        NormTensor &t = A.t[i];
        if (!t.heads) continue;
        t.x = x[i]; t.g = g[i]; t.out = out[i]; t.gain = gain[i];
        for (int k = 0; k < 3; ++k) { t.xs[k] = xs[i][k]; t.gs[k] = ys[i][k]; t.os[k] = os[i][k]; }
        if (((uintptr_t)t.x | (uintptr_t)t.g | (uintptr_t)t.out) % es || (uintptr_t)t.gain % gs) return op_failed(XSM_ERR_INVALID_ARG, "tensors must be aligned to their elements");
        wide = wide && aligned(t.x, xs[i], es) && aligned(t.g, ys[i], es) && aligned(t.out, os[i], es);
    }
    const int blocks = cut_norm(A, lanes_of(A.d, es, wide));
    A.t[0].part = (float *)a->workspace;
    A.t[1].part = A.t[0].part + (size_t)A.t[0].blocks * A.d;
    for (int i = 0; i < 2; ++i) A.t[i].d_gain = d_gain[i];
    // (few blocks: the last one adds up; of 296 that is 6 us longer than a kernel of its own)
    A.counter = blocks <= 64 ? a->counters : nullptr;
    const Pages P = {};
    cudaError_t e = cudaSuccess;
    with_dtype(a->dtype, [&](auto in) { e = launch_norm<decltype(in), decltype(in), NM_GRAD>(A, P, blocks, wide, a->interleaved != 0, st); });
    if (e == cudaSuccess && !A.counter) {
        GainArgs R;
        for (int i = 0; i < 2; ++i) { R.part[i] = A.t[i].part; R.out[i] = A.t[i].heads ? d_gain[i] : nullptr; R.blocks[i] = A.t[i].blocks; }
        R.d = A.d; R.dtype = A.gain_dtype;
        e = launch_early(gain_kernel, dim3(A.d / 32, 2), dim3(1024), 0, st, R);
    }
    return launched(e);
}

xsm_status xsm_kv_append_norm(const xsm_kv *kv, const xsm_kv_append_args *a, const xsm_head_norm *n, void *cuda_stream) {
    if (!kv || !a || !n) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (a->batch < 0 || a->m < 0 || a->n_heads < 0 || a->max_pages < 0) return op_failed(XSM_ERR_INVALID_ARG, "batch, m, n_heads and max_pages must not be negative");
    if (a->n_heads > 4096) return op_failed(XSM_ERR_INVALID_ARG, "n_heads must not exceed 4096");
    if (const char *w = wrong_norm(a->in_dtype, n->gain_dtype, n->eps, a->rope, a->rope_positions, a->rope_dims, kv->cfg.d_head)) return op_failed(XSM_ERR_INVALID_ARG, w);
    const long long tokens = (long long)a->batch * a->m;
    if (tokens == 0) return XSM_OK;
    const int most = a->n_heads > kv->cfg.n_kv_heads ? a->n_heads : kv->cfg.n_kv_heads;
    if (tokens * most > INT_MAX) return op_failed(XSM_ERR_INVALID_ARG, "more than 2^31 - 1 heads of tokens");
    if (!a->k || !a->v || (!a->block_table && a->max_pages) || !a->starts || !n->k_gain) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (a->n_heads && (!a->q || !a->q_out || !n->q_gain)) return op_failed(XSM_ERR_INVALID_ARG, "n_heads without q, q_out or q_gain");
    const NormSizes s = {a->batch, a->m, a->n_heads, kv->cfg.n_kv_heads, kv->cfg.d_head, a->in_dtype, n->gain_dtype, a->rope_positions, a->rope_dims, n->eps};
    NormArgs A = norm_args(s, nullptr, a->rope);
    A.starts = a->starts; A.counts = a->counts;
    A.t[2].heads = kv->cfg.n_kv_heads;
    const void *x[3] = {a->q, a->k, a->v}, *gain[3] = {n->q_gain, n->k_gain, nullptr};
    const int64_t *xs[3] = {a->q_stride, a->k_stride, a->v_stride};
    const int es = element_size(a->in_dtype);
    bool wide = A.rot % (32 / es) == 0 && (uintptr_t)a->rope % 16 == 0;
    for (int i = 0; i < 3; ++i) {
        NormTensor &t = A.t[i];
        if (!t.heads) continue;
        t.x = x[i]; t.gain = gain[i];
        for (int k = 0; k < 3; ++k) { t.xs[k] = xs[i][k]; t.os[k] = a->q_out_stride[k]; }
        if ((uintptr_t)t.x % es || (uintptr_t)t.gain % element_size(n->gain_dtype)) return op_failed(XSM_ERR_INVALID_ARG, "tensors must be aligned to their elements");
        wide = wide && aligned(t.x, xs[i], es);
    }
    if (a->n_heads) {
        A.t[0].out = a->q_out;
        if ((uintptr_t)a->q_out % es) return op_failed(XSM_ERR_INVALID_ARG, "tensors must be aligned to their elements");
        wide = wide && aligned(a->q_out, a->q_out_stride, es);
    }
    const Pages P = pages_of(*kv, a->block_table, a->table_stride, a->max_pages);
    const int blocks = cut_norm(A, lanes_of(A.d, es, wide));
    cudaError_t e = cudaSuccess;
    with_dtype(a->in_dtype, [&](auto in) {
        with_dtype(kv->cfg.dtype, [&](auto stored) { e = launch_norm<decltype(in), decltype(stored), NM_APPEND>(A, P, blocks, wide, a->interleaved != 0, (cudaStream_t)cuda_stream); });
    });
    return launched(e);
}
