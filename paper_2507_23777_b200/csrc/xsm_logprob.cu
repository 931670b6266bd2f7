// Log probabilities of given tokens with entropy and top alternatives, and their gradient by the logits.
//
// Forward: one pass over a row with a running maximum m, s = sum exp((z - m)/T) and t = sum exp((z - m)/T) (z - m)/T; then
// lse = m/T + log s, logprob = (z_token - m)/T - log s, entropy = log s - t/s.  A block of 128 threads takes a row; where
// there are fewer rows than keep the chip busy a cluster of blocks takes a part of the row each and joins through shared memory.
// Alternatives: the largest logits of every thread bound the k-th largest of the row from below; what reaches the bound, usually little more
// than k logits, is collected in a second look at the row (out of registers, or the caches) and sorted by counting.
// Backward: one pass, every element from its own logit and a few numbers of its row.
//
// What bounds them.  Many rows: forward the instructions (8192 x 8192 of bf16 31 us where the bytes take 21: five and a half an element, of which
// one is the exponential, and a row's 700 warp instructions of beginning and end), backward memory (42 us; 41 without any
// arithmetic).  Two numbers an instruction (f32x2) took the pair from 111 to 78 us, blocks of 128 threads with four pieces of 16 bits
// (eight of 32) under way to 72.  Few rows: a chain: 4.3 us for 5 x 4096 with 5 alternatives, of which a launch is 2; 96 x 131071 takes 8.0
// without alternatives (the bytes 3.9) and 15.9 with 20, the parts' alternatives one behind the other: bound, second look, order, cluster, order.
#include "xsm_ops.h"

#include <math.h>

#include <type_traits>

namespace xsm {

constexpr int kMaxTop = 32;
constexpr int kBlock = 128;               // threads
constexpr int kWarpRowBytes = 8192;       // rows up to this size are a warp's each, where there are many

struct LogprobArgs {
    const void *logits, *tokens;
    float *logprob, *entropy, *lse;
    int *top_ids;
    float *top_logprobs;
    long long row_ld, token_ld;
    int rows, vocab, token_bytes, top;
    int cuts, cut_shift;                  // blocks of a cluster, each with a part of the row: 2^cut_shift
    float inv_t;
};

__device__ __forceinline__ long long token_at(const void *tokens, int bytes, long long i) {
    return bytes == 8 ? reinterpret_cast<const long long *>(tokens)[i] : reinterpret_cast<const int *>(tokens)[i];
}

// A number that orders as the logit does; NaN comes last (0), zeros of either sign are the same.
__device__ __forceinline__ unsigned order_of(float z) {
    const unsigned u = __float_as_uint(z + 0.f);
    return z != z ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_order(unsigned o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
// (logit descending, index ascending): the first of them is the largest
__device__ __forceinline__ unsigned long long rank_key(float z, int i) { return ((unsigned long long)order_of(z) << 32) | (unsigned)~i; }

// The elements of a run of a row as single ones up to a 16-byte boundary, 16-byte pieces, and single ones again.
template <typename T> struct Pieces {
    static constexpr int n = 16 / sizeof(T);
    const T *p;
    int head, pieces, tail;
    __device__ __forceinline__ Pieces(const T *first, int count) : p(first) {
        head = min(count, (int)((16 - ((uintptr_t)first & 15)) & 15) / (int)sizeof(T));
        pieces = (count - head) / n;
        tail = count - head - pieces * n;
    }
    __device__ __forceinline__ uint4 piece(int i) const { return reinterpret_cast<const uint4 *>(p + head)[i]; }
    // thread i's single element, if it has one: its index in the run, or -1 (there are fewer than eight at each end)
    __device__ __forceinline__ int single(int i) const { return i < head ? i : i >= 8 && i < 8 + tail ? head + pieces * n + i - 8 : -1; }
};
// two fp32 numbers that are worked on together
typedef unsigned long long Two;
__device__ __forceinline__ Two two(float a, float b) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 apart(Two v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// elements 2i and 2i + 1 of a piece
template <typename T> __device__ __forceinline__ float2 pair(const uint4 &v, int i) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    else if constexpr (std::is_same<T, bf16>::value) return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    else return __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
}
template <typename T> __device__ __forceinline__ void widen(const uint4 &v, float (&x)[Pieces<T>::n]) {
#pragma unroll
    for (int i = 0; i < Pieces<T>::n / 2; ++i) {
        const float2 f = pair<T>(v, i);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
// largest element of a piece (NaN aside)
template <typename T> __device__ __forceinline__ float largest(const uint4 &v) {
    if constexpr (sizeof(T) == 4) {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    } else if constexpr (std::is_same<T, bf16>::value) {
        const __nv_bfloat162 *h = reinterpret_cast<const __nv_bfloat162 *>(&v);
        const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__low2float(m), __high2float(m));
    } else {
        const __half2 *h = reinterpret_cast<const __half2 *>(&v);
        const __half2 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
}
template <typename T> __device__ __forceinline__ uint4 nothing() {      // -infinity everywhere
    const unsigned w = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, bf16>::value ? 0xff80ff80u : 0xfc00fc00u;
    return make_uint4(w, w, w, w);
}

// Running maximum m and sums of a part of a row: s = sum 2^x, t = sum 2^x x, x = (z - m) c with c = log2(e) / T.
struct Part {
    float m, s, t;
    // the same sums against a maximum that is no smaller
    __device__ __forceinline__ void rebase(float top, float c) {
        const float d = fmaxf((m - top) * c, -1e30f), f = m == -INFINITY ? 0.f : ex2(d);      // (nothing yet: s = t = 0, but -infinity times 0 is none)
        t = f * (t + s * d);
        s *= f;
        m = top;
    }
    // over the first `lanes` lanes of a warp, in every one of them
    __device__ __forceinline__ void join(int lanes, float c) {
        float top = m;
        for (int o = lanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (m != top) rebase(top, c);
        for (int o = lanes / 2; o > 0; o >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, o);
            t += __shfl_xor_sync(0xffffffffu, t, o);
        }
    }
};
// Two more elements.  (The difference first: that of the maximum to itself is zero, and nothing overflows.)
__device__ __forceinline__ void take(float2 z, Two minus_m, Two c, Two &s, Two &t) {
    const float2 x = apart(mul2(add2(two(z.x, z.y), minus_m), c));
    const Two e = two(ex2(x.x), ex2(x.y));
    s = add2(s, e);
    t = fma2(e, two(fmaxf(x.x, -1e30f), fmaxf(x.y, -1e30f)), t);
}

// Warps that share a row: a block's four, or one, and the block has four rows.
template <int W> __device__ __forceinline__ void meet() {
    if (W == 1) __syncwarp();
    else __syncthreads();
}
template <int W> struct RowShared {
    static constexpr int room = W == 1 ? 256 : 512;
    __align__(16) unsigned long long candidate[room + 8];
    unsigned long long key[W], best[kMaxTop];
    Part part[W];
    unsigned bound[W];
    int found;
    // of a cluster's first block: what every block has found
    __align__(16) unsigned long long gathered[W == 1 ? 1 : 8 * kMaxTop + 8];
    Part parts[W == 1 ? 1 : 8];
};

// how many of n keys are larger than this one (what lies behind them up to a multiple of eight is zero)
__device__ __forceinline__ int larger(const unsigned long long *keys, int n, unsigned long long key) {
    int count = 0;
    for (int k = 0; k < n; k += 8) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(keys + k + 2 * q);
            count += (v.x > key) + (v.y > key);
        }
    }
    return count;
}

// The `top` largest of a run one after the other, each the largest below the one before: for rows whose bound collects too many (all
// alike, or -infinity) or too few (NaN).
template <typename T, int W> __device__ __noinline__ void best_one_by_one(const T *z, int count, int index0, int top, RowShared<W> &sh) {
    const int tid = W == 1 ? threadIdx.x & 31 : threadIdx.x;
    unsigned long long last = ~0ull;
    for (int k = 0; k < top; ++k) {
        unsigned long long best = 0;
        for (int i = tid; i < count; i += 32 * W) {
            const unsigned long long key = rank_key(to_f(z[i]), index0 + i);
            if (key < last && key > best) best = key;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const unsigned long long w = __shfl_xor_sync(0xffffffffu, best, o);
            best = w > best ? w : best;
        }
        meet<W>();
        if ((tid & 31) == 0) sh.key[tid >> 5] = best;
        meet<W>();
        last = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) last = sh.key[w] > last ? sh.key[w] : last;
        if (tid == 0) sh.best[k] = last;
    }
    meet<W>();
}

template <typename T, bool kTop, int W> __global__ void __launch_bounds__(kBlock, kTop || sizeof(T) == 4 ? 8 : 12) logprob_kernel(const __grid_constant__ LogprobArgs A) {
    constexpr int N = Pieces<T>::n, kThreads = 32 * W, kAhead = 32 / N;      // pieces that a thread has under way: 32 logits
    __shared__ RowShared<W> shared[W == 1 ? kBlock / 32 : 1];
    chain_go();
    chain_wait();
    RowShared<W> &sh = shared[W == 1 ? threadIdx.x >> 5 : 0];
    const int tid = W == 1 ? threadIdx.x & 31 : threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int cut = W == 1 ? 0 : blockIdx.x & (A.cuts - 1);          // (clusters start at multiples of their size: this is the rank)
    const long long row = W == 1 ? (long long)blockIdx.x * (kBlock / 32) + (threadIdx.x >> 5) : blockIdx.x >> A.cut_shift;
    if (W == 1 && row >= A.rows) return;
    const T *z = reinterpret_cast<const T *>(A.logits) + row * A.row_ld;
    const int i0 = W == 1 ? 0 : (int)(((long long)A.vocab * cut) >> A.cut_shift);
    const int count = (W == 1 ? A.vocab : (int)(((long long)A.vocab * (cut + 1)) >> A.cut_shift)) - i0;
    const Pieces<T> in(z + i0, count);
    const float c = A.inv_t * kLog2e;
    if (W > 1 && A.cuts > 1) cluster_arrive_relaxed();          // (nothing is told but that this block runs)
    if (kTop && tid == 0) sh.found = 0;
    float given = 0.f;
    long long token = -1;
    if (tid == 0 && cut == 0) {
        token = token_at(A.tokens, A.token_bytes, row * A.token_ld);
        if (token < 0 || token >= A.vocab) token = -1;
        if (token >= 0) given = to_f(z[token]);
    }

    Part a{-INFINITY, 0.f, 0.f};
    const int one = in.single(tid);
    const float single = one >= 0 ? to_f(in.p[one]) : -INFINITY;
    uint4 v[kAhead];
    // kTop: the largest logits of this thread's best pieces, the best two's places
    float best[3] = {-INFINITY, -INFINITY, -INFINITY};
    int place[2] = {in.pieces, in.pieces};
    for (int at = 0; at == 0 || at < in.pieces; at += kThreads * kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = at + u * kThreads + tid;
            v[u] = i < in.pieces ? in.piece(i) : nothing<T>();
        }
        float top = at == 0 ? single : a.m;
        if (!(top == top)) top = a.m;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const float x = largest<T>(v[u]);
            top = fmaxf(top, x);
            if (kTop) {
                const bool first = x > best[0], second = x > best[1];
                best[2] = second ? best[1] : fmaxf(best[2], x);
                place[1] = first ? place[0] : second ? at + u * kThreads + tid : place[1];
                best[1] = first ? best[0] : fmaxf(best[1], x);
                place[0] = first ? at + u * kThreads + tid : place[0];
                best[0] = fmaxf(best[0], x);
            }
        }
        if (top > a.m) a.rebase(top, c);
        const float ref = a.m == -INFINITY ? 0.f : a.m;
        const Two cc = two(c, c), minus = two(-ref, -ref);
        Two s = two(0.f, 0.f), t = s;
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int i = 0; i < N / 2; ++i) take(pair<T>(v[u], i), minus, cc, s, t);
        if (at == 0) take(make_float2(single, -INFINITY), minus, cc, s, t);
        const float2 s2 = apart(s), t2 = apart(t);
        a.s += s2.x + s2.y;
        a.t += t2.x + t2.y;
    }
    const unsigned mine = kTop ? order_of(a.m) : 0u;
    const int full_warps = min(W, max(1, in.pieces / 32));
    a.join(32, c);
    unsigned bound = 0;
    if (kTop) {
        // the j-th largest of the maxima of a warp's threads, as many as make `top` over the warps that are full of pieces: at least `top` logits
        // reach the least of these warps' bounds
        bool in_play = true;
        for (int j = 0; j < A.top; j += full_warps) {
            bound = __reduce_max_sync(0xffffffffu, in_play ? mine : 0u);
            const unsigned who = __ballot_sync(0xffffffffu, in_play && mine == bound);
            if (who && lane == __ffs(who) - 1) in_play = false;
        }
        if (W > 1 && lane == 0) sh.bound[warp] = bound;
    }
    if (W > 1) {
        if (lane == 0) sh.part[warp] = a;
        meet<W>();
        if (warp == 0) {
            a = lane < W ? sh.part[lane] : Part{-INFINITY, 0.f, 0.f};
            a.join(W, c);
        }
    } else {
        meet<W>();
    }
    if (kTop) {
        if (W > 1) {
            bound = sh.bound[0];
#pragma unroll
            for (int w = 1; w < W; ++w) if (w < full_warps) bound = min(bound, sh.bound[w]);
        }
        const float least = of_order(bound);
        const int want = min(A.top, count);
        int found = 0;
        if (bound > order_of(-INFINITY) || count <= RowShared<W>::room) {
            auto offer = [&](float x, int i) {
                if (x >= least) {
                    const int at = atomicAdd(&sh.found, 1);
                    if (at < RowShared<W>::room) sh.candidate[at] = rank_key(x, i0 + i);
                }
            };
            auto offer_piece = [&](const uint4 &w, int i) {
                if (!(largest<T>(w) >= least)) return;
                float x[N];
                widen<T>(w, x);
#pragma unroll
                for (int k = 0; k < N; ++k) offer(x[k], in.head + i * N + k);
            };
            if (one >= 0) offer(single, one);
            if (in.pieces <= kThreads * kAhead) {             // the row's pieces are still in registers
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int i = u * kThreads + tid;
                    if (i < in.pieces) offer_piece(v[u], i);
                }
            } else {
                // a second look at the pieces that reach the bound: a thread's best two, and where there may be more all of its pieces, one for every lane
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const bool worth = best[q] >= least && best[2] < least && place[q] < in.pieces;
                    v[q] = worth ? in.piece(place[q]) : nothing<T>();
                }
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    if (best[q] >= least && best[2] < least && place[q] < in.pieces) offer_piece(v[q], place[q]);
                unsigned who = __ballot_sync(0xffffffffu, best[2] >= least);
                while (who) {
                    const int p = warp * 32 + __ffs(who) - 1;
                    who &= who - 1;
                    for (int at = lane * kThreads + p; at < in.pieces; at += 32 * kThreads) offer_piece(in.piece(at), at);
                }
            }
            meet<W>();
            found = sh.found;
            if (found <= RowShared<W>::room) {
                if (tid < 8) sh.candidate[found + tid] = 0;
                meet<W>();
            }
        }
        if (found < want || found > RowShared<W>::room) {
            best_one_by_one<T, W>(z + i0, count, i0, want, sh);
        } else {
            for (int i = tid; i < found; i += kThreads) {
                const unsigned long long key = sh.candidate[i];
                const int before = larger(sh.candidate, found, key);
                if (before < want) sh.best[before] = key;
            }
        }
        if (tid < A.top && tid >= want) sh.best[tid] = 0;                 // a part of the row that is shorter than `top`
        meet<W>();
    }
    if (W > 1 && A.cuts > 1) {
        // every block writes what it has found to the first one's shared memory
        __syncwarp();
        cluster_wait();
        if (kTop && tid < A.top) st_cluster_u64(map_rank(smem_u32(&sh.gathered[cut * A.top + tid]), 0), sh.best[tid]);
        if (tid == 0) {
            const uint32_t to = map_rank(smem_u32(&sh.parts[cut]), 0);
            st_cluster_f32(to, a.m);
            st_cluster_f32(to + 4, a.s);
            st_cluster_f32(to + 8, a.t);
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        if (cut != 0) return;
        if (warp == 0) {
            a = lane < A.cuts ? sh.parts[lane] : Part{-INFINITY, 0.f, 0.f};
            a.join(8, c);
        }
        if (kTop) {
            const int n = A.cuts * A.top;
            if (tid < 8) sh.gathered[n + tid] = 0;
            meet<W>();
            for (int i = tid; i < n; i += kThreads) {
                const unsigned long long key = sh.gathered[i];
                const int before = larger(sh.gathered, n, key);
                if (key != 0 && before < A.top) sh.best[before] = key;
            }
            meet<W>();
        }
    }
    // lane 0 has the row's sums
    const float log_s = logf(a.s), ref = a.m == -INFINITY ? 0.f : a.m;
    const bool none = a.s == 0.f;                                     // nothing but -infinity
    if (tid == 0) {
        A.logprob[row] = token < 0 ? 0.f : none ? -INFINITY : (given - ref) * A.inv_t - log_s;
        A.entropy[row] = none ? 0.f : log_s - a.t / a.s * 0.69314718055994531f;
        A.lse[row] = none ? -INFINITY : ref * A.inv_t + log_s;
    }
    if (kTop && warp == 0) {
        const float m0 = __shfl_sync(0xffffffffu, ref, 0), log0 = __shfl_sync(0xffffffffu, none ? INFINITY : log_s, 0);
        if (lane < A.top) {
            const unsigned long long key = sh.best[lane];
            A.top_ids[row * A.top + lane] = (int)~(unsigned)key;
            // (its logit out of the key, where NaN has none)
            const float x = (key >> 32) == 0 ? NAN : of_order((unsigned)(key >> 32));
            A.top_logprobs[row * A.top + lane] = log0 == INFINITY ? -INFINITY : (x - m0) * A.inv_t - log0;
        }
    }
}

struct GradArgs {
    const void *logits, *tokens;
    const float *logprob, *lse, *entropy;      // logprob may be missing
    const int *top_ids;
    const float *g_logprob, *g_entropy, *g_lse, *g_top;
    void *d_logits;
    long long row_ld, token_ld, gl_ld, ge_ld, gs_ld, d_ld;
    int rows, vocab, token_bytes, top, per_block;      // per_block: pieces of a row that a block takes
    float inv_t, temperature;
};

// The numbers of a row that its elements' gradients are made of: with x = log2 p = (z - ref) c + off, the gradient is -p (total' + ge' x), where
// total' has the entropy's share and everything the factor 1/T.  The reference is the token's logit, which is known with its log probability, so that what all
// logits have in common does not matter (an lse of 1000 is rounded to 3e-5, p to as much); where there is no token, or its log probability is larger than the lse
// (a masked one's), it is lse T.  A row with nothing left: off = -infinity, so p = 0, and the rest zero.
struct RowGrad {
    float c, minus_ref, off, total, ge;
    __device__ __forceinline__ float of(float z) const {
        const float x = fmaf(z + minus_ref, c, off);
        return -ex2(x) * fmaf(ge, fmaxf(x, -1e3f), total);                // (p is zero below -150: the bound only keeps 0 * -infinity out)
    }
};

template <typename T> __device__ __forceinline__ uint4 narrow(const float (&x)[Pieces<T>::n]) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            w[i] = __float_as_uint(x[i]);
        } else if constexpr (std::is_same<T, bf16>::value) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const unsigned *>(&h);
        } else {
            w[i] = pack_f16x2(x[2 * i], x[2 * i + 1]);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// W warps take per_block pieces of a row (and the first of its row the single elements at both ends).  What falls on single logits directly,
// the token's and the alternatives' gradients, is a list; when all elements are written, the listed ones among them are written again with
// it, from logits that were read before (the gradient may take the place of the logits).
template <typename T, bool kTop, int W> __global__ void __launch_bounds__(kBlock) logprob_grad_kernel(const __grid_constant__ GradArgs A) {
    constexpr int N = Pieces<T>::n, kLoads = 4, kThreads = 32 * W, kGroups = W == 1 ? kBlock / 32 : 1;
    __shared__ RowGrad rows[kGroups];
    __shared__ int ids[kGroups][kMaxTop + 1];
    __shared__ float gs[kGroups][kMaxTop + 1];
    chain_go();
    chain_wait();
    const int tid = W == 1 ? threadIdx.x & 31 : threadIdx.x, group = W == 1 ? threadIdx.x >> 5 : 0;
    int *const s_id = ids[group];
    float *const s_g = gs[group];
    const long long row = (long long)blockIdx.x * kGroups + group;
    if (W == 1 && row >= A.rows) return;
    const T *z = reinterpret_cast<const T *>(A.logits) + row * A.row_ld;
    T *out = reinterpret_cast<T *>(A.d_logits) + row * A.d_ld;
    const Pieces<T> in(z, A.vocab);
    const int first = blockIdx.y * A.per_block, last = min(in.pieces, first + A.per_block);
    uint4 v[kLoads];
    auto fetch = [&](int at) {
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int i = at + u * kThreads + tid;
            if (i < last) v[u] = in.piece(i);
        }
    };
    fetch(first);
    const int one = blockIdx.y == 0 ? in.single(tid) : -1;
    const float single = one >= 0 ? to_f(in.p[one]) : 0.f;
    const int listed = kTop ? A.top + 1 : 1;
    if (tid < 32) {
        const float lse = A.lse[row], logprob = A.logprob ? A.logprob[row] : 0.f;
        const long long token = token_at(A.tokens, A.token_bytes, row * A.token_ld);
        const bool has = token >= 0 && token < A.vocab;
        const bool by_token = A.logprob && has && fabsf(logprob) < fabsf(lse);      // (an lse may be beyond fp32 where the differences are not)
        const bool none = lse == -INFINITY && !by_token;
        float more = 0.f;
        if (kTop) {
            if (tid < A.top) {
                more = none ? 0.f : A.g_top[row * A.top + tid] * A.inv_t;
                s_id[tid + 1] = A.top_ids[row * A.top + tid];
                s_g[tid + 1] = more;
            }
            more = warp_sum(more);
        }
        if (tid == 0) {
            const float g = A.g_logprob && has && !none ? A.g_logprob[row * A.gl_ld] * A.inv_t : 0.f;
            const float ge = A.g_entropy && !none ? A.g_entropy[row * A.ge_ld] * A.inv_t : 0.f;
            s_id[0] = has ? (int)token : -1;
            s_g[0] = g;
            RowGrad r;
            r.ge = ge * 0.69314718055994531f;
            r.total = none ? 0.f : g + more - (A.g_lse ? A.g_lse[row * A.gs_ld] * A.inv_t : 0.f) + (A.g_entropy ? ge * A.entropy[row] : 0.f);
            r.off = none ? -INFINITY : by_token ? logprob * kLog2e : 0.f;
            r.minus_ref = by_token ? -to_f(z[token]) : none ? 0.f : -lse * A.temperature;
            r.c = A.inv_t * kLog2e;
            rows[group] = r;
        }
    }
    meet<W>();
    const RowGrad r = rows[group];
    // this thread's entries of the list whose logits are of this block's part, and these
    constexpr int kEntries = W == 1 ? 2 : 1;
    static_assert(kEntries * kThreads > kMaxTop, "the list has a thread for every entry");
    float listed_z[kEntries];
    int listed_id[kEntries];
#pragma unroll
    for (int q = 0; q < kEntries; ++q) {
        const int k = tid + q * kThreads;
        int id = k < listed ? s_id[k] : -1;
        if (id >= A.vocab) id = -1;
        if (id >= in.head && id < in.head + in.pieces * N) {
            const int piece = (id - in.head) / N;
            if (piece < first || piece >= last) id = -1;
        } else if (blockIdx.y != 0) {
            id = -1;
        }
        listed_id[q] = id;
        listed_z[q] = id >= 0 ? to_f(z[id]) : 0.f;
    }
    meet<W>();
    if (one >= 0) out[one] = rounded<T>(r.of(single));
    const bool alike = (((uintptr_t)z ^ (uintptr_t)out) & 15) == 0;
    const Two cc = two(r.c, r.c), minus = two(r.minus_ref, r.minus_ref), off = two(r.off, r.off), ge = two(-r.ge, -r.ge), total = two(-r.total, -r.total);
    for (int at = first; at < last; at += kThreads * kLoads) {
        if (at != first) fetch(at);
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int i = at + u * kThreads + tid, e = in.head + i * N;
            if (i >= last) continue;
            float d[N];
#pragma unroll
            for (int k = 0; k < N / 2; ++k) {
                const float2 y = pair<T>(v[u], k), x = apart(fma2(add2(two(y.x, y.y), minus), cc, off));
                const Two w = fma2(ge, two(fmaxf(x.x, -1e3f), fmaxf(x.y, -1e3f)), total);
                const float2 f = apart(mul2(two(ex2(x.x), ex2(x.y)), w));
                d[2 * k] = f.x;
                d[2 * k + 1] = f.y;
            }
            if (alike) {
                *reinterpret_cast<uint4 *>(out + e) = narrow<T>(d);
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) out[e + k] = rounded<T>(d[k]);
            }
        }
    }
    meet<W>();
#pragma unroll
    for (int q = 0; q < kEntries; ++q) {
        const int id = listed_id[q];
        if (id < 0) continue;
        float d = r.of(listed_z[q]);
        for (int k = 0; k < listed; ++k) d += s_id[k] == id ? s_g[k] : 0.f;
        out[id] = rounded<T>(d);
    }
}

// Blocks that share a row, as a power of two: as many as the chip takes at a time (six an SM) over the rows, each with 4096 logits at least.
// (96 x 131071 without alternatives: a block a row 13.5 us, two 11.5, four and eight 8.0.)
static int cut_shift_of(int rows, int vocab, int sms) {
    int shift = 0;
    while (shift < 3 && ((long long)rows << (shift + 1)) <= 6LL * sms && (vocab >> (shift + 1)) >= 4096) ++shift;
    return shift;
}

static cudaError_t sm_count(int *sms) {
    static int known[kMaxDevices];            // (a race writes the same number twice)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    if (known[dev] == 0 && (e = cudaDeviceGetAttribute(&known[dev], cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    *sms = known[dev];
    return cudaSuccess;
}

// Short rows are a warp's each, where there are enough of them (16000 x 1000 with its gradient 56 us as blocks, 23 as warps; 16000 x 3001 78 and 57;
// 8192 x 8192, past the line, 72 as blocks and 76 as warps).
static bool by_warp(int rows, long long row_bytes, int sms) { return row_bytes <= kWarpRowBytes && rows >= 4 * sms; }

template <typename T, bool kTop> static cudaError_t launch_logprob(const LogprobArgs &A, bool warps, cudaStream_t st) {
    if (warps) return launch_early(logprob_kernel<T, kTop, 1>, dim3((A.rows + kBlock / 32 - 1) / (kBlock / 32)), dim3(kBlock), 0, st, A);
    if (A.cuts == 1) return launch_early(logprob_kernel<T, kTop, kBlock / 32>, dim3(A.rows), dim3(kBlock), 0, st, A);
    cudaLaunchConfig_t cfg = {};             // (clusters gain nothing by starting early: 96 x 131071 17.2 us without, 19.9 with)
    cfg.gridDim = dim3((unsigned)(A.rows * A.cuts));
    cfg.blockDim = dim3(kBlock);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = A.cuts;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, logprob_kernel<T, kTop, kBlock / 32>, A);
}
template <typename T, bool kTop> static cudaError_t launch_grad(const GradArgs &A, int blocks, bool warps, cudaStream_t st) {
    if (warps) return launch_early(logprob_grad_kernel<T, kTop, 1>, dim3((A.rows + kBlock / 32 - 1) / (kBlock / 32)), dim3(kBlock), 0, st, A);
    return launch_early(logprob_grad_kernel<T, kTop, kBlock / 32>, dim3(A.rows, blocks), dim3(kBlock), 0, st, A);
}

static const char *check_logits(const void *logits, const void *tokens, int rows, int vocab, int dtype, int token_bytes, int top, float temperature) {
    if (rows < 0 || vocab < 1) return "rows must not be negative and vocab must be positive";
    if (!is_dtype(dtype)) return "dtype must be 0 (fp32), 1 (bf16) or 2 (fp16)";
    if (token_bytes != 4 && token_bytes != 8) return "token_bytes must be 4 or 8";
    if (top < 0 || top > kMaxTop || top > vocab) return "top must be in [0, 32] and at most vocab";
    if (!(temperature > 0.f) || !(temperature < INFINITY) || !(1.f / temperature < INFINITY)) return "temperature must be positive and finite";
    if (rows > 0 && (!logits || !tokens)) return "null argument";
    if ((uintptr_t)logits % element_size(dtype) || (uintptr_t)tokens % token_bytes) return "logits and tokens must be aligned to their elements";
    return nullptr;
}

}  // namespace xsm

using namespace xsm;

xsm_status xsm_token_logprobs(const xsm_logprob_args *a, void *cuda_stream) {
    if (!a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (const char *m = check_logits(a->logits, a->tokens, a->rows, a->vocab, a->dtype, a->token_bytes, a->top, a->temperature)) return op_failed(XSM_ERR_INVALID_ARG, m);
    if (a->rows == 0) return XSM_OK;
    if (!a->logprob || !a->entropy || !a->lse || (a->top && (!a->top_ids || !a->top_logprobs))) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    int sms = 0;
    const cudaError_t e = sm_count(&sms);
    if (e != cudaSuccess) return launched(e);
    const bool warps = by_warp(a->rows, (long long)a->vocab * element_size(a->dtype), sms);
    const int shift = warps ? 0 : cut_shift_of(a->rows, a->vocab, sms);
    const LogprobArgs A{a->logits, a->tokens, a->logprob, a->entropy, a->lse, a->top_ids, a->top_logprobs, a->row_stride, a->token_stride,
                        a->rows, a->vocab, a->token_bytes, a->top, 1 << shift, shift, 1.f / a->temperature};
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t r = cudaSuccess;
    with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        r = a->top ? launch_logprob<T, true>(A, warps, st) : launch_logprob<T, false>(A, warps, st);
    });
    return launched(r);
}

xsm_status xsm_token_logprobs_grad(const xsm_logprob_grad_args *a, void *cuda_stream) { return xsm_token_logprobs_grad_near(a, nullptr, cuda_stream); }

xsm_status xsm_token_logprobs_grad_near(const xsm_logprob_grad_args *a, const float *logprob, void *cuda_stream) {
    if (!a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (const char *m = check_logits(a->logits, a->tokens, a->rows, a->vocab, a->dtype, a->token_bytes, a->top, a->temperature)) return op_failed(XSM_ERR_INVALID_ARG, m);
    if (a->rows == 0) return XSM_OK;
    if (!a->lse || !a->d_logits || (a->g_entropy && !a->entropy) || (a->g_top && a->top && !a->top_ids)) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if ((uintptr_t)a->d_logits % element_size(a->dtype)) return op_failed(XSM_ERR_INVALID_ARG, "d_logits must be aligned to its elements");
    int sms = 0;
    const cudaError_t e = sm_count(&sms);
    if (e != cudaSuccess) return launched(e);
    const long long row_bytes = (long long)a->vocab * element_size(a->dtype);
    const bool warps = by_warp(a->rows, row_bytes, sms), top = a->top && a->g_top;
    // A block takes 2048 pieces of a row where there are rows enough for the eight blocks and more that an SM takes, else 512 (2045 rows of 1250 pieces
    // 33.1 -> 32.6 us, 1300 of 5000 58.0 -> 56.1, 1300 of 1000 13.6 -> 14.5).
    const int pieces = (int)((row_bytes + 15) / 16), per_block = warps ? pieces : a->rows >= 8 * sms ? 2048 : 512;
    const int blocks = pieces > per_block ? (pieces + per_block - 1) / per_block : 1;
    if (blocks > 65535) return op_failed(XSM_ERR_INVALID_ARG, "vocab is too large");
    // (every block of a row reads the token's logit: not where another one may have written the gradient to its place)
    const int es = element_size(a->dtype);
    const char *from = (const char *)a->logits, *to = (const char *)a->d_logits;
    const long long ends_from = ((a->rows - 1) * a->row_stride + a->vocab) * es, ends_to = ((a->rows - 1) * a->d_row_stride + a->vocab) * es;
    if (blocks > 1 && from < to + ends_to && to < from + ends_from) logprob = nullptr;
    const GradArgs A{a->logits, a->tokens, logprob, a->lse, a->entropy, a->top_ids, a->g_logprob, a->g_entropy, a->g_lse, a->g_top, a->d_logits,
                     a->row_stride, a->token_stride, a->g_logprob_stride, a->g_entropy_stride, a->g_lse_stride, a->d_row_stride,
                     a->rows, a->vocab, a->token_bytes, a->top, per_block, 1.f / a->temperature, a->temperature};
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t r = cudaSuccess;
    with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        r = top ? launch_grad<T, true>(A, blocks, warps, st) : launch_grad<T, false>(A, blocks, warps, st);
    });
    return launched(r);
}
