// Log probabilities of given tokens with entropy and top alternatives, and their gradient by the logits.
//
// Forward: one pass over a row with a running maximum m, s = sum exp((z - m)/T) and t = sum exp((z - m)/T) (z - m); then
// lse = m/T + log s, logprob = (z_token - m)/T - log s, entropy = log s - t/(s T).  A block of 256 threads takes a row; where
// there are fewer rows than keep the chip busy a cluster of blocks takes a part of the row each and joins through shared memory.
// Alternatives: the largest logits of every thread bound the k-th largest of the row from below; what reaches the bound, usually little more
// than k logits, is collected in a second look at the row (out of registers, or the caches) and sorted by counting.
// Backward: one pass, every element from its own logit and a few numbers of its row.
#include "xsm_ops.h"

#include <math.h>

#include <type_traits>

namespace xsm {

constexpr int kMaxTop = 32;
constexpr int kRowThreads = 256, kRowWarps = kRowThreads / 32;
constexpr int kAhead = 4;                 // 16-byte pieces that a thread has under way
constexpr int kCandidates = 512;

struct LogprobArgs {
    const void *logits, *tokens;
    float *logprob, *entropy, *lse;
    int *top_ids;
    float *top_logprobs;
    long long row_ld, token_ld;
    int vocab, token_bytes, top, cuts;    // cuts: blocks of a cluster, each with a part of the row
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
    // this thread's single element, if it has one: its index in the run, or -1
    __device__ __forceinline__ int single() const {
        const int i = threadIdx.x;
        return i < head ? i : i >= 32 && i < 32 + tail ? head + pieces * n + i - 32 : -1;
    }
};
template <typename T> __device__ __forceinline__ void widen(const uint4 &v, float (&x)[Pieces<T>::n]) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            x[i] = __uint_as_float(w[i]);
        } else if constexpr (std::is_same<T, bf16>::value) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
}
template <typename T> __device__ __forceinline__ uint4 nothing() {      // -infinity everywhere
    const unsigned w = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, bf16>::value ? 0xff80ff80u : 0xfc00fc00u;
    return make_uint4(w, w, w, w);
}

// Running maximum and sums of a part of a row.
struct Part {
    float m, s, t;
    // the same sums against a maximum that is no smaller
    __device__ __forceinline__ void rebase(float top, float c) {
        const float d = fmaxf(m - top, -1e30f), f = m == -INFINITY ? 0.f : ex2(d * c);      // (nothing yet: s = t = 0, but -infinity times 0 is none)
        t = f * (t + s * d);
        s *= f;
        m = top;
    }
    __device__ __forceinline__ void join(Part o, float c) {
        const float top = fmaxf(m, o.m);
        if (m != top) rebase(top, c);
        if (o.m != top) o.rebase(top, c);
        s += o.s;
        t += o.t;
    }
};
template <int N> __device__ __forceinline__ void take(Part &a, const float (&x)[N], float ref, float c, float &s, float &t) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float d = x[i] - ref, e = ex2(d * c);
        s += e;
        t = fmaf(e, fmaxf(d, -1e30f), t);
    }
}

struct RowShared {
    Part part[kRowWarps], joined;
    unsigned bound[kRowWarps];
    int found;
    unsigned long long key[kRowWarps];
    unsigned long long candidate[kCandidates];
    unsigned long long best[kMaxTop];
};

// The `top` largest of a run one after the other, each the largest below the one before: for rows whose bound collects too many (all
// alike, or -infinity) or too few (NaN).
template <typename T> __device__ __noinline__ void best_one_by_one(const T *z, int count, int index0, int top, RowShared &sh) {
    unsigned long long last = ~0ull;
    for (int k = 0; k < top; ++k) {
        unsigned long long best = 0;
        for (int i = threadIdx.x; i < count; i += kRowThreads) {
            const unsigned long long key = rank_key(to_f(z[i]), index0 + i);
            if (key < last && key > best) best = key;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const unsigned long long w = __shfl_xor_sync(0xffffffffu, best, o);
            best = w > best ? w : best;
        }
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh.key[threadIdx.x >> 5] = best;
        __syncthreads();
        last = 0;
        for (int w = 0; w < kRowWarps; ++w) last = sh.key[w] > last ? sh.key[w] : last;
        if (threadIdx.x == 0) sh.best[k] = last;
    }
    __syncthreads();
}

template <typename T, bool kTop> __global__ void __launch_bounds__(kRowThreads, 4) logprob_kernel(const __grid_constant__ LogprobArgs A) {
    constexpr int N = Pieces<T>::n;
    __shared__ RowShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int cut = A.cuts > 1 ? (int)cluster_rank() : 0;
    const long long row = blockIdx.x / A.cuts;
    const T *z = reinterpret_cast<const T *>(A.logits) + row * A.row_ld;
    const int i0 = (int)((long long)A.vocab * cut / A.cuts), count = (int)((long long)A.vocab * (cut + 1) / A.cuts) - i0;
    const Pieces<T> in(z + i0, count);
    const float c = A.inv_t * kLog2e;
    if (kTop && tid == 0) sh.found = 0;
    float given = 0.f;
    long long token = -1;
    if (tid == 0 && cut == 0) {
        token = token_at(A.tokens, A.token_bytes, row * A.token_ld);
        if (token < 0 || token >= A.vocab) token = -1;
        if (token >= 0) given = to_f(z[token]);
    }

    Part a{-INFINITY, 0.f, 0.f};
    const int one = in.single();
    const float single = one >= 0 ? to_f(in.p[one]) : -INFINITY;
    uint4 v[kAhead];
    for (int at = 0; at == 0 || at < in.pieces; at += kRowThreads * kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = at + u * kRowThreads + tid;
            v[u] = i < in.pieces ? in.piece(i) : nothing<T>();
        }
        float top = at == 0 ? fmaxf(a.m, single) : a.m;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            float x[N];
            widen<T>(v[u], x);
#pragma unroll
            for (int i = 0; i < N; ++i) top = fmaxf(top, x[i]);
        }
        if (top > a.m) a.rebase(top, c);
        const float ref = a.m == -INFINITY ? 0.f : a.m;
        float s = 0.f, t = 0.f;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            float x[N];
            widen<T>(v[u], x);
            take(a, x, ref, c, s, t);
        }
        if (at == 0) {
            const float x[1] = {single};
            take(a, x, ref, c, s, t);
        }
        a.s += s;
        a.t += t;
    }
    const unsigned mine = kTop ? order_of(a.m) : 0u;
    const int full_warps = min(kRowWarps, max(1, in.pieces / 32));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Part b;
        b.m = __shfl_xor_sync(0xffffffffu, a.m, o); b.s = __shfl_xor_sync(0xffffffffu, a.s, o); b.t = __shfl_xor_sync(0xffffffffu, a.t, o);
        a.join(b, c);
    }
    if (kTop) {
        // the j-th largest of the maxima of a warp's threads, as many as make `top` over the warps that are full of pieces: at least `top` logits
        // reach the least of these warps' bounds
        bool in_play = true;
        unsigned bound = 0;
        for (int j = 0; j < A.top; j += full_warps) {
            bound = __reduce_max_sync(0xffffffffu, in_play ? mine : 0u);
            const unsigned who = __ballot_sync(0xffffffffu, in_play && mine == bound);
            if (who && lane == __ffs(who) - 1) in_play = false;
        }
        if (lane == 0) sh.bound[warp] = bound;
    }
    if (lane == 0) sh.part[warp] = a;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kRowWarps; ++w) a.join(sh.part[w], c);
        if (A.cuts > 1) sh.joined = a;
    }
    if (kTop) {
        unsigned bound = sh.bound[0];
#pragma unroll
        for (int w = 1; w < kRowWarps; ++w) if (w < full_warps) bound = min(bound, sh.bound[w]);
        const float least = of_order(bound);
        const int want = min(A.top, count);
        int found = 0;
        if (bound > order_of(-INFINITY) || count <= kCandidates) {
            auto offer = [&](float x, int i) {
                if (x >= least) {
                    const int at = atomicAdd(&sh.found, 1);
                    if (at < kCandidates) sh.candidate[at] = rank_key(x, i0 + i);
                }
            };
            if (one >= 0) offer(single, one);
            const bool kept = in.pieces <= kRowThreads * kAhead;          // the row's pieces are still in registers
            for (int at = 0; at < in.pieces; at += kRowThreads * kAhead) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int i = at + u * kRowThreads + tid;
                    if (i >= in.pieces) continue;
                    if (!kept) v[u] = in.piece(i);
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int i = at + u * kRowThreads + tid;
                    if (i >= in.pieces) continue;
                    float x[N];
                    widen<T>(v[u], x);
#pragma unroll
                    for (int k = 0; k < N; ++k) offer(x[k], in.head + i * N + k);
                }
            }
            __syncthreads();
            found = sh.found;
        }
        if (found < want || found > kCandidates) {
            best_one_by_one(z + i0, count, i0, want, sh);
        } else {
            for (int i = tid; i < found; i += kRowThreads) {
                const unsigned long long key = sh.candidate[i];
                int before = 0;
                for (int k = 0; k < found; ++k) before += sh.candidate[k] > key;
                if (before < want) sh.best[before] = key;
            }
        }
        if (tid < A.top && tid >= want) sh.best[tid] = 0;                 // a part of the row that is shorter than `top`
        __syncthreads();
    }
    if (A.cuts > 1) {
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        if (cut == 0) {
            const uint32_t theirs = smem_u32(&sh.joined);
            if (tid == 0) {
                for (int r = 1; r < A.cuts; ++r) {
                    const uint32_t at = map_rank(theirs, r);
                    Part b{ld_cluster_f32(at), ld_cluster_f32(at + 4), ld_cluster_f32(at + 8)};
                    a.join(b, c);
                }
            }
            if (kTop) {
                // the parts' best, in order, side by side; the first of them all
                const int n = A.cuts * A.top;
                unsigned long long key = 0;
                if (tid < n) {
                    const uint32_t at = map_rank(smem_u32(&sh.best[tid % A.top]), tid / A.top);
                    const unsigned lo = __float_as_uint(ld_cluster_f32(at)), hi = __float_as_uint(ld_cluster_f32(at + 4));
                    key = ((unsigned long long)hi << 32) | lo;
                    sh.candidate[tid] = key;
                }
                __syncthreads();
                if (tid < n) {
                    int before = 0;
                    for (int k = 0; k < n; ++k) before += sh.candidate[k] > key || (sh.candidate[k] == key && k < tid);
                    if (before < A.top) sh.best[before] = key;
                }
                __syncthreads();
            }
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        if (cut != 0) return;
    }
    if (tid == 0) {
        const float log_s = logf(a.s), ref = a.m == -INFINITY ? 0.f : a.m;
        const bool none = a.s == 0.f;                                     // nothing but -infinity
        A.logprob[row] = token < 0 ? 0.f : none ? -INFINITY : (given - ref) * A.inv_t - log_s;
        A.entropy[row] = none ? 0.f : log_s - a.t / a.s * A.inv_t;
        A.lse[row] = none ? -INFINITY : ref * A.inv_t + log_s;
        if (kTop) sh.part[0] = Part{ref, log_s, none ? 1.f : 0.f};
    }
    if (kTop) {
        __syncthreads();
        if (tid < A.top) {
            const int id = (int)~(unsigned)sh.best[tid];
            A.top_ids[row * A.top + tid] = id;
            A.top_logprobs[row * A.top + tid] = sh.part[0].t != 0.f ? -INFINITY : (to_f(z[id]) - sh.part[0].m) * A.inv_t - sh.part[0].s;
        }
    }
}

struct GradArgs {
    const void *logits, *tokens;
    const float *lse, *entropy;
    const int *top_ids;
    const float *g_logprob, *g_entropy, *g_lse, *g_top;
    void *d_logits;
    long long row_ld, token_ld, gl_ld, ge_ld, gs_ld, d_ld;
    int vocab, token_bytes, top, chunks;   // chunks: blocks of a row
    float inv_t;
};

// The numbers of a row that its elements' gradients are made of, divided by T where they enter linearly.
struct RowGrad {
    float lse, entropy, total, ge, inv_t;
    bool none;
    __device__ __forceinline__ float of(float z) const {
        const float logp = fmaf(z, inv_t, -lse), p = ex2(logp * kLog2e);
        return -p * fmaf(ge, fmaxf(logp, -1e3f) + entropy, total);        // (p is zero below -104: the bound only keeps 0 * -infinity out)
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

// A block takes kRowThreads * kAhead pieces of a row (and the first of its row the single elements at both ends).
template <typename T, bool kTop> __global__ void __launch_bounds__(kRowThreads) logprob_grad_kernel(const __grid_constant__ GradArgs A) {
    constexpr int N = Pieces<T>::n;
    __shared__ unsigned s_marked[kRowThreads];
    __shared__ int s_id[kMaxTop];
    __shared__ float s_g[kMaxTop];
    const int tid = threadIdx.x, lane = tid & 31, chunk = blockIdx.x % A.chunks;
    const long long row = blockIdx.x / A.chunks;
    const T *z = reinterpret_cast<const T *>(A.logits) + row * A.row_ld;
    T *out = reinterpret_cast<T *>(A.d_logits) + row * A.d_ld;
    const Pieces<T> in(z, A.vocab);
    const int at0 = chunk * kRowThreads * kAhead;
    uint4 v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        const int i = at0 + u * kRowThreads + tid;
        if (i < in.pieces) v[u] = in.piece(i);
    }
    const int one = chunk == 0 ? in.single() : -1;
    const float single = one >= 0 ? to_f(in.p[one]) : 0.f;
    const long long token = token_at(A.tokens, A.token_bytes, row * A.token_ld);
    const bool has = token >= 0 && token < A.vocab;
    const float g = A.g_logprob && has ? A.g_logprob[row * A.gl_ld] * A.inv_t : 0.f;
    RowGrad r;
    r.lse = A.lse[row];
    r.entropy = A.entropy ? A.entropy[row] : 0.f;
    r.ge = A.g_entropy ? A.g_entropy[row * A.ge_ld] * A.inv_t : 0.f;
    r.total = g - (A.g_lse ? A.g_lse[row * A.gs_ld] * A.inv_t : 0.f);
    r.inv_t = A.inv_t;
    r.none = r.lse == -INFINITY;
    const int t = has ? (int)token : -1;
    // which of its pieces hold the token or an alternative, a bit each
    unsigned marked = 0;
    auto mark_of = [&](int id, int &owner) {
        const int i = id - in.head, piece = i / N - at0;
        owner = -1;
        if (i < 0 || i >= in.pieces * N || piece < 0 || piece >= kRowThreads * kAhead) return 0u;
        owner = piece % kRowThreads;
        return 1u << (piece / kRowThreads);
    };
    if (kTop) {
        const float gk = lane < A.top ? A.g_top[row * A.top + lane] * A.inv_t : 0.f;
        r.total += warp_sum(gk);
        s_marked[tid] = 0;
        __syncthreads();
        if (tid < A.top) {
            const int id = A.top_ids[row * A.top + tid];
            s_id[tid] = id;
            s_g[tid] = gk;
            int owner;
            const unsigned bit = mark_of(id, owner);
            if (owner >= 0) atomicOr(&s_marked[owner], bit);
        }
        __syncthreads();
        marked = s_marked[tid];
    }
    if (t >= 0) {
        int owner;
        const unsigned bit = mark_of(t, owner);
        if (owner == tid) marked |= bit;
    }
    auto full = [&](float x, int i) {             // of element i, with what falls on it directly
        float d = r.of(x);
        if (i == t) d += g;
        if (kTop) for (int k = 0; k < A.top; ++k) if (s_id[k] == i) d += s_g[k];
        return r.none ? 0.f : d;
    };
    if (one >= 0) out[one] = rounded<T>(full(single, one));
    const bool alike = (((uintptr_t)z ^ (uintptr_t)out) & 15) == 0;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        const int i = at0 + u * kRowThreads + tid, e = in.head + i * N;
        if (i >= in.pieces) continue;
        float x[N];
        widen<T>(v[u], x);
        if ((marked >> u) & 1u) {
#pragma unroll 1
            for (int k = 0; k < N; ++k) {         // (x stays in registers: the one element that counts is picked by comparison)
                float y = 0.f;
#pragma unroll
                for (int q = 0; q < N; ++q) if (q == k) y = x[q];
                y = full(y, e + k);
#pragma unroll
                for (int q = 0; q < N; ++q) if (q == k) x[q] = y;
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = r.none ? 0.f : r.of(x[k]);
        }
        if (alike) {
            *reinterpret_cast<uint4 *>(out + e) = narrow<T>(x);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) out[e + k] = rounded<T>(x[k]);
        }
    }
}

// Blocks that share a row: as many as the chip takes at a time (four an SM) over the rows, each with 4096 logits at least.
static int cuts_of(int rows, int vocab, int sms) {
    int cuts = 1;
    while (cuts < 8 && (long long)rows * cuts * 2 <= 4LL * sms && vocab / (2 * cuts) >= 4096) cuts *= 2;
    return cuts;
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

template <typename T, bool kTop> static cudaError_t launch_logprob(const LogprobArgs &A, int rows, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * A.cuts));
    cfg.blockDim = dim3(kRowThreads);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = A.cuts;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = A.cuts > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, logprob_kernel<T, kTop>, A);
}

static const char *check_logits(const void *logits, const void *tokens, int rows, int vocab, int dtype, int token_bytes, int top, float temperature) {
    if (rows < 0 || vocab < 1) return "rows must not be negative and vocab must be positive";
    if (!is_dtype(dtype)) return "dtype must be 0 (fp32), 1 (bf16) or 2 (fp16)";
    if (token_bytes != 4 && token_bytes != 8) return "token_bytes must be 4 or 8";
    if (top < 0 || top > kMaxTop || top > vocab) return "top must be in [0, 32] and at most vocab";
    if (!(temperature > 0.f) || !(temperature < INFINITY) || !(1.f / temperature < INFINITY)) return "temperature must be positive and finite";
    if (rows > 0 && (!logits || !tokens)) return "null argument";
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
    const LogprobArgs A{a->logits, a->tokens, a->logprob, a->entropy, a->lse, a->top_ids, a->top_logprobs, a->row_stride, a->token_stride,
                        a->vocab, a->token_bytes, a->top, cuts_of(a->rows, a->vocab, sms), 1.f / a->temperature};
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t r = cudaSuccess;
    with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        r = a->top ? launch_logprob<T, true>(A, a->rows, st) : launch_logprob<T, false>(A, a->rows, st);
    });
    return launched(r);
}

xsm_status xsm_token_logprobs_grad(const xsm_logprob_grad_args *a, void *cuda_stream) {
    if (!a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (const char *m = check_logits(a->logits, a->tokens, a->rows, a->vocab, a->dtype, a->token_bytes, a->top, a->temperature)) return op_failed(XSM_ERR_INVALID_ARG, m);
    if (a->rows == 0) return XSM_OK;
    if (!a->lse || !a->d_logits || (a->g_entropy && !a->entropy) || (a->g_top && a->top && !a->top_ids)) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    const int per = kRowThreads * kAhead * 16 / element_size(a->dtype), chunks = (a->vocab + per - 1) / per;
    if ((long long)a->rows * chunks > 0x7fffffff) return op_failed(XSM_ERR_INVALID_ARG, "rows * vocab is too large");
    const bool top = a->top && a->g_top;
    const GradArgs A{a->logits, a->tokens, a->lse, a->entropy, a->top_ids, a->g_logprob, a->g_entropy, a->g_lse, a->g_top, a->d_logits,
                     a->row_stride, a->token_stride, a->g_logprob_stride, a->g_entropy_stride, a->g_lse_stride, a->d_row_stride,
                     a->vocab, a->token_bytes, a->top, chunks, 1.f / a->temperature};
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        if (top) logprob_grad_kernel<T, true><<<a->rows * chunks, kRowThreads, 0, st>>>(A);
        else logprob_grad_kernel<T, false><<<a->rows * chunks, kRowThreads, 0, st>>>(A);
    });
    return launched(cudaGetLastError());
}
