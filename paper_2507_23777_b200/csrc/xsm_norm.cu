// Norms of queries and keys for each head with the rotation of the positions in the same pass: whole sequences for training, with the gradients, and new
// tokens on their way to the pages of a cache.
//
// y = R(position) (gain x r), r = (mean x^2 + eps)^(-1/2) over a head.  Gradient: u = R^-1 dy, d_gain = sum over rows of u x r, dx = r (w - x r^2 mean(w x)), w = gain u.
// A head is 2 to 16 neighbouring lanes, which hold two runs of eight elements each, the two halves of eight pairs, so that norm and rotation need nothing but
// the lanes' own registers and a sum over them.  A group of lanes takes some heads of a token one behind the other, the angles and the gains in registers, the
// next head on its way.  d_gain is added up in registers over all rows of a group, then over a block, then over blocks in their order: no atomics.
#include "xsm_ops.h"
#include "xsm_chain.cuh"

#include <limits.h>

#include <type_traits>

namespace xsm {

enum NormMode { NM_FORWARD, NM_APPEND, NM_GRAD };
constexpr int kNormThreads = 256;
constexpr int kNormBlocksPerSm = 4;

struct NormTensor {
    const void *x, *g;              // rows, gradients of the result
    void *out;                      // result, or gradient by x
    const void *gain;
    float *part;                    // NM_GRAD: [block][d]
    long long xs[3], gs[3], os[3];  // strides of sequence, token, head
    int heads, chunks, blocks;      // heads, units of a token, blocks that work on the tensor
};
struct NormArgs {
    NormTensor t[3];                // queries, keys, values
    const int *starts, *counts, *positions;
    const float2 *rope;
    unsigned tokens, m;
    int d, rope_n, rot, hp, gain_dtype;      // hp: heads of a unit
    float eps;
};

template <typename T, int N> struct __align__(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Run { T e[N]; };

__device__ __forceinline__ float gain_at(const void *p, int dtype, int i) {
    return dtype == XSM_F32 ? reinterpret_cast<const float *>(p)[i] : dtype == XSM_BF16 ? to_f(reinterpret_cast<const bf16 *>(p)[i]) : to_f(reinterpret_cast<const __half *>(p)[i]);
}

// N = 8: 16-byte pieces, L lanes a head, an item (two runs of N elements) each.  N = 1, for rows or angles that are not aligned to that: a warp a head, up to four pairs
// of elements a lane.  kNear: pairs are neighbours.
template <typename TI, typename TC, int N, int L, bool kNear, int MODE>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(const __grid_constant__ NormArgs A, const __grid_constant__ Pages P) {
    constexpr int I = N == 8 ? 1 : 4, G = kNormThreads / L;
    chain_go();
    chain_wait();
    int blk = (int)blockIdx.x, job = 0;
    while (job < 2 && blk >= A.t[job].blocks) blk -= A.t[job++].blocks;
    const NormTensor &T = A.t[job];
    const bool norm = job < 2;
    const int lane = threadIdx.x % L, group = threadIdx.x / L, items = A.d / (2 * N), rotated = A.rot / (2 * N);
    const unsigned mask = L == 32 ? 0xffffffffu : ((1u << L) - 1u) << ((threadIdx.x & 31) & ~(L - 1));
    int e0[I], e1[I];
    bool have[I], turn[I];
    float g0[I][N], g1[I][N], a0[I][N], a1[I][N];
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int c = lane + L * i;
        have[i] = c < items;
        turn[i] = have[i] && c < rotated && norm;
        e0[i] = turn[i] && !kNear ? c * N : c * 2 * N;
        e1[i] = turn[i] && !kNear ? e0[i] + A.rot / 2 : e0[i] + N;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            g0[i][k] = norm && have[i] ? gain_at(T.gain, A.gain_dtype, e0[i] + k) : 0.f;
            g1[i][k] = norm && have[i] ? gain_at(T.gain, A.gain_dtype, e1[i] + k) : 0.f;
            a0[i][k] = a1[i][k] = 0.f;
        }
    }
    const unsigned units = A.tokens * (unsigned)T.chunks, stride = (unsigned)T.blocks * G;
    for (unsigned u = (unsigned)blk * G + group; u < units; u += stride) {
        const unsigned token = u / (unsigned)T.chunks;
        const int h0 = (int)(u - token * (unsigned)T.chunks) * A.hp, h1 = min(h0 + A.hp, T.heads);
        const int b = (int)(token / A.m), j = (int)(token - (unsigned)b * A.m);
        const TI *x = reinterpret_cast<const TI *>(T.x) + b * T.xs[0] + j * T.xs[1];
        const TI *dy = MODE == NM_GRAD ? reinterpret_cast<const TI *>(T.g) + b * T.gs[0] + j * T.gs[1] : nullptr;
        Run<TI, N> in0[I], in1[I], d0[I], d1[I];
        auto fetch = [&](int h) {
#pragma unroll
            for (int i = 0; i < I; ++i)
                if (have[i]) {
                    in0[i] = *reinterpret_cast<const Run<TI, N> *>(x + h * T.xs[2] + e0[i]);
                    in1[i] = *reinterpret_cast<const Run<TI, N> *>(x + h * T.xs[2] + e1[i]);
                    if (MODE == NM_GRAD) {
                        d0[i] = *reinterpret_cast<const Run<TI, N> *>(dy + h * T.gs[2] + e0[i]);
                        d1[i] = *reinterpret_cast<const Run<TI, N> *>(dy + h * T.gs[2] + e1[i]);
                    }
                }
        };
        fetch(h0);        // on its way before anybody waits for the position and the page
        long long pos = 0, place = -1;
        bool real = true;
        if (MODE == NM_APPEND) {
            real = A.counts == nullptr || j < A.counts[b];
            pos = (long long)A.starts[b] + j;
        } else if (A.rope != nullptr) {
            pos = A.positions ? A.positions[token] : j;
        }
        const bool has_angle = A.rope == nullptr || (pos >= 0 && pos < A.rope_n);
        if (MODE == NM_APPEND && real && has_angle && pos >= 0 && pos <= INT_MAX) {
            const int at = (int)pos / P.size;
            const int page = at < P.max_pages ? P.table[b * P.table_ld + at] : -1;
            if (page >= 0 && page < P.n_pages) place = page * P.page + ((int)pos - at * P.size) * P.row;
        }
        const bool live = real && has_angle;
        if (MODE == NM_APPEND && job > 0 && place < 0) continue;
        float2 cs[I][N];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const float2 *from = A.rope + pos * (A.rot / 2) + (lane + L * i) * N;
#pragma unroll
            for (int k = 0; k < N; ++k) cs[i][k] = make_float2(1.f, 0.f);
            if (turn[i] && live) {
                if constexpr (N > 1) {
#pragma unroll
                    for (int k = 0; k < N / 2; ++k) {
                        const float4 t = reinterpret_cast<const float4 *>(from)[k];
                        cs[i][2 * k] = make_float2(t.x, t.y);
                        cs[i][2 * k + 1] = make_float2(t.z, t.w);
                    }
                } else {
                    cs[i][0] = from[0];
                }
            }
        }
        for (int h = h0; h < h1; ++h) {
            float p[I][N], q[I][N], up[I][N], uq[I][N];
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    p[i][k] = have[i] ? to_f(in0[i].e[k]) : 0.f;
                    q[i][k] = have[i] ? to_f(in1[i].e[k]) : 0.f;
                    if (MODE == NM_GRAD) {
                        up[i][k] = have[i] ? to_f(d0[i].e[k]) : 0.f;
                        uq[i][k] = have[i] ? to_f(d1[i].e[k]) : 0.f;
                    }
                    ss = fmaf(p[i][k], p[i][k], ss);
                    ss = fmaf(q[i][k], q[i][k], ss);
                }
            if (h + 1 < h1) fetch(h + 1);
            float r = 1.f;
            if (norm) {
#pragma unroll
                for (int o = L / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(mask, ss, o);
                r = 1.f / sqrtf(ss / (float)A.d + A.eps);
            }
            // pair k of a lane: elements k of both runs; interleaved: neighbours, the first half of the pairs in the first run.  back: by the angle's negative
            auto rotate = [&](float (&s)[N], float (&t)[N], const float2 (&angle)[N], bool back) {
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    constexpr bool near = N > 1 && kNear;
                    float &a = near ? (k < N / 2 ? s[2 * k % N] : t[2 * k % N]) : s[k], &d = near ? (k < N / 2 ? s[(2 * k + 1) % N] : t[(2 * k + 1) % N]) : t[k];
                    const float sn = back ? -angle[k].y : angle[k].y, f = a * angle[k].x - d * sn, w = a * sn + d * angle[k].x;
                    a = f;
                    d = w;
                }
            };
            if (MODE == NM_GRAD) {
                float dot = 0.f;
#pragma unroll
                for (int i = 0; i < I; ++i) {
                    if (turn[i]) rotate(up[i], uq[i], cs[i], true);
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        if (!live) up[i][k] = uq[i][k] = 0.f;
                        a0[i][k] = live ? fmaf(up[i][k], p[i][k] * r, a0[i][k]) : a0[i][k];
                        a1[i][k] = live ? fmaf(uq[i][k], q[i][k] * r, a1[i][k]) : a1[i][k];
                        up[i][k] *= g0[i][k];
                        uq[i][k] *= g1[i][k];
                        dot = fmaf(up[i][k], p[i][k], dot);
                        dot = fmaf(uq[i][k], q[i][k], dot);
                    }
                }
#pragma unroll
                for (int o = L / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(mask, dot, o);
                const float c = r * r * dot / (float)A.d;
                TI *dst = reinterpret_cast<TI *>(T.out) + b * T.os[0] + j * T.os[1] + h * T.os[2];
#pragma unroll
                for (int i = 0; i < I; ++i)
                    if (have[i]) {
                        Run<TI, N> o0, o1;
#pragma unroll
                        for (int k = 0; k < N; ++k) {
                            o0.e[k] = rounded<TI>(live ? r * (up[i][k] - p[i][k] * c) : 0.f);
                            o1.e[k] = rounded<TI>(live ? r * (uq[i][k] - q[i][k] * c) : 0.f);
                        }
                        *reinterpret_cast<Run<TI, N> *>(dst + e0[i]) = o0;
                        *reinterpret_cast<Run<TI, N> *>(dst + e1[i]) = o1;
                    }
            } else {
#pragma unroll
                for (int i = 0; i < I; ++i) {
                    if (norm) {
#pragma unroll
                        for (int k = 0; k < N; ++k) {
                            p[i][k] = p[i][k] * r * g0[i][k];
                            q[i][k] = q[i][k] * r * g1[i][k];
                        }
                        if (turn[i]) rotate(p[i], q[i], cs[i], false);
                    }
                    if (!have[i]) continue;
                    if (MODE == NM_APPEND && job > 0) {
                        TC *dst = reinterpret_cast<TC *>(job == 1 ? P.k : P.v) + place + h * P.head;
                        Run<TC, N> o0, o1;
#pragma unroll
                        for (int k = 0; k < N; ++k) { o0.e[k] = to_stored<TC>(p[i][k]); o1.e[k] = to_stored<TC>(q[i][k]); }
                        *reinterpret_cast<Run<TC, N> *>(dst + e0[i]) = o0;
                        *reinterpret_cast<Run<TC, N> *>(dst + e1[i]) = o1;
                    } else {
                        TI *dst = reinterpret_cast<TI *>(T.out) + b * T.os[0] + j * T.os[1] + h * T.os[2];
                        Run<TI, N> o0, o1;
#pragma unroll
                        for (int k = 0; k < N; ++k) { o0.e[k] = rounded<TI>(live ? p[i][k] : 0.f); o1.e[k] = rounded<TI>(live ? q[i][k] : 0.f); }
                        *reinterpret_cast<Run<TI, N> *>(dst + e0[i]) = o0;
                        *reinterpret_cast<Run<TI, N> *>(dst + e1[i]) = o1;
                    }
                }
            }
        }
    }
    if constexpr (MODE == NM_GRAD) {
        __shared__ float s[G][(N == 8 ? 16 * L : 256) + 1];
#pragma unroll
        for (int i = 0; i < I; ++i)
            if (have[i])
#pragma unroll
                for (int k = 0; k < N; ++k) { s[group][e0[i] + k] = a0[i][k]; s[group][e1[i] + k] = a1[i][k]; }
        __syncthreads();
        for (int e = threadIdx.x; e < A.d; e += kNormThreads) {
            float v = 0.f;
            for (int g = 0; g < G; ++g) v += s[g][e];
            T.part[(long long)blk * A.d + e] = v;
        }
    }
}

struct GainArgs {
    const float *part[2];
    void *out[2];
    int blocks[2], d, dtype;
};
// d_gain: 32 elements a block, eight threads an element
__global__ void __launch_bounds__(256) gain_kernel(const __grid_constant__ GainArgs A) {
    chain_go();
    chain_wait();
    __shared__ float s[8][32];
    const int which = blockIdx.y, x = threadIdx.x & 31, y = threadIdx.x >> 5, e = blockIdx.x * 32 + x;
    if (A.out[which] == nullptr) return;
    float v = 0.f;
#pragma unroll 8
    for (int b = y; b < A.blocks[which]; b += 8) v += A.part[which][(long long)b * A.d + e];
    s[y][x] = v;
    __syncthreads();
    if (y) return;
    for (int i = 1; i < 8; ++i) v += s[i][x];
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
static int lanes_of(int d, bool wide) { return !wide ? 32 : d == 96 ? 8 : d / 16; }

// Units of a token and blocks of each tensor.  Few tokens: a head a unit, a block for each of its groups; many: eight heads a unit, as many blocks as the chip
// runs at a time, shared out by the tensors' heads.
static int cut_norm(NormArgs &A, int lanes, bool bounded) {
    const int groups = kNormThreads / lanes, most = norm_sms() * kNormBlocksPerSm;
    int heads = 0, all = 0;
    for (const NormTensor &t : A.t) heads += t.heads;
    A.hp = (long long)A.tokens * heads <= (long long)most * groups ? 1 : 8;
    for (NormTensor &t : A.t) {
        t.chunks = (t.heads + A.hp - 1) / A.hp;
        const long long need = ((long long)A.tokens * t.chunks + groups - 1) / groups, share = ((long long)most * t.heads + heads - 1) / heads;
        t.blocks = (int)(bounded || A.hp > 1 ? (need < share ? need : share) : need);
        all += t.blocks;
    }
    return all;
}

template <typename TI, typename TC, int MODE>
static cudaError_t launch_norm(const NormArgs &A, const Pages &P, int blocks, bool wide, bool near, cudaStream_t st) {
    auto go = [&](auto fn) { return launch_early(fn, dim3(blocks), dim3(kNormThreads), 0, st, A, P); };
    if (!wide) return near ? go(norm_kernel<TI, TC, 1, 32, true, MODE>) : go(norm_kernel<TI, TC, 1, 32, false, MODE>);
    switch (lanes_of(A.d, true)) {
        case 2: return near ? go(norm_kernel<TI, TC, 8, 2, true, MODE>) : go(norm_kernel<TI, TC, 8, 2, false, MODE>);
        case 4: return near ? go(norm_kernel<TI, TC, 8, 4, true, MODE>) : go(norm_kernel<TI, TC, 8, 4, false, MODE>);
        case 8: return near ? go(norm_kernel<TI, TC, 8, 8, true, MODE>) : go(norm_kernel<TI, TC, 8, 8, false, MODE>);
        default: return near ? go(norm_kernel<TI, TC, 8, 16, true, MODE>) : go(norm_kernel<TI, TC, 8, 16, false, MODE>);
    }
}

static bool aligned16(const void *p, const int64_t *s, int es) {
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
    A.d = s.d_head; A.rope_n = s.rope_positions; A.rot = rope ? s.rope_dims : 0;
    A.gain_dtype = s.gain_dtype; A.eps = s.eps;
    A.t[0].heads = s.n_heads;
    A.t[1].heads = s.n_kv_heads;
    return A;
}

static size_t up(size_t n) { return (n + 255) & ~(size_t)255; }
static size_t gain_parts(int d) { return up((size_t)(norm_sms() * kNormBlocksPerSm + 3) * d * 4); }

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
    bool wide = A.rot % 16 == 0 && (uintptr_t)a->rope % 16 == 0;
    for (int i = 0; i < 2; ++i) {
        NormTensor &t = A.t[i];
        if (!t.heads) continue;
        t.x = x[i]; t.out = out[i]; t.gain = gain[i];
        for (int k = 0; k < 3; ++k) { t.xs[k] = xs[i][k]; t.os[k] = os[i][k]; }
        if (((uintptr_t)t.x | (uintptr_t)t.out) % es || (uintptr_t)t.gain % element_size(a->gain_dtype)) return op_failed(XSM_ERR_INVALID_ARG, "tensors must be aligned to their elements");
        wide = wide && aligned16(t.x, xs[i], es) && aligned16(t.out, os[i], es);
    }
    const int blocks = cut_norm(A, lanes_of(A.d, wide), false);
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
    if ((a->n_heads && (!a->q || !a->g_q || !a->d_q)) || (a->n_kv_heads && (!a->k || !a->g_k || !a->d_k)) || !a->workspace) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if ((uintptr_t)a->workspace % 16) return op_failed(XSM_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    if (a->workspace_bytes < (int64_t)gain_parts(a->d_head)) return op_failed(XSM_ERR_CAPACITY, "the workspace is too small");
    NormArgs A = norm_args(s, a->positions, a->rope);
    const void *x[2] = {a->q, a->k}, *g[2] = {a->g_q, a->g_k}, *gain[2] = {a->q_gain, a->k_gain};
    void *out[2] = {a->d_q, a->d_k}, *d_gain[2] = {a->d_q_gain, a->d_k_gain};
    const int64_t *xs[2] = {a->q_stride, a->k_stride}, *ys[2] = {a->g_q_stride, a->g_k_stride}, *os[2] = {a->d_q_stride, a->d_k_stride};
    const int es = element_size(a->dtype);
    bool wide = A.rot % 16 == 0 && (uintptr_t)a->rope % 16 == 0;
    for (int i = 0; i < 2; ++i) {
        NormTensor &t = A.t[i];
        if (!t.heads) continue;
        t.x = x[i]; t.g = g[i]; t.out = out[i]; t.gain = gain[i];
        for (int k = 0; k < 3; ++k) { t.xs[k] = xs[i][k]; t.gs[k] = ys[i][k]; t.os[k] = os[i][k]; }
        if (((uintptr_t)t.x | (uintptr_t)t.g | (uintptr_t)t.out) % es || (uintptr_t)t.gain % gs) return op_failed(XSM_ERR_INVALID_ARG, "tensors must be aligned to their elements");
        wide = wide && aligned16(t.x, xs[i], es) && aligned16(t.g, ys[i], es) && aligned16(t.out, os[i], es);
    }
    const int blocks = cut_norm(A, lanes_of(A.d, wide), true);
    A.t[0].part = (float *)a->workspace;
    A.t[1].part = A.t[0].part + (size_t)A.t[0].blocks * A.d;
    const Pages P = {};
    cudaError_t e = cudaSuccess;
    with_dtype(a->dtype, [&](auto in) { e = launch_norm<decltype(in), decltype(in), NM_GRAD>(A, P, blocks, wide, a->interleaved != 0, st); });
    if (e == cudaSuccess) {
        GainArgs R;
        for (int i = 0; i < 2; ++i) { R.part[i] = A.t[i].part; R.out[i] = A.t[i].heads ? d_gain[i] : nullptr; R.blocks[i] = A.t[i].blocks; }
        R.d = A.d; R.dtype = A.gain_dtype;
        e = launch_early(gain_kernel, dim3(A.d / 32, 2), dim3(256), 0, st, R);
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
    bool wide = A.rot % 16 == 0 && (uintptr_t)a->rope % 16 == 0;
    for (int i = 0; i < 3; ++i) {
        NormTensor &t = A.t[i];
        if (!t.heads) continue;
        t.x = x[i]; t.gain = gain[i];
        for (int k = 0; k < 3; ++k) { t.xs[k] = xs[i][k]; t.os[k] = a->q_out_stride[k]; }
        if ((uintptr_t)t.x % es || (uintptr_t)t.gain % element_size(n->gain_dtype)) return op_failed(XSM_ERR_INVALID_ARG, "tensors must be aligned to their elements");
        wide = wide && aligned16(t.x, xs[i], es);
    }
    if (a->n_heads) {
        A.t[0].out = a->q_out;
        if ((uintptr_t)a->q_out % es) return op_failed(XSM_ERR_INVALID_ARG, "tensors must be aligned to their elements");
        wide = wide && aligned16(a->q_out, a->q_out_stride, es);
    }
    const Pages P = pages_of(*kv, a->block_table, a->table_stride, a->max_pages);
    const int blocks = cut_norm(A, lanes_of(A.d, wide), false);
    cudaError_t e = cudaSuccess;
    with_dtype(a->in_dtype, [&](auto in) {
        with_dtype(kv->cfg.dtype, [&](auto stored) { e = launch_norm<decltype(in), decltype(stored), NM_APPEND>(A, P, blocks, wide, a->interleaved != 0, (cudaStream_t)cuda_stream); });
    });
    return launched(e);
}
