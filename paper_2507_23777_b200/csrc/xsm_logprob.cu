// Log probabilities of given tokens with entropy and top alternatives, and their gradient by the logits.
#include "xsm_ops.h"

#include <math.h>

namespace xsm {

constexpr int kMaxTop = 32;

struct LogprobArgs {
    const void *logits, *tokens;
    float *logprob, *entropy, *lse;
    int *top_ids;
    float *top_logprobs;
    long long row_ld, token_ld;
    int vocab, token_bytes, top;
    float inv_t;
};

__device__ __forceinline__ long long token_at(const void *tokens, int bytes, long long i) {
    return bytes == 8 ? reinterpret_cast<const long long *>(tokens)[i] : reinterpret_cast<const int *>(tokens)[i];
}

// An unsigned number that orders as (logit descending, index ascending) does, the first of them the largest.  NaN comes last; zeros of
// either sign are the same.
__device__ __forceinline__ unsigned long long rank_key(float z, int i) {
    const unsigned u = __float_as_uint(z + 0.f);
    const unsigned o = z != z ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
    return ((unsigned long long)o << 32) | (unsigned)~i;
}

// largest key (sum of values) of the block, in every thread
__device__ __forceinline__ unsigned long long block_max(unsigned long long v, unsigned long long *s) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) { const unsigned long long w = __shfl_xor_sync(0xffffffffu, v, o); v = w > v ? w : v; }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = s[0];
    for (int w = 1; w < (int)blockDim.x / 32; ++w) v = s[w] > v ? s[w] : v;
    return v;
}
__device__ __forceinline__ float block_sum(float v, float *s) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) v += s[w];
    return v;
}
__device__ __forceinline__ float block_max_f(float v, float *s) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = s[0];
    for (int w = 1; w < (int)blockDim.x / 32; ++w) v = fmaxf(v, s[w]);
    return v;
}

// A block for every row: maximum, sums, then the alternatives one after the other.
template <typename T> __global__ void __launch_bounds__(256) logprob_kernel(const __grid_constant__ LogprobArgs A) {
    __shared__ unsigned long long s_key[8];
    __shared__ float s_f[8];
    const long long row = blockIdx.x;
    const T *z = reinterpret_cast<const T *>(A.logits) + row * A.row_ld;
    float mx = -INFINITY;
    for (int i = threadIdx.x; i < A.vocab; i += 256) mx = fmaxf(mx, to_f(z[i]));
    mx = block_max_f(mx, s_f);
    float sum = 0.f, dot = 0.f;
    for (int i = threadIdx.x; i < A.vocab; i += 256) {
        const float x = (to_f(z[i]) - mx) * A.inv_t, e = expf(x);
        sum += e;
        dot += e == 0.f ? 0.f : e * x;
    }
    sum = block_sum(sum, s_f);
    dot = block_sum(dot, s_f);
    const bool none = mx == -INFINITY && sum != sum;      // nothing but -infinity, or NaN beside it
    float lse = mx * A.inv_t + logf(sum), entropy = logf(sum) - dot / sum;
    bool nan = false;
    if (none) {
        for (int i = threadIdx.x; i < A.vocab; i += 256) nan |= to_f(z[i]) != to_f(z[i]);
        nan = __syncthreads_or(nan);
        if (!nan) { lse = -INFINITY; entropy = 0.f; }
    }
    const bool empty = none && !nan;
    if (threadIdx.x == 0) {
        const long long t = token_at(A.tokens, A.token_bytes, row * A.token_ld);
        const bool has = t >= 0 && t < A.vocab;
        A.logprob[row] = !has ? 0.f : empty ? -INFINITY : (to_f(z[t]) - mx) * A.inv_t - logf(sum);
        A.entropy[row] = entropy;
        A.lse[row] = lse;
    }
    unsigned long long last = ~0ull;
    for (int k = 0; k < A.top; ++k) {
        unsigned long long best = 0;
        for (int i = threadIdx.x; i < A.vocab; i += 256) {
            const unsigned long long key = rank_key(to_f(z[i]), i);
            if (key < last && key > best) best = key;
        }
        last = block_max(best, s_key);
        if (threadIdx.x == 0) {
            const int id = (int)~(unsigned)last;
            A.top_ids[row * A.top + k] = id;
            A.top_logprobs[row * A.top + k] = empty ? -INFINITY : (to_f(z[id]) - mx) * A.inv_t - logf(sum);
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
    int vocab, token_bytes, top;
    float inv_t;
};

template <typename T> __global__ void __launch_bounds__(256) logprob_grad_kernel(const __grid_constant__ GradArgs A) {
    const long long row = blockIdx.x;
    const T *z = reinterpret_cast<const T *>(A.logits) + row * A.row_ld;
    T *d = reinterpret_cast<T *>(A.d_logits) + row * A.d_ld;
    const long long t = token_at(A.tokens, A.token_bytes, row * A.token_ld);
    const float lse = A.lse[row], h = A.entropy ? A.entropy[row] : 0.f;
    const float g = A.g_logprob && t >= 0 && t < A.vocab ? A.g_logprob[row * A.gl_ld] : 0.f, ge = A.g_entropy ? A.g_entropy[row * A.ge_ld] : 0.f;
    float total = g - (A.g_lse ? A.g_lse[row * A.gs_ld] : 0.f);
    if (A.g_top) for (int k = 0; k < A.top; ++k) total += A.g_top[row * A.top + k];
    for (int i = threadIdx.x; i < A.vocab; i += 256) {
        const float logp = to_f(z[i]) * A.inv_t - lse, p = expf(logp);
        float v = -p * (total + ge * ((p == 0.f ? 0.f : logp) + h));
        if (i == t) v += g;
        if (A.g_top) for (int k = 0; k < A.top; ++k) if (A.top_ids[row * A.top + k] == i) v += A.g_top[row * A.top + k];
        d[i] = rounded<T>(lse == -INFINITY ? 0.f : v * A.inv_t);
    }
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
    LogprobArgs A{a->logits, a->tokens, a->logprob, a->entropy, a->lse, a->top_ids, a->top_logprobs, a->row_stride, a->token_stride,
                  a->vocab, a->token_bytes, a->top, 1.f / a->temperature};
    with_dtype(a->dtype, [&](auto t) { logprob_kernel<decltype(t)><<<a->rows, 256, 0, (cudaStream_t)cuda_stream>>>(A); });
    return launched(cudaGetLastError());
}

xsm_status xsm_token_logprobs_grad(const xsm_logprob_grad_args *a, void *cuda_stream) {
    if (!a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (const char *m = check_logits(a->logits, a->tokens, a->rows, a->vocab, a->dtype, a->token_bytes, a->top, a->temperature)) return op_failed(XSM_ERR_INVALID_ARG, m);
    if (a->rows == 0) return XSM_OK;
    if (!a->lse || !a->d_logits || (a->g_entropy && !a->entropy) || (a->g_top && a->top && !a->top_ids)) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    GradArgs A{a->logits, a->tokens, a->lse, a->entropy, a->top_ids, a->g_logprob, a->g_entropy, a->g_lse, a->top ? a->g_top : nullptr, a->d_logits,
               a->row_stride, a->token_stride, a->g_logprob_stride, a->g_entropy_stride, a->g_lse_stride, a->d_row_stride, a->vocab, a->token_bytes, a->top, 1.f / a->temperature};
    with_dtype(a->dtype, [&](auto t) { logprob_grad_kernel<decltype(t)><<<a->rows, 256, 0, (cudaStream_t)cuda_stream>>>(A); });
    return launched(cudaGetLastError());
}
