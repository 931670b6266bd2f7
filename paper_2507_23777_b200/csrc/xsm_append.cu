// Pools of keys and values of a caller (xsm_kv), and new tokens appended to them: keys and queries rotated by their position on
// the way.
//
// A stream of its inputs (prompts of 8001 tokens, 327 MB, 62 us = 82 % of the measured copy rate), for few tokens a chain of two loads
// behind one another, position and page (2.0 us for a window of five tokens, 2.9 for 96 tokens: little more than a launch).
#include "xsm_ops.h"

#include <cuda.h>
#include <limits.h>

#include <atomic>
#include <new>
#include <type_traits>

namespace xsm {

struct AppendArgs {
    const void *q, *k, *v;
    void *q_out;
    const int *starts, *counts;
    const float2 *rope;
    long long qs[3], ks[3], vs[3], os[3];       // strides of sequence, token, head
    unsigned tokens, m;
    int heads, d, rope_n, rot;
};

template <typename T, int N> struct __align__(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Vec { T e[N]; };

template <bool kPool, typename T, int N> __device__ __forceinline__ void store_f(T *p, const float (&x)[N]) {
    Vec<T, N> v;
#pragma unroll
    for (int i = 0; i < N; ++i) v.e[i] = kPool ? to_stored<T>(x[i]) : rounded<T>(x[i]);
    *reinterpret_cast<Vec<T, N> *>(p) = v;
}

// The items of a token are the heads of q, of k and of v in runs of N pairs of elements, d / 2N items a head, the rotated ones first.  N = 8 takes whole 16-byte
// pieces; where the rotated part or the alignment does not allow that, N = 1.
// kOnce: a block has a thread for every item of its token, or of several tokens where they have few; otherwise 128 threads go from item to item of one token.
// kNear: pairs are neighbours.
template <typename TI, typename TC, int N, bool kNear, bool kOnce>
__global__ void __launch_bounds__(kOnce ? 512 : 128) append_kernel(const __grid_constant__ AppendArgs A, const __grid_constant__ Pages P) {
    chain_go();
    chain_wait();
    const unsigned token = kOnce ? blockIdx.x * blockDim.y + threadIdx.y : blockIdx.x;
    if (kOnce && token >= A.tokens) return;
    const int b = (int)(token / A.m), j = (int)(token - (unsigned)b * A.m);
    const int per_head = A.d / (2 * N), rotated = A.rot / (2 * N), n = (A.heads + 2 * P.kv_heads) * per_head;
    struct Item {
        bool is_q, is_v, turn;
        int head, c, e0, e1;                     // the two runs of N elements of the head
    };
    auto item_of = [&](int it) {
        Item i;
        const int slot = it / per_head;
        i.c = it - slot * per_head;
        i.is_q = slot < A.heads;
        i.is_v = slot >= A.heads + P.kv_heads;
        i.head = i.is_q ? slot : i.is_v ? slot - A.heads - P.kv_heads : slot - A.heads;
        i.turn = !i.is_v && i.c < rotated;
        i.e0 = i.turn && !kNear ? i.c * N : i.c * 2 * N;
        i.e1 = i.turn && !kNear ? i.e0 + A.rot / 2 : i.e0 + N;
        return i;
    };
    Vec<TI, N> in0, in1;
    auto fetch = [&](const Item &i) {
        const long long *s = i.is_q ? A.qs : i.is_v ? A.vs : A.ks;
        const TI *src = reinterpret_cast<const TI *>(i.is_q ? A.q : i.is_v ? A.v : A.k) + b * s[0] + j * s[1] + i.head * s[2];
        in0 = *reinterpret_cast<const Vec<TI, N> *>(src + i.e0);
        in1 = *reinterpret_cast<const Vec<TI, N> *>(src + i.e1);
    };
    if (kOnce) fetch(item_of(min((int)threadIdx.x, n - 1)));        // on their way before anybody waits for the position and the page
    const bool real = A.counts == nullptr || j < A.counts[b];
    const long long pos = (long long)A.starts[b] + j;
    const bool has_angle = A.rope == nullptr || (pos >= 0 && pos < A.rope_n);
    long long place = -1;                        // of the row in head 0, in elements
    if (real && has_angle && pos >= 0 && pos <= INT_MAX) {
        const int at = (int)pos / P.size;
        const int page = at < P.max_pages ? P.table[b * P.table_ld + at] : -1;
        if (page >= 0 && page < P.n_pages) place = page * P.page + ((int)pos - at * P.size) * P.row;
    }
    for (int it = threadIdx.x; it < n; it += blockDim.x) {
        const Item i = item_of(it);
        if (!i.is_q && place < 0) continue;
        if (!kOnce) fetch(i);
        const bool is_q = i.is_q, is_v = i.is_v, turn = i.turn;
        const int head = i.head, c = i.c, e0 = i.e0, e1 = i.e1;
        float x[N], y[N];
#pragma unroll
        for (int k = 0; k < N; ++k) { x[k] = to_f(in0.e[k]); y[k] = to_f(in1.e[k]); }
        if (turn && real && has_angle) {
            const float2 *from = A.rope + pos * (A.rot / 2) + c * N;
            float2 cs[N];
            if constexpr (N > 1) {
#pragma unroll
                for (int i = 0; i < N / 2; ++i) {
                    const float4 t = reinterpret_cast<const float4 *>(from)[i];
                    cs[2 * i] = make_float2(t.x, t.y);
                    cs[2 * i + 1] = make_float2(t.z, t.w);
                }
            } else {
                cs[0] = from[0];
            }
            // pair i: elements i of both runs; interleaved: neighbours, the first half of the pairs in the first run
#pragma unroll
            for (int i = 0; i < N; ++i) {
                constexpr bool near = N > 1 && kNear;
                float &a = near ? (i < N / 2 ? x[2 * i % N] : y[2 * i % N]) : x[i], &d = near ? (i < N / 2 ? x[(2 * i + 1) % N] : y[(2 * i + 1) % N]) : y[i];
                const float u = a * cs[i].x - d * cs[i].y, w = a * cs[i].y + d * cs[i].x;
                a = u;
                d = w;
            }
        }
        if (is_q) {
            if (!real || !has_angle) {
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = y[i] = 0.f;
            }
            TI *dst = reinterpret_cast<TI *>(A.q_out) + b * A.os[0] + j * A.os[1] + head * A.os[2];
            store_f<false>(dst + e0, x);
            store_f<false>(dst + e1, y);
        } else {
            TC *dst = reinterpret_cast<TC *>(is_v ? P.v : P.k) + place + head * P.head;
            store_f<true>(dst + e0, x);
            store_f<true>(dst + e1, y);
        }
    }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// tensor map of a pool: elements, rows of a page, heads, pages
static bool pool_map(EncodeTiledFn encode, TensorMap *out, const xsm_kv_config &c, void *pool, int box_rows) {
    const int es = element_size(c.dtype), box_w = es == 4 ? 32 : c.d_head % 64 == 0 ? 64 : 32;
    cuuint64_t dims[4] = {(cuuint64_t)c.d_head, (cuuint64_t)c.page_size, (cuuint64_t)c.n_kv_heads, (cuuint64_t)c.n_pages};
    cuuint64_t strides[3] = {(cuuint64_t)c.row_stride * es, (cuuint64_t)c.head_stride * es, (cuuint64_t)c.page_stride * es};
    cuuint32_t box[4] = {(cuuint32_t)box_w, (cuuint32_t)box_rows, 1, 1}, estr[4] = {1, 1, 1, 1};
    return encode(reinterpret_cast<CUtensorMap *>(out),
                  c.dtype == XSM_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : c.dtype == XSM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                  4, pool, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, box_w * es == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static bool aligned(const void *p, const int64_t (&s)[3], int es) {
    return ((uintptr_t)p | (uintptr_t)(s[0] * es) | (uintptr_t)(s[1] * es) | (uintptr_t)(s[2] * es)) % 16 == 0;
}

}  // namespace xsm

using namespace xsm;

xsm_status xsm_kv_create(const xsm_kv_config *cfg, void *d_k, void *d_v, xsm_kv **out) {
    if (!cfg || !d_k || !d_v || !out) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    const xsm_kv_config &c = *cfg;
    if (!is_dtype(c.dtype)) return op_failed(XSM_ERR_INVALID_ARG, "dtype must be 0 (fp32), 1 (bf16) or 2 (fp16)");
    if (c.d_head != 32 && c.d_head != 64 && c.d_head != 96 && c.d_head != 128 && c.d_head != 256)
        return op_failed(XSM_ERR_INVALID_ARG, "d_head must be 32, 64, 96, 128 or 256");
    if (c.page_size < 16 || c.page_size % 16) return op_failed(XSM_ERR_INVALID_ARG, "page_size must be a positive multiple of 16");
    if (c.n_pages < 1 || c.n_kv_heads < 1 || c.n_kv_heads > 1024) return op_failed(XSM_ERR_INVALID_ARG, "n_pages must be positive and n_kv_heads in [1, 1024]");
    const int per16 = 16 / element_size(c.dtype);
    if (c.row_stride < c.d_head || c.head_stride < c.d_head || c.page_stride < c.d_head || c.row_stride % per16 || c.head_stride % per16 || c.page_stride % per16)
        return op_failed(XSM_ERR_INVALID_ARG, "strides of the pools must be multiples of 16 bytes and no shorter than a row");
    if (((uintptr_t)d_k | (uintptr_t)d_v) % 16) return op_failed(XSM_ERR_INVALID_ARG, "the pools must be 16-byte aligned");
    xsm_kv *kv = new (std::nothrow) xsm_kv;
    if (!kv) return op_failed(XSM_ERR_CAPACITY, "out of host memory");
    kv->cfg = c;
    kv->k = d_k;
    kv->v = d_v;
    kv->box_rows = c.page_size % 32 ? 16 : 32;
    kv->tries = kMbarSpinLimit;
    kv->starve = 0;
    int dev = 0;
    void *encode = nullptr;
    cudaDriverEntryPointQueryResult q;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&kv->sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &encode, cudaEnableDefault, &q);
    if (e != cudaSuccess) {
        delete kv;
        return launched(e);
    }
    if (q != cudaDriverEntryPointSuccess || !pool_map((EncodeTiledFn)encode, &kv->k_map, c, d_k, kv->box_rows) ||
        !pool_map((EncodeTiledFn)encode, &kv->v_map, c, d_v, kv->box_rows)) {
        delete kv;
        return op_failed(XSM_ERR_CUDA, "the tensor maps of the pools could not be made");
    }
    *out = kv;
    return XSM_OK;
}

xsm_status xsm_kv_destroy(xsm_kv *kv) {
    if (!kv) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    delete kv;
    return XSM_OK;
}

xsm_status xsm_debug_kv_waits(xsm_kv *kv, uint32_t tries, int starve) {
    if (!kv) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    kv->tries = tries ? tries : kMbarSpinLimit;
    kv->starve = starve != 0;
    return XSM_OK;
}

// One word that the graph's end sets, on a thread of the driver's: nothing of the caller's is touched there.
struct xsm_capture {
    std::atomic<int> gone{0};
};
static void CUDART_CB graph_gone(void *c) { static_cast<xsm_capture *>(c)->gone.store(1, std::memory_order_release); }

uint64_t xsm_capture_id(void *cuda_stream) {
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    unsigned long long id = 0;
    if (cudaStreamGetCaptureInfo((cudaStream_t)cuda_stream, &status, &id) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    return status == cudaStreamCaptureStatusActive ? id : 0;
}

xsm_status xsm_capture_watch(void *cuda_stream, xsm_capture **out) {
    if (!out) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    unsigned long long id = 0;
    cudaGraph_t graph = nullptr;
    cudaError_t e = cudaStreamGetCaptureInfo((cudaStream_t)cuda_stream, &status, &id, &graph);
    if (e != cudaSuccess) return launched(e);
    if (status != cudaStreamCaptureStatusActive) return op_failed(XSM_ERR_INVALID_ARG, "the stream is not being recorded");
    xsm_capture *c = new (std::nothrow) xsm_capture;
    if (!c) return op_failed(XSM_ERR_CAPACITY, "out of host memory");
    cudaUserObject_t object = nullptr;
    e = cudaUserObjectCreate(&object, c, graph_gone, 1, cudaUserObjectNoDestructorSync);
    if (e != cudaSuccess) {
        delete c;
        return launched(e);
    }
    e = cudaGraphRetainUserObject(graph, object, 1, cudaGraphUserObjectMove);
    if (e != cudaSuccess) {
        (void)cudaUserObjectRelease(object, 1);      // (its end may still be on its way: the word stays allocated)
        return launched(e);
    }
    *out = c;
    return XSM_OK;
}

int xsm_capture_gone(xsm_capture *c) {
    if (!c || !c->gone.load(std::memory_order_acquire)) return 0;
    delete c;
    return 1;
}

int xsm_capture_mode(int mode) {
    cudaStreamCaptureMode m = (cudaStreamCaptureMode)mode;
    if (mode < 0 || mode > 2 || cudaThreadExchangeStreamCaptureMode(&m) != cudaSuccess) {
        (void)cudaGetLastError();
        return -1;
    }
    return (int)m;
}

xsm_status xsm_kv_append(const xsm_kv *kv, const xsm_kv_append_args *a, void *cuda_stream) {
    if (!kv || !a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (a->batch < 0 || a->m < 0 || a->n_heads < 0 || a->max_pages < 0) return op_failed(XSM_ERR_INVALID_ARG, "batch, m, n_heads and max_pages must not be negative");
    if (a->n_heads > 4096) return op_failed(XSM_ERR_INVALID_ARG, "n_heads must not exceed 4096");
    if (!is_dtype(a->in_dtype)) return op_failed(XSM_ERR_INVALID_ARG, "in_dtype must be 0 (fp32), 1 (bf16) or 2 (fp16)");
    if (a->rope && (a->rope_dims < 2 || a->rope_dims % 2 || a->rope_dims > kv->cfg.d_head || a->rope_positions < 1))
        return op_failed(XSM_ERR_INVALID_ARG, "rope_dims must be even and in [2, d_head], rope_positions positive");
    const long long tokens = (long long)a->batch * a->m;
    if (tokens == 0) return XSM_OK;
    if (tokens > 0x7fffffff) return op_failed(XSM_ERR_INVALID_ARG, "more than 2^31 - 1 tokens");
    if (!a->k || !a->v || (!a->block_table && a->max_pages) || !a->starts) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (a->n_heads && (!a->q || !a->q_out)) return op_failed(XSM_ERR_INVALID_ARG, "n_heads without q or q_out");
    AppendArgs A;
    A.q = a->q; A.k = a->k; A.v = a->v; A.q_out = a->q_out;
    A.starts = a->starts; A.counts = a->counts;
    A.rope = reinterpret_cast<const float2 *>(a->rope);
    for (int i = 0; i < 3; ++i) { A.qs[i] = a->q_stride[i]; A.ks[i] = a->k_stride[i]; A.vs[i] = a->v_stride[i]; A.os[i] = a->q_out_stride[i]; }
    A.tokens = (unsigned)tokens; A.m = (unsigned)a->m; A.heads = a->n_heads; A.d = kv->cfg.d_head; A.rope_n = a->rope_positions;
    A.rot = a->rope ? a->rope_dims : 0;
    const Pages P = pages_of(*kv, a->block_table, a->table_stride, a->max_pages);
    const int es = element_size(a->in_dtype);
    if (((uintptr_t)a->k | (uintptr_t)a->v | (uintptr_t)(a->n_heads ? a->q : nullptr) | (uintptr_t)(a->n_heads ? a->q_out : nullptr)) % es)
        return op_failed(XSM_ERR_INVALID_ARG, "q, k, v and q_out must be aligned to their elements");
    if (((uintptr_t)a->rope) % 8) return op_failed(XSM_ERR_INVALID_ARG, "rope must be 8-byte aligned");
    const bool wide = A.rot % 16 == 0 && (uintptr_t)a->rope % 16 == 0 && aligned(a->k, a->k_stride, es) && aligned(a->v, a->v_stride, es) &&
                      (a->n_heads == 0 || (aligned(a->q, a->q_stride, es) && aligned(a->q_out, a->q_out_stride, es)));
    const int items = (A.heads + 2 * P.kv_heads) * (A.d / (wide ? 16 : 2));
    // Few tokens: a thread for every item, whose elements are requested before the token's place is known (a window of five tokens 2.45 -> 2.1 us); many:
    // 128 threads a token, fewer registers a thread (prompts of 8001 tokens 62 us, 73 the other way, 65 with 256 threads).
    const bool once = items <= 64 || (tokens < 1024 && items <= 512);
    const int threads = !once && items > 128 ? 128 : (items + 31) / 32 * 32;
    // few items a token, many tokens: as many of them a block as make 128 threads (269790 tokens of four heads of 128: 281 us with one a block, 128 with four)
    const int packed = tokens < 1024 || threads > 64 ? 1 : 128 / threads;
    cudaError_t e = cudaSuccess;
    with_dtype(a->in_dtype, [&](auto in) {
        with_dtype(kv->cfg.dtype, [&](auto stored) {
            using TI = decltype(in);
            using TC = decltype(stored);
            auto go = [&](auto n, auto near, auto one) {
                e = launch_early(append_kernel<TI, TC, decltype(n)::value, decltype(near)::value, decltype(one)::value>, dim3((unsigned)((tokens + packed - 1) / packed)), dim3(threads, packed), 0,
                                 (cudaStream_t)cuda_stream, A, P);
            };
            auto by_order = [&](auto n, auto near) { once ? go(n, near, std::true_type()) : go(n, near, std::false_type()); };
            auto by_width = [&](auto n) { a->interleaved ? by_order(n, std::true_type()) : by_order(n, std::false_type()); };
            wide ? by_width(std::integral_constant<int, 8>()) : by_width(std::integral_constant<int, 1>());
        });
    });
    return launched(e);
}
