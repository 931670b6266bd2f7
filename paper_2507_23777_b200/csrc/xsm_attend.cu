// Attention of the newest tokens of each sequence over a caller's paged pools (xsm_kv).
//
// A unit is a sequence, a key head and up to 64 of the query rows (tokens x heads of the group) that read it.  What a unit has to do is
// counted in granules of 128 positions, and all granules of the call, in one row, are cut into equal runs, one for every CTA of a grid
// that fills the chip once: lengths are known on the device alone, and neither short nor long sequences leave SMs without work.
// A unit that a cut goes through leaves partial results (maximum, sum, unnormalised output) in the workspace; the CTA that is the last
// to arrive at the unit's counter adds them up in the order of the positions, so results do not depend on which one that is.
//
// In a CTA up to four producer warps stream stages of 32 positions (boxes of the keys' and values' tensor maps; page numbers looked up 32
// stages at a time) through a ring in shared memory.  Eight warps attend (four where heads are 256 wide): row tiles of sixteen rows (one, two or four of
// them) times as many groups as that leaves, which take the stages in turn.  A warp keeps its rows' output and running maximum in registers:
// S = Q K^T, online softmax, O += P V with mma.sync; over 16-bit pools weights enter as the sum of a rounded part and its remainder, fp32
// operands as parts of eleven bits whose three large products are added up.
//
// What bounds it.  Long contexts: the pools' bytes, at the rate of a copy (4 x 20000 positions of sixteen heads of 128 in fp16, 655 MB, 103 us = 98 %
// of the measured rate; 48 ragged sequences of eight key heads in bf16, 804 MB, 129 us = 97 %).  A producer warp needs 0.4 to 0.6 us a stage: one
// alone fed 33 GB/s an SM (158 us), four feed 46.  Short ones: a chain.  0.3 us to past the wait for the kernel before, 1.8 until lengths are
// read and the cut is known, 0.6 for page numbers, 0.6 for the first stage, a microsecond a stage, 1.2 for joining the warps: 5.6 us for
// 190 positions; where a unit is cut 1 us for the counter and 2 for adding up (12288 positions of sixteen heads of 64: 17 us of which the
// bytes are 7.8).  Starting under the kernel before saves 1 us.  fp32: the chain too, with three products for one (12 us; the bytes 1.4).
// Many rows a key head: mma.sync (8 x 4000 positions, 64 rows a key head: 42 us, the bytes 12).
#include "xsm_ops.h"

#include <limits.h>
#include <math.h>
#include <string.h>

#include <type_traits>

namespace xsm {

constexpr int kStage = 32;            // positions of a stage
// Stages that are never cut apart (2, 4, 8: 142, 138, 137 us on the ragged batch, 15.0, 15.0, 16.6 on fp32 with a window); granules that a unit counts for
// beside its stages: its queries, the joining of its warps, its output (0, 2, 3: 133, 125, 126 us on the ragged batch, 18.2, 17.3, 16.4 on 12288
// positions, 104.8, 103.8, 103.0 on 20000).
constexpr int kGranule = 4, kOpening = 3;
// Units up to this many bytes of keys and values are not cut at all: joining what two CTAs have done takes 3 us, in which one of them reads as much (190
// positions 7.6 -> 5.9 us).
constexpr int kWholeBytes = 128 * 1024;
constexpr int kProducers = 4;
// Attending warps of a CTA: heads of 256 want 255 registers a thread, which eight warps and the producers do not have.
__host__ __device__ constexpr int attend_warps(int dh) { return dh == 256 ? 4 : 8; }
// Warps that share a stage's positions: where stages are so large that few fit, and a warp works on one for long (all that follows from a position's
// key is a warp's own, so that the shares meet at the end of a unit like any others).
__host__ __device__ constexpr int slices_of(int dh, int es) { return es == 4 ? dh >= 128 ? 4 : dh >= 64 ? 2 : 1 : dh == 256 ? 2 : 1; }
constexpr int kRing = 16;             // most stages in shared memory
constexpr int kMaxRowTiles = 4;       // of a unit
constexpr int kDeclared = 4096;       // shared memory that the kernel declares, at most
// Workspace: status word and counters, which every call leaves at zero, in a place that does not depend on the call; then the partial results.
constexpr int kHeadBytes = 4096, kMaxGrid = kHeadBytes / 4 - 4;

struct AttendArgs {
    const void *q;
    void *out;
    float *lse;
    const int *lengths, *counts, *table;
    int *counters, *status;           // a counter for every CTA, used for the unit that the next CTA shares with it; status word of the waits
    float *partial;                   // two places for every CTA
    long long qs[3], os[3], table_ld;
    int batch, m, heads, group, kv_heads;
    int whole;                        // stages of a unit that is not cut, at most
    float part_scale, all_units;      // see run_of
    int rt, row_groups, n_rows;       // row tiles of a unit, units that share a key head, query rows of a key head
    int causal, window, page, max_pages, n_pages, box_rows;
    int parked;                       // warps that park their state at the end of a unit
    int ring, turns, producers;       // stages in shared memory; groups of warps that take them in turn, warps that fetch them: every place is one of each's
    float c;                          // scale * log2(e)
    unsigned tries;                   // of a barrier, before whoever waits gives up
    int starve;                       // nothing is fetched (a test of the waits)
};

template <typename T, int DH> struct Shape {
    static constexpr int es = sizeof(T), box_w = es == 4 ? 32 : DH % 64 == 0 ? 64 : 32;      // elements of a box's row
    static constexpr int rb = box_w * es, boxes = DH / box_w, box_bytes = kStage * rb;
    static constexpr int half = boxes * box_bytes, stage = 2 * half;                          // keys, then values
    static constexpr int steps = DH * es / 32;                                                // products over 32 bytes of a row
    static constexpr int ld = DH + 4;                                                         // rows of parked outputs
    // Shared-memory address of 16-byte chunk ch of row r.  Rows are 128 (64) bytes, so a lane's row and the chunk that it begins with are one number
    // (`lane_at`), and an even number of chunks further is an exclusive or of constants (`step`).
    static __device__ __forceinline__ uint32_t at(uint32_t base, int r, int ch) {
        constexpr int per = rb / 16;
        const int x = ch % per, s = rb == 128 ? r & 7 : (r >> 1) & 3;
        return base + (ch / per) * box_bytes + r * rb + ((x ^ s) << 4);
    }
    static __device__ __forceinline__ uint32_t lane_at(int r, int first) { return at(0, r, first); }
    static __device__ __forceinline__ uint32_t step(uint32_t from, int ch) {
        constexpr int per = rb / 16;
        return (from ^ (uint32_t)((ch % per) << 4)) + (uint32_t)((ch / per) * box_bytes);
    }
};
__host__ __device__ constexpr int parked_bytes(int dh, int warps) { return warps * 16 * ((dh + 4) + 2) * 4; }
// query operands of a row tile, in the order in which the lanes take them
__host__ __device__ constexpr int query_bytes(int dh, int es, bool split) { return dh * es / 32 * 512 * (split ? 2 : 1); }

// query rows as they are in memory, on their way to that
__host__ __device__ constexpr int raw_bytes(int dh, int es) { return 16 * (dh * es + 16); }

// What a sequence has to do.  Row j of its nq queries sees [begin_j, end_j): end_j = end - nq + 1 + j (all: end), begin_j = end_j - window.
struct Span {
    int base, end, first_end, first_begin, last_begin, nq, stages;
};
__device__ __forceinline__ Span span_of(const AttendArgs &A, int b) {
    Span s;
    const long long room = (long long)A.max_pages * A.page;
    int len = A.lengths[b];
    len = len > room ? (int)room : len < 0 ? 0 : len;
    len = min(len, INT_MAX - 2 * kStage);
    s.nq = A.counts ? max(0, min(A.counts[b], A.m)) : A.m;
    s.end = s.nq == 0 ? 0 : len;
    s.first_end = A.causal ? s.end - s.nq + 1 : s.end;
    s.first_begin = A.window > 0 ? max(0, s.first_end - A.window) : 0;
    s.last_begin = A.window > 0 ? max(0, s.end - A.window) : 0;
    s.base = s.first_begin & ~(A.box_rows - 1);
    s.stages = max(1, (s.end - s.base + kStage - 1) / kStage);
    return s;
}
// (a unit takes a granule's time more than its stages do: queries, joining of warps, output)
__device__ __forceinline__ int granules(int stages) { return (stages + kGranule - 1) / kGranule + kOpening; }

// The run of granules of this CTA, and where it starts.  Every warp works it out for itself.  (The host has made sure that the granules
// of all units fit 31 bits.)
struct Run {
    int at, end, before;                     // granules; before: those of the sequences before b
    int b;
    int ctas, quot, rem;                     // CTAs that have work: the first `rem` have quot + 1 granules, the others quot
    __device__ __forceinline__ int start(int cta) const { return cta * quot + min(cta, rem); }
    __device__ __forceinline__ int owner(int granule) const {
        const int more = rem * (quot + 1);
        return granule < more ? granule / (quot + 1) : rem + (granule - more) / quot;
    }
};
__device__ __forceinline__ Run run_of(const AttendArgs &A, int units) {
    const int lane = threadIdx.x & 31;
    int sum = 0, all = 0, first = 0;         // granules; stages; stages of the first 32 sequences, which most calls end with
    for (int b = lane; b < A.batch; b += 32) {
        const int stages = span_of(A, b).stages;
        if (b == lane) first = stages;
        sum += granules(stages);
        all += stages;
    }
    Run r;
    const int total = (int)__reduce_add_sync(0xffffffffu, (unsigned)sum) * units;
    // Few long units: a unit's parts are read by their CTAs side by side, n stages of 32 * 2 * d_head elements, and joined by one, C rows of d_head
    // sums, both at about the same bytes a second, so C = sqrt(16 * element size * n / rows) parts are the quickest (one key head at 20000 positions: 148
    // parts 21.7 us, 50 parts 15.3).
    // (part_scale has what the lengths do not change: times all stages it is the square of C times the number of units.)
    float parts;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(parts) : "f"(A.part_scale * (float)__reduce_add_sync(0xffffffffu, (unsigned)all)));
    r.ctas = min(min((int)gridDim.x, total), (int)fminf(fmaxf(parts, A.all_units), 65535.f));      // every one of them has a granule at least
    r.quot = total / r.ctas;
    r.rem = total - r.quot * r.ctas;
    r.at = r.start(blockIdx.x);
    r.end = r.start(blockIdx.x + 1);
    r.b = 0;
    r.before = 0;
    if ((int)blockIdx.x >= r.ctas) {
        r.end = r.at;
        return r;
    }
    // where both ends lie; one inside a unit that is not cut, or in front of a unit's first stage, goes to the unit's beginning
    int ends[2] = {r.at, r.end};
    int before = 0, open = 2;
    for (int b0 = 0; b0 < A.batch && open; b0 += 32) {
        const int b = b0 + lane, stages = b < A.batch ? b0 == 0 ? first : span_of(A, b).stages : 0, mine = b < A.batch ? granules(stages) : 0;
        int up = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, up, o);
            if (lane >= o) up += v;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int at = e == 0 ? r.at : r.end;
            const unsigned past = __ballot_sync(0xffffffffu, b < A.batch && (before + up) * units > at);
            if (!past || before * units > at) continue;
            const int l = __ffs(past) - 1, per = __shfl_sync(0xffffffffu, mine, l), start = (before + __shfl_sync(0xffffffffu, up - mine, l)) * units;
            const int unit = start + (at - start) / per * per;
            if (__shfl_sync(0xffffffffu, stages, l) <= A.whole || at - unit <= kOpening) ends[e] = unit;
            if (e == 0) { r.b = b0 + l; r.before = start; }
            --open;
        }
        before += __shfl_sync(0xffffffffu, up, 31);
    }
    r.at = ends[0];
    r.end = ends[1];
    return r;
}

// The part of a unit that a CTA does.
struct Segment {
    int unit, stage0, stage1;                // of the sequence; stages
    int first, last;                         // the whole unit's granules
    bool whole, more;                        // the CTA does all of the unit; has another one behind it (the next of the sequence, or the next sequence's first)
};

template <typename F> __device__ __forceinline__ void walk(const AttendArgs &A, int units, F &&f) {
    Run r = run_of(A, units);
    while (r.at < r.end) {
        const Span sp = span_of(A, r.b);
        const int per = granules(sp.stages), behind = r.before + per * units;
        while (r.at < r.end && r.at < behind) {
            Segment s;
            const int rel = r.at - r.before;
            s.unit = rel / per;
            const int g0 = rel - s.unit * per, g1 = min(per, g0 + (r.end - r.at));
            s.stage0 = max(0, g0 - kOpening) * kGranule;
            s.stage1 = min(sp.stages, (g1 - kOpening) * kGranule);
            s.first = r.before + s.unit * per;
            s.last = s.first + per;
            s.whole = g0 == 0 && g1 == per;
            s.more = r.at + g1 - g0 < r.end;
            f(r.b, sp, s, r);
            r.at += g1 - g0;
        }
        r.before = behind;
        ++r.b;
    }
}

__device__ __forceinline__ void tma_box4(uint32_t dst, const void *tmap, int x, int row, int head, int page, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 :: "r"(dst), "l"(tmap), "r"(x), "r"(row), "r"(head), "r"(page), "r"(bar) : "memory");
}
__device__ __forceinline__ void mma1688_tf32(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16(float (&c)[4], const uint4 &a, unsigned b0, unsigned b1, __half) { mma16816_f16(c, a.x, a.y, a.z, a.w, b0, b1); }
__device__ __forceinline__ void mma16(float (&c)[4], const uint4 &a, unsigned b0, unsigned b1, bf16) { mma16816_bf16(c, a.x, a.y, a.z, a.w, b0, b1); }

// x = part + rest: part is x rounded to eleven bits (a tf32 operand), the rest is at most 2^-12 of it, of which a tf32 operand keeps eleven bits again
__device__ __forceinline__ unsigned tf32_weight(float x) { return (__float_as_uint(x) + 0x1000u) & 0xffffe000u; }      // (far from the largest number)
// What would round to an infinity is cut off instead.  Infinities and NaN have a part of some finite number and are their own rest (the difference of two
// infinities would be NaN where the products are right), so that the rest is a subtraction without a question.
__device__ __forceinline__ unsigned tf32_part(float x) {
    const unsigned u = __float_as_uint(x), up = u + 0x1000u;
    return (up & 0x7f800000u) == 0x7f800000u ? u & 0xff7fe000u : up & 0xffffe000u;
}
__device__ __forceinline__ unsigned tf32_rest(float x, unsigned part) { return __float_as_uint(x - __uint_as_float(part)); }

// two values as 16-bit operands, first in the low half, and what the rounding took off
template <typename T> __device__ __forceinline__ unsigned pack2(float a, float b);
template <> __device__ __forceinline__ unsigned pack2<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const unsigned *>(&h);
}
template <> __device__ __forceinline__ unsigned pack2<bf16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const unsigned *>(&h);
}
template <typename T> __device__ __forceinline__ unsigned rest2(float a, float b, unsigned p);
template <> __device__ __forceinline__ unsigned rest2<__half>(float a, float b, unsigned p) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&p));
    return pack2<__half>(a - f.x, b - f.y);
}
template <> __device__ __forceinline__ unsigned rest2<bf16>(float a, float b, unsigned p) {
    return pack2<bf16>(a - __uint_as_float(p << 16), b - __uint_as_float(p & 0xffff0000u));
}
__device__ __forceinline__ unsigned lds32(uint32_t a) {
    unsigned v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}

// A warp's sixteen rows: lane 4g + t has rows g and g + 8, columns 8j + 2t and + 1.
template <int DH> struct RowState {
    float o[DH / 8][4], m[2], l[2];           // l: this lane's keys only
};

// bits of the positions base..base+31 inside [begin, end)
__device__ __forceinline__ unsigned inside(int base, int begin, int end) {
    const int lo = max(0, begin - base), hi = min(kStage, end - base);
    if (lo >= hi) return 0u;
    return (hi == 32 ? ~0u : (1u << hi) - 1u) & ~((1u << lo) - 1u);
}

// O += P V over 8 NT positions.  kept: positions that take part; the others' values may be anything (kMask: they are
// read as zeros, so that zero weights do not meet infinities).  kSome: only rows of which `mine` is set get anything.
template <typename T, int DH, int NT, bool kMask, bool kSome>
__device__ __forceinline__ void add_values(const float (&p)[NT][4], uint32_t v_base, unsigned kept, const bool (&mine)[2], RowState<DH> &st) {
    using S = Shape<T, DH>;
    const int lane = threadIdx.x & 31, t = lane & 3, g = lane >> 2;
    if constexpr (std::is_same<T, float>::value) {
        // The tensor core cuts off what its sum has no place for, towards zero: a stage's products are added up by themselves, and to the output by rounding.
        unsigned a[NT][4], r[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = p[nt][(i & 1) * 2 + (i >> 1)];
                a[nt][i] = tf32_weight(w);
                r[nt][i] = __float_as_uint(w - __uint_as_float(a[nt][i]));
            }
#pragma unroll
        for (int j = 0; j < DH / 8; ++j) {
            float add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int k0 = nt * 8 + 2 * t;
                unsigned x = lds32(S::at(v_base, k0, 2 * j + (g >> 2)) + (g & 3) * 4), y = lds32(S::at(v_base, k0 + 1, 2 * j + (g >> 2)) + (g & 3) * 4);
                if (kMask) { x = (kept >> k0) & 1u ? x : 0u; y = (kept >> (k0 + 1)) & 1u ? y : 0u; }
                const unsigned xh = tf32_part(__uint_as_float(x)), yh = tf32_part(__uint_as_float(y));
                const unsigned xl = tf32_rest(__uint_as_float(x), xh), yl = tf32_rest(__uint_as_float(y), yh);
                mma1688_tf32(add, r[nt][0], r[nt][1], r[nt][2], r[nt][3], xh, yh);
                mma1688_tf32(add, a[nt][0], a[nt][1], a[nt][2], a[nt][3], xl, yl);
                mma1688_tf32(add, a[nt][0], a[nt][1], a[nt][2], a[nt][3], xh, yh);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) if (!kSome || mine[i >> 1]) st.o[j][i] += add[i];
        }
    } else {
#pragma unroll
        for (int kk = 0; kk < NT / 2; ++kk) {
            const float (&u)[4] = p[2 * kk], (&w)[4] = p[2 * kk + 1];
            const uint4 a = make_uint4(pack2<T>(u[0], u[1]), pack2<T>(u[2], u[3]), pack2<T>(w[0], w[1]), pack2<T>(w[2], w[3]));
            const uint4 r = make_uint4(rest2<T>(u[0], u[1], a.x), rest2<T>(u[2], u[3], a.y), rest2<T>(w[0], w[1], a.z), rest2<T>(w[2], w[3], a.w));
            const uint32_t from = v_base + kk * 16 * S::rb + S::lane_at((lane & 7) + (((lane >> 3) & 1) << 3), lane >> 4);
            unsigned m0 = ~0u, m1 = ~0u;
            if (kMask) {
                const unsigned b0 = kept >> (kk * 16 + 2 * t), b1 = kept >> (kk * 16 + 2 * t + 8);
                m0 = (b0 & 1u ? 0xffffu : 0u) | (b0 & 2u ? 0xffff0000u : 0u);
                m1 = (b1 & 1u ? 0xffffu : 0u) | (b1 & 2u ? 0xffff0000u : 0u);
            }
#pragma unroll
            for (int j = 0; j < DH / 8; j += 2) {
                unsigned v[4];
                ldmatrix_x4_trans(v, S::step(from, j));
                if (kMask) { v[0] &= m0; v[1] &= m1; v[2] &= m0; v[3] &= m1; }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float add[4] = {0.f, 0.f, 0.f, 0.f};
                    float (&o)[4] = kSome ? add : st.o[j + h];
                    mma16(o, r, v[2 * h], v[2 * h + 1], T());
                    mma16(o, a, v[2 * h], v[2 * h + 1], T());
                    if (kSome) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) if (mine[i >> 1]) st.o[j + h][i] += add[i];
                    }
                }
            }
        }
    }
}

// Whether a position of `some` holds a value that is not finite.  (An exponent of ones and one more carry into the sign's place; the order of
// a row's pieces does not matter.)
template <typename T, int DH, int NT> __device__ __forceinline__ bool odd_values(uint32_t v_base, unsigned some) {
    using S = Shape<T, DH>;
    constexpr unsigned ones = S::es == 4 ? 0x7f800000u : std::is_same<T, bf16>::value ? 0x7f807f80u : 0x7c007c00u;
    constexpr unsigned more = S::es == 4 ? 0x00800000u : std::is_same<T, bf16>::value ? 0x00800080u : 0x04000400u;
    constexpr int chunks = DH * S::es / 16, per = S::rb / 16;
    const int lane = threadIdx.x & 31, first = __ffs(some) - 1, last = 32 - __clz(some);
    unsigned odd = 0;
#pragma unroll 4
    for (int i = first * chunks + lane; i < last * chunks; i += 32) {
        const int r = i / chunks, c = i - r * chunks;
        const uint4 v = lds128(v_base + (c / per) * S::box_bytes + r * S::rb + c % per * 16);
        const unsigned bits = ((v.x & ones) + more) | ((v.y & ones) + more) | ((v.z & ones) + more) | ((v.w & ones) + more);
        odd |= (some >> r) & 1u ? bits : 0u;
    }
    return __any_sync(0xffffffffu, (odd & (S::es == 4 ? 0x80000000u : 0x80008000u)) != 0u);
}

// What masks a stage for a warp: positions that its two rows see, that any row of the sequence sees, that all of them do.
struct StageMask {
    unsigned row[2], any, all, valid;
};

// 8 NT positions of a stage (`stage`, masks and `base` begin with them) for the sixteen rows of a warp.
template <typename T, int DH, int NT, bool kSplitQ, bool kMask>
__device__ __forceinline__ void attend_stage(uint32_t q_base, uint32_t stage, float c, const StageMask &mask, const AttendArgs &A, const Span &sp, int base,
                                             const int (&token)[2], RowState<DH> &st) {
    using S = Shape<T, DH>;
    const int lane = threadIdx.x & 31, t = lane & 3;
    // Weights over fp16 pools are the type's numbers, of which 2^-24 is the least step: they are up to 2^15 instead of 1, so that a key whose weight is 2^-18 of
    // the largest still has its 22 bits, and the error of any is below 2^-40 of the largest (17.5 nats below a key without a value: off by half, and by 2^-15 now).
    constexpr int kHead = std::is_same<T, __half>::value ? 15 : 0;
    constexpr bool kHalves = S::es == 4 && NT <= 2;      // of fp32 the products of either half of the head are added up by themselves too
    float half[kHalves ? NT : 1][4];
    float s[NT][4], small[NT][4];             // fp32 operands, or queries in two parts: products of the smaller parts, in a chain of their own
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
        small[nt][0] = small[nt][1] = small[nt][2] = small[nt][3] = 0.f;
        if (kHalves) half[nt][0] = half[nt][1] = half[nt][2] = half[nt][3] = 0.f;
    }
    const uint32_t from = stage + (NT > 1 ? S::lane_at((lane & 7) + ((lane >> 4) << 3), (lane >> 3) & 1) : S::lane_at(lane & 7, (lane >> 3) & 1));
#pragma unroll
    for (int ks = 0; ks < S::steps; ++ks) {
        const uint4 a = lds128(q_base + ks * 512 + lane * 16);
        uint4 al;
        if (kSplitQ || S::es == 4) al = lds128(q_base + (S::steps + ks) * 512 + lane * 16);
#pragma unroll
        for (int kt = 0; kt < (NT + 1) / 2; ++kt) {
            unsigned k[4];
            if constexpr (NT > 1) ldmatrix_x4(k, S::step(from, 2 * ks) + kt * 16 * S::rb);
            else ldmatrix_x2(k, S::step(from, 2 * ks));
            if constexpr (S::es == 4) {
                unsigned h[4], l[4];
#pragma unroll
                for (int i = 0; i < (NT > 1 ? 4 : 2); ++i) { h[i] = tf32_part(__uint_as_float(k[i])); l[i] = tf32_rest(__uint_as_float(k[i]), h[i]); }
#pragma unroll
                for (int n = 0; n < (NT > 1 ? 2 : 1); ++n) {
                    mma1688_tf32(small[2 * kt + n], al.x, al.y, al.z, al.w, h[2 * n], h[2 * n + 1]);
                    mma1688_tf32(small[2 * kt + n], a.x, a.y, a.z, a.w, l[2 * n], l[2 * n + 1]);
                    mma1688_tf32(kHalves && ks >= S::steps / 2 ? half[kHalves ? 2 * kt + n : 0] : s[2 * kt + n], a.x, a.y, a.z, a.w, h[2 * n], h[2 * n + 1]);
                }
            } else {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    if (kSplitQ) mma16(small[2 * kt + n], al, k[2 * n], k[2 * n + 1], T());
                    mma16(s[2 * kt + n], a, k[2 * n], k[2 * n + 1], T());
                }
            }
        }
    }
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (kHalves) s[nt][i] += half[nt][i];
            s[nt][i] = kSplitQ || S::es == 4 ? (s[nt][i] + small[nt][i]) * c : s[nt][i] * c;
            if (kMask && !((mask.row[i >> 1] >> (nt * 8 + 2 * t + (i & 1))) & 1u)) s[nt][i] = -INFINITY;
            top[i >> 1] = fmaxf(top[i >> 1], s[nt][i]);
        }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
        top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
        // the reference that the weights are taken against (kHead below the largest score; rounded up, so that no weight is above 2^kHead however large the
        // scores are)
        top[r] = fmaxf(st.m[r], kHead > 0 ? __fadd_ru(top[r], (float)-kHead) : top[r]);
    }
    // nothing seen so far: any finite reference will do, the weights are zero
    const float ref0 = kMask && top[0] == -INFINITY ? 0.f : top[0], ref1 = kMask && top[1] == -INFINITY ? 0.f : top[1];
    if (__any_sync(0xffffffffu, top[0] != st.m[0] || top[1] != st.m[1])) {
        const float f0 = ex2(st.m[0] - ref0), f1 = ex2(st.m[1] - ref1);
        st.l[0] *= f0; st.l[1] *= f1;
#pragma unroll
        for (int j = 0; j < DH / 8; ++j) { st.o[j][0] *= f0; st.o[j][1] *= f0; st.o[j][2] *= f1; st.o[j][3] *= f1; }
        st.m[0] = top[0]; st.m[1] = top[1];
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        s[nt][0] = ex2(s[nt][0] - ref0); s[nt][1] = ex2(s[nt][1] - ref0);
        s[nt][2] = ex2(s[nt][2] - ref1); s[nt][3] = ex2(s[nt][3] - ref1);
        st.l[0] += s[nt][0] + s[nt][1];
        st.l[1] += s[nt][2] + s[nt][3];
    }
    const uint32_t v_base = stage + S::half;
    const bool all[2] = {true, true};
    if (!kMask) {
        add_values<T, DH, NT, false, false>(s, v_base, ~0u, all, st);
    } else {
        const unsigned some = mask.any & ~mask.all;       // positions that some rows see and others do not
        if (some == 0u || !odd_values<T, DH, NT>(v_base, some)) {
            add_values<T, DH, NT, true, false>(s, v_base, mask.any, all, st);
        } else {                                          // one of them holds an infinity or NaN: the rows of one token after the other
            for (int j = 0; j < sp.nq; ++j) {
                const int end = A.causal ? sp.first_end + j : sp.end, begin = A.window > 0 ? max(0, end - A.window) : 0;
                const bool mine[2] = {token[0] == j, token[1] == j};
                add_values<T, DH, NT, true, true>(s, v_base, inside(base, begin, end) & mask.valid, mine, st);
            }
        }
    }
}

// the attending warps
template <int W> __device__ __forceinline__ void bar_attend() { bar_sync<W * 32>(1); }

template <typename TQ> __device__ __forceinline__ void store4(TQ *p, float4 v) {
    if constexpr (sizeof(TQ) == 4) *reinterpret_cast<float4 *>(p) = v;
    else *reinterpret_cast<uint2 *>(p) = make_uint2(pack2<TQ>(v.x, v.y), pack2<TQ>(v.z, v.w));
}

// Where a unit's rows come out.  Written by a thread a row: who needs them would divide.
struct RowPlace {
    long long out, lse;                       // elements; lse -1: not wanted
    int token;                                // of the sequence's queries
    bool real;                                // there is such a query
};
__device__ __forceinline__ void place_row(const AttendArgs &A, int b, int unit, int nq, int r, RowPlace *places) {
    const int kvh = unit / A.row_groups, row = (unit - kvh * A.row_groups) * A.rt * 16 + r, j = row / A.group, h = kvh * A.group + (row - j * A.group);
    places[r] = RowPlace{b * A.os[0] + j * A.os[1] + h * A.os[2], A.lse ? ((long long)b * A.m + j) * A.heads + h : -1, j, j < nq};
}
// output of one row's four elements and its lse, from the joined state
template <typename TQ> __device__ __forceinline__ void finish(const AttendArgs &A, const RowPlace &p, int d, float4 o, float m, float l) {
    const bool none = !p.real || l == 0.f;
    const float f = none ? 0.f : 1.f / l;
    store4<TQ>(reinterpret_cast<TQ *>(A.out) + p.out + d, none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
    if (d == 0 && p.lse >= 0) A.lse[p.lse] = none ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

template <typename T, typename TQ, int DH>
__global__ void __launch_bounds__((attend_warps(DH) + kProducers) * 32, 1)
attend_kernel(const __grid_constant__ TensorMap k_map, const __grid_constant__ TensorMap v_map, const __grid_constant__ AttendArgs A) {
    using S = Shape<T, DH>;
    constexpr int W = attend_warps(DH), kSlices = slices_of(DH, S::es), NT = 4 / kSlices;
    // queries with more bits than the pools' type enter as two parts
    constexpr bool kSplitQ = S::es == 2 && sizeof(TQ) == 4;
    extern __shared__ __align__(1024) unsigned char smem[];
    __shared__ __align__(8) unsigned long long s_full[kRing], s_empty[kRing];
    __shared__ int2 s_info[kRing];            // first position of a stage, which halves exist
    struct Left { int b, unit, nq, c0, c1; bool second, last; };
    __shared__ RowPlace s_rows[2][kMaxRowTiles * 16];      // of the unit at work; at the end of two that are joined
    __shared__ Left s_left[2];                // units that other CTAs share: at most the run's first and its last
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t ring = smem_u32(smem), full = smem_u32(s_full), empty = smem_u32(s_empty);
    float *parked = reinterpret_cast<float *>(smem + A.ring * S::stage), *parked_ml = parked + A.parked * 16 * S::ld;
    unsigned char *queries = smem + A.ring * S::stage + parked_bytes(DH, A.parked);
    chain_go();
    if (threadIdx.x == 0) {
        for (int i = 0; i < A.ring; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, A.rt * kSlices); }
        mbar_init_fence();
    }
    __syncthreads();
    chain_wait();
    const int units = A.kv_heads * A.row_groups;

    if (warp >= W) {
        // producer p of n takes stages p, p + n, ... of the CTA; slot and phase are those of its next one
        const int p = warp - W;
        if (p >= A.producers) return;
        int it = 0, slot = 0, phase = 1, next = p;                    // it: stages of the segments before
        // (lane 0) The stage behind the last that was requested: once a wait has run out, none is any more.  A place is filled again only when all its readers
        // have said that they are through, which one that has given up never says: so no barrier is armed twice in a phase.
        int past = A.starve ? -1 : p;
        auto advance = [&](int by) {
            slot += by;
            while (slot >= A.ring) { slot -= A.ring; phase ^= 1; }
        };
        advance(p);
        walk(A, units, [&](int b, const Span &sp, const Segment &seg, const Run &) {
            const int kvh = seg.unit / A.row_groups, halves = A.box_rows == kStage ? 1 : 2, n = seg.stage1 - seg.stage0;
            while (next < it + n) {
                // page and first row in it of both halves of the stage that is this lane's of the next 32
                int page[2] = {-1, -1}, row[2] = {0, 0};
                const int mine = next - it + lane * A.producers, first = sp.base + (seg.stage0 + mine) * kStage;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int pos = first + h * 16;
                    if (h < halves && mine < n && pos < sp.end) {
                        const int at = pos / A.page;
                        page[h] = A.table[b * A.table_ld + at];
                        row[h] = pos - at * A.page;
                    }
                    if (page[h] < 0 || page[h] >= A.n_pages) page[h] = -1;        // outside the pool: zeros are read, nobody sees them
                }
                for (int i = 0; i < 32 && next < it + n; ++i, next += A.producers) {
                    int pg[2], rw[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) { pg[h] = __shfl_sync(0xffffffffu, page[h], i); rw[h] = __shfl_sync(0xffffffffu, row[h], i); }
                    const int pos = __shfl_sync(0xffffffffu, first, i);
                    if (lane == 0 && next == past && (next < A.ring || mbar_wait(empty + 8 * slot, phase, A.tries, A.status))) {
                        const uint32_t bar = full + 8 * slot, dst = ring + slot * S::stage;
                        past += A.producers;
                        s_info[slot] = make_int2(pos, halves == 1 ? (pg[0] >= 0 ? 3 : 0) : (pg[0] >= 0 ? 1 : 0) | (pg[1] >= 0 ? 2 : 0));
                        mbar_arrive_expect_tx(bar, S::stage);
#pragma unroll
                        for (int x = 0; x < S::boxes; ++x) {
                            tma_box4(dst + x * S::box_bytes, &k_map, x * S::box_w, rw[0], kvh, pg[0], bar);
                            if (halves == 2) tma_box4(dst + x * S::box_bytes + 16 * S::rb, &k_map, x * S::box_w, rw[1], kvh, pg[1], bar);
                        }
#pragma unroll
                        for (int x = 0; x < S::boxes; ++x) {
                            tma_box4(dst + S::half + x * S::box_bytes, &v_map, x * S::box_w, rw[0], kvh, pg[0], bar);
                            if (halves == 2) tma_box4(dst + S::half + x * S::box_bytes + 16 * S::rb, &v_map, x * S::box_w, rw[1], kvh, pg[1], bar);
                        }
                    }
                    advance(A.producers);
                }
            }
            it += n;
        });
        // every copy lands before the CTA ends, also where an attending warp has given up: each producer looks at its own places, whose phases before it knows to
        // be over
        if (lane == 0)
            for (int i = past - A.producers; i >= 0 && i > past - A.producers - A.ring; i -= A.producers) mbar_wait(full + 8 * (i % A.ring), (i / A.ring) & 1, A.tries, A.status);
        return;
    }

    const int tile = warp % A.rt, share = warp / A.rt % kSlices * NT, turns = A.turns, turn = warp / (A.rt * kSlices);      // row tile; first eight positions of a stage; groups that take stages, which of them (behind the last: none)
    const int g = lane >> 2, t = lane & 3, tid = threadIdx.x;
    const int slot_floats = A.rt * 16 * (DH + 2);
    unsigned char *raw = queries + A.rt * query_bytes(DH, S::es, kSplitQ || S::es == 4);
    constexpr int raw_ld = DH * (int)sizeof(TQ) + 16;
    // requests the query rows of a unit
    auto fetch_rows = [&](int b, int unit) {
        constexpr int chunks = DH * (int)sizeof(TQ) / 16;
        const int kvh = unit / A.row_groups, row0 = (unit % A.row_groups) * A.rt * 16, rows = min(A.rt * 16, A.n_rows - row0);
        for (int i = tid; i < rows * chunks; i += W * 32) {
            const int r = i / chunks, c = i - r * chunks, j = (row0 + r) / A.group, h = kvh * A.group + (row0 + r - j * A.group);
            const TQ *p = reinterpret_cast<const TQ *>(A.q) + b * A.qs[0] + j * A.qs[1] + h * A.qs[2];
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(smem_u32(raw) + r * raw_ld + c * 16), "l"(reinterpret_cast<const char *>(p) + c * 16) : "memory");
        }
    };
    bool opening = true;
    int pending = 0;
    int it0 = 0, next = turn < turns ? turn : INT_MAX, slot = turn, phase = 0;      // stages of the segments before; this warp's next one
    walk(A, units, [&](int b, const Span &sp, const Segment &seg, const Run &run) {
        const int kvh = seg.unit / A.row_groups, row0 = (seg.unit % A.row_groups) * A.rt * 16, rows = min(A.rt * 16, A.n_rows - row0);
        if (opening) fetch_rows(b, seg.unit);
        opening = false;
        asm volatile("cp.async.wait_all;" ::: "memory");
        bar_attend<W>();                            // the rows are here; what the segment before parked has been read
        if (tid < rows) place_row(A, b, seg.unit, sp.nq, tid, s_rows[0]);
        // A thread takes 16 bytes of the operands (eight elements, or four of fp32) at a time and puts their words where the lanes of the products
        // look for them: 32 bytes of a row a step; lane 4 (row mod 8) + (word mod 4), register (row / 8) + 2 (word / 4).
        constexpr int per = S::es == 4 ? 4 : 8, chunks = DH / per;
        for (int i = tid; i < A.rt * 16 * chunks; i += W * 32) {
            const int r = (i / (16 * chunks)) * 16 + i % 16, ch = i / 16 % chunks, in = r & 15;      // neighbouring lanes take neighbouring rows: fewer of them meet in a bank
            struct __align__(16) Some { TQ e[per]; };
            const Some some = *reinterpret_cast<const Some *>(raw + r * raw_ld + ch * per * (int)sizeof(TQ));
            float x[per];
#pragma unroll
            for (int k = 0; k < per; ++k) x[k] = r < rows ? to_f(some.e[k]) : 0.f;
            unsigned *dst = reinterpret_cast<unsigned *>(queries + (r >> 4) * query_bytes(DH, S::es, kSplitQ || S::es == 4) + (ch >> 1) * 512 + (in & 7) * 64) +
                            (in >> 3) + 2 * (ch & 1);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if constexpr (S::es == 4) {
                    const unsigned hi = tf32_part(x[w]);
                    dst[4 * w] = hi;
                    dst[4 * w + S::steps * 128] = tf32_rest(x[w], hi);
                } else {
                    const unsigned hi = pack2<T>(x[2 * w], x[2 * w + 1]);
                    dst[4 * w] = hi;
                    if (kSplitQ) dst[4 * w + S::steps * 128] = rest2<T>(x[2 * w], x[2 * w + 1], hi);
                }
            }
        }
        bar_attend<W>();
        if (seg.more) {
            const bool same = seg.unit + 1 < units;
            fetch_rows(same ? b : b + 1, same ? seg.unit + 1 : 0);
        }

        RowState<DH> st;
#pragma unroll
        for (int j = 0; j < DH / 8; ++j) st.o[j][0] = st.o[j][1] = st.o[j][2] = st.o[j][3] = 0.f;
        st.m[0] = st.m[1] = -INFINITY;
        st.l[0] = st.l[1] = 0.f;
        const uint32_t q_base = smem_u32(queries) + tile * query_bytes(DH, S::es, kSplitQ || S::es == 4);
        int token[2], begin[2], end[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int row = tile * 16 + g + 8 * r;
            token[r] = row < rows ? s_rows[0][row].token : sp.nq;
            end[r] = token[r] >= sp.nq ? 0 : A.causal ? sp.first_end + token[r] : sp.end;
            begin[r] = A.window > 0 ? max(0, end[r] - A.window) : 0;
        }
        const int n = seg.stage1 - seg.stage0;
        for (; next < it0 + n; next += turns) {
            // (the results are void once a wait has run out: this warp waits for nothing more, and tells no producer to go on)
            if (!__all_sync(0xffffffffu, mbar_wait(full + 8 * slot, phase, A.tries, A.status))) {
                next = INT_MAX;
                break;
            }
            const int2 info = s_info[slot];
            const int base = info.x + share * 8;
            const uint32_t stage = ring + slot * S::stage + share * 8 * S::rb;
            StageMask mask;
            if (info.y == 3 && base >= sp.last_begin && base + 8 * NT <= sp.first_end) {
                attend_stage<T, DH, NT, kSplitQ, false>(q_base, stage, A.c, mask, A, sp, base, token, st);
            } else {
                constexpr unsigned mine = NT == 4 ? ~0u : (1u << (8 * NT)) - 1u;
                mask.valid = (((info.y & 1 ? 0xffffu : 0u) | (info.y & 2 ? 0xffff0000u : 0u)) >> (share * 8)) & mine;
                mask.row[0] = inside(base, begin[0], end[0]) & mask.valid;
                mask.row[1] = inside(base, begin[1], end[1]) & mask.valid;
                mask.any = inside(base, sp.first_begin, sp.end) & mask.valid;
                mask.all = inside(base, sp.last_begin, sp.first_end);
                attend_stage<T, DH, NT, kSplitQ, true>(q_base, stage, A.c, mask, A, sp, base, token, st);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + 8 * slot);
            slot += turns;
            if (slot >= A.ring) { slot -= A.ring; phase ^= 1; }
        }
        it0 += n;

        // the states of the warps: where they are more than have a place, the second half hand theirs to the first, which park the joined ones
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            st.l[r] += __shfl_xor_sync(0xffffffffu, st.l[r], 1);
            st.l[r] += __shfl_xor_sync(0xffffffffu, st.l[r], 2);
        }
        const int spot = warp & (A.parked - 1);
        float *mine = parked + spot * 16 * S::ld, *mine_ml = parked_ml + spot * 32;
        auto park = [&] {
#pragma unroll
            for (int j = 0; j < DH / 8; ++j) {
                *reinterpret_cast<float2 *>(mine + g * S::ld + 8 * j + 2 * t) = make_float2(st.o[j][0], st.o[j][1]);
                *reinterpret_cast<float2 *>(mine + (g + 8) * S::ld + 8 * j + 2 * t) = make_float2(st.o[j][2], st.o[j][3]);
            }
            if (t == 0) {
                mine_ml[2 * g] = st.m[0]; mine_ml[2 * g + 1] = st.l[0];
                mine_ml[2 * g + 16] = st.m[1]; mine_ml[2 * g + 17] = st.l[1];
            }
        };
        const bool halved = turns * A.rt * kSlices == 2 * A.parked;
        if (halved) {
            if (warp >= A.parked && warp < 2 * A.parked) park();
            bar_attend<W>();
        }
        if (halved && warp < A.parked) {
            float f[2], h[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float m = mine_ml[2 * g + 16 * r], l = mine_ml[2 * g + 16 * r + 1], top = fmaxf(m, st.m[r]), ref = top == -INFINITY ? 0.f : top;
                f[r] = ex2(st.m[r] - ref); h[r] = ex2(m - ref);
                st.l[r] = st.l[r] * f[r] + l * h[r];
                st.m[r] = top;
            }
#pragma unroll
            for (int j = 0; j < DH / 8; ++j) {
                const float2 x = *reinterpret_cast<float2 *>(mine + g * S::ld + 8 * j + 2 * t), y = *reinterpret_cast<float2 *>(mine + (g + 8) * S::ld + 8 * j + 2 * t);
                st.o[j][0] = st.o[j][0] * f[0] + x.x * h[0]; st.o[j][1] = st.o[j][1] * f[0] + x.y * h[0];
                st.o[j][2] = st.o[j][2] * f[1] + y.x * h[1]; st.o[j][3] = st.o[j][3] * f[1] + y.y * h[1];
            }
            __syncwarp();
        }
        if (warp < A.parked) park();
        bar_attend<W>();
        const int items = rows * (DH / 4), tiles = A.rt;
        float *place = A.partial;
        if (!seg.whole) {
            place += (2 * (long long)blockIdx.x + (run.start(blockIdx.x) < seg.first ? 1 : 0)) * slot_floats;
        }
        for (int i = tid; i < items; i += W * 32) {
            const int r = i / (DH / 4), d = (i - r * (DH / 4)) * 4;
            float m = -INFINITY, l = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
            float2 ml[4];
            float4 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int w = (r >> 4) + k * tiles;
                ml[k] = make_float2(-INFINITY, 0.f);
                x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (w < A.parked) {
                    ml[k] = *reinterpret_cast<const float2 *>(parked_ml + w * 32 + 2 * (r & 15));
                    x[k] = *reinterpret_cast<const float4 *>(parked + (w * 16 + (r & 15)) * S::ld + d);
                }
                m = fmaxf(m, ml[k].x);
            }
            const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float f = ex2(ml[k].x - ref);
                l += ml[k].y * f;
                o.x += x[k].x * f; o.y += x[k].y * f; o.z += x[k].z * f; o.w += x[k].w * f;
            }
            if (seg.whole) {
                finish<TQ>(A, s_rows[0][r], d, o, m, l);
            } else {
                __stcg(reinterpret_cast<float4 *>(place + r * DH + d), o);
                if (d == 0) __stcg(reinterpret_cast<float2 *>(place + A.rt * 16 * DH + 2 * r), make_float2(m, l));
            }
        }
        if (!seg.whole) {
            // CTAs whose runs meet this unit: the one with its first granule to the one with its last.  Whether this CTA is the last of them to
            // be there is asked at its end, when all its runs' writes are done.
            if (tid == 0) {
                const int c0 = run.owner(seg.first + kOpening), c1 = run.owner(seg.last - 1);
                s_left[pending] = Left{b, seg.unit, sp.nq, c0, c1, run.start(c0) < seg.first, false};
            }
            ++pending;
        }
    });
    if (pending == 0) return;
    bar_attend<W>();
    if (tid < pending) {
        // c0 is the first at no other unit that is cut: its counter is this unit's
        int *counter = A.counters + s_left[tid].c0, before;
        asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
        const bool last = before == s_left[tid].c1 - s_left[tid].c0;
        if (last) *counter = 0;                  // as the next call wants it
        s_left[tid].last = last;
    }
    bar_attend<W>();
    // two of them: half of the warps each
    const bool both = pending == 2 && s_left[0].last && s_left[1].last;
    const int first = both ? tid % (W * 16) : tid, step = both ? W * 16 : W * 32;
    for (int u = 0; u < pending; ++u) {
        const Left &left = s_left[u];
        if (left.last && tid < min(A.rt * 16, A.n_rows - (left.unit % A.row_groups) * A.rt * 16)) place_row(A, left.b, left.unit, left.nq, tid, s_rows[u]);
    }
    bar_attend<W>();
    for (int u = both ? tid / (W * 16) : 0; u < (both ? tid / (W * 16) + 1 : pending); ++u) {
        const Left left = s_left[u];
        if (!left.last) continue;
        const int n = min(A.rt * 16, A.n_rows - (left.unit % A.row_groups) * A.rt * 16) * (DH / 4);
        // kItems pieces of the output times kWay parts on their way at a time
        auto join = [&](auto items_, auto way_) {
            constexpr int kItems = decltype(items_)::value, kWay = decltype(way_)::value;
            for (int i0 = first; i0 < n; i0 += step * kItems) {
                float m[kItems], l[kItems];
                float4 o[kItems];
#pragma unroll
                for (int q = 0; q < kItems; ++q) { m[q] = -INFINITY; l[q] = 0.f; o[q] = make_float4(0.f, 0.f, 0.f, 0.f); }
                for (int c = left.c0; c <= left.c1; c += kWay) {
                    float2 ml[kItems][kWay];
                    float4 x[kItems][kWay];
#pragma unroll
                    for (int k = 0; k < kWay; ++k) {
                        const float *from = A.partial + (2 * (long long)(c + k) + (c + k == left.c0 && left.second ? 1 : 0)) * slot_floats;
#pragma unroll
                        for (int q = 0; q < kItems; ++q) {
                            const int i = i0 + q * step;
                            ml[q][k] = make_float2(-INFINITY, 0.f);
                            x[q][k] = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (c + k <= left.c1 && i < n) {
                                ml[q][k] = __ldcg(reinterpret_cast<const float2 *>(from + A.rt * 16 * DH) + i / (DH / 4));
                                x[q][k] = __ldcg(reinterpret_cast<const float4 *>(from) + i);
                            }
                        }
                    }
#pragma unroll
                    for (int q = 0; q < kItems; ++q) {
                        float top = m[q];
#pragma unroll
                        for (int k = 0; k < kWay; ++k) top = fmaxf(top, ml[q][k].x);
                        const float ref = top == -INFINITY ? 0.f : top, f0 = ex2(m[q] - ref);
                        l[q] *= f0; o[q].x *= f0; o[q].y *= f0; o[q].z *= f0; o[q].w *= f0;
                        m[q] = top;
#pragma unroll
                        for (int k = 0; k < kWay; ++k) {
                            const float f = ex2(ml[q][k].x - ref);
                            l[q] += ml[q][k].y * f;
                            o[q].x += x[q][k].x * f; o[q].y += x[q][k].y * f; o[q].z += x[q][k].z * f; o[q].w += x[q][k].w * f;
                        }
                    }
                }
#pragma unroll
                for (int q = 0; q < kItems; ++q) {
                    const int i = i0 + q * step, r = i / (DH / 4);
                    if (i < n) finish<TQ>(A, s_rows[u][r], (i - r * (DH / 4)) * 4, o[q], m[q], l[q]);
                }
            }
        };
        if (left.c1 - left.c0 < 4 && n > step) join(std::integral_constant<int, 2>(), std::integral_constant<int, 4>());
        else join(std::integral_constant<int, 1>(), std::integral_constant<int, 8>());
    }
}

// --------------------------------------------------------------------------------------------- host

struct AttendPlan {
    int rt, row_groups, ring, turns, producers, parked, smem, grid;
    long long units;
    size_t workspace;
};

static AttendPlan plan_attend(const xsm_kv &kv, int batch, int m, int n_heads, int q_dtype) {
    const xsm_kv_config &c = kv.cfg;
    const int es = element_size(c.dtype), rows = m * (n_heads / c.n_kv_heads), tiles = (rows + 15) / 16;
    AttendPlan p;
    const int q = query_bytes(c.d_head, es, es == 4 || q_dtype == XSM_F32) + raw_bytes(c.d_head, element_size(q_dtype)), stage = 2 * kStage * c.d_head * es;
    const int warps = attend_warps(c.d_head) / slices_of(c.d_head, es);      // that could take stages of their own
    p.rt = tiles >= 3 ? 4 : tiles;
    while (p.rt > warps) p.rt /= 2;
    // Shared memory: the ring gets what the parked states and the queries leave.  A group of warps that takes stages wants two places, one to
    // work on and one that fills; so few groups that wide rows leave no room, then fewer row tiles.
    const int most = attend_warps(c.d_head) / 2;
    auto parked = [&](int rt, int turns) { const int n = rt * turns * slices_of(c.d_head, es); return n < most ? n : most; };
    auto left = [&](int rt, int turns) { return kCtaSmem - kDeclared - parked_bytes(c.d_head, parked(rt, turns)) - rt * q; };
    for (;; p.rt /= 2) {
        p.turns = warps / p.rt;
        while (p.turns > 1 && left(p.rt, p.turns) / stage < 2 * p.turns) p.turns /= 2;
        if (p.rt == 1 || left(p.rt, p.turns) / stage >= 2) break;
    }
    p.parked = parked(p.rt, p.turns);
    p.ring = left(p.rt, p.turns) / stage < kRing ? left(p.rt, p.turns) / stage : kRing;
    // Whoever waits for a stage must have seen the one before it in the same place (a barrier tells one phase from the next, not from the
    // one after): groups of warps, and producers, have places of the ring of their own.  (All are powers of two, none larger than the ring.)
    p.producers = kProducers;
    while (p.producers > p.ring) p.producers /= 2;
    p.ring -= p.ring % (p.turns > p.producers ? p.turns : p.producers);
    p.row_groups = (tiles + p.rt - 1) / p.rt;
    p.smem = p.ring * stage + parked_bytes(c.d_head, p.parked) + p.rt * q;
    p.units = (long long)batch * c.n_kv_heads * p.row_groups;
    p.grid = kv.sms < kMaxGrid ? kv.sms : kMaxGrid;
    p.workspace = kHeadBytes + 2 * (size_t)p.grid * p.rt * 16 * (c.d_head + 2) * 4;
    return p;
}

template <typename T, typename TQ, int DH>
static cudaError_t launch_attend(const xsm_kv &kv, const AttendArgs &A, const AttendPlan &p, cudaStream_t st) {
    const void *fn = (const void *)attend_kernel<T, TQ, DH>;
    const cudaError_t e = open_kernel(fn, p.smem, false);
    if (e != cudaSuccess) return e;
    return launch_early(attend_kernel<T, TQ, DH>, dim3(p.grid), dim3((attend_warps(DH) + kProducers) * 32), p.smem, st, kv.k_map, kv.v_map, A);
}
template <typename T, typename TQ> static cudaError_t launch_width(const xsm_kv &kv, const AttendArgs &A, const AttendPlan &p, cudaStream_t st) {
    switch (kv.cfg.d_head) {
        case 32: return launch_attend<T, TQ, 32>(kv, A, p, st);
        case 64: return launch_attend<T, TQ, 64>(kv, A, p, st);
        case 96: return launch_attend<T, TQ, 96>(kv, A, p, st);
        case 128: return launch_attend<T, TQ, 128>(kv, A, p, st);
        default: return launch_attend<T, TQ, 256>(kv, A, p, st);
    }
}

}  // namespace xsm

using namespace xsm;

size_t xsm_kv_attend_workspace(const xsm_kv *kv, int batch, int m, int n_heads) {
    if (!kv || batch < 1 || m < 1 || m > XSM_MAX_DRAFT || n_heads < 1 || n_heads > 4096 || n_heads % kv->cfg.n_kv_heads) return 0;
    const size_t a = plan_attend(*kv, batch, m, n_heads, kv->cfg.dtype).workspace, b = plan_attend(*kv, batch, m, n_heads, XSM_F32).workspace;
    return a > b ? a : b;
}

xsm_status xsm_kv_attend(const xsm_kv *kv, const xsm_kv_attend_args *a, void *cuda_stream) {
    if (!kv || !a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    const xsm_kv_config &c = kv->cfg;
    if (a->batch < 0 || a->max_pages < 0) return op_failed(XSM_ERR_INVALID_ARG, "batch and max_pages must not be negative");
    if (a->m < 1 || a->m > XSM_MAX_DRAFT) return op_failed(XSM_ERR_INVALID_ARG, "m must be in [1, 16]");
    if (a->n_heads < 1 || a->n_heads > 4096 || a->n_heads % c.n_kv_heads) return op_failed(XSM_ERR_INVALID_ARG, "n_heads must be a multiple of n_kv_heads, at most 4096");
    if (!is_dtype(a->q_dtype) || (a->q_dtype != c.dtype && c.dtype != XSM_F16))
        return op_failed(XSM_ERR_INVALID_ARG, "q_dtype must be the pools' type (over an fp16 pool: any)");
    if (a->window < 0 || (a->window && !a->causal)) return op_failed(XSM_ERR_INVALID_ARG, "window must not be negative, and needs causal");
    if (!(fabsf(a->scale) < INFINITY)) return op_failed(XSM_ERR_INVALID_ARG, "scale must be finite");
    if (a->batch == 0) return XSM_OK;
    if (!a->q || !a->out || (!a->block_table && a->max_pages) || !a->lengths || !a->workspace) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    const AttendPlan p = plan_attend(*kv, a->batch, a->m, a->n_heads, a->q_dtype);
    if ((double)p.units * ((double)a->max_pages * c.page_size / (kStage * kGranule) + kOpening + 2) > INT_MAX / 2) return op_failed(XSM_ERR_INVALID_ARG, "batch * heads * positions is too large");
    if (a->workspace_bytes < (int64_t)p.workspace) return op_failed(XSM_ERR_CAPACITY, "the workspace is too small");
    const int per16 = 16 / element_size(a->q_dtype);
    for (int i = 0; i < 3; ++i)
        if (a->q_stride[i] % per16 || a->out_stride[i] % per16) return op_failed(XSM_ERR_INVALID_ARG, "strides of q and out must be multiples of 16 bytes");
    if (((uintptr_t)a->q | (uintptr_t)a->out | (uintptr_t)a->workspace) % 16) return op_failed(XSM_ERR_INVALID_ARG, "q, out and workspace must be 16-byte aligned");
    AttendArgs A;
    A.q = a->q; A.out = a->out; A.lse = a->lse; A.lengths = a->lengths; A.counts = a->counts; A.table = a->block_table; A.table_ld = a->table_stride;
    A.status = (int *)a->workspace;
    A.counters = A.status + 4;
    A.partial = reinterpret_cast<float *>((char *)a->workspace + kHeadBytes);
    for (int i = 0; i < 3; ++i) { A.qs[i] = a->q_stride[i]; A.os[i] = a->out_stride[i]; }
    A.batch = a->batch; A.m = a->m; A.heads = a->n_heads; A.group = a->n_heads / c.n_kv_heads; A.kv_heads = c.n_kv_heads;
    A.whole = kWholeBytes / (2 * kStage * c.d_head * element_size(c.dtype)); A.rt = p.rt; A.row_groups = p.row_groups; A.n_rows = A.m * A.group; A.ring = p.ring; A.turns = p.turns; A.producers = p.producers; A.parked = p.parked;
    A.causal = a->causal != 0; A.page = c.page_size; A.max_pages = a->max_pages; A.n_pages = c.n_pages; A.box_rows = kv->box_rows;
    A.c = (float)((double)a->scale * 1.4426950408889634);
    A.tries = kv->tries;
    A.starve = kv->starve;
    // (lengths end at INT_MAX - 2 kStage: a larger window sees no more, and would not go below a first end of -15)
    A.window = a->window < INT_MAX - kStage ? a->window : INT_MAX - kStage;
    A.all_units = (float)p.units;
    A.part_scale = A.all_units * A.all_units * 16.f * element_size(c.dtype) / ((float)A.batch * (float)(A.n_rows < 16 * A.rt ? A.n_rows : 16 * A.rt));
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    if (c.dtype == XSM_F32) return launched(launch_width<float, float>(*kv, A, p, st));
    if (c.dtype == XSM_BF16) return launched(launch_width<bf16, bf16>(*kv, A, p, st));
    if (a->q_dtype == XSM_F32) return launched(launch_width<__half, float>(*kv, A, p, st));
    if (a->q_dtype == XSM_BF16) return launched(launch_width<__half, bf16>(*kv, A, p, st));
    return launched(launch_width<__half, __half>(*kv, A, p, st));
}
