// Rows of logits (fp32 or bf16): loads under a mask of legal entries, the sums that
// every loss over a row needs, and their combination over the threads that share it.
#pragma once

#include "internal.hpp"

#include "chunk.hpp"
#include "device.hpp"

namespace malib {

namespace {   // (each kernel file's own)

typedef float f32x4 __attribute__((ext_vector_type(4)));

enum { kPolicy, kPolicyRef, kDistill };   // template KIND

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kNegInf = -__builtin_inff();

// 2^x on the hardware (1 ulp; results below 2^-126 are 0)
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// e is 0 below 2^-126: exponents under this one are replaced by it, so that e d is 0
// and not NaN where d is -inf
constexpr float kLeast = -256.0f;

struct Stats {
    float m, s, t;     // of the logits
    float my, sy, v;   // of the reference
};

__device__ __forceinline__ Stats empty_stats()
{
    return Stats{kNegInf, 0.0f, 0.0f, kNegInf, 0.0f, 0.0f};
}

// a + b, both parts of one row.  An empty part (or one of -inf only) has s = 0.
template <int KIND>
__device__ __forceinline__ Stats merge(const Stats& a, const Stats& b, float c)
{
    Stats r;
    r.m = fmaxf(a.m, b.m);
    const float da = a.s == 0.0f ? 0.0f : fmaxf((a.m - r.m) * c, kLeast);
    const float db = b.s == 0.0f ? 0.0f : fmaxf((b.m - r.m) * c, kLeast);
    const float ra = exp2_hw(da), rb = exp2_hw(db);   // 0 at kLeast
    r.s = a.s * ra + b.s * rb;
    r.t = 0.0f;
    if (KIND != kDistill)
        r.t = ra * (a.t + a.s * da) + rb * (b.t + b.s * db);
    r.my = r.sy = r.v = 0.0f;
    if (KIND == kPolicyRef) {
        r.my = fmaxf(a.my, b.my);
        const float fa = a.my == kNegInf ? kNegInf : (a.my - r.my) * kLog2e;
        const float fb = b.my == kNegInf ? kNegInf : (b.my - r.my) * kLog2e;
        r.sy = a.sy * exp2_hw(fa) + b.sy * exp2_hw(fb);
        r.v = (a.s == 0.0f || ra == 0.0f ? 0.0f : ra * (a.v + a.s * fa)) +
              (b.s == 0.0f || rb == 0.0f ? 0.0f : rb * (b.v + b.s * fb));
    }
    return r;
}

// The sums of one entry, relative to the maxima m and my (0 where -inf).
template <int KIND>
__device__ __forceinline__ void add_entry(Stats& r, float x, float y, float m, float my, float c)
{
    const float d = (x - m) * c, e = exp2_hw(d);
    r.s += e;
    if (KIND != kDistill)
        r.t = __builtin_fmaf(e, fmaxf(d, kLeast), r.t);
    if (KIND == kPolicyRef) {
        const float f = (y - my) * kLog2e;
        r.sy += exp2_hw(f);
        r.v = __builtin_fmaf(e, e > 0.0f ? f : 0.0f, r.v);
    }
}

// What a row's gradient needs.
struct RowGrad {
    float m, my, c0, c1, c2;
    float with_ref;       // the reference enters where e is above: 0, or inf (nowhere)
    float at_action;      // policy: added at the action
};

template <int KIND>
__device__ __forceinline__ float grad_entry(const RowGrad& g, float x, float y, float c)
{
    const float d = (x - g.m) * c, e = exp2_hw(d);
    float k = g.c0;
    if (KIND != kDistill)
        k = __builtin_fmaf(g.c1, fmaxf(d, kLeast), k);
    if (KIND == kPolicyRef)
        k = __builtin_fmaf(g.c2, e > g.with_ref ? (y - g.my) * kLog2e : 0.0f, k);
    return e * k;
}

constexpr uint32_t kNegInfBits = 0xFF800000u;

// v with -inf as entry i
template <typename E>
__device__ __forceinline__ void exclude(u32x4& v, int i, bool out)
{
    if constexpr (sizeof(E) == 4) {
        v[i] = out ? kNegInfBits : v[i];
    } else {
        const uint32_t w = v[i >> 1];
        v[i >> 1] = out ? ((i & 1) ? (w & 0xFFFFu) | kNegInfBits
                                   : (w & 0xFFFF0000u) | (kNegInfBits >> 16))
                        : w;
    }
}

typedef uint32_t u32_any __attribute__((aligned(1)));
typedef uint64_t u64_any __attribute__((aligned(1)));

// Chunk at p of a row of which n entries are left and `before` lie in front, with -inf
// in the entries behind the row's end and those that are not legal.
template <typename E>
__device__ __forceinline__ u32x4 load_masked(const E* p, int n, const uint8_t* mask, int64_t before)
{
    constexpr int CH = kChunk<E>;
    if (n >= CH) {
        u32x4 v = *(const u32x4_any*)p;
        if (mask) {
#pragma unroll
            for (int i = 0; i < CH; i += 4) {
                const uint32_t b = *(const u32_any*)(mask + i);
                exclude<E>(v, i, (b & 0xFFu) == 0);
                exclude<E>(v, i + 1, (b & 0xFF00u) == 0);
                exclude<E>(v, i + 2, (b & 0xFF0000u) == 0);
                exclude<E>(v, i + 3, (b & 0xFF000000u) == 0);
            }
        }
        return v;
    }
    u32x4 v = {0, 0, 0, 0};
    uint64_t m = 0;   // bit 8 i up: entry i is legal
    if (n > 0) {
        v = load_chunk(p, n, before);
        m = ~0ull >> (64 - 8 * n);
        if (mask) {
            if (before + n >= 8) {   // the 8 bytes before the row's end
                m = *(const u64_any*)(mask + n - 8) >> (64 - 8 * n);
            } else {
                m = 0;
                for (int i = 0; i < n; ++i)
                    m |= (uint64_t)mask[i] << (8 * i);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < CH; ++i)
        exclude<E>(v, i, ((uint32_t)(m >> (32 * (i / 4))) >> (8 * (i % 4)) & 0xFFu) == 0);
    return v;
}

// ------------------------------------------------- few actions: a lane per row

// 64 rows per wavefront, up to kLaneMost entries each: rows go through LDS as one run
// of values, so that memory is read and written in its own order, 16 bytes per
// lane where rows follow each other without gaps, while each lane works on a row
// alone in registers: no reductions, and a row's scalar work is not repeated by
// other lanes.  A lane moves its row in the widest pieces that rows are aligned
// to: pieces of neighbouring rows then fall into different banks unless A is a
// multiple of 8 (up to 4 lanes per bank at 16).  (Rows padded to an odd stride
// instead, their places found element by element: 105 us against 94 us for 2^21
// rows of 18.)
// Bound by memory for many rows: 2097152 x 18 fp32 86 us, 4.2 TB/s; 192 rows with masks and
// reference logits 9 us, one chain of loads, LDS and stores.
constexpr int kLaneThreads = 256, kLaneRows = 64, kLaneMost = 31;

// i / w for i < 2048, w <= 32
struct SmallDiv {
    uint32_t magic;
    __device__ __forceinline__ explicit SmallDiv(int w) : magic((1u << 20) / (uint32_t)w + 1u) {}
    __device__ __forceinline__ int operator()(int i) const
    {
        return (int)(((uint32_t)i * magic) >> 20);
    }
};

// n rows of w values (rows ld apart) into LDS, value j of row r at r * w + j, or at
// r * (w + 1) + j with PAD; -inf where the mask excludes an entry.  With BOTH a
// second array of the same shape under the same mask goes along: a round of the
// loop asks for everything it needs before it waits.
template <bool PAD, bool BOTH, typename E>
__device__ __forceinline__ void rows_to_lds(const E* p, int64_t ld, const E* p2, int64_t ld2,
                                            const uint8_t* mask, int64_t mask_ld, int n, int w,
                                            float* to, float* to2, int lane)
{
    constexpr int CH = kChunk<E>;
    const int count = n * w;
    const SmallDiv div(w);
    auto put = [&](float* t, int i, u32x4 raw) {
        float v[CH];
        unpack<E>(raw, v);
        if (!PAD && i + CH <= count) {
#pragma unroll
            for (int e = 0; e < CH; e += 4)
                *(f32x4*)(t + i + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
        } else {
#pragma unroll
            for (int e = 0; e < CH; ++e)
                if (i + e < count)
                    t[i + e + (PAD ? div(i + e) : 0)] = v[e];
        }
    };
    if (ld == w && (!BOTH || ld2 == w) && (!mask || mask_ld == w)) {
        constexpr int U = 2;
        for (int i0 = lane * CH; i0 < count; i0 += U * 64 * CH) {
            u32x4 v[U], v2[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * 64 * CH;
                v[u] = load_masked(p + i, count - i, mask ? mask + i : nullptr, i);
                if (BOTH)
                    v2[u] = load_masked(p2 + i, count - i, mask ? mask + i : nullptr, i);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * 64 * CH;
                if (i < count) {
                    put(to, i, v[u]);
                    if (BOTH)
                        put(to2, i, v2[u]);
                }
            }
        }
        return;
    }
    constexpr int U = 4;
    for (int i0 = lane; i0 < count; i0 += U * 64) {
        float v[U], v2[U];
        int at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * 64;
            v[u] = v2[u] = kNegInf;
            at[u] = -1;
            if (i < count) {
                const int r = div(i), j = i - r * w;
                const bool legal = !mask || mask[r * mask_ld + j] != 0;
                const float x = to_f32(p[r * ld + j]);
                v[u] = legal ? x : kNegInf;
                if (BOTH) {
                    const float y = to_f32(p2[r * ld2 + j]);
                    v2[u] = legal ? y : kNegInf;
                }
                at[u] = i + (PAD ? r : 0);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (at[u] >= 0) {
                to[at[u]] = v[u];
                if (BOTH)
                    to2[at[u]] = v2[u];
            }
    }
}

template <typename E>
__device__ __forceinline__ void rows_from_lds(const float* from, E* p, int64_t ld, int n, int w,
                                              int lane)
{
    constexpr int CH = kChunk<E>;
    const int count = n * w;
    if (ld == w) {
        for (int i = lane * CH; i < count; i += 64 * CH) {
            float v[CH];
            if (i + CH <= count) {
#pragma unroll
                for (int e = 0; e < CH; e += 4) {
                    const f32x4 q = *(const f32x4*)(from + i + e);
                    v[e] = q[0];
                    v[e + 1] = q[1];
                    v[e + 2] = q[2];
                    v[e + 3] = q[3];
                }
            } else {
#pragma unroll
                for (int e = 0; e < CH; ++e)
                    v[e] = i + e < count ? from[i + e] : 0.0f;
            }
            store_chunk(p + i, count - i, pack<E>(v));
        }
        return;
    }
    const SmallDiv div(w);
    for (int i = lane; i < count; i += 64) {
        const int r = div(i), j = i - r * w;
        p[r * ld + j] = from_f32<E>(from[i]);
    }
}

// A lane's row of A <= NA values between LDS and registers, in pieces of W values
// (A a multiple of W).
template <int NA, int W>
__device__ __forceinline__ void row_read(const float* p, int A, float (&x)[NA])
{
    typedef float piece __attribute__((ext_vector_type(W)));
#pragma unroll
    for (int j = 0; j < NA; j += W) {
        if (j >= A)
            break;
        const piece q = *(const piece*)(p + j);
#pragma unroll
        for (int e = 0; e < W; ++e)
            x[j + e] = q[e];
    }
}
template <int NA, int W>
__device__ __forceinline__ void row_write(float* p, int A, const float (&x)[NA])
{
    typedef float piece __attribute__((ext_vector_type(W)));
#pragma unroll
    for (int j = 0; j < NA; j += W) {
        if (j >= A)
            break;
        piece q;
#pragma unroll
        for (int e = 0; e < W; ++e)
            q[e] = x[j + e];
        *(piece*)(p + j) = q;
    }
}
template <int NA>
__device__ __forceinline__ void row_read(const float* p, int A, float (&x)[NA])
{
    if (A % 4 == 0)
        row_read<NA, 4>(p, A, x);
    else if (A % 2 == 0)
        row_read<NA, 2>(p, A, x);
    else {
#pragma unroll
        for (int j = 0; j < NA; ++j) {
            if (j >= A)
                break;
            x[j] = p[j];
        }
    }
}
template <int NA>
__device__ __forceinline__ void row_write(float* p, int A, const float (&x)[NA])
{
    if (A % 4 == 0)
        row_write<NA, 4>(p, A, x);
    else if (A % 2 == 0)
        row_write<NA, 2>(p, A, x);
    else {
#pragma unroll
        for (int j = 0; j < NA; ++j) {
            if (j >= A)
                break;
            p[j] = x[j];
        }
    }
}

// ------------------------------------------------------- a group of lanes per row

// T threads per row: neighbouring lanes of one wavefront (T <= 64) or a workgroup.
template <int T>
__device__ __forceinline__ void group_sync()
{
    if constexpr (T <= 64)
        wave_lds_sync();
    else
        __syncthreads();
}

struct MaxOp {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct SumOp {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

template <int CTRL>
__device__ __forceinline__ float dpp(float v)
{
    return __uint_as_float(
        __builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}

// v combined over groups of N lanes (N a power of two up to 64), in every lane:
// neighbours, pairs, then mirrored halves of 8 and 16 lanes (whose lanes are equal by
// then), which need no LDS; the last two steps cross rows of 16 lanes.
template <int N, typename Op>
__device__ __forceinline__ float lanes_combine(float v, Op op)
{
    if constexpr (N >= 2)
        v = op(v, dpp<0xB1>(v));     // quad_perm 1 0 3 2
    if constexpr (N >= 4)
        v = op(v, dpp<0x4E>(v));     // quad_perm 2 3 0 1
    if constexpr (N >= 8)
        v = op(v, dpp<0x141>(v));    // row_half_mirror
    if constexpr (N >= 16)
        v = op(v, dpp<0x140>(v));    // row_mirror
    if constexpr (N >= 32)
        v = op(v, __shfl_xor(v, 16));
    if constexpr (N >= 64)
        v = op(v, __shfl_xor(v, 32));
    return v;
}

// n values combined over the group, in every thread, always in the same order.
// T > 64: through half HALF (0 or 1) of `scratch`, with one barrier.  Calls use the
// halves in turn: a thread writes a half again only after the barrier of the call
// on the other half, by when all have read it.
constexpr int kScratch = 16 * 4;   // floats of a half

template <int T, int HALF, int NV, typename Op>
__device__ __forceinline__ void group_combine(float (&v)[NV], Op op, float* scratch)
{
#pragma unroll
    for (int i = 0; i < NV; ++i)
        v[i] = lanes_combine<(T < 64 ? T : 64)>(v[i], op);
    if constexpr (T > 64) {
        constexpr int W = T / 64;
        float* half = scratch + HALF * kScratch;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                half[(threadIdx.x >> 6) * NV + i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i)
            v[i] = lanes_combine<W>(half[(threadIdx.x & (W - 1)) * NV + i], op);
    }
}

// The group's parts of a row as one, in every thread: the common maxima first, then
// each thread's sums rescaled to them.  `flag` (in LDS, set before the call) clears
// `counts` where it is 0.
template <int T, int KIND>
__device__ __forceinline__ Stats group_merge(const Stats& st, float c, float* scratch,
                                             const int* flag, bool& counts)
{
    Stats r = empty_stats();
    if constexpr (KIND == kPolicyRef) {
        float mx[2] = {st.m, st.my};
        group_combine<T, 0>(mx, MaxOp(), scratch);
        r.m = mx[0];
        r.my = mx[1];
    } else {
        float mx[1] = {st.m};
        group_combine<T, 0>(mx, MaxOp(), scratch);
        r.m = mx[0];
    }
    if (flag)
        counts = counts && *flag != 0;
    const float d = st.s == 0.0f ? 0.0f : fmaxf((st.m - r.m) * c, kLeast);
    const float k = exp2_hw(d);   // 0 at kLeast
    if constexpr (KIND == kPolicyRef) {
        const float f = st.my == kNegInf ? kNegInf : (st.my - r.my) * kLog2e;
        float sum[4] = {st.s * k, k * (st.t + st.s * d), st.sy * exp2_hw(f),
                        st.s == 0.0f || k == 0.0f ? 0.0f : k * (st.v + st.s * f)};
        group_combine<T, 1>(sum, SumOp(), scratch);
        r.s = sum[0];
        r.t = sum[1];
        r.sy = sum[2];
        r.v = sum[3];
    } else if constexpr (KIND == kPolicy) {
        float sum[2] = {st.s * k, k * (st.t + st.s * d)};
        group_combine<T, 1>(sum, SumOp(), scratch);
        r.s = sum[0];
        r.t = sum[1];
    } else {
        float sum[1] = {st.s * k};
        group_combine<T, 1>(sum, SumOp(), scratch);
        r.s = sum[0];
    }
    return r;
}

// Between two uses of a thread's chunks: the raw chunks are what stays in registers,
// not their unpacked values (twice as many in bf16).
template <int KIND, int C>
__device__ __forceinline__ void keep_raw(u32x4 (&x)[C], u32x4* y)
{
#pragma unroll
    for (int i = 0; i < C; ++i) {
        asm volatile("" : "+v"(x[i]));
        if (KIND == kPolicyRef)
            asm volatile("" : "+v"(y[i]));
    }
}

// The sums over the first `used` of C chunks that a thread holds.
template <typename E, int KIND, int C>
__device__ __forceinline__ Stats chunk_stats(u32x4 (&x)[C], u32x4* y, int used, float c)
{
    constexpr int CH = kChunk<E>;
    Stats st = empty_stats();
#pragma unroll
    for (int i = 0; i < C; ++i) {
        if (i >= used)
            break;
        float f[CH];
        unpack<E>(x[i], f);
#pragma unroll
        for (int e = 0; e < CH; ++e)
            st.m = fmaxf(st.m, f[e]);
        if (KIND == kPolicyRef) {
            unpack<E>(y[i], f);
#pragma unroll
            for (int e = 0; e < CH; ++e)
                st.my = fmaxf(st.my, f[e]);
        }
    }
    const float m = st.m == kNegInf ? 0.0f : st.m, my = st.my == kNegInf ? 0.0f : st.my;
    keep_raw<KIND>(x, y);
#pragma unroll
    for (int i = 0; i < C; ++i) {
        if (i >= used)
            break;
        float f[CH], r[CH];
        unpack<E>(x[i], f);
        if (KIND == kPolicyRef)
            unpack<E>(y[i], r);
#pragma unroll
        for (int e = 0; e < CH; ++e)
            add_entry<KIND>(st, f[e], KIND == kPolicyRef ? r[e] : 0.0f, m, my, c);
        __builtin_amdgcn_sched_barrier(0);
    }
    return st;
}

// A row's chunks into registers, -inf in the entries that are not legal or not there,
// and everywhere in a row that does not count.  Within a wavefront (T <= 64) every
// chunk has its own conditions, so that all are asked for together; in workgroups the
// chunks that all threads hold whole take none, and the one round that the row's end
// falls into comes first, which leaves registers for more wavefronts (fp32, 2048 x
// 32000 with reference logits: 173 us, with conditions on every chunk 290 us, with that
// round last 196 us; 559269 x 91: 120, as workgroups' rows 139 us).
template <typename E, int KIND, int T, int C>
__device__ __forceinline__ void load_row(int A, bool counts, const E* px, const E* py,
                                         const uint8_t* pm, int lane, u32x4 (&x)[C], u32x4* y)
{
    constexpr int CH = kChunk<E>;
    if constexpr (T <= 64) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = (lane + i * T) * CH, n = counts ? A - j : 0;
            x[i] = load_masked(px + j, n, pm ? pm + j : nullptr, j);
            if (KIND == kPolicyRef)
                y[i] = load_masked(py + j, n, pm ? pm + j : nullptr, j);
        }
        return;
    }
    const int whole = A / (T * CH);
    const int jt = (lane + whole * T) * CH, nt = counts ? A - jt : 0;
    const u32x4 tx = load_masked(px + jt, nt, pm ? pm + jt : nullptr, jt);
    u32x4 ty = tx;
    if (KIND == kPolicyRef)
        ty = load_masked(py + jt, nt, pm ? pm + jt : nullptr, jt);
    const u32x4 none = load_masked((const E*)nullptr, 0, nullptr, 0);
#pragma unroll
    for (int i = 0; i < C; ++i) {
        x[i] = i == whole ? tx : none;
        if (KIND == kPolicyRef)
            y[i] = i == whole ? ty : none;
    }
    if (!counts)
        return;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        if (i < whole) {
            const int j = (lane + i * T) * CH;
            x[i] = *(const u32x4_any*)(px + j);
            if (KIND == kPolicyRef)
                y[i] = *(const u32x4_any*)(py + j);
        }
    }
    if (!pm)
        return;
    uint32_t legal[C][CH / 4];
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
        for (int e = 0; e < CH / 4; ++e)
            legal[i][e] = 0x01010101u;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        if (i < whole) {
            const int j = (lane + i * T) * CH;
#pragma unroll
            for (int e = 0; e < CH / 4; ++e)
                legal[i][e] = *(const u32_any*)(pm + j + 4 * e);
        }
    }
#pragma unroll
    for (int i = 0; i < C; ++i) {
#pragma unroll
        for (int e = 0; e < CH; ++e) {
            const bool out = (legal[i][e / 4] >> (8 * (e % 4)) & 0xFFu) == 0;
            exclude<E>(x[i], e, out);
            if (KIND == kPolicyRef)
                exclude<E>(y[i], e, out);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

}  // namespace

}  // namespace malib
