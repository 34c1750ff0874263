// The learner's losses over rows of logits, each with its gradient: the clipped
// policy loss with a divergence term, and the distillation of teachers' top
// logits.
//
// With x a row's legal logits, c = log2(e) / T and m = max x, everything a row
// needs comes from sums over e_j = 2^((x_j - m) c):
//   s = sum e,  t = sum e (x - m) c,  and, against reference logits y with
//   f = (y - max y) log2(e):  s_y = sum 2^f,  v = sum e f.
//   log p_j = (x_j - m) / T - ln s,  H = ln s - ln2 t / s,
//   KL = ln2 (t - v) / s - ln s + ln s_y.
// The gradient of either loss is e_j (c0 + c1 d_j + c2 f_j) with the row's c0, c1,
// c2, plus a term at the action or at the teacher's entries.  Parts of a row
// combine by rescaling their sums to the common maximum.
//
// All of it is bound by memory: logits (and reference, mask) in, gradient out.
#include "internal.hpp"

#include "chunk.hpp"
#include "device.hpp"

namespace malib {

namespace {

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

// A row's scalar inputs of the policy loss.
struct PolicyRow {
    int64_t action;
    float w, old_logp, advantage, ref_logp;
    bool counts;
};

template <int KIND>
__device__ __forceinline__ PolicyRow policy_row(const LossArgs& a, int64_t row)
{
    PolicyRow r;
    r.action = a.action_bytes == 1   ? (int64_t)((const uint8_t*)a.actions)[row]
               : a.action_bytes == 4 ? (int64_t)((const int32_t*)a.actions)[row]
                                     : ((const int64_t*)a.actions)[row];
    r.w = a.weight ? a.weight[row] : a.row_weight;
    r.old_logp = a.old_logp[row];
    r.advantage = a.advantage[row];
    r.ref_logp = KIND == kPolicy && a.ref_logp ? a.ref_logp[row] : 0.0f;
    r.counts = r.action >= 0 && r.action < a.A && r.w != 0.0f;
    if (r.counts && a.mask)
        r.counts = a.mask[row * a.mask_ld + r.action] != 0;
    return r;
}

struct PolicyOut {
    float loss, logp, kl, entropy;
};

// The loss of a row that counts and its gradient's coefficients; x_a: the action's
// logit.
template <int KIND>
__device__ __forceinline__ PolicyOut policy_finish(const LossArgs& a, const PolicyRow& row,
                                                   const Stats& st, float x_a, RowGrad& g)
{
    PolicyOut o;
    const float m = st.m == kNegInf ? 0.0f : st.m, my = st.my == kNegInf ? 0.0f : st.my;
    const float ln_s = logf(st.s), inv = 1.0f / st.s;
    o.logp = (x_a - m) - ln_s;
    o.entropy = ln_s - kLn2 * st.t * inv;
    const float adv = row.advantage, w = row.w;
    const float ratio = expf(o.logp - row.old_logp);
    const float lo = 1.0f - a.clip_low, hi = 1.0f + a.clip_high;
    const float s1 = ratio * adv, s2 = (ratio < lo ? lo : ratio > hi ? hi : ratio) * adv;
    float slope = s1 <= s2 ? -s1 : s1 != s1 ? s1 : 0.0f;   // d loss / d log p[action]
    o.loss = -(s2 < s1 ? s2 : s1);
    o.kl = 0.0f;
    // (a divergence with a coefficient of 0 is a statistic only: infinite or NaN, it
    // leaves loss and gradient alone)
    const bool with_kl = a.kl_coef != 0.0f;
    float pull = 0.0f;   // of the divergence, in every logit
    if (KIND == kPolicyRef) {
        const float ln_sy = logf(st.sy);
        o.kl = kLn2 * (st.t - st.v) * inv - ln_s + ln_sy;
        if (with_kl)
            pull = a.kl_coef * (ln_sy - ln_s - o.kl);
    } else if (a.ref_logp) {
        const float d = row.ref_logp - o.logp;
        const float em = expm1f(d);
        o.kl = em - d;
        if (with_kl)
            slope -= a.kl_coef * em;
    }
    if (with_kl)
        o.loss += a.kl_coef * o.kl;
    if (a.entropy_coef != 0.0f)
        o.loss -= a.entropy_coef * o.entropy;
    const float k = w * inv;
    g.m = m;
    g.my = my;
    g.c0 = k * (pull + a.entropy_coef * (o.entropy - ln_s) - slope);
    g.c1 = k * kLn2 * (a.entropy_coef + (KIND == kPolicyRef ? a.kl_coef : 0.0f));
    g.c2 = KIND == kPolicyRef ? -k * kLn2 * a.kl_coef : 0.0f;
    g.with_ref = with_kl ? 0.0f : -kNegInf;
    g.at_action = w * slope;
    return o;
}

__device__ __forceinline__ void store_policy(const LossArgs& a, int64_t row, const PolicyOut& o)
{
    if (!a.stats)
        return;
    a.stats[row] = o.loss;
    a.stats[a.rows + row] = o.logp;
    a.stats[2 * a.rows + row] = o.kl;
    a.stats[3 * a.rows + row] = o.entropy;
}

// Sum of one value per thread over the workgroup (in a fixed order), in thread 0.
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double part[16];
#pragma unroll
    for (int o = 32; o; o >>= 1)
        v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = v;
    __syncthreads();
    double t = 0.0;
    if (threadIdx.x == 0)
        for (int i = 0; i < (int)(blockDim.x >> 6); ++i)
            t += part[i];
    return t;
}

__device__ __forceinline__ void store_total(const LossArgs& a, double t)
{
    if (!a.total || threadIdx.x != 0)
        return;
    if (gridDim.x == 1)
        *a.total = (float)t;
    else
        a.part_total[blockIdx.x] = t;
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

// Floats of LDS per row: logits, the reference's or the teacher's dense
// probabilities, the teacher's list.
__host__ __device__ constexpr int lane_floats(int kind, int A, int top)
{
    return A * (kind == kPolicy ? 1 : 2) + (kind == kDistill ? 2 * (top + 1) : 0);
}

// NA: entries in registers, A rounded up to 8
template <typename E, int KIND, int NA>
__global__ __launch_bounds__(kLaneThreads) void loss_lane_kernel(LossArgs a)
{
    extern __shared__ float lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int A = a.A, top = KIND == kDistill ? a.top : 0, ldt = top + 1;
    float* bx = lds + wave * kLaneRows * lane_floats(KIND, A, top);
    float* by = bx + kLaneRows * A;
    float* bv = by + kLaneRows * A;                  // distillation: the list's logits
    float* bi = bv + kLaneRows * ldt;                  // and indices (as floats' bits)
    const float c = kLog2e / a.temperature;
    double total = 0.0;
    const int64_t tiles = (a.rows + kLaneThreads - 1) / kLaneThreads;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t r0 = tile * kLaneThreads + wave * kLaneRows;
        const int64_t left = a.rows - r0;
        const int n = left < kLaneRows ? (left > 0 ? (int)left : 0) : kLaneRows;
        const uint8_t* mask = a.mask ? a.mask + r0 * a.mask_ld : nullptr;
        const int64_t row = r0 + lane;
        PolicyRow pr{};
        if (lane < n) {
            if (KIND != kDistill)
                pr = policy_row<KIND>(a, row);
            else
                pr.w = a.weight ? a.weight[row] : a.row_weight;
        }
        wave_lds_sync();
        rows_to_lds<false, KIND == kPolicyRef>((const E*)a.logits + r0 * a.logits_ld, a.logits_ld,
                                               (const E*)a.ref_logits + r0 * a.ref_ld, a.ref_ld,
                                               mask, a.mask_ld, n, A, bx, by, lane);
        if (KIND == kDistill)
            rows_to_lds<true, true>(a.val + r0 * top, top, (const float*)a.idx + r0 * top, top,
                                    nullptr, 0, n, top, bv, bi, lane);
        wave_lds_sync();
        if (lane < n) {
            float* xr = bx + lane * A;
            float* yr = by + lane * A;
            float x[NA], y[KIND == kPolicy ? 1 : NA];
            float m = kNegInf, my = kNegInf;
#pragma unroll
            for (int j = 0; j < NA; ++j) {
                x[j] = kNegInf;
                if (KIND == kPolicyRef)
                    y[j] = kNegInf;
            }
            row_read(xr, A, x);
            if constexpr (KIND == kPolicyRef)
                row_read(yr, A, y);
            // (four entries per uniform branch)
#pragma unroll
            for (int q = 0; q < NA; q += 4) {
                if (q >= A)
                    break;
#pragma unroll
                for (int j = q; j < q + 4; ++j) {
                    m = fmaxf(m, x[j]);
                    if (KIND == kPolicyRef)
                        my = fmaxf(my, y[j]);
                }
            }
            Stats st = empty_stats();
            st.m = m;
            st.my = my;
            m = m == kNegInf ? 0.0f : m;
            my = my == kNegInf ? 0.0f : my;
#pragma unroll
            for (int q = 0; q < NA; q += 4) {
                if (q >= A)
                    break;
#pragma unroll
                for (int j = q; j < q + 4; ++j)
                    add_entry<KIND>(st, x[j], KIND == kPolicyRef ? y[j] : 0.0f, m, my, c);
            }
            RowGrad g{};
            bool counts;
            float ts = 0.0f;   // distillation: sum of the teacher's exponentials
            if (KIND != kDistill) {
                counts = pr.counts && st.s != 0.0f;
                PolicyOut o{0.0f, 0.0f, 0.0f, 0.0f};
                if (counts) {
                    o = policy_finish<KIND>(a, pr, st, xr[pr.action], g);
                    total += (double)pr.w * o.loss;
                }
                store_policy(a, row, o);
            } else {
                const float T = a.temperature;
                const float* v = bv + lane * ldt;
                float* ix = bi + lane * ldt;
                float tm = kNegInf;
#pragma unroll
                for (int j = 0; j < NA; ++j)
                    y[j] = 0.0f;
                row_write(yr, A, y);
                // an entry counts if its index is a legal entry (-inf logits that are legal
                // count: the loss is then infinite); the others' index becomes -1
#pragma unroll 4
                for (int k = 0; k < top; ++k) {
                    const int i = (int)__float_as_uint(ix[k]);
                    if (i < 0 || i >= A || (mask && mask[lane * a.mask_ld + i] == 0))
                        ix[k] = __uint_as_float(0xFFFFFFFFu);
                    else
                        tm = fmaxf(tm, v[k]);
                }
                tm = tm == kNegInf ? 0.0f : tm;
                float own = 0.0f, ce = 0.0f;   // sums of e b and e (x - m) over the list
                for (int k = 0; k < top; ++k) {
                    const int i = (int)__float_as_uint(ix[k]);
                    if (i < 0)
                        continue;
                    const float b = v[k] - tm, e = exp2_hw(b * c);
                    ts += e;
                    yr[i] += e;
                    if (e != 0.0f) {
                        own = __builtin_fmaf(e, b, own);
                        ce = __builtin_fmaf(e, xr[i] - m, ce);
                    }
                }
                counts = pr.w != 0.0f && st.s != 0.0f && ts != 0.0f;
                float loss = 0.0f;
                if (counts) {
                    loss = T * T * ((own - ce) / (T * ts) + (logf(st.s) - logf(ts)));
                    total += (double)pr.w * loss;
                    g.m = m;
                    g.c0 = pr.w * T / st.s;
                }
                if (a.stats)
                    a.stats[row] = loss;
            }
            if (a.dlogits) {
                const float wt = KIND == kDistill && counts ? pr.w * a.temperature / ts : 0.0f;
                if constexpr (KIND == kDistill)
                    row_read(yr, A, y);
#pragma unroll
                for (int q = 0; q < NA; q += 4) {
                    if (q >= A)
                        break;
#pragma unroll
                    for (int j = q; j < q + 4; ++j) {
                        float d = grad_entry<KIND>(g, x[j], KIND == kPolicyRef ? y[j] : 0.0f, c);
                        if (KIND == kDistill)
                            d = __builtin_fmaf(-wt, y[j], d);
                        x[j] = counts ? d : 0.0f;
                    }
                }
                row_write(xr, A, x);
                if (KIND != kDistill && counts)
                    xr[pr.action] += g.at_action;
            }
        }
        wave_lds_sync();
        if (a.dlogits)
            rows_from_lds(bx, (E*)a.dlogits + r0 * a.dlogits_ld, a.dlogits_ld, n, A, lane);
    }
    if (a.total)
        store_total(a, block_sum(total));
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

// WHOLE: the chunk does not cross the row's end.
template <typename E, int KIND, bool WHOLE>
__device__ __forceinline__ void write_grad(const LossArgs& a, const RowGrad& g, bool counts,
                                           int64_t row, int q, u32x4 x, u32x4 y, float c)
{
    constexpr int CH = kChunk<E>;
    const int j0 = q * CH, n = WHOLE || a.A - j0 > CH ? CH : a.A - j0;
    if (n <= 0)
        return;
    float f[CH], r[CH];
    if (counts) {
        unpack<E>(x, f);
        if (KIND == kPolicyRef)
            unpack<E>(y, r);
#pragma unroll
        for (int e = 0; e < CH; ++e)
            f[e] = grad_entry<KIND>(g, f[e], KIND == kPolicyRef ? r[e] : 0.0f, c);
    } else {
#pragma unroll
        for (int e = 0; e < CH; ++e)
            f[e] = 0.0f;
    }
    store_chunk((E*)a.dlogits + row * a.dlogits_ld + j0, n, pack<E>(f));
}

// The action's entry, over what write_grad left there, by the thread that wrote it (a
// thread's stores to one place stay in order).
template <typename E, int KIND>
__device__ __forceinline__ void write_action(const LossArgs& a, const RowGrad& g, int64_t row,
                                             int j, float x, float y, float c)
{
    ((E*)a.dlogits)[row * a.dlogits_ld + j] = from_f32<E>(grad_entry<KIND>(g, x, y, c) + g.at_action);
}

// The teacher's list of a row, handled by TL lanes (the row's own, or its first
// wavefront): index (-1 where an entry does not count), probability and the
// student's logit of each entry, in LDS, and two bitmaps over the indices, `seen` and
// `twice`: bits that an entry, or more than one, falls on.  Rows in registers have a
// bit for each of their entries; longer ones share bits, so that a bit in `twice` says
// only that the list has to be searched.
template <int T>
struct List {
    static constexpr int kWords = T <= 64 ? T : 256;
    int* i;
    float *p, *x;
    uint32_t *seen, *twice;
    int top, padded;   // padded: top rounded up to 4

    // of row `slot` of the workgroup's `rows`
    __device__ __forceinline__ List(void* lds, int slot, int rows, int top_)
        : top(top_), padded((top_ + 3) & ~3)
    {
        i = (int*)lds + slot * padded * 3;
        p = (float*)(i + padded);
        x = p + padded;
        seen = (uint32_t*)lds + rows * padded * 3 + slot * 2 * kWords;
        twice = seen + kWords;
    }
    __device__ __forceinline__ static uint32_t word(int i)
    {
        return (uint32_t)i / 32 % (uint32_t)kWords;
    }
    __device__ __forceinline__ static uint32_t bit(int i) { return 1u << (i & 31); }
};
// of a workgroup's lists, with T threads per row
constexpr int list_bytes(int top, int T, int threads)
{
    return T <= 64 ? ((top + 3) & ~3) * 12 * (threads / T) + 8 * threads
                   : ((top + 3) & ~3) * 12 + 8 * 256;
}

// Loads the list and forms the probabilities.  Returns whether any entry counts (in
// the TL lanes): its index is a legal entry.  `part`: this lane's sum of t ln t.
template <typename E, int T>
__device__ __forceinline__ bool load_list(const LossArgs& a, const List<T>& l, int64_t row,
                                          int lane, bool live_row, float c, float& part)
{
    constexpr int TL = T < 64 ? T : 64, U = 4;
    for (int w = lane; w < List<T>::kWords; w += TL)
        l.seen[w] = l.twice[w] = 0;
    wave_lds_sync();
    const E* x = (const E*)a.logits + row * a.logits_ld;
    const uint8_t* mask = a.mask ? a.mask + row * a.mask_ld : nullptr;
    float tm = kNegInf;
    for (int k0 = lane; k0 < l.padded; k0 += U * TL) {
        int i[U];
        float v[U], f[U];
        bool in[U];
        if (live_row) {   // (entries behind the list's end read its last)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = k0 + u * TL < l.top ? k0 + u * TL : l.top - 1;
                i[u] = a.idx[row * a.top + k];
                v[u] = a.val[row * a.top + k];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                in[u] = k0 + u * TL < l.top && i[u] >= 0 && i[u] < a.A;
                const int j = in[u] ? i[u] : 0;
                f[u] = to_f32(x[j]);
                if (mask)
                    in[u] = in[u] && mask[j] != 0;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u * TL;
            if (k >= l.padded)
                break;
            const bool ok = live_row && in[u];
            l.i[k] = ok ? i[u] : -1;
            l.p[k] = ok ? v[u] : kNegInf;
            l.x[k] = ok ? f[u] : 0.0f;
            if (ok) {
                tm = fmaxf(tm, v[u]);
                const uint32_t w = l.word(i[u]), b = l.bit(i[u]);
                if (a.dlogits && (atomicOr(l.seen + w, b) & b))
                    atomicOr(l.twice + w, b);
            }
        }
    }
    tm = lanes_combine<TL>(tm, MaxOp());
    tm = tm == kNegInf ? 0.0f : tm;
    float s = 0.0f;
    for (int k = lane; k < l.padded; k += TL)
        if (l.i[k] >= 0)
            s += exp2_hw((l.p[k] - tm) * c);
    s = lanes_combine<TL>(s, SumOp());
    const float inv = 1.0f / s, ln_s = logf(s);
    part = 0.0f;
    for (int k = lane; k < l.padded; k += TL) {
        const float b = l.p[k] - tm;
        const float p = l.i[k] >= 0 ? exp2_hw(b * c) * inv : 0.0f;
        l.p[k] = p;
        if (p != 0.0f)
            part = __builtin_fmaf(p, b / a.temperature - ln_s, part);
    }
    return s != 0.0f;
}

// The row's loss in the TL lanes, from load_list's part.
template <int T>
__device__ __forceinline__ float list_loss(const LossArgs& a, const List<T>& l, int lane,
                                           float part, float m, float ln_s)
{
    constexpr int TL = T < 64 ? T : 64;
    for (int k = lane; k < l.padded; k += TL)
        if (l.p[k] != 0.0f)
            part -= l.p[k] * ((l.x[k] - m) / a.temperature - ln_s);
    return lanes_combine<TL>(part, SumOp()) * a.temperature * a.temperature;
}

// The entries' part of the gradient, over what write_grad left there: an index that
// the list holds more than once is written by its first entry with the sum of all, in
// their order.
template <typename E, int T>
__device__ __forceinline__ void write_list(const LossArgs& a, const List<T>& l, const RowGrad& g,
                                           int64_t row, int lane, float c, float w, int j_lo,
                                           int j_hi)
{
    constexpr int TL = T < 64 ? T : 64;
    E* o = (E*)a.dlogits + row * a.dlogits_ld;
    for (int k = lane; k < l.top; k += TL) {
        const int i = l.i[k];
        if (i < j_lo || i >= j_hi)
            continue;
        float p = l.p[k];
        if (l.twice[l.word(i)] & l.bit(i)) {
            bool first = true;
            for (int q = 0; q < l.top; ++q) {
                if (q == k || l.i[q] != i)
                    continue;
                first = first && q > k;
                p += l.p[q];
            }
            if (!first)
                continue;
        }
        o[i] = from_f32<E>(grad_entry<kDistill>(g, l.x[k], 0.0f, c) - w * a.temperature * p);
    }
}

// A row's chunks into registers, -inf in the entries that are not legal or not there,
// and everywhere in a row that does not count.  Within a wavefront (T <= 64) every
// chunk has its own conditions, so that all are asked for together; in workgroups the
// chunks that all threads hold whole take none, and the one round that the row's end
// falls into comes first, which leaves registers for more wavefronts (fp32, 2048 x
// 32000 with reference logits: 173 us, with conditions on every chunk 290 us, with that
// round last 196 us; 559269 x 91: 120, as workgroups' rows 139 us).
template <typename E, int KIND, int T, int C>
__device__ __forceinline__ void load_row(const LossArgs& a, bool counts, const E* px, const E* py,
                                         const uint8_t* pm, int lane, u32x4 (&x)[C], u32x4* y)
{
    constexpr int CH = kChunk<E>;
    if constexpr (T <= 64) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = (lane + i * T) * CH, n = counts ? a.A - j : 0;
            x[i] = load_masked(px + j, n, pm ? pm + j : nullptr, j);
            if (KIND == kPolicyRef)
                y[i] = load_masked(py + j, n, pm ? pm + j : nullptr, j);
        }
        return;
    }
    const int whole = a.A / (T * CH);
    const int jt = (lane + whole * T) * CH, nt = counts ? a.A - jt : 0;
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

// Rows that fit the registers of T threads, C chunks each: read once, written once.
// Bound by memory: 16384 x 8192 bf16 123 us, 4.4 TB/s; 4096 x 65536 bf16 with reference
// logits 389 us, 4.1 TB/s; 2048 x 32000 fp32 distilled 123 us, 4.3 TB/s.
template <typename E, int KIND, int T, int C>
__global__ __launch_bounds__(T <= 64 ? 1024 : T) void loss_row_kernel(LossArgs a)
{
    const int ROWS = T <= 64 ? (int)blockDim.x / T : 1;
    constexpr int CH = kChunk<E>;
    extern __shared__ float lds[];
    __shared__ float scratch[T > 64 ? 2 * kScratch : 1];
    const int lane = threadIdx.x % T, slot = threadIdx.x / T;
    constexpr int TL = T < 64 ? T : 64;
    const List<T> list(lds, slot, ROWS, KIND == kDistill ? a.top : 0);
    __shared__ int any_entry;
    const bool lists = KIND == kDistill && lane < TL;
    const float c = kLog2e / a.temperature;
    double total = 0.0;
    const int64_t tiles = (a.rows + ROWS - 1) / ROWS;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t row = tile * ROWS + slot;
        const bool live = row < a.rows;
        PolicyRow pr{};
        if (live) {
            if (KIND != kDistill) {
                pr = policy_row<KIND>(a, row);
            } else {
                pr.w = a.weight ? a.weight[row] : a.row_weight;
                pr.counts = pr.w != 0.0f;
            }
        }
        bool counts = pr.counts;
        const E* px = (const E*)a.logits + row * a.logits_ld;
        const E* py = (const E*)a.ref_logits + row * a.ref_ld;
        const uint8_t* pm = a.mask ? a.mask + row * a.mask_ld : nullptr;
        u32x4 x[C], y[KIND == kPolicyRef ? C : 1];
        load_row<E, KIND, T, C>(a, counts, px, py, pm, lane, x, y);
        const int used = (a.A + T * CH - 1) / (T * CH);   // chunks that any thread holds
        float part = 0.0f;
        if (lists) {
            // (the group's other wavefronts learn from LDS whether the list counts: written
            // before the barriers of the merge, read between them)
            wave_lds_sync();
            const bool any = load_list<E>(a, list, row, lane, counts, c, part);
            if (T > 64) {
                if (lane == 0)
                    any_entry = any;
            } else {
                counts = counts && any;
            }
            wave_lds_sync();
        }
        Stats st = group_merge<T, KIND>(chunk_stats<E, KIND, C>(x, y, used, c), c, scratch,
                                        KIND == kDistill && T > 64 ? &any_entry : nullptr, counts);
        counts = counts && st.s != 0.0f;
        RowGrad g{};
        float x_a = 0.0f, y_a = 0.0f;   // the action's logits
        if (KIND != kDistill) {
            PolicyOut o{0.0f, 0.0f, 0.0f, 0.0f};
            if (counts) {
                x_a = to_f32(px[pr.action]);
                if (KIND == kPolicyRef)
                    y_a = to_f32(py[pr.action]);
                o = policy_finish<KIND>(a, pr, st, x_a, g);
            }
            if (live && lane == 0) {
                if (counts)
                    total += (double)pr.w * o.loss;
                store_policy(a, row, o);
            }
        } else {
            g.m = st.m == kNegInf ? 0.0f : st.m;
            g.c0 = pr.w * a.temperature / st.s;
            float loss = 0.0f;
            if (lists)
                loss = list_loss(a, list, lane, part, g.m, logf(st.s));
            if (live && lane == 0) {
                if (counts)
                    total += (double)pr.w * loss;
                if (a.stats)
                    a.stats[row] = counts ? loss : 0.0f;
            }
        }
        if (a.dlogits && live) {
            keep_raw<KIND>(x, y);
            if constexpr (T <= 64) {
#pragma unroll
                for (int i = 0; i < C; ++i)
                    write_grad<E, KIND, false>(a, g, counts, row, lane + i * T, x[i],
                                               KIND == kPolicyRef ? y[i] : x[i], c);
            } else {
                const int whole = a.A / (T * CH);
                u32x4 tx = x[0], ty = KIND == kPolicyRef ? y[0] : x[0];
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    if (i < whole)
                        write_grad<E, KIND, true>(a, g, counts, row, lane + i * T, x[i],
                                                  KIND == kPolicyRef ? y[i] : x[i], c);
                    tx = i == whole ? x[i] : tx;
                    if (KIND == kPolicyRef)
                        ty = i == whole ? y[i] : ty;
                    __builtin_amdgcn_sched_barrier(0);
                }
                write_grad<E, KIND, false>(a, g, counts, row, lane + whole * T, tx, ty, c);
            }
            if (KIND != kDistill && counts && (int)pr.action / CH % T == lane)
                write_action<E, KIND>(a, g, row, (int)pr.action, x_a, y_a, c);
        }
        if (KIND == kDistill && a.dlogits) {
            group_sync<T>();
            if (counts && lists)
                write_list<E>(a, list, g, row, lane, c, pr.w, 0, a.A);
        }
    }
    if (a.total)
        store_total(a, block_sum(total));
}

// ------------------------------------------- long rows: a workgroup per part of a row

// PHASE 0: a workgroup takes a row whole, once for its sums and once for its
// gradient (the second time from the caches).  PHASE 1: the sums of one of
// `splits` parts of a row, into a.part; PHASE 2: the parts merged (by every workgroup
// alike) and the gradient of one part.
// 3 x 131071 bf16 in parts 13.5 us: three dependent launches.
constexpr int kLongThreads = 512, kLongUnroll = 4;

template <typename E, int KIND, int PHASE>
__global__ __launch_bounds__(kLongThreads) void loss_long_kernel(LossArgs a)
{
    constexpr int T = kLongThreads, U = kLongUnroll, CH = kChunk<E>;
    extern __shared__ float lds[];
    __shared__ float scratch[2 * kScratch];
    const int tid = threadIdx.x;
    const List<T> list(lds, 0, 1, KIND == kDistill ? a.top : 0);
    __shared__ int any_entry;
    const bool lists = KIND == kDistill && tid < 64;
    const float c = kLog2e / a.temperature;
    double total = 0.0;
    const int64_t items = PHASE == 0 ? a.rows : a.rows * a.splits;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t row = PHASE == 0 ? item : item / a.splits;
        const int part = PHASE == 0 ? 0 : (int)(item % a.splits);
        const int q0 = PHASE == 0 ? 0 : part * a.part_chunks;
        const int chunks = (a.A + CH - 1) / CH;
        const int q1 = PHASE == 0 || q0 + a.part_chunks > chunks ? chunks : q0 + a.part_chunks;
        PolicyRow pr{};
        if (KIND != kDistill) {
            pr = policy_row<KIND>(a, row);
        } else {
            pr.w = a.weight ? a.weight[row] : a.row_weight;
            pr.counts = pr.w != 0.0f;
        }
        bool counts = pr.counts;
        const E* px = (const E*)a.logits + row * a.logits_ld;
        const E* py = (const E*)a.ref_logits + row * a.ref_ld;
        const uint8_t* pm = a.mask ? a.mask + row * a.mask_ld : nullptr;
        Stats st = empty_stats();
        if (PHASE != 2) {
            if (counts) {
                for (int q = q0 + tid; q < q1; q += T * U) {
                    u32x4 x[U], y[KIND == kPolicyRef ? U : 1];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int j = (q + u * T) * CH;
                        const int n = q + u * T < q1 ? a.A - j : 0;
                        x[u] = load_masked(px + j, n, pm ? pm + j : nullptr, j);
                        if (KIND == kPolicyRef)
                            y[u] = load_masked(py + j, n, pm ? pm + j : nullptr, j);
                    }
                    st = merge<KIND>(st, chunk_stats<E, KIND, U>(x, y, U, c), c);
                }
            }
            st = group_merge<T, KIND>(st, c, scratch, nullptr, counts);
            if (PHASE == 1) {
                if (tid == 0)
                    ((Stats*)a.part)[row * a.splits + part] = st;
                continue;
            }
        } else {
            // (each thread takes every T-th part, then as within a row)
            for (int i = tid; i < a.splits; i += T)
                st = merge<KIND>(st, ((const Stats*)a.part)[row * a.splits + i], c);
            st = group_merge<T, KIND>(st, c, scratch, nullptr, counts);
        }
        float from_list = 0.0f;
        if (KIND == kDistill) {
            __syncthreads();   // (the last row's flag has been read)
            if (lists) {
                const bool any = load_list<E>(a, list, row, tid, counts, c, from_list);
                if (tid == 0)
                    any_entry = any;
                wave_lds_sync();
            }
            __syncthreads();
            counts = counts && any_entry != 0;
        }
        counts = counts && st.s != 0.0f;
        RowGrad g{};
        float x_a = 0.0f, y_a = 0.0f;   // the action's logits
        if (KIND != kDistill) {
            PolicyOut o{0.0f, 0.0f, 0.0f, 0.0f};
            if (counts) {
                x_a = to_f32(px[pr.action]);
                if (KIND == kPolicyRef)
                    y_a = to_f32(py[pr.action]);
                o = policy_finish<KIND>(a, pr, st, x_a, g);
            }
            if (tid == 0 && part == 0) {
                if (counts)
                    total += (double)pr.w * o.loss;
                store_policy(a, row, o);
            }
        } else {
            g.m = st.m == kNegInf ? 0.0f : st.m;
            g.c0 = pr.w * a.temperature / st.s;
            float loss = 0.0f;
            if (lists)
                loss = list_loss(a, list, tid, from_list, g.m, logf(st.s));
            if (tid == 0 && part == 0) {
                if (counts)
                    total += (double)pr.w * loss;
                if (a.stats)
                    a.stats[row] = counts ? loss : 0.0f;
            }
        }
        if (a.dlogits) {
            for (int q = q0 + tid; q < q1; q += T * U) {
                u32x4 x[U], y[KIND == kPolicyRef ? U : 1];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int j = (q + u * T) * CH;
                    const int n = counts && q + u * T < q1 ? a.A - j : 0;
                    x[u] = load_masked(px + j, n, pm ? pm + j : nullptr, j);
                    if (KIND == kPolicyRef)
                        y[u] = load_masked(py + j, n, pm ? pm + j : nullptr, j);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (q + u * T < q1)
                        write_grad<E, KIND, false>(a, g, counts, row, q + u * T, x[u],
                                                   KIND == kPolicyRef ? y[u] : x[u], c);
            }
            if (KIND != kDistill && counts) {
                const int q = (int)pr.action / CH;
                if (q >= q0 && q < q1 && (q - q0) % T == tid)
                    write_action<E, KIND>(a, g, row, (int)pr.action, x_a, y_a, c);
            }
            if (KIND == kDistill) {
                __syncthreads();
                if (counts && lists)
                    write_list<E>(a, list, g, row, tid, c, pr.w, q0 * CH, q1 * CH);
            }
        }
    }
    if (PHASE != 1 && a.total)
        store_total(a, block_sum(total));
}

__global__ __launch_bounds__(256) void loss_total_kernel(const double* part, int64_t n, float* total)
{
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 256)
        v += part[i];
    v = block_sum(v);
    if (threadIdx.x == 0)
        *total = (float)v;
}

template <typename E, int KIND>
hipError_t launch_kind(const LossArgs& a, const LossPlan& p, hipStream_t s)
{
    const unsigned nb = (unsigned)p.blocks, nt = (unsigned)p.threads;
    const size_t lds = p.variant == kLossLane
                           ? (size_t)kLaneThreads * 4 * lane_floats(KIND, a.A, a.top)
                       : KIND == kDistill ? (size_t)list_bytes(a.top, p.group, p.threads) : 0;
    switch (p.variant) {
    case kLossLane:
        if (a.A <= 8)
            loss_lane_kernel<E, KIND, 8><<<nb, nt, lds, s>>>(a);
        else if (a.A <= 16)
            loss_lane_kernel<E, KIND, 16><<<nb, nt, lds, s>>>(a);
        else if (a.A <= 24)
            loss_lane_kernel<E, KIND, 24><<<nb, nt, lds, s>>>(a);
        else
            loss_lane_kernel<E, KIND, 32><<<nb, nt, lds, s>>>(a);
        break;
    case kLossRow:
        switch (p.group) {
        case 4:
            loss_row_kernel<E, KIND, 4, 4><<<nb, nt, lds, s>>>(a);
            break;
        case 8:
            loss_row_kernel<E, KIND, 8, 4><<<nb, nt, lds, s>>>(a);
            break;
        case 16:
            loss_row_kernel<E, KIND, 16, 4><<<nb, nt, lds, s>>>(a);
            break;
        case 32:
            loss_row_kernel<E, KIND, 32, 4><<<nb, nt, lds, s>>>(a);
            break;
        case 64:
            loss_row_kernel<E, KIND, 64, 4><<<nb, nt, lds, s>>>(a);
            break;
        case 128:
            loss_row_kernel<E, KIND, 128, 4><<<nb, nt, lds, s>>>(a);
            break;
        case 256:
            loss_row_kernel<E, KIND, 256, 4><<<nb, nt, lds, s>>>(a);
            break;
        case 512:
            loss_row_kernel<E, KIND, 512, 4><<<nb, nt, lds, s>>>(a);
            break;
        case 1024:
            loss_row_kernel<E, KIND, 1024, 4><<<nb, nt, lds, s>>>(a);
            break;
        default:
            loss_row_kernel<E, KIND, 1024, 8><<<nb, nt, lds, s>>>(a);
        }
        break;
    case kLossLong:
        loss_long_kernel<E, KIND, 0><<<nb, nt, lds, s>>>(a);
        break;
    default:
        loss_long_kernel<E, KIND, 1><<<nb, nt, lds, s>>>(a);
        loss_long_kernel<E, KIND, 2><<<nb, nt, lds, s>>>(a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.total || p.blocks == 1)
        return e;
    loss_total_kernel<<<1, 256, 0, s>>>(a.part_total, p.blocks, a.total);
    return hipGetLastError();
}

__global__ void zero_total_kernel(float* total) { *total = 0.0f; }

}  // namespace

// Up to 31 actions a lane per row (in fp32 with reference logits, against 4 or more
// threads per row: 10^6 x 8 29 and 62 us, x 24 72 and 88, x 31 118 and 135; 100000 x 31
// 19.6 and 19.0; 2000 x 8 12.2 and 11.6, x 31 14.1 and 12.1); up to 8 chunks of 16 bytes for each of 1024 threads
// (65536 bf16 or 32768 fp32 entries) a row stays in the registers of as few threads as
// hold it; above, and where a workgroup per row would leave half of the CUs idle, rows
// are read twice, in parts where there are few.  Rows in registers against rows read
// twice: 4096 x 65536 bf16 with reference logits 394 and 411 us, 2048 x 32000 fp32 with
// them 172 and 227 us, 2047 x 50001 bf16 distilled 122 and 129 us, 4096 x 50000 bf16 207
// and 205 us.  128 threads against 256: 20888 x 3602 bf16 89 and 118 us.
LossPlan loss_plan(int64_t rows, int64_t A, int top, int size)
{
    constexpr int64_t kCus = 256;
    LossPlan p{};
    const int64_t ch = 16 / size;
    p.splits = 1;
    int64_t per = 1;   // rows per workgroup
    int64_t most = 2048;
    // (the rows of a workgroup fit 64 KB of LDS)
    if (A <= kLaneMost && (top == 0 || (top <= 32 && lane_floats(kDistill, (int)A, top) <= 64))) {
        p.variant = kLossLane;
        per = p.threads = kLaneThreads;
    } else if (A <= 256 * 4 * ch || (A <= 1024 * 8 * ch && rows >= kCus / 2)) {
        p.variant = kLossRow;
        p.group = 4;
        // at most 8 entries of a teacher's list per lane
        while (p.group * 4 * ch < A || (p.group < 64 && p.group * 8 < top))
            p.group *= 2;
        // rows that 1024 threads hold at once are one workgroup's, which leaves no totals
        // of others to add in a launch of its own: 10 x 266 fp32 distilled 7.7 us, in
        // workgroups of 256 threads 11.4 us.  (Two rounds: 128 x 281 bf16 14.8 and 11.5 us.)
        p.threads = p.group <= 64 ? 256 : std::min(p.group, 1024);
        if (p.group <= 64 && rows > 0 && rows * p.group <= 1024) {
            const int one = (int)((rows * p.group + 63) / 64 * 64);
            if (list_bytes(top, p.group, one) <= 65536)
                p.threads = one;
        }
        per = std::max(1, p.threads / p.group);
        if (p.threads == 128)
            most = 4096;
    } else {
        p.variant = kLossLong;
        p.threads = p.group = kLongThreads;
        const int64_t chunks = (A + ch - 1) / ch;
        if (rows < 2 * kCus) {
            // parts of at least 512 chunks (8 KB)
            const int64_t want = std::max<int64_t>(1, 2 * kCus / std::max<int64_t>(1, rows));
            p.splits = (int)std::min(want, std::max<int64_t>(1, chunks / 512));
        }
        if (p.splits > 1) {
            p.variant = kLossSplit;
            p.part_chunks = (int)((chunks + p.splits - 1) / p.splits);
            p.splits = (int)((chunks + p.part_chunks - 1) / p.part_chunks);
        }
    }
    p.blocks = std::min(most, (rows + per - 1) / per * p.splits);
    p.part_bytes = p.splits > 1 ? rows * p.splits * (int64_t)sizeof(Stats) : 0;
    p.part_bytes = (p.part_bytes + 255) / 256 * 256;
    p.work_bytes = p.part_bytes + (p.blocks > 1 ? p.blocks * 8 : 0);
    return p;
}

hipError_t launch_loss(LossArgs a, int dtype, bool distill, const LossPlan& p, void* work,
                       hipStream_t s)
{
    if (a.rows == 0) {
        if (a.total)
            zero_total_kernel<<<1, 1, 0, s>>>(a.total);
        return hipGetLastError();
    }
    a.splits = p.splits;
    a.part_chunks = p.part_chunks;
    a.part = work;
    a.part_total = (double*)((char*)work + p.part_bytes);
    const bool ref = a.ref_logits != nullptr;
    if (dtype == MALIB_DT_BF16)
        return distill ? launch_kind<bf16_t, kDistill>(a, p, s)
               : ref   ? launch_kind<bf16_t, kPolicyRef>(a, p, s)
                       : launch_kind<bf16_t, kPolicy>(a, p, s);
    return distill ? launch_kind<float, kDistill>(a, p, s)
           : ref   ? launch_kind<float, kPolicyRef>(a, p, s)
                   : launch_kind<float, kPolicy>(a, p, s);
}

}  // namespace malib
