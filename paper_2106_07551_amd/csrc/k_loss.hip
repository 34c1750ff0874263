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
        k = __builtin_fmaf(g.c2, e > 0.0f ? (y - g.my) * kLog2e : 0.0f, k);
    return e * k;
}

// A row's scalar inputs of the policy loss.
struct PolicyRow {
    int64_t action;
    float w;
    bool counts;
};

__device__ __forceinline__ PolicyRow policy_row(const LossArgs& a, int64_t row)
{
    PolicyRow r;
    r.action = a.action_bytes == 1   ? (int64_t)((const uint8_t*)a.actions)[row]
               : a.action_bytes == 4 ? (int64_t)((const int32_t*)a.actions)[row]
                                     : ((const int64_t*)a.actions)[row];
    r.w = a.weight ? a.weight[row] : a.row_weight;
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
__device__ __forceinline__ PolicyOut policy_finish(const LossArgs& a, int64_t row, float w,
                                                   const Stats& st, float x_a, RowGrad& g)
{
    PolicyOut o;
    const float m = st.m == kNegInf ? 0.0f : st.m, my = st.my == kNegInf ? 0.0f : st.my;
    const float ln_s = logf(st.s), inv = 1.0f / st.s;
    o.logp = (x_a - m) - ln_s;
    o.entropy = ln_s - kLn2 * st.t * inv;
    const float adv = a.advantage[row];
    const float ratio = expf(o.logp - a.old_logp[row]);
    const float lo = 1.0f - a.clip_low, hi = 1.0f + a.clip_high;
    const float s1 = ratio * adv, s2 = (ratio < lo ? lo : ratio > hi ? hi : ratio) * adv;
    float slope = s1 <= s2 ? -s1 : s1 != s1 ? s1 : 0.0f;   // d loss / d log p[action]
    o.loss = -(s2 < s1 ? s2 : s1);
    o.kl = 0.0f;
    float pull = 0.0f;   // of the divergence, in every logit
    if (KIND == kPolicyRef) {
        const float ln_sy = logf(st.sy);
        o.kl = kLn2 * (st.t - st.v) * inv - ln_s + ln_sy;
        pull = a.kl_coef * (ln_sy - ln_s - o.kl);
    } else if (a.ref_logp) {
        const float d = a.ref_logp[row] - o.logp;
        const float em = expm1f(d);
        o.kl = em - d;
        slope -= a.kl_coef * em;
    }
    if (a.kl_coef != 0.0f)
        o.loss += a.kl_coef * o.kl;
    if (a.entropy_coef != 0.0f)
        o.loss -= a.entropy_coef * o.entropy;
    const float k = w * inv;
    g.m = m;
    g.my = my;
    g.c0 = k * (pull + a.entropy_coef * (o.entropy - ln_s) - slope);
    g.c1 = k * kLn2 * (a.entropy_coef + (KIND == kPolicyRef ? a.kl_coef : 0.0f));
    g.c2 = KIND == kPolicyRef ? -k * kLn2 * a.kl_coef : 0.0f;
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

// Whether entry k of a row's list counts: its index (or -1).
__device__ __forceinline__ int list_index(const LossArgs& a, int64_t row, int k)
{
    const int i = a.idx[row * a.top + k];
    if (i < 0 || i >= a.A || (a.mask && a.mask[row * a.mask_ld + i] == 0))
        return -1;
    return i;
}

// Sum of one value per thread over the workgroup (in a fixed order), in thread 0.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double part[THREADS / 64];
#pragma unroll
    for (int o = 32; o; o >>= 1)
        v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = v;
    __syncthreads();
    double t = 0.0;
    if (threadIdx.x == 0)
        for (int i = 0; i < THREADS / 64; ++i)
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

// ------------------------------------------------- few actions: a lane per row

// 64 rows per wavefront: their logits go through LDS (row stride odd, so that lanes
// that read the same column of neighbouring rows fall into different banks), so
// that memory is read and written in its own order while each lane works on a row
// alone: no reductions, and a row's scalar work is not repeated by other lanes.
constexpr int kLaneThreads = 256, kLaneRows = 64;

template <typename E, int KIND>
__global__ __launch_bounds__(kLaneThreads) void loss_lane_kernel(LossArgs a)
{
    extern __shared__ float lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int A = a.A, ldw = A | 1;
    constexpr int kBufs = KIND == kPolicyRef ? 2 : 1;
    float* bx = lds + wave * kLaneRows * ldw * kBufs;
    float* by = bx + kLaneRows * ldw;
    float* xr = bx + lane * ldw;
    float* yr = by + lane * ldw;
    const float c = kLog2e / a.temperature;
    double total = 0.0;
    const int64_t tiles = (a.rows + kLaneThreads - 1) / kLaneThreads;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t r0 = tile * kLaneThreads + wave * kLaneRows;
        const int n = (int)(a.rows - r0 < kLaneRows ? a.rows - r0 : kLaneRows);   // may be <= 0
        const int count = n > 0 ? n * A : 0;
        wave_lds_sync();
        for (int i = lane; i < count; i += 64) {
            const int r = i / A, j = i - r * A;
            float x = to_f32(((const E*)a.logits)[(r0 + r) * a.logits_ld + j]);
            const bool legal = !a.mask || a.mask[(r0 + r) * a.mask_ld + j] != 0;
            bx[r * ldw + j] = legal ? x : kNegInf;
            if (KIND == kPolicyRef) {
                const float y = to_f32(((const E*)a.ref_logits)[(r0 + r) * a.ref_ld + j]);
                by[r * ldw + j] = legal ? y : kNegInf;
            }
        }
        wave_lds_sync();
        const int64_t row = r0 + lane;
        if (lane < n) {
            PolicyRow pr{};
            bool counts;
            float w;
            if (KIND == kDistill) {
                w = a.weight ? a.weight[row] : a.row_weight;
                counts = w != 0.0f;
            } else {
                pr = policy_row(a, row);
                w = pr.w;
                counts = pr.counts;
            }
            Stats st = empty_stats();
            float m = kNegInf, my = kNegInf;
            for (int j = 0; j < A; ++j) {
                m = fmaxf(m, xr[j]);
                if (KIND == kPolicyRef)
                    my = fmaxf(my, yr[j]);
            }
            st.m = m;
            st.my = my;
            m = m == kNegInf ? 0.0f : m;
            my = my == kNegInf ? 0.0f : my;
            for (int j = 0; j < A; ++j)
                add_entry<KIND>(st, xr[j], KIND == kPolicyRef ? yr[j] : 0.0f, m, my, c);
            counts = counts && st.s != 0.0f;
            RowGrad g{};
            if (KIND != kDistill) {
                PolicyOut o{0.0f, 0.0f, 0.0f, 0.0f};
                if (counts) {
                    o = policy_finish<KIND>(a, row, w, st, xr[pr.action], g);
                    total += (double)w * o.loss;
                }
                store_policy(a, row, o);
            } else {
                // the teacher's softmax over the entries that count
                const float T = a.temperature;
                float tm = kNegInf, ts = 0.0f, loss = 0.0f;
                for (int k = 0; k < a.top; ++k)
                    if (list_index(a, row, k) >= 0)
                        tm = fmaxf(tm, a.val[row * a.top + k]);
                const float tm0 = tm == kNegInf ? 0.0f : tm;
                for (int k = 0; k < a.top; ++k)
                    if (list_index(a, row, k) >= 0)
                        ts += exp2_hw((a.val[row * a.top + k] - tm0) * c);
                counts = counts && ts != 0.0f;
                if (counts) {
                    const float ln_ts = logf(ts), ln_s = logf(st.s);
                    for (int k = 0; k < a.top; ++k) {
                        const int i = list_index(a, row, k);
                        if (i < 0)
                            continue;
                        const float b = (a.val[row * a.top + k] - tm0) / T;
                        const float p = exp2_hw((a.val[row * a.top + k] - tm0) * c) / ts;
                        if (p != 0.0f)
                            loss += p * ((b - ln_ts) - ((xr[i] - m) / T - ln_s));
                    }
                    loss *= T * T;
                    total += (double)w * loss;
                    g.m = m;
                    g.c0 = w * T / st.s;
                }
                if (a.stats)
                    a.stats[row] = loss;
                if (a.dlogits) {
                    for (int j = 0; j < A; ++j)
                        xr[j] = counts ? grad_entry<KIND>(g, xr[j], 0.0f, c) : 0.0f;
                    if (counts)
                        for (int k = 0; k < a.top; ++k) {
                            const int i = list_index(a, row, k);
                            if (i >= 0)
                                xr[i] -= w * T *
                                         (exp2_hw((a.val[row * a.top + k] - tm0) * c) / ts);
                        }
                }
            }
            if (KIND != kDistill && a.dlogits) {
                for (int j = 0; j < A; ++j)
                    xr[j] = counts ? grad_entry<KIND>(g, xr[j], KIND == kPolicyRef ? yr[j] : 0.0f,
                                                      c)
                                   : 0.0f;
                if (counts)
                    xr[pr.action] += g.at_action;
            }
        }
        wave_lds_sync();
        if (a.dlogits)
            for (int i = lane; i < count; i += 64) {
                const int r = i / A, j = i - r * A;
                ((E*)a.dlogits)[(r0 + r) * a.dlogits_ld + j] = from_f32<E>(bx[r * ldw + j]);
            }
    }
    if (a.total)
        store_total(a, block_sum<kLaneThreads>(total));
}

// ------------------------------------------------------- a group of lanes per row

// T threads per row: lanes of one wavefront (T <= 64) or a workgroup.
template <int T>
__device__ __forceinline__ void group_sync()
{
    if constexpr (T <= 64)
        wave_lds_sync();
    else
        __syncthreads();
}

// Merge over the group; every thread gets the result.  `scratch`: LDS, T > 64 only.
template <int T, int KIND>
__device__ __forceinline__ Stats group_merge(Stats st, float c, float* scratch)
{
#pragma unroll
    for (int o = (T < 64 ? T : 64) / 2; o; o >>= 1) {
        Stats b;
        b.m = __shfl_xor(st.m, o);
        b.s = __shfl_xor(st.s, o);
        b.t = KIND != kDistill ? __shfl_xor(st.t, o) : 0.0f;
        if (KIND == kPolicyRef) {
            b.my = __shfl_xor(st.my, o);
            b.sy = __shfl_xor(st.sy, o);
            b.v = __shfl_xor(st.v, o);
        }
        st = merge<KIND>(st, b, c);
    }
    if constexpr (T > 64) {
        Stats* w = (Stats*)scratch;
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
            w[threadIdx.x >> 6] = st;
        __syncthreads();
        st = w[0];
#pragma unroll
        for (int i = 1; i < T / 64; ++i)
            st = merge<KIND>(st, w[i], c);
    }
    return st;
}

template <int T>
__device__ __forceinline__ float group_max(float v, float* scratch)
{
#pragma unroll
    for (int o = (T < 64 ? T : 64) / 2; o; o >>= 1)
        v = fmaxf(v, __shfl_xor(v, o));
    if constexpr (T > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
            scratch[threadIdx.x >> 6] = v;
        __syncthreads();
        v = scratch[0];
        for (int i = 1; i < T / 64; ++i)
            v = fmaxf(v, scratch[i]);
    }
    return v;
}

template <int T>
__device__ __forceinline__ float group_sum(float v, float* scratch)
{
#pragma unroll
    for (int o = (T < 64 ? T : 64) / 2; o; o >>= 1)
        v += __shfl_xor(v, o);
    if constexpr (T > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
            scratch[threadIdx.x >> 6] = v;
        __syncthreads();
        v = scratch[0];
        for (int i = 1; i < T / 64; ++i)
            v += scratch[i];
    }
    return v;
}

constexpr uint32_t kNegInfBits = 0xFF800000u;

// Raw chunk with -inf in the entries that do not exist or are not legal.
template <typename E>
__device__ __forceinline__ u32x4 load_masked(const E* p, int n, const uint8_t* mask)
{
    constexpr int CH = kChunk<E>;
    u32x4 v = n > 0 ? load_chunk(p, n) : u32x4{0, 0, 0, 0};
    uint32_t out = 0;   // bit i: entry i does not count
    if (n < CH)
        out = n > 0 ? (0xFFu << n) & 0xFFu : 0xFFu;
    if (mask && n > 0) {
        if (n >= CH) {
            typedef uint32_t u32_any __attribute__((aligned(1)));
            uint32_t b[CH / 4];
#pragma unroll
            for (int i = 0; i < CH / 4; ++i)
                b[i] = ((const u32_any*)mask)[i];
#pragma unroll
            for (int i = 0; i < CH; ++i)
                out |= ((b[i / 4] >> (8 * (i % 4))) & 0xFFu) == 0 ? 1u << i : 0u;
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i)
                if (i < n)
                    out |= mask[i] == 0 ? 1u << i : 0u;
        }
    }
    if (out) {
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if ((out >> i) & 1u) {
                if constexpr (sizeof(E) == 4)
                    v[i] = kNegInfBits;
                else
                    v[i >> 1] = (i & 1) ? (v[i >> 1] & 0xFFFFu) | kNegInfBits
                                        : (v[i >> 1] & 0xFFFF0000u) | (kNegInfBits >> 16);
            }
    }
    return v;
}

// The sums over C chunks that a thread holds.
template <typename E, int KIND, int C>
__device__ __forceinline__ Stats chunk_stats(const u32x4 (&x)[C], const u32x4* y, float c)
{
    constexpr int CH = kChunk<E>;
    Stats st = empty_stats();
#pragma unroll
    for (int i = 0; i < C; ++i) {
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
#pragma unroll
    for (int i = 0; i < C; ++i) {
        float f[CH], r[CH];
        unpack<E>(x[i], f);
        if (KIND == kPolicyRef)
            unpack<E>(y[i], r);
#pragma unroll
        for (int e = 0; e < CH; ++e)
            add_entry<KIND>(st, f[e], KIND == kPolicyRef ? r[e] : 0.0f, m, my, c);
    }
    return st;
}

template <typename E, int KIND>
__device__ __forceinline__ void write_grad(const LossArgs& a, const RowGrad& g, bool counts,
                                           int64_t row, int64_t action, int q, u32x4 x, u32x4 y,
                                           float c)
{
    constexpr int CH = kChunk<E>;
    const int j0 = q * CH, n = a.A - j0 < CH ? a.A - j0 : CH;
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
        if (KIND != kDistill && action >= j0 && action < j0 + CH) {
#pragma unroll
            for (int e = 0; e < CH; ++e)
                if (action == j0 + e)
                    f[e] += g.at_action;
        }
    } else {
#pragma unroll
        for (int e = 0; e < CH; ++e)
            f[e] = 0.0f;
    }
    store_chunk((E*)a.dlogits + row * a.dlogits_ld + j0, n, pack<E>(f));
}

// The teacher's list of a row: softmax over the entries that count into LDS (index
// and probability; probability 0 and index -1 elsewhere).  Returns whether any
// entry counts.
template <int T>
__device__ __forceinline__ bool load_list(const LossArgs& a, int64_t row, int lane, bool live_row,
                                          int* li, float* lp, float* scratch, float c,
                                          float& tm0, float& ts)
{
    float tm = kNegInf;
    for (int k = lane; k < a.top; k += T) {
        const int i = live_row ? list_index(a, row, k) : -1;
        const float v = live_row ? a.val[row * a.top + k] : 0.0f;
        li[k] = i;
        lp[k] = v;
        if (i >= 0)
            tm = fmaxf(tm, v);
    }
    tm = group_max<T>(tm, scratch);
    tm0 = tm == kNegInf ? 0.0f : tm;
    float s = 0.0f;
    for (int k = lane; k < a.top; k += T)
        if (li[k] >= 0)
            s += exp2_hw((lp[k] - tm0) * c);
    ts = group_sum<T>(s, scratch);
    return ts != 0.0f;
}

// This lane's share of the list's part of the loss (before the factor T^2): sum of
// t (ln t - ln q) over entries with t > 0.
template <typename E, int T>
__device__ __forceinline__ float list_loss(const LossArgs& a, int64_t row, int lane,
                                           const int* li, const float* lp, float c, float tm0,
                                           float ts, float m, float ln_s)
{
    const E* x = (const E*)a.logits + row * a.logits_ld;
    const float ln_ts = logf(ts);
    float loss = 0.0f;
    for (int k = lane; k < a.top; k += T) {
        const int i = li[k];
        if (i < 0)
            continue;
        const float b = lp[k] - tm0;
        const float p = exp2_hw(b * c) / ts;
        if (p != 0.0f)
            loss += p * ((b / a.temperature - ln_ts) - ((to_f32(x[i]) - m) / a.temperature - ln_s));
    }
    return loss;
}

// The entries' part of the gradient, over what write_grad left there: an index that
// the list holds more than once is written by its first entry with the sum of all.
template <typename E, int T>
__device__ __forceinline__ void write_list(const LossArgs& a, const RowGrad& g, int64_t row,
                                           int lane, const int* li, const float* lp, float c,
                                           float tm0, float ts, float w, int j_lo, int j_hi)
{
    const E* x = (const E*)a.logits + row * a.logits_ld;
    E* o = (E*)a.dlogits + row * a.dlogits_ld;
    for (int k = lane; k < a.top; k += T) {
        const int i = li[k];
        if (i < j_lo || i >= j_hi)
            continue;
        bool first = true;
        float p = 0.0f;
        for (int q = 0; q < a.top; ++q)
            if (li[q] == i) {
                first = first && q >= k;
                p += exp2_hw((lp[q] - tm0) * c) / ts;
            }
        if (first)
            o[i] = from_f32<E>(grad_entry<kDistill>(g, to_f32(x[i]), 0.0f, c) -
                               w * a.temperature * p);
    }
}

// Rows that fit the registers of T threads, C chunks each: read once, written once.
template <typename E, int KIND, int T, int C>
__global__ __launch_bounds__(T < 256 ? 256 : T) void loss_row_kernel(LossArgs a)
{
    constexpr int THREADS = T < 256 ? 256 : T, ROWS = THREADS / T;
    constexpr int CH = kChunk<E>;
    extern __shared__ float lds[];
    __shared__ Stats scratch[T > 64 ? T / 64 : 1];
    const int lane = threadIdx.x % T, slot = threadIdx.x / T;
    int* li = (int*)lds + slot * a.top * 2;
    float* lp = (float*)(li + a.top);
    const float c = kLog2e / a.temperature;
    double total = 0.0;
    const int64_t tiles = (a.rows + ROWS - 1) / ROWS;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t row = tile * ROWS + slot;
        const bool live = row < a.rows;
        PolicyRow pr{0, 0.0f, false};
        if (live) {
            if (KIND != kDistill) {
                pr = policy_row(a, row);
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
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int j = (lane + i * T) * CH;
            const int n = counts ? a.A - j : 0;
            x[i] = load_masked(px + j, n, pm ? pm + j : nullptr);
            if (KIND == kPolicyRef)
                y[i] = load_masked(py + j, n, pm ? pm + j : nullptr);
        }
        float tm0 = 0.0f, ts = 1.0f;
        if (KIND == kDistill) {
            group_sync<T>();
            const bool any = load_list<T>(a, row, lane, counts, li, lp, (float*)scratch, c, tm0, ts);
            counts = counts && any;
        }
        Stats st = group_merge<T, KIND>(chunk_stats<E, KIND, C>(x, y, c), c, (float*)scratch);
        counts = counts && st.s != 0.0f;
        RowGrad g{};
        if (KIND != kDistill) {
            PolicyOut o{0.0f, 0.0f, 0.0f, 0.0f};
            if (counts)
                o = policy_finish<KIND>(a, row, pr.w, st, to_f32(px[pr.action]), g);
            if (live && lane == 0) {
                if (counts)
                    total += (double)pr.w * o.loss;
                store_policy(a, row, o);
            }
        } else {
            float loss = 0.0f;
            const float m = st.m == kNegInf ? 0.0f : st.m;
            group_sync<T>();   // the list is whole
            if (counts)
                loss = list_loss<E, T>(a, row, lane, li, lp, c, tm0, ts, m, logf(st.s));
            loss = group_sum<T>(loss, (float*)scratch) * a.temperature * a.temperature;
            g.m = m;
            g.c0 = pr.w * a.temperature / st.s;
            if (live && lane == 0) {
                if (counts)
                    total += (double)pr.w * loss;
                if (a.stats)
                    a.stats[row] = counts ? loss : 0.0f;
            }
        }
        if (a.dlogits && live) {
#pragma unroll
            for (int i = 0; i < C; ++i)
                write_grad<E, KIND>(a, g, counts, row, pr.action, lane + i * T, x[i],
                                    KIND == kPolicyRef ? y[i] : x[i], c);
        }
        if (KIND == kDistill && a.dlogits) {
            group_sync<T>();
            if (counts)
                write_list<E, T>(a, g, row, lane, li, lp, c, tm0, ts, pr.w, 0, a.A);
        }
    }
    if (a.total)
        store_total(a, block_sum<THREADS>(total));
}

// ------------------------------------------- long rows: a workgroup per part of a row

// PHASE 0: a workgroup takes a row whole, once for its sums and once for its
// gradient (the second time from the caches).  PHASE 1: the sums of one of
// `splits` parts of a row, into a.part; PHASE 2: the parts merged (in order, by every
// workgroup alike) and the gradient of one part.
constexpr int kLongThreads = 512, kLongUnroll = 4;

template <typename E, int KIND, int PHASE>
__global__ __launch_bounds__(kLongThreads) void loss_long_kernel(LossArgs a)
{
    constexpr int T = kLongThreads, U = kLongUnroll, CH = kChunk<E>;
    extern __shared__ float lds[];
    __shared__ Stats scratch[T / 64];
    const int tid = threadIdx.x;
    int* li = (int*)lds;
    float* lp = (float*)(li + a.top);
    const float c = kLog2e / a.temperature;
    double total = 0.0;
    const int64_t items = PHASE == 0 ? a.rows : a.rows * a.splits;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t row = PHASE == 0 ? item : item / a.splits;
        const int part = PHASE == 0 ? 0 : (int)(item % a.splits);
        const int q0 = PHASE == 0 ? 0 : part * a.part_chunks;
        const int chunks = (a.A + CH - 1) / CH;
        const int q1 = PHASE == 0 || q0 + a.part_chunks > chunks ? chunks : q0 + a.part_chunks;
        PolicyRow pr{0, 0.0f, false};
        if (KIND != kDistill) {
            pr = policy_row(a, row);
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
                        x[u] = load_masked(px + j, n, pm ? pm + j : nullptr);
                        if (KIND == kPolicyRef)
                            y[u] = load_masked(py + j, n, pm ? pm + j : nullptr);
                    }
                    st = merge<KIND>(st, chunk_stats<E, KIND, U>(x, y, c), c);
                }
            }
            st = group_merge<T, KIND>(st, c, (float*)scratch);
            if (PHASE == 1) {
                if (tid == 0)
                    ((Stats*)a.part)[row * a.splits + part] = st;
                continue;
            }
        } else {
            for (int i = 0; i < a.splits; ++i)
                st = merge<KIND>(st, ((const Stats*)a.part)[row * a.splits + i], c);
        }
        float tm0 = 0.0f, ts = 1.0f;
        if (KIND == kDistill) {
            __syncthreads();
            const bool any = load_list<T>(a, row, tid, counts, li, lp, (float*)scratch, c, tm0, ts);
            counts = counts && any;
        }
        counts = counts && st.s != 0.0f;
        RowGrad g{};
        if (KIND != kDistill) {
            PolicyOut o{0.0f, 0.0f, 0.0f, 0.0f};
            if (counts)
                o = policy_finish<KIND>(a, row, pr.w, st, to_f32(px[pr.action]), g);
            if (tid == 0 && part == 0) {
                if (counts)
                    total += (double)pr.w * o.loss;
                store_policy(a, row, o);
            }
        } else {
            float loss = 0.0f;
            const float m = st.m == kNegInf ? 0.0f : st.m;
            __syncthreads();
            if (counts)
                loss = list_loss<E, T>(a, row, tid, li, lp, c, tm0, ts, m, logf(st.s));
            loss = group_sum<T>(loss, (float*)scratch) * a.temperature * a.temperature;
            g.m = m;
            g.c0 = pr.w * a.temperature / st.s;
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
                    x[u] = load_masked(px + j, n, pm ? pm + j : nullptr);
                    if (KIND == kPolicyRef)
                        y[u] = load_masked(py + j, n, pm ? pm + j : nullptr);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (q + u * T < q1)
                        write_grad<E, KIND>(a, g, counts, row, pr.action, q + u * T, x[u],
                                            KIND == kPolicyRef ? y[u] : x[u], c);
            }
            if (KIND == kDistill) {
                __syncthreads();
                if (counts)
                    write_list<E, T>(a, g, row, tid, li, lp, c, tm0, ts, pr.w, q0 * CH, q1 * CH);
            }
        }
    }
    if (PHASE != 1 && a.total)
        store_total(a, block_sum<T>(total));
}

__global__ __launch_bounds__(256) void loss_total_kernel(const double* part, int64_t n, float* total)
{
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 256)
        v += part[i];
    v = block_sum<256>(v);
    if (threadIdx.x == 0)
        *total = (float)v;
}

template <typename E, int KIND>
hipError_t launch_kind(const LossArgs& a, const LossPlan& p, hipStream_t s)
{
    const size_t list = KIND == kDistill ? (size_t)a.top * 8 : 0;
    const unsigned nb = (unsigned)p.blocks;
    switch (p.variant) {
    case kLossLane: {
        const size_t lds = (size_t)kLaneThreads * (a.A | 1) * 4 * (KIND == kPolicyRef ? 2 : 1);
        loss_lane_kernel<E, KIND><<<nb, kLaneThreads, lds, s>>>(a);
        break;
    }
    case kLossRow16:
        loss_row_kernel<E, KIND, 16, 2><<<nb, 256, list * 16, s>>>(a);
        break;
    case kLossRow64:
        loss_row_kernel<E, KIND, 64, 4><<<nb, 256, list * 4, s>>>(a);
        break;
    case kLossRow256:
        loss_row_kernel<E, KIND, 256, 4><<<nb, 256, list, s>>>(a);
        break;
    case kLossRow1024:
        loss_row_kernel<E, KIND, 1024, 4><<<nb, 1024, list, s>>>(a);
        break;
    case kLossLong:
        loss_long_kernel<E, KIND, 0><<<nb, kLongThreads, list, s>>>(a);
        break;
    default:
        loss_long_kernel<E, KIND, 1><<<nb, kLongThreads, list, s>>>(a);
        loss_long_kernel<E, KIND, 2><<<nb, kLongThreads, list, s>>>(a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.total || p.blocks == 1)
        return e;
    loss_total_kernel<<<1, 256, 0, s>>>(a.part_total, p.blocks, a.total);
    return hipGetLastError();
}

__global__ void zero_total_kernel(float* total) { *total = 0.0f; }

}  // namespace

LossPlan loss_plan(int64_t rows, int64_t A, int size)
{
    constexpr int64_t kCus = 256;
    LossPlan p{};
    const int64_t ch = 16 / size;
    p.splits = 1;
    int64_t per = 1;   // rows per workgroup
    int64_t most = 2048;
    if (A < 32) {   // two buffers of 256 rows of 31 fit 64 KB of LDS
        p.variant = kLossLane;
        per = kLaneThreads;
    } else if (A <= 16 * 2 * ch) {
        p.variant = kLossRow16;
        per = 16;
    } else if (A <= 64 * 4 * ch) {
        p.variant = kLossRow64;
        per = 4;
    } else if (A <= 256 * 4 * ch) {
        p.variant = kLossRow256;
    } else if (A <= 1024 * 4 * ch && rows >= kCus / 2) {
        p.variant = kLossRow1024;
    } else {
        p.variant = kLossLong;
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
