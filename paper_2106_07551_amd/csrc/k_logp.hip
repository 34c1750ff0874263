// Log probabilities of given actions, the entropy and the top alternatives of rows of
// logits, and the gradient of the first two.
//
// With x a row's legal logits, c = log2(e) / T and m = max x: s = sum_j 2^((x_j - m) c),
// t = sum_j 2^((x_j - m) c) (x_j - m) c, and
//   l = (x_a - m) / T - ln s (as a product with 2 / T),  H = ln s - ln2 t / s,
//   dx_j = 2^((x_j - m) c) (c0 + c1 (x_j - m) c) + dl [j = a] / T.
// Lists: rows of up to kShortMost entries stay in the registers of a few lanes, which
// find one place after the other, or, for longer lists, in LDS, where a wavefront finds the value
// of the last place bit by bit.  Longer rows stream through a wavefront or a workgroup, whose
// sums need the largest entry of every chunk of 16 bytes anyway: chunks with an entry that
// can still be listed (one per hundreds) go to LDS, and the bound for that rises as the
// row goes by.
#include "rows.hpp"

namespace malib {

namespace {

// ---------------------------------------------------------------- order of entries

// The order of a list as whole numbers: the value's (NaN above everything, -0 as 0) in the
// high half, the index reversed in the low one.  Entries up to kUnlisted are not listed.
constexpr uint32_t kUnlisted = 0x007FFFFFu;   // of -inf
constexpr uint32_t kAboveInf = 0xFF800000u;   // the values above are NaN
constexpr float kLeastFinite = -3.402823466e38f;

__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return x != x ? 0xFFFFFFFFu : b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k)
{
    return __uint_as_float(k >> 31 ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ uint64_t entry_key(float x, int64_t index)
{
    return (uint64_t)order_of(x) << 32 | (uint32_t)~(uint32_t)index;
}
__device__ __forceinline__ int key_index(uint64_t k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_value(uint64_t k) { return value_of((uint32_t)(k >> 32)); }

// How many of the n keys in LDS are larger; zeros behind them up to a multiple of kPad (which
// are not larger than any).
constexpr int kPad = 8;
typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int place_of(const uint64_t* keys, int n, uint64_t key)
{
    int place = 0;
    for (int q = 0; q < n; q += kPad) {
        u64x2 k[kPad / 2];
#pragma unroll
        for (int i = 0; i < kPad / 2; ++i)
            k[i] = *(const u64x2*)(keys + q + 2 * i);
#pragma unroll
        for (int i = 0; i < kPad / 2; ++i)
            place += (k[i][0] > key) + (k[i][1] > key);
    }
    return place;
}

// ------------------------------------------------------------------ a row's scalars

// The action of a row as it is, -1 without one
__device__ __forceinline__ int64_t given_action(const LogpArgs& a, int64_t row)
{
    if (!a.actions)
        return -1;
    return a.action_bytes == 1   ? (int64_t)((const uint8_t*)a.actions)[row]
           : a.action_bytes == 4 ? (int64_t)((const int32_t*)a.actions)[row]
                                 : ((const int64_t*)a.actions)[row];
}
// -1 where it is not a legal entry
__device__ __forceinline__ int legal_action(const LogpArgs& a, int64_t row, int64_t v)
{
    if (v < 0 || v >= a.A || (a.mask && a.mask[row * a.mask_ld + v] == 0))
        return -1;
    return (int)v;
}
__device__ __forceinline__ int row_action(const LogpArgs& a, int64_t row)
{
    return legal_action(a, row, given_action(a, row));
}

struct RowOut {
    float l, H, m, ln_s;
};

// (x - m) / T, of halves: x - m itself can leave fp32 where the result does not (3e38 and -3e38
// with T = 4)
__device__ __forceinline__ float below_max(const LogpArgs& a, float x, float m)
{
    return __builtin_fmaf(0.5f, x, -0.5f * m) * a.two_over_t;
}

__device__ __forceinline__ RowOut row_finish(const LogpArgs& a, const Stats& st, int action,
                                             float x_a)
{
    RowOut o{0.0f, 0.0f, st.m, 0.0f};
    if (st.s != 0.0f) {
        const float m = st.m == kNegInf ? 0.0f : st.m;   // (only NaN above -inf)
        o.ln_s = logf(st.s);
        o.H = o.ln_s - kLn2 * st.t / st.s;
        if (action >= 0)
            o.l = below_max(a, x_a, m) - o.ln_s;
    }
    return o;
}

__device__ __forceinline__ void store_row(const LogpArgs& a, int64_t row, const RowOut& o)
{
    a.stats[row] = o.l;
    a.stats[a.rows + row] = o.H;
    a.stats[2 * a.rows + row] = o.m;
    a.stats[3 * a.rows + row] = o.ln_s;
}

__device__ __forceinline__ float entry_logp(const LogpArgs& a, const RowOut& o, float x)
{
    return below_max(a, x, o.m == kNegInf ? 0.0f : o.m) - o.ln_s;
}

// ------------------------------------------------ few actions: a lane per row

// 64 rows per wavefront, as in the losses (rows.hpp): rows go through LDS in memory's own
// order.  A list is found in as many rounds as it has places, each over the row's
// entries in registers.  Bound by their instructions: 131072 x 18 fp32, 6 places 12 us, of
// which 5 are the transfer (17.8 MB at the copy's rate: 3.7).
template <typename E, int NA>
__global__ __launch_bounds__(kLaneThreads) void logp_lane_kernel(LogpArgs a)
{
    extern __shared__ float lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int A = a.A, w = a.top < A ? a.top : A;   // w: places that entries can fill
    float* bx = lds + wave * kLaneRows * (A + w);
    float* bv = bx + kLaneRows * A;
    const float c = kLog2e / a.temperature;
    const int64_t tiles = (a.rows + kLaneThreads - 1) / kLaneThreads;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t r0 = tile * kLaneThreads + wave * kLaneRows;
        const int64_t left = a.rows - r0;
        const int n = left < kLaneRows ? (left > 0 ? (int)left : 0) : kLaneRows;
        const uint8_t* mask = a.mask ? a.mask + r0 * a.mask_ld : nullptr;
        const int64_t row = r0 + lane;
        const int64_t given = lane < n ? given_action(a, row) : -1;
        wave_lds_sync();
        rows_to_lds<false, false>((const E*)a.logits + r0 * a.logits_ld, a.logits_ld,
                                  (const E*)nullptr, 0, mask, a.mask_ld, n, A, bx, bx, lane);
        wave_lds_sync();
        // (asked for behind the rows, in the caches by now)
        const int action = lane < n ? legal_action(a, row, given) : -1;
        float x[NA];
        RowOut o{};
        if (lane < n) {
            float* xr = bx + lane * A;
#pragma unroll
            for (int j = 0; j < NA; ++j)
                x[j] = kNegInf;
            row_read(xr, A, x);
            Stats st = empty_stats();
#pragma unroll
            for (int j = 0; j < NA; ++j)
                st.m = fmaxf(st.m, x[j]);
            const float m = st.m == kNegInf ? 0.0f : st.m;
#pragma unroll
            for (int q = 0; q < NA; q += 4) {
                if (q >= A)
                    break;
#pragma unroll
                for (int j = q; j < q + 4; ++j)
                    add_entry<kPolicy>(st, x[j], 0.0f, m, 0.0f, c);
            }
            o = row_finish(a, st, action, action >= 0 ? xr[action] : 0.0f);
            store_row(a, row, o);
        }
        if (w == 0)
            continue;
        wave_lds_sync();   // (the rows in bx have been read)
        if (lane < n) {
            // bf16: order and index fit one number (2M x 18, 6 places 78 us, as in fp32 86; fp32
            // with the index looked for behind the maximum took 5% longer)
            constexpr bool kOne = sizeof(E) == 2;
            uint32_t k[NA];
#pragma unroll
            for (int j = 0; j < NA; ++j) {
                k[j] = order_of(x[j]);
                if (kOne)
                    k[j] = k[j] <= kUnlisted ? 0u : (k[j] & 0xFFFF0000u) | (31u - j);
            }
            for (int p = 0; p < w; ++p) {
                uint32_t best = kOne ? 0u : kUnlisted;
                int at = -1;
#pragma unroll
                for (int q = 0; q < NA; q += 4) {
                    if (q >= A)
                        break;
#pragma unroll
                    for (int j = q; j < q + 4; ++j) {
                        if (!kOne)
                            at = k[j] > best ? j : at;
                        best = k[j] > best ? k[j] : best;
                    }
                }
#pragma unroll
                for (int q = 0; q < NA; q += 4) {
                    if (q >= A)
                        break;
#pragma unroll
                    for (int j = q; j < q + 4; ++j)
                        k[j] = (kOne ? k[j] == best : j == at) ? 0u : k[j];
                }
                if (kOne && best) {   // (a NaN's order lost its low half, which leaves a NaN)
                    at = 31 - (int)(best & 31u);
                    best = best >> 31 ? best & 0xFFFF0000u : best | 0xFFFFu;
                }
                bx[lane * w + p] = __uint_as_float((uint32_t)at);
                bv[lane * w + p] = at < 0 ? 0.0f : entry_logp(a, o, value_of(best));
            }
        }
        wave_lds_sync();
        rows_from_lds<float>(bx, (float*)a.top_idx + r0 * a.top, a.top, n, w, lane);
        rows_from_lds<float>(bv, a.top_logp + r0 * a.top, a.top, n, w, lane);
        const int more = a.top - w;   // places that no entry can fill
        for (int i = lane; i < n * more; i += 64) {
            const int64_t to = (r0 + i / more) * a.top + w + i % more;
            a.top_idx[to] = -1;
            a.top_logp[to] = 0.0f;
        }
    }
}

// ------------------------------------------------ the exact search, in registers

// Sum of a whole number over the group (a wavefront or a workgroup, as all below), in every
// thread; `half`: which half of scratch is next (see group_combine).
template <int T>
__device__ __forceinline__ int group_count(int v, float* scratch, int& half)
{
    static_assert(T >= 64, "");
    float f = lanes_combine<64>((float)v, SumOp());   // (below 2^24: exact)
    if constexpr (T > 64) {
        float* h = scratch + half * kScratch;
        if ((threadIdx.x & 63) == 0)
            h[threadIdx.x >> 6] = f;
        __syncthreads();
        f = lanes_combine<T / 64>(h[threadIdx.x & (T / 64 - 1)], SumOp());
        half ^= 1;
    }
    return (int)f;
}

// f(value, index in the row's part) for each entry in a lane's registers
template <typename E, int T, int C, typename F>
__device__ __forceinline__ void for_entries(u32x4 (&x)[C], int used, int lane, F f)
{
    constexpr int CH = kChunk<E>;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        if (i >= used)
            break;
        float v[CH];
        unpack<E>(x[i], v);
#pragma unroll
        for (int e = 0; e < CH; ++e)
            f(v[e], (lane + i * T) * CH + e);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// A value that at least k of the group's entries are not below, or the least finite
// one: of each of its wavefronts the j-th largest lane's, the least.
constexpr int kBoundRounds = 16;
template <int T>
__device__ __forceinline__ float lower_bound(float m, int k, float* scratch, int& half)
{
    constexpr int W = T / 64;
    const int j = (k + W - 1) / W;
    float bound = kLeastFinite;
    if (j <= kBoundRounds) {   // (uniform)
        const int lane = threadIdx.x & 63;
        for (int r = 0; r < j; ++r) {
            bound = lanes_combine<64>(m, MaxOp());
            const uint64_t who = __ballot(m == bound);
            if (lane == __builtin_ctzll(who | 1ull << 63))   // (without NaN some lane is)
                m = kNegInf;
        }
    }
    if constexpr (W > 1) {
        float* h = scratch + half * kScratch;
        if ((threadIdx.x & 63) == 0)
            h[threadIdx.x >> 6] = -bound;
        __syncthreads();
        bound = -lanes_combine<W>(h[threadIdx.x & (W - 1)], MaxOp());
        half ^= 1;
    }
    return fmaxf(bound, kLeastFinite);
}

// The k first entries of a row's part in the order of lists: out(place, key) for each,
// by any of the group's threads; returns how many there are.  m: the lane's largest
// value; keys: LDS for `cap` >= k keys; *count: LDS, 0.  All threads of a workgroup come here
// together (T > 64), or all lanes of a wavefront.
template <typename E, int T, int C, typename F>
__device__ __forceinline__ int select_top(u32x4 (&x)[C], int used, int lane, float m, int k,
                                          int64_t base, uint64_t* keys, int cap, int* count,
                                          float* scratch, F out)
{
    int half = 0;
    float at_least = lower_bound<T>(m, k, scratch, half);
    int mine = 0;
    for_entries<E, T, C>(x, used, lane, [&](float v, int) { mine += !(v < at_least); });
    int slot = mine ? atomicAdd(count, mine) : 0;
    group_sync<T>();
    int n = *count;
    bool is_nan = false;          // the least listed value is NaN
    int index_below = 1 << 30;    // of the entries at that value, those with an index below
    // Too many, by chance (a part of the row's entries in few lanes), by ties or since the
    // list is long for so few lanes: the exact value of place k, bit by bit, then, where ties
    // are too many, the index up to which they are listed.
    if (n > cap) {   // (uniform, as all counts)
        auto count_if = [&](auto pred) {
            int v = 0;
            for_entries<E, T, C>(x, used, lane, [&](float f, int i) { v += pred(f, i); });
            return group_count<T>(v, scratch, half);
        };
        int above = count_if([&](float f, int) { return f > at_least || f != f; });
        if (above >= k) {
            constexpr int kLast = sizeof(E) == 2 ? 16 : 0;   // (bf16 has no bits below)
            uint32_t t = 0;
            for (int b = 31; b >= kLast; --b) {
                const uint32_t next = t | 1u << b;
                const float v = value_of(next);
                const bool beyond = next > kAboveInf;
                if (count_if([&](float f, int) { return beyond ? f != f : !(f < v); }) >= k)
                    t = next;
            }
            if (kLast > 0 && !(t >> 31))
                t |= (1u << kLast) - 1u;
            is_nan = t > kAboveInf;
            at_least = value_of(t);
            above = count_if(
                [&](float f, int) { return is_nan ? false : f > at_least || f != f; });
        }
        const int ties =
            count_if([&](float f, int) { return is_nan ? f != f : f == at_least; });
        if (above + ties > cap) {
            int lo = 0;
            for (int b = 30 - __builtin_clz(T * C * kChunk<E>); b >= 0; --b) {
                const int next = lo | 1 << b;
                if (count_if([&](float f, int i) {
                        return (is_nan ? f != f : f == at_least) && i < next;
                    }) <= k - above)
                    lo = next;
            }
            index_below = lo;
        }
        auto listed = [&](float f, int i) {
            return is_nan ? f != f && i < index_below
                          : f > at_least || f != f || (f == at_least && i < index_below);
        };
        mine = 0;
        for_entries<E, T, C>(x, used, lane, [&](float f, int i) { mine += listed(f, i); });
        group_sync<T>();
        if (lane == 0)
            *count = 0;
        group_sync<T>();
        slot = mine ? atomicAdd(count, mine) : 0;
        group_sync<T>();
        n = *count;
    }
    if (mine) {
        for_entries<E, T, C>(x, used, lane, [&](float f, int i) {
            const bool listed = is_nan ? f != f && i < index_below
                                       : f > at_least || f != f ||
                                             (f == at_least && i < index_below);
            if (listed)
                keys[slot++] = entry_key(f, base + i);
        });
    }
    group_sync<T>();
    for (int i = lane; i < n; i += T) {
        const uint64_t key = keys[i];
        int place = 0;
        int q = 0;
        for (; q + 4 <= n; q += 4) {
            const uint64_t k0 = keys[q], k1 = keys[q + 1], k2 = keys[q + 2], k3 = keys[q + 3];
            place += (k0 > key) + (k1 > key) + (k2 > key) + (k3 > key);
        }
        for (; q < n; ++q)
            place += keys[q] > key;
        if (place < k)
            out(place, key);
    }
    return n < k ? n : k;
}

// --------------------------------------------- short rows: 4 to 64 lanes per row

// Rows of up to kShortMost entries, C chunks a lane: 4, or 1 where there are few rows, whose lanes
// then have less to do one after the other.  Few rows are bound by latency (192 x 18 fp32 4.6
// us), many by the lists' instructions (65536 x 512 bf16 with one place 28 us, 2.4 TB/s).
constexpr int kShortMost = 1024, kShortThreads = 256;

// The places up to which a group of T lanes with C chunks each finds a list by rounds: their time
// rises with every place, that of a list by the whole wavefront hardly (us, lists by rounds and by
// the wavefront at the last size of rounds here and behind it.  1024 rows, C = 1: fp32 x 63, 14
// and 20 places 5.9 and 6.3, 7.1 and 6.5; x 127, 6 and 8 4.8 and 4.8, 5.3 and 4.9; x 255, 2 and 3
// 4.1 and 4.3, 4.4 and 4.3; bf16 x 127, 20 and 28 6.8 and 7.6, 8.2 and 8.1; x 255, 10 and 14 5.6
// and 5.7, 6.5 and 5.7; x 511, 4 and 6 4.8 and 4.9, 5.4 and 5.0.  65536 rows, C = 4: fp32 x 63, 28
// and 40 28.4 and 29.0, 38.1 and 32.2; x 127, 10 and 14 24.0 and 28.4, 29.9 and 28.8; x 255, 6 and
// 8 32.7 and 34.4, 37.8 and 35.2; x 511, 4 and 6 51.8 and 57.0, 62.5 and 57.6; bf16 x 127, 40 and
// 56 37.7 and 43.0, 49.3 and 47.7; x 255, 20 and 28 37.8 and 38.7, 47.9 and 42.3; x 511, 14 and 20
// 54.0 and 56.2, 67.5 and 58.5; 2040 x 1023, 10 and 14 9.0 and 9.6, 10.6 and 9.8, fp32 3 and 4 6.2
// and 6.7, 6.9 and 6.8).
template <typename E>
constexpr int rounds_most(int T, int C)
{
    const int i = T == 4 ? 0 : T == 8 ? 1 : T == 16 ? 2 : T == 32 ? 3 : 4;
    constexpr int one[2][5] = {{40, 40, 17, 6, 2}, {56, 56, 27, 10, 4}};
    constexpr int four[2][5] = {{28, 13, 6, 5, 3}, {50, 20, 15, 11, 11}};
    return C == 1 ? one[sizeof(E) == 2][i] : four[sizeof(E) == 2][i];
}

struct MaxU32 {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const
    {
        return a > b ? a : b;
    }
};

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true);
}

// The largest of N lanes' numbers (N up to 64), in each; as lanes_combine
template <int N>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
    const MaxU32 op;
    if constexpr (N >= 2)
        v = op(v, dpp_u32<0xB1>(v));
    if constexpr (N >= 4)
        v = op(v, dpp_u32<0x4E>(v));
    if constexpr (N >= 8)
        v = op(v, dpp_u32<0x141>(v));
    if constexpr (N >= 16)
        v = op(v, dpp_u32<0x140>(v));
    if constexpr (N >= 32)
        v = op(v, (uint32_t)__shfl_xor((int)v, 16));
    if constexpr (N >= 64)
        v = op(v, (uint32_t)__shfl_xor((int)v, 32));
    return v;
}

// A list place after place by the row's T lanes.  bf16: order and index fit one number.
template <typename E, int T, int C>
__device__ __forceinline__ void list_by_rounds(const LogpArgs& a, u32x4 (&x)[C], int lane,
                                               int64_t row, bool live, const RowOut& o)
{
    constexpr int CH = kChunk<E>, N = C * CH;
    constexpr bool kOne = sizeof(E) == 2;
    uint32_t k[N];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        float v[CH];
        unpack<E>(x[i], v);
#pragma unroll
        for (int e = 0; e < CH; ++e) {
            const uint32_t key = order_of(v[e]);
            const uint32_t at = (lane + i * T) * CH + e;
            k[i * CH + e] = key <= kUnlisted ? 0u : kOne ? (key & 0xFFFF0000u) | (0xFFFFu - at)
                                                         : key;
        }
    }
    int idx = -1;
    float val = 0.0f;
    for (int p = 0; p < a.top; ++p) {
        uint32_t best = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            best = k[i] > best ? k[i] : best;
        best = lanes_max<T>(best);
        uint32_t at = 0;   // 65535 less the index
        if constexpr (kOne) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                k[i] = k[i] == best ? 0u : k[i];
            at = best & 0xFFFFu;
        } else {
#pragma unroll
            for (int i = N - 1; i >= 0; --i)
                at = k[i] == best ? 0xFFFFu - ((lane + i / CH * T) * CH + i % CH) : at;
            at = lanes_max<T>(at);
#pragma unroll
            for (int i = 0; i < N; ++i)
                k[i] = at == 0xFFFFu - ((lane + i / CH * T) * CH + i % CH) ? 0u : k[i];
        }
        if (p % T == lane) {
            // (bf16: a NaN's order lost its low half, which leaves a NaN)
            const uint32_t order = kOne ? (best >> 31 ? best & 0xFFFF0000u : best | 0xFFFFu) : best;
            idx = best ? (int)(0xFFFFu - at) : -1;
            val = best ? entry_logp(a, o, value_of(order)) : 0.0f;
        }
        if ((p + 1) % T == 0 || p + 1 == a.top) {
            const int64_t to = row * a.top + p - p % T + lane;
            if (live && lane <= p % T) {
                a.top_idx[to] = idx;
                a.top_logp[to] = val;
            }
        }
    }
}

// A list by a wavefront: the row's entries in LDS, lane l takes every 64th.  keys: LDS for
// as many keys and kPad more.
template <typename E, int T, int C>
__device__ __forceinline__ void list_by_wave(const LogpArgs& a, const E* from, uint64_t* keys,
                                             int lane, int64_t row, const RowOut& o)
{
    constexpr int COUNT = T * C * kChunk<E>, N = (COUNT + 63) / 64;
    uint32_t k[N];
    int listed = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        k[i] = COUNT >= 64 || lane < COUNT ? order_of(to_f32(from[lane + 64 * i])) : 0u;
        k[i] = k[i] <= kUnlisted ? 0u : k[i];
        listed += __popcll(__ballot(k[i] != 0));
    }
    const int most = a.top;
    uint32_t t = 1;       // the least order that is listed
    int ties = kShortMost;   // how many entries of that order
    bool search = listed > most;
    if (search && N > 1 && most <= 32) {
        // at least `most` lanes' largest entries are not below t: about as many entries as that
        // (one count a step, not N) as long as they lie in different lanes
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            m = k[i] > m ? k[i] : m;
        uint32_t low = 0;
        for (int b = 31; b >= 16; --b)
            if (__popcll(__ballot(m >= (low | 1u << b))) >= most)
                low |= 1u << b;
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            n += __popcll(__ballot(k[i] >= low));
        if (low > kUnlisted && n <= 2 * most + 32) {
            t = low;
            search = false;
        }
    }
    if (search) {
        auto count = [&](uint32_t c) {
            int n = 0;
#pragma unroll
            for (int i = 0; i < N; ++i)
                n += __popcll(__ballot(k[i] >= c));
            return n;
        };
        t = 0;
        for (int b = 31; b >= 16; --b)
            if (count(t | 1u << b) >= most)
                t |= 1u << b;
        int n = sizeof(E) == 4 ? count(t) : 0;
        if (sizeof(E) == 4 && n > most + 16) {
            for (int b = 15; b >= 0; --b)
                if (count(t | 1u << b) >= most)
                    t |= 1u << b;
            n = 0;
        }
        if (sizeof(E) == 2 && !(t >> 31))
            t |= 0xFFFFu;
        if (sizeof(E) == 2 && t > kAboveInf)
            t = 0xFFFFFFFFu;
        if (n == 0)   // t is an entry's
            ties = most - count(t + 1 > t ? t + 1 : 0xFFFFFFFFu) * (t != 0xFFFFFFFFu);
    }
    int n = 0, tied = 0;
    const uint64_t before = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint64_t same = __ballot(k[i] == t);
        const bool in = k[i] > t || (k[i] == t && tied + __popcll(same & before) < ties);
        const uint64_t who = __ballot(in);
        if (in)
            keys[n + __popcll(who & before)] = (uint64_t)k[i] << 32 | (uint32_t)~(lane + 64 * i);
        n += __popcll(who);
        tied += __popcll(same);
    }
    if (lane < kPad)
        keys[n + lane] = 0;
    wave_lds_sync();
    const int64_t to = row * most;
    for (int i = lane; i < n; i += 64) {
        const uint64_t key = keys[i];
        const int place = place_of(keys, n, key);
        if (place < most) {
            a.top_idx[to + place] = key_index(key);
            a.top_logp[to + place] = entry_logp(a, o, key_value(key));
        }
    }
    for (int i = n + lane; i < most; i += 64) {
        a.top_idx[to + i] = -1;
        a.top_logp[to + i] = 0.0f;
    }
    wave_lds_sync();
}

template <typename E, int T, int C>
__global__ __launch_bounds__(kShortThreads) void logp_short_kernel(LogpArgs a)
{
    constexpr int ROWS = kShortThreads / T, CH = kChunk<E>;
    extern __shared__ u32x4 staged[];   // lists by wavefronts: rows, then keys
    const int lane = threadIdx.x % T, slot = threadIdx.x / T;
    const int wave = threadIdx.x >> 6, wl = threadIdx.x & 63;
    const float c = kLog2e / a.temperature;
    const int64_t tiles = (a.rows + ROWS - 1) / ROWS;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t row = tile * ROWS + slot;
        const bool live = row < a.rows;
        const E* px = (const E*)a.logits + row * a.logits_ld;
        const uint8_t* pm = a.mask ? a.mask + row * a.mask_ld : nullptr;
        const int64_t given = live ? given_action(a, row) : -1;
        u32x4 x[C];
        load_row<E, kPolicy, T, C>(a.A, live, px, (const E*)nullptr, pm, lane, x, nullptr);
        keep_raw<kPolicy>(x, nullptr);   // (asked for behind the row, in the caches by now)
        const int action = live ? legal_action(a, row, given) : -1;
        const float x_a = action >= 0 ? to_f32(px[action]) : 0.0f;
        const int used = (a.A + T * CH - 1) / (T * CH);
        bool unused = true;
        const Stats st = group_merge<T, kPolicy>(chunk_stats<E, kPolicy, C>(x, nullptr, used, c),
                                                 c, nullptr, nullptr, unused);
        const RowOut o = row_finish(a, st, action, x_a);
        if (lane == 0 && live)
            store_row(a, row, o);
        if (a.top == 0)
            continue;
        if (a.top <= rounds_most<E>(T, C)) {
            list_by_rounds<E, T, C>(a, x, lane, row, live, o);
            continue;
        }
        u32x4* mine = staged + wave * 64 * C;
        uint64_t* keys = (uint64_t*)(staged + kShortThreads * C) + wave * (T * C * CH + kPad);
#pragma unroll
        for (int i = 0; i < C; ++i)
            mine[wl / T * T * C + lane + i * T] = x[i];
        wave_lds_sync();
        for (int r = 0; r < 64 / T; ++r) {
            const int64_t at = tile * ROWS + wave * (64 / T) + r;
            if (at >= a.rows)
                break;
            RowOut of = o;
            of.m = __shfl(o.m, r * T);
            of.ln_s = __shfl(o.ln_s, r * T);
            list_by_wave<E, T, C>(a, (const E*)(mine + r * T * C), keys, wl, at, of);
        }
    }
}

// -------------------------------------------------------------- long rows, streamed

// T threads per row, or per part of one (PART: its sums and list go to the workspace): a
// wavefront (lists of up to kWaveTop places) or a workgroup.  They go through the row in tiles
// of U chunks each.  A chunk with an entry that is not below `bound` goes to LDS; the first
// tile's bound is the least of its wavefronts' j-th largest chunks' maxima, j = ceil(k /
// wavefronts).  After 2, 8, 32, ... tiles (long lists: 1, 2, 4, ...) and the last one the chunks'
// entries join the list's candidates, which are cut to about k, the bound becoming the last one's
// value: three times as many (as many) come in from one cut to the next.  Values are cut by the
// high half of their order (bf16 exactly).  Where LDS does not hold them, the row's list is made in
// a second pass, from its end on, in which a tile that brings too many gets a bound of its own
// (4096 x 65536 bf16, 64 places, a first tile without entries or of low ones: 270 us); or, where a
// tile's own entries are too alike for that or a NaN is about, by the exact search, tile by tile,
// which passes over tiles that add nothing (many equal entries: 1.1 ms; entries that rise: 1.8 ms;
// fp32 entries that share the high half of their order, as all from 300 up to 302 do: 16384 x 8192
// of 300 +- 0.5, 64 places, 0.77 ms, around 0 0.16).
// Bound by memory without lists: 4096 x 65536 bf16 102 us, 5.3 TB/s; with 64 places 131 us: the
// cuts' and the first tile's barriers leave their workgroups without loads on the way, and the
// registers of the lists' code keep more workgroups out (tiles half as wide for eight a CU, or the
// next tile's loads ahead of the cuts, took longer).
constexpr int kStreamU = 4, kWaveTop = 64;
template <int T>
struct StreamSize {
    static constexpr int kChunks = T == 64 ? 160 : 512, kKeys = T == 64 ? 256 : 1024;
    static constexpr int kRows = T == 64 ? 4 : 1;   // per workgroup
};

template <int T>
struct Candidates {
    u32x4 raw[StreamSize<T>::kChunks];
    uint64_t keys[StreamSize<T>::kKeys + kPad];
    int at[StreamSize<T>::kChunks];   // first index of each chunk
    float scratch[T > 64 ? 2 * kScratch : 1];
    int n_raw, n_keys;
    float bound;
    bool over;
};

// A number of which nothing is formed ahead: what hangs on a lane's alone would be, before the
// loops over rows and tiles, and in registers that are not there (4096 x 65536 bf16 wrote 57 MB
// of them to memory; 16384 x 8192 fp32, 8 places, takes 124 us for 131).
__device__ __forceinline__ int apart(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// The largest 16-bit prefix of an order, from `lo` (which at least k entries are not below) to
// that of +inf, that at least k of the wavefront's entries are not below.  count(p): how many
// are not below the lowest value of prefix p.  The steps double, then halve: the result lies
// near lo.
template <typename F>
__device__ __forceinline__ uint32_t prefix_bound(uint32_t lo, int k, F count)
{
    uint32_t hi = 0xFF81u, step = 1;   // behind +inf's
    while (lo + step < hi) {   // (uniform)
        const uint32_t p = lo + step;
        if (count(p) < k)
            hi = p;
        else {
            lo = p;
            step *= 2;
        }
    }
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (count(mid) >= k)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}
// The same from the least finite value's prefix, halving alone
template <typename F>
__device__ __forceinline__ uint32_t halved_bound(int k, F count)
{
    uint32_t lo = 0x0080u, hi = 0xFF81u;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (count(mid) >= k)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}
constexpr uint32_t kLeastPrefix = 0x0080u;   // of the least finite value
// the lowest value of a prefix
__device__ __forceinline__ float prefix_value(uint32_t p) { return value_of(p << 16); }

// The chunks' entries become candidates; the candidates are cut to k or a few more.
template <typename E, int T>
__device__ __forceinline__ void tighten(Candidates<T>& l, int lane, int k)
{
    using S = StreamSize<T>;
    constexpr int CH = kChunk<E>;
    group_sync<T>();
    const int chunks = l.n_raw;
    if (chunks > S::kChunks) {   // (uniform over the group)
        l.over = true;
        return;
    }
    const float bound = l.bound;
    for (int i = lane; i < chunks * CH; i += T) {
        const float v = to_f32(((const E*)l.raw)[i]);
        if (!(v < bound)) {
            const int slot = atomicAdd(&l.n_keys, 1);
            if (slot < S::kKeys)
                l.keys[slot] = entry_key(v, l.at[i / CH] + i % CH);
        }
    }
    group_sync<T>();
    const int n = l.n_keys;
    if (n > S::kKeys) {
        l.over = true;
        return;
    }
    if (n > k) {
        if (T == 64 || lane < 64) {
            constexpr int R = 4;   // keys of a lane in registers
            uint32_t order[R];
#pragma unroll
            for (int r = 0; r < R; ++r)
                order[r] =
                    r * 64 + lane < n ? (uint32_t)(l.keys[r * 64 + lane] >> 32) : kUnlisted;
            auto count = [&](uint32_t p) {
                int m = 0;
#pragma unroll
                for (int r = 0; r < R; ++r)
                    m += __popcll(__ballot(order[r] >= p << 16));
                for (int i = R * 64; i < n; i += 64)
                    m += __popcll(__ballot(i + lane < n &&
                                           (uint32_t)(l.keys[i + lane] >> 32) >= p << 16));
                return m;
            };
            const uint32_t p = prefix_bound(order_of(bound) >> 16, k, count);
            int kept = 0;
            for (int i = 0; i < n; i += 64) {
                const uint64_t key = i + lane < n ? l.keys[i + lane] : 0;
                const bool in = (uint32_t)(key >> 32) >= p << 16;
                const uint64_t who = __ballot(in);
                wave_lds_sync();
                if (in)
                    l.keys[kept + __popcll(who & ((1ull << lane) - 1))] = key;
                wave_lds_sync();
                kept += __popcll(who);
            }
            if (lane == 0) {
                l.n_keys = kept;
                l.bound = fmaxf(bound, prefix_value(p));
            }
        }
    }
    if (lane == 0)
        l.n_raw = 0;
    group_sync<T>();
    if (lane < kPad)   // (for place_of; before the next candidates, or the last barrier)
        l.keys[l.n_keys + lane] = 0;
    group_sync<T>();
}

// A row's part once more where LDS did not hold what the first pass asked for: candidates are cut
// before they are too many, and a tile that alone brings too many gets a bound of its own.  The
// last tile comes first: the first pass was misled by the first.  False where that does not help.
template <typename E, int T>
__device__ __forceinline__ bool careful_list(Candidates<T>& l, const E* px, const uint8_t* pm,
                                             int len, int64_t base, int k, int lane)
{
    using S = StreamSize<T>;
    constexpr int U = kStreamU, CH = kChunk<E>, TILE = T * U * CH, W = T / 64;
    group_sync<T>();   // (all have read what the first pass left)
    if (lane == 0) {   // (the first pass' bound holds)
        l.n_raw = l.n_keys = 0;
        l.over = false;
    }
    group_sync<T>();
    int before = 0;   // chunks of the tiles before this one
    for (int j0 = (len - 1) / TILE * TILE; j0 >= 0; j0 -= TILE) {
        u32x4 x[U];
        float top[U];   // of each chunk
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + (lane + u * T) * CH;
            x[u] = load_masked(px + j, len - j, pm ? pm + j : nullptr, j);
            float v[CH];
            unpack<E>(x[u], v);
            top[u] = kNegInf;
#pragma unroll
            for (int e = 0; e < CH; ++e)
                top[u] = fmaxf(top[u], v[e]);
        }
        keep_raw<kPolicy>(x, nullptr);
        auto add = [&]() {
            const float bound = l.bound;
            int mine = 0;
#pragma unroll
            for (int u = 0; u < U; ++u)
                mine += top[u] >= bound;
            int to = mine ? atomicAdd(&l.n_raw, mine) : 0;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (top[u] >= bound) {
                    if (to < S::kChunks) {
                        l.raw[to] = x[u];
                        l.at[to] = (int)base + j0 + (lane + u * T) * CH;
                    }
                    ++to;
                }
            group_sync<T>();
        };
        add();
        const int keys = l.n_keys;
        int n = l.n_raw;   // (uniform: no one adds or cuts before all have passed another barrier)
        if (n * CH + keys > S::kKeys) {
            auto entries = [&](uint32_t p) {
                const float v = prefix_value(p);
                int n = 0;
                for_entries<E, T, U>(x, U, lane,
                                     [&](float f, int) { n += __popcll(__ballot(f >= v)); });
                return n;
            };
            auto chunks = [&](uint32_t p) {
                const float v = prefix_value(p);
                int n = 0;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    n += __popcll(__ballot(top[u] >= v));
                return n;
            };
            // of each wavefront the j-th largest chunk's maximum (or entry, of few chunks), the
            // least; wavefronts with fewer entries than j leave the k to the others
            const int any = chunks(kLeastPrefix);
            const int own = any >= 3 * k ? any : entries(kLeastPrefix);
            int j = k, with = own >= k;
            if constexpr (W > 1) {
                if ((lane & 63) == 0)
                    l.scratch[lane >> 6] = (float)own;
                __syncthreads();
                with = W;
                do {
                    j = (k + with - 1) / with;
                    with = 0;
                    for (int i = 0; i < W; ++i)
                        with += (int)l.scratch[i] >= j;
                } while (with > 0 && with * j < k);
            }
            float bound = any >= 3 * j ? prefix_value(halved_bound(j, chunks))
                          : own >= j   ? prefix_value(halved_bound(j, entries))
                                       : -kNegInf;
            if constexpr (W > 1) {
                if ((lane & 63) == 0)
                    l.scratch[kScratch + (lane >> 6)] = bound;
                __syncthreads();
                for (int i = 0; i < W; ++i)
                    bound = fminf(bound, l.scratch[kScratch + i]);
            }
            if (with > 0 && bound > l.bound) {
                group_sync<T>();   // (all have read the counts and the bound)
                if (lane == 0) {
                    l.n_raw = before;
                    l.bound = bound;
                }
                group_sync<T>();
                add();
                n = l.n_raw;
            }
        }
        if (n * CH + keys > S::kKeys / 2 || j0 == 0) {
            tighten<E, T>(l, lane, k);
            if (l.over)
                return false;
            before = 0;
        } else {
            before = n;
            group_sync<T>();
        }
    }
    return true;
}

// The exact list of a row's part, tile by tile, into l.keys in order; returns its length.
template <typename E, int T>
__device__ __forceinline__ int exact_list(Candidates<T>& l, const E* px, const uint8_t* pm, int len,
                                          int64_t base, int k, int lane)
{
    constexpr int U = kStreamU, CH = kChunk<E>, TILE = T * U * CH;
    uint64_t* best = (uint64_t*)l.raw;   // the list so far, and behind it the tile's
    uint64_t* more = best + k;
    static_assert(sizeof(l.raw) >= 16 * (T == 64 ? kWaveTop : 256), "two lists");
    int n = 0;
    for (int64_t j0 = 0; j0 < len; j0 += TILE) {
        u32x4 x[U];
        float m = kNegInf;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t j = j0 + (lane + u * T) * CH;
            x[u] = load_masked(px + j, len - j < CH ? (int)(len - j) : CH, pm ? pm + j : nullptr,
                               j);
            float v[CH];
            unpack<E>(x[u], v);
#pragma unroll
            for (int e = 0; e < CH; ++e)
                m = fmaxf(m, v[e]);
        }
        group_sync<T>();
        if (n == k) {   // (later entries are listed above the last one's value alone)
            const float last = key_value(best[k - 1]);
            bool above = false;
            for_entries<E, T, U>(x, U, lane, [&](float f, int) { above |= !(f <= last); });
            above &= last == last;
            // (__syncthreads_or here costs every row of the kernel: 4096 x 65536 bf16 142 us
            // for 130)
            bool some = __ballot(above) != 0;
            if constexpr (T > 64) {
                if (lane == 0)
                    l.n_keys = 0;
                group_sync<T>();
                if (some && (lane & 63) == 0)
                    l.n_keys = 1;
                group_sync<T>();
                some = l.n_keys != 0;
                group_sync<T>();
            }
            if (!some)
                continue;
        }
        if (lane == 0)
            l.n_keys = 0;
        group_sync<T>();
        const int got = select_top<E, T, U>(x, U, lane, m, k, base + j0, l.keys,
                                            StreamSize<T>::kKeys, &l.n_keys, l.scratch,
                                            [&](int place, uint64_t key) { more[place] = key; });
        group_sync<T>();
        for (int i = lane; i < n + got; i += T) {   // merged through l.keys
            const uint64_t key = i < n ? best[i] : more[i - n];
            int place = 0;
            for (int q = 0; q < n; ++q)
                place += best[q] > key;
            for (int q = 0; q < got; ++q)
                place += more[q] > key;
            if (place < k)
                l.keys[place] = key;
        }
        n = n + got < k ? n + got : k;
        group_sync<T>();
        for (int i = lane; i < n; i += T)
            best[i] = l.keys[i];
        group_sync<T>();
    }
    for (int i = lane; i < n; i += T)
        l.keys[i] = best[i];
    group_sync<T>();
    return n;
}

template <typename V>
using InLds = __attribute__((address_space(3))) V;
template <typename V>
using InGlobal = __attribute__((address_space(1))) V;

// The list of a row's part in a second pass, into l.keys in order; returns its length.  (A call of
// its own leaves the first pass its registers.  Its pointers say what memory they are of, which a
// call forgets: a first tile without entries, as above, 540 us.)
template <typename E, int T>
__device__ __attribute__((noinline)) int list_again(InLds<Candidates<T>>* lists,
                                                    InGlobal<const E>* logits,
                                                    InGlobal<const uint8_t>* mask, int len,
                                                    int64_t base, int k, int lane, bool any_nan)
{
    Candidates<T>& l = *(Candidates<T>*)lists;
    const E* px = (const E*)logits;
    const uint8_t* pm = (const uint8_t*)mask;
    if (any_nan || !careful_list<E, T>(l, px, pm, len, base, k, lane))
        return exact_list<E, T>(l, px, pm, len, base, k, lane);
    uint64_t* best = (uint64_t*)l.raw;
    const int n = l.n_keys;
    for (int i = lane; i < n; i += T) {
        const uint64_t key = l.keys[i];
        const int place = place_of(l.keys, n, key);
        if (place < k)
            best[place] = key;
    }
    group_sync<T>();
    const int listed = n < k ? n : k;
    for (int i = lane; i < listed; i += T)
        l.keys[i] = best[i];
    group_sync<T>();
    return listed;
}

// LIST: top > 0.  (Without lists the sums alone need no more than four wavefronts a SIMD, and
// registers for the next tile's loads: 4096 x 65536 bf16 108 us, with six 122.)
template <typename E, int T, bool PART, bool LIST>
__global__ __launch_bounds__(256, LIST ? 6 : 4) void logp_stream_kernel(LogpArgs a)
{
    using S = StreamSize<T>;
    constexpr int U = kStreamU, CH = kChunk<E>, TILE = T * U * CH, W = T / 64;
    extern __shared__ u32x4 lists[];
    __shared__ float scratch[T > 64 ? 2 * kScratch : 1];
    // (in fp32 a row is said to be the whole workgroup's: 16384 x 8192, 8 places 133 us, else 149;
    // bf16 rows, and wavefronts', take longer by it: 4096 x 65536, 64 places 157 and 135)
    const int slot = T > 64 && sizeof(E) == 4 ? 0 : threadIdx.x / T;
    Candidates<T>& l = ((Candidates<T>*)lists)[slot];
    const float c = kLog2e / a.temperature;
    const int k = LIST ? a.top : 0;
    const int64_t items = PART ? a.rows * a.splits : a.rows;
    for (int64_t item = (int64_t)blockIdx.x * S::kRows + slot; item < items;
         item += (int64_t)gridDim.x * S::kRows) {   // (a wavefront's, or a workgroup's, alone)
        const int lane = apart(threadIdx.x % T);
        const int64_t row = PART ? item / a.splits : item;
        const int part = PART ? (int)(item % a.splits) : 0;
        const int64_t base = PART ? (int64_t)part * a.part_len : 0;
        const int len = PART ? (int)(a.A - base < a.part_len ? a.A - base : a.part_len) : a.A;
        const E* px = (const E*)a.logits + row * a.logits_ld + base;
        const uint8_t* pm = a.mask ? a.mask + row * a.mask_ld + base : nullptr;
        int action = -1;
        float x_a = 0.0f;
        if (!PART) {
            action = row_action(a, row);
            if (action >= 0)
                x_a = to_f32(px[action]);
        }
        if (k > 0 && lane == 0) {
            l.n_raw = l.n_keys = apart(0);
            l.over = false;
            l.bound = kLeastFinite;
        }
        Stats st = empty_stats();
        float bound = 0.0f;
        // (the tile of the next cut: each comes when three times as many tiles as before it, or
        // as many, have gone by)
        const bool seldom = 4 * k <= S::kChunks;
        int next = seldom ? 1 : 0, tile = 0;
        for (int j0 = 0; j0 < len; j0 += TILE, ++tile) {
            u32x4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + (lane + u * T) * CH;
                x[u] = load_masked(px + j, len - j, pm ? pm + j : nullptr, j);
            }
            float top[U];   // of each chunk
            Stats own = empty_stats();
            const int here = (len - j0 + T * CH - 1) / (T * CH);   // rounds with any chunk
#pragma unroll
            for (int u = 0; u < U; ++u) {
                top[u] = kNegInf;
                if (u >= here)
                    continue;
                float v[CH];
                unpack<E>(x[u], v);
                top[u] = v[0];
#pragma unroll
                for (int e = 1; e < CH; ++e)
                    top[u] = fmaxf(top[u], v[e]);
                own.m = fmaxf(own.m, top[u]);
            }
            const float m = own.m == kNegInf ? 0.0f : own.m;
            keep_raw<kPolicy>(x, nullptr);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u >= here)
                    break;
                float v[CH];
                unpack<E>(x[u], v);
#pragma unroll
                for (int e = 0; e < CH; ++e)
                    add_entry<kPolicy>(own, v[e], 0.0f, m, 0.0f, c);
                __builtin_amdgcn_sched_barrier(0);
            }
            st = tile == 0 ? own : merge<kPolicy>(st, own, c);
            if constexpr (!LIST)
                continue;
            if (tile == 0) {
                const int j = T > 64 ? a.wave_places : k;
                // (entries instead of chunks where the list is long for so few)
                auto entries = [&](uint32_t p) {
                    const float v = prefix_value(p);
                    int n = 0;
                    for_entries<E, T, U>(x, here, lane,
                                         [&](float f, int) { n += __popcll(__ballot(f >= v)); });
                    return n;
                };
                auto count = [&](uint32_t p) {
                    const float v = prefix_value(p);
                    int n = 0;
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        n += __popcll(__ballot(top[u] >= v));
                    return n;
                };
                const int chunks = count(kLeastPrefix);
                uint32_t p = kLeastPrefix;
                if (chunks >= 3 * j)
                    p = halved_bound(j, count);
                else if (entries(kLeastPrefix) >= j)
                    p = halved_bound(j, entries);
                bound = prefix_value(p);
                if constexpr (W > 1) {
                    if ((lane & 63) == 0)
                        scratch[lane >> 6] = (lane >> 6) < a.tile_waves ? bound : -kNegInf;
                    __syncthreads();
                    bound = scratch[0];
#pragma unroll
                    for (int i = 1; i < W; ++i)
                        bound = fminf(bound, scratch[i]);
                }
                bound = fmaxf(bound, kLeastFinite);
                if (lane == 0)
                    l.bound = bound;
                group_sync<T>();   // (and the counts are 0 before others add)
            }
            int mine = 0;
#pragma unroll
            for (int u = 0; u < U; ++u)
                mine += top[u] >= bound;
            if (mine) {
                int to = atomicAdd(&l.n_raw, mine);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (top[u] >= bound) {
                        if (to < S::kChunks) {
                            l.raw[to] = x[u];
                            l.at[to] = (int)base + j0 + (lane + u * T) * CH;
                        }
                        ++to;
                    }
            }
            if (tile == next || j0 + TILE >= len) {
                tighten<E, T>(l, apart(lane), k);
                if (l.over) {   // (no later chunk counts)
                    bound = -kNegInf;
                    next = 1 << 30;
                } else {
                    bound = l.bound;
                    next = seldom ? 4 * next + 3 : 2 * next + 1;
                }
            }
        }
        bool unused = true;
        st = group_merge<T, kPolicy>(st, c, scratch, nullptr, unused);
        RowOut o{};
        if constexpr (PART) {
            if (lane == 0)
                ((Stats*)a.part_stats)[item] = st;
        } else {
            o = row_finish(a, st, action, x_a);
            if (lane == 0)
                store_row(a, row, o);
        }
        if constexpr (!LIST)
            continue;
        int n = l.n_keys;
        bool sorted = false;
        const int own = apart(lane);
        if (__builtin_expect(l.over || st.s != st.s, false)) {
            n = list_again<E, T>((InLds<Candidates<T>>*)&l, (InGlobal<const E>*)px,
                                 (InGlobal<const uint8_t>*)pm, len, base, k, own, st.s != st.s);
            sorted = true;
        }
        const int64_t to = item * k;
        for (int i = own; i < n; i += T) {
            const uint64_t key = l.keys[i];
            const int place = sorted ? i : place_of(l.keys, n, key);
            if (place < k) {
                if constexpr (PART) {
                    a.part_keys[to + place] = key;
                } else {
                    a.top_idx[to + place] = key_index(key);
                    a.top_logp[to + place] = entry_logp(a, o, key_value(key));
                }
            }
        }
        for (int i = n + own; i < k; i += T) {
            if constexpr (PART) {
                a.part_keys[to + i] = 0;
            } else {
                a.top_idx[to + i] = -1;
                a.top_logp[to + i] = 0.0f;
            }
        }
        group_sync<T>();   // (lists and scratch are the next row's)
    }
}

// ------------------------------------------------------------- parts of rows, merged

// A workgroup per row: the parts' sums, and the first of their lists (each in order,
// zeros behind its entries).  At least `top` entries are not below the j-th of every list,
// j = ceil(top / lists), nor below the last place of any one list; with more lists than
// places, nor below the top-th largest of their first entries.  Bound by latency, a chain of
// loads, barriers and stores: 3 x 131071 bf16, 40 places 6 us, the parts before it 9.6.
constexpr int kMergeThreads = 256, kMergeCap = 1024, kMergeAll = 512;
constexpr int kMergeLists = 2;   // of a thread, at most
static_assert(kMergeThreads * kMergeLists <= kMergeCap, "");   // (a key of each list fits)

__global__ __launch_bounds__(kMergeThreads) void logp_merge_kernel(LogpArgs a)
{
    constexpr int T = kMergeThreads;
    __shared__ float scratch[2 * kScratch];
    __shared__ __align__(16) uint64_t keys[kMergeCap + kPad];
    __shared__ uint64_t wave_key[T / 64];
    __shared__ int total;
    const int tid = threadIdx.x, top = a.top;
    const float c = kLog2e / a.temperature;
    auto block_max = [&](uint64_t v) {   // (ends with all having read wave_key)
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            const uint64_t u = __shfl_xor(v, o);
            v = u > v ? u : v;
        }
        __syncthreads();
        if ((tid & 63) == 0)
            wave_key[tid >> 6] = v;
        __syncthreads();
        v = wave_key[0];
        for (int i = 1; i < T / 64; ++i)
            v = wave_key[i] > v ? wave_key[i] : v;
        return v;
    };
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        // (everything that is known to be needed is asked for at once)
        const int64_t given = given_action(a, row);
        const uint64_t* lists = a.part_keys + row * a.splits * top;
        const bool all = a.splits * top <= kMergeAll;
        uint64_t own[kMergeAll / T];
#pragma unroll
        for (int i = 0; i < kMergeAll / T; ++i)
            own[i] = all && tid + i * T < a.splits * top ? lists[tid + i * T] : 0;
        Stats st = empty_stats();
        const Stats* parts = (const Stats*)a.part_stats + row * a.splits;
        for (int i = tid; i < a.splits; i += T)
            st = merge<kPolicy>(st, parts[i], c);
        const int action = legal_action(a, row, given);
        const float x_a =
            action < 0 ? 0.0f
            : a.bf16   ? to_f32(((const bf16_t*)a.logits)[row * a.logits_ld + action])
                       : ((const float*)a.logits)[row * a.logits_ld + action];
        if (all) {
#pragma unroll
            for (int i = 0; i < kMergeAll / T; ++i)
                keys[tid + i * T] = own[i];   // (zeros behind the last one)
        }
        bool unused = true;
        st = group_merge<T, kPolicy>(st, c, scratch, nullptr, unused);   // (with barriers)
        const RowOut o = row_finish(a, st, action, x_a);
        if (tid == 0)
            store_row(a, row, o);
        if (top == 0) {
            __syncthreads();
            continue;
        }
        const int64_t to = row * top;
        auto write = [&](int place, uint64_t key) {
            a.top_idx[to + place] = key ? key_index(key) : -1;
            a.top_logp[to + place] = key ? entry_logp(a, o, key_value(key)) : 0.0f;
        };
        if (all) {   // (zeros are no entries)
            const int n = a.splits * top;
#pragma unroll
            for (int i = 0; i < kMergeAll / T; ++i) {
                if (tid + i * T >= n)
                    continue;
                const int place = place_of(keys, n, own[i]);
                if (own[i] != 0 && place < top)
                    write(place, own[i]);
            }
            const int entries = place_of(keys, n, 0);
            for (int i = entries + tid; i < top; i += T)
                write(i, 0);
            __syncthreads();
            continue;
        }
        // the bound: the largest last place, the least j-th (as the largest of ~key)
        uint64_t last = 0, jth = 0;
        const int j = (top + a.splits - 1) / a.splits;
        for (int i = tid; i < a.splits; i += T) {
            const uint64_t l = lists[(int64_t)i * top + top - 1];
            const uint64_t f = ~lists[(int64_t)i * top + j - 1];
            last = l > last ? l : last;
            jth = f > jth ? f : jth;
        }
        last = block_max(last);
        jth = ~block_max(jth);
        uint64_t bound = last > jth ? last : jth;
        if (a.splits > top) {   // (j = 1)
            for (int i = tid; i < a.splits + kPad; i += T)
                keys[i] = i < a.splits ? lists[(int64_t)i * top] : 0;
            __syncthreads();
            uint64_t best = 0;
            for (int i = tid; i < a.splits; i += T) {
                const uint64_t key = keys[i];
                if (place_of(keys, a.splits, key) == top - 1)
                    best = key;
            }
            best = block_max(best);
            bound = best > bound ? best : bound;
        }
        if (bound == 0)
            bound = 1;   // (zeros are no entries)
        if (tid == 0)
            total = 0;
        __syncthreads();
        // kSide places of every list at a time, until none of them reaches the bound
        constexpr int kSide = 16;
        for (int p0 = 0; p0 < top; p0 += kSide) {
            bool any = false;
            for (int i = tid; i < a.splits * kSide; i += T) {
                const int p = p0 + i % kSide;
                const uint64_t key = p < top ? lists[(int64_t)(i / kSide) * top + p] : 0;
                if (key >= bound) {
                    any = true;
                    const int slot = atomicAdd(&total, 1);
                    if (slot < kMergeCap)
                        keys[slot] = key;
                }
            }
            if (!__syncthreads_or(any))
                break;
        }
        __syncthreads();
        const int n = total;
        if (n <= kMergeCap) {
            if (tid < kPad)
                keys[n + tid] = 0;
            __syncthreads();
            for (int i = tid; i < n; i += T) {
                const uint64_t key = keys[i];
                const int place = place_of(keys, n, key);
                if (place < top)
                    write(place, key);
            }
            for (int i = n + tid; i < top; i += T)
                write(i, 0);
        } else {   // place after place: the largest of the lists' next entries
            int next[kMergeLists] = {};
            for (int p = 0; p < top; ++p) {
                uint64_t head[kMergeLists], best = 0;
#pragma unroll
                for (int q = 0; q < kMergeLists; ++q) {
                    const int i = tid + q * T;
                    head[q] = i < a.splits && next[q] < top ? lists[(int64_t)i * top + next[q]]
                                                            : 0;
                    best = head[q] > best ? head[q] : best;
                }
                best = block_max(best);
#pragma unroll
                for (int q = 0; q < kMergeLists; ++q)
                    next[q] += head[q] == best;
                if (tid == 0)
                    write(p, best);
            }
        }
        __syncthreads();
    }
}

// --------------------------------------------------------------------- gradient

// What a row's gradient needs: 2^d (c0 + c1 d) and, at the action, `at_action` more.
struct GradRow {
    RowGrad g;
    int action;
    bool some;
};

__device__ __forceinline__ GradRow grad_row(const LogpArgs& a, int64_t row)
{
    GradRow r{};
    r.action = a.dlogp ? row_action(a, row) : -1;
    const float H = a.stats[a.rows + row], m = a.stats[2 * a.rows + row];
    const float ln_s = a.stats[3 * a.rows + row];
    const float dl = r.action >= 0 ? a.dlogp[row] : 0.0f;
    const float dh = a.dentropy ? a.dentropy[row] : 0.0f;
    const float k = expf(-ln_s) / a.temperature;
    r.some = m != kNegInf || ln_s != 0.0f;   // (only NaN above -inf: m is -inf, ln s NaN)
    r.g.m = m == kNegInf ? 0.0f : m;
    r.g.c0 = -k * (dl + dh * (H - ln_s));
    r.g.c1 = -k * kLn2 * dh;
    r.g.at_action = dl / a.temperature;
    return r;
}

__device__ __forceinline__ float grad_at(const GradRow& r, float x, int j, float c)
{
    const float v = grad_entry<kPolicy>(r.g, x, 0.0f, c) + (j == r.action ? r.g.at_action : 0.0f);
    return x == kNegInf || !r.some ? 0.0f : v;
}

// As the lane kernel above.
template <typename E, int NA>
__global__ __launch_bounds__(kLaneThreads) void logp_grad_lane_kernel(LogpArgs a)
{
    extern __shared__ float lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int A = a.A;
    float* bx = lds + wave * kLaneRows * A;
    const float c = kLog2e / a.temperature;
    const int64_t tiles = (a.rows + kLaneThreads - 1) / kLaneThreads;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t r0 = tile * kLaneThreads + wave * kLaneRows;
        const int64_t left = a.rows - r0;
        const int n = left < kLaneRows ? (left > 0 ? (int)left : 0) : kLaneRows;
        const uint8_t* mask = a.mask ? a.mask + r0 * a.mask_ld : nullptr;
        GradRow r{};
        if (lane < n)
            r = grad_row(a, r0 + lane);
        wave_lds_sync();
        rows_to_lds<false, false>((const E*)a.logits + r0 * a.logits_ld, a.logits_ld,
                                  (const E*)nullptr, 0, mask, a.mask_ld, n, A, bx, bx, lane);
        wave_lds_sync();
        if (lane < n) {
            float* xr = bx + lane * A;
            float x[NA];
#pragma unroll
            for (int j = 0; j < NA; ++j)
                x[j] = kNegInf;
            row_read(xr, A, x);
#pragma unroll
            for (int q = 0; q < NA; q += 4) {
                if (q >= A)
                    break;
#pragma unroll
                for (int j = q; j < q + 4; ++j)
                    x[j] = grad_at(r, x[j], j, c);
            }
            row_write(xr, A, x);
        }
        wave_lds_sync();
        rows_from_lds(bx, (E*)a.dlogits + r0 * a.dlogits_ld, a.dlogits_ld, n, A, lane);
    }
}

// T lanes per row, or per part of one (splits > 1): every entry apart, in chunks of 16
// bytes.  Bound by memory: 2047 x 50001 bf16, 410 MB, 90 us, 4.5 TB/s.
constexpr int kGradThreads = 256, kGradUnroll = 4;
constexpr int64_t kFewGrad = 1 << 17;   // threads

template <typename E, int T>
__global__ __launch_bounds__(kGradThreads) void logp_grad_kernel(LogpArgs a)
{
    constexpr int ROWS = kGradThreads / T, U = kGradUnroll, CH = kChunk<E>;
    const int lane = threadIdx.x % T, slot = threadIdx.x / T;
    const float c = kLog2e / a.temperature;
    const int64_t items = a.rows * a.splits;
    const int64_t tiles = (items + ROWS - 1) / ROWS;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t item = tile * ROWS + slot;
        if (item >= items)
            continue;
        const int64_t row = a.splits > 1 ? item / a.splits : item;
        const int64_t base = a.splits > 1 ? item % a.splits * a.part_len : 0;
        const int len = a.splits > 1 && a.A - base > a.part_len ? a.part_len : (int)(a.A - base);
        const GradRow r = grad_row(a, row);
        const E* px = (const E*)a.logits + row * a.logits_ld + base;
        E* po = (E*)a.dlogits + row * a.dlogits_ld + base;
        const uint8_t* pm = a.mask ? a.mask + row * a.mask_ld + base : nullptr;
        for (int j0 = lane * CH; j0 < len; j0 += U * T * CH) {
            u32x4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + u * T * CH;
                x[u] = load_masked(px + j, len - j, pm ? pm + j : nullptr, j);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + u * T * CH;
                if (j >= len)
                    break;
                float f[CH];
                unpack<E>(x[u], f);
#pragma unroll
                for (int e = 0; e < CH; ++e)
                    f[e] = grad_at(r, f[e], (int)base + j + e, c);
                store_chunk(po + j, len - j, pack<E>(f));
            }
        }
    }
}

// ---------------------------------------------------------------------- launches

template <typename E, int C>
void launch_short(const LogpArgs& a, int T, unsigned nb, size_t lds, hipStream_t s)
{
    if (T == 4)
        logp_short_kernel<E, 4, C><<<nb, kShortThreads, lds, s>>>(a);
    else if (T == 8)
        logp_short_kernel<E, 8, C><<<nb, kShortThreads, lds, s>>>(a);
    else if (T == 16)
        logp_short_kernel<E, 16, C><<<nb, kShortThreads, lds, s>>>(a);
    else if (T == 32)
        logp_short_kernel<E, 32, C><<<nb, kShortThreads, lds, s>>>(a);
    else if constexpr (sizeof(E) == 4 || C == 1)   // (4 chunks: bf16 rows fit 32 lanes)
        logp_short_kernel<E, 64, C><<<nb, kShortThreads, lds, s>>>(a);
}

template <typename E, int T, bool PART>
void launch_stream(const LogpArgs& a, unsigned nb, hipStream_t s)
{
    if (a.top == 0)
        logp_stream_kernel<E, T, PART, false><<<nb, 256, 0, s>>>(a);
    else
        logp_stream_kernel<E, T, PART, true>
            <<<nb, 256, sizeof(Candidates<T>) * StreamSize<T>::kRows, s>>>(a);
}

template <typename E>
hipError_t launch_as(const LogpArgs& a, const LogpPlan& p, hipStream_t s)
{
    const unsigned nb = (unsigned)p.blocks;
    if (p.variant == kLogpLane) {
        const int w = a.top < a.A ? a.top : a.A;
        const size_t lds = (size_t)kLaneThreads * 4 * (a.A + w);
        if (a.A <= 8)
            logp_lane_kernel<E, 8><<<nb, kLaneThreads, lds, s>>>(a);
        else if (a.A <= 16)
            logp_lane_kernel<E, 16><<<nb, kLaneThreads, lds, s>>>(a);
        else if (a.A <= 24)
            logp_lane_kernel<E, 24><<<nb, kLaneThreads, lds, s>>>(a);
        else
            logp_lane_kernel<E, 32><<<nb, kLaneThreads, lds, s>>>(a);
    } else if (p.variant == kLogpShort) {
        const size_t lds = a.top > rounds_most<E>(p.group, p.chunks)
                               ? (size_t)kShortThreads * p.chunks * 16 +
                                     (size_t)kShortThreads / 64 *
                                         (p.group * p.chunks * kChunk<E> + kPad) * 8
                               : 0;
        if (p.chunks == 1)
            launch_short<E, 1>(a, p.group, nb, lds, s);
        else
            launch_short<E, 4>(a, p.group, nb, lds, s);
    } else if (p.variant == kLogpWave) {
        launch_stream<E, 64, false>(a, nb, s);
    } else if (p.splits == 1) {
        launch_stream<E, 256, false>(a, nb, s);
    } else {
        launch_stream<E, 256, true>(a, nb, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
        logp_merge_kernel<<<(unsigned)std::min<int64_t>(a.rows, 4096), kMergeThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

template <typename E>
hipError_t launch_grad_as(LogpArgs a, hipStream_t s)
{
    constexpr int64_t kCus = 256, CH = kChunk<E>;
    a.splits = 1;
    if (a.A <= kLaneMost) {
        const unsigned nb = (unsigned)std::min<int64_t>(
            2048, (a.rows + kLaneThreads - 1) / kLaneThreads);
        const size_t lds = (size_t)kLaneThreads * 4 * a.A;
        if (a.A <= 8)
            logp_grad_lane_kernel<E, 8><<<nb, kLaneThreads, lds, s>>>(a);
        else if (a.A <= 16)
            logp_grad_lane_kernel<E, 16><<<nb, kLaneThreads, lds, s>>>(a);
        else if (a.A <= 24)
            logp_grad_lane_kernel<E, 24><<<nb, kLaneThreads, lds, s>>>(a);
        else
            logp_grad_lane_kernel<E, 32><<<nb, kLaneThreads, lds, s>>>(a);
        return hipGetLastError();
    }
    // Lanes of four chunks each, a round of the loop, or of two where that leaves the CUs few
    // threads (us, two and four: bf16 65536 x 1000 53 and 43, 65536 x 250 17.5 and 15.4, 4096 x
    // 2000 10.3 and 9.0, fp32 65536 x 1000 101 and 98; but bf16 4096 x 500 5.3 and 5.5, 200 x 1000
    // 4.2 and 4.7, 4096 x 100 4.5 and 4.8).  Few wide rows in parts (against one each: fp32 3 x
    // 131071 4.4 and 35, 40 x 20000 5.0 and 8.3, 300 x 131071 59 and 70, 1500 x 20000 39 and 39).
    const int64_t chunks = (a.A + CH - 1) / CH;
    int T = 4;
    while (T < kGradThreads && T * (a.rows * T >= kFewGrad ? 4 : 2) < chunks)
        T *= 2;
    if (T == kGradThreads && a.rows < 8 * kCus) {   // parts of at least a round of the loop
        const int64_t want = 8 * kCus / a.rows;
        a.splits = (int)std::max<int64_t>(
            1, std::min<int64_t>(want, chunks / (kGradThreads * kGradUnroll)));
        const int64_t per = (chunks + a.splits - 1) / a.splits;
        a.part_len = (int)(per * CH);
        a.splits = (int)((chunks + per - 1) / per);
    }
    const int64_t tiles = (a.rows * a.splits + kGradThreads / T - 1) / (kGradThreads / T);
    const unsigned nb = (unsigned)std::min<int64_t>(65536, tiles);
    switch (T) {
    case 4:
        logp_grad_kernel<E, 4><<<nb, kGradThreads, 0, s>>>(a);
        break;
    case 8:
        logp_grad_kernel<E, 8><<<nb, kGradThreads, 0, s>>>(a);
        break;
    case 16:
        logp_grad_kernel<E, 16><<<nb, kGradThreads, 0, s>>>(a);
        break;
    case 32:
        logp_grad_kernel<E, 32><<<nb, kGradThreads, 0, s>>>(a);
        break;
    case 64:
        logp_grad_kernel<E, 64><<<nb, kGradThreads, 0, s>>>(a);
        break;
    case 128:
        logp_grad_kernel<E, 128><<<nb, kGradThreads, 0, s>>>(a);
        break;
    default:
        logp_grad_kernel<E, 256><<<nb, kGradThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

// Up to 31 entries a lane per row; up to kShortMost a few lanes.  From half of that on, with many
// rows and, in fp32, without lists, or with more than 6 places, a wavefront (us, 65536 rows of
// 1024 bf16, few lanes and a wavefront, lists of 1, 8 and 64 places: 51 and 76, 97 and 82, 184 and
// 157; of 512: 28 and 73, 42 and 80, 95 and 126; without lists 29 and 37, 8192 x 640 5.2 and 7.4,
// fp32 46 and 40, 6.8 and 5.7).  Above, a wavefront where there are rows enough and short lists
// (700 rows of 3000 bf16, lists of 3 and 64 places 8.6 and 14.0, a workgroup 10.4 and 12.5; 1657
// rows of 1553 fp32 9.2 and 14.2, a workgroup 16.3 and 18.9), else a workgroup, or several where
// there are fewer rows than fill the CUs: of at least a tile (16 KB) each.  Few rows: a chunk per
// lane, while that takes no more threads than fill the CUs a few times (us, lists of 6 places,
// against a lane per row: fp32 4096 x 18 5.4 and 10.0, 65536 x 18 10.4 and 10.8, 131072 x 18 16.6
// and 12.9; against four chunks per lane: 4096 x 60 5.3 and 7.0, 65536 x 60 15.7 and 12.6, 4096 x
// 250 7.7 and 7.7, 16384 x 250 18.7 and 13.0; bf16 131072 x 18 12.4 and 12.5, 4096 x 250 6.3 and
// 8.2, 16384 x 250 11.9 and 9.9).
constexpr int64_t kFewLane = 1 << 19, kFewShort = 1 << 18;
LogpPlan logp_plan(int64_t rows, int64_t A, int top, int size)
{
    constexpr int64_t kCus = 256;
    LogpPlan p{};
    const int64_t ch = 16 / size, chunks = (A + ch - 1) / ch;
    p.splits = 1;
    int64_t per = 1;   // rows per workgroup
    int64_t lanes = 4;   // of a row, a chunk each
    while (lanes < chunks && lanes < 128)
        lanes *= 2;
    const bool few = lanes <= 64 && rows * lanes <= (A <= kLaneMost ? kFewLane : kFewShort);
    if (A <= kLaneMost && !few) {
        p.variant = kLogpLane;
        per = kLaneThreads;
    } else if (A <= kShortMost &&
               !(A > kShortMost / 2 && rows >= 8 * kCus &&
                 (top == 0 ? size == 4 : top > 6 && top <= kWaveTop))) {
        p.variant = kLogpShort;
        p.chunks = few ? 1 : 4;
        p.group = 4;
        while (p.group * p.chunks * ch < A)
            p.group *= 2;
        per = kShortThreads / p.group;
    } else if (top <= kWaveTop && chunks <= 1024 &&
               rows >= (chunks > 512 ? 8 : top > 32 ? 4 : 1) * kCus) {
        p.variant = kLogpWave;
        per = StreamSize<64>::kRows;
    } else {
        p.variant = kLogpGroup;
        const int64_t want = (8 * kCus + rows - 1) / std::max<int64_t>(1, rows);
        const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(
            {want, (int64_t)kMergeThreads * kMergeLists, chunks / (256 * kStreamU)}));
        const int64_t each = (chunks + parts - 1) / parts;
        p.part_len = (int)(each * ch);
        p.splits = (int)((chunks + each - 1) / each);
    }
    p.blocks = std::min<int64_t>(1 << 20, (rows * p.splits + per - 1) / per);
    if (p.splits > 1) {
        p.stats_bytes = (rows * p.splits * (int64_t)sizeof(Stats) + 255) / 256 * 256;
        p.work_bytes = p.stats_bytes + rows * p.splits * top * 8;
    }
    return p;
}

hipError_t launch_logp(LogpArgs a, int dtype, const LogpPlan& p, void* work, hipStream_t s)
{
    a.bf16 = dtype == MALIB_DT_BF16;
    a.two_over_t = 2.0f / a.temperature;
    a.splits = p.splits;
    a.part_len = p.part_len;
    // wavefronts of a streaming workgroup that a row's end leaves 32 chunks at least: the others
    // have too few for a bound (parts have a tile, but for the last one)
    const int64_t chunks = p.splits > 1 ? 1024 : (a.A * (a.bf16 ? 2 : 4) + 15) / 16;
    a.tile_waves = (int)std::max<int64_t>(1, std::min<int64_t>(4, (chunks + 32) / 64));
    a.wave_places = (a.top + a.tile_waves - 1) / a.tile_waves;
    a.part_stats = work;
    a.part_keys = (uint64_t*)((char*)work + p.stats_bytes);
    return a.bf16 ? launch_as<bf16_t>(a, p, s) : launch_as<float>(a, p, s);
}

hipError_t launch_logp_grad(const LogpArgs& a, int dtype, hipStream_t s)
{
    return dtype == MALIB_DT_BF16 ? launch_grad_as<bf16_t>(a, s) : launch_grad_as<float>(a, s);
}

}  // namespace malib
