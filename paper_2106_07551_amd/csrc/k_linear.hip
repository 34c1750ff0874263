// The learner's linear layer, forward and backward:
//
//   forward    z = x W^T + b,  y = act(z) + residual
//   backward   dz = dy act'(z),  dx = dz W,  dW = dz^T x,  db = sum over rows of dz
//
// All three products are one kernel, C[m][n] = sum_k A(m, k) B(n, k), where each
// operand lies in memory either with k contiguous ("KC": x, W of the forward, dz
// of dx) or with its row index contiguous ("RC": W of dx, dz and x of dW).
#include "internal.hpp"

#include <cmath>
#include <type_traits>

#include "chunk.hpp"
#include "device.hpp"

namespace malib {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// k per tile: 128 bytes
template <typename E>
constexpr int kBK = 128 / (int)sizeof(E);

// The activations and their derivatives at z, in fp32.  relu passes a NaN on, as the
// policies' hidden layers do; its derivative at 0 is 0.
__device__ __forceinline__ float relu_f32(float z) { return z != z ? z : (z > 0.0f ? z : 0.0f); }

// e^-x^2 / 2 (`e`) and Phi(x), the normal distribution function.  With ax = |x|,
// 1 - Phi(ax) = e^(-x^2 / 2) R(ax), where R is smooth and falls like 1 / ax: a polynomial
// in t = 1 / (1 + 0.32 ax), fitted to R for the least relative error over all ax >= 0
// (3.2e-8).  To the left the exponent's rounding is the larger part: Phi is within 4e-7 of
// itself down to -2, 2e-6 at -6 (0.5 (1 + erf) in fp32: 1e-5 at -3, 5% at -5).
__device__ __forceinline__ float normal_cdf(float x, float& e)
{
    constexpr int N = 10;
    constexpr float kR[N] = {1.276615262e-01f, 1.276609451e-01f,  1.146223545e-01f,
                             8.782909811e-02f, 5.865395442e-02f,  -9.377530776e-03f,
                             6.532797217e-02f, -1.467074007e-01f, 9.540722519e-02f,
                             -2.107816003e-02f};
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.32f, __builtin_fabsf(x), 1.0f));
    float p = kR[N - 1];
#pragma unroll
    for (int i = N - 2; i >= 0; --i)
        p = __builtin_fmaf(p, t, kR[i]);
    e = __builtin_amdgcn_exp2f(-0.72134752044448170f * (x * x));
    const float tail = (p * t) * e;
    return x > 0.0f ? 1.0f - tail : tail;
}

__device__ __forceinline__ float sigmoid_f32(float z)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * z));
}

template <int N>
__device__ __forceinline__ void activate(int act, float (&v)[N])
{
    switch (act) {
    case MALIB_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = relu_f32(v[i]);
        break;
    case MALIB_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float e;
            v[i] *= normal_cdf(v[i], e);
        }
        break;
    case MALIB_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] *= sigmoid_f32(v[i]);
        break;
    }
}

// v[i] *= act'(z[i])
template <int N>
__device__ __forceinline__ void times_slope(int act, const float (&z)[N], float (&v)[N])
{
    switch (act) {
    case MALIB_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] *= z[i] > 0.0f ? 1.0f : 0.0f;
        break;
    case MALIB_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float e;
            const float p = normal_cdf(z[i], e);
            v[i] *= __builtin_fmaf(z[i] * 0.39894228040143268f, e, p);
        }
        break;
    case MALIB_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float s = sigmoid_f32(z[i]);
            v[i] *= s * __builtin_fmaf(z[i], 1.0f - s, 1.0f);
        }
        break;
    }
}

// ------------------------------------------------------------------- epilogue

// Bias of columns n .. n + cnt - 1 (zeros without one, and behind cnt)
template <int N>
__device__ __forceinline__ void load_bias(const GemmArgs& a, int g, int64_t n, int cnt,
                                          float (&b)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const u32x4 t = a.bias && cnt > i
                            ? load_chunk(a.bias + (int64_t)g * a.N + n + i, cnt - i, n + i)
                            : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            b[i + e] = __uint_as_float(t[e]);
    }
}

template <typename E>
__device__ __forceinline__ u32x4 load_residual(const GemmArgs& a, int g, int64_t m, int64_t n,
                                               int cnt)
{
    return load_chunk((const E*)a.res.p + g * a.res.gs + m * a.res.ld + n, cnt, n);
}

// One chunk of an output row: columns n .. n + cnt - 1 of row m of group g.
template <typename E>
__device__ __forceinline__ void finish_chunk(const GemmArgs& a, int g, int64_t m, int64_t n,
                                             int cnt, const float (&bias)[kChunk<E>], u32x4 res,
                                             float (&v)[kChunk<E>])
{
    if (a.bias) {
#pragma unroll
        for (int i = 0; i < kChunk<E>; ++i)
            v[i] += bias[i];
    }
    if (a.pre.p)
        store_chunk((E*)a.pre.p + g * a.pre.gs + m * a.pre.ld + n, cnt, pack<E>(v));
    activate(a.act, v);
    if (a.res.p) {
        float r[kChunk<E>];
        unpack<E>(res, r);
#pragma unroll
        for (int i = 0; i < kChunk<E>; ++i)
            v[i] += r[i];
    }
    store_chunk((E*)a.c.p + g * a.c.gs + m * a.c.ld + n, cnt, pack<E>(v));
}

// ----------------------------------------------------------------- LDS layout

// A tile of BR rows (of A or B) by 128 bytes of k, as BR * 8 chunks.  KC: row r's
// chunks of k side by side; RC: row k's chunks of r side by side.  The chunk index
// is xor-ed with bits of the row, so that the lanes of one read fall into
// different banks: a KC read takes one chunk from each of 32 rows, an RC read 4
// rows of k from 64 bytes each (bf16, transposing) or 128 bytes from two rows
// (f32).
template <typename E, bool KC, int BR>
__device__ __forceinline__ int chunk_slot(int row, int c)
{
    if constexpr (KC)
        return row * 8 + (c ^ ((row >> 1) & 7));
    constexpr int CPR = BR / kChunk<E>;   // chunks per row of k
    if constexpr (sizeof(E) == 2)
        return row * CPR + (CPR >= 16 ? c ^ ((row & 3) << 2)
                                      : CPR == 8 ? c ^ (((row >> 1) & 1) << 2) : c);
    return row * CPR + (CPR >= 16 ? c ^ (((row >> 2) & 1) << 3) : c);
}

// Row and chunk of slot s (the inverse of chunk_slot).
template <typename E, bool KC, int BR>
__device__ __forceinline__ void slot_chunk(int s, int& row, int& c)
{
    constexpr int CPR = KC ? 8 : BR / kChunk<E>;
    row = s / CPR;
    c = chunk_slot<E, KC, BR>(row, s % CPR) - row * CPR;
}

// Transposing LDS reads: 16 lanes read a block of 4 rows of k by 16, each lane 8
// bytes of it, and get a column each.  Written as assembly because the compiler
// puts a wait for all loads from memory to LDS in front of the builtin, which
// would end the overlap of the next tile's loads with this tile's products; the
// wait for the reads themselves is in the same block.
constexpr int kHalfRows = 4;   // rows of k between a fragment's two reads

template <int OFF, int STEP>
__device__ __forceinline__ void read_transposed(const uint32_t (&p)[1], u32x4 (&v)[1])
{
    uint64_t a, b;
    asm volatile("ds_read_b64_tr_b16 %0, %2 offset:%3\n\t"
                 "ds_read_b64_tr_b16 %1, %2 offset:%4\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b)
                 : "v"(p[0]), "n"(OFF), "n"(OFF + STEP)
                 : "memory");
    v[0] = u32x4{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
}

template <int OFF, int STEP>
__device__ __forceinline__ void read_transposed(const uint32_t (&p)[2], u32x4 (&v)[2])
{
    uint64_t a, b, c, d;
    asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%6\n\t"
                 "ds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
                 "ds_read_b64_tr_b16 %2, %5 offset:%6\n\t"
                 "ds_read_b64_tr_b16 %3, %5 offset:%7\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d)
                 : "v"(p[0]), "v"(p[1]), "n"(OFF), "n"(OFF + STEP)
                 : "memory");
    v[0] = u32x4{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
    v[1] = u32x4{(uint32_t)c, (uint32_t)(c >> 32), (uint32_t)d, (uint32_t)(d >> 32)};
}

template <int OFF, int STEP>
__device__ __forceinline__ void read_transposed(const uint32_t (&p)[4], u32x4 (&v)[4])
{
    uint64_t a, b, c, d, e, f, g, h;
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %2, %9 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %4, %10 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %6, %11 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d), "=&v"(e), "=&v"(f), "=&v"(g), "=&v"(h)
                 : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "n"(OFF), "n"(OFF + STEP)
                 : "memory");
    v[0] = u32x4{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
    v[1] = u32x4{(uint32_t)c, (uint32_t)(c >> 32), (uint32_t)d, (uint32_t)(d >> 32)};
    v[2] = u32x4{(uint32_t)e, (uint32_t)(e >> 32), (uint32_t)f, (uint32_t)(f >> 32)};
    v[3] = u32x4{(uint32_t)g, (uint32_t)(g >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
}

// Operand fragments of step kk (0 .. 3) of a tile for N times 32 rows from rb: 8
// values of k per lane in bf16 (one 32x32x16 product), 4 in f32 (four 32x32x2
// products); lanes 0-31 hold the first half of the step's k, lanes 32-63 the
// second, the same for both operands.
template <typename E, bool KC, int BR, int N>
struct Fragments {
    uint32_t at[N];   // RC in bf16: LDS address of this lane's part at kk = 0 of the first stage
    const char* tile0;
    int rb, lane;

    __device__ __forceinline__ Fragments(const char* tile, int rb_, int lane_)
        : tile0(tile), rb(rb_), lane(lane_)
    {
        if constexpr (!KC && sizeof(E) == 2) {
            const int k = 8 * (lane >> 5) + ((lane >> 2) & 3);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int row = rb + 32 * i + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
                at[i] = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)tile +
                        16 * chunk_slot<E, false, BR>(k, row >> 3) + 2 * (row & 7);
            }
        }
    }

    // of the stage `stage` bytes behind the first
    template <int KK>
    __device__ __forceinline__ void read(int stage, u32x4 (&v)[N]) const
    {
        const int r = lane & 31, h = lane >> 5;
        if constexpr (KC) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] = *(const u32x4*)(tile0 + stage +
                                       16 * chunk_slot<E, true, BR>(rb + 32 * i + r, 2 * KK + h));
        } else if constexpr (sizeof(E) == 2) {
            // (the chunk index is xor-ed with bits of k mod 4 only: rows 4 and 16 further
            // are at fixed distances)
            constexpr int kRow = BR * 2;
            uint32_t p[N];
#pragma unroll
            for (int i = 0; i < N; ++i)
                p[i] = at[i] + (uint32_t)stage;
            read_transposed<16 * KK * kRow, kHalfRows * kRow>(p, v);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    v[i][j] = *(const uint32_t*)(
                        tile0 + stage +
                        16 * chunk_slot<E, false, BR>(8 * KK + 4 * h + j, (rb + 32 * i + r) >> 2) +
                        4 * (r & 3));
        }
    }
};

template <typename E>
__device__ __forceinline__ f32x16 multiply(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (sizeof(E) == 2) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[j]), __uint_as_float(b[j]),
                                                     c, 0, 0, 0);
        return c;
    }
}

// -------------------------------------------------------------- tile loading

// How operand tiles get to LDS: straight from memory (rows on 16-byte boundaries
// that end with whole chunks), or through registers (any alignment, any extent),
// or through registers with A = dy act'(pre) formed on the way (backward pass).
enum { kDirect, kStaged, kFused };

constexpr uint32_t kNoOffset = 0xF0000000u;   // beyond every buffer: reads as zero

// One operand's share of a thread: NI chunks of every tile.
template <typename E, bool KC, int BR, int THREADS, int LOAD>
struct TileLoader {
    static constexpr int NI = BR * 8 / THREADS;
    static constexpr int CH = kChunk<E>;
    const E* base;       // kDirect: the tile's first row (KC) or column (RC) at k = 0
    int64_t ld;
    uint32_t off[NI];    // kDirect: byte offset from the tile's start, or kNoOffset
    // else: this thread's chunks of the next tile, in the operand and in the values
    // before the activation.  What lies behind the operand's end is not read: rows
    // (KC) behind the last repeat it, as what they give is not written; a chunk that
    // crosses the end is read from the last 16 bytes before it, and the first `drop`
    // elements dropped (all of them: not read).  An operand narrower than a chunk goes
    // element by element.
    const E *at[NI], *pre[NI];
    int drop[NI];
    bool narrow, trim;   // (the same for the whole workgroup)
    int k[NI];           // first k of the chunk in the tile
    int64_t step, pre_step;
    int act;
    u32x4 reg[LOAD == kDirect ? 1 : NI], reg_z[LOAD == kFused ? NI : 1];
    int cut[LOAD == kDirect ? 1 : NI];   // elements to drop from what `reg` holds
    bool cuts;

    // R rows by K; the first tile starts at k0
    __device__ __forceinline__ TileLoader(const MatArg& m, const MatArg& z, int act_, int g,
                                          int64_t r0, int R, int K, int64_t k0, int tid)
    {
        ld = m.ld;
        base = (const E*)m.p + g * m.gs + (KC ? r0 * m.ld : r0);
        act = act_;
        step = KC ? kBK<E> : kBK<E> * m.ld;
        pre_step = KC ? kBK<E> : kBK<E> * z.ld;
        const int n_rows = (int)(R - r0);   // rows of the operand from the tile's first on
        narrow = (KC ? K : (int64_t)R) < CH;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            int rr, c;
            slot_chunk<E, KC, BR>(tid + i * THREADS, rr, c);
            const int row = KC ? rr : c * CH;
            k[i] = KC ? c * CH : rr;
            if constexpr (LOAD == kDirect) {
                off[i] = row < n_rows
                             ? (uint32_t)(((int64_t)rr * ld + c * CH) * (int64_t)sizeof(E))
                             : kNoOffset;
            } else {
                const int last = n_rows - CH;   // (RC; below 0 also where the operand is wider)
                const int64_t r = KC ? (row < n_rows ? row : n_rows - 1) : k0 + k[i];
                const int64_t col = KC ? k0 + k[i] : narrow ? row : row < last ? row : last;
                at[i] = base + r * ld + col;
                if (LOAD == kFused)
                    pre[i] = (const E*)z.p + g * z.gs + (KC ? r0 * z.ld : r0) + r * z.ld + col;
                const int behind = KC || narrow || row <= last ? 0 : row - last;
                drop[i] = behind < CH ? behind : CH;
                if (narrow && !KC)   // elements that are there
                    drop[i] = n_rows - row;
            }
        }
        trim = !KC && n_rows < BR;
    }

    // kDirect: the chunks of the tile at k0; a wavefront's 64 chunks are
    // consecutive slots.  Chunks at or behind k1 read as zeros.
    __device__ __forceinline__ void issue(char* tile, int64_t k0, int64_t k1, int tid)
    {
        const E* p = base + (KC ? k0 : k0 * ld);
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, 0x7FFFFFF0, 0x00027000);
        const int left = (int)(k1 - k0 < kBK<E> ? k1 - k0 : kBK<E>);
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const uint32_t o = k[i] < left ? off[i] : kNoOffset;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rsrc, (__attribute__((address_space(3))) void*)(tile + (wave * 64 + i * THREADS) * 16),
                16, o, 0, 0, 0);
        }
    }

    // kStaged, kFused: the next tile's chunks into registers; `left` (> 0): k from its
    // first on
    __device__ __forceinline__ void load(int64_t left)
    {
        const bool end = left < kBK<E>;   // the tile ends with k
        cuts = trim || end;
        if (narrow) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int kl = (int)(end ? left : kBK<E>) - k[i];
                const int n = KC ? kl : kl > 0 ? drop[i] : 0;
                reg[i] = n > 0 ? load_chunk(at[i], n, 0) : u32x4{0, 0, 0, 0};
                if (LOAD == kFused)
                    reg_z[i] = n > 0 ? load_chunk(pre[i], n, 0) : u32x4{0, 0, 0, 0};
                cut[i] = 0;
            }
        } else if (!cuts) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                reg[i] = *(const u32x4_any*)at[i];
                if (LOAD == kFused)
                    reg_z[i] = *(const u32x4_any*)pre[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                int over = 0;   // KC: elements of the chunk behind the end of k
                cut[i] = KC ? 0 : drop[i];
                if (end) {
                    const int rest = (int)left;
                    if (KC) {
                        over = k[i] + CH - rest;
                        over = over < 0 ? 0 : over;
                        cut[i] = over < CH ? over : CH;
                    } else if (k[i] >= rest) {
                        cut[i] = CH;
                    }
                }
                reg[i] = u32x4{0, 0, 0, 0};
                if (LOAD == kFused)
                    reg_z[i] = u32x4{0, 0, 0, 0};
                if (cut[i] < CH) {
                    reg[i] = *(const u32x4_any*)(at[i] - over);
                    if (LOAD == kFused)
                        reg_z[i] = *(const u32x4_any*)(pre[i] - over);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            at[i] += step;
            if (LOAD == kFused)
                pre[i] += pre_step;
        }
    }
    __device__ __forceinline__ void store(char* tile, int tid)
    {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            if constexpr (LOAD == kFused) {
                float v[CH], z[CH];
                unpack<E>(reg[i], v);
                unpack<E>(reg_z[i], z);
                times_slope(act, z, v);
                reg[i] = pack<E>(v);
            }
            if (cuts)
                reg[i] = drop_front<E>(reg[i], cut[i]);
            *(u32x4*)(tile + (tid + i * THREADS) * 16) = reg[i];
        }
    }
};

// --------------------------------------------------------------------- kernel

template <int TILE>
struct GemmShape {
    static constexpr int kWm = 2, kWn = TILE == 256 ? 4 : 2;     // wavefronts
    static constexpr int kThreads = kWm * kWn * 64;
    static constexpr int kTm = TILE / kWm / 32, kTn = TILE / kWn / 32;   // 32x32 tiles of each
    static constexpr int kStage = 2 * TILE * 128;                // bytes of one stage
    static constexpr int kOutLd = kTn * 32 + 4;                  // floats per staged output row
    static constexpr int kOut = kWm * kWn * 32 * kOutLd * 4;
    static constexpr int lds(int stages)
    {
        return stages * kStage > kOut ? stages * kStage : kOut;
    }
};

// s_waitcnt: at most `vm` vector loads outstanding, no LDS operation
constexpr int wait_code(int vm) { return (vm & 15) | ((vm >> 4) << 14) | (7 << 4); }

// Bound by the matrix cores where k is long (8192 x 4096 -> 4096 bf16 forward 241 us, 1.14
// PFLOP/s, backward 488 us; 4096 x 2048 -> 2048 fp32 256 us, 134 TFLOP/s), by memory where
// it is short (131072 x 256 -> 512 bf16 with z kept 84 to 94 us by machine, 4.0 to 3.6 TB/s): LDS holds two stages
// of the largest tile, so one workgroup of it per CU, whose output phase nothing
// overlaps.
// One workgroup's tile of C, number `block` of `n_blocks` of this product.
// STAGES (kDirect): tiles in LDS, in use and on the way.  Four small ones hide the
// latency of products that leave few workgroups per CU; where there are many, two
// leave LDS for more of them.
template <typename E, bool AKC, bool BKC, int TILE, int LOAD, int STAGES>
__device__ __forceinline__ void gemm_tile(const GemmArgs& a, uint32_t block, uint32_t n_blocks,
                                          char* lds)
{
    using S = GemmShape<TILE>;
    constexpr int CH = kChunk<E>, TM = S::kTm, TN = S::kTn;
    // column sums of A beside dW; the largest tile has no registers for them
    constexpr bool kSums = !AKC && TILE < 256;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / S::kWn, wn = wave % S::kWn;

    // Workgroup -> tile: consecutive workgroups go to the 8 XCDs in turn, so each
    // XCD gets one run of the tile order; within it, bands of 8 tile rows are
    // walked column by column, which keeps both operands' tiles in its L2.
    uint32_t id;
    {
        const uint32_t q = n_blocks / 8, r = n_blocks % 8, x = block % 8;
        id = x * q + (x < r ? x : r) + block / 8;
    }
    const uint32_t tiles = (uint32_t)a.mt * (uint32_t)a.nt;   // below 2^31, as the grid
    const uint32_t sg = id / tiles, t0 = id % tiles;
    const int split = (int)(sg / (uint32_t)a.groups), g = (int)(sg % (uint32_t)a.groups);
    int mt, nt;
    {
        const uint32_t band = t0 / 8 / (uint32_t)a.nt, rows_left = (uint32_t)a.mt - band * 8;
        const uint32_t rows = rows_left < 8 ? rows_left : 8;
        const uint32_t u = t0 - band * 8 * (uint32_t)a.nt;
        mt = (int)(band * 8 + u % rows);
        nt = (int)(u / rows);
    }
    const int64_t m0 = (int64_t)mt * TILE, n0 = (int64_t)nt * TILE;
    const int64_t kb = (int64_t)split * a.k_split;
    const int64_t ke = kb + a.k_split < a.K ? kb + a.k_split : a.K;
    const int n_k = (int)((ke - kb + kBK<E> - 1) / kBK<E>);

    TileLoader<E, AKC, TILE, S::kThreads, LOAD> la(a.a, a.a_pre, a.a_act, g, m0, a.M, a.K, kb,
                                                        tid);
    TileLoader<E, BKC, TILE, S::kThreads, LOAD == kFused ? kStaged : LOAD> lb(a.b, a.b, 0, g, n0,
                                                                              a.N, a.K, kb, tid);

    f32x16 acc[TM][TN], sum[kSums ? TM : 1];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
                acc[i][j][r] = 0.0f;
#pragma unroll
        for (int i = 0; i < (kSums ? TM : 1); ++i)
            sum[i][r] = 0.0f;
    }
    const Fragments<E, AKC, TILE, TM> fa(lds, wm * TM * 32, lane);
    const Fragments<E, BKC, TILE, TN> fb(lds + TILE * 128, wn * TN * 32, lane);
    const bool sums = kSums && a.sum && nt == 0 && wn == 0;
    const uint32_t one = sizeof(E) == 2 ? 0x3F803F80u : 0x3F800000u;

    if constexpr (LOAD == kDirect) {
#pragma unroll
        for (int t = 0; t < STAGES - 1; ++t) {
            const int64_t k = kb + (int64_t)t * kBK<E>;
            la.issue(lds + t * S::kStage, k, ke, tid);
            lb.issue(lds + t * S::kStage + TILE * 128, k, ke, tid);
        }
    } else if (n_k > 0) {
        la.load(ke - kb);
        lb.load(ke - kb);
    }
    for (int t = 0; t < n_k; ++t) {
        char* cur = lds + (t & (STAGES - 1)) * S::kStage;
        const int next = LOAD == kDirect ? t + STAGES - 1 : t + 1;
        const int64_t k_next = kb + (int64_t)next * kBK<E>;
        if constexpr (LOAD == kDirect) {
            // this tile has arrived (later ones may be on the way: the loads of each
            // tile are issued in every round, behind the end as reads of nothing, so
            // that the count holds), and every wavefront is done with the stage that is
            // filled next
            constexpr int kLater = (STAGES - 2) * (decltype(la)::NI + decltype(lb)::NI);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(wait_code(kLater));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            char* to = lds + (next & (STAGES - 1)) * S::kStage;
            if (STAGES > 2 || next < n_k) {
                la.issue(to, k_next, ke, tid);
                lb.issue(to + TILE * 128, k_next, ke, tid);
            }
        } else {
            la.store(cur, tid);
            lb.store(cur + TILE * 128, tid);
            __syncthreads();
            if (next < n_k) {
                la.load(ke - k_next);
                lb.load(ke - k_next);
            }
        }
        const int stage = (t & (STAGES - 1)) * S::kStage;
        auto step = [&](auto kk) {
            u32x4 va[TM], vb[TN];
            fa.template read<decltype(kk)::value>(stage, va);
            fb.template read<decltype(kk)::value>(stage, vb);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = multiply<E>(va[i], vb[j], acc[i][j]);
            if constexpr (kSums) {
                if (sums) {
#pragma unroll
                    for (int i = 0; i < TM; ++i)
                        sum[i] = multiply<E>(va[i], u32x4{one, one, one, one}, sum[i]);
                }
            }
        };
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
    }

    // nothing may still land in LDS
    if constexpr (LOAD == kDirect)
        __builtin_amdgcn_s_waitcnt(wait_code(0));
    const int h = lane >> 5;
    if constexpr (kSums) {
        if (sums && (lane & 31) == 0) {
            float* o = a.sum + ((int64_t)split * a.groups + g) * a.M;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int64_t m = m0 + (wm * TM + i) * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
                    if (m < a.M)
                        o[m] = sum[i][r];
                }
        }
    }

    // Output: 32 rows at a time through the wavefront's own part of LDS, so that
    // a lane holds 16 bytes of a row and a row's lanes are neighbours.
    __syncthreads();
    float* buf = (float*)lds + wave * 32 * S::kOutLd;
    constexpr int LPR = TN * 32 / CH, RPP = 64 / LPR;   // lanes per row, rows per pass
    const int64_t n = n0 + wn * TN * 32 + lane % LPR * CH;
    const int cnt = n < a.N ? (int)(a.N - n < CH ? a.N - n : CH) : 0;
    float bias[CH];
    load_bias(a, g, n, a.part ? 0 : cnt, bias);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t mi = m0 + (wm * TM + i) * 32 + lane / LPR;
        u32x4 res[32 / RPP];
#pragma unroll
        for (int p = 0; p < 32 / RPP; ++p)
            res[p] = a.res.p && !a.part && cnt > 0 && mi + p * RPP < a.M
                         ? load_residual<E>(a, g, mi + p * RPP, n, cnt)
                         : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                buf[(8 * (r >> 2) + 4 * h + (r & 3)) * S::kOutLd + j * 32 + (lane & 31)] =
                    acc[i][j][r];
        wave_lds_sync();
        float* row = buf + lane / LPR * S::kOutLd + lane % LPR * CH;
#pragma unroll
        for (int p = 0; p < 32 / RPP; ++p) {
            const int64_t m = mi + p * RPP;
            if (m < a.M && cnt > 0) {
                float v[CH];
#pragma unroll
                for (int e = 0; e < CH; e += 4) {
                    const f32x4 q = *(const f32x4*)(row + p * RPP * S::kOutLd + e);
                    v[e] = q[0];
                    v[e + 1] = q[1];
                    v[e + 2] = q[2];
                    v[e + 3] = q[3];
                }
                if (a.part) {
                    float* o = a.part + (((int64_t)split * a.groups + g) * a.M + m) * a.N + n;
#pragma unroll
                    for (int e = 0; e < CH; e += 4)
                        store_chunk(o + e, cnt - e,
                                    u32x4{__float_as_uint(v[e]), __float_as_uint(v[e + 1]),
                                          __float_as_uint(v[e + 2]), __float_as_uint(v[e + 3])});
                } else {
                    finish_chunk<E>(a, g, m, n, cnt, bias, res[p], v);
                }
            }
        }
        wave_lds_sync();
    }
}

template <typename E, int TILE, int LOAD, int STAGES>
__global__ __launch_bounds__(GemmShape<TILE>::kThreads) void forward_kernel(GemmArgs a,
                                                                            uint32_t first)
{
    __shared__ __attribute__((aligned(16))) char lds[GemmShape<TILE>::lds(STAGES)];
    gemm_tile<E, true, true, TILE, LOAD, STAGES>(a, first + blockIdx.x, (uint32_t)a.blocks, lds);
}

// dW's tiles, then dx's, in one launch: neither waits for the other's last tiles.
template <typename E, int TILE, int LOAD, int STAGES>
__global__ __launch_bounds__(GemmShape<TILE>::kThreads) void backward_kernel(GemmArgs dw,
                                                                             GemmArgs dx,
                                                                             uint32_t first)
{
    __shared__ __attribute__((aligned(16))) char lds[GemmShape<TILE>::lds(STAGES)];
    const uint32_t block = first + blockIdx.x, n_dw = (uint32_t)dw.blocks;
    if (block < n_dw)
        gemm_tile<E, false, false, TILE, LOAD, STAGES>(dw, block, n_dw, lds);
    else
        gemm_tile<E, true, false, TILE, LOAD, STAGES>(dx, block - n_dw, (uint32_t)dx.blocks, lds);
}

// -------------------------------------------------------------- few rows, forward

// At most 16 rows of x: the product reads W once and does little else.  A workgroup
// takes 16 output units, each of its wavefronts a share of k in pieces of 256 bytes
// per unit, straight from memory to registers, W as the first operand of 16x16
// products and x as the second; the shares are added through LDS.  Units and rows
// that do not exist repeat the last one: their results are not written.  Bound by
// the read of W: 3 rows x 8192 -> 8192 bf16 32 us, 4.3 TB/s (with 4 wavefronts 35 us,
// 16 32 us; as 64-wide tiles with split sums 33 us and more, in two launches).
template <typename E>
__global__ __launch_bounds__(512) void few_rows_kernel(GemmArgs a)
{
    constexpr int WAVES = 8;
    constexpr int CH = kChunk<E>, PIECE = 16 * CH;   // k of a piece
    constexpr int AHEAD = 4;                         // pieces on the way
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = blockIdx.y;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int r = lane & 15, h = lane >> 4;
    const int64_t unit = n0 + r < a.N ? n0 + r : a.N - 1, row = r < a.M ? r : a.M - 1;
    const E* w = (const E*)a.b.p + g * a.b.gs + unit * a.b.ld + h * CH;
    const E* x = (const E*)a.a.p + g * a.a.gs + row * a.a.ld + h * CH;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    auto product = [&](const u32x4 (&vw)[4], const u32x4 (&vx)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(E) == 2) {
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vw[i]),
                                                              __builtin_bit_cast(bf16x8, vx[i]),
                                                              acc, 0, 0, 0);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vw[i][j]),
                                                               __uint_as_float(vx[i][j]), acc, 0,
                                                               0, 0);
            }
        }
    };
    const int64_t whole = a.K / PIECE;
    int64_t p = wave;
    for (; p + (AHEAD - 1) * WAVES < whole; p += AHEAD * WAVES) {
        u32x4 vw[AHEAD][4], vx[AHEAD][4];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                vw[u][i] = *(const u32x4_any*)(w + (p + u * WAVES) * PIECE + i * 4 * CH);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                vx[u][i] = *(const u32x4_any*)(x + (p + u * WAVES) * PIECE + i * 4 * CH);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            product(vw[u], vx[u]);
    }
    for (; p * PIECE < a.K; p += WAVES) {   // single pieces, the last one short
        u32x4 vw[4], vx[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t left = a.K - p * PIECE - (i * 4 + h) * CH;
            const int n = left > 0 ? (int)(left < CH ? left : CH) : 0;
            vw[i] = vx[i] = u32x4{0, 0, 0, 0};
            if (n > 0) {
                const int64_t k = p * PIECE + i * 4 * CH;
                vw[i] = load_chunk(w + k, n, k + h * CH);
                vx[i] = load_chunk(x + k, n, k + h * CH);
            }
        }
        product(vw, vx);
    }
    // lane: row r of x, output units 4 h .. 4 h + 3
    __shared__ f32x4 part[WAVES][64];
    part[wave][lane] = acc;
    __syncthreads();
    if (wave != 0 || r >= a.M)
        return;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        const f32x4 t = part[i][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] += t[e];
    }
    const int64_t n = n0 + 4 * h;
    const int cnt = n < a.N ? (int)(a.N - n < 4 ? a.N - n : 4) : 0;
    float bias[4];
    load_bias(a, g, n, cnt, bias);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] += a.bias ? bias[e] : 0.0f;
    if (a.pre.p)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < cnt)
                ((E*)a.pre.p)[g * a.pre.gs + r * a.pre.ld + n + e] = from_f32<E>(v[e]);
    activate(a.act, v);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < cnt) {
            if (a.res.p)
                v[e] += to_f32(((const E*)a.res.p)[g * a.res.gs + r * a.res.ld + n + e]);
            ((E*)a.c.p)[g * a.c.gs + r * a.c.ld + n + e] = from_f32<E>(v[e]);
        }
}

// Bound by memory and launch: 64 parts of 512 x 512 fp32 21 us, most of it from the
// caches; small layers 4 us.
// Sums of the splits' parts, then the epilogue, of up to two products: a workgroup
// takes 256 / SHARES chunks of output, each thread a share of the splits, the shares
// added in order.  Column sums are further items behind a product's chunks.
constexpr int kSumThreads = 256;

template <typename E, int SHARES>
__device__ __forceinline__ void split_sum_block(const GemmArgs& a, int64_t block, float* red)
{
    constexpr int CH = kChunk<E>, ITEMS = kSumThreads / SHARES;
    const int item = threadIdx.x % ITEMS, share = threadIdx.x / ITEMS;
    const int64_t per_row = (a.N + CH - 1) / CH;
    const int64_t n_chunks = (int64_t)a.groups * a.M * per_row;
    const int64_t n_sums = a.sum_out ? (int64_t)a.groups * a.M : 0;
    const int64_t q = block * ITEMS + item;
    const int64_t gm = q < n_chunks ? q / per_row : q - n_chunks;
    const int n = q < n_chunks ? (int)(q - gm * per_row) * CH : 0;
    const int cnt = q < n_chunks ? (a.N - n < CH ? a.N - n : CH) : q < n_chunks + n_sums ? 1 : 0;
    const int64_t plane = (int64_t)a.groups * a.M * (q < n_chunks ? a.N : 1);
    const float* p = q < n_chunks ? a.part + gm * a.N + n : a.sum + gm;
    float v[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e)
        v[e] = 0.0f;
    if (cnt == CH) {
#pragma unroll 4
        for (int s = share; s < a.splits; s += SHARES) {
#pragma unroll
            for (int e = 0; e < CH; e += 4) {
                const u32x4 t = *(const u32x4_any*)(p + s * plane + e);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[e + i] += __uint_as_float(t[i]);
            }
        }
    } else if (cnt > 0) {
#pragma unroll 4
        for (int s = share; s < a.splits; s += SHARES)
#pragma unroll
            for (int e = 0; e < CH; ++e)
                if (e < cnt)
                    v[e] += p[s * plane + e];
    }
    if constexpr (SHARES > 1) {
#pragma unroll
        for (int e = 0; e < CH; ++e)
            red[(share * CH + e) * ITEMS + item] = v[e];
        __syncthreads();
        if (share != 0)
            return;
#pragma unroll
        for (int e = 0; e < CH; ++e)
            for (int t = 1; t < SHARES; ++t)
                v[e] += red[(t * CH + e) * ITEMS + item];
    }
    if (cnt == 0)
        return;
    if (q >= n_chunks) {
        a.sum_out[gm] = v[0];
        return;
    }
    const int g = (int)(gm / a.M);
    float bias[CH];
    load_bias(a, g, n, cnt, bias);
    const u32x4 res = a.res.p ? load_residual<E>(a, g, gm % a.M, n, cnt) : u32x4{0, 0, 0, 0};
    finish_chunk<E>(a, g, gm % a.M, n, cnt, bias, res, v);
}

// db[i] = sum over the row ranges: shares of the ranges by thread, added in order.
constexpr int kDbItems = 8, kDbShares = kSumThreads / kDbItems;

__device__ __forceinline__ void db_block(const DbArgs& d, int64_t block, float* red)
{
    const int item = threadIdx.x % kDbItems, share = threadIdx.x / kDbItems;
    const int64_t i = block * kDbItems + item;
    float t = 0.0f;
    if (i < d.n) {
#pragma unroll 4
        for (int p = share; p < d.count; p += kDbShares)
            t += d.parts[p * d.n + i];
    }
    red[share * kDbItems + item] = t;
    __syncthreads();
    if (share == 0 && i < d.n) {
        for (int k = 1; k < kDbShares; ++k)
            t += red[k * kDbItems + item];
        d.out[i] = t;
    }
}

// The sums of dW's splits (n_a workgroups), of dx's (up to n_b) and of db's ranges
template <typename E, int SHARES>
__global__ __launch_bounds__(kSumThreads) void split_sum_kernel(GemmArgs a, uint32_t n_a,
                                                                GemmArgs b, uint32_t n_b, DbArgs d)
{
    __shared__ float red[SHARES > 1 ? kSumThreads * kChunk<E> : kSumThreads];
    if (blockIdx.x < n_a)
        split_sum_block<E, SHARES>(a, blockIdx.x, red);
    else if (blockIdx.x < n_b)
        split_sum_block<E, SHARES>(b, blockIdx.x - n_a, red);
    else
        db_block(d, blockIdx.x - n_b, red);
}

__global__ __launch_bounds__(kSumThreads) void db_kernel(DbArgs d)
{
    __shared__ float red[kSumThreads];
    db_block(d, blockIdx.x, red);
}

// Threads per chunk: as many as bring about four loads each (512 parts of 6 x 64 fp32 with
// 8 threads: 18 us)
static int sum_shares(const GemmArgs& a)
{
    return a.splits >= 128 ? 32 : a.splits >= 24 ? 8 : a.splits >= 6 ? 2 : 1;
}

template <typename E>
int64_t split_sum_blocks(const GemmArgs& a, int shares)
{
    const int64_t per_row = (a.N + kChunk<E> - 1) / kChunk<E>;
    const int64_t items = (int64_t)a.groups * a.M * (per_row + (a.sum_out ? 1 : 0));
    return (items * shares + kSumThreads - 1) / kSumThreads;
}

// Bound by memory: 131072 x 512 bf16 73 to 79 us by machine (404 MB).  dz = dy act'(z) rounded to the layer's
// type (where there is an activation; the matrix cores take operands of that type), and
// the column sums of the unrounded dz: a workgroup takes 32 chunks of columns
// and a range of rows, eight rows at a time.
constexpr int kDzCols = 32, kDzRows = 8;

template <typename E>
__global__ __launch_bounds__(kDzCols* kDzRows) void dz_kernel(MatArg dy, MatArg pre, MatArg dz,
                                                              int act, int M, int N,
                                                              int rows_per_block, float* sums)
{
    constexpr int CH = kChunk<E>;
    const int cx = threadIdx.x % kDzCols, ry = threadIdx.x / kDzCols;
    const int n = (blockIdx.x * kDzCols + cx) * CH, g = blockIdx.z;
    const int cnt = N - n < CH ? N - n : CH;
    const int64_t r0 = (int64_t)blockIdx.y * rows_per_block;
    const int64_t r1 = r0 + rows_per_block < M ? r0 + rows_per_block : M;
    float s[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e)
        s[e] = 0.0f;
    if (cnt > 0) {
        constexpr int U = 4;   // rows asked for together
        for (int64_t m0 = r0 + ry; m0 < r1; m0 += U * kDzRows) {
            u32x4 vy[U], vz[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t m = m0 + u * kDzRows;
                vy[u] = vz[u] = u32x4{0, 0, 0, 0};
                if (m < r1) {
                    vy[u] = load_chunk((const E*)dy.p + g * dy.gs + m * dy.ld + n, cnt, n);
                    if (act != MALIB_ACT_NONE)
                        vz[u] = load_chunk((const E*)pre.p + g * pre.gs + m * pre.ld + n, cnt, n);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t m = m0 + u * kDzRows;
                if (m >= r1)
                    break;
                float v[CH];
                unpack<E>(vy[u], v);
                if (act != MALIB_ACT_NONE) {
                    float z[CH];
                    unpack<E>(vz[u], z);
                    times_slope(act, z, v);
                    if (dz.p)
                        store_chunk((E*)dz.p + g * dz.gs + m * dz.ld + n, CH, pack<E>(v));
                }
#pragma unroll
                for (int e = 0; e < CH; ++e)
                    s[e] += v[e];
            }
        }
    }
    if (!sums)
        return;
    __shared__ float red[kDzRows][kDzCols * CH + 1];
#pragma unroll
    for (int e = 0; e < CH; ++e)
        red[ry][cx * CH + e] = s[e];
    __syncthreads();
    for (int c = threadIdx.x; c < kDzCols * CH; c += kDzCols * kDzRows) {
        const int col = blockIdx.x * kDzCols * CH + c;
        if (col < N) {
            float t = 0.0f;
#pragma unroll
            for (int r = 0; r < kDzRows; ++r)
                t += red[r][c];
            sums[((int64_t)blockIdx.y * gridDim.z + g) * N + col] = t;
        }
    }
}

// Stages of 64-wide tiles: see gemm_tile.  (16 groups of 8192 x 24 -> 64 fp32: 28 us
// with four, 20 us with two; 1024 x 1024 -> 1024 bf16: 11 us and 13 us.)
int small_stages(int64_t blocks, int64_t k_split, int bk)
{
    return blocks >= 1024 || k_split <= 2 * bk ? 2 : 4;
}

// launch(first, count) for n workgroups: a launch takes fewer than 2^32 threads
template <typename F>
hipError_t in_launches(uint32_t n, F launch)
{
    constexpr uint64_t kMost = (uint64_t)1 << 22;   // (a multiple of the 8 XCDs)
    for (uint64_t first = 0; first < n; first += kMost)
        launch((uint32_t)first, (unsigned)std::min(kMost, n - first));
    return hipGetLastError();
}

template <typename E>
hipError_t launch_forward_as(const GemmArgs& a, int tile, bool direct, hipStream_t s)
{
    auto run = [&](auto kernel, int threads) {
        return in_launches((uint32_t)a.blocks, [&](uint32_t first, unsigned nb) {
            kernel<<<nb, threads, 0, s>>>(a, first);
        });
    };
    if constexpr (sizeof(E) == 2) {   // (fp32 plans take no larger tile than 128)
        if (tile == 256)
            return run(forward_kernel<E, 256, kDirect, 2>, 512);
    }
    if (tile == 128 && direct)
        return run(forward_kernel<E, 128, kDirect, 2>, 256);
    if (tile == 128)
        return run(forward_kernel<E, 128, kStaged, 2>, 256);
    if (!direct)
        return run(forward_kernel<E, 64, kStaged, 2>, 256);
    if (small_stages(a.blocks, a.k_split, kBK<E>) == 2)
        return run(forward_kernel<E, 64, kDirect, 2>, 256);
    return run(forward_kernel<E, 64, kDirect, 4>, 256);
}

template <typename E>
hipError_t launch_few_rows_as(const GemmArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.N + 15) / 16), (unsigned)a.groups);
    few_rows_kernel<E><<<grid, 512, 0, s>>>(a);
    return hipGetLastError();
}

template <typename E>
hipError_t launch_backward_as(const GemmArgs& dw, const GemmArgs& dx, int tile, int load,
                              hipStream_t s)
{
    const uint32_t nb = (uint32_t)dw.blocks + (uint32_t)dx.blocks;   // (each below 2^31)
    if (nb == 0)
        return hipSuccess;
    auto run = [&](auto kernel, int threads) {
        return in_launches(nb, [&](uint32_t first, unsigned n) {
            kernel<<<n, threads, 0, s>>>(dw, dx, first);
        });
    };
    const int64_t k = std::max(dw.blocks ? dw.k_split : 0, dx.blocks ? dx.k_split : 0);
    if constexpr (sizeof(E) == 2) {
        if (tile == 256)
            return run(backward_kernel<E, 256, kDirect, 2>, 512);
    }
    if (tile == 128 && load == kDirect)
        return run(backward_kernel<E, 128, kDirect, 2>, 256);
    if (tile == 128 && load == kStaged)
        return run(backward_kernel<E, 128, kStaged, 2>, 256);
    if (tile == 128)
        return run(backward_kernel<E, 128, kFused, 2>, 256);
    if (load == kStaged)
        return run(backward_kernel<E, 64, kStaged, 2>, 256);
    if (load == kFused)
        return run(backward_kernel<E, 64, kFused, 2>, 256);
    if (small_stages(nb, k, kBK<E>) == 2)
        return run(backward_kernel<E, 64, kDirect, 2>, 256);
    return run(backward_kernel<E, 64, kDirect, 4>, 256);
}

template <typename E>
hipError_t launch_split_sums(const GemmArgs& a, const GemmArgs& b, const DbArgs& d, hipStream_t s)
{
    const bool pa = a.blocks && a.part, pb = b.blocks && b.part;
    const int shares = std::max(pa ? sum_shares(a) : 1, pb ? sum_shares(b) : 1);
    const uint32_t na = pa ? (uint32_t)split_sum_blocks<E>(a, shares) : 0;
    const uint32_t nb = na + (pb ? (uint32_t)split_sum_blocks<E>(b, shares) : 0);
    const uint32_t n = nb + (d.parts ? (uint32_t)((d.n + kDbItems - 1) / kDbItems) : 0);
    if (n == 0)
        return hipSuccess;
    if (nb == 0)
        db_kernel<<<n, kSumThreads, 0, s>>>(d);
    else if (shares == 32)
        split_sum_kernel<E, 32><<<n, kSumThreads, 0, s>>>(a, na, b, nb, d);
    else if (shares == 8)
        split_sum_kernel<E, 8><<<n, kSumThreads, 0, s>>>(a, na, b, nb, d);
    else if (shares == 2)
        split_sum_kernel<E, 2><<<n, kSumThreads, 0, s>>>(a, na, b, nb, d);
    else
        split_sum_kernel<E, 1><<<n, kSumThreads, 0, s>>>(a, na, b, nb, d);
    return hipGetLastError();
}

}  // namespace

// Whether an operand's tiles can go straight to LDS: rows on 16-byte boundaries
// that end with whole chunks, and a tile's bytes within 31 bits.
static bool chunked(const MatArg& m, int size, int64_t contiguous, int groups,
                    bool padded = false)
{
    const int64_t ch = 16 / size;
    if (padded)
        contiguous = 0;   // (a chunk that crosses the end holds zeros there)
    return (uintptr_t)m.p % 16 == 0 && m.ld % ch == 0 && (groups == 1 || m.gs % ch == 0) &&
           contiguous % ch == 0 && m.ld * size <= (int64_t)(0x70000000 / 256);
}

// Tile and splits by estimated time on 256 CUs, from measured constants (us; bf16,
// fp32): a CU's time per 128 bytes of k of a tile with several workgroups on it
// (`busy`) and with one (`alone`; at least 1 us through registers, 2 us element by
// element: 898 x 4 -> 1280 bf16 backward 43 us without splits), and the time of a
// tile's output (`out`).  The
// sum of the splits' parts is a launch and their bytes at about 3.5 TB/s.
//   8192 x 4096 -> 4096 bf16: 64 480 us, 128 279 us, 256 238 us; 2048^3: 64 33 us,
//   128 28 us, 256 53 us, 128 with two splits 64 us; 4096 x 2048 -> 2048 fp32: 64
//   307 us, 128 267 us; 20000 x 256 -> 256 fp32: 64 31 us, 128 43 us; 27815 x 61 -> 281
//   fp32 with ReLU and residual: 64 26 us, 128 41 us.
GemmPlan gemm_plan(int64_t groups, int64_t M, int64_t N, int64_t K, int size, int loads, int tile)
{
    struct Cost {
        int tile;
        double busy, alone, out;
    };
    static constexpr Cost kCosts[2][3] = {{{64, 0.23, 0.30, 1.3}, {128, 0.55, 0.75, 3.1}, {256, 1.75, 1.75, 10.0}},
                                          {{64, 0.60, 0.70, 1.4}, {128, 2.08, 2.1, 7.5}, {0, 0, 0, 0}}};
    constexpr double kCus = 256, kSumLaunch = 5.0, kSumBytes = 3.5e6;
    const int bk = 128 / size;
    const int64_t k_tiles = std::max<int64_t>(1, (K + bk - 1) / bk);
    GemmPlan best{};
    double least = 1e30;
    for (const Cost& c : kCosts[size == 4]) {
        if (c.tile == 0 || (tile == 0 ? c.tile > 64 && std::max(M, N) <= c.tile / 2 : c.tile != tile))
            continue;
        const double alone = std::max(c.alone, loads == kLoadsNarrow   ? 2.0
                                               : loads == kLoadsStaged ? 1.0 : 0.0);
        const double blocks = (double)groups * (double)((M + c.tile - 1) / c.tile) *
                              (double)((N + c.tile - 1) / c.tile);
        for (int64_t s = 1; s <= 512; s *= 2) {
            if (s > 1 && (k_tiles < 2 * s || blocks * (double)(s / 2) >= 2 * kCus))
                break;
            const int64_t per = (k_tiles + s - 1) / s;
            const int64_t splits = (k_tiles + per - 1) / per;
            const double n = std::max(1.0, std::ceil(blocks * (double)splits / kCus));
            double t = (double)per * std::max(alone, n * c.busy) + n * c.out;
            if (splits > 1)
                t += kSumLaunch + (double)splits * (double)groups * (double)M * (double)N * 4.0 / kSumBytes;
            if (t < least) {
                least = t;
                best.tile = c.tile;
                best.splits = (int)splits;
                best.k_split = per * bk;
            }
        }
    }
    best.us = least;
    best.part_bytes = best.splits > 1 ? best.splits * groups * M * N * 4 : 0;
    best.sum_bytes = best.splits > 1 ? best.splits * groups * M * 4 : 0;
    return best;
}

// On different tiles the products are two launches, of which the second waits for the
// first's last workgroups: 5 us and more (34998 x 225 -> 64 fp32).
void backward_plans(int64_t groups, int64_t rows, int64_t in, int64_t out, int size, int loads,
                    GemmPlan& dw, GemmPlan& dx)
{
    constexpr double kLaunch = 5.0;
    dw = gemm_plan(groups, out, in, rows, size, loads);
    dx = gemm_plan(groups, rows, in, out, size, loads);
    if (dw.tile == dx.tile)
        return;
    const GemmPlan w = gemm_plan(groups, out, in, rows, size, loads, dx.tile);
    const GemmPlan x = gemm_plan(groups, rows, in, out, size, loads, dw.tile);
    const double apart = dw.us + dx.us + kLaunch, as_dx = w.us + dx.us, as_dw = dw.us + x.us;
    if (as_dx < apart && as_dx <= as_dw)
        dw = w;
    else if (as_dw < apart)
        dx = x;
}

// The plan's part of a product's arguments
static void apply(GemmArgs& a, const GemmPlan& p, float* part)
{
    a.mt = (int)(((int64_t)a.M + p.tile - 1) / p.tile);   // (M may be 2^31 - 1)
    a.nt = (a.N + p.tile - 1) / p.tile;
    a.splits = p.splits;
    a.k_split = p.k_split;
    a.part = p.splits > 1 ? part : nullptr;
    a.blocks = (int64_t)a.mt * a.nt * a.groups * a.splits;
}

GemmPlan linear_plan(int64_t groups, int64_t M, int64_t N, int64_t K, int size)
{
    if (M <= kFewRows) {
        GemmPlan p{};
        p.splits = 1;
        p.k_split = K;
        return p;
    }
    return gemm_plan(groups, M, N, K, size, loads_of(K, size));
}

hipError_t launch_linear(int dtype, GemmArgs a, GemmPlan p, float* part, hipStream_t s)
{
    const bool bf = dtype == MALIB_DT_BF16;
    if (p.tile == 0)
        return bf ? launch_few_rows_as<bf16_t>(a, s) : launch_few_rows_as<float>(a, s);
    const int size = bf ? 2 : 4;
    const bool direct = chunked(a.a, size, a.K, a.groups) && chunked(a.b, size, a.K, a.groups);
    if (p.tile == 256 && !direct)
        p.tile = 128;   // the largest tile takes aligned rows only
    apply(a, p, part);
    const GemmArgs none{};
    const hipError_t e = bf ? launch_forward_as<bf16_t>(a, p.tile, direct, s)
                            : launch_forward_as<float>(a, p.tile, direct, s);
    if (e != hipSuccess)
        return e;
    const DbArgs no_db{};
    return bf ? launch_split_sums<bf16_t>(a, none, no_db, s)
              : launch_split_sums<float>(a, none, no_db, s);
}

template <typename E>
static hipError_t backward_as(const GemmArgs& dw, int dw_tile, const GemmArgs& dx, int dx_tile,
                              int load, const DbArgs& db, hipStream_t s)
{
    const GemmArgs none{};
    hipError_t e;
    if (dw_tile == dx_tile) {
        e = launch_backward_as<E>(dw, dx, dw_tile, load, s);
    } else {
        e = launch_backward_as<E>(dw, none, dw_tile, load, s);
        if (e == hipSuccess)
            e = launch_backward_as<E>(none, dx, dx_tile, load, s);
    }
    return e != hipSuccess ? e : launch_split_sums<E>(dw, dx, db, s);
}

hipError_t launch_linear_backward(int dtype, GemmArgs dw, GemmPlan pw, float* dw_part,
                                  float* sum_part, GemmArgs dx, GemmPlan px, float* dx_part,
                                  const DbArgs& db, hipStream_t s)
{
    const int size = dtype == MALIB_DT_BF16 ? 2 : 4;
    bool direct = true, fused = false;
    if (dw.c.p) {
        direct = chunked(dw.a, size, dw.M, dw.groups, dw.a_padded) && chunked(dw.b, size, dw.N, dw.groups);
        fused = dw.a_act != MALIB_ACT_NONE;
    }
    if (dx.c.p) {
        direct = direct && chunked(dx.a, size, dx.K, dx.groups, dx.a_padded) &&
                 chunked(dx.b, size, dx.N, dx.groups);
        fused = fused || dx.a_act != MALIB_ACT_NONE;
    }
    const int load = fused ? kFused : direct ? kDirect : kStaged;
    if (load != kDirect) {   // the largest tile takes aligned rows only
        pw.tile = std::min(pw.tile, 128);
        px.tile = std::min(px.tile, 128);
    }
    if (dw.c.p) {
        apply(dw, pw, dw_part);
        if (dw.sum_out)
            dw.sum = pw.splits > 1 ? sum_part : dw.sum_out;
    }
    if (dx.c.p)
        apply(dx, px, dx_part);
    return dtype == MALIB_DT_BF16
               ? backward_as<bf16_t>(dw, pw.tile, dx, px.tile, load, db, s)
               : backward_as<float>(dw, pw.tile, dx, px.tile, load, db, s);
}

DzPlan dz_plan(int64_t groups, int64_t M, int64_t N, int size)
{
    DzPlan p;
    const int64_t cols = (N + kDzCols * (16 / size) - 1) / (kDzCols * (16 / size));
    int64_t parts = std::max<int64_t>(1, 2048 / (cols * groups));
    parts = std::max<int64_t>(1, std::min(parts, (M + 4 * kDzRows - 1) / (4 * kDzRows)));
    p.rows_per_block = (int)std::max<int64_t>(1, (M + parts - 1) / parts);
    p.parts = (int)std::max<int64_t>(1, (M + p.rows_per_block - 1) / p.rows_per_block);
    p.col_blocks = (int)cols;
    p.sum_bytes = p.parts > 1 ? (int64_t)p.parts * groups * N * 4 : 0;
    return p;
}

hipError_t launch_dz(int dtype, const DzPlan& p, const MatArg& dy, const MatArg& pre,
                     const MatArg& dz, int act, int groups, int M, int N, float* sums,
                     hipStream_t s)
{
    const dim3 grid(p.col_blocks, p.parts, groups);
    if (dtype == MALIB_DT_BF16)
        dz_kernel<bf16_t><<<grid, kDzCols * kDzRows, 0, s>>>(dy, pre, dz, act, M, N,
                                                             p.rows_per_block, sums);
    else
        dz_kernel<float><<<grid, kDzCols * kDzRows, 0, s>>>(dy, pre, dz, act, M, N,
                                                            p.rows_per_block, sums);
    return hipGetLastError();
}

}  // namespace malib
