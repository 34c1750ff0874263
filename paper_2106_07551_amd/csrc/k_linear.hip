// The learner's linear layer, forward and backward:
//
//   forward    z = x W^T + b,  y = act(z) + residual
//   backward   dz = dy act'(z),  dx = dz W,  dW = dz^T x,  db = sum over rows of dz
//
// All three products are one kernel, C[m][n] = sum_k A(m, k) B(n, k), where each
// operand lies in memory either with k contiguous ("KC": x, W of the forward, dz
// of dx) or with its row index contiguous ("RC": W of dx, dz and x of dW).
#include "internal.hpp"

#include "chunk.hpp"
#include "device.hpp"

namespace malib {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// k per tile: 128 bytes
template <typename E>
constexpr int kBK = 128 / (int)sizeof(E);

// The activation and its derivative at z, in fp32.  relu passes a NaN on, as the
// policies' hidden layers do; its derivative at 0 is 0.
__device__ __forceinline__ float act_f32(int act, float z)
{
    switch (act) {
    case MALIB_ACT_RELU:
        return z != z ? z : (z > 0.0f ? z : 0.0f);
    case MALIB_ACT_GELU:
        return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    case MALIB_ACT_SILU:
        return z / (1.0f + expf(-z));
    default:
        return z;
    }
}

__device__ __forceinline__ float act_slope_f32(int act, float z)
{
    switch (act) {
    case MALIB_ACT_RELU:
        return z > 0.0f ? 1.0f : 0.0f;
    case MALIB_ACT_GELU:
        return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) +
               z * (0.39894228040143268f * expf(-0.5f * z * z));
    case MALIB_ACT_SILU: {
        const float s = 1.0f / (1.0f + expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    default:
        return 1.0f;
    }
}

// ------------------------------------------------------------------- epilogue

// One chunk of an output row: columns n .. n + cnt - 1 of row m of group g.
template <typename E>
__device__ __forceinline__ void epilogue_chunk(const GemmArgs& a, int g, int64_t m, int n, int cnt,
                                               float (&v)[kChunk<E>])
{
    if (a.bias) {
        const float* b = a.bias + (int64_t)g * a.N + n;
#pragma unroll
        for (int i = 0; i < kChunk<E>; ++i)
            if (i < cnt)
                v[i] += b[i];
    }
    if (a.pre.p)
        store_chunk((E*)a.pre.p + g * a.pre.gs + m * a.pre.ld + n, cnt, pack<E>(v));
    if (a.act != MALIB_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < kChunk<E>; ++i)
            v[i] = act_f32(a.act, v[i]);
    }
    if (a.res.p) {
        float r[kChunk<E>];
        unpack<E>(load_chunk((const E*)a.res.p + g * a.res.gs + m * a.res.ld + n, cnt), r);
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

// Operand fragment of step kk (0 .. 3) of a tile for the 32 rows from rb: 8
// values of k per lane in bf16 (one 32x32x16 product), 4 in f32 (four 32x32x2
// products); lanes 0-31 hold the first half of the step's k, lanes 32-63 the
// second, the same for both operands.
template <typename E, bool KC, int BR>
__device__ __forceinline__ u32x4 fragment(const char* tile, int rb, int kk, int lane)
{
    const int r = lane & 31, h = lane >> 5;
    if constexpr (KC) {
        return *(const u32x4*)(tile + 16 * chunk_slot<E, true, BR>(rb + r, 2 * kk + h));
    } else if constexpr (sizeof(E) == 2) {
        // 16 lanes read a 4 x 16 block (4 of k) and get its transpose
        const int row = rb + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
        const int k = 16 * kk + 8 * h + ((lane >> 2) & 3);
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const char* p = tile + 16 * chunk_slot<E, false, BR>(k + 4 * i, row >> 3) + 2 * (row & 7);
            const s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
            const uint64_t u = __builtin_bit_cast(uint64_t, t);
            v[2 * i] = (uint32_t)u;
            v[2 * i + 1] = (uint32_t)(u >> 32);
        }
        return v;
    } else {
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = *(const uint32_t*)(tile + 16 * chunk_slot<E, false, BR>(8 * kk + 4 * h + j,
                                                                           (rb + r) >> 2) +
                                      4 * (r & 3));
        return v;
    }
}

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

constexpr uint32_t kNoOffset = 0xF0000000u;   // beyond every buffer: reads as zero

// One operand's share of a thread: NI chunks of every tile.
template <typename E, bool KC, int BR, int THREADS, bool FAST>
struct TileLoader {
    static constexpr int NI = BR * 8 / THREADS;
    static constexpr int CH = kChunk<E>;
    const E* base;       // the tile's first row (KC) or column (RC) at k = 0
    int64_t ld;
    uint32_t off[NI];    // FAST: byte offset from the tile's start, or kNoOffset
    int row[NI], k[NI];  // !FAST: row and first k (KC) / first row and k (RC) in the tile
    int n_rows;          // rows of the operand from the tile's first on
    u32x4 reg[FAST ? 1 : NI];

    __device__ __forceinline__ TileLoader(const MatArg& m, int g, int64_t r0, int R, int tid)
    {
        ld = m.ld;
        base = (const E*)m.p + g * m.gs + (KC ? r0 * m.ld : r0);
        n_rows = (int)(R - r0);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            int rr, c;
            slot_chunk<E, KC, BR>(tid + i * THREADS, rr, c);
            row[i] = KC ? rr : c * CH;
            k[i] = KC ? c * CH : rr;
            if constexpr (FAST)
                off[i] = row[i] < n_rows
                             ? (uint32_t)(((int64_t)rr * ld + c * CH) * (int64_t)sizeof(E))
                             : kNoOffset;
        }
    }

    // FAST: chunks of the tile at k0 straight into LDS; a wavefront's 64 chunks
    // are consecutive slots.  Chunks at or behind k1 read as zeros.
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

    // !FAST: the same through registers, any alignment, any extent
    __device__ __forceinline__ void load(int64_t k0, int64_t k1)
    {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int64_t left = k1 - k0 - k[i];
            const int rl = n_rows - row[i];
            int n;
            if constexpr (KC)
                n = rl > 0 ? (int)(left < CH ? left : CH) : 0;
            else
                n = left > 0 ? rl : 0;
            const E* p = base + (KC ? row[i] * ld + k0 + k[i] : (k0 + k[i]) * ld + row[i]);
            reg[i] = n > 0 ? load_chunk(p, n) : u32x4{0, 0, 0, 0};
        }
    }
    __device__ __forceinline__ void store(char* tile, int tid)
    {
#pragma unroll
        for (int i = 0; i < NI; ++i)
            *(u32x4*)(tile + (tid + i * THREADS) * 16) = reg[i];
    }
};

// --------------------------------------------------------------------- kernel

template <int BM, int BN, int WM, int WN>
struct GemmShape {
    static constexpr int kThreads = WM * WN * 64;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;   // 32x32 tiles per wavefront
    static constexpr int kStage = (BM + BN) * 128;               // bytes of one stage
    static constexpr int kOutLd = TN * 32 + 4;                   // floats per staged output row
    static constexpr int kLds = 2 * kStage > WM * WN * 32 * kOutLd * 4 ? 2 * kStage
                                                                      : WM * WN * 32 * kOutLd * 4;
};

template <typename E, bool AKC, bool BKC, int BM, int BN, int WM, int WN, bool FAST>
__global__ __launch_bounds__(WM* WN * 64) void gemm_kernel(GemmArgs a)
{
    using S = GemmShape<BM, BN, WM, WN>;
    constexpr int CH = kChunk<E>;
    __shared__ __attribute__((aligned(16))) char lds[S::kLds];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;

    // Workgroup -> tile: consecutive workgroups go to the 8 XCDs in turn, so each
    // XCD gets one run of the tile order; within it, bands of 8 tile rows are
    // walked column by column, which keeps both operands' tiles in its L2.
    uint32_t id;
    {
        const uint32_t nb = gridDim.x, q = nb / 8, r = nb % 8, x = blockIdx.x % 8;
        id = x * q + (x < r ? x : r) + blockIdx.x / 8;
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
    const int64_t m0 = (int64_t)mt * BM, n0 = (int64_t)nt * BN;
    const int64_t kb = (int64_t)split * a.k_split;
    const int64_t ke = kb + a.k_split < a.K ? kb + a.k_split : a.K;
    const int n_k = (int)((ke - kb + kBK<E> - 1) / kBK<E>);

    TileLoader<E, AKC, BM, S::kThreads, FAST> la(a.a, g, m0, a.M, tid);
    TileLoader<E, BKC, BN, S::kThreads, FAST> lb(a.b, g, n0, a.N, tid);

    f32x16 acc[S::TM][S::TN];
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                acc[i][j][r] = 0.0f;

    if (n_k > 0) {
        if constexpr (FAST) {
            la.issue(lds, kb, ke, tid);
            lb.issue(lds + BM * 128, kb, ke, tid);
        } else {
            la.load(kb, ke);
            lb.load(kb, ke);
        }
    }
    for (int t = 0; t < n_k; ++t) {
        char* cur = lds + (t & 1) * S::kStage;
        char* nxt = lds + ((t + 1) & 1) * S::kStage;
        const int64_t k_next = kb + (int64_t)(t + 1) * kBK<E>;
        if constexpr (!FAST) {
            la.store(cur, tid);
            lb.store(cur + BM * 128, tid);
        }
        // this tile has arrived; every wavefront is done with the other stage
        __syncthreads();
        if (t + 1 < n_k) {
            if constexpr (FAST) {
                la.issue(nxt, k_next, ke, tid);
                lb.issue(nxt + BM * 128, k_next, ke, tid);
            } else {
                la.load(k_next, ke);
                lb.load(k_next, ke);
            }
        }
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            u32x4 fa[S::TM], fb[S::TN];
#pragma unroll
            for (int i = 0; i < S::TM; ++i)
                fa[i] = fragment<E, AKC, BM>(cur, (wm * S::TM + i) * 32, kk, lane);
#pragma unroll
            for (int j = 0; j < S::TN; ++j)
                fb[j] = fragment<E, BKC, BN>(cur + BM * 128, (wn * S::TN + j) * 32, kk, lane);
#pragma unroll
            for (int i = 0; i < S::TM; ++i)
#pragma unroll
                for (int j = 0; j < S::TN; ++j)
                    acc[i][j] = multiply<E>(fa[i], fb[j], acc[i][j]);
        }
    }

    // Output: 32 rows at a time through the wavefront's own part of LDS, so that
    // a lane holds 16 bytes of a row and a row's lanes are neighbours.
    __syncthreads();
    float* buf = (float*)lds + wave * 32 * S::kOutLd;
    const int h = lane >> 5;
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                buf[(8 * (r >> 2) + 4 * h + (r & 3)) * S::kOutLd + j * 32 + (lane & 31)] =
                    acc[i][j][r];
        wave_lds_sync();
        constexpr int LPR = S::TN * 32 / CH;   // lanes per row
#pragma unroll 1
        for (int p = 0; p < 32; p += 64 / LPR) {
            const int r = p + lane / LPR, c = (lane % LPR) * CH;
            const int64_t m = m0 + (wm * S::TM + i) * 32 + r;
            const int64_t n = n0 + wn * S::TN * 32 + c;
            if (m < a.M && n < a.N) {
                const int cnt = (int)(a.N - n < CH ? a.N - n : CH);
                float v[CH];
#pragma unroll
                for (int e = 0; e < CH; e += 4) {
                    const f32x4 q = *(const f32x4*)(buf + r * S::kOutLd + c + e);
                    v[e] = q[0];
                    v[e + 1] = q[1];
                    v[e + 2] = q[2];
                    v[e + 3] = q[3];
                }
                if (a.part) {
                    float* o = a.part + (((int64_t)split * a.groups + g) * a.M + m) * a.N + n;
#pragma unroll
                    for (int e = 0; e < CH; ++e)
                        if (e < cnt)
                            o[e] = v[e];
                } else {
                    epilogue_chunk<E>(a, g, m, (int)n, cnt, v);
                }
            }
        }
        wave_lds_sync();
    }
}

// Sum of the splits' parts in split order, then the epilogue.
template <typename E>
__global__ __launch_bounds__(256) void split_sum_kernel(GemmArgs a)
{
    constexpr int CH = kChunk<E>;
    const int64_t per_row = (a.N + CH - 1) / CH;
    const int64_t n_chunks = (int64_t)a.groups * a.M * per_row;
    const int64_t plane = (int64_t)a.groups * a.M * a.N;
    for (int64_t q = blockIdx.x * 256ll + threadIdx.x; q < n_chunks; q += gridDim.x * 256ll) {
        const int64_t gm = q / per_row;
        const int n = (int)(q % per_row) * CH;
        const int cnt = a.N - n < CH ? a.N - n : CH;
        float v[CH];
#pragma unroll
        for (int e = 0; e < CH; ++e)
            v[e] = 0.0f;
        const float* p = a.part + gm * a.N + n;
        for (int s = 0; s < a.splits; ++s, p += plane) {
#pragma unroll
            for (int e = 0; e < CH; ++e)
                if (e < cnt)
                    v[e] += p[e];
        }
        epilogue_chunk<E>(a, (int)(gm / a.M), gm % a.M, n, cnt, v);
    }
}

// dz = dy act'(z) rounded to the layer's type (where there is an activation), and
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
        for (int64_t m = r0 + ry; m < r1; m += kDzRows) {
            float v[CH];
            unpack<E>(load_chunk((const E*)dy.p + g * dy.gs + m * dy.ld + n, cnt), v);
            if (act != MALIB_ACT_NONE) {
                float z[CH];
                unpack<E>(load_chunk((const E*)pre.p + g * pre.gs + m * pre.ld + n, cnt), z);
#pragma unroll
                for (int e = 0; e < CH; ++e)
                    v[e] *= act_slope_f32(act, z[e]);
                if (dz.p)
                    store_chunk((E*)dz.p + g * dz.gs + m * dz.ld + n, cnt, pack<E>(v));
            }
#pragma unroll
            for (int e = 0; e < CH; ++e)
                s[e] += v[e];
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

// db[i] = sum over the row ranges, in order.
__global__ __launch_bounds__(256) void db_kernel(const float* sums, int64_t n, int parts, float* db)
{
    const int64_t i = blockIdx.x * 256ll + threadIdx.x;
    if (i >= n)
        return;
    float t = 0.0f;
    for (int p = 0; p < parts; ++p)
        t += sums[p * n + i];
    db[i] = t;
}

template <typename E, bool AKC, bool BKC, int BM, int BN, int WM, int WN>
hipError_t launch_shape(const GemmArgs& a, bool fast, int64_t blocks, hipStream_t s)
{
    if (fast)
        gemm_kernel<E, AKC, BKC, BM, BN, WM, WN, true>
            <<<(unsigned)blocks, WM * WN * 64, 0, s>>>(a);
    else
        gemm_kernel<E, AKC, BKC, BM, BN, WM, WN, false>
            <<<(unsigned)blocks, WM * WN * 64, 0, s>>>(a);
    return hipGetLastError();
}

template <typename E, bool AKC, bool BKC>
hipError_t launch_form(const GemmArgs& a, int tile, bool fast, int64_t blocks, hipStream_t s)
{
    if (tile == 256)
        return launch_shape<E, AKC, BKC, 256, 256, 2, 4>(a, fast, blocks, s);
    if (tile == 128)
        return launch_shape<E, AKC, BKC, 128, 128, 2, 2>(a, fast, blocks, s);
    return launch_shape<E, AKC, BKC, 64, 64, 2, 2>(a, fast, blocks, s);
}

}  // namespace

// Whether an operand's tiles can go straight to LDS: rows on 16-byte boundaries
// that end with whole chunks, and a tile's bytes within 31 bits.
static bool chunked(const MatArg& m, int size, int64_t contiguous, int groups)
{
    const int64_t ch = 16 / size;
    return (uintptr_t)m.p % 16 == 0 && m.ld % ch == 0 && (groups == 1 || m.gs % ch == 0) &&
           contiguous % ch == 0 && m.ld * size <= (int64_t)(0x70000000 / 256);
}

GemmPlan gemm_plan(int64_t groups, int64_t M, int64_t N, int64_t K, int size)
{
    GemmPlan p;
    const int bk = 128 / size;
    auto blocks = [&](int t) { return groups * ((M + t - 1) / t) * ((N + t - 1) / t); };
    const int64_t k_tiles = std::max<int64_t>(1, (K + bk - 1) / bk);
    p.tile = 64;
    if (blocks(128) * k_tiles >= 1024 && std::min(M, N) > 64)
        p.tile = 128;
    if (size == 2 && blocks(256) * k_tiles >= 8192 && std::min(M, N) > 128)
        p.tile = 256;
    const int64_t b = std::max<int64_t>(1, blocks(p.tile));
    const int64_t want = p.tile == 256 ? 256 : p.tile == 128 ? 512 : 1024;
    int64_t splits = 1;
    if (b < want && k_tiles > 4)
        splits = std::min(std::min(want / b, k_tiles / 4), (int64_t)128);
    splits = std::max<int64_t>(1, splits);
    const int64_t per = (k_tiles + splits - 1) / splits;
    p.splits = (int)((k_tiles + per - 1) / per);
    p.k_split = per * bk;
    p.part_bytes = p.splits > 1 ? p.splits * groups * M * N * 4 : 0;
    return p;
}

hipError_t launch_gemm(int form, int dtype, GemmArgs a, const GemmPlan& p, float* part,
                       hipStream_t s)
{
    const int size = dtype == MALIB_DT_BF16 ? 2 : 4;
    const int64_t t = p.tile;
    a.mt = (int)((a.M + t - 1) / t);
    a.nt = (int)((a.N + t - 1) / t);
    a.splits = p.splits;
    a.k_split = p.k_split;
    a.part = p.splits > 1 ? part : nullptr;
    const bool fast = chunked(a.a, size, form == kGemmDw ? a.M : a.K, a.groups) &&
                      chunked(a.b, size, form == kGemmForward ? a.K : a.N, a.groups);
    const int64_t blocks = (int64_t)a.mt * a.nt * a.groups * a.splits;
    if (blocks == 0)
        return hipSuccess;
    hipError_t e;
    const bool bf = dtype == MALIB_DT_BF16;
    switch (form) {
    case kGemmForward:
        e = bf ? launch_form<bf16_t, true, true>(a, p.tile, fast, blocks, s)
               : launch_form<float, true, true>(a, p.tile, fast, blocks, s);
        break;
    case kGemmDx:
        e = bf ? launch_form<bf16_t, true, false>(a, p.tile, fast, blocks, s)
               : launch_form<float, true, false>(a, p.tile, fast, blocks, s);
        break;
    default:
        e = bf ? launch_form<bf16_t, false, false>(a, p.tile, fast, blocks, s)
               : launch_form<float, false, false>(a, p.tile, fast, blocks, s);
    }
    if (e != hipSuccess || !a.part)
        return e;
    const int64_t chunks = (int64_t)a.groups * a.M * ((a.N + 16 / size - 1) / (16 / size));
    const unsigned nb = (unsigned)std::min<int64_t>((chunks + 255) / 256, 8192);
    if (bf)
        split_sum_kernel<bf16_t><<<nb, 256, 0, s>>>(a);
    else
        split_sum_kernel<float><<<nb, 256, 0, s>>>(a);
    return hipGetLastError();
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
    p.sum_bytes = (int64_t)p.parts * groups * N * 4;
    return p;
}

hipError_t launch_dz(int dtype, const DzPlan& p, const MatArg& dy, const MatArg& pre,
                     const MatArg& dz, int act, int groups, int M, int N, float* sums, float* db,
                     hipStream_t s)
{
    const dim3 grid(p.col_blocks, p.parts, groups);
    if (dtype == MALIB_DT_BF16)
        dz_kernel<bf16_t><<<grid, kDzCols * kDzRows, 0, s>>>(dy, pre, dz, act, M, N,
                                                             p.rows_per_block, sums);
    else
        dz_kernel<float><<<grid, kDzCols * kDzRows, 0, s>>>(dy, pre, dz, act, M, N,
                                                            p.rows_per_block, sums);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !db)
        return e;
    const int64_t n = (int64_t)groups * N;
    db_kernel<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(sums, n, p.parts, db);
    return hipGetLastError();
}

}  // namespace malib
