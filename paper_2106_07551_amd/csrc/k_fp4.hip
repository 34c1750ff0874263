// Layers of frozen policies in 4 bits: weights v s, v one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and
// their negatives, s a bf16 scale shared by 32, 64 or 128 weights along the input.
//
// Codes lie in the order of the second operand of 16x16x32 products: a lane of a wavefront
// holds the codes of one output and 32 of 128 inputs in 16 bytes, four products' worth.
// gfx950 turns two codes into bf16 in one instruction, exactly; products with bf16 are exact,
// too, and a scale goes onto the fp32 sum of its weights' products.
#include "internal.hpp"

#include <type_traits>

#include "act.hpp"
#include "chunk.hpp"
#include "device.hpp"

namespace malib {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// The bf16 values of eight codes, times a power of two
__device__ __forceinline__ u32x4 code_values(uint32_t c, float times = 1.0f)
{
    u32x4 v;
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, times, 0));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, times, 1));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, times, 2));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, times, 3));
    return v;
}

__device__ __forceinline__ float scale_value(uint16_t s)
{
    return __uint_as_float((uint32_t)s << 16);
}

// ------------------------------------------------------------- weights to codes and back

constexpr int kPackThreads = 256;
constexpr float kSixth = 1.0f / 6.0f;   // of the largest magnitude: a group's scale
// The largest scale (85 x 2^119) whose product with 6 fits fp32, and bf16: with the next one, that
// of fp32 weights beyond 1023 x 2^118 (bf16's end before it), they would come back infinite
constexpr uint16_t kMostScale = 0x7E2A;

// A wavefront per block of 16 outputs x 128 inputs; a lane has output lane & 15 and, of
// each 32 inputs, the eight from 8 (lane >> 4) on.  Bound by memory, without a second round of
// loads on the way in a wavefront: 8192 x 4096 bf16 to codes 16.9 us, 5.1 TB/s, and back 16.2.
struct BlockOf {
    int64_t g, tile, kb;
    __device__ __forceinline__ BlockOf(const Fp4Args& a, int64_t i)
    {
        int64_t q = i;
        if (i >> 31 == 0) {   // (uniform; 64-bit divisions take far longer)
            q = (uint32_t)i / (uint32_t)a.blocks_k;
            kb = i - q * a.blocks_k;
            g = (uint32_t)q / (uint32_t)a.tiles;
        } else {
            q = i / a.blocks_k;
            kb = i - q * a.blocks_k;
            g = q / a.tiles;
        }
        tile = q - g * a.tiles;
    }
};

// Nearest value's code: the comparisons with the borders between values are exact (a
// border times a bf16 scale fits fp32), ties go to the even code.  Bit by bit from the highest: the
// borders below codes 4, 2 and 6 belong to the upper code, the others to the lower.
struct Borders {
    float b1, b2, b3, b4, b5, b6, b7;   // below each code
    __device__ __forceinline__ explicit Borders(float s)
    {
        const float t = s == 0.0f ? __builtin_inff() : s;   // (NaN: no comparison holds)
        b1 = t * 0.25f;
        b2 = t * 0.75f;
        b3 = t * 1.25f;
        b4 = t * 1.75f;
        b5 = t * 2.5f;
        b6 = t * 3.5f;
        b7 = t * 5.0f;
    }
    __device__ __forceinline__ uint32_t code(float w) const
    {
        const float m = __builtin_fabsf(w);
        const bool c2 = m >= b4;
        const float second = c2 ? b6 : b2, low = c2 ? b5 : b1, high = c2 ? b7 : b3;
        const bool c1 = m >= second;
        const bool c0 = m > (c1 ? high : low);
        uint32_t c = c2;
        c = c + c + c1;
        c = c + c + c0;
        return c | (__float_as_uint(w) >> 28 & 8u);   // (-0 is a code, too)
    }
};

// The codes of eight weights.  bf16: a weight and a border of 3 bits times a bf16 scale are
// equal or differ by 2^-11 of themselves at least, so their quotient, formed to a few
// units in its last place and then rounded to 14 bits, lies on a border where it should and on the
// right side of it elsewhere: gfx950's own conversion (nearest, ties to the even code) takes it
// from there.
template <typename E>
__device__ __forceinline__ uint32_t codes_of(const float (&w)[8], float s)
{
    uint32_t c = 0;
    if (sizeof(E) == 2 && s >= 0x1p-120f && s <= 0x1p120f) {
        const float inv = __builtin_amdgcn_rcpf(s);
        float q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            q[e] = __uint_as_float((__float_as_uint(w[e] * inv) + 0x100u) & 0xFFFFFE00u);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[0], q[1], 1.0f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[2], q[3], 1.0f, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[4], q[5], 1.0f, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[6], q[7], 1.0f, 3);
        return c;
    }
    const Borders borders(s);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        c |= borders.code(w[e]) << (4 * e);
    return c;
}

template <typename E>
__global__ __launch_bounds__(kPackThreads) void quantize_kernel(Fp4Args a)
{
    constexpr int CH = kChunk<E>;
    const int lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int per = 128 / a.scale_group;   // scales of an output in a block
    const int64_t n_blocks = (int64_t)a.groups * a.tiles * a.blocks_k;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t i = (int64_t)blockIdx.x * (kPackThreads / 64) + wave; i < n_blocks;
         i += (int64_t)gridDim.x * (kPackThreads / 64)) {
        const BlockOf at(a, i);
        const int64_t n = at.tile * 16 + r, k0 = at.kb * 128 + h * 8;
        const E* w = (const E*)a.w.p + at.g * a.w.gs + n * a.w.ld;
        float v[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int q = 0; q < 8; q += CH) {
                const int64_t k = k0 + j * 32 + q, left = a.K - k;
                u32x4 c = {0, 0, 0, 0};
                if (n < a.N && left > 0)
                    c = load_chunk(w + k, left < CH ? (int)left : CH, k);
                float f[CH];
                unpack<E>(c, f);
#pragma unroll
                for (int e = 0; e < CH; ++e)
                    v[j][q + e] = f[e];
            }
        // (as whole numbers the magnitudes of inf and NaN are above all others)
        uint32_t most[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            most[j] = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t m = __float_as_uint(v[j][e]) & 0x7FFFFFFFu;
                most[j] = m > most[j] ? m : most[j];
            }
#pragma unroll
            for (int o = 16; o <= 32; o *= 2) {
                const uint32_t m = (uint32_t)__shfl_xor((int)most[j], o);
                most[j] = m > most[j] ? m : most[j];
            }
        }
        if (a.scale_group >= 64) {
            most[0] = most[1] = most[0] > most[1] ? most[0] : most[1];
            most[2] = most[3] = most[2] > most[3] ? most[2] : most[3];
        }
        if (a.scale_group == 128)
            most[0] = most[1] = most[2] = most[3] = most[0] > most[2] ? most[0] : most[2];
        u32x4 codes;
        uint16_t scale = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint16_t s = from_f32<bf16_t>(__uint_as_float(most[j]) * kSixth).b;
            if (sizeof(E) == 4 && s > kMostScale)
                s = kMostScale;
            if (most[j] >= 0x7F800000u)
                s = 0x7FC0u;
            if (j * 32 / a.scale_group == h)
                scale = s;
            codes[j] = codes_of<E>(v[j], scale_value(s));
        }
        *(u32x4*)(a.codes + i * 1024 + lane * 16) = codes;
        if (h < per)
            a.scales[(i * 16 + r) * per + h] = scale;
    }
}

template <typename E>
__global__ __launch_bounds__(kPackThreads) void dequantize_kernel(Fp4Args a)
{
    constexpr int CH = kChunk<E>;
    const int lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int per = 128 / a.scale_group;
    const int64_t n_blocks = (int64_t)a.groups * a.tiles * a.blocks_k;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t i = (int64_t)blockIdx.x * (kPackThreads / 64) + wave; i < n_blocks;
         i += (int64_t)gridDim.x * (kPackThreads / 64)) {
        const BlockOf at(a, i);
        const int64_t n = at.tile * 16 + r, k0 = at.kb * 128 + h * 8;
        if (n >= a.N)
            continue;
        E* w = (E*)const_cast<void*>(a.w.p) + at.g * a.w.gs + n * a.w.ld;
        const u32x4 codes = *(const u32x4*)(a.codes + i * 1024 + lane * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t left = a.K - k0 - j * 32;
            if (left <= 0)
                break;
            const float s = scale_value(a.scales[(i * 16 + r) * per + j * 32 / a.scale_group]);
            float v[8];
            unpack<bf16_t>(code_values(codes[j]), v);
#pragma unroll
            for (int q = 0; q < 8; q += CH) {
                float f[CH];
#pragma unroll
                for (int e = 0; e < CH; ++e)
                    f[e] = v[q + e] * s;
                if (left > q)
                    store_chunk(w + k0 + j * 32 + q, left - q < CH ? (int)(left - q) : CH,
                                pack<E>(f));
            }
        }
    }
}

// ----------------------------------------------------------------------- the layer

// Eight consecutive inputs of a row as operands: bf16, or fp32 in three bf16 parts whose
// sum it is (each part the leading 8 bits of what the ones before leave over).
template <typename E>
constexpr int kParts = sizeof(E) == 2 ? 1 : 3;

template <typename E>
__device__ __forceinline__ void split_parts(const u32x4 (&raw)[8 / kChunk<E>],
                                            bf16x8 (&out)[kParts<E>])
{
    if constexpr (sizeof(E) == 2) {
        out[0] = __builtin_bit_cast(bf16x8, raw[0]);
    } else {
        uint32_t b[3][8];
        float check = 0.0f;   // NaN where any input is inf or NaN
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t x = raw[i / 4][i % 4];
            const float rest = __uint_as_float(x) - __uint_as_float(x & 0xFFFF0000u);
            const float mid = __uint_as_float(__float_as_uint(rest) & 0xFFFF0000u);
            b[0][i] = x;
            b[1][i] = __float_as_uint(rest);
            b[2][i] = __float_as_uint(rest - mid);
            check += rest;
        }
        if (__any(check != check)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float f = __uint_as_float(b[0][i]);
                if (f - f != 0.0f) {   // inf or NaN: the first part alone
                    b[0][i] = f != f ? 0x7FC00000u : b[0][i];
                    b[1][i] = b[2][i] = 0;
                }
            }
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            u32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i)   // the high halves of two
                v[i] = __builtin_amdgcn_perm(b[p][2 * i + 1], b[p][2 * i], 0x07060302u);
            out[p] = __builtin_bit_cast(bf16x8, v);
        }
    }
}

// The scales of an output in a block, two in a register
template <int PER>
__device__ __forceinline__ void load_scales(const uint16_t* p, uint32_t (&s)[(PER + 1) / 2])
{
    if constexpr (PER == 4) {
        const uint64_t v = *(const uint64_t*)p;
        s[0] = (uint32_t)v;
        s[1] = (uint32_t)(v >> 32);
    } else if constexpr (PER == 2) {
        s[0] = *(const uint32_t*)p;
    } else {
        s[0] = *p;
    }
}
// (padding's scales may hold anything)
template <int PER>
__device__ __forceinline__ float scale_of(const uint32_t (&s)[(PER + 1) / 2], int i, bool there)
{
    const uint32_t v = s[i / 2];
    return there ? __uint_as_float(i % 2 ? v & 0xFFFF0000u : v << 16) : 0.0f;
}

// Output n of rows m .. m + 3: the sum of COUNT shares, `stride` apart in LDS, and the epilogue.
template <typename E, int COUNT>
__device__ __forceinline__ void finish_tile(const Fp4Args& a, int64_t g, int64_t m, int64_t n,
                                            const f32x4* part, int stride)
{
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const f32x4 f = part[i * stride];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] += f[e];
    }
    if (n >= a.N)
        return;
    if (a.bias) {
        const float b = a.bias[g * a.N + n];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] += b;
    }
    activate(a.act, v);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (m + e < a.M) {
            if (a.res.p)
                v[e] += to_f32(((const E*)a.res.p)[g * a.res.gs + (m + e) * a.res.ld + n]);
            ((E*)const_cast<void*>(a.y.p))[g * a.y.gs + (m + e) * a.y.ld + n] = from_f32<E>(v[e]);
        }
}

// Whether a wavefront's sums are not all finite
template <int N>
__device__ __forceinline__ bool beyond_fp32(const f32x4 (&acc)[N])
{
    f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};   // NaN where a sum is inf or NaN
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            zero[e] = __builtin_fmaf(acc[t][e], 0.0f, zero[e]);
    const bool beyond = (zero[0] + zero[1]) + (zero[2] + zero[3]) != 0.0f;
    return __builtin_expect(__ballot(beyond) != 0, false);
}

// A sum without its scale can leave fp32 where their product would not: it has up to 128 terms of
// up to 6 |x| (one of |x| = 1e38 does, or 128 of 1e36).  A tile's sums (of 16 rows from m0 on,
// blocks kb, kb + step, ..) that are not finite are formed again from the codes' values times
// kSmall, with which no sum of finite terms leaves fp32.  The others stay as they are: inputs below
// 2^-116 would lose bits by kSmall.  (Finite sums pay for the look at them: 0.6% over 84 sizes.)
constexpr float kSmall = 0x1p-10f;
static_assert(128 * 6 * kSmall < 1.0f, "");

template <typename E, int SG>
__device__ __forceinline__ f32x4 mended(const Fp4Args& a, int64_t g, int64_t m0, int64_t tile,
                                        int64_t kb, int step, int lane, f32x4 acc)
{
    constexpr int CH = kChunk<E>, P = kParts<E>, PER = 128 / SG;
    asm volatile("" : "+v"(lane));   // (no address of the loops before is kept for this one)
    const int r = lane & 15, h = lane >> 4;
    tile = tile < a.tiles ? tile : a.tiles - 1;
    const int64_t first = (g * a.tiles + tile) * a.blocks_k, row = m0 + r < a.M ? m0 + r : a.M - 1;
    const E* x = (const E*)a.x.p + g * a.x.gs + row * a.x.ld;
    f32x4 again = {0.0f, 0.0f, 0.0f, 0.0f}, sum = again;
    for (; kb < a.blocks_k; kb += step) {
        const u32x4 codes = *(const u32x4*)(a.codes + (first + kb) * 1024 + lane * 16);
        uint32_t scales[(PER + 1) / 2];
        load_scales<PER>(a.scales + ((first + kb) * 16 + r) * PER, scales);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4 raw[8 / CH];
#pragma unroll
            for (int q = 0; q < 8; q += CH) {
                const int64_t k = kb * 128 + j * 32 + h * 8 + q, left = a.K - k;
                raw[q / CH] = left > 0 ? load_chunk(x + k, left < CH ? (int)left : CH, k)
                                       : u32x4{0, 0, 0, 0};
            }
            bf16x8 xp[P];
            split_parts<E>(raw, xp);
            const bf16x8 w = __builtin_bit_cast(bf16x8, code_values(codes[j], kSmall));
            if (j * 32 % SG == 0)
                sum = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int p = P - 1; p >= 0; --p)
                sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xp[p], w, sum, 0, 0, 0);
            if ((j * 32 + 32) % SG == 0) {
                const float s =
                    scale_of<PER>(scales, j * 32 / SG, kb * 128 + j * 32 / SG * SG < a.K);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    again[e] = __builtin_fmaf(sum[e] * s, 1.0f / kSmall, again[e]);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        acc[e] = acc[e] - acc[e] != 0.0f ? again[e] : acc[e];
    return acc;
}

// A wavefront takes 16 rows of x, 16 NT outputs and a share of the blocks of 128 inputs, straight
// from memory to registers, a block ahead of the products.  WK = 8: a workgroup's wavefronts
// share the inputs, and their sums are added through LDS in their order; WK = 1 (few blocks of
// inputs): each has outputs of its own.  Rows and outputs that do not exist repeat the last
// row, or use the padding's codes: their results are not written.  One row is bound by the read
// of the codes: 8192 -> 8192 bf16, groups of 32, 37.7 MB, 8.4 us, 4.5 TB/s.
constexpr int kWaves = 8;

template <typename E, int SG, int NT, int WK>
__global__ __launch_bounds__(kWaves * 64) void linear_fp4_kernel(Fp4Args a)
{
    constexpr int CH = kChunk<E>, P = kParts<E>, PER = 128 / SG;
    const int lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t g = a.first_group + blockIdx.z;
    const int64_t m0 = (int64_t)blockIdx.y * 16;
    const int64_t t0 = (WK == 1 ? (int64_t)blockIdx.x * kWaves + wave : blockIdx.x) * NT;
    const int share = WK == 1 ? 0 : wave;
    if (WK == 1 && t0 >= a.tiles)
        return;
    const uint8_t* codes[NT];
    const uint16_t* scales[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t tile = t0 + t < a.tiles ? t0 + t : a.tiles - 1;
        const int64_t first = (g * a.tiles + tile) * a.blocks_k;
        codes[t] = a.codes + first * 1024 + lane * 16;
        scales[t] = a.scales + (first * 16 + r) * PER;
    }
    const int64_t row = m0 + r < a.M ? m0 + r : a.M - 1;
    const E* x = (const E*)a.x.p + g * a.x.gs + row * a.x.ld + h * 8;
    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
        acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    struct Block {
        u32x4 c[NT];
        uint32_t s[NT][(PER + 1) / 2];   // two scales each
        u32x4 raw[4][8 / CH];
    };
    auto load = [&](Block& b, int64_t kb, bool whole) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            b.c[t] = *(const u32x4*)(codes[t] + kb * 1024);
            load_scales<PER>(scales[t] + kb * 16 * PER, b.s[t]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int q = 0; q < 8; q += CH) {
                const int64_t k = kb * 128 + j * 32 + q;
                if (whole) {
                    b.raw[j][q / CH] = *(const u32x4_any*)(x + k);
                } else {
                    const int64_t left = a.K - k - h * 8;
                    b.raw[j][q / CH] = u32x4{0, 0, 0, 0};
                    if (left > 0)
                        b.raw[j][q / CH] =
                            load_chunk(x + k, left < CH ? (int)left : CH, k + h * 8);
                }
            }
    };
    auto multiply = [&](const Block& b, int64_t kb, bool whole) {
        f32x4 sum[NT];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x8 xp[P];
            split_parts<E>(b.raw[j], xp);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const bf16x8 w = __builtin_bit_cast(bf16x8, code_values(b.c[t][j]));
                const float s = scale_of<PER>(b.s[t], j * 32 / SG,
                                              whole || kb * 128 + j * 32 / SG * SG < a.K);
                if (j * 32 % SG == 0)
                    sum[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int p = P - 1; p >= 0; --p)
                    sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xp[p], w, sum[t], 0, 0, 0);
                if ((j * 32 + 32) % SG == 0) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[t][e] = __builtin_fmaf(sum[t][e], s, acc[t][e]);
                }
            }
        }
    };
    const int64_t whole = a.K / 128;
    int64_t kb = share;
    if (kb < whole) {
        Block now, next;
        load(now, kb, true);
        for (; kb + WK < whole; kb += WK) {
            load(next, kb + WK, true);
            multiply(now, kb, true);
            now = next;
        }
        multiply(now, kb, true);
        kb += WK;
    }
    if (kb < a.blocks_k) {
        Block b;
        load(b, kb, false);
        multiply(b, kb, false);
    }
    // lane: output r of a tile, its rows 4 h .. 4 h + 3
    const bool beyond = beyond_fp32(acc);
    if constexpr (WK == 1) {
        if (beyond) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
                acc[t] = mended<E, SG>(a, g, m0, t0 + t, share, WK, lane, acc[t]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
            finish_tile<E, 1>(a, g, m0 + 4 * h, (t0 + t) * 16 + r, &acc[t], 0);
    } else {
        __shared__ f32x4 part[kWaves][NT][64];
#pragma unroll
        for (int t = 0; t < NT; ++t)
            part[wave][t][lane] = acc[t];
        if (beyond) {
            for (int t = 0; t < NT; ++t)
                part[wave][t][lane] =
                    mended<E, SG>(a, g, m0, t0 + t, share, WK, lane, part[wave][t][lane]);
        }
        __syncthreads();
        if (wave < NT)
            finish_tile<E, kWaves>(a, g, m0 + 4 * h, (t0 + wave) * 16 + r, &part[0][wave][lane],
                                   NT * 64);
    }
}

// More rows, bf16: a workgroup takes 32 rows and 64 outputs.  Rows go through LDS, a wavefront's
// own 32 x 128 at a time (whole lines of memory, where a 16-row operand takes half ones);
// 16-byte chunk c of row m lies at c ^ (m mod 16), so that a wavefront's reads of one
// operand fall into different banks.  192 x 4096 -> 4096 13.8 us, 0.47 PFLOP/s: the matrix cores
// are busy an eighth of the time, the rest goes to codes (taken apart again for every 32
// rows), scales and the way through LDS.
constexpr int kTallWaves = 4, kTallRows = 32, kTallTiles = 4;

template <int SG>
__global__ __launch_bounds__(kTallWaves * 64, SG == 64 ? 1 : 2) void tall_fp4_kernel(Fp4Args a)
{
    constexpr int NT = kTallTiles, MT = kTallRows / 16, PER = 128 / SG, IN = kTallRows / 4;
    const int lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t g = a.first_group + blockIdx.z;
    const int64_t m0 = (int64_t)blockIdx.y * kTallRows, t0 = (int64_t)blockIdx.x * NT;
    __shared__ u32x4 lds[kTallWaves][kTallRows * 16];
    u32x4* staged = lds[wave];
    const uint8_t* codes[NT];
    const uint16_t* scales[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t tile = t0 + t < a.tiles ? t0 + t : a.tiles - 1;
        const int64_t first = (g * a.tiles + tile) * a.blocks_k;
        codes[t] = a.codes + first * 1024 + lane * 16;
        scales[t] = a.scales + (first * 16 + r) * PER;
    }
    // on the way to LDS a lane has chunk r of rows 4 i + h
    const bf16_t* x[IN];
#pragma unroll
    for (int i = 0; i < IN; ++i) {
        const int64_t m = m0 + 4 * i + h;
        x[i] = (const bf16_t*)a.x.p + g * a.x.gs + (m < a.M ? m : a.M - 1) * a.x.ld + r * 8;
    }
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
            acc[i][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    struct Block {
        u32x4 c[NT], raw[IN];
        uint32_t s[NT][(PER + 1) / 2];
    };
    auto load = [&](Block& b, int64_t kb, auto whole) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            b.c[t] = *(const u32x4*)(codes[t] + kb * 1024);
            load_scales<PER>(scales[t] + kb * 16 * PER, b.s[t]);
        }
        if constexpr (whole()) {
#pragma unroll
            for (int i = 0; i < IN; ++i)
                b.raw[i] = *(const u32x4_any*)(x[i] + kb * 128);
        } else {
            const int64_t left = a.K - kb * 128 - r * 8;
#pragma unroll
            for (int i = 0; i < IN; ++i)
                b.raw[i] = left > 0 ? load_chunk(x[i] + kb * 128, left < 8 ? (int)left : 8,
                                                 kb * 128 + r * 8)
                                    : u32x4{0, 0, 0, 0};
        }
    };
    using Whole = std::true_type;
    using Short = std::false_type;
    // `b` holds block kb; block `next` (whole) takes its place
    auto step = [&](Block& b, int64_t kb, int64_t next, auto whole, auto more) {
        wave_lds_sync();   // (the last block's operands have been read)
#pragma unroll
        for (int i = 0; i < IN; ++i) {
            const int m = 4 * i + h;
            staged[m * 16 + (r ^ (m & 15))] = b.raw[i];
        }
        wave_lds_sync();
        u32x4 c[NT];
        uint32_t s[NT][(PER + 1) / 2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            c[t] = b.c[t];
#pragma unroll
            for (int i = 0; i < (PER + 1) / 2; ++i)
                s[t][i] = b.s[t][i];
        }
        if constexpr (more())
            load(b, next, Whole());
        f32x4 sum[MT][NT];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x8 xp[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i)
                xp[i] = __builtin_bit_cast(bf16x8, staged[(i * 16 + r) * 16 + ((j * 4 + h) ^ r)]);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const bf16x8 w = __builtin_bit_cast(bf16x8, code_values(c[t][j]));
                const float sc = scale_of<PER>(s[t], j * 32 / SG,
                                               whole() || kb * 128 + j * 32 / SG * SG < a.K);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if (j * 32 % SG == 0)
                        sum[i][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                    sum[i][t] =
                        __builtin_amdgcn_mfma_f32_16x16x32_bf16(xp[i], w, sum[i][t], 0, 0, 0);
                    if ((j * 32 + 32) % SG == 0) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[i][t][e] = __builtin_fmaf(sum[i][t][e], sc, acc[i][t][e]);
                    }
                }
            }
        }
    };
    // whole blocks, two ahead (behind the last one it is loaded again), then the short one
    const int64_t whole = a.K / 128, last = whole - 1;
    int64_t kb = wave;
    if (kb < whole) {
        Block even, odd;
        load(even, kb, Whole());
        load(odd, kb + kTallWaves < whole ? kb + kTallWaves : last, Whole());
        for (; kb + kTallWaves < whole; kb += 2 * kTallWaves) {
            const int64_t n0 = kb + 2 * kTallWaves, n1 = n0 + kTallWaves;
            step(even, kb, n0 < whole ? n0 : last, Whole(), Whole());
            step(odd, kb + kTallWaves, n1 < whole ? n1 : last, Whole(), Whole());
        }
        if (kb < whole) {
            step(even, kb, 0, Whole(), Short());
            kb += kTallWaves;
        }
    }
    if (kb == whole && whole < a.blocks_k) {
        Block b;
        load(b, kb, Short());
        step(b, kb, 0, Short(), Short());
    }
    static_assert(MT == 2, "");
    static_assert(sizeof lds == sizeof(f32x4) * kTallWaves * MT * NT * 64, "");
    f32x4* part = (f32x4*)lds;   // [wavefront][tile][lane], each wavefront's over its own rows
    wave_lds_sync();
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
            part[(wave * MT * NT + i * NT + t) * 64 + lane] = acc[i][t];
    if (beyond_fp32(acc[0]) || beyond_fp32(acc[1])) {
        for (int q = 0; q < MT * NT; ++q) {
            f32x4& sums = part[(wave * MT * NT + q) * 64 + lane];
            sums = mended<bf16_t, SG>(a, g, m0 + q / NT * 16, t0 + q % NT, wave, kTallWaves, lane,
                                      sums);
        }
    }
    __syncthreads();
    for (int q = wave; q < MT * NT; q += kTallWaves)
        finish_tile<bf16_t, kTallWaves>(a, g, m0 + q / NT * 16 + 4 * h, (t0 + q % NT) * 16 + r,
                                        part + q * 64 + lane, MT * NT * 64);
}

template <typename E, int NT, int WK>
void launch_tiles(const Fp4Args& a, dim3 grid, hipStream_t s)
{
    if (a.scale_group == 32)
        linear_fp4_kernel<E, 32, NT, WK><<<grid, kWaves * 64, 0, s>>>(a);
    else if (a.scale_group == 64)
        linear_fp4_kernel<E, 64, NT, WK><<<grid, kWaves * 64, 0, s>>>(a);
    else
        linear_fp4_kernel<E, 128, NT, WK><<<grid, kWaves * 64, 0, s>>>(a);
}

void launch_tall(const Fp4Args& a, dim3 grid, hipStream_t s)
{
    if (a.scale_group == 32)
        tall_fp4_kernel<32><<<grid, kTallWaves * 64, 0, s>>>(a);
    else if (a.scale_group == 64)
        tall_fp4_kernel<64><<<grid, kTallWaves * 64, 0, s>>>(a);
    else
        tall_fp4_kernel<128><<<grid, kTallWaves * 64, 0, s>>>(a);
}

template <typename E>
hipError_t launch_linear_as(Fp4Args a, const Fp4Plan& p, hipStream_t s)
{
    // at most 2^22 workgroups a launch (and 65535 blocks of rows)
    constexpr int64_t kMost = (int64_t)1 << 22;
    const int64_t nt = (a.tiles + p.tiles * p.apart - 1) / (p.tiles * p.apart);
    const int64_t groups = std::max<int64_t>(1, std::min<int64_t>(a.groups, kMost / nt));
    const int64_t per =
        std::max<int64_t>(1, std::min<int64_t>(65535, kMost / (nt * groups))) * 16 * p.rows;
    const int64_t es = sizeof(E);
    for (int64_t m = 0; m < a.M; m += per) {
        Fp4Args b = a;
        b.M = (int)std::min<int64_t>(per, a.M - m);
        b.x.p = (const char*)a.x.p + m * a.x.ld * es;
        b.y.p = (const char*)a.y.p + m * a.y.ld * es;
        if (a.res.p)
            b.res.p = (const char*)a.res.p + m * a.res.ld * es;
        for (int64_t g = 0; g < a.groups; g += groups) {
            b.first_group = (int)g;
            const dim3 grid((unsigned)nt, (unsigned)((b.M + 16 * p.rows - 1) / (16 * p.rows)),
                            (unsigned)std::min<int64_t>(groups, a.groups - g));
            if (p.rows == 2)
                launch_tall(b, grid, s);
            else if (p.apart > 1 && p.tiles == 4)
                launch_tiles<E, 4, 1>(b, grid, s);
            else if (p.apart > 1)
                launch_tiles<E, 1, 1>(b, grid, s);
            else if (p.tiles == 4)
                launch_tiles<E, 4, kWaves>(b, grid, s);
            else if (p.tiles == 2)
                launch_tiles<E, 2, kWaves>(b, grid, s);
            else
                launch_tiles<E, 1, kWaves>(b, grid, s);
        }
    }
    return hipGetLastError();
}

template <typename F>
hipError_t launch_pack(const Fp4Args& a, F kernel, hipStream_t s)
{
    const int64_t n = (int64_t)a.groups * a.tiles * a.blocks_k;
    const unsigned nb = (unsigned)std::min<int64_t>((int64_t)1 << 20, (n + 3) / 4);
    kernel<<<nb, kPackThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

// bf16 rows through LDS against straight to registers (us, groups of 128 and of 32 weights): 96
// rows x 4096 -> 4096 9.4 and 13.6, 15.6 and 14.6; 128 rows x 8192 -> 8192 25.4 and 44.2, 37.9
// and 48.8; 256 x 512 -> 16384 15.7 and 25.5, 18.8 and 22.8; but 48 x 4096 -> 4096 9.8 and 8.1,
// 15.5 and 9.0, and with few workgroups 256 x 16384 -> 512 23.9 and 21.1, 43.8 and 24.8, 112 x
// 11504 -> 1856 41 and 19 (groups of 32).  Straight to registers, as many tiles as leave a
// workgroup for most CUs: 1 row x 8192 -> 8192 with 1, 2, 4 tiles 9.1, 8.5, 11.0; 16 rows 19.2,
// 12.5, 14.6; 32 rows 34.8, 21.8, 15.3.  Wavefronts with outputs of their own where there is one
// block of inputs: 21 x 58 x 112 -> 2624 fp32 12 and 41; with four 16 x 512 -> 512 bf16 6.4 and
// 3.5.
constexpr int64_t kApartMost = 128;
Fp4Plan fp4_plan(int64_t groups, int64_t M, int64_t N, int64_t K, int size)
{
    constexpr int64_t kFill = 192;   // workgroups
    Fp4Plan p{};
    p.tiles = 4;
    p.rows = p.apart = 1;
    const int64_t tiles = (N + 15) / 16, blocks = (M + 15) / 16 * groups;
    if (size == 2 && M > 64 && K >= 512 &&
        (tiles + 3) / 4 * ((M + kTallRows - 1) / kTallRows) * groups >= kFill) {
        p.rows = kTallRows / 16;
    } else if (K <= kApartMost) {
        p.apart = kWaves;
        if ((tiles + 4 * kWaves - 1) / (4 * kWaves) * blocks < kFill)
            p.tiles = 1;
    } else {
        while (p.tiles > 1 && (tiles + p.tiles - 1) / p.tiles * blocks < kFill)
            p.tiles /= 2;
    }
    return p;
}

hipError_t launch_quantize_fp4(const Fp4Args& a, int dtype, hipStream_t s)
{
    return dtype == MALIB_DT_BF16 ? launch_pack(a, quantize_kernel<bf16_t>, s)
                                  : launch_pack(a, quantize_kernel<float>, s);
}

hipError_t launch_dequantize_fp4(const Fp4Args& a, int dtype, hipStream_t s)
{
    return dtype == MALIB_DT_BF16 ? launch_pack(a, dequantize_kernel<bf16_t>, s)
                                  : launch_pack(a, dequantize_kernel<float>, s);
}

hipError_t launch_linear_fp4(Fp4Args a, int dtype, const Fp4Plan& p, hipStream_t s)
{
    return dtype == MALIB_DT_BF16 ? launch_linear_as<bf16_t>(a, p, s)
                                  : launch_linear_as<float>(a, p, s);
}

}  // namespace malib
