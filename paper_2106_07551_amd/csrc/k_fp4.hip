// Layers of frozen policies in 4 bits: weights v s, v one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and
// their negatives, s a bf16 scale shared by 32, 64 or 128 weights along the input.
//
// Codes lie in the order of the second operand of 16x16x32 products: a lane of a wavefront
// holds the codes of one output and 32 of 128 inputs in 16 bytes, four products' worth.
// gfx950 turns two codes into bf16 in one instruction, exactly; products with bf16 are exact,
// too, and a scale goes onto the fp32 sum of its weights' products.
#include "internal.hpp"

#include "act.hpp"
#include "chunk.hpp"
#include "device.hpp"

namespace malib {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// The bf16 values of eight codes
__device__ __forceinline__ u32x4 code_values(uint32_t c)
{
    u32x4 v;
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, 1.0f, 0));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, 1.0f, 1));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, 1.0f, 2));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, 1.0f, 3));
    return v;
}

__device__ __forceinline__ float scale_value(uint16_t s)
{
    return __uint_as_float((uint32_t)s << 16);
}

// ------------------------------------------------------------- weights to codes and back

constexpr int kPackThreads = 256;
constexpr float kSixth = 1.0f / 6.0f;   // of the largest magnitude: a group's scale

// A wavefront per block of 16 outputs x 128 inputs; a lane has output lane & 15 and, of
// each 32 inputs, the eight from 8 (lane >> 4) on.
struct BlockOf {
    int64_t g, tile, kb;
    __device__ __forceinline__ BlockOf(const Fp4Args& a, int64_t i)
    {
        kb = i % a.blocks_k;
        tile = i / a.blocks_k % a.tiles;
        g = i / a.blocks_k / a.tiles;
    }
};

// Nearest value's code: the comparisons with the borders between values are exact (a
// border times a bf16 scale fits fp32), ties go to the even code.
__device__ __forceinline__ uint32_t code_of(float w, float s)
{
    const float m = __builtin_fabsf(w);
    uint32_t c = (m > s * 0.25f) + (m >= s * 0.75f) + (m > s * 1.25f) + (m >= s * 1.75f) +
                 (m > s * 2.5f) + (m >= s * 3.5f) + (m > s * 5.0f);
    c = s > 0.0f ? c : 0u;
    return c && w < 0.0f ? c | 8u : c;
}

template <typename E>
__global__ __launch_bounds__(kPackThreads) void quantize_kernel(Fp4Args a)
{
    constexpr int CH = kChunk<E>;
    const int lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int per = 128 / a.scale_group;   // scales of an output in a block
    const int64_t n_blocks = (int64_t)a.groups * a.tiles * a.blocks_k;
    for (int64_t i = (int64_t)blockIdx.x * (kPackThreads / 64) + (threadIdx.x >> 6); i < n_blocks;
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
            const uint16_t s = most[j] >= 0x7F800000u
                                   ? (uint16_t)0x7FC0u
                                   : from_f32<bf16_t>(__uint_as_float(most[j]) * kSixth).b;
            if (j * 32 / a.scale_group == h)
                scale = s;
            uint32_t c = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                c |= code_of(v[j][e], scale_value(s)) << (4 * e);
            codes[j] = c;
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
    for (int64_t i = (int64_t)blockIdx.x * (kPackThreads / 64) + (threadIdx.x >> 6); i < n_blocks;
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
        uint32_t part[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t b[2][3];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t x = raw[i / 2][2 * (i % 2) + e];
                const bool special = (x & 0x7F800000u) == 0x7F800000u;
                const float f = __uint_as_float(x);
                const float hi = __uint_as_float(x & 0xFFFF0000u);
                const float rest = special ? 0.0f : f - hi;
                const uint32_t mid = __float_as_uint(rest) & 0xFFFF0000u;
                b[e][0] = f != f ? 0x7FC00000u : x;
                b[e][1] = mid;
                b[e][2] = __float_as_uint(rest - __uint_as_float(mid));
            }
#pragma unroll
            for (int p = 0; p < 3; ++p)
                part[p][i] = b[0][p] >> 16 | (b[1][p] & 0xFFFF0000u);
        }
#pragma unroll
        for (int p = 0; p < 3; ++p)
            out[p] = __builtin_bit_cast(bf16x8, u32x4{part[p][0], part[p][1], part[p][2],
                                                      part[p][3]});
    }
}

// A workgroup takes 16 MT rows of x and 16 NT outputs, each of its wavefronts a share of the
// blocks of 128 inputs; the shares are added through LDS in their order.  Rows and
// outputs that do not exist repeat the last row, or use the padding's codes: their
// results are not written.
constexpr int kWaves = 8;

template <typename E, int SG, int MT, int NT>
__global__ __launch_bounds__(kWaves * 64) void linear_fp4_kernel(Fp4Args a)
{
    constexpr int CH = kChunk<E>, P = kParts<E>, PER = 128 / SG;
    const int lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t g = a.first_group + blockIdx.z;
    const int64_t m0 = (int64_t)blockIdx.y * 16 * MT;
    const int64_t t0 = (int64_t)blockIdx.x * NT;
    const uint8_t* codes[NT];
    const uint16_t* scales[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t tile = t0 + t < a.tiles ? t0 + t : a.tiles - 1;
        const int64_t first = (g * a.tiles + tile) * a.blocks_k;
        codes[t] = a.codes + first * 1024 + lane * 16;
        scales[t] = a.scales + (first * 16 + r) * PER;
    }
    const E* x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int64_t m = m0 + t * 16 + r;
        x[t] = (const E*)a.x.p + g * a.x.gs + (m < a.M ? m : a.M - 1) * a.x.ld + h * 8;
    }
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto block = [&](int64_t kb, bool whole) {
        u32x4 c[NT];
        float s[NT][PER];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            c[t] = *(const u32x4*)(codes[t] + kb * 1024);
            const uint16_t* p = scales[t] + kb * 16 * PER;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                s[t][i] = whole || kb * 128 + i * SG < a.K ? scale_value(p[i]) : 0.0f;
        }
        u32x4 raw[MT][4][8 / CH];
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int q = 0; q < 8; q += CH) {
                    const int64_t k = kb * 128 + j * 32 + q;
                    if (whole) {
                        raw[t][j][q / CH] = *(const u32x4_any*)(x[t] + k);
                    } else {
                        const int64_t left = a.K - k - h * 8;
                        raw[t][j][q / CH] = u32x4{0, 0, 0, 0};
                        if (left > 0)
                            raw[t][j][q / CH] =
                                load_chunk(x[t] + k, left < CH ? (int)left : CH, k + h * 8);
                    }
                }
        f32x4 sum[MT][NT];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x8 w[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t)
                w[t] = __builtin_bit_cast(bf16x8, code_values(c[t][j]));
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                bf16x8 xp[P];
                split_parts<E>(raw[i][j], xp);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    if (j * 32 % SG == 0)
                        sum[i][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int p = P - 1; p >= 0; --p)
                        sum[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xp[p], w[t], sum[i][t],
                                                                            0, 0, 0);
                    if ((j * 32 + 32) % SG == 0) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[i][t][e] = __builtin_fmaf(sum[i][t][e], s[t][j * 32 / SG],
                                                          acc[i][t][e]);
                    }
                }
            }
        }
    };
    const int64_t whole = a.K / 128;
    int64_t kb = wave;
    for (; kb < whole; kb += kWaves)
        block(kb, true);
    if (kb < a.blocks_k)
        block(kb, false);
    __shared__ f32x4 part[kWaves][MT * NT][64];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            part[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    // lane: output r of a tile, its rows 4 h .. 4 h + 3
    for (int q = wave; q < MT * NT; q += kWaves) {
        const int64_t n = (t0 + q % NT) * 16 + r, m = m0 + q / NT * 16 + 4 * h;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            const f32x4 t = part[i][q][lane];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] += t[e];
        }
        if (n >= a.N)
            continue;
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
                ((E*)const_cast<void*>(a.y.p))[g * a.y.gs + (m + e) * a.y.ld + n] =
                    from_f32<E>(v[e]);
            }
    }
}

template <typename E, int MT, int NT>
void launch_tiles(const Fp4Args& a, dim3 grid, hipStream_t s)
{
    if (a.scale_group == 32)
        linear_fp4_kernel<E, 32, MT, NT><<<grid, kWaves * 64, 0, s>>>(a);
    else if (a.scale_group == 64)
        linear_fp4_kernel<E, 64, MT, NT><<<grid, kWaves * 64, 0, s>>>(a);
    else
        linear_fp4_kernel<E, 128, MT, NT><<<grid, kWaves * 64, 0, s>>>(a);
}

template <typename E>
hipError_t launch_linear_as(Fp4Args a, const Fp4Plan& p, hipStream_t s)
{
    // at most 2^22 workgroups a launch (and 65535 blocks of rows)
    constexpr int64_t kMost = (int64_t)1 << 22;
    const int64_t nt = (a.tiles + p.tiles - 1) / p.tiles;
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
            if (p.rows == 1)
                launch_tiles<E, 1, 1>(b, grid, s);
            else if (p.rows == 2)
                launch_tiles<E, 2, 1>(b, grid, s);
            else
                launch_tiles<E, 4, 1>(b, grid, s);
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

Fp4Plan fp4_plan(int64_t groups, int64_t M, int64_t N, int64_t K, int size)
{
    Fp4Plan p{};
    p.rows = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    p.tiles = 1;
    p.splits = 1;
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
