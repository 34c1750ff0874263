// Dropout from the library's random stream: y = x k / q + residual, the mask formed again
// wherever it is needed.
//
// A thread takes 16 consecutive values (in the matrix's own order, whatever its
// strides), which share one block of the stream: 16 bits each.  Bound by memory: with 32 bits
// a value the stream's 64-bit products would take longer than the values' transfer.
// 131072 x 512 bf16 with a residual, 402 MB: 68 us, 5.9 TB/s (two thirds of it are reads, which
// are faster than a copy).  5003 x 777 fp32, rows apart, 31 MB: 9 us, 3.5 TB/s.
#include "internal.hpp"

#include "chunk.hpp"
#include "device.hpp"

namespace malib {

namespace {

constexpr int kThreads = 256, kRun = 16;   // values per block of the stream

// i / cols for i < 2^55 and a quotient below 2^31: the product with 1 / cols is off by less than
// one
__device__ __forceinline__ uint32_t row_of(int64_t i, int64_t cols, double inv, int64_t& col)
{
    uint32_t q = (uint32_t)((double)i * inv);
    col = i - (int64_t)q * cols;
    if (col < 0) {
        --q;
        col += cols;
    } else if (col >= cols) {
        ++q;
        col -= cols;
    }
    return q;
}

template <typename E>
__device__ __forceinline__ E dropped(const DropoutArgs& a, E x, const E* residual, uint32_t bits)
{
    float v = bits >= a.drop ? to_f32(x) * a.scale : 0.0f;
    if (residual)
        v += to_f32(*residual);
    return from_f32<E>(v);
}

// FLAT: x, residual and y have no gaps between their rows.  Runs across a row's end (and the
// matrix's) are written value by value, four runs at a time by the whole wavefront: a lane on
// its own took 16 values' loads for all of its wavefront (65536 x 777 bf16, rows apart,
// 79 us).
template <typename E, bool FLAT>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutArgs a)
{
    constexpr int CH = kChunk<E>, NC = kRun / CH;
    const int64_t n = a.rows * a.cols, runs = (n + kRun - 1) / kRun;
    const uint64_t step = a.step + (a.device_step ? (uint64_t)*a.device_step : 0);
    const E *x = (const E*)a.x, *res = (const E*)a.residual;
    E* y = (E*)a.y;
    const int lane = threadIdx.x & 63;
    // (a wavefront's lanes stay together)
    for (int64_t b0 = (int64_t)blockIdx.x * kThreads + (threadIdx.x & ~63); b0 < runs;
         b0 += (int64_t)gridDim.x * kThreads) {
        const int64_t b = b0 + lane, i = b * kRun;
        int64_t row = 0, col = i;
        if (!FLAT)
            row = row_of(i, a.cols, a.inv_cols, col);
        const bool whole = i + kRun <= n && (FLAT || col + kRun <= a.cols);
        const int64_t px = FLAT ? i : row * a.x_ld + col, py = FLAT ? i : row * a.y_ld + col;
        const int64_t pr = FLAT ? i : row * a.residual_ld + col;
        u32x4 cx[NC], cr[NC];
        if (whole) {
#pragma unroll
            for (int q = 0; q < NC; ++q)
                cx[q] = *(const u32x4_any*)(x + px + q * CH);
            if (res) {
#pragma unroll
                for (int q = 0; q < NC; ++q)
                    cr[q] = *(const u32x4_any*)(res + pr + q * CH);
            }
        }
        const u64x4 bits = stream_block(a.seed, (uint64_t)b, step, kPurposeDropout, a.layer, 0);
        if (whole) {
#pragma unroll
            for (int q = 0; q < NC; ++q) {
                float f[CH], g[CH];
                unpack<E>(cx[q], f);
                if (res)
                    unpack<E>(cr[q], g);
#pragma unroll
                for (int e = 0; e < CH; ++e) {
                    const int at = q * CH + e;
                    const uint32_t u = block_lane(bits, at / 2) >> (16 * (at % 2)) & 0xFFFFu;
                    f[e] = u >= a.drop ? f[e] * a.scale : 0.0f;
                    if (res)
                        f[e] += g[e];
                }
                *(u32x4_any*)(y + py + q * CH) = pack<E>(f);
            }
        }
        uint64_t rest = __ballot(!whole && i < n);
        if (rest == 0)
            continue;
        // value e of its run: bits 16 (e % 4) up of word e / 4
        const int e = lane & 15;
        while (rest) {
            int from = -1;   // the lane whose run these 16 lanes take
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (rest) {
                    const int who = __builtin_ctzll(rest);
                    rest &= rest - 1;
                    from = lane >> 4 == q ? who : from;
                }
            }
            const int src = from < 0 ? 0 : from;
            uint32_t u = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                const uint32_t v = (uint32_t)__shfl((int)block_lane(bits, w), src);
                u = e / 2 == w ? v : u;
            }
            u = e % 2 ? u >> 16 : u & 0xFFFFu;
            const int64_t at = (b0 + src) * kRun + e;
            if (from >= 0 && at < n) {
                int64_t rr = 0, cc = at;
                if (!FLAT)
                    rr = row_of(at, a.cols, a.inv_cols, cc);
                y[FLAT ? at : rr * a.y_ld + cc] =
                    dropped(a, x[FLAT ? at : rr * a.x_ld + cc],
                            res ? res + (FLAT ? at : rr * a.residual_ld + cc) : nullptr, u);
            }
        }
    }
}

template <typename E>
hipError_t launch_as(DropoutArgs a, hipStream_t s)
{
    a.inv_cols = 1.0 / (double)a.cols;
    const int64_t runs = (a.rows * a.cols + kRun - 1) / kRun;
    const unsigned nb =
        (unsigned)std::min<int64_t>((int64_t)1 << 22, (runs + kThreads - 1) / kThreads);
    const bool flat = a.rows == 1 || (a.x_ld == a.cols && a.y_ld == a.cols &&
                                      (!a.residual || a.residual_ld == a.cols));
    if (flat)
        dropout_kernel<E, true><<<nb, kThreads, 0, s>>>(a);
    else
        dropout_kernel<E, false><<<nb, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, int dtype, hipStream_t s)
{
    return dtype == MALIB_DT_BF16 ? launch_as<bf16_t>(a, s) : launch_as<float>(a, s);
}

}  // namespace malib
