// Dropout from the library's random stream: y = x k / q + residual, the mask formed again
// wherever it is needed.
//
// A thread takes 16 consecutive values (in the matrix's own order, whatever its
// strides), which share one block of the stream: 16 bits each.  Bound by memory: with 32 bits
// a value the stream's 64-bit products would take longer than the values' transfer.
#include "internal.hpp"

#include "chunk.hpp"
#include "device.hpp"

namespace malib {

namespace {

constexpr int kThreads = 256, kRun = 16;   // values per block of the stream

// FLAT: x, residual and y have no gaps between their rows.
template <typename E, bool FLAT>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutArgs a)
{
    constexpr int CH = kChunk<E>, NC = kRun / CH;
    const int64_t n = a.rows * a.cols, runs = (n + kRun - 1) / kRun;
    const uint64_t step = a.step + (a.device_step ? (uint64_t)*a.device_step : 0);
    const E *x = (const E*)a.x, *res = (const E*)a.residual;
    E* y = (E*)a.y;
    for (int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x; b < runs;
         b += (int64_t)gridDim.x * kThreads) {
        const int64_t i = b * kRun;
        int64_t row = 0, col = i;
        if (!FLAT) {
            row = i / a.cols;
            col = i - row * a.cols;
        }
        const int left = n - i < kRun ? (int)(n - i) : kRun;
        const bool whole = left == kRun && (FLAT || col + kRun <= a.cols);
        const int64_t px = FLAT ? i : row * a.x_ld + col, py = FLAT ? i : row * a.y_ld + col;
        const int64_t pr = FLAT ? i : row * a.residual_ld + col;
        float v[kRun], r[kRun];
#pragma unroll
        for (int e = 0; e < kRun; ++e)
            v[e] = r[e] = 0.0f;
        if (whole) {
            u32x4 cx[NC], cr[NC];
#pragma unroll
            for (int q = 0; q < NC; ++q)
                cx[q] = *(const u32x4_any*)(x + px + q * CH);
            if (res) {
#pragma unroll
                for (int q = 0; q < NC; ++q)
                    cr[q] = *(const u32x4_any*)(res + pr + q * CH);
            }
#pragma unroll
            for (int q = 0; q < NC; ++q) {
                float f[CH];
                unpack<E>(cx[q], f);
#pragma unroll
                for (int e = 0; e < CH; ++e)
                    v[q * CH + e] = f[e];
                if (res) {
                    unpack<E>(cr[q], f);
#pragma unroll
                    for (int e = 0; e < CH; ++e)
                        r[q * CH + e] = f[e];
                }
            }
        } else {   // across a row's end, or the matrix's
            int64_t rr = row, cc = col;
#pragma unroll
            for (int e = 0; e < kRun; ++e) {
                if (e < left) {
                    v[e] = to_f32(x[FLAT ? i + e : rr * a.x_ld + cc]);
                    if (res)
                        r[e] = to_f32(res[FLAT ? i + e : rr * a.residual_ld + cc]);
                }
                if (++cc == a.cols) {
                    cc = 0;
                    ++rr;
                }
            }
        }
        const u64x4 bits = stream_block(a.seed, (uint64_t)b, step, kPurposeDropout, a.layer, 0);
#pragma unroll
        for (int e = 0; e < kRun; ++e) {
            const uint32_t u = block_lane(bits, e / 2) >> (16 * (e % 2)) & 0xFFFFu;
            v[e] = u >= a.drop ? v[e] * a.scale : 0.0f;
            if (res)
                v[e] += r[e];
        }
        if (whole) {
#pragma unroll
            for (int q = 0; q < NC; ++q) {
                float f[CH];
#pragma unroll
                for (int e = 0; e < CH; ++e)
                    f[e] = v[q * CH + e];
                *(u32x4_any*)(y + py + q * CH) = pack<E>(f);
            }
        } else {
            int64_t rr = row, cc = col;
#pragma unroll
            for (int e = 0; e < kRun; ++e) {
                if (e < left)
                    y[FLAT ? i + e : rr * a.y_ld + cc] = from_f32<E>(v[e]);
                if (++cc == a.cols) {
                    cc = 0;
                    ++rr;
                }
            }
        }
    }
}

template <typename E>
hipError_t launch_as(const DropoutArgs& a, hipStream_t s)
{
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
