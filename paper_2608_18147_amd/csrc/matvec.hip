// Products with 4-bit weights: y[r][o] = sum_g s[o][g] sum_{i in g} c[sym[o][i]] x[r][i].
#include "half16.hpp"
#include "serve.hpp"

namespace ecasq {
namespace {

// One dword of symbols, one scale or one codebook value per thread.
template <int DT>
__global__ __launch_bounds__(256) void k_weights_pack(const uint8_t* __restrict__ sym,
                                                      const double* __restrict__ cb, int32_t t,
                                                      const uint16_t* __restrict__ scales,
                                                      Weights w, char* __restrict__ packed) {
    const int64_t nw = w.tiles() * w.blocks() * 256, ns = w.tiles() * w.groups() * 16;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < nw + ns + kWHead / 2;
         at += (int64_t)gridDim.x * 256) {
        if (at < nw) {
            const int l = (int)(at / 4 % 64), j = (int)(at % 4);
            const int64_t block = at / 256;
            const int64_t o = block / w.blocks() * 16 + l % 16;
            const int64_t i0 = block % w.blocks() * 128 + 32 * j + 8 * (l / 16);
            uint32_t v = 0;
            if (o < w.n_out) {
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if (i0 + i < w.n_in) {
                        const uint32_t s = sym[o * w.n_in + i0 + i];
                        v |= (s < (uint32_t)t ? s : (uint32_t)t - 1u) << (4 * i);
                    }
            }
            reinterpret_cast<uint32_t*>(packed + kWHead)[at] = v;
        } else if (at < nw + ns) {
            const int64_t k = at - nw, o = k / 16 / w.groups() * 16 + k % 16;
            reinterpret_cast<uint16_t*>(packed + w.scales_at())[k] =
                o < w.n_out ? scales[o * w.groups() + k / 16 % w.groups()] : (uint16_t)0;
        } else {
            const int64_t k = at - nw - ns;
            reinterpret_cast<uint16_t*>(packed)[k] = k < t ? to16<DT>(cb[k]) : (uint16_t)0;
        }
    }
}

// A wavefront per tile of 16 rows and row of x: lane l takes quarter l / 16 of
// the columns of row l % 16.
template <int DT>
__global__ __launch_bounds__(64) void k_matvec(const char* __restrict__ packed, Weights w,
                                               const uint16_t* __restrict__ x, int64_t x_stride,
                                               uint16_t* __restrict__ y) {
    __shared__ float book[16];
    const int l = threadIdx.x, q = l / 16;
    if (l < 16) book[l] = from16<DT>(reinterpret_cast<const uint16_t*>(packed)[l]);
    __syncthreads();
    const int64_t tile = blockIdx.x;
    x += blockIdx.y * x_stride;
    const uint32_t* words =
        reinterpret_cast<const uint32_t*>(packed + kWHead) + tile * w.blocks() * 256 + l * 4;
    const uint16_t* scales = reinterpret_cast<const uint16_t*>(packed + w.scales_at()) +
                             tile * w.groups() * 16 + l % 16;
    float total = 0.0f;
    for (int64_t b = 0; b < w.blocks(); b++) {
        for (int j = 0; j < 4; j++) {
            const uint32_t v = words[b * 256 + j];
            const int64_t i0 = b * 128 + 32 * j + 8 * q;
            float dot = 0.0f;
            for (int i = 0; i < 8; i++)
                if (i0 + i < w.n_in) dot += book[(v >> (4 * i)) & 15] * from16<DT>(x[i0 + i]);
            const int64_t g = (b * 128 + 32 * j) / w.group;
            if (g < w.groups()) total += dot * from16<DT>(scales[g * 16]);
        }
    }
    total += __shfl_xor(total, 16);
    total += __shfl_xor(total, 32);
    const int64_t o = tile * 16 + l % 16;
    if (q == 0 && o < w.n_out) y[blockIdx.y * w.n_out + o] = to16<DT>(total);
}

}  // namespace

hipError_t launch_weights_pack(const uint8_t* symbols, const double* codebook, int32_t t,
                               const void* scales, int dt, const Weights& w, char* packed,
                               hipStream_t st) {
    const int64_t n = w.bytes() / 4;
    const unsigned g = (unsigned)(n < ((int64_t)1 << 28) ? (n + 255) / 256 : (int64_t)1 << 20);
    const auto* sc = static_cast<const uint16_t*>(scales);
    if (dt == ECASQ_F16)
        k_weights_pack<1><<<g, 256, 0, st>>>(symbols, codebook, t, sc, w, packed);
    else
        k_weights_pack<2><<<g, 256, 0, st>>>(symbols, codebook, t, sc, w, packed);
    return hipGetLastError();
}

hipError_t launch_matvec(const char* packed, int dt, const Weights& w, const void* x, int64_t m,
                         int64_t x_stride, void* y, hipStream_t st) {
    const auto* xs = static_cast<const uint16_t*>(x);
    auto* ys = static_cast<uint16_t*>(y);
    for (int64_t r = 0; r < m; r += 32768) {
        const dim3 g((unsigned)w.tiles(), (unsigned)(m - r < 32768 ? m - r : 32768));
        if (dt == ECASQ_F16)
            k_matvec<1><<<g, 64, 0, st>>>(packed, w, xs + r * x_stride, x_stride,
                                          ys + r * w.n_out);
        else
            k_matvec<2><<<g, 64, 0, st>>>(packed, w, xs + r * x_stride, x_stride,
                                          ys + r * w.n_out);
    }
    return hipGetLastError();
}

}  // namespace ecasq
