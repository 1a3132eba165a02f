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

// Products on the matrix cores, 16 rows of W by 16 NT rows of x per wavefront.  A
// workgroup's 16 wavefronts take 16 / S tiles, S of them a part of the columns each,
// and add their sums at the end.  Symbols become operands two at a time: a byte
// selects its pair of values from a table of all 256 pairs in LDS, one dword each,
// held in 64 copies so that every lane reads its own bank; the address is one byte
// permutation (the byte above the lane's four).  A block's sums (fp32, exact
// products) are multiplied by the scales of their rows as they leave the matrix
// cores, STEP products of 32 columns at a time.
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMW = 16, kMT = 64 * kMW;

template <int DT>
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (DT == 1)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, a),
                                                      __builtin_bit_cast(h16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a),
                                                       __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
}

// The rows' scales of one tile and group for a lane's four results.
template <int DT>
__device__ __forceinline__ f32x4 scales4(uint2 w) {
    return f32x4{from16<DT>(w.x & 0xFFFFu), from16<DT>(w.x >> 16), from16<DT>(w.y & 0xFFFFu),
                 from16<DT>(w.y >> 16)};
}

struct MatvecArgs {
    const char* packed;
    const uint16_t* x;
    uint16_t* y;
    int64_t x_stride, n_out, tiles, scales_at;
    int32_t n_in, m, blocks, groups;
    int32_t unit, unit_shift;  // a group's products of 32 STEP columns; its log2, -1 if none
    int32_t split_shift;       // log2 of S
};

template <int DT, int NT, int STEP>
__global__ __launch_bounds__(kMT) void k_matvec(MatvecArgs p) {
    __shared__ __align__(256) char lds[65536];
    const int lane = threadIdx.x % 64, n16 = lane % 16, g = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int S = 1 << p.split_shift, part = wave & (S - 1);
    const int64_t tile = (int64_t)blockIdx.x * (kMW >> p.split_shift) + (wave >> p.split_shift);
    const int32_t t0 = blockIdx.y * (16 * NT);
    const bool live = tile < p.tiles;
    const int32_t b0 = (int32_t)((int64_t)p.blocks * part >> p.split_shift);
    const int32_t b1 = live ? (int32_t)((int64_t)p.blocks * (part + 1) >> p.split_shift) : b0;
    const int32_t whole = p.n_in / 128 < b1 ? p.n_in / 128 : b1;  // blocks without padding

    const char* words = p.packed + kWHead + (tile * p.blocks + b0) * 1024 + lane * 16;
    const char* scales = p.packed + p.scales_at + tile * p.groups * 32 + g * 8;
    u32x4 next = {0u, 0u, 0u, 0u};
    if (b0 < b1) next = *reinterpret_cast<const u32x4*>(words);

    {  // the table: pair e, copy k at 256 e + 4 k
        const uint16_t* cb = reinterpret_cast<const uint16_t*>(p.packed);
        const uint32_t lo = cb[threadIdx.x / 16 % 16];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t v = lo | (uint32_t)cb[4 * i + threadIdx.x / 256] << 16;
            *reinterpret_cast<u32x4*>(lds + i * 16384 + threadIdx.x * 16) = u32x4{v, v, v, v};
        }
    }
    const uint16_t* xs[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const int32_t r = t0 + 16 * t + n16;
        xs[t] = p.x + (int64_t)(r < p.m ? r : p.m - 1) * p.x_stride + 8 * g;
    }
    f32x4 total[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) total[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    __syncthreads();

    const uint32_t at = 4 * lane;
    auto operand = [&](uint32_t w) {  // eight symbols
        u32x4 a;
#pragma unroll
        for (int k = 0; k < 4; k++)
            a[k] = *reinterpret_cast<const uint32_t*>(
                lds + __builtin_amdgcn_perm(w, at, 0x0C0C0000u | (uint32_t)(4 + k) << 8));
        return a;
    };
    auto group_of = [&](int32_t u) {  // of unit u of 32 STEP columns
        return p.unit_shift >= 0 ? u >> p.unit_shift : u / p.unit;
    };

    for (int32_t b = b0; b < whole; b++) {
        const u32x4 now = next;
        words += 1024;
        if (b + 1 < b1) next = *reinterpret_cast<const u32x4*>(words);
        uint2 sw[4 / STEP];
#pragma unroll
        for (int u = 0; u < 4 / STEP; u++)
            sw[u] = *reinterpret_cast<const uint2*>(
                scales + (int64_t)group_of(b * (4 / STEP) + u) * 32);
        u32x4 xv[NT][4];
#pragma unroll
        for (int t = 0; t < NT; t++)
#pragma unroll
            for (int j = 0; j < 4; j++)
                __builtin_memcpy(&xv[t][j], xs[t] + (int64_t)b * 128 + 32 * j, 16);
#pragma unroll
        for (int u = 0; u < 4 / STEP; u++) {
            f32x4 sum[NT];
#pragma unroll
            for (int t = 0; t < NT; t++) sum[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = u * STEP; j < (u + 1) * STEP; j++) {
                const u32x4 a = operand(now[j]);
#pragma unroll
                for (int t = 0; t < NT; t++) sum[t] = mfma<DT>(a, xv[t][j], sum[t]);
            }
            const f32x4 s = scales4<DT>(sw[u]);
#pragma unroll
            for (int t = 0; t < NT; t++)
#pragma unroll
                for (int r = 0; r < 4; r++)
                    total[t][r] = __builtin_fmaf(s[r], sum[t][r], total[t][r]);
        }
    }
    if (whole < b1 && b0 < b1) {  // the last block, with columns past the matrix: both operands 0 there
        const int32_t i0 = (b1 - 1) * 128;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int32_t i = i0 + 32 * j;
            if (i >= p.n_in) break;
            u32x4 a = operand(next[j]);
#pragma unroll
            for (int k = 0; k < 8; k++)
                if (i + 8 * g + k >= p.n_in) a[k / 2] &= k % 2 ? 0x0000FFFFu : 0xFFFF0000u;
            const f32x4 s = scales4<DT>(*reinterpret_cast<const uint2*>(
                scales + (int64_t)group_of(i / (32 * STEP)) * 32));
#pragma unroll
            for (int t = 0; t < NT; t++) {
                u32x4 xv = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int k = 0; k < 8; k++)
                    if (i + 8 * g + k < p.n_in)
                        xv[k / 2] |= (uint32_t)xs[t][i + k] << (k % 2 * 16);
                const f32x4 sum = mfma<DT>(a, xv, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
                for (int r = 0; r < 4; r++) total[t][r] = __builtin_fmaf(s[r], sum[r], total[t][r]);
            }
        }
    }

    // sums of the S parts in order; result r of lane l of part w at 256 (w NT + t) + 64 r + l
    __syncthreads();
    float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int t = 0; t < NT; t++)
#pragma unroll
        for (int r = 0; r < 4; r++) sums[(wave * NT + t) * 256 + 64 * r + lane] = total[t][r];
    __syncthreads();
    if (!live) return;
    const float* mine = sums + (wave - part) * NT * 256;
    for (int k = part * 64 + lane; k < NT * 256; k += S * 64) {
        const int row = k % 16, col = k / 16 % 16, t = k / 256;
        const float* from = mine + t * 256 + row % 4 * 64 + row / 4 * 16 + col;
        float v = from[0];
        for (int w = 1; w < S; w++) v += from[w * NT * 256];
        const int64_t o = tile * 16 + row;
        const int32_t r = t0 + 16 * t + col;
        if (o < p.n_out && r < p.m) p.y[(int64_t)r * p.n_out + o] = to16<DT>(v);
    }
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

namespace {

template <int DT, int NT>
void matvec_step(const MatvecArgs& a, int step, dim3 g, hipStream_t st) {
    if (step == 4)
        k_matvec<DT, NT, 4><<<g, kMT, 0, st>>>(a);
    else
        k_matvec<DT, NT, 1><<<g, kMT, 0, st>>>(a);
}

template <int DT>
void matvec_rows(const MatvecArgs& a, int nt, int step, dim3 g, hipStream_t st) {
    if (nt == 1)
        matvec_step<DT, 1>(a, step, g, st);
    else if (nt == 2)
        matvec_step<DT, 2>(a, step, g, st);
    else
        matvec_step<DT, 4>(a, step, g, st);
}

}  // namespace

hipError_t launch_matvec(const char* packed, int dt, const Weights& w, const void* x, int64_t m,
                         int64_t x_stride, void* y, hipStream_t st) {
    MatvecArgs a{};
    a.packed = packed;
    a.x = static_cast<const uint16_t*>(x);
    a.y = static_cast<uint16_t*>(y);
    a.x_stride = x_stride;
    a.n_out = w.n_out;
    a.n_in = (int32_t)w.n_in;
    a.m = (int32_t)m;
    a.tiles = w.tiles();
    a.blocks = (int32_t)w.blocks();
    a.groups = (int32_t)w.groups();
    a.scales_at = w.scales_at();
    // scales change at whole blocks of 128 columns, or anywhere between products of 32
    const int step = w.group % 128 == 0 ? 4 : 1;
    a.unit = (int32_t)(w.group / (32 * step));
    a.unit_shift = (a.unit & (a.unit - 1)) == 0 ? __builtin_ctz((unsigned)a.unit) : -1;
    // parts of the columns: until there are 4096 wavefronts, 16 for each CU
    while (a.split_shift < 4 && (a.tiles << a.split_shift) < 4096 &&
           (2 << a.split_shift) <= a.blocks)
        a.split_shift++;
    const int nt = m <= 16 ? 1 : m <= 32 ? 2 : 4;
    const int64_t per = kMW >> a.split_shift;
    const dim3 g((unsigned)((a.tiles + per - 1) / per), (unsigned)((m + 16 * nt - 1) / (16 * nt)));
    if (dt == ECASQ_F16)
        matvec_rows<1>(a, nt, step, g, st);
    else
        matvec_rows<2>(a, nt, step, g, st);
    return hipGetLastError();
}

}  // namespace ecasq
