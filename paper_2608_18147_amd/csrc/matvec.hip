// Products with 4-bit weights: y[r][o] = sum_g s[o][g] sum_{i in g} c[sym[o][i]] x[r][i].
#include <type_traits>

#include "half16.hpp"
#include "serve.hpp"

namespace ecasq {
namespace {

// Eight symbols' bytes to a dword; a symbol of t or more counts as t - 1.
__device__ __forceinline__ uint32_t pack8(const uint32_t (&b)[2], uint32_t t) {
    // (no carries: a byte's low seven bits plus 128 - t stay below 256)
    const uint32_t add = (0x80u - t) * 0x01010101u;
    const uint32_t over = (((b[0] & 0x7F7F7F7Fu) + add) | b[0] | ((b[1] & 0x7F7F7F7Fu) + add) |
                           b[1]) & 0x80808080u;
    uint32_t v = 0;
    if (over == 0u) {
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const uint32_t two = (b[k] | b[k] >> 4) & 0x00FF00FFu;
            v |= ((two | two >> 8) & 0xFFFFu) << (16 * k);
        }
        return v;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const uint32_t s = b[i / 4] >> (i % 4 * 8) & 0xFFu;
        v |= (s < t ? s : t - 1u) << (4 * i);
    }
    return v;
}

// A wavefront per tile of 16 rows and block of 128 columns, 16 bytes a lane: every line that
// it reads is read whole (28672 x 8192, 356 MB read and written: 265 us with a dword a
// thread and its place by 64-bit divisions, 68 so).  Then a scale or a codebook value a thread.
template <int DT>
__global__ __launch_bounds__(256) void k_weights_pack(const uint8_t* __restrict__ sym,
                                                      const double* __restrict__ cb, int32_t t,
                                                      const uint16_t* __restrict__ scales,
                                                      Weights w, char* __restrict__ packed) {
    const int lane = threadIdx.x % 64;
    const int32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int32_t blocks = (int32_t)w.blocks();
    const int64_t units = w.tiles() * blocks;  // below 2^30
    // What fills up tiles and blocks meets zeros of x and is not to make NaN of them: a
    // symbol whose value is finite (0 if there is none).
    uint32_t pad = 0;
    for (int k = 15; k >= 0; k--)
        if (k < t && __builtin_isfinite(from16<DT>(to16<DT>(cb[k])))) pad = (uint32_t)k;
    for (int32_t u = (int32_t)blockIdx.x * 4 + wave; u < units; u += (int32_t)gridDim.x * 4) {
        const int32_t tile = u / blocks, block = u - tile * blocks;
        const int64_t o = (int64_t)tile * 16 + lane % 16;
        const int32_t i0 = block * 128 + 8 * (lane / 16);
        const uint8_t* from = sym + o * w.n_in + i0;
        uint32_t bytes[4][2];
        if (o < w.n_out && block * 128 + 128 <= w.n_in) {
#pragma unroll
            for (int j = 0; j < 4; j++) __builtin_memcpy(bytes[j], from + 32 * j, 8);
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++) {
                bytes[j][0] = bytes[j][1] = 0u;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    uint32_t s = pad;
                    if (o < w.n_out && i0 + 32 * j + i < w.n_in) s = from[32 * j + i];
                    bytes[j][i / 4] |= s << (i % 4 * 8);
                }
            }
        }
        const uint4 v = {pack8(bytes[0], (uint32_t)t), pack8(bytes[1], (uint32_t)t),
                         pack8(bytes[2], (uint32_t)t), pack8(bytes[3], (uint32_t)t)};
        reinterpret_cast<uint4*>(packed + kWHead)[(int64_t)u * 64 + lane] = v;
    }
    const int64_t ns = w.tiles() * w.groups() * 16;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < ns + kWHead / 2;
         k += (int64_t)gridDim.x * 256) {
        if (k < ns) {
            const int64_t o = k / 16 / w.groups() * 16 + k % 16;
            reinterpret_cast<uint16_t*>(packed + w.scales_at())[k] =
                o < w.n_out ? scales[o * w.groups() + k / 16 % w.groups()] : (uint16_t)0;
        } else {
            const int64_t at = k - ns;
            reinterpret_cast<uint16_t*>(packed)[at] = at < t ? to16<DT>(cb[at]) : (uint16_t)0;
        }
    }
}

// Products on the matrix cores, 16 rows of W (a tile) by up to 16 rows of x.  The
// columns are cut into chunks of 128 NB (NB KB of a tile's symbols); S of a workgroup's
// 16 wavefronts take the chunks of one tile, and go over their tiles with the next
// chunk's symbols always on the way; their sums are added when a tile ends.  Up to
// 8192 columns a wavefront has one chunk and reads its part of x once for all tiles:
// loads return in order, so a wait for x was one for the symbols behind it (28672 x
// 8192, one row of x: 41 us against 30).  Above, it has several; the rows of x are then
// in LDS where they fit (32256 columns for one row, 15872 for two, 10752 for three), or a part of x is
// read again for every `turns` tiles (8192 x 28672, one row: 28 us by the first, 32 by the
// second).
//
// Symbols become operands two at a time: a byte selects its pair of values from a
// table of all 256 pairs in LDS, one dword each, held in 64 copies so that every
// lane reads its own bank; the address is one byte permutation (the byte above the
// lane's four).  Sums (fp32, exact products) are multiplied by the scales of their
// rows as they leave the matrix cores, STEP products of 32 columns at a time.  What a
// row of x gives depends on the matrix alone, not on the other rows.
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

// The scales of a lane's four results, of which lane `u` of each 16 has those of
// product u (32 columns) of the chunk.
template <int DT, int U>
__device__ __forceinline__ f32x4 scales4(uint2 w) {
    const uint32_t x = __builtin_amdgcn_update_dpp(0, (int)w.x, 0x150 + U, 0xF, 0xF, true);
    const uint32_t y = __builtin_amdgcn_update_dpp(0, (int)w.y, 0x150 + U, 0xF, 0xF, true);
    return f32x4{from16<DT>(x & 0xFFFFu), from16<DT>(x >> 16), from16<DT>(y & 0xFFFFu),
                 from16<DT>(y >> 16)};
}

struct MatvecArgs {
    const char* packed;
    const uint16_t* x;
    uint16_t* y;
    int64_t x_stride, n_out, scales_at;
    int32_t n_in, m, tiles, blocks, groups;
    int32_t unit, unit_shift;  // products of 32 columns per group; its log2, -1 if none
    int32_t parts;             // S
    int32_t slots;             // tiles that a workgroup has at a time
    int32_t turns;             // MANY: tiles for which a part of x is kept
    int32_t odd;               // many rows of x, some of which begin between two dwords
};

// Eight entries of a row of x, some of whose rows begin between two dwords (odd, the same for
// all lanes).  Loads that begin there take a lane after the other: the dwords begin an entry
// early then, but for the row's first entry, in front of which nothing may be.
__device__ __forceinline__ u32x4 load8(const uint16_t* p, int32_t odd, bool first) {
    u32x4 v;
    if (!odd || first) {
        __builtin_memcpy(&v, p, 16);
        return v;
    }
    const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(p) & 2u;
    uint32_t w[4];
    __builtin_memcpy(w, __builtin_assume_aligned(reinterpret_cast<const char*>(p) - off, 4), 16);
    const uint32_t last = p[7];
#pragma unroll
    for (int k = 0; k < 4; k++)
        v[k] = __builtin_amdgcn_alignbyte(k < 3 ? w[k + 1] : last, w[k], off);
    return v;
}
constexpr int kTurns = 4, kXBytes = 65536;

// A wavefront has one chunk; or several (then S is 16 and a workgroup has one tile at a
// time), with x in registers or in LDS.
enum Mode { kOne, kMany, kManyLds };

template <int DT, int STEP, int NB, int MODE>
__global__ __launch_bounds__(kMT) void k_matvec(MatvecArgs p) {
    __shared__ __align__(256) char table[65536];
    __shared__ float sums[MODE == kMany ? kTurns : 2][kMW * 256];
    __shared__ __align__(16) char xlds[MODE == kManyLds ? kXBytes : 16];
    const int lane = threadIdx.x % 64, n16 = lane % 16, g = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int S = p.parts, slot = wave / S, part = wave - slot * S;
    const int32_t t0 = blockIdx.y * 16, chunks = (p.blocks + NB - 1) / NB;
    const int32_t turns = MODE == kMany ? p.turns : 1, stride = gridDim.x * p.slots * turns;
    int32_t tile = blockIdx.x * p.slots * turns + slot;
    const bool busy = slot < p.slots && part < chunks;

    // this lane's part of chunk c of tile t (the last tile's for those past it)
    auto words_of = [&](int32_t t, int32_t c, int i) {
        const int64_t row = t < p.tiles ? t : p.tiles - 1;
        const int32_t b = NB * c + i < p.blocks ? NB * c + i : p.blocks - 1;
        return *reinterpret_cast<const u32x4*>(p.packed + kWHead + (row * p.blocks + b) * 1024 +
                                               lane * 16);
    };
    auto scales_of = [&](int32_t t, int32_t c) {
        const int64_t row = t < p.tiles ? t : p.tiles - 1;
        const int32_t u = 4 * NB * c + n16;
        const int32_t k = p.unit_shift >= 0 ? u >> p.unit_shift : u / p.unit;
        uint2 v = {0u, 0u};  // past the matrix, where x is 0 and the symbols' values are finite
        if (k < p.groups)
            v = *reinterpret_cast<const uint2*>(p.packed + p.scales_at +
                                                (row * p.groups + k) * 32 + g * 8);
        return v;
    };
    u32x4 q[NB];
    uint2 scale = {0u, 0u};
    if (busy) {
#pragma unroll
        for (int i = 0; i < NB; i++) q[i] = words_of(tile, part, i);
        scale = scales_of(tile, part);
    }

    // x of chunk c: entries of this lane's row, 0 past the matrix and past the rows
    const bool has = t0 + n16 < p.m;
    const uint16_t* xr = p.x + (int64_t)(has ? t0 + n16 : t0) * p.x_stride + 8 * g;
    u32x4 x[MODE == kManyLds ? 1 : 4 * NB];
    auto read_x = [&](int32_t c) {
        const int32_t i0 = 128 * NB * c, left = p.n_in - i0;
        if (left >= 128 * NB) {
#pragma unroll
            for (int k = 0; k < 4 * NB; k++) {
                x[k] = u32x4{0u, 0u, 0u, 0u};
                if (has) x[k] = load8(xr + i0 + 32 * k, p.odd, i0 + 32 * k == 0);
            }
            return;
        }
        // the product that the matrix ends in, entry by entry
        u32x4 edge = {0u, 0u, 0u, 0u};
        const int32_t e0 = i0 + left / 32 * 32;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const bool in = has && e0 + 8 * g + e < p.n_in;
            const uint32_t v = in ? xr[e0 + e] : 0u;
            edge[e / 2] |= v << (e % 2 * 16);
        }
#pragma unroll
        for (int k = 0; k < 4 * NB; k++) {
            x[k] = u32x4{0u, 0u, 0u, 0u};
            if (32 * (k + 1) <= left) {
                // (several chunks: one in three or more, and the registers are full)
                if (has)
                    x[k] = load8(xr + i0 + 32 * k, MODE == kMany ? 0 : p.odd, i0 + 32 * k == 0);
            } else if (32 * k < left) {
                x[k] = edge;
            }
        }
    };
    if constexpr (MODE == kOne) {
        if (busy) read_x(part);
    }
    const int32_t x_bytes = chunks * 256 * NB + 16;  // of a row in LDS
    const char* x_row = xlds + (has ? n16 * x_bytes : 0) + 16 * g;
    if constexpr (MODE == kManyLds) {
        const int32_t rows = p.m - t0 < 16 ? p.m - t0 : 16, per = chunks * 16 * NB;
        for (int32_t k = threadIdx.x; k < rows * per; k += kMT) {
            const int32_t r = k / per, i = k % per * 8;
            const uint16_t* from = p.x + (int64_t)(t0 + r) * p.x_stride;
            u32x4 v = {0u, 0u, 0u, 0u};
            if (i + 8 <= p.n_in)
                __builtin_memcpy(&v, from + i, 16);
            else
                for (int e = 0; e < 8; e++)
                    if (i + e < p.n_in) v[e / 2] |= (uint32_t)from[i + e] << (e % 2 * 16);
            *reinterpret_cast<u32x4*>(xlds + r * x_bytes + 2 * i) = v;
        }
    }
    {  // the table: pair e, copy k at 256 e + 4 k
        const uint16_t* cb = reinterpret_cast<const uint16_t*>(p.packed);
        const uint32_t lo = cb[threadIdx.x / 16 % 16];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t v = lo | (uint32_t)cb[4 * i + threadIdx.x / 256] << 16;
            *reinterpret_cast<u32x4*>(table + i * 16384 + threadIdx.x * 16) = u32x4{v, v, v, v};
        }
    }
    __syncthreads();

    const uint32_t at = 4 * lane;
    auto operand = [&](uint32_t w) {  // eight symbols
        u32x4 a;
#pragma unroll
        for (int k = 0; k < 4; k++)
            a[k] = *reinterpret_cast<const uint32_t*>(
                table + __builtin_amdgcn_perm(w, at, 0x0C0C0000u | (uint32_t)(4 + k) << 8));
        return a;
    };
    // the symbols q, with the scales `scale`, of chunk c; the next to come are those of tile2, c2
    auto chunk = [&](auto WHOLE, int32_t c, int32_t tile2, int32_t c2) {
        f32x4 total = {0.0f, 0.0f, 0.0f, 0.0f};
        const uint2 scale2 = scales_of(tile2, c2);
        auto block = [&](auto I) {
            constexpr int i = decltype(I)::value;
            if (WHOLE.value || NB * c + i < p.blocks) {
                f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
                auto product = [&](auto J) {
                    constexpr int j = decltype(J)::value;
                    u32x4 v;
                    if constexpr (MODE == kManyLds)
                        v = *reinterpret_cast<const u32x4*>(x_row + 256 * (NB * c + i) + 64 * j);
                    else
                        v = x[4 * i + j];
                    sum = mfma<DT>(operand(q[i][j]), v, sum);
                    if (STEP == 1 || j == 3) {
                        const f32x4 s = scales4<DT, 4 * i + (STEP == 1 ? j : 0)>(scale);
#pragma unroll
                        for (int k = 0; k < 4; k++)
                            total[k] = __builtin_fmaf(s[k], sum[k], total[k]);
                        sum = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                    }
                };
                product(std::integral_constant<int, 0>{});
                product(std::integral_constant<int, 1>{});
                product(std::integral_constant<int, 2>{});
                product(std::integral_constant<int, 3>{});
            }
            q[i] = words_of(tile2, c2, i);
        };
        block(std::integral_constant<int, 0>{});
        if constexpr (NB > 1) block(std::integral_constant<int, 1>{});
        if constexpr (NB > 2) block(std::integral_constant<int, 2>{});
        if constexpr (NB > 3) block(std::integral_constant<int, 3>{});
        scale = scale2;
        return total;
    };
    auto either = [&](int32_t c, int32_t tile2, int32_t c2) {
        return 128 * NB * (c + 1) <= p.n_in ? chunk(std::true_type{}, c, tile2, c2)
                                            : chunk(std::false_type{}, c, tile2, c2);
    };

    // result k of lane l of wavefront w at 256 w + 64 k + l of its tile's sums
    auto finish = [&](const float* mine, int32_t t, int k) {
        const int row = k % 16, col = k / 16;
        const float* from = mine + row % 4 * 64 + row / 4 * 16 + col;
        float v = from[0];
        for (int w = 1; w < S; w++) v += from[w * 256];
        const int64_t o = (int64_t)t * 16 + row;
        if (t < p.tiles && o < p.n_out && t0 + col < p.m)
            p.y[(int64_t)(t0 + col) * p.n_out + o] = to16<DT>(v);
    };
    const int32_t begin = blockIdx.x * p.slots * turns;
    if constexpr (MODE != kMany) {
        int turn = 0;
        for (int32_t first = begin; first < p.tiles; first += stride) {
            if (busy) {
                f32x4 total;
                if constexpr (MODE == kOne)
                    total = either(part, tile + stride, part);
                else
                    for (int32_t c = part; c < chunks; c += kMW) {
                        const bool last = c + kMW >= chunks;
                        const f32x4 v =
                            either(c, last ? tile + stride : tile, last ? part : c + kMW);
                        total = c == part ? v : total + v;
                    }
#pragma unroll
                for (int k = 0; k < 4; k++) sums[turn][wave * 256 + 64 * k + lane] = total[k];
            }
            __syncthreads();
            if (slot < p.slots)
                for (int k = part * 64 + lane; k < 256; k += S * 64)
                    finish(sums[turn] + slot * S * 256, tile, k);
            turn ^= 1;  // (the next sums go where nobody reads)
            tile += stride;
        }
    } else {
        for (int32_t first = begin; first < p.tiles; first += stride) {
            for (int32_t c = part; c < chunks; c += kMW) {
                read_x(c);
                for (int t = 0; t < turns; t++) {
                    const bool end = t + 1 == turns, last = end && c + kMW >= chunks;
                    const f32x4 total = either(c, last ? first + stride : first + (end ? 0 : t + 1),
                                               last ? part : end ? c + kMW : c);
                    float* to = sums[t] + wave * 256 + lane;
#pragma unroll
                    for (int k = 0; k < 4; k++)
                        to[64 * k] = c == part ? total[k] : to[64 * k] + total[k];
                }
            }
            __syncthreads();
            for (int k = threadIdx.x; k < turns * 256; k += kMT)
                finish(sums[k / 256], first + k / 256, k % 256);
            __syncthreads();
        }
    }
}

}  // namespace

hipError_t launch_weights_pack(const uint8_t* symbols, const double* codebook, int32_t t,
                               const void* scales, int dt, const Weights& w, char* packed,
                               hipStream_t st) {
    const int64_t n = (w.tiles() * w.blocks() + 3) / 4;
    const unsigned g = (unsigned)(n < 4096 ? n : 4096);  // twice what is resident at once
    const auto* sc = static_cast<const uint16_t*>(scales);
    if (dt == ECASQ_F16)
        k_weights_pack<1><<<g, 256, 0, st>>>(symbols, codebook, t, sc, w, packed);
    else
        k_weights_pack<2><<<g, 256, 0, st>>>(symbols, codebook, t, sc, w, packed);
    return hipGetLastError();
}

namespace {

template <int NB, int MODE>
void matvec_go(const MatvecArgs& a, int dt, int step, dim3 g, hipStream_t st) {
    if (dt == ECASQ_F16) {
        if (step == 4)
            k_matvec<1, 4, NB, MODE><<<g, kMT, 0, st>>>(a);
        else
            k_matvec<1, 1, NB, MODE><<<g, kMT, 0, st>>>(a);
    } else {
        if (step == 4)
            k_matvec<2, 4, NB, MODE><<<g, kMT, 0, st>>>(a);
        else
            k_matvec<2, 1, NB, MODE><<<g, kMT, 0, st>>>(a);
    }
}

}  // namespace

hipError_t launch_matvec(const char* packed, int dt, const Weights& w, const void* x, int64_t m,
                         int64_t x_stride, void* y, hipStream_t st) {
    MatvecArgs a{};
    a.packed = packed;
    a.x_stride = x_stride;
    a.n_out = w.n_out;
    a.n_in = (int32_t)w.n_in;
    a.tiles = (int32_t)w.tiles();
    a.blocks = (int32_t)w.blocks();
    a.groups = (int32_t)w.groups();
    a.scales_at = w.scales_at();
    a.unit = (int32_t)(w.group / 32);
    a.unit_shift = (a.unit & (a.unit - 1)) == 0 ? __builtin_ctz((unsigned)a.unit) : -1;
    // scales change at whole blocks of 128 columns, or anywhere between products of 32
    const int step = w.group % 128 == 0 ? 4 : 1;

    // A workgroup per CU.  Chunks of nb blocks give every tile S wavefronts and a
    // workgroup 16 / S tiles; a round takes about nb and as much as a block for its end.  Larger
    // chunks where they save a fifth, since the tiles of a workgroup read x each for itself
    // (14336 x 4096 for 16 rows: 14 us with 2 blocks, 17 with 4; 32124 x 1091 for 3: 15 with
    // 1, 11 with 2).
    constexpr int32_t cus = 256;
    int32_t nb = 4, least = INT32_MAX;
    const bool many = a.blocks > 4 * kMW;
    for (int32_t k = 1; !many && k <= 4; k++) {
        const int32_t parts = (a.blocks + k - 1) / k;
        if (parts > kMW) continue;
        const int32_t at_once = cus * (kMW / parts);
        const int32_t cost = (a.tiles + at_once - 1) / at_once * (k + 1);
        if (least == INT32_MAX || 5 * (int64_t)cost < 4 * (int64_t)least) {
            least = cost;
            nb = k;
        }
    }
    a.parts = many ? kMW : (a.blocks + nb - 1) / nb;
    a.slots = (a.tiles + cus - 1) / cus;
    const bool in_lds = many && (m < 16 ? m : 16) * ((a.blocks + 3) / 4 * 1024 + 16) <= kXBytes;
    a.turns = !many || in_lds ? 1 : a.slots < kTurns ? a.slots : kTurns;
    if (a.slots > kMW / a.parts) a.slots = kMW / a.parts;
    const int32_t each = a.slots * a.turns, wgs = (a.tiles + each - 1) / each;
    constexpr int64_t most = (int64_t)1 << 19;  // rows of one launch (its grid's second side)
    for (int64_t r0 = 0; r0 < m; r0 += most) {
        const int64_t rows = m - r0 < most ? m - r0 : most;
        a.x = static_cast<const uint16_t*>(x) + r0 * x_stride;
        // (8191 x 4096 for 12 rows 26 us, 16 so; 4101 x 11000 for 5 rows 11.8 and 12.8)
        a.odd = rows > 5 && (reinterpret_cast<uintptr_t>(a.x) % 4 != 0 || x_stride % 2 != 0);
        a.y = static_cast<uint16_t*>(y) + r0 * w.n_out;
        a.m = (int32_t)rows;
        const dim3 g((unsigned)(wgs < cus ? wgs : cus), (unsigned)((rows + 15) / 16));
        if (in_lds)
            matvec_go<4, kManyLds>(a, dt, step, g, st);
        else if (many)
            matvec_go<4, kMany>(a, dt, step, g, st);
        else if (nb == 1)
            matvec_go<1, kOne>(a, dt, step, g, st);
        else if (nb == 2)
            matvec_go<2, kOne>(a, dt, step, g, st);
        else if (nb == 3)
            matvec_go<3, kOne>(a, dt, step, g, st);
        else
            matvec_go<4, kOne>(a, dt, step, g, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ecasq
