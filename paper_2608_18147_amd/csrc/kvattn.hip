// Attention of one new token per sequence over the paged cache.
//
// A wavefront takes 32 slots at a time, two tiles of 16 (a tile lies in one page),
// and 16 query heads of one key/value head:
//   S' = K Q'   (16 slots x heads per tile),  p = 2^(S' - m),  O' += V' P',
// transposed, so that every lane keeps one head (lane % 16) throughout: the four
// slots 4 g .. 4 g + 3 of a tile (g = lane / 16) that its results of S' belong to
// are the ones that the second product takes from it, and the running maximum,
// the sum and the scale of O' are the lane's own.  The order of the slots in the
// second product is free; V' follows it.
//
// The running maximum m moves only when a score passes it by 2^8 (the weights
// stay below 2^15 in f16, 2^8 in bf16, and the sums are fp32), so that the four
// lanes of a head seldom have to agree on a new one.  Weights enter the second
// product as two 16-bit numbers, rounded and remainder: one alone would add an
// error as large as the result's own rounding.  Neither part may meet an infinity (a
// remainder is 0 or, in bf16, of either sign; a small weight of f16 is 0 in both), and bf16
// values near the largest pass the floats before they are divided by the sum: where a
// result is no finite number though the sum of the weights is, the wavefront takes it again
// from the definition (by_definition).
#include "half16.hpp"
#include "serve.hpp"

namespace ecasq {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4, kAT = 64 * kWaves;
constexpr float kLazy = 8.0f;  // log2 of what a weight may pass 1 by
template <int DT>
constexpr float kLift = DT == 1 ? 7.0f : 0.0f;  // keeps f16 weights off its smallest steps

// The plan of one call, the same on the host and the device.
struct Plan {
    int32_t q_heads, group, tiles;  // tiles of 16 query heads per key/value head
    int32_t chunk, chunks;          // slots per workgroup, chunks of the longest sequence
    int32_t tile_shift;             // log2 of a page's tiles, -1 where that is no whole number
};

template <int DT>
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (DT == 1)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, a),
                                                      __builtin_bit_cast(h16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a),
                                                       __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
}

// Two weights as 16-bit numbers, and their remainders.
template <int DT>
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
    if constexpr (DT == 1) {
        typedef __fp16 fp16x2 __attribute__((ext_vector_type(2)));
        const fp16x2 h = __builtin_amdgcn_cvt_pkrtz(a, b);
        const fp16x2 l = __builtin_amdgcn_cvt_pkrtz(a - (float)h.x, b - (float)h.y);
        hi = __builtin_bit_cast(uint32_t, h);
        lo = __builtin_bit_cast(uint32_t, l);
    } else {
        typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        const f32x2 v = {a, b};
        hi = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b16x2));
        const f32x2 r = {a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xFFFF0000u)};
        lo = __builtin_bit_cast(uint32_t, __builtin_convertvector(r, b16x2));
    }
}

// What O and l grow by when the maximum goes from m to M >= m.
__device__ __forceinline__ float down_to(float m, float M) {
    return m == M ? 1.0f : __builtin_amdgcn_exp2f(m - M);
}

template <int W>
struct Words {
    uint32_t w[W];
};
template <int W>
__device__ __forceinline__ Words<W> load_words(const void* p) {
    Words<W> r;
    if constexpr (W == 1)
        r.w[0] = *static_cast<const uint32_t*>(p);
    else
        __builtin_memcpy(&r, __builtin_assume_aligned(p, W == 2 ? 8 : 16), 4 * W);
    return r;
}

// Eight values of a row from eight symbols (a dword) and its codebook's byte planes:
// lo[k], hi[k] hold the low and high bytes of values 4 k .. 4 k + 3.  A byte
// permutation looks four symbols up in eight bytes; the two halves of the codebook
// are looked up by the symbols' low three bits and chosen between by the fourth.
// Order: symbols 0 2, 4 6, 1 3, 5 7.
struct Planes {
    uint32_t lo[4], hi[4];
};
__device__ __forceinline__ Planes planes(const Words<8>& b) {
    Planes p;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        p.lo[k] = __builtin_amdgcn_perm(b.w[2 * k + 1], b.w[2 * k], 0x06040200u);
        p.hi[k] = __builtin_amdgcn_perm(b.w[2 * k + 1], b.w[2 * k], 0x07050301u);
    }
    return p;
}
__device__ __forceinline__ void lookup4(const Planes& p, uint32_t low3, uint32_t half,
                                        uint32_t& first, uint32_t& second) {
    const uint32_t a0 = __builtin_amdgcn_perm(p.lo[1], p.lo[0], low3);
    const uint32_t b0 = __builtin_amdgcn_perm(p.lo[3], p.lo[2], low3);
    const uint32_t a1 = __builtin_amdgcn_perm(p.hi[1], p.hi[0], low3);
    const uint32_t b1 = __builtin_amdgcn_perm(p.hi[3], p.hi[2], low3);
    const uint32_t lo = __builtin_amdgcn_perm(b0, a0, half);
    const uint32_t hi = __builtin_amdgcn_perm(b1, a1, half);
    first = __builtin_amdgcn_perm(hi, lo, 0x05010400u);
    second = __builtin_amdgcn_perm(hi, lo, 0x07030602u);
}
__device__ __forceinline__ u32x4 lookup8(const Planes& p, uint32_t w) {
    uint32_t r0, r1, r2, r3;
    lookup4(p, w & 0x07070707u, ((w >> 1) & 0x04040404u) | 0x03020100u, r0, r1);
    lookup4(p, (w >> 4) & 0x07070707u, ((w >> 5) & 0x04040404u) | 0x03020100u, r2, r3);
    return u32x4{r0, r1, r2, r3};
}

// A tile of 16 slots: its first row in the cache, and how many of its slots hold one.
struct Tile {
    int64_t row;
    int32_t live;
};

// LDS of a wavefront's value codebooks: the 8 slots of lane group g at 288 g, 32
// bytes each, so that the groups' reads meet different banks and every address
// is a byte (the symbol's, with the group's bits) and a constant high byte.
constexpr int kBookBytes = 1280;

template <int DT, bool CODED, int D>
__device__ __forceinline__ float entry(const void* rows, const void* books, int64_t row, int e) {
    if constexpr (CODED) {
        const uint32_t two = static_cast<const uint8_t*>(rows)[row * (D / 2) + e / 2];
        return from16<DT>(
            static_cast<const uint16_t*>(books)[row * 16 + (two >> (e % 2 * 4) & 15u)]);
    } else {
        return from16<DT>(static_cast<const uint16_t*>(rows)[row * D + e]);
    }
}

// o = sum_t p_t V_t over the slots lo .. end - 1, entries E quad and up of a head, for the 16
// consecutive lanes `quad` of each of a wavefront's four heads: scores of 16 slots by a lane each,
// then weights p = 2^(score - up) by (at most 1, so sums of finite values are finite), slot after
// slot.  The smallest float is added to a weight, so that it is no 0 by underflow: that makes an
// infinity of an infinity and nothing of a finite value; a score of -inf has weight 0, and 0
// times an infinity is NaN.  A path for rare values, not for speed (64 sequences of about 4000
// 16-bit slots with one infinity each: 1.4 ms, 0.19 with none).
template <int DT, bool CODED, int D>
__device__ __forceinline__ void by_definition(const ecasq_kv_cache& c, int32_t b, int32_t head,
                                              const uint16_t* __restrict__ q, int32_t lo,
                                              int32_t end, float scale, float up, float by,
                                              float (&o)[D / 16]) {
    constexpr int E = D / 16;
    const int lane = threadIdx.x % 64, quad = lane % 16;
#pragma unroll
    for (int i = 0; i < E; i++) o[i] = 0.0f;
#pragma unroll 1
    for (int32_t s0 = lo; s0 < end; s0 += 16) {
        const int64_t mine = s0 + quad < end ? kv_row(c, b, head, s0 + quad) : -1;
        float z = 0.0f;
        if (mine >= 0)
#pragma unroll 8
            for (int e = 0; e < D; e++)
                z = __builtin_fmaf(entry<DT, CODED, D>(c.k, c.k_books, mine, e), from16<DT>(q[e]),
                                   z);
        z *= scale;
#pragma unroll 1
        for (int k = 0; k < 16; k++) {
            const float score = __shfl(z, lane - quad + k);
            const int64_t row = s0 + k < end ? kv_row(c, b, head, s0 + k) : -1;
            if (row < 0) continue;
            const float weight = __builtin_fmaf(__builtin_amdgcn_exp2f(score - up), by,
                                                score > -INFINITY ? 0x1p-149f : 0.0f);
#pragma unroll
            for (int i = 0; i < E; i++)
                o[i] = __builtin_fmaf(
                    weight, entry<DT, CODED, D>(c.v, c.v_books, row, quad * E + i), o[i]);
        }
    }
}

template <int DT, bool CODED, int D>
__global__ __launch_bounds__(kAT, D == 256 ? 2 : 3) void k_attend(ecasq_kv_cache c, Plan p,
                                                const uint16_t* __restrict__ q, int64_t q_stride,
                                                float scale, uint16_t* __restrict__ out,
                                                float* __restrict__ scores,
                                                float2* __restrict__ ml, float* __restrict__ part) {
    constexpr int J = D / 32;   // products per tile of S'
    constexpr int E = D / 16;   // entries of a value row per lane
    constexpr int MERGE = kWaves * (64 * D + 128);  // a wavefront's O', m and l
    constexpr int LDS = CODED && kWaves * kBookBytes > MERGE ? kWaves * kBookBytes : MERGE;
    __shared__ __align__(256) uint8_t lds[LDS];

    const int lane = threadIdx.x % 64, n16 = lane % 16, g = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    // workgroups: head, then sequence, head tile and chunk.  Workgroups go to the eight
    // dies in turn; with the chunks first, the first chunks, which every sequence has,
    // came to lie on one die and the last ones on another (16 ragged sequences: 3 of 53 us).
    // The tiles of a head meet on one die where
    // the heads of all sequences are a multiple of eight.
    int32_t id = blockIdx.x;
    const int32_t head = id % c.heads;
    id /= c.heads;
    const int32_t b = id % c.batch;
    id /= c.batch;
    const int32_t ht = id % p.tiles, ch = id / p.tiles;
    const int32_t n = (int32_t)kv_len(c, b);
    const int32_t lo = ch * p.chunk;
    if (lo >= n && ch > 0) return;
    const int32_t end = n - lo < p.chunk ? n : lo + p.chunk;
    const int32_t used = (n + p.chunk - 1) / p.chunk;  // chunks of this sequence
    const int32_t h = ht * 16 + n16;                   // this lane's head within the group
    const bool mine = h < p.group;
    const int64_t row_out = ((int64_t)b * c.heads + head) * p.group + h;

    // Q': lane's head, entries in the order of K's
    u32x4 qv[J];
    {
        const uint16_t* qr = q + (int64_t)b * q_stride + ((int64_t)head * p.group + h) * D;
#pragma unroll
        for (int j = 0; j < J; j++) {
            qv[j] = u32x4{0u, 0u, 0u, 0u};
            if (mine) {
                if constexpr (CODED) {
                    Words<4> w;
                    __builtin_memcpy(&w, qr + g * (D / 4) + 8 * j, 16);
                    qv[j] = u32x4{__builtin_amdgcn_perm(w.w[1], w.w[0], 0x05040100u),
                                  __builtin_amdgcn_perm(w.w[3], w.w[2], 0x05040100u),
                                  __builtin_amdgcn_perm(w.w[1], w.w[0], 0x07060302u),
                                  __builtin_amdgcn_perm(w.w[3], w.w[2], 0x07060302u)};
                } else {
                    __builtin_memcpy(&qv[j], qr + 32 * j + 8 * g, 16);
                }
            }
        }
    }

    const int32_t per_page = c.page_size / 16;
    auto tile_at = [&](int32_t t) {
        Tile r{0, 0};
        if (t * 16 < end) {
            const int32_t at = p.tile_shift >= 0 ? t >> p.tile_shift : t / per_page;
            const int32_t page = c.table[(int64_t)b * c.max_pages + at];
            if (page >= 0 && page < c.n_pages) {
                r.row = ((int64_t)page * c.heads + head) * c.page_size + (t - at * per_page) * 16;
                r.live = end - t * 16 < 16 ? end - t * 16 : 16;
            }
        }
        return r;
    };

    // where a lane's part of a tile's keys and values begins, in bytes
    constexpr uint32_t kRow = CODED ? D / 2 : 2 * D;
    const uint32_t k_at = n16 * kRow + g * (CODED ? D / 8 : 16);
    const uint32_t v_at = 4 * g * kRow + n16 * (kRow / 16);

    f32x4 acc[E];
#pragma unroll
    for (int i = 0; i < E; i++) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, ref = 0.0f, l = 0.0f;
    uint8_t* book = lds + wave * kBookBytes;
    const uint32_t group_bits = 0x20202020u * (uint32_t)g;
    const uint32_t high = (uint32_t)(wave * kBookBytes / 256 + g);

    for (int32_t t0 = lo / 16 + 2 * wave; t0 * 16 < end; t0 += 2 * kWaves) {
        const Tile tile[2] = {tile_at(t0), tile_at(t0 + 1)};
        f32x4 s[2];
        Words<CODED ? E / 8 + (E < 8) : E / 2> v[8];
        if constexpr (CODED) {
            Words<D / 32> kc[2];
            Words<8> kb[2];
#pragma unroll
            for (int t = 0; t < 2; t++) {
                kc[t] = load_words<D / 32>(static_cast<const uint8_t*>(c.k) +
                                           tile[t].row * (D / 2) + k_at);
                kb[t] = load_words<8>(static_cast<const uint8_t*>(c.k_books) + tile[t].row * 32 +
                                      n16 * 32u);
            }
            const int64_t vb_row = lane < 32 ? tile[0].row : tile[1].row;
            const Words<4> vb = load_words<4>(static_cast<const uint8_t*>(c.v_books) +
                                              vb_row * 32 + lane % 32 * 16);
#pragma unroll
            for (int k = 0; k < 8; k++) {
                const uint8_t* at = static_cast<const uint8_t*>(c.v) + tile[k / 4].row * (D / 2) +
                                    v_at + k % 4 * (D / 2);
                if constexpr (E == 4)
                    v[k].w[0] = *reinterpret_cast<const uint16_t*>(at);
                else
                    v[k] = load_words<E / 8>(at);
            }
            {
                const int slot = lane / 2 % 16;
                const bool live = slot < (lane < 32 ? tile[0].live : tile[1].live);
                uint8_t* to = book + slot / 4 * 288 + (slot % 4 + lane / 32 * 4) * 32 +
                              lane % 2 * 16;
                Words<4> w;
#pragma unroll
                for (int k = 0; k < 4; k++) w.w[k] = live ? vb.w[k] : 0u;
                __builtin_memcpy(__builtin_assume_aligned(to, 16), &w, 16);
            }
#pragma unroll
            for (int t = 0; t < 2; t++) {
                const Planes pl = planes(kb[t]);
                s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < J; j++) s[t] = mfma<DT>(lookup8(pl, kc[t].w[j]), qv[j], s[t]);
            }
        } else {
            u32x4 kv[2][J];
#pragma unroll
            for (int t = 0; t < 2; t++)
#pragma unroll
                for (int j = 0; j < J; j++)
                    kv[t][j] = *reinterpret_cast<const u32x4*>(
                        static_cast<const uint8_t*>(c.k) + tile[t].row * (2 * D) + k_at + 64 * j);
#pragma unroll
            for (int k = 0; k < 8; k++)
                v[k] = load_words<E / 2>(static_cast<const uint8_t*>(c.v) +
                                         tile[k / 4].row * (2 * D) + v_at + k % 4 * (2 * D));
#pragma unroll
            for (int t = 0; t < 2; t++) {
                s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < J; j++) s[t] = mfma<DT>(kv[t][j], qv[j], s[t]);
            }
            if (tile[0].live < 16 || tile[1].live < 16) {  // no NaN of slots that hold nothing
#pragma unroll
                for (int k = 0; k < 8; k++)
                    if (4 * g + k % 4 >= tile[k / 4].live)
#pragma unroll
                        for (int i = 0; i < E / 2; i++) v[k].w[i] = 0u;
            }
        }

        float z[8], top = -INFINITY;
#pragma unroll
        for (int k = 0; k < 8; k++) {
            z[k] = 4 * g + k % 4 < tile[k / 4].live ? s[k / 4][k % 4] * scale : -INFINITY;
            top = fmaxf(top, z[k]);
        }
        if (scores && mine) {
#pragma unroll
            for (int t = 0; t < 2; t++)
                if ((t0 + t) * 16 < end) {
                    const f32x4 w = {z[4 * t], z[4 * t + 1], z[4 * t + 2], z[4 * t + 3]};
                    *reinterpret_cast<f32x4*>(scores + row_out * kv_slots(c) + (t0 + t) * 16 +
                                              4 * g) = w;
                }
        }
        float down = 1.0f;
        if (__any(top > m + kLazy)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float M = fmaxf(m, top);
            down = down_to(m, M);
            m = M;
            ref = M == -INFINITY ? 0.0f : M - kLift<DT>;
        }
        // by 1 where nothing moved: 32 products cost less than the copies of O' that the
        // compiler makes where a branch may change it
        l *= down;
#pragma unroll
        for (int i = 0; i < E; i++) acc[i] *= down;
        u32x4 hi, rest;
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; k++) {
            w[k] = __builtin_amdgcn_exp2f(z[k] - ref);
            l += w[k];
        }
#pragma unroll
        for (int k = 0; k < 4; k++) {
            uint32_t a, r;
            split2<DT>(w[2 * k], w[2 * k + 1], a, r);
            hi[k] = a;
            rest[k] = r;
        }

        if constexpr (CODED) {
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int wd = 0; wd < (E + 7) / 8; wd++) {
                uint32_t even[8], odd[8];
#pragma unroll
                for (int k = 0; k < 8; k++) {
                    even[k] = ((v[k].w[wd] << 1) & 0x1E1E1E1Eu) | group_bits;
                    odd[k] = ((v[k].w[wd] >> 3) & 0x1E1E1E1Eu) | group_bits;
                }
#pragma unroll
                for (int i = 0; i < (E < 8 ? E : 8); i++) {
                    uint32_t x[8];
#pragma unroll
                    for (int k = 0; k < 8; k++) {
                        const uint32_t at = __builtin_amdgcn_perm(
                            high, i % 2 ? odd[k] : even[k], 0x0C0C0400u + i / 2);
                        x[k] = *reinterpret_cast<const uint16_t*>(lds + at + 32 * k);
                    }
                    const u32x4 a = {x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16,
                                     x[6] | x[7] << 16};
                    f32x4& o = acc[8 * wd + i];
                    o = mfma<DT>(a, hi, o);
                    o = mfma<DT>(a, rest, o);
                }
            }
            __builtin_amdgcn_wave_barrier();
        } else {
#pragma unroll
            for (int i = 0; i < E; i++) {
                const uint32_t sel = i % 2 ? 0x07060302u : 0x05040100u;
                u32x4 a;
#pragma unroll
                for (int k = 0; k < 4; k++)
                    a[k] = __builtin_amdgcn_perm(v[2 * k + 1].w[i / 2], v[2 * k].w[i / 2], sel);
                acc[i] = mfma<DT>(a, hi, acc[i]);
                acc[i] = mfma<DT>(a, rest, acc[i]);
            }
        }
    }

    // The wavefronts' parts meet in LDS: O' as [E][head][g] of four entries, so that 16 threads
    // a head read them in order, then m and l (summed over the head's four lanes).
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    __syncthreads();
    if (mine) {
        float* to = reinterpret_cast<float*>(lds) + wave * (16 * D + 32);
#pragma unroll
        for (int i = 0; i < E; i++)
            *reinterpret_cast<f32x4*>(to + i * 256 + (n16 * 4 + g) * 4) = acc[i];
        if (g == 0) {
            to[16 * D + n16] = m;
            to[16 * D + 16 + n16] = l;
        }
    }
    __syncthreads();
    // entries (4 g + r) E + i of head o16, by thread 16 o16 + 4 g + r
    static_assert(kAT == 256, "16 heads by 16 threads");
    const int o16 = threadIdx.x / 16, quad = threadIdx.x % 16;
    if (ht * 16 + o16 >= p.group) return;
    const float* from = reinterpret_cast<const float*>(lds);
    constexpr int kPart = 16 * D + 32;
    float M = -INFINITY, L = 0.0f, down[kWaves], o[E];
#pragma unroll
    for (int w = 0; w < kWaves; w++) M = fmaxf(M, from[w * kPart + 16 * D + o16]);
#pragma unroll
    for (int w = 0; w < kWaves; w++) {
        down[w] = down_to(from[w * kPart + 16 * D + o16], M);
        L += from[w * kPart + 16 * D + 16 + o16] * down[w];
    }
#pragma unroll
    for (int i = 0; i < E; i++) {
        o[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; w++)
            o[i] += from[w * kPart + i * 256 + threadIdx.x] * down[w];
    }
    // (no weight at all: 0, or the NaN of the values, which a join hands on)
    const float by = L == 0.0f ? 1.0f : 1.0f / L;
    float none = 0.0f;  // NaN if one of the entries is no finite number
#pragma unroll
    for (int i = 0; i < E; i++) {
        none += o[i] * 0.0f;
        o[i] *= by;
    }
    const bool again = none != 0.0f && L > 0.0f && L < INFINITY;
    if (__any(again)) {  // (heads are the group's: the others' threads have returned)
        float exact[E];
        by_definition<DT, CODED, D>(
            c, b, head, q + (int64_t)b * q_stride + ((int64_t)head * p.group + ht * 16 + o16) * D, lo,
            end, scale, M - kLift<DT>, by, exact);
#pragma unroll
        for (int i = 0; i < E; i++) o[i] = again ? exact[i] : o[i];
    }
    const int64_t row = ((int64_t)b * c.heads + head) * p.group + ht * 16 + o16;
    if (ml && quad == 0) ml[row * p.chunks + ch] = make_float2(M, L);
    if (used > 1) {
        __builtin_memcpy(
            __builtin_assume_aligned(part + (row * p.chunks + ch) * D + quad * E, 16), o, 4 * E);
        return;
    }
    uint32_t w[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; i++)  // (no weight at all: zeros, whatever the values are)
        w[i] = L == 0.0f ? 0u : to16<DT>(o[2 * i]) | (uint32_t)to16<DT>(o[2 * i + 1]) << 16;
    __builtin_memcpy(__builtin_assume_aligned(out + row * D + quad * E, 8), w, 2 * E);
}

// Joins the chunks of every sequence that has more than one, a workgroup per query
// head; the workgroups after those give the slots their weights, 1024 slots of a
// key/value head at a time: the sum over the group's heads in order.
constexpr int kJT = 256, kSpan = 4 * kJT;

// Maximum and sum of a head's chunks, by one wavefront; the same for every lane.  (A chunk's
// part is divided by its sum already.)
__device__ __forceinline__ float2 joined(const float2* __restrict__ ml, int32_t used) {
    const int lane = threadIdx.x % 64;
    float m = -INFINITY, l = 0.0f;
    for (int32_t k = lane; k < used; k += 64) m = fmaxf(m, ml[k].x);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
    for (int32_t k = lane; k < used; k += 64) l += ml[k].y * down_to(ml[k].x, m);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off);
    return make_float2(m, l);
}

template <int DT, int D>
__device__ __forceinline__ void join_row(const Plan& p, int64_t row, int32_t used,
                                         const float2* __restrict__ ml,
                                         const float* __restrict__ part,
                                         uint16_t* __restrict__ out) {
    // a chunk's entries by D / 4 threads, kSide chunks side by side
    constexpr int kSide = kJT / (D / 4);
    __shared__ f32x4 sums[kJT];
    const int side = threadIdx.x / (D / 4), e = threadIdx.x % (D / 4);
    const float2* at = ml + row * p.chunks;
    const float2 all = joined(at, used);
    const auto* from = reinterpret_cast<const f32x4*>(part + row * p.chunks * D) + e;
    const float by = 1.0f / all.y;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int32_t k = side; k < used; k += kSide) {
        // a chunk's share, at most 1, and no 0 by underflow (by_definition)
        const float2 v = at[k];
        const float share =
            __builtin_fmaf(v.y * down_to(v.x, all.x), by, v.y > 0.0f ? 0x1p-149f : 0.0f);
        o += from[(int64_t)k * (D / 4)] * share;
    }
    sums[threadIdx.x] = o;
    __syncthreads();
    if (side != 0) return;
#pragma unroll
    for (int k = 1; k < kSide; k++) o += sums[k * (D / 4) + e];
    if (all.y == 0.0f) o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};  // no weight at all
    const uint32_t w[2] = {to16<DT>(o[0]) | (uint32_t)to16<DT>(o[1]) << 16,
                           to16<DT>(o[2]) | (uint32_t)to16<DT>(o[3]) << 16};
    __builtin_memcpy(__builtin_assume_aligned(out + row * D + 4 * e, 8), w, 8);
}

template <int DT>
__global__ __launch_bounds__(kJT) void k_join(ecasq_kv_cache c, Plan p, int32_t join_groups,
                                              const float* __restrict__ scores,
                                              const float2* __restrict__ ml,
                                              const float* __restrict__ part,
                                              uint16_t* __restrict__ out, float* mass_out) {
    if ((int32_t)blockIdx.x < join_groups) {
        const int64_t row = blockIdx.x;
        const int32_t b = (int32_t)(row / p.q_heads);
        const int32_t n = (int32_t)kv_len(c, b), used = (n + p.chunk - 1) / p.chunk;
        if (used <= 1) return;
        if (c.head_dim == 64)
            join_row<DT, 64>(p, row, used, ml, part, out);
        else if (c.head_dim == 128)
            join_row<DT, 128>(p, row, used, ml, part, out);
        else
            join_row<DT, 256>(p, row, used, ml, part, out);
        return;
    }
    __shared__ float2 each[64];
    const int64_t slots = kv_slots(c);
    const int32_t spans = (int32_t)((slots + kSpan - 1) / kSpan);
    const int64_t id = (int64_t)blockIdx.x - join_groups;
    const int64_t kvh = id / spans;
    const int32_t b = (int32_t)(kvh / c.heads), n = (int32_t)kv_len(c, b);
    const int32_t first = (int32_t)(id % spans) * kSpan;
    if (first >= n) return;
    const int32_t used = (n + p.chunk - 1) / p.chunk;
    for (int32_t h = threadIdx.x / 64; h < p.group; h += kJT / 64) {
        const float2 v = joined(ml + (kvh * p.group + h) * p.chunks, used);
        if (threadIdx.x % 64 == 0)
            each[h] = make_float2(v.x == -INFINITY ? 0.0f : v.x - kLift<DT>,
                                  v.y == 0.0f ? 0.0f : 1.0f / v.y);
    }
    __syncthreads();
    const int32_t i = first + 4 * (int32_t)threadIdx.x;
    if (i >= n) return;
    // four slots: all within the row of scores, whose length is a multiple of 16
    f32x4 w = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int32_t h = 0; h < p.group; h++) {
        const f32x4 z = *reinterpret_cast<const f32x4*>(scores + (kvh * p.group + h) * slots + i);
#pragma unroll
        for (int k = 0; k < 4; k++)
            w[k] += __builtin_amdgcn_exp2f(z[k] - each[h].x) * each[h].y;
    }
    const int64_t at = kvh * slots + i;
#pragma unroll
    for (int k = 0; k < 4; k++)
        if (i + k < n) mass_out[at + k] = (c.mass ? c.mass[at + k] : 0.0f) + w[k];
}

size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }

// Workgroups of four wavefronts where every sequence is as long as the table allows: as
// many as are resident at once for a single sequence; more for several, because
// they seldom are of one length (131071 coded slots alone: 54 us with 1024, 60 with
// 1792; 16 sequences of 0 to 8191: 49 and 39 us; 64 of 3500 to 4500 in 16 bits: 190 and
// 193 us).  A chunk has 256 slots at least: two rounds of a workgroup take less than
// the launch that joins two chunks (4 sequences of up to 200: 6.1 us, 7.9 with 128); 128 where
// there are chunks to join anyway, few workgroups otherwise and few chunks to a head (8 heads of
// 3000 coded slots: 96 workgroups, 9.1 us and 10.3 with 256; 8 heads of 8000 slots: 250, 14.3
// and 12.7; one head of 45000: 18.5 and 15.1).
constexpr int64_t kGroupsOne = 1024, kGroupsMany = 1792, kGroupsFew = 192, kChunkLeast = 256;

Plan plan(const ecasq_kv_cache& c, int32_t q_heads) {
    Plan p;
    p.q_heads = q_heads;
    p.group = q_heads / c.heads;
    p.tiles = (p.group + 15) / 16;
    const int64_t rows = (int64_t)c.batch * c.heads * p.tiles, slots = kv_slots(c);
    const int64_t groups = c.batch > 1 ? kGroupsMany : kGroupsOne;
    int64_t chunk = (rows * slots + groups - 1) / groups;
    chunk = (chunk + 127) / 128 * 128;
    if (chunk < kChunkLeast)
        chunk = slots > kChunkLeast && slots <= 32 * kChunkLeast &&
                        rows * slots < kGroupsFew * kChunkLeast
                    ? kChunkLeast / 2
                    : kChunkLeast;
    if (chunk > slots) chunk = slots;
    p.chunk = (int32_t)chunk;
    p.chunks = (int32_t)((slots + chunk - 1) / chunk);
    const int32_t per_page = c.page_size / 16;
    p.tile_shift = (per_page & (per_page - 1)) == 0 ? __builtin_ctz((unsigned)per_page) : -1;
    return p;
}

struct Layout {
    size_t ml, part, scores, total;
};
Layout layout(const ecasq_kv_cache& c, const Plan& p, bool mass) {
    const size_t rows = (size_t)c.batch * p.q_heads, parts = rows * (size_t)p.chunks;
    Layout l;
    l.ml = 0;
    l.part = align256(p.chunks > 1 || mass ? parts * sizeof(float2) : 0);
    l.scores = l.part + align256(p.chunks > 1 ? parts * (size_t)c.head_dim * sizeof(float) : 0);
    l.total = l.scores + (mass ? rows * (size_t)kv_slots(c) * sizeof(float) : 0) + 256;
    return l;
}

template <int DT, bool CODED>
void attend(const ecasq_kv_cache& c, const Plan& p, const uint16_t* q, int64_t q_stride,
            float scale, uint16_t* out, float* scores, float2* ml, float* part, hipStream_t st) {
    const unsigned g = (unsigned)((int64_t)c.batch * c.heads * p.tiles * p.chunks);
    auto go = [&](auto kernel) {
        kernel<<<g, kAT, 0, st>>>(c, p, q, q_stride, scale, out, scores, ml, part);
    };
    if (c.head_dim == 64)
        go(k_attend<DT, CODED, 64>);
    else if (c.head_dim == 128)
        go(k_attend<DT, CODED, 128>);
    else
        go(k_attend<DT, CODED, 256>);
}

}  // namespace

size_t kv_attention_bytes(const ecasq_kv_cache& c, int32_t q_heads, bool mass) {
    return layout(c, plan(c, q_heads), mass).total;
}

hipError_t launch_kv_attention(const ecasq_kv_cache& c, const void* q, int64_t q_stride,
                               int32_t q_heads, float scale, float* mass_out, void* out, char* ws,
                               hipStream_t st) {
    const Plan p = plan(c, q_heads);
    const Layout l = layout(c, p, mass_out != nullptr);
    auto* ml = p.chunks > 1 || mass_out ? reinterpret_cast<float2*>(ws + l.ml) : nullptr;
    auto* part = reinterpret_cast<float*>(ws + l.part);
    auto* scores = mass_out ? reinterpret_cast<float*>(ws + l.scores) : nullptr;
    const auto* qs = static_cast<const uint16_t*>(q);
    auto* o = static_cast<uint16_t*>(out);
    const float log2_scale = scale * 1.44269504f;  // weights are powers of two
    if (c.dt == ECASQ_F16)
        c.coded ? attend<1, true>(c, p, qs, q_stride, log2_scale, o, scores, ml, part, st)
                : attend<1, false>(c, p, qs, q_stride, log2_scale, o, scores, ml, part, st);
    else
        c.coded ? attend<2, true>(c, p, qs, q_stride, log2_scale, o, scores, ml, part, st)
                : attend<2, false>(c, p, qs, q_stride, log2_scale, o, scores, ml, part, st);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || (p.chunks == 1 && !mass_out)) return e;
    const int32_t join = p.chunks > 1 ? c.batch * q_heads : 0;
    const int64_t weigh =
        mass_out ? (int64_t)c.batch * c.heads * ((kv_slots(c) + kSpan - 1) / kSpan) : 0;
    if (c.dt == ECASQ_F16)
        k_join<1><<<(unsigned)(join + weigh), kJT, 0, st>>>(c, p, join, scores, ml, part, o,
                                                            mass_out);
    else
        k_join<2><<<(unsigned)(join + weigh), kJT, 0, st>>>(c, p, join, scores, ml, part, o,
                                                            mass_out);
    return hipGetLastError();
}

}  // namespace ecasq
