// The paged key/value cache: new rows written into it (rounded with a codebook
// per row where it holds symbols), and slots of least weight given up.
#include "half16.hpp"
#include "philox.hpp"
#include "serve.hpp"

namespace ecasq {
namespace {

constexpr int kWT = 256;

// Sequence of new row i: the number of sequences that end at or before it.
__device__ __forceinline__ int32_t sequence_of(const int32_t* __restrict__ starts, int32_t batch,
                                               int64_t i) {
    int32_t n = 0;
    for (int32_t b0 = 0; b0 < batch; b0 += 64) {
        const int32_t b = b0 + (int32_t)(threadIdx.x % 64);
        const bool ended = b < batch && (int64_t)starts[b + 1] <= i;
        n += __popcll(__ballot(ended));
    }
    return n;
}

// A row's codebook in LDS, its values rounded to the cache's type beside them.
struct RowBook {
    double q[16];
    int32_t t;
};

// A workgroup per new token.
template <int DT>
__global__ __launch_bounds__(kWT) void k_kv_write(ecasq_kv_cache c, KvNew n) {
    const int64_t i = blockIdx.x, slots = kv_slots(c);
    const int32_t b = sequence_of(n.starts, c.batch, i);
    if (b >= c.batch || n.starts[b] > i) return;
    const int64_t slot = (int64_t)c.lens[b] - n.starts[b + 1] + i;
    if (slot < 0 || slot >= slots) return;
    for (int32_t h = threadIdx.x; h < c.heads; h += kWT) {
        const int64_t at = ((int64_t)b * c.heads + h) * slots + slot;
        if (c.mass) c.mass[at] = 0.0f;
        if (c.pos) c.pos[at] = n.positions ? n.positions[i] : (int32_t)slot;
    }
    const int32_t d = c.head_dim;
    if (!c.coded) {
        const int32_t chunks = d / 8;
        for (int32_t e = threadIdx.x; e < 2 * c.heads * chunks; e += kWT) {
            const bool value = e >= c.heads * chunks;
            const int32_t r = value ? e - c.heads * chunks : e;
            const int64_t row = kv_row(c, b, r / chunks, slot);
            if (row < 0) return;
            const auto* from = static_cast<const uint16_t*>(value ? n.v : n.k) +
                               i * (value ? n.v_stride : n.k_stride) + (int64_t)r * 8;
            uint4 v;
            __builtin_memcpy(&v, from, 16);
            reinterpret_cast<uint4*>(value ? c.v : c.k)[row * chunks + r % chunks] = v;
        }
        return;
    }
    __shared__ RowBook books[kWT / 32];
    const int32_t lanes = d / 2, per = kWT / lanes;  // a thread per pair of entries
    const int32_t mine = threadIdx.x / lanes, pair = threadIdx.x % lanes;
    const uint32_t k0 = (uint32_t)n.seed, k1 = (uint32_t)(n.seed >> 32);
    for (int32_t r0 = 0; r0 < 2 * c.heads; r0 += per) {
        const int32_t r = r0 + mine;
        const bool live = r < 2 * c.heads, value = r >= c.heads;
        const int32_t head = value ? r - c.heads : r;
        const int64_t row = live ? kv_row(c, b, head, slot) : -1, in = i * c.heads + head;
        __syncthreads();
        if (row >= 0 && pair < 16) {
            const int32_t t = (value ? n.v_counts : n.k_counts)[in];
            const bool good = t >= 1 && t <= 16 && t <= n.s;
            const double q =
                good && pair < t ? (value ? n.v_books : n.k_books)[in * n.s + pair] : 0.0;
            books[mine].q[pair] = q;
            if (pair == 0) books[mine].t = good ? t : 0;
            static_cast<uint16_t*>(value ? c.v_books : c.k_books)[row * 16 + pair] =
                good ? to16<DT>(q) : kNan16<DT>;
        }
        __syncthreads();
        if (row < 0) continue;
        const RowBook& B = books[mine];
        uint32_t sym[2] = {0u, 0u};
        if (B.t > 1) {
            const int64_t h = (in * d) / 2 + pair;
            uint32_t w[4] = {(uint32_t)h, (uint32_t)(h >> 32), value ? 3u : 2u, 0u};
            philox4x32_10(w, k0, k1);
            const auto* from = static_cast<const uint16_t*>(value ? n.v : n.k) +
                               i * (value ? n.v_stride : n.k_stride) + (int64_t)head * d + 2 * pair;
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const double x = (double)from16<DT>(from[e]);
                int32_t at = 0;
                for (int32_t k = 1; k <= B.t - 2; k++)
                    if (B.q[k] < x) at = k;
                const double p = (x - B.q[at]) / (B.q[at + 1] - B.q[at]);
                sym[e] = at + (uniform53(w[2 * e], w[2 * e + 1]) < p ? 1 : 0);
            }
        }
        static_cast<uint8_t*>(value ? c.v : c.k)[row * lanes + pair] =
            (uint8_t)(sym[0] | (sym[1] << 4));
        if (n.k_hat) {
            auto* to = static_cast<uint16_t*>(value ? n.v_hat : n.k_hat) + in * d + 2 * pair;
#pragma unroll
            for (int e = 0; e < 2; e++) to[e] = B.t ? to16<DT>(B.q[sym[e]]) : kNan16<DT>;
        }
    }
}

// ---------------------------------------------------------------------------
// Eviction

constexpr int kET = 1024;

// Rank of a slot: larger is kept first.  A float's bits in an order that whole
// numbers have; NaN below all others, slots of recent positions above.
__device__ __forceinline__ uint32_t evict_key(float mass, int32_t pos, int64_t newest_but) {
    if ((int64_t)pos > newest_but) return 0xFFFFFFFFu;
    if (mass != mass) return 0u;
    const uint32_t b = __float_as_uint(mass + 0.0f);  // -0 as +0
    return (b >> 31) ? ~b : b | 0x80000000u;
}

// Sum over the workgroup, the same for every thread.
__device__ __forceinline__ int32_t block_count(int32_t v, int32_t* red) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    __syncthreads();
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
    __syncthreads();
    int32_t s = 0;
    for (int k = 0; k < kET / 64; k++) s += red[k];
    return s;
}

// Exclusive prefix count of `on` over the workgroup's threads, and the total.
__device__ __forceinline__ int32_t block_rank(bool on, int32_t* red, int32_t& total) {
    const uint64_t m = __ballot(on);
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    __syncthreads();
    if (lane == 0) red[wave] = __popcll(m);
    __syncthreads();
    int32_t before = 0, all = 0;
    for (int k = 0; k < kET / 64; k++) {
        if (k < wave) before += red[k];
        all += red[k];
    }
    total = all;
    return before + __popcll(m & ((1ull << lane) - 1));
}

// A workgroup per sequence and head: the rank of the last kept slot by bisection
// over the keys' bits, then the lists of freed and moving slots, then the moves.
__global__ __launch_bounds__(kET) void k_kv_evict(ecasq_kv_cache c, int32_t keep, int32_t recent,
                                                  float* mass_out, int32_t* pos_out,
                                                  int32_t* __restrict__ lists) {
    __shared__ int32_t red[kET / 64];
    __shared__ int32_t newest;
    const int32_t b = blockIdx.x / c.heads, head = blockIdx.x % c.heads;
    const int64_t slots = kv_slots(c), n = kv_len(c, b);
    const int64_t base = ((int64_t)b * c.heads + head) * slots;
    const float* mass = c.mass + base;
    const int32_t* pos = c.pos + base;
    if (threadIdx.x == 0) newest = INT32_MIN;
    __syncthreads();
    const int64_t most = n < keep ? n : keep;
    if (n > keep) {
        int32_t p = INT32_MIN;
        for (int64_t i = threadIdx.x; i < n; i += kET) p = max(p, pos[i]);
        atomicMax(&newest, p);
        __syncthreads();
        const int64_t but = (int64_t)newest - recent;
        // the largest key T with at least keep keys at or above it
        uint32_t T = 0;
        for (int bit = 31; bit >= 0; bit--) {
            const uint32_t at = T | (1u << bit);
            int32_t k = 0;
            for (int64_t i = threadIdx.x; i < n; i += kET) k += evict_key(mass[i], pos[i], but) >= at;
            if (block_count(k, red) >= keep) T = at;
        }
        int32_t above = 0;
        for (int64_t i = threadIdx.x; i < n; i += kET) above += evict_key(mass[i], pos[i], but) > T;
        int32_t ties = keep - block_count(above, red);  // slots of key T that are kept
        int32_t* freed = lists + (int64_t)blockIdx.x * 2 * keep;
        int32_t* moving = freed + keep;
        int32_t nf = 0, nm = 0;
        for (int64_t i0 = 0; i0 < n; i0 += kET) {
            const int64_t i = i0 + threadIdx.x;
            const uint32_t key = i < n ? evict_key(mass[i], pos[i], but) : 0u;
            int32_t got = 0;
            const bool tie = i < n && key == T;
            const int32_t place = block_rank(tie, red, got);
            const bool kept = i < n && (key > T || (tie && place < ties));
            ties = max(0, ties - got);
            const bool fr = i < keep && !kept, mv = i >= keep && kept;
            int32_t at = block_rank(fr, red, got);
            if (fr) freed[nf + at] = (int32_t)i;
            nf += got;
            at = block_rank(mv, red, got);
            if (mv) moving[nm + at] = (int32_t)i;
            nm += got;
        }
        __syncthreads();
        // the moves: a wavefront each
        const int lane = threadIdx.x % 64;
        const int32_t row16 = c.coded ? c.head_dim / 32 : c.head_dim / 8;
        for (int32_t m = threadIdx.x / 64; m < nf; m += kET / 64) {
            const int64_t to = kv_row(c, b, head, freed[m]), from = kv_row(c, b, head, moving[m]);
            if (to < 0 || from < 0) continue;
            for (int e = lane; e < row16; e += 64) {
                static_cast<uint4*>(c.k)[to * row16 + e] =
                    static_cast<const uint4*>(c.k)[from * row16 + e];
                static_cast<uint4*>(c.v)[to * row16 + e] =
                    static_cast<const uint4*>(c.v)[from * row16 + e];
            }
            if (c.coded && lane < 4) {
                uint4* books = static_cast<uint4*>(lane < 2 ? c.k_books : c.v_books);
                books[to * 2 + lane % 2] = books[from * 2 + lane % 2];
            }
        }
        __syncthreads();
        if (mass_out != c.mass)
            for (int64_t i = threadIdx.x; i < most; i += kET) mass_out[base + i] = mass[i];
        if (pos_out != c.pos)
            for (int64_t i = threadIdx.x; i < most; i += kET) pos_out[base + i] = pos[i];
        __syncthreads();
        for (int32_t m = threadIdx.x; m < nf; m += kET) {
            mass_out[base + freed[m]] = mass[moving[m]];
            pos_out[base + freed[m]] = pos[moving[m]];
        }
        return;
    }
    for (int64_t i = threadIdx.x; i < most; i += kET) {
        mass_out[base + i] = mass[i];
        pos_out[base + i] = pos[i];
    }
}

__global__ __launch_bounds__(256) void k_kv_lens(ecasq_kv_cache c, int32_t keep,
                                                 int32_t* lens_out) {
    const int32_t b = blockIdx.x * 256 + threadIdx.x;
    if (b >= c.batch) return;
    const int64_t n = kv_len(c, b);
    lens_out[b] = (int32_t)(n < keep ? n : keep);
}

}  // namespace

hipError_t launch_kv_write(const ecasq_kv_cache& c, const KvNew& n, hipStream_t st) {
    if (c.dt == ECASQ_F16)
        k_kv_write<1><<<(unsigned)n.rows, kWT, 0, st>>>(c, n);
    else
        k_kv_write<2><<<(unsigned)n.rows, kWT, 0, st>>>(c, n);
    return hipGetLastError();
}

size_t kv_evict_bytes(const ecasq_kv_cache& c, int32_t keep) {
    const int64_t most = keep < kv_slots(c) ? keep : kv_slots(c);
    return 256 + (size_t)c.batch * c.heads * 2 * most * sizeof(int32_t);
}

hipError_t launch_kv_evict(const ecasq_kv_cache& c, int32_t keep, int32_t recent, float* mass_out,
                           int32_t* pos_out, int32_t* lens_out, char* ws, hipStream_t st) {
    if (keep > kv_slots(c)) keep = (int32_t)kv_slots(c);
    k_kv_evict<<<(unsigned)(c.batch * c.heads), kET, 0, st>>>(c, keep, recent, mass_out, pos_out,
                                                              reinterpret_cast<int32_t*>(ws));
    k_kv_lens<<<(unsigned)((c.batch + 255) / 256), 256, 0, st>>>(c, keep, lens_out);
    return hipGetLastError();
}

}  // namespace ecasq
