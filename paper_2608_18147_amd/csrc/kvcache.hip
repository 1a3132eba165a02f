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

// Where new row i goes, for a whole workgroup: its sequence, slot and page (-1: none), with
// the slot's weight and position set; false if it is left out.
struct Place {
    int32_t b, page, offset;
};
__device__ __forceinline__ bool place_of(const ecasq_kv_cache& c, const KvNew& n, int64_t i,
                                         Place& p) {
    const int64_t slots = kv_slots(c);
    p.b = sequence_of(n.starts, c.batch, i);
    if (p.b >= c.batch || n.starts[p.b] > i) return false;
    const int64_t slot = (int64_t)c.lens[p.b] - n.starts[p.b + 1] + i;
    if (slot < 0 || slot >= slots) return false;
    for (int32_t h = threadIdx.x; blockIdx.y == 0 && h < c.heads; h += kWT) {
        const int64_t at = ((int64_t)p.b * c.heads + h) * slots + slot;
        if (c.mass) c.mass[at] = 0.0f;
        if (c.pos) c.pos[at] = n.positions ? n.positions[i] : (int32_t)slot;
    }
    const uint32_t at = (uint32_t)slot, size = (uint32_t)c.page_size;  // below 2^30
    p.page = c.table[(int64_t)p.b * c.max_pages + at / size];
    p.offset = (int32_t)(at % size);
    return p.page >= 0 && p.page < c.n_pages;
}

// Rows of 16-bit values: a workgroup per token, 16 bytes a thread.
__global__ __launch_bounds__(kWT) void k_kv_write(ecasq_kv_cache c, KvNew n) {
    const int64_t i = blockIdx.x;
    Place p;
    if (!place_of(c, n, i, p)) return;
    const int32_t chunks = c.head_dim / 8;
    for (int32_t e = threadIdx.x; e < 2 * c.heads * chunks; e += kWT) {
        const bool value = e >= c.heads * chunks;
        const int32_t r = value ? e - c.heads * chunks : e;
        const int64_t row = ((int64_t)p.page * c.heads + r / chunks) * c.page_size + p.offset;
        const auto* from = static_cast<const uint16_t*>(value ? n.v : n.k) +
                           i * (value ? n.v_stride : n.k_stride) + (int64_t)r * 8;
        uint4 v;
        __builtin_memcpy(&v, from, 16);
        reinterpret_cast<uint4*>(value ? c.v : c.k)[row * chunks + r % chunks] = v;
    }
}

// A row's codebook in a wavefront's LDS: the values; the largest floats not above the
// values 1 .. t - 2, and infinity (a float x is above value k exactly if it is above that
// float); about one over the intervals' widths (NaN where that is no ordinary float); the
// values in the cache's type.
struct RowBook {
    double q[16];
    float s[16], over[16];
    uint16_t h[16];
    int32_t t;
};

__device__ __forceinline__ float float_not_above(double q) {
    const float f = (float)q;
    if (!((double)f > q)) return f;
    const uint32_t b = __float_as_uint(f);
    return __uint_as_float((b & 0x7FFFFFFFu) == 0u ? 0x80000001u : (b >> 31) ? b + 1u : b - 1u);
}

// Rows of symbols: a workgroup per token, a wavefront per 128 entries (a row, two or half
// of one), two entries a lane from one call of the generator.  Brackets and comparisons are
// made in 32 bits where those decide, as in ecasq_quantize: the quotient in 32 bits is within
// 2^-21 of the one in 64 up to 2, and the uniform within 2^-24, so that only a difference
// below 2^-20 (one entry in 2^19, or NaN) takes the 64-bit division (4000 tokens of 8 heads of
// 128: 50 us with 64-bit comparisons, 30 so).  Of the 30 us the generator is 5, the bracket
// search 2.4 and the books' preparation, by 16 lanes of 64 where a row is 128 entries or more,
// 2.4; without generator and search 23.6 remain.
template <int DT, int D>
__global__ __launch_bounds__(kWT) void k_kv_round(ecasq_kv_cache c, KvNew n) {
    constexpr int kRows = D < 128 ? 128 / D : 1, kParts = D < 128 ? 1 : D / 128;
    __shared__ RowBook lds[kWT / 64][kRows];
    const int64_t i = blockIdx.x;
    const int lane = threadIdx.x % 64, r = lane / 16, k = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int mine = kRows > 1 ? lane / (D / 2) : 0;
    const uint32_t k0 = (uint32_t)n.seed, k1 = (uint32_t)(n.seed >> 32);
    const int32_t units = (c.heads + kRows - 1) / kRows * kParts;  // of keys, and of values
    const int32_t last = min(2 * units, (int32_t)(blockIdx.y + 1) * n.units);
    RowBook* books = lds[wave];
    // what a unit reads, on the way while the one before is rounded (and, the first, while
    // the row's place is found): a lane's count and value of the books, and two entries
    struct Unit {
        bool value;
        int32_t part, head0, t, pair;
        uint32_t two;
        double q;
    };
    auto read = [&](int32_t u) {
        Unit x;
        x.value = u >= units;
        const int32_t v = x.value ? u - units : u;
        x.part = v % kParts;
        x.head0 = v / kParts * kRows;
        x.pair = kRows > 1 ? lane % (D / 2) : x.part * 64 + lane;
        x.t = 0;
        x.two = 0u;
        x.q = 0.0;
        if (u >= last) return x;
        const int64_t in0 = i * c.heads + x.head0;
        if (x.head0 + mine < c.heads)
            __builtin_memcpy(&x.two,
                             static_cast<const uint16_t*>(x.value ? n.v : n.k) +
                                 i * (x.value ? n.v_stride : n.k_stride) +
                                 (int64_t)(x.head0 + mine) * D + 2 * x.pair,
                             4);
        if (r < kRows && x.head0 + r < c.heads) {
            x.t = (x.value ? n.v_counts : n.k_counts)[in0 + r];
            if (k < n.s) x.q = (x.value ? n.v_books : n.k_books)[(in0 + r) * n.s + k];
        }
        return x;
    };
    int32_t u = (int32_t)blockIdx.y * n.units + wave;
    Unit next = read(u);
    Place p;
    if (!place_of(c, n, i, p)) return;
    for (; u < last; u += kWT / 64) {
        const Unit now = next;
        next = read(u + kWT / 64);
        const bool value = now.value;
        const int32_t head0 = now.head0, part = now.part, pair = now.pair;
        const uint32_t two = now.two;
        const int64_t row0 = ((int64_t)p.page * c.heads + head0) * c.page_size + p.offset;
        const int64_t in0 = i * c.heads + head0;
        // the books: a lane per value
        {
            const bool live = r < kRows && head0 + r < c.heads;
            const bool good = now.t >= 1 && now.t <= 16 && now.t <= n.s;
            const int32_t t = good ? now.t : 0;
            const double q = k < t ? now.q : 0.0;
            const double width = __shfl_down(q, 1) - q;
            const uint16_t h = good ? to16<DT>(q) : kNan16<DT>;
            __builtin_amdgcn_wave_barrier();  // the last unit's reads come first
            if (live) {
                RowBook& B = books[r];
                B.q[k] = q;
                B.s[k] = k >= 1 && k <= t - 2 ? float_not_above(q) : __builtin_huge_valf();
                B.over[k] = k < t - 1 && width >= 0x1p-100 && width <= 0x1p+100
                                ? 1.0f / (float)width
                                : __builtin_nanf("");
                B.h[k] = h;
                if (k == 0) B.t = t;
                if (part == 0) {
                    auto* to = static_cast<uint16_t*>(value ? c.v_books : c.k_books);
                    to[(row0 + (int64_t)r * c.page_size) * 16 + k] = h;
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (head0 + mine >= c.heads) continue;
        const RowBook& B = books[mine];
        const int64_t in = in0 + mine, row = row0 + (int64_t)mine * c.page_size;
        uint32_t sym[2] = {0u, 0u};
        if (B.t > 1) {
            const float x[2] = {from16<DT>(two & 0xFFFFu), from16<DT>(two >> 16)};
            uint32_t at[2] = {0u, 0u};
#pragma unroll
            for (uint32_t step = 8; step > 0; step /= 2)
#pragma unroll
                for (int e = 0; e < 2; e++)
                    if (B.s[at[e] + step] < x[e]) at[e] += step;
            const int64_t h = (in * D) / 2 + pair;
            uint32_t w[4] = {(uint32_t)h, (uint32_t)(h >> 32), value ? 3u : 2u, 0u};
            philox4x32_10(w, k0, k1);
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const double a = B.q[at[e]], N = (double)x[e] - a;
                const float d = (float)w[2 * e + 1] * 0x1p-32f - (float)N * B.over[at[e]];
                bool up = d < 0.0f;
                if (!(__builtin_fabsf(d) > 0x1p-20f))
                    up = uniform53(w[2 * e], w[2 * e + 1]) < N / (B.q[at[e] + 1] - a);
                sym[e] = at[e] + (up ? 1u : 0u);
            }
        }
        static_cast<uint8_t*>(value ? c.v : c.k)[row * (D / 2) + pair] =
            (uint8_t)(sym[0] | (sym[1] << 4));
        if (n.k_hat) {
            const uint32_t hat = B.h[sym[0]] | (uint32_t)B.h[sym[1]] << 16;
            __builtin_memcpy(static_cast<uint16_t*>(value ? n.v_hat : n.k_hat) + in * D + 2 * pair,
                             &hat, 4);
        }
    }
}

// ---------------------------------------------------------------------------
// Eviction

// Rank of a slot: larger is kept first.  A float's bits in an order that whole
// numbers have; NaN below all others, slots of recent positions above.
__device__ __forceinline__ uint32_t evict_key(float mass, int32_t pos, int64_t newest_but) {
    if ((int64_t)pos > newest_but) return 0xFFFFFFFFu;
    if (mass != mass) return 0u;
    const uint32_t b = __float_as_uint(mass + 0.0f);  // -0 as +0
    return (b >> 31) ? ~b : b | 0x80000000u;
}

// Inclusive sums over a wavefront: within rows of 16 lanes, then over the rows.
__device__ __forceinline__ int32_t wave_sums(int32_t v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
    return v;
}

// The workgroup's hold on one head's keys: every wavefront has a span of consecutive
// slots, 256 at a time and four to a lane, so that ranks in slot order are four ballots'
// and three barriers' work.  The keys are in LDS (KEYS of them); longer heads (KEYS = 0)
// read mass and pos again for every pass.  A long head is bounded by what one CU reads and
// issues (32768 slots: 34 us), a short one by the passes' latencies (640 slots: 7 us).
constexpr int kBins = 2048;
constexpr int kKeysFew = 1024, kKeysSome = 4096, kKeysMany = 32768;

struct EvictPlan {
    int32_t keep, recent, moves;  // moves: the most a head can make
    int32_t* lists;               // per head: freed slots, then moving ones, `moves` each
    int32_t* counts;              // per head: moves made
};

template <int KEYS, int T>
__global__ __launch_bounds__(T) void k_kv_evict(ecasq_kv_cache c, EvictPlan e,
                                                float* __restrict__ mass_out,
                                                int32_t* __restrict__ pos_out) {
    constexpr int kEW = T / 64, kEach = kBins / T;  // wavefronts; bins of a thread
    constexpr int kRounds = KEYS > 4 * T ? KEYS / (4 * T) : 1;
    __shared__ int32_t newest;
    __shared__ uint32_t hist[3][kBins];
    __shared__ int32_t sums[3][kEW];
    __shared__ int32_t found[3][2];
    __shared__ int4 counts[kEW];
    __shared__ uint4 keys[KEYS ? kRounds * T : 1];
    const int32_t b = blockIdx.x / c.heads;
    const int32_t slots = (int32_t)kv_slots(c), n = (int32_t)kv_len(c, b), keep = e.keep;
    const int64_t base = (int64_t)blockIdx.x * slots;
    // (these may be c.mass and c.pos; nothing is read again after it is written)
    const float* mass = c.mass + base;
    const int32_t* pos = c.pos + base;
    mass_out += base;
    pos_out += base;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    if (n <= keep) {
        if (mass_out != mass)
            for (int32_t i = threadIdx.x; i < n; i += T) mass_out[i] = mass[i];
        if (pos_out != pos)
            for (int32_t i = threadIdx.x; i < n; i += T) pos_out[i] = pos[i];
        if (threadIdx.x == 0) e.counts[blockIdx.x] = 0;
        return;
    }
    // slots start + 256 r + 4 lane .. + 3 in round r
    const int32_t rounds = (n + 4 * T - 1) / (4 * T), start = wave * rounds * 256;
    const bool copy_mass = mass_out != mass, copy_pos = pos_out != pos;
    auto read4 = [&](const auto* from, int32_t i, auto past, auto (&v)[4])
                     __attribute__((always_inline)) {
        if (i + 4 <= n) {
            __builtin_memcpy(v, from + i, 16);
        } else {
#pragma unroll
            for (int u = 0; u < 4; u++) {
                v[u] = past;
                if (i + u < n) v[u] = from[i + u];
            }
        }
    };
    // slots below keep go to the outputs as they are (the moves overwrite the freed ones)
    auto copy4 = [&](auto* to, int32_t i, const auto (&v)[4]) __attribute__((always_inline)) {
        if (i + 4 <= keep) {
            __builtin_memcpy(to + i, v, 16);
        } else {
#pragma unroll
            for (int u = 0; u < 4; u++)
                if (i + u < keep) to[i + u] = v[u];
        }
    };
    int32_t top = INT32_MIN;
    if (threadIdx.x == 0) newest = INT32_MIN;
    for (int k = threadIdx.x; k < 3 * kBins; k += T) hist[0][k] = 0u;
    float m[KEYS ? kRounds : 1][4];
    int32_t p[KEYS ? kRounds : 1][4];
    if constexpr (KEYS > 0) {
#pragma unroll
        for (int r = 0; r < kRounds; r++)
            if (r < rounds) {
                const int32_t i = start + 256 * r + 4 * lane;
                read4(mass, i, 0.0f, m[r]);
                read4(pos, i, (int32_t)INT32_MIN, p[r]);
            }
#pragma unroll
        for (int r = 0; r < kRounds; r++)
            if (r < rounds) {
                const int32_t i = start + 256 * r + 4 * lane;
                top = max(max(top, max(p[r][0], p[r][1])), max(p[r][2], p[r][3]));
                if (copy_mass) copy4(mass_out, i, m[r]);
                if (copy_pos) copy4(pos_out, i, p[r]);
            }
    } else {
#pragma unroll 2
        for (int32_t r = 0; r < rounds; r++) {
            const int32_t i = start + 256 * r + 4 * lane;
            read4(pos, i, (int32_t)INT32_MIN, p[0]);
            top = max(max(top, max(p[0][0], p[0][1])), max(p[0][2], p[0][3]));
            if (copy_pos) copy4(pos_out, i, p[0]);
            if (copy_mass) {
                read4(mass, i, 0.0f, m[0]);
                copy4(mass_out, i, m[0]);
            }
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = max(top, __shfl_xor(top, off));
    __syncthreads();
    if (lane == 0) atomicMax(&newest, top);
    __syncthreads();
    const int64_t but = (int64_t)newest - e.recent;
    // Slots past the end rank below or with the last (0), and behind all others of that rank:
    // they are never among the first `keep`.
    auto key4 = [&](int32_t i, const float (&mv)[4], const int32_t (&pv)[4])
                    __attribute__((always_inline)) {
        uint32_t k[4];
#pragma unroll
        for (int u = 0; u < 4; u++) k[u] = i + u < n ? evict_key(mv[u], pv[u], but) : 0u;
        return make_uint4(k[0], k[1], k[2], k[3]);
    };
    if constexpr (KEYS > 0) {  // (every lane's own slots, here and in every pass)
#pragma unroll
        for (int r = 0; r < kRounds; r++)
            if (r < rounds)
                keys[wave * rounds * 64 + 64 * r + lane] =
                    key4(start + 256 * r + 4 * lane, m[r], p[r]);
    }
    // f(first slot of the wavefront's, of this lane's, the lane's four keys)
    auto each = [&](auto f) __attribute__((always_inline)) {
        for (int32_t r = 0; r < rounds; r++) {
            const int32_t i0 = start + 256 * r, i = i0 + 4 * lane;
            if (i0 >= n) break;
            uint4 k;
            if constexpr (KEYS > 0) {
                k = keys[wave * rounds * 64 + 64 * r + lane];
            } else {
                read4(mass, i, 0.0f, m[0]);
                read4(pos, i, (int32_t)0, p[0]);
                k = key4(i, m[0], p[0]);
            }
            const uint32_t four[4] = {k.x, k.y, k.z, k.w};
            f(i0, i, four);
        }
    };

    // the key of the last slot that is kept, by its leading 11, 11 and 10 bits
    uint32_t prefix = 0, mask = 0;
    int32_t left = keep;  // slots to keep among those with the prefix
#pragma unroll
    for (int pass = 0; pass < 3; pass++) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
        each([&](int32_t, int32_t i, const uint32_t (&k)[4]) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < 4; u++)
                if ((k[u] & mask) == prefix && i + u < n)
                    atomicAdd(&hist[pass][(k[u] >> shift) & (bins - 1)], 1u);
        });
        __syncthreads();
        // from the top: this thread's bins, and how many slots are in those above
        const int32_t hi = bins - 1 - kEach * (int)threadIdx.x;
        int32_t h[kEach], own = 0;
#pragma unroll
        for (int k = 0; k < kEach; k++) {
            h[k] = hi > 0 ? (int32_t)hist[pass][hi - k] : 0;
            own += h[k];
        }
        int32_t run = wave_sums(own);
        if (lane == 63) sums[pass][wave] = run;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kEW; w++) {
            const int32_t v = sums[pass][w];
            run += w < wave ? v : 0;
        }
        int32_t above = run - own;
        if (above < left && left <= run) {
#pragma unroll
            for (int k = 0; k < kEach; k++) {
                if (above < left && left <= above + h[k]) {
                    found[pass][0] = hi - k;
                    found[pass][1] = left - above;
                }
                above += h[k];
            }
        }
        __syncthreads();
        prefix |= (uint32_t)found[pass][0] << shift;
        mask |= (uint32_t)(bins - 1) << shift;
        left = found[pass][1];
    }

    // Slots below keep and at or above it whose key is larger, and ties (of which the first
    // `left` are kept), in every wavefront's span; from these, what the spans before this one
    // keep, free and move.
    {
        int4 v = {0, 0, 0, 0};
        each([&](int32_t i0, int32_t i, const uint32_t (&k)[4]) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const int32_t more = k[u] > prefix, same = k[u] == prefix;
                if (i0 + 256 <= keep || (i0 < keep && i + u < keep)) {
                    v.x += more;
                    v.y += same;
                } else {
                    v.z += more;
                    v.w += same;
                }
            }
        });
        v = {wave_sums(v.x), wave_sums(v.y), wave_sums(v.z), wave_sums(v.w)};
        if (lane == 63) counts[wave] = v;
    }
    __syncthreads();
    int32_t ties = 0, some = 0, nf = 0, nm = 0, all = 0, t = 0;
#pragma unroll
    for (int w = 0; w < kEW; w++) {
        const int4 v = counts[w];
        const int32_t open = max(left - t, 0), low = min(v.y, open), high = min(v.w, open - low);
        const int32_t slots_low = min(max(keep - w * rounds * 256, 0), rounds * 256);
        if (w == wave) {
            ties = t;
            nf = all;
            some = v.y + v.w;
        }
        if (w < wave) nm += v.z + high;
        all += slots_low - v.x - low;
        t += v.y + v.w;
    }
    if (threadIdx.x == 0) e.counts[blockIdx.x] = all;
    const uint64_t below = (1ull << lane) - 1;
    int32_t* freed = e.lists + (int64_t)blockIdx.x * 2 * e.moves;
    // f(u, rank) for the lane's marked slots, ranks in slot order from `from` on; all marked in
    // the wavefront are added to it
    auto ranked = [&](const bool (&on)[4], int32_t& from, auto f) __attribute__((always_inline)) {
        int32_t at = from;
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const uint64_t v = __ballot(on[u]);
            at += __popcll(v & below);
            from += __popcll(v);
        }
#pragma unroll
        for (int u = 0; u < 4; u++)
            if (on[u]) f(u, at++);
    };
    each([&](int32_t i0, int32_t i, const uint32_t (&k)[4]) __attribute__((always_inline)) {
        bool on[4], mark[4];
#pragma unroll
        for (int u = 0; u < 4; u++) on[u] = k[u] > prefix;
        if (some) {
#pragma unroll
            for (int u = 0; u < 4; u++) mark[u] = k[u] == prefix;
            ranked(mark, ties, [&](int u, int32_t at) { on[u] = at < left; });
        }
        if (i0 < keep) {
#pragma unroll
            for (int u = 0; u < 4; u++) mark[u] = i + u < keep && !on[u];
            ranked(mark, nf, [&](int u, int32_t at) { freed[at] = i + u; });
        }
        if (i0 + 256 > keep) {
#pragma unroll
            for (int u = 0; u < 4; u++) mark[u] = i + u >= keep && on[u];
            ranked(mark, nm, [&](int u, int32_t at) { freed[e.moves + at] = i + u; });
        }
    });
}

// The moves, 64 of a head to a workgroup: where each goes from and to, then the rows
// (and their codebooks) in pieces of 16 bytes.
constexpr int kMoves = 64, kVT = 256;
typedef uint32_t Piece __attribute__((ext_vector_type(4)));

__global__ __launch_bounds__(kVT) void k_kv_move(ecasq_kv_cache c, EvictPlan e, float* mass_out,
                                                 int32_t* pos_out, int32_t* lens_out) {
    __shared__ int64_t from[kMoves], to[kMoves];
    const int32_t rows = c.batch * c.heads;
    const int32_t row = blockIdx.x % rows, m0 = blockIdx.x / rows * kMoves;
    const int32_t b = row / c.heads, head = row % c.heads;
    if (m0 == 0 && head == 0 && threadIdx.x == 0) {  // (nothing else of this kernel reads lens)
        const int64_t n = kv_len(c, b);
        lens_out[b] = (int32_t)(n < e.keep ? n : e.keep);
    }
    const int32_t count = min(e.counts[row] - m0, kMoves);
    if (count <= 0) return;
    if ((int)threadIdx.x < count) {
        const int32_t* freed = e.lists + (int64_t)row * 2 * e.moves + m0 + threadIdx.x;
        const int32_t t = freed[0], f = freed[e.moves];
        const int64_t base = (int64_t)row * kv_slots(c);
        mass_out[base + t] = c.mass[base + f];
        pos_out[base + t] = c.pos[base + f];
        const int64_t rt = kv_row(c, b, head, t), rf = kv_row(c, b, head, f);
        to[threadIdx.x] = rf < 0 ? -1 : rt;
        from[threadIdx.x] = rf;
    }
    __syncthreads();
    const int32_t piece = c.coded ? c.head_dim / 32 : c.head_dim / 8;  // of a row
    const int32_t books = c.coded ? 2 : 0, each = 2 * (piece + books);
    // A thread keeps its piece of a row for all moves, with four of them on the way at a time (no
    // row is read that another move writes); 1304 of 8 heads of 256 in 16 bits: 21 us by the
    // call with one, 17 so.
    const int32_t per = kVT / each, u0 = threadIdx.x % each;
    const bool value = u0 >= piece + books;
    const int32_t u1 = value ? u0 - piece - books : u0;
    const bool book = u1 >= piece;
    const int32_t size = book ? 2 : piece, u = book ? u1 - piece : u1;
    Piece* x = static_cast<Piece*>(book ? value ? c.v_books : c.k_books : value ? c.v : c.k) + u;
    for (int32_t m = threadIdx.x / each; m < count && threadIdx.x < per * each; m += 4 * per) {
        Piece v[4];
        int64_t at[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {  // (past the last or without a page: row 0, not written)
            const int32_t k = min(m + i * per, kMoves - 1);
            at[i] = m + i * per < count ? to[k] : -1;
            v[i] = x[(at[i] < 0 ? 0 : from[k]) * size];
        }
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (at[i] >= 0) x[at[i] * size] = v[i];
    }
}

EvictPlan evict_plan(const ecasq_kv_cache& c, int32_t keep, int32_t recent, char* ws) {
    const int64_t slots = kv_slots(c);
    EvictPlan e;
    e.keep = (int32_t)(keep < slots ? keep : slots);
    e.recent = recent;
    e.moves = (int32_t)(slots - e.keep < e.keep ? slots - e.keep : e.keep);
    e.counts = reinterpret_cast<int32_t*>(ws);
    e.lists = e.counts + (int64_t)c.batch * c.heads;
    return e;
}

}  // namespace

namespace {

template <int DT, int D>
void kv_round(const ecasq_kv_cache& c, KvNew n, hipStream_t st) {
    // Units of 128 entries: four for each wavefront of a workgroup, or fewer while there are
    // not four workgroups to a CU (152 tokens of 8 heads of 256: 6.9 us with four, 5.0 with two;
    // 4000 of 8 of 128: 30 and 32).
    const int64_t units = 2 * (((int64_t)c.heads * D + 127) / 128);
    n.units = 4 * kWT / 64;
    while (n.units > kWT / 64 && n.rows * ((units + n.units - 1) / n.units) < 1024) n.units /= 2;
    const dim3 g((unsigned)n.rows, (unsigned)((units + n.units - 1) / n.units));
    k_kv_round<DT, D><<<g, kWT, 0, st>>>(c, n);
}

template <int DT>
void kv_round(const ecasq_kv_cache& c, const KvNew& n, hipStream_t st) {
    if (c.head_dim == 64)
        kv_round<DT, 64>(c, n, st);
    else if (c.head_dim == 128)
        kv_round<DT, 128>(c, n, st);
    else
        kv_round<DT, 256>(c, n, st);
}

}  // namespace

hipError_t launch_kv_write(const ecasq_kv_cache& c, const KvNew& n, hipStream_t st) {
    if (!c.coded)
        k_kv_write<<<(unsigned)n.rows, kWT, 0, st>>>(c, n);
    else if (c.dt == ECASQ_F16)
        kv_round<1>(c, n, st);
    else
        kv_round<2>(c, n, st);
    return hipGetLastError();
}

size_t kv_evict_bytes(const ecasq_kv_cache& c, int32_t keep) {
    const EvictPlan e = evict_plan(c, keep, 0, nullptr);
    return 256 + (size_t)c.batch * c.heads * (1 + 2 * (size_t)e.moves) * sizeof(int32_t);
}

hipError_t launch_kv_evict(const ecasq_kv_cache& c, int32_t keep, int32_t recent, float* mass_out,
                           int32_t* pos_out, int32_t* lens_out, char* ws, hipStream_t st) {
    const EvictPlan e = evict_plan(c, keep, recent, ws);
    const unsigned rows = (unsigned)(c.batch * c.heads);
    // eight wavefronts up to 1024 slots, where barriers count (347 slots: 10.3 us, 11.3 with
    // sixteen; 2347: 14.1 and 13.2)
    if (kv_slots(c) <= kKeysFew)
        k_kv_evict<kKeysFew, 512><<<rows, 512, 0, st>>>(c, e, mass_out, pos_out);
    else if (kv_slots(c) <= kKeysSome)
        k_kv_evict<kKeysSome, 1024><<<rows, 1024, 0, st>>>(c, e, mass_out, pos_out);
    else if (kv_slots(c) <= kKeysMany)
        k_kv_evict<kKeysMany, 1024><<<rows, 1024, 0, st>>>(c, e, mass_out, pos_out);
    else
        k_kv_evict<0, 1024><<<rows, 1024, 0, st>>>(c, e, mass_out, pos_out);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    const unsigned parts = (unsigned)(e.moves < 1 ? 1 : (e.moves + kMoves - 1) / kMoves);
    k_kv_move<<<rows * parts, kVT, 0, st>>>(c, e, mass_out, pos_out, lens_out);
    return hipGetLastError();
}

}  // namespace ecasq
