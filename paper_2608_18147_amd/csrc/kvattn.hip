// Attention of one new token per sequence over the paged cache.
#include "half16.hpp"
#include "serve.hpp"

namespace ecasq {
namespace {

constexpr int kAT = 256;

// Entry e of the cache's row `row` of keys or values.
template <int DT, bool CODED>
__device__ __forceinline__ float entry(const void* rows, const void* books, int32_t d, int64_t row,
                                       int32_t e) {
    if (!CODED) return from16<DT>(static_cast<const uint16_t*>(rows)[row * d + e]);
    const uint32_t two = static_cast<const uint8_t*>(rows)[row * (d / 2) + e / 2];
    const uint32_t s = e % 2 ? two >> 4 : two & 15u;
    return from16<DT>(static_cast<const uint16_t*>(books)[row * 16 + s]);
}

// A workgroup per sequence and query head, 256 slots at a time with the running
// maximum and sum of the softmax.
template <int DT, bool CODED>
__global__ __launch_bounds__(kAT) void k_attend(ecasq_kv_cache c, const uint16_t* __restrict__ q,
                                                int64_t q_stride, int32_t q_heads, float scale,
                                                uint16_t* __restrict__ out,
                                                float* __restrict__ scores, float2* __restrict__ ml) {
    __shared__ float qs[256], p[kAT], red[4], part[kAT];
    const int32_t b = blockIdx.x / q_heads, h = blockIdx.x % q_heads, d = c.head_dim;
    const int32_t head = h / (q_heads / c.heads);
    const int tid = threadIdx.x;
    const int64_t n = kv_len(c, b);
    if (tid < d) qs[tid] = from16<DT>(q[b * q_stride + (int64_t)h * d + tid]);
    __syncthreads();
    float m = -INFINITY, l = 0.0f, acc = 0.0f;
    const int e = tid % d, g = tid / d, ng = kAT / d;
    for (int64_t i0 = 0; i0 < n; i0 += kAT) {
        const int64_t i = i0 + tid;
        const int64_t row = i < n ? kv_row(c, b, head, i) : -1;
        float s = -INFINITY;
        if (row >= 0) {
            float a = 0.0f;
            for (int32_t k = 0; k < d; k++)
                a += qs[k] * entry<DT, CODED>(c.k, c.k_books, d, row, k);
            s = a * scale;
        }
        if (scores && i < n) scores[(int64_t)blockIdx.x * kv_slots(c) + i] = s;
        float t = s;
        for (int off = 32; off > 0; off >>= 1) t = fmaxf(t, __shfl_xor(t, off));
        __syncthreads();
        if (tid % 64 == 0) red[tid / 64] = t;
        __syncthreads();
        const float m2 = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
        const float fix = m2 == -INFINITY ? 0.0f : m2;
        const float down = __expf(m - fix);
        m = m2;
        p[tid] = row >= 0 ? __expf(s - fix) : 0.0f;
        l = l * down + p[tid];
        acc *= down;
        __syncthreads();
        const int64_t end = n - i0 < kAT ? n - i0 : kAT;
        for (int k = g; k < end; k += ng) {
            const int64_t r = kv_row(c, b, head, i0 + k);
            if (r >= 0) acc += p[k] * entry<DT, CODED>(c.v, c.v_books, d, r, e);
        }
    }
    for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off);
    __syncthreads();
    if (tid % 64 == 0) red[tid / 64] = l;
    part[tid] = acc;
    __syncthreads();
    l = red[0] + red[1] + red[2] + red[3];
    if (tid < d) {
        float o = 0.0f;
        for (int k = 0; k < ng; k++) o += part[k * d + tid];
        out[(int64_t)blockIdx.x * d + tid] = to16<DT>(l == 0.0f ? 0.0f : o / l);
    }
    if (scores && tid == 0) ml[blockIdx.x] = make_float2(m, l);
}

// The slots' weights: the sum over the group's query heads, added to c.mass.
__global__ __launch_bounds__(kAT) void k_mass(ecasq_kv_cache c, int32_t group,
                                              const float* __restrict__ scores,
                                              const float2* __restrict__ ml, float* mass_out) {
    const int32_t b = blockIdx.y / c.heads;
    const int64_t slots = kv_slots(c), n = kv_len(c, b);
    for (int64_t i = (int64_t)blockIdx.x * kAT + threadIdx.x; i < n; i += (int64_t)gridDim.x * kAT) {
        float w = 0.0f;
        for (int32_t g = 0; g < group; g++) {
            const int64_t r = (int64_t)blockIdx.y * group + g;
            const float2 v = ml[r];
            const float s = scores[r * slots + i];
            if (v.y != 0.0f) w += __expf(s - v.x) / v.y;
        }
        const int64_t at = blockIdx.y * slots + i;
        mass_out[at] = (c.mass ? c.mass[at] : 0.0f) + w;
    }
}

size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }

}  // namespace

size_t kv_attention_bytes(const ecasq_kv_cache& c, int32_t q_heads, bool mass) {
    size_t n = 256;
    const size_t rows = (size_t)c.batch * q_heads;
    if (mass) n += align256(rows * sizeof(float2)) + rows * (size_t)kv_slots(c) * sizeof(float);
    return n;
}

hipError_t launch_kv_attention(const ecasq_kv_cache& c, const void* q, int64_t q_stride,
                               int32_t q_heads, float scale, float* mass_out, void* out, char* ws,
                               hipStream_t st) {
    const size_t rows = (size_t)c.batch * q_heads;
    auto* ml = mass_out ? reinterpret_cast<float2*>(ws) : nullptr;
    auto* scores =
        mass_out ? reinterpret_cast<float*>(ws + align256(rows * sizeof(float2))) : nullptr;
    const auto* qs = static_cast<const uint16_t*>(q);
    auto* o = static_cast<uint16_t*>(out);
    auto go = [&](auto kernel) {
        kernel<<<(unsigned)rows, kAT, 0, st>>>(c, qs, q_stride, q_heads, scale, o, scores, ml);
    };
    if (c.dt == ECASQ_F16)
        c.coded ? go(k_attend<1, true>) : go(k_attend<1, false>);
    else
        c.coded ? go(k_attend<2, true>) : go(k_attend<2, false>);
    if (mass_out) {
        const dim3 g((unsigned)((kv_slots(c) + kAT - 1) / kAT < 1024 ? (kv_slots(c) + kAT - 1) / kAT
                                                                      : 1024),
                     (unsigned)(c.batch * c.heads));
        k_mass<<<g, kAT, 0, st>>>(c, q_heads / c.heads, scores, ml, mass_out);
    }
    return hipGetLastError();
}

}  // namespace ecasq
