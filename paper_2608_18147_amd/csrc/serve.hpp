// Launchers of the operators that serve a quantized model: products with
// 4-bit weights and the paged key/value cache.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/ecasq.h"

namespace ecasq {

// ---- matvec.hip ----
// A packed matrix: 16 codebook values (32 bytes) and padding to kWHead; then for
// every tile of 16 rows and block of 128 columns 1024 bytes of symbols, 16
// for each lane l = (row l % 16, quarter q = l / 16): dword j holds columns 32 j +
// 8 q + i, i = 0 .. 7, at bits 4 i; then for every tile and group the 16 rows'
// scales.  Rows and columns past the matrix hold the first symbol of a finite value and
// scale 0.
constexpr int64_t kWHead = 256;
struct Weights {
    int64_t n_out, n_in, group;
    __host__ __device__ int64_t tiles() const { return (n_out + 15) / 16; }
    __host__ __device__ int64_t blocks() const { return (n_in + 127) / 128; }
    __host__ __device__ int64_t groups() const { return (n_in + group - 1) / group; }
    __host__ __device__ int64_t scales_at() const { return kWHead + tiles() * blocks() * 1024; }
    __host__ __device__ int64_t bytes() const { return scales_at() + tiles() * groups() * 32; }
};
hipError_t launch_weights_pack(const uint8_t* symbols, const double* codebook, int32_t t,
                               const void* scales, int dt, const Weights& w, char* packed,
                               hipStream_t st);
hipError_t launch_matvec(const char* packed, int dt, const Weights& w, const void* x, int64_t m,
                         int64_t x_stride, void* y, hipStream_t st);

// ---- kvcache.hip ----
// Where a slot's rows are: an index of rows of the cache, or -1.
__device__ __forceinline__ int64_t kv_row(const ecasq_kv_cache& c, int32_t b, int32_t head,
                                          int32_t slot) {
    const uint32_t at = (uint32_t)slot, size = (uint32_t)c.page_size;
    const int32_t page = c.table[(int64_t)b * c.max_pages + at / size];
    if (page < 0 || page >= c.n_pages) return -1;
    return ((int64_t)page * c.heads + head) * c.page_size + at % size;
}
__host__ __device__ __forceinline__ int64_t kv_slots(const ecasq_kv_cache& c) {
    return (int64_t)c.max_pages * c.page_size;
}
__device__ __forceinline__ int64_t kv_len(const ecasq_kv_cache& c, int32_t b) {
    const int64_t n = c.lens[b], most = kv_slots(c);
    return n < 0 ? 0 : n > most ? most : n;
}
struct KvNew {
    const void *k, *v;
    int64_t k_stride, v_stride, rows;
    const int32_t *starts, *positions;
    const double *k_books, *v_books;
    const int32_t *k_counts, *v_counts;
    int32_t s;
    uint64_t seed;
    void *k_hat, *v_hat;
    int32_t units;  // of a workgroup (set by the launch)
};
hipError_t launch_kv_write(const ecasq_kv_cache& c, const KvNew& n, hipStream_t st);
size_t kv_evict_bytes(const ecasq_kv_cache& c, int32_t keep);
hipError_t launch_kv_evict(const ecasq_kv_cache& c, int32_t keep, int32_t recent, float* mass_out,
                           int32_t* pos_out, int32_t* lens_out, char* ws, hipStream_t st);

// ---- kvattn.hip ----
size_t kv_attention_bytes(const ecasq_kv_cache& c, int32_t q_heads, bool mass);
hipError_t launch_kv_attention(const ecasq_kv_cache& c, const void* q, int64_t q_stride,
                               int32_t q_heads, float scale, float* mass_out, void* out, char* ws,
                               hipStream_t st);

}  // namespace ecasq
