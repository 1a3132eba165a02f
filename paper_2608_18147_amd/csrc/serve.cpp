// Host side of the serving operators: argument checks and launches (see
// include/ecasq.h for the contract).  Nothing here allocates or waits, so every
// call can be captured into a graph.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/ecasq.h"
#include "serve.hpp"

using namespace ecasq;

namespace {

bool half_type(int dt) { return dt == ECASQ_F16 || dt == ECASQ_BF16; }

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

bool weights_ok(int64_t n_out, int64_t n_in, int64_t group) {
    constexpr int64_t most = (int64_t)1 << 24;
    return n_out >= 1 && n_out <= most && n_in >= 1 && n_in <= most &&
           n_out <= ((int64_t)1 << 40) / n_in && group >= 32 && group <= most && group % 32 == 0;
}

// The sizes alone: what the workspace functions need.
bool kv_sizes_ok(const ecasq_kv_cache* c) {
    return c && half_type(c->dt) && (c->coded == 0 || c->coded == 1) && c->heads >= 1 &&
           c->heads <= 1024 && (c->head_dim == 64 || c->head_dim == 128 || c->head_dim == 256) &&
           c->page_size >= 16 && c->page_size <= 65536 && c->page_size % 16 == 0 &&
           c->batch >= 1 && c->batch <= 65535 && (int64_t)c->batch * c->heads <= (1 << 20) &&
           c->max_pages >= 1 && c->n_pages >= 1 &&
           kv_slots(*c) <= ((int64_t)1 << 30);
}

bool kv_ok(const ecasq_kv_cache* c) {
    if (!kv_sizes_ok(c) || !c->k || !c->v || !c->table || !c->lens) return false;
    if (!aligned(c->k, 16) || !aligned(c->v, 16)) return false;
    return c->coded == 0 || (c->k_books && c->v_books && aligned(c->k_books, 16) &&
                             aligned(c->v_books, 16));
}

bool heads_ok(const ecasq_kv_cache* c, int32_t q_heads) {
    return q_heads >= c->heads && q_heads % c->heads == 0 && q_heads / c->heads <= 64 &&
           (int64_t)c->batch * q_heads <= (1 << 23);
}

// Per-slot work (weights, eviction): one launch covers all slots of all heads.
bool slots_ok(const ecasq_kv_cache* c) {
    return (int64_t)c->batch * c->heads * kv_slots(*c) <= ((int64_t)1 << 30);
}

// Do na bytes at a meet nb at b?
bool meet(const void* a, size_t na, const void* b, size_t nb) {
    const auto a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return a0 < b0 + nb && b0 < a0 + na;
}

// Do `rows` rows of `row` 16-bit entries, a_stride apart at a, meet n at b?
bool overlap(const void* a, int64_t rows, int64_t row, int64_t a_stride, const void* b, int64_t n) {
    return meet(a, 2 * ((size_t)(rows - 1) * a_stride + row), b, 2 * (size_t)n);
}

// Does a result of n bytes lie partly over its operand (NULL: there is none)?  It may be the
// operand itself.
bool partly(const void* result, const void* operand, size_t n) {
    return operand && result != operand && meet(result, n, operand, n);
}

size_t slots_bytes(const ecasq_kv_cache* c) {
    return 4 * (size_t)c->batch * c->heads * (size_t)kv_slots(*c);
}

ecasq_status status(hipError_t e) { return e == hipSuccess ? ECASQ_OK : ECASQ_EHIP; }

}  // namespace

extern "C" {

size_t ecasq_weights_size(int64_t n_out, int64_t n_in, int64_t group) {
    if (!weights_ok(n_out, n_in, group)) return 0;
    return (size_t)Weights{n_out, n_in, group}.bytes();
}

ecasq_status ecasq_weights_pack(const uint8_t* symbols, const double* codebook, int32_t t,
                                const void* scales, ecasq_dtype dt, int64_t n_out, int64_t n_in,
                                int64_t group, void* stream, void* packed, size_t packed_bytes) {
    if (!symbols || !codebook || t < 1 || t > 16 || !scales || !half_type(dt) || !packed ||
        !aligned(packed, 16) || !aligned(scales, 2) || !weights_ok(n_out, n_in, group))
        return ECASQ_EINVAL;
    const Weights w{n_out, n_in, group};
    if (packed_bytes < (size_t)w.bytes()) return ECASQ_EINVAL;
    return status(launch_weights_pack(symbols, codebook, t, scales, dt, w,
                                      static_cast<char*>(packed),
                                      static_cast<hipStream_t>(stream)));
}

ecasq_status ecasq_matvec(const void* packed, ecasq_dtype dt, int64_t n_out, int64_t n_in,
                          int64_t group, const void* x, int64_t m, int64_t x_stride, void* stream,
                          void* y) {
    if (!packed || !aligned(packed, 16) || !half_type(dt) || !weights_ok(n_out, n_in, group) ||
        !x || !y || !aligned(x, 2) || !aligned(y, 2) || m < 1 || m > ((int64_t)1 << 20) ||
        x_stride < n_in || x_stride > ((int64_t)1 << 40) ||
        overlap(x, m, n_in, x_stride, y, m * n_out))
        return ECASQ_EINVAL;
    const Weights w{n_out, n_in, group};
    if (meet(packed, (size_t)w.bytes(), y, 2 * (size_t)(m * n_out))) return ECASQ_EINVAL;
    return status(launch_matvec(static_cast<const char*>(packed), dt, w, x, m, x_stride, y,
                                static_cast<hipStream_t>(stream)));
}

ecasq_status ecasq_kv_write(const ecasq_kv_cache* c, const void* new_k, int64_t k_stride,
                            const void* new_v, int64_t v_stride, int64_t rows,
                            const int32_t* starts, const int32_t* positions, void* stream,
                            const double* k_codebooks, const int32_t* k_counts,
                            const double* v_codebooks, const int32_t* v_counts, int32_t s,
                            uint64_t seed, void* k_hat, void* v_hat) {
    if (!kv_ok(c) || !new_k || !new_v || !aligned(new_k, 2) || !aligned(new_v, 2) || !starts ||
        rows < 1 || rows > (1 << 23))
        return ECASQ_EINVAL;
    const int64_t row = (int64_t)c->heads * c->head_dim, most = (int64_t)1 << 30;
    if (k_stride < row || v_stride < row || k_stride > most || v_stride > most)
        return ECASQ_EINVAL;
    KvNew n{};
    n.k = new_k;
    n.v = new_v;
    n.k_stride = k_stride;
    n.v_stride = v_stride;
    n.rows = rows;
    n.starts = starts;
    n.positions = positions;
    if (c->coded) {
        if (!k_codebooks || !k_counts || !v_codebooks || !v_counts || s < 2 || s > 32 ||
            (k_hat == nullptr) != (v_hat == nullptr) || !aligned(k_hat, 2) || !aligned(v_hat, 2))
            return ECASQ_EINVAL;
        // (a row's entries are read before they are written; in one place, that is all)
        const int64_t all = rows * row;
        const bool k_there = k_hat == new_k && (k_stride == row || rows == 1);
        const bool v_there = v_hat == new_v && (v_stride == row || rows == 1);
        if (k_hat && (overlap(k_hat, 1, all, all, v_hat, all) ||
                      overlap(new_v, rows, row, v_stride, k_hat, all) ||
                      overlap(new_k, rows, row, k_stride, v_hat, all) ||
                      (!k_there && overlap(new_k, rows, row, k_stride, k_hat, all)) ||
                      (!v_there && overlap(new_v, rows, row, v_stride, v_hat, all))))
            return ECASQ_EINVAL;
        n.k_books = k_codebooks;
        n.v_books = v_codebooks;
        n.k_counts = k_counts;
        n.v_counts = v_counts;
        n.s = s;
        n.seed = seed;
        n.k_hat = k_hat;
        n.v_hat = v_hat;
    } else if (k_hat || v_hat) {
        return ECASQ_EINVAL;
    }
    return status(launch_kv_write(*c, n, static_cast<hipStream_t>(stream)));
}

size_t ecasq_kv_attention_workspace(const ecasq_kv_cache* c, int32_t q_heads, int32_t with_mass) {
    if (!kv_sizes_ok(c) || !heads_ok(c, q_heads) || (with_mass && !slots_ok(c))) return 0;
    return kv_attention_bytes(*c, q_heads, with_mass != 0);
}

ecasq_status ecasq_kv_attention(const ecasq_kv_cache* c, const void* q, int64_t q_stride,
                                int32_t q_heads, double scale, float* mass_out, void* stream,
                                void* out, void* workspace, size_t workspace_bytes) {
    if (!kv_ok(c) || !heads_ok(c, q_heads) || !q || !aligned(q, 2) || !out || !aligned(out, 16) ||
        q_stride < (int64_t)q_heads * c->head_dim || q_stride > ((int64_t)1 << 40) ||
        !std::isfinite((float)scale * 1.5f) || (mass_out && !slots_ok(c)))
        return ECASQ_EINVAL;
    if (!workspace || !aligned(workspace, 256)) return ECASQ_EINVAL;
    if (workspace_bytes < kv_attention_bytes(*c, q_heads, mass_out != nullptr))
        return ECASQ_EWORKSPACE;
    const int64_t row = (int64_t)q_heads * c->head_dim;
    if (overlap(q, c->batch, row, q_stride, out, c->batch * row)) return ECASQ_EINVAL;
    if (mass_out && partly(mass_out, c->mass, slots_bytes(c))) return ECASQ_EINVAL;
    return status(launch_kv_attention(*c, q, q_stride, q_heads, (float)scale, mass_out, out,
                                      static_cast<char*>(workspace),
                                      static_cast<hipStream_t>(stream)));
}

size_t ecasq_kv_evict_workspace(const ecasq_kv_cache* c, int32_t keep) {
    if (!kv_sizes_ok(c) || !slots_ok(c) || keep < 1) return 0;
    return kv_evict_bytes(*c, keep);
}

ecasq_status ecasq_kv_evict(const ecasq_kv_cache* c, int32_t keep, int32_t recent, float* mass_out,
                            int32_t* pos_out, int32_t* lens_out, void* stream, void* workspace,
                            size_t workspace_bytes) {
    if (!kv_ok(c) || !slots_ok(c) || !c->mass || !c->pos || keep < 1 || recent < 0 ||
        recent > keep || !mass_out || !pos_out || !lens_out)
        return ECASQ_EINVAL;
    if (!workspace || !aligned(workspace, 256)) return ECASQ_EINVAL;
    if (workspace_bytes < kv_evict_bytes(*c, keep)) return ECASQ_EWORKSPACE;
    const size_t n = slots_bytes(c);
    if (partly(mass_out, c->mass, n) || partly(pos_out, c->pos, n) || meet(mass_out, n, pos_out, n) ||
        meet(mass_out, n, c->pos, n) || meet(pos_out, n, c->mass, n) ||
        partly(lens_out, c->lens, 4 * (size_t)c->batch))
        return ECASQ_EINVAL;
    return status(launch_kv_evict(*c, keep, recent, mass_out, pos_out, lens_out,
                                  static_cast<char*>(workspace),
                                  static_cast<hipStream_t>(stream)));
}

}  // extern "C"
