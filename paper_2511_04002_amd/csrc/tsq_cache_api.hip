// Host side of include/tsq_cache.h: validation and the order of kernel launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "tsq_cache.h"
#include "tsq_cache_internal.hpp"

using namespace tsq;

struct tsq_cache {
    CacheShape s;
};

namespace {

tsq_status hip_rc(int e) { return e == 0 ? TSQ_OK : e == kTooLarge ? TSQ_ERR_UNSUPPORTED : TSQ_ERR_HIP; }
bool misaligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// rows of 16-bit elements: 16-byte aligned, a stride of whole 16-byte pieces that holds a row (any for one row)
bool bad_rows(const void *p, uint64_t stride, uint64_t row, uint32_t rows) {
    return !p || misaligned(p, 16) || stride % 8 != 0 || (rows > 1 && stride < row) || stride >= (1ull << 40);
}

bool bad_memory(const tsq_cache_memory *m) {
    return !m || !m->d_k || !m->d_v || !m->d_k_scale || !m->d_v_scale || misaligned(m->d_k, 16) || misaligned(m->d_v, 16) ||
           misaligned(m->d_k_scale, 16) || misaligned(m->d_v_scale, 16);
}

bool bad_words(const void *p) { return !p || misaligned(p, 4); }

}  // namespace

extern "C" {

tsq_status tsq_cache_create(const tsq_cache_config *cfg, tsq_cache **out) { return tsq_cache_create_bits(cfg, 8, out); }

tsq_status tsq_cache_create_bits(const tsq_cache_config *cfg, uint32_t bits, tsq_cache **out) {
    if (!cfg || !out || (bits != 8 && bits != 4)) return TSQ_ERR_INVALID_ARG;
    if (cfg->blocks == 0 || cfg->q_heads == 0 || cfg->kv_heads == 0 || cfg->head_dim == 0 || cfg->max_blocks == 0 ||
        cfg->block_tokens == 0 || cfg->reserved != 0)
        return TSQ_ERR_INVALID_ARG;
    if (cfg->dtype != TSQ_F16 && cfg->dtype != TSQ_BF16) return TSQ_ERR_INVALID_ARG;
    if (cfg->q_heads % cfg->kv_heads != 0) return TSQ_ERR_INVALID_ARG;
    const uint32_t b = cfg->block_tokens, d = cfg->head_dim;
    if ((b != 16 && b != 32 && b != 64 && b != 128) || (d != 64 && d != 128 && d != 256) || cfg->q_heads > 1024)
        return TSQ_ERR_UNSUPPORTED;
    // slots and positions are 32-bit signed
    if ((uint64_t)cfg->blocks * b >= (1ull << 31) || (uint64_t)cfg->max_blocks * b >= (1ull << 31)) return TSQ_ERR_UNSUPPORTED;
    tsq_cache *c = new (std::nothrow) tsq_cache();
    if (!c) return TSQ_ERR_NO_MEMORY;
    c->s = CacheShape{cfg->blocks, b, b == 16 ? 4u : b == 32 ? 5u : b == 64 ? 6u : 7u, cfg->q_heads, cfg->kv_heads, d,
                      cfg->max_blocks, cfg->dtype == TSQ_BF16, bits};
    *out = c;
    return TSQ_OK;
}

void tsq_cache_destroy(tsq_cache *cache) { delete cache; }

tsq_status tsq_cache_memory_sizes(const tsq_cache *c, tsq_cache_sizes *out) {
    if (!c || !out) return TSQ_ERR_INVALID_ARG;
    const uint64_t heads = (uint64_t)c->s.blocks * c->s.kv_heads, elements = heads * c->s.block_tokens * c->s.head_dim;
    out->code_bytes = c->s.bits == 4 ? elements / 2 : elements;
    out->scale_bytes = c->s.bits == 4 ? elements / 32 : 4 * heads;
    return TSQ_OK;
}

tsq_status tsq_cache_schedule(const tsq_cache *c, uint32_t requests, const void *d_new, const void *d_lengths, void *d_table,
                              void *d_ring, const void *d_counters, uint32_t capacity, void *d_lengths_out, void *d_counters_out,
                              void *d_starts, void *d_positions, void *d_slots, void *d_status, void *stream) {
    if (!c || requests == 0 || bad_words(d_new) || bad_words(d_lengths) || bad_words(d_table) || bad_words(d_ring) ||
        !d_counters || misaligned(d_counters, 8) || bad_words(d_lengths_out) || !d_counters_out || misaligned(d_counters_out, 8) ||
        bad_words(d_starts) || (capacity && (bad_words(d_positions) || bad_words(d_slots))) || bad_words(d_status) ||
        d_lengths_out == d_lengths || d_counters_out == d_counters || capacity >= (1u << 31))
        return TSQ_ERR_INVALID_ARG;
    if (requests > kMaxScheduleRequests) return TSQ_ERR_UNSUPPORTED;
    ScheduleArgs a;
    a.fresh = static_cast<const int32_t *>(d_new);
    a.lengths = static_cast<const int32_t *>(d_lengths);
    a.table = static_cast<int32_t *>(d_table);
    a.ring = static_cast<int32_t *>(d_ring);
    a.counters = static_cast<const int64_t *>(d_counters);
    a.lengths_out = static_cast<int32_t *>(d_lengths_out);
    a.counters_out = static_cast<int64_t *>(d_counters_out);
    a.starts = static_cast<int32_t *>(d_starts);
    a.positions = static_cast<int32_t *>(d_positions);
    a.slots = static_cast<int32_t *>(d_slots);
    a.status = static_cast<int32_t *>(d_status);
    a.requests = requests;
    a.capacity = capacity;
    a.blocks = c->s.blocks;
    a.block_tokens = c->s.block_tokens;
    a.block_log2 = c->s.block_log2;
    a.max_blocks = c->s.max_blocks;
    return hip_rc(launch_schedule(a, stream));
}

}  // extern "C"

namespace {

// axes 0: one row of positions, and d_axis is not used
tsq_status norm_rotate(const tsq_cache *c, uint32_t tokens, const void *d_q, uint64_t q_stride, const void *d_k, uint64_t k_stride,
                       uint32_t axes, const void *d_positions, const void *d_axis, const void *d_angles, uint32_t angle_rows,
                       uint32_t rotary, int32_t pairs, const void *d_q_weight, const void *d_k_weight, float eps, void *d_q_out,
                       uint64_t q_out_stride, void *d_k_out, uint64_t k_out_stride, void *stream) {
    if (!c || (pairs != TSQ_PAIRS_HALVES && pairs != TSQ_PAIRS_NEIGHBOURS) || !(eps >= 0.0f) || std::isinf(eps) || tokens >= (1u << 31))
        return TSQ_ERR_INVALID_ARG;
    const uint32_t d = c->s.head_dim;
    if (rotary < 16 || rotary % 16 != 0 || rotary > d) return TSQ_ERR_INVALID_ARG;
    if (tokens == 0) return TSQ_OK;
    const uint64_t qw = (uint64_t)c->s.q_heads * d, kw = (uint64_t)c->s.kv_heads * d;
    if (bad_rows(d_q, q_stride, qw, tokens) || bad_rows(d_k, k_stride, kw, tokens) || bad_rows(d_q_out, q_out_stride, qw, tokens) ||
        bad_rows(d_k_out, k_out_stride, kw, tokens) || bad_words(d_positions) || !d_angles || misaligned(d_angles, 16) ||
        misaligned(d_q_weight, 16) || misaligned(d_k_weight, 16))
        return TSQ_ERR_INVALID_ARG;
    NormRotateArgs a;
    a.q = d_q; a.k = d_k; a.q_weight = d_q_weight; a.k_weight = d_k_weight;
    a.q_out = d_q_out; a.k_out = d_k_out;
    a.positions = static_cast<const int32_t *>(d_positions);
    a.angles = static_cast<const float *>(d_angles);
    a.q_stride = q_stride; a.k_stride = k_stride; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
    a.tokens = tokens; a.angle_rows = angle_rows; a.rotary = rotary; a.neighbours = pairs == TSQ_PAIRS_NEIGHBOURS;
    a.q_heads = c->s.q_heads; a.kv_heads = c->s.kv_heads; a.eps = eps;
    a.axes = axes; a.axis = static_cast<const uint8_t *>(d_axis);
    return hip_rc(launch_norm_rotate(c->s, a, stream));
}

}  // namespace

extern "C" {

tsq_status tsq_cache_norm_rotate(const tsq_cache *c, uint32_t tokens, const void *d_q, uint64_t q_stride, const void *d_k,
                                 uint64_t k_stride, const void *d_positions, const void *d_angles, uint32_t angle_rows,
                                 uint32_t rotary, int32_t pairs, const void *d_q_weight, const void *d_k_weight, float eps,
                                 void *d_q_out, uint64_t q_out_stride, void *d_k_out, uint64_t k_out_stride, void *stream) {
    return norm_rotate(c, tokens, d_q, q_stride, d_k, k_stride, 0, d_positions, nullptr, d_angles, angle_rows, rotary, pairs, d_q_weight,
                       d_k_weight, eps, d_q_out, q_out_stride, d_k_out, k_out_stride, stream);
}

tsq_status tsq_cache_norm_rotate_axes(const tsq_cache *c, uint32_t tokens, const void *d_q, uint64_t q_stride, const void *d_k,
                                      uint64_t k_stride, uint32_t axes, const void *d_positions, const void *d_axis,
                                      const void *d_angles, uint32_t angle_rows, uint32_t rotary, int32_t pairs,
                                      const void *d_q_weight, const void *d_k_weight, float eps, void *d_q_out,
                                      uint64_t q_out_stride, void *d_k_out, uint64_t k_out_stride, void *stream) {
    if (axes == 0 || axes > kMaxAxes) return TSQ_ERR_INVALID_ARG;
    if (tokens && (!d_axis || misaligned(d_axis, 8))) return TSQ_ERR_INVALID_ARG;
    return norm_rotate(c, tokens, d_q, q_stride, d_k, k_stride, axes, d_positions, d_axis, d_angles, angle_rows, rotary, pairs, d_q_weight,
                       d_k_weight, eps, d_q_out, q_out_stride, d_k_out, k_out_stride, stream);
}

tsq_status tsq_cache_append(const tsq_cache *c, const tsq_cache_memory *m, uint32_t tokens, const void *d_k, uint64_t k_stride,
                            const void *d_v, uint64_t v_stride, const void *d_slots, void *stream) {
    if (!c || bad_memory(m) || tokens >= (1u << 31)) return TSQ_ERR_INVALID_ARG;
    if (tokens == 0) return TSQ_OK;
    const uint64_t w = (uint64_t)c->s.kv_heads * c->s.head_dim;
    if (bad_rows(d_k, k_stride, w, tokens) || bad_rows(d_v, v_stride, w, tokens) || bad_words(d_slots)) return TSQ_ERR_INVALID_ARG;
    if (c->s.bits == 4) {
        AppendFourArgs a;
        a.k = d_k; a.v = d_v; a.k_stride = k_stride; a.v_stride = v_stride;
        a.k_codes = static_cast<uint8_t *>(m->d_k); a.v_codes = static_cast<uint8_t *>(m->d_v);
        a.k_scale = static_cast<uint8_t *>(m->d_k_scale); a.v_scale = static_cast<uint8_t *>(m->d_v_scale);
        a.slots = static_cast<const int32_t *>(d_slots);
        a.tokens = tokens; a.kv_heads = c->s.kv_heads; a.blocks = c->s.blocks; a.block_log2 = c->s.block_log2;
        return hip_rc(launch_append_four(c->s, a, stream));
    }
    AppendArgs a;
    a.x[0] = d_k; a.x[1] = d_v;
    a.stride[0] = k_stride; a.stride[1] = v_stride;
    a.codes[0] = static_cast<int8_t *>(m->d_k); a.codes[1] = static_cast<int8_t *>(m->d_v);
    a.scale[0] = static_cast<float *>(m->d_k_scale); a.scale[1] = static_cast<float *>(m->d_v_scale);
    a.slots = static_cast<const int32_t *>(d_slots);
    a.tokens = tokens; a.kv_heads = c->s.kv_heads; a.blocks = c->s.blocks;
    a.block_tokens = c->s.block_tokens; a.block_log2 = c->s.block_log2;
    a.window = a.waves_each = 0;
    return hip_rc(launch_append(c->s, a, stream));
}

tsq_status tsq_cache_gather(const tsq_cache *c, const tsq_cache_memory *m, uint32_t requests, const void *d_table,
                            const void *d_starts, const void *d_lengths, uint32_t tokens, void *d_k_out, uint64_t k_out_stride,
                            void *d_v_out, uint64_t v_out_stride, void *stream) {
    if (!c || bad_memory(m) || requests == 0 || tokens >= (1u << 31) || bad_words(d_table) || bad_words(d_starts) || bad_words(d_lengths))
        return TSQ_ERR_INVALID_ARG;
    if (requests > 65535) return TSQ_ERR_UNSUPPORTED;
    if (tokens == 0) return TSQ_OK;
    const uint64_t w = (uint64_t)c->s.kv_heads * c->s.head_dim;
    if (bad_rows(d_k_out, k_out_stride, w, tokens) || bad_rows(d_v_out, v_out_stride, w, tokens)) return TSQ_ERR_INVALID_ARG;
    GatherArgs a;
    a.out[0] = d_k_out; a.out[1] = d_v_out;
    a.stride[0] = k_out_stride; a.stride[1] = v_out_stride;
    a.codes[0] = m->d_k; a.codes[1] = m->d_v;
    a.scale[0] = m->d_k_scale; a.scale[1] = m->d_v_scale;
    a.table = static_cast<const int32_t *>(d_table);
    a.starts = static_cast<const int32_t *>(d_starts);
    a.lengths = static_cast<const int32_t *>(d_lengths);
    a.requests = requests; a.tokens = tokens; a.kv_heads = c->s.kv_heads; a.blocks = c->s.blocks;
    a.block_tokens = c->s.block_tokens; a.block_log2 = c->s.block_log2; a.max_blocks = c->s.max_blocks;
    a.waves_each = 0;
    return hip_rc(c->s.bits == 4 ? launch_gather_four(c->s, a, stream) : launch_gather(c->s, a, stream));
}

size_t tsq_cache_attend_workspace_bytes(const tsq_cache *c, uint32_t requests, uint32_t tokens, uint32_t max_new, uint32_t max_length,
                                        uint32_t window) {
    if (!c || requests == 0 || tokens == 0) return 0;
    return attend_launch(c->s, requests, tokens, max_new, max_length, window).workspace;
}

tsq_status tsq_cache_attend(const tsq_cache *c, const tsq_cache_memory *m, uint32_t requests, const void *d_table,
                            const void *d_starts, const void *d_lengths, uint32_t tokens, uint32_t max_new, uint32_t max_length,
                            const void *d_q, uint64_t q_stride, float scale, int32_t causal, uint32_t window, void *d_out,
                            uint64_t out_stride, void *d_lse, void *d_ws, void *stream) {
    if (!c || bad_memory(m) || requests == 0 || bad_words(d_table) || bad_words(d_starts) || bad_words(d_lengths) ||
        !(scale > 0.0f) || std::isinf(scale) || (causal != 0 && causal != 1) || (d_lse && misaligned(d_lse, 4)))
        return TSQ_ERR_INVALID_ARG;
    if (requests > 65535 || (uint64_t)tokens * c->s.q_heads >= (1ull << 31)) return TSQ_ERR_UNSUPPORTED;
    if (tokens == 0) return TSQ_OK;
    const uint64_t w = (uint64_t)c->s.q_heads * c->s.head_dim;
    if (bad_rows(d_q, q_stride, w, tokens) || bad_rows(d_out, out_stride, w, tokens)) return TSQ_ERR_INVALID_ARG;
    const AttendLaunch l = attend_launch(c->s, requests, tokens, max_new, max_length, window);
    if (l.workspace && (!d_ws || misaligned(d_ws, 256))) return TSQ_ERR_INVALID_ARG;
    AttendArgs a;
    a.k = m->d_k; a.v = m->d_v; a.k_scale = m->d_k_scale; a.v_scale = m->d_v_scale;
    a.table = static_cast<const int32_t *>(d_table);
    a.starts = static_cast<const int32_t *>(d_starts);
    a.lengths = static_cast<const int32_t *>(d_lengths);
    a.q = d_q; a.out = d_out; a.lse = static_cast<float *>(d_lse); a.parts = static_cast<float *>(d_ws);
    a.q_stride = q_stride; a.out_stride = out_stride; a.part_rows = l.part_rows;
    a.slots_each = 0;
    a.requests = requests; a.tokens = tokens; a.q_heads = c->s.q_heads; a.kv_heads = c->s.kv_heads;
    a.group = c->s.q_heads / c->s.kv_heads; a.blocks = c->s.blocks; a.block_log2 = c->s.block_log2; a.max_blocks = c->s.max_blocks;
    a.tiles = l.tiles; a.tiles_each = l.tiles_each; a.splits = l.splits; a.chunk = l.chunk; a.by_length = l.by_length; a.by_tile = 0;
    a.rows_from = 0; a.rows_to = ~0u;
    a.window = window; a.causal = causal; a.scale_log2 = scale * 1.44269504088896340736f;
    return hip_rc(launch_attend(c->s, l, a, stream));
}

}  // extern "C"
