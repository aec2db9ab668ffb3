// Shared between the host side of tsq_cache.h (tsq_cache_api.hip) and its kernels (tsq_cache_rows.hip,
// tsq_attend.hip).  Plain data, and what the kernels have in common.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace tsq {

constexpr uint32_t kMaxScheduleRequests = 4096;   // three words of LDS each in k_schedule: 48 KB

struct CacheShape {
    uint32_t blocks, block_tokens, block_log2, q_heads, kv_heads, head_dim, max_blocks;
    bool bf16;
};

struct ScheduleArgs {
    const int32_t *fresh, *lengths;
    int32_t *table, *ring;
    const int64_t *counters;
    int32_t *lengths_out;
    int64_t *counters_out;
    int32_t *starts, *positions, *slots, *status;
    uint32_t requests, capacity, blocks, block_tokens, block_log2, max_blocks;
};

struct NormRotateArgs {
    const void *q, *k, *q_weight, *k_weight;
    void *q_out, *k_out;
    const int32_t *positions;
    const float *angles;
    uint64_t q_stride, k_stride, q_out_stride, k_out_stride;
    uint32_t tokens, angle_rows, rotary, neighbours, q_heads, kv_heads;
    float eps;
};

struct AppendArgs {
    const void *x[2];            // keys, values
    uint64_t stride[2];
    int8_t *codes[2];
    float *scale[2];
    const int32_t *slots;
    uint32_t tokens, kv_heads, blocks, block_tokens, block_log2;
    uint32_t window, waves_each; // rows that are looked through for runs together, and the waves that share them
};

struct GatherArgs {
    void *out[2];
    uint64_t stride[2];
    const int8_t *codes[2];
    const float *scale[2];
    const int32_t *table, *starts, *lengths;
    uint32_t requests, tokens, kv_heads, blocks, block_tokens, block_log2, max_blocks;
    uint32_t waves_each;         // waves that share the heads of 16 rows
};

struct AttendArgs {
    const int8_t *k, *v;
    const float *k_scale, *v_scale;
    const int32_t *table, *starts, *lengths;
    const void *q;
    void *out;
    float *lse;
    float *parts;                // binary32 [part_rows][splits][head_dim] sums, then [..][splits][2] their maximum and weight
    uint64_t q_stride, out_stride, part_rows;
    uint32_t slots_each;         // rows of a kv head that a request has in the parts of that launch; 0: part_rows are rows of the output
    uint32_t requests, tokens, q_heads, kv_heads, group, blocks, block_log2, max_blocks;
    uint32_t tiles, tiles_each;  // row tiles of the call; of each request, or 0: they follow one another (see find_place)
    uint32_t splits, chunk;      // pieces of a tile's reach along the cache, and the tokens of a piece (a multiple of 128)
    uint32_t by_length;          // the requests' workgroups in the order of their lengths, the longest first (2 .. 64 requests)
    uint32_t by_tile;            // the requests' first tiles before their second ones
    uint32_t rows_from, rows_to; // a launch is for the requests with so many rows of a kv head: rows_from <= rows <= rows_to
    uint32_t window;
    int32_t causal;
    float scale_log2;            // scale * log2(e)
};

// A launch counts its threads in 32 bits: one of more is refused before anything is enqueued.
constexpr int kTooLarge = -1;    // what the functions below return then; 0, or a hipError_t, in all other cases
inline bool fits(uint64_t workgroups, uint32_t threads) { return workgroups * threads < (1ull << 32); }

// The join has both launches' parts; what the others do not need is no argument of theirs.
struct JoinArgs {
    AttendArgs a;                // of the first launch
    float *few_parts;
    uint64_t few_part_rows;
    uint32_t few_splits;         // (1: no join)
    uint32_t slots_each;         // of the second launch
};

int launch_schedule(const ScheduleArgs &a, void *stream);
int launch_norm_rotate(const CacheShape &s, const NormRotateArgs &a, void *stream);
int launch_append(const CacheShape &s, const AppendArgs &a, void *stream);
int launch_gather(const CacheShape &s, const GatherArgs &a, void *stream);
// How an attend call is split: by the shape and the caller's numbers alone, so that the workspace's size and the
// launch agree.
struct AttendLaunch {
    uint32_t rows, tiles, tiles_each, splits, chunk, by_length;
    uint64_t part_rows;
    // a second launch, for the requests of few rows among those of many, with pieces of its own
    uint32_t few_tiles;          // 0: there is none
    uint32_t few_splits, few_chunk, slots_each;
    uint64_t few_part_rows;
    uint64_t few_at, workspace;  // bytes: where the second launch's parts begin, and of both
};
AttendLaunch attend_launch(const CacheShape &s, uint32_t requests, uint32_t tokens, uint32_t max_new, uint32_t max_length,
                           uint32_t window);
int launch_attend(const CacheShape &s, const AttendLaunch &l, const AttendArgs &a, void *stream);

// f(head_dim, bfloat16 or not), both as types whose value is known when compiling.
template <class F> void by_shape(const CacheShape &s, F f) {
    auto kind = [&](auto d) { if (s.bf16) f(d, std::true_type{}); else f(d, std::false_type{}); };
    if (s.head_dim == 64) kind(std::integral_constant<int, 64>{});
    else if (s.head_dim == 128) kind(std::integral_constant<int, 128>{});
    else kind(std::integral_constant<int, 256>{});
}

#ifdef __HIPCC__
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float float16_t __attribute__((ext_vector_type(16)));
typedef uint32_t uint2_t __attribute__((ext_vector_type(2)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));

// 16-bit patterns to binary32 and back (to nearest, ties to even; a NaN stays one).
template <bool BF16> __device__ __forceinline__ float widen(uint32_t bits16) {
    if constexpr (BF16) return __builtin_bit_cast(float, bits16 << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)bits16);
}
template <bool BF16> __device__ __forceinline__ uint32_t narrow(float v) {
    if constexpr (BF16) return __builtin_bit_cast(uint16_t, (__bf16)v);
    else return __builtin_bit_cast(uint16_t, (_Float16)v);
}
template <bool BF16> __device__ __forceinline__ uint32_t narrow2(float a, float b) {
    return narrow<BF16>(a) | (narrow<BF16>(b) << 16);
}

// Four codes as halves, exactly: a byte under the exponent of 1024 is 1024 + its value, so with the sign bit
// turned the code is that less 1152.  Five instructions for four codes.
__device__ __forceinline__ half4_t codes_to_half(uint32_t w) {
    w ^= 0x80808080u;
    const half2_t off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    const half2_t a = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) + off;
    const half2_t b = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) + off;
    return half4_t{a[0], a[1], b[0], b[1]};
}
__device__ __forceinline__ float code_at(uint32_t w, int byte) { return (float)(int8_t)(w >> (8 * byte)); }
#endif

}  // namespace tsq
