// Shared between the host side of tsq_cache.h (tsq_cache_api.hip) and its kernels (tsq_cache_rows.hip,
// tsq_attend.hip).  Plain data, and what the kernels have in common.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace tsq {

constexpr uint32_t kMaxScheduleRequests = 4096;   // three words of LDS each in k_schedule: 48 KB
constexpr uint32_t kMaxAxes = 4;                  // axes of a position

struct CacheShape {
    uint32_t blocks, block_tokens, block_log2, q_heads, kv_heads, head_dim, max_blocks;
    bool bf16;
    uint32_t bits;               // 8 or 4
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
    uint32_t axes;               // rows of positions; 0: one, which all pairs turn by
    const uint8_t *axis;         // [rotary / 2], with axes
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

// Of a cache in 4 bits: codes [blocks][kv_heads][block_tokens][head_dim / 2], scales [blocks][kv_heads][head_dim / 32][block_tokens].
struct AppendFourArgs {
    const void *k, *v;
    uint64_t k_stride, v_stride;
    uint8_t *k_codes, *v_codes, *k_scale, *v_scale;
    const int32_t *slots;
    uint32_t tokens, kv_heads, blocks, block_log2;
};

struct GatherArgs {
    void *out[2];
    uint64_t stride[2];
    const void *codes[2], *scale[2];
    const int32_t *table, *starts, *lengths;
    uint32_t requests, tokens, kv_heads, blocks, block_tokens, block_log2, max_blocks;
    uint32_t waves_each;         // waves that share the heads of 16 rows
};

struct AttendArgs {
    const void *k, *v, *k_scale, *v_scale;
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
    uint32_t by_length;          // the requests' workgroups in the order of their lengths, the longest first (2 .. 64 requests); n + 1: n
                                 // of them, and then the shortest first
    uint32_t by_tile;            // the requests' first tiles before their second ones
    uint32_t rows_from, rows_to; // a launch is for the requests with so many rows of a kv head: rows_from <= rows <= rows_to
    uint32_t window;
    int32_t causal;
    float scale_log2;            // scale * log2(e)
};

// A launch counts its threads in 32 bits: one of more is refused before anything is enqueued.
constexpr int kTooLarge = -1;    // what the functions below return then; 0, or a hipError_t, in all other cases
inline bool fits(uint64_t workgroups, uint32_t threads) { return workgroups * threads < (1ull << 32); }
// A grid of n waves in workgroups of four.
inline int workgroups(uint64_t waves, uint32_t *out) {
    const uint64_t n = (waves + 3) / 4;
    if (!fits(n, 256)) return kTooLarge;
    *out = (uint32_t)n;
    return 0;
}

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
int launch_append_four(const CacheShape &s, const AppendFourArgs &a, void *stream);
int launch_gather(const CacheShape &s, const GatherArgs &a, void *stream);
int launch_gather_four(const CacheShape &s, const GatherArgs &a, void *stream);
// How an attend call is split: by the shape and the caller's numbers alone, so that the workspace's size and the
// launch agree.
struct AttendLaunch {
    uint32_t rows, tiles, tiles_each, splits, chunk, by_length;     // (by_length: as in AttendArgs)
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
// The kernels of a cache in 4 bits, for tiles of `rows` rows of a kv head; once: no request has more of few rows.
void launch_attend_four(const CacheShape &s, uint32_t rows, bool once, uint32_t grid, const AttendArgs &a, void *stream);

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

// a wave's number in its workgroup, as a value that the compiler knows to be the wave's
__device__ __forceinline__ uint32_t wave_in_group() { return (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// Where the 16 rows from `begin` on of a gather lie, one a lane of each 16: the request, the block that it has there (-1: none
// that the table holds) as its nth, and the place in that.
struct GatherRow { uint32_t r, nth, place; int32_t block; bool owned; };
__device__ __forceinline__ GatherRow gather_row(const GatherArgs &a, uint64_t begin) {
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t i = (uint32_t)begin + (lane & 15);
    // the last request that begins at or before the first row, 64 requests at a time, ...
    uint32_t lo = 0, hi = a.requests;
    while (hi - lo > 1) {
        const uint32_t step = (hi - lo + 63) / 64, at = lo + lane * step;
        const uint64_t below = __ballot(at < hi && a.starts[at] <= (int32_t)begin);
        const uint32_t last = 63 - (uint32_t)__builtin_clzll(below | 1);
        hi = min(hi, lo + (last + 1) * step);
        lo += last * step;
    }
    // ... and the others' among the 64 that follow, or by search where those all begin in these rows
    const int32_t next = lo + 1 + lane < a.requests ? a.starts[lo + 1 + lane] : 0x7FFFFFFF;
    uint32_t r = lo;
    if (__builtin_expect(__ballot(next <= (int32_t)(begin + 15)) != ~0ull, 1)) {
        for (uint32_t j = 0; j < 16; ++j) {
            const uint32_t passed = (uint32_t)__builtin_popcountll(__ballot(next <= (int32_t)(begin + j)));
            if ((lane & 15) == j) r = lo + passed;
        }
    } else {
        uint32_t top = a.requests;
        while (top - r > 1) {
            const uint32_t mid = (r + top) >> 1;
            if (a.starts[mid] <= (int32_t)i) r = mid; else top = mid;
        }
    }
    const int32_t s0 = a.starts[r], s1 = a.starts[r + 1];
    const bool owned = i < a.tokens && s0 >= 0 && (int32_t)i >= s0 && (int32_t)i < s1;
    const int64_t position = (int64_t)a.lengths[r] - s1 + (int32_t)i;
    const uint32_t nth = (uint32_t)((uint64_t)position >> a.block_log2);
    int32_t block = -1;
    if (owned && position >= 0 && ((uint64_t)position >> a.block_log2) < a.max_blocks) block = a.table[(uint64_t)r * a.max_blocks + nth];
    if ((uint32_t)block >= a.blocks) block = -1;
    return GatherRow{r, nth, (uint32_t)position & (a.block_tokens - 1), block, owned};
}
#endif

}  // namespace tsq
