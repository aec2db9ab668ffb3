// Attention over a cache held in 8 bits (tsq_cache_attend).
//
// With a key c_k * s_k and a value c_v * s_v (codes of the cache, and one scale for a block of tokens and a head),
//   out = sum_t w_t s_v c_v / sum_t w_t,   w_t = exp(scale * s_k * (q . c_k))
// The codes go into the matrix instructions as they are: whole numbers up to 127 are exact as halves, so q . c_k is
// exact up to its binary32 sum.  Both scales belong to 16 or more tokens in a row and stay outside: s_k multiplies
// the scores, and s_v goes into the exponent, P_t = 2^(score_t + log2 s_v - m), so that one exponential makes the
// weight that the values' codes want; the softmax's denominator takes P_t / s_v back, once for 16 tokens.  The
// reference m follows the largest exponent of a row in steps: it moves only when an exponent is more than 8 above
// what it was set for, and is then set 7 below the largest.  P is then at most 2^15, in a half's range, and
// 11-bit weights down to 2^-21 of the row's largest: the matrix instructions' operands, as fine as an output of binary16
// and three bits finer than one of bfloat16.  The denominator adds the weights as they are before that rounding.
//
// Scores are computed transposed, S^T = K Q^T: a lane then has all its scores in one row of the softmax (a query),
// and the registers that hold P^T are, in the order they are in, an operand of O^T = V^T P^T.  A matrix
// instruction does not care which tokens its k index stands for as long as both operands agree, so the tokens of
// a tile are dealt to the lanes such that nothing has to be moved.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "tsq_attend.hpp"

namespace tsq {
namespace {

constexpr float kRoom = 7.0f;        // the reference is set this far below the largest exponent ...
constexpr float kSlack = 8.0f;       // ... and kept until one exceeds that by as much
constexpr float kCoarse = 0x1p22f;   // beyond this a reference's last bit is worth 1/2 or more: the difference of a score that
                                     // is not rounded and one that is would pass a half's range

// What the tokens of a block have in common for a head: the factor of the scores, and the values' scale as log2 and
// as reciprocal.  Values that are all 0 weigh nothing whatever their scale is: 2^-60 keeps their tokens in the
// denominator without touching the reference of the others.
//
// A row's exponents hold scales of 2^-60 to 2^40 together, all that values of magnitudes from 2^-53 to 2^47 bring: with
// scales farther apart, tokens of small ones would be lost from the denominator, and of scales below about 2^-110 it would
// pass binary32's range.  A tile that meets others is gone through twice more: once for the softmax of the scores
// alone (kScores), and once for the sums of the values (kValues), each with a reference of its own, in 2.4 to 2.7 times the time.
enum Mode : uint32_t { kAll, kScores, kValues };
__device__ __forceinline__ bool is_far(float log_v) { return fabsf(log_v + 10.0f) > 50.0f; }
struct Scale { float k, v; bool bad; };
__device__ __forceinline__ Scale scale_at(const AttendArgs &a, const Place &p, uint32_t entry) {
    const uint64_t at = (uint64_t)id_of(a, entry) * a.kv_heads + p.h;
    return Scale{static_cast<const float *>(a.k_scale)[at], static_cast<const float *>(a.v_scale)[at], is_bad(a, p, entry)};
}
struct Block { float c, log_v, back_v; };
__device__ __forceinline__ Block block_of(Scale s, float row_factor, uint32_t mode) {
    const float v = s.v == 0.0f || s.bad ? 0x1p-60f : s.v;         // (what is read for a block that there is not may be anything)
    Block b{s.bad ? __builtin_nanf("") : s.k * row_factor, log2_of(v), 1.0f / v};
    if (mode == kScores) { b.log_v = s.v - s.v; b.back_v = 1.0f; }           // (0, or NaN)
    if (mode == kValues && s.v == 0.0f) b.log_v = -INFINITY;
    return b;
}
struct Softmax { float ref, weight; };                   // of a row, from kScores

// What a row ends with: its statistics, and what its sums are to be multiplied by, f h h (h twice, since binary32 may
// not hold its square).  The sums of a piece along the cache stay as they are; from kValues they become an average, which
// goes to the join at 2^-10 of its size, so that the join can add a thousand of them.
struct Ending { float top, total, f, h; };
__device__ __forceinline__ Ending ending(const AttendArgs &a, uint32_t mode, float top, float total, Softmax x) {
    Ending e{top, total, 1.0f, 1.0f};
    if (mode == kValues) {
        e.top = x.ref;
        e.total = x.weight;
        e.h = x.weight == 0.0f ? 0.0f : pow2(0.5f * (top - x.ref));
    }
    const float back = e.total == 0.0f ? 0.0f : 1.0f / e.total;
    if (a.splits == 1) e.f = back;
    else if (mode == kValues) {
        e.f = back * 0x1p-10f;
        e.top = x.weight == 0.0f ? kNone : x.ref + log2_of(x.weight) + 10.0f;
        e.total = x.weight * e.f;
    }
    return e;
}

// A query's 16-bit elements as halves, and what the scores are to be multiplied by for it: binary16 as it is,
// bfloat16 at a power of two that brings the row's largest element to 2^13 .. 2^14, which leaves every bit of
// elements down to 2^-27 of it.
template <bool BF16>
__device__ __forceinline__ half8_t query_piece(uint4_t w, float f) {
    if constexpr (!BF16) return __builtin_bit_cast(half8_t, w);
    else {
        half8_t o;
        for (int i = 0; i < 4; ++i) {
            o[2 * i] = (_Float16)(widen<true>(w[i] & 0xFFFFu) * f);
            o[2 * i + 1] = (_Float16)(widen<true>(w[i] >> 16) * f);
        }
        return o;
    }
}
__device__ __forceinline__ uint32_t piece_most(uint4_t w) {
    uint32_t m = 0;
    for (int i = 0; i < 4; ++i) m = max(m, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
    return m;
}
// largest magnitude's bits (bfloat16) -> the factor that its row is multiplied by; `back` undoes it
__device__ __forceinline__ float query_factor(uint32_t most, float &back) {
    int e = (int)(most >> 7) - 127;
    if (e > 127) e = 13;             // a NaN or infinity shows in any case
    if (e < -100) e = -100;
    back = __builtin_bit_cast(float, (uint32_t)(e - 13 + 127) << 23);
    return __builtin_bit_cast(float, (uint32_t)(13 - e + 127) << 23);
}

// Few rows: 16 of a kv head's, or 32 (SETS = 2, which share the codes once they are halves).  Each of four waves takes
// every fourth tile of 64 tokens straight from memory to registers and keeps a softmax of its own; they meet in LDS at
// the end.
// Lane (m = lane % 16, g = lane / 16).  The tokens of a tile: group g has 16g .. 16g + 15, all of one block.
//   S^T tile t (16 tokens x 16 rows): row 4g + i is token 16g + 4t + i, so that a lane's 16 scores (t, i) are the
//   16 tokens of its group, in the order of its 16 bytes of a value's row; its row of the softmax is m.
//   Keys: operand row m is token 16 (m / 4) + 4t + m % 4; the lane's k indices are the elements 64f + 16g .. + 15.
//
// The cache's bytes bound it: 64 requests of 1024 to 4096 tokens on 40 heads of 128, blocks of 16, are 1.79 GB and
// 297 to 303 us, 5.9 to 6.0 TB/s.  The same 2 KB pieces read and thrown away take 300 us, 283 with the longest request first; a
// stream of reads reaches 7.0 TB/s.  One query of 64 heads on 8 over 131072 tokens: 269 MB, 56 us with the
// join.  With two sets a wave does twice the exponents, maxima and sums for the same bytes, two waves a SIMD: 4 queries of
// 32 requests over 8192 tokens, 64 heads on 8, are 537 MB and 130 us, 8 of 16 requests over 4096, in two tiles, 134 MB
// and 48.
template <int D, bool BF16, int SETS>
__global__ __launch_bounds__(256, D == 256 ? 1 : D == 128 || SETS == 2 ? 2 : 3) void k_attend_few(AttendArgs a) {
    constexpr int F = D / 64;                            // 64-element pieces of a head
    constexpr int ROWS = 16 * SETS;
    __shared__ alignas(16) float sums[4][16][132];
    __shared__ float stats[4][16][2];
    __shared__ Softmax softmax[ROWS];                    // (of the pass kScores)
    __shared__ uint32_t far[4];
    Place p;
    if (!find_place<ROWS>(a, p)) return;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
    const uint32_t B = 1u << a.block_log2;
    uint32_t mode = kAll;
    for (uint32_t tile = p.tile;;) {
        const AttendArgs here = SETS == 2 || D == 256 ? args_again() : a;
        const uint32_t rows = p.n * here.group;
        const Reach reach = reach_of<ROWS>(here, p, tile);
        const bool done = !p.last || (uint64_t)(tile + 1) * ROWS >= rows;
        if (here.splits > 1 && reach.begin >= reach.end) {
            nothing_seen<ROWS>(here, p, tile, D);
            if (done) return;
            ++tile;
            continue;
        }
        half8_t q[SETS][F][2];
        float back[SETS];
        uint32_t from[SETS], to[SETS];
#pragma unroll
        for (int c = 0; c < SETS; ++c) {
            const uint32_t row = tile * ROWS + 16 * c + m;
            uint4_t w[F][2];
            uint32_t most = 0;
            for (int f = 0; f < F; ++f)
                for (int e = 0; e < 2; ++e) {
                    w[f][e] = uint4_t{0, 0, 0, 0};
                    if (row < rows) {
                        const uint16_t *src = static_cast<const uint16_t *>(here.q) + (uint64_t)(p.begin + row / a.group) * here.q_stride +
                                              (uint64_t)(p.h * a.group + row % a.group) * D + 64 * f + 16 * g + 8 * e;
                        w[f][e] = *reinterpret_cast<const uint4_t *>(src);
                    }
                    most = max(most, piece_most(w[f][e]));
                }
            float factor = 1.0f;
            back[c] = 1.0f;
            if constexpr (BF16) {
                most = max(most, (uint32_t)__shfl_xor((int)most, 16));
                most = max(most, (uint32_t)__shfl_xor((int)most, 32));
                factor = query_factor(most, back[c]);
            }
            for (int f = 0; f < F; ++f)
                for (int e = 0; e < 2; ++e) q[c][f][e] = query_piece<BF16>(w[f][e], factor);
            row_sees(here, p, row, from[c], to[c]);
        }

        float4_t acc[SETS][D / 16];
        float ref[SETS], weight[SETS];
        bool met_far = false;
#pragma unroll
        for (int c = 0; c < SETS; ++c) {
            for (int d = 0; d < D / 16; ++d) acc[c][d] = float4_t{0, 0, 0, 0};
            ref[c] = kNone;
            weight[c] = 0.0f;
        }

        // Loads are always on their way: a tile's keys are asked for while the tile before it is worked on, its values
        // when that one's are used up, and its block numbers a tile earlier still.
        uint4_t kw[4][F], vw[D / 16];
        Scale scale = {};
        const int8_t *my_keys = static_cast<const int8_t *>(a.k) + (m & 3) * D + 16 * g;
        auto ask_keys = [&](uint32_t t0, uint32_t entry) {
            const uint32_t key_id = (uint32_t)__shfl((int)id_of(a, entry), (int)(m >> 2) << 4), token = t0 + 16 * (m >> 2);
            const int8_t *keys = my_keys + (((uint64_t)key_id * a.kv_heads + p.h) * B + (token & (B - 1))) * D;
            scale = scale_at(a, p, entry);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                for (int f = 0; f < F; ++f) kw[t][f] = *reinterpret_cast<const uint4_t *>(keys + 4 * t * D + 64 * f);
        };
        auto ask_values = [&](uint32_t t0, uint32_t entry) {
            const int8_t *values = static_cast<const int8_t *>(a.v) + (((uint64_t)id_of(a, entry) * a.kv_heads + p.h) * D + m) * B + ((t0 + 16 * g) & (B - 1));
#pragma unroll
            for (int d = 0; d < D / 16; ++d) vw[d] = *reinterpret_cast<const uint4_t *>(values + (uint64_t)(16 * d) * B);
        };
        uint32_t t0 = reach.begin + 64 * wave, next = 0;
        if (t0 < reach.end) {
            const uint32_t entry = table_entry(a, p, t0 + 16 * g, reach.end, reach.first);
            next = table_entry(a, p, t0 + 256 + 16 * g, reach.end);
            ask_keys(t0, entry);
            ask_values(t0, entry);
        }
        for (; t0 < reach.end; t0 += 256) {
            float4_t s[SETS][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                for (int c = 0; c < SETS; ++c) s[c][t] = float4_t{0, 0, 0, 0};
                for (int f = 0; f < F; ++f)
                    for (int e = 0; e < 2; ++e) {
                        const half4_t x = codes_to_half(kw[t][f][2 * e]), y = codes_to_half(kw[t][f][2 * e + 1]);
                        const half8_t k = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
                        for (int c = 0; c < SETS; ++c) s[c][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[c][f][e], s[c][t], 0, 0, 0);
                    }
            }
            const Block b = block_of(scale, a.scale_log2, mode);
            met_far |= is_far(b.log_v);
            const uint32_t entry = next;
            ask_keys(t0 + 256, entry);
            next = table_entry(a, p, t0 + 512 + 16 * g, reach.end);
            // exponents, and the reference
            const uint32_t mine = t0 + 16 * g;
            half8_t pw[SETS][2];
#pragma unroll
            for (int c = 0; c < SETS; ++c) {
                const bool whole = __ballot(mine < from[c] || mine + 16 > to[c]) == 0;
                const float f = BF16 ? b.c * back[c] : b.c;
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    for (int i = 0; i < 4; ++i) s[c][t][i] = __builtin_fmaf(s[c][t][i], f, b.log_v);
                if (!whole) {
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t token = mine + 4 * t + i;
                            s[c][t][i] = token < from[c] || token >= to[c] ? -INFINITY : s[c][t][i];
                        }
                }
                float top = -INFINITY;
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, s[c][t][i]);
                top = fmaxf(top, __shfl_xor(top, 16));
                top = max_across_halves(top);
                if (__ballot(top > ref[c] + (kRoom + kSlack))) {
                    const float now = fmaxf(ref[c], top - kRoom), down = pow2(ref[c] - now);
                    ref[c] = now;
                    weight[c] *= down;
                    for (int d = 0; d < D / 16; ++d) acc[c][d] *= down;
                }
                float sum = 0.0f;
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    for (int i = 0; i < 4; ++i) {
                        const float e = pow2(s[c][t][i] - ref[c]);
                        sum += e;
                        pw[c][t / 2][4 * (t & 1) + i] = (_Float16)e;
                    }
                // (a group that a row sees nothing of stays out, whatever its scale is)
                weight[c] += sum == 0.0f ? 0.0f : sum * b.back_v;
            }
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
                for (int u = 0; u < 2; ++u) {
                    const half4_t x = codes_to_half(vw[d][2 * u]), y = codes_to_half(vw[d][2 * u + 1]);
                    const half8_t v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
                    for (int c = 0; c < SETS; ++c) acc[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pw[c][u], acc[c][d], 0, 0, 0);
                }
            ask_values(t0 + 256, entry);
        }

        // the four waves' sums, at one reference
        const bool any_far = __ballot(met_far) != 0;
        if (lane == 0) far[wave] = mode == kAll && any_far;
        bool again = false;
#pragma unroll
        for (int c = 0; c < SETS; ++c) {
            weight[c] += __shfl_xor(weight[c], 16);
            weight[c] += __shfl_xor(weight[c], 32);
            if (c) __syncthreads();
            if (g == 0) { stats[wave][m][0] = ref[c]; stats[wave][m][1] = weight[c]; }
            __syncthreads();
            if (c == 0) again = (far[0] | far[1] | far[2] | far[3]) != 0;
            if (again) break;
            const float all = fmaxf(fmaxf(stats[0][m][0], stats[1][m][0]), fmaxf(stats[2][m][0], stats[3][m][0]));
            const float mine = pow2(ref[c] - all);
            const uint32_t out_row = threadIdx.x >> 4, piece = threadIdx.x & 15, o = tile * ROWS + 16 * c + out_row;
            float total = 0.0f, top = fmaxf(fmaxf(stats[0][out_row][0], stats[1][out_row][0]), fmaxf(stats[2][out_row][0], stats[3][out_row][0]));
            for (int w = 0; w < 4; ++w) total += stats[w][out_row][1] * pow2(stats[w][out_row][0] - top);
            if (is_lost(a, p, o)) total = __builtin_nanf("");
            if (mode == kScores) {
                if (piece == 0) softmax[16 * c + out_row] = Softmax{top, total};
                continue;
            }
            const AttendArgs e = SETS == 2 || D == 256 ? args_again() : a;
            const Ending end = ending(e, mode, top, total, softmax[16 * c + out_row]);
            const uint64_t id = e.splits == 1 ? row_id(e, p, o) : part_row(e, p, o);
            for (int part = 0; part < (D + 127) / 128; ++part) {
                constexpr int N = D < 128 ? D : 128;     // elements at a time
                if (part) __syncthreads();
                for (int d = 0; d < N / 16; ++d) *reinterpret_cast<float4_t *>(&sums[wave][m][16 * d + 4 * g]) = acc[c][part * 8 + d] * mine;
                __syncthreads();
                if (piece * 8 < N && o < rows) {
                    float y[8];
                    for (int i = 0; i < 8; ++i) {
                        y[i] = sums[0][out_row][8 * piece + i] + sums[1][out_row][8 * piece + i] + sums[2][out_row][8 * piece + i] + sums[3][out_row][8 * piece + i];
                        y[i] = y[i] * end.f * end.h * end.h;
                    }
                    if (e.splits == 1) {
                        uint4_t w;
                        for (int i = 0; i < 4; ++i) w[i] = narrow2<BF16>(y[2 * i], y[2 * i + 1]);
                        uint16_t *dst = static_cast<uint16_t *>(e.out) + (uint64_t)(p.begin + o / e.group) * e.out_stride +
                                        (uint64_t)(p.h * e.group + o % e.group) * D + part * 128 + piece * 8;
                        *reinterpret_cast<uint4_t *>(dst) = w;
                    } else {
                        float *dst = e.parts + (id * e.splits + p.split) * D + part * 128 + piece * 8;
                        *reinterpret_cast<float4_t *>(dst) = float4_t{y[0], y[1], y[2], y[3]};
                        *reinterpret_cast<float4_t *>(dst + 4) = float4_t{y[4], y[5], y[6], y[7]};
                    }
                }
            }
            if (piece == 0 && o < rows) {
                if (e.splits > 1) {
                    float *dst = e.parts + e.part_rows * e.splits * D + (id * e.splits + p.split) * 2;
                    dst[0] = end.top;
                    dst[1] = end.total;
                } else if (e.lse) {
                    e.lse[id] = end.total == 0.0f ? -INFINITY : (end.top + log2_of(end.total)) * 0.69314718055994530942f;
                }
            }
        }
        if (again || mode == kScores) {
            mode = again ? kScores : kValues;
        } else {
            if (done) return;
            mode = kAll;
            ++tile;
        }
        __syncthreads();
    }
}

// Many rows: 32 of a kv head's a wave, eight waves a workgroup (four, where a request has no more than 128 rows, and for
// heads of 256, whose sums and queries take the registers of two).  A tile of 128 tokens (64) goes through registers
// into LDS, as halves, once for all rows: the threads convert a share of it each, and one barrier a tile is all that
// they wait for.  A piece from LDS feeds one product of 32 x 32 x 16, so LDS is read at about half its rate.
//
// Instruction issue bounds it: a wave's 64 tokens by 32 rows of 128 are 1024 cycles of products, and some 1300 of
// exponentials, maxima, sums, conversions and addresses, which run beside them only as far as two waves of a SIMD
// complement each other (a product keeps 12 cycles of issue from the other wave).  8192 queries over as many tokens,
// causal, 64 heads on 8 of 128: 1.10 PFLOP in 1.12 to 1.14 ms, 0.96 to 0.99 PFLOP/s; a large library product of halves
// reaches 1.2.  Heads of 64 have the exponentials of 128 for half the products: 0.69 PFLOP/s (two requests of 8000 tokens,
// 20 heads).  Heads of 256 leave registers for one wave a SIMD, whose products nothing runs beside: 0.59 to 0.63 PFLOP/s (4096
// tokens, 16 heads on 8).  Chunks: 512 queries after 7680, 64 heads on 8, 154 us, 0.87 PFLOP/s; 300 after 4000 of four
// requests, 32 on 8, 122 us, 0.67 (160 workgroups for 256 places).
// The maxima could be left out of nearly all tiles, since the sums of the weights show when the reference is too low;
// the second pass that this needs costs more registers than there are (spilled, 1.44 ms).
// Lane (n = lane % 32, hi = lane / 32).  S^T in two 32 x 32 pieces: register i of a piece is token
// 8 (i / 4) + 4 hi + i % 4, row n.  P^T as an operand of 16 tokens wants eight of them from each half of the wave:
// registers 8u .. 8u + 7 are tokens 4 hi + (0..3) and 8 + 4 hi + (0..3) of the 16, so the values' rows in LDS hold
// each 16 tokens in the order 0-3, 8-11, 4-7, 12-15.
template <int D, int TOKENS>
struct alignas(16) ManyTile {                            // rows padded by 16 bytes: neighbours begin four banks apart
    _Float16 k[TOKENS][D + 8];
    _Float16 v[D][TOKENS + 8];
    float factor[TOKENS / 16], log_v[TOKENS / 16], back_v[TOKENS / 16];      // of each 16 tokens
};

// How a block's N loads from LDS and N products are to be issued: four loads, then one behind each product.
template <int N, int GROUP> __device__ __forceinline__ void loads_among_products() {
    constexpr int kLoad = 0x100, kProduct = 0x8;
    __builtin_amdgcn_sched_group_barrier(kLoad, 4, GROUP);
#pragma unroll
    for (int i = 0; i < N - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(kProduct, 1, GROUP);
        __builtin_amdgcn_sched_group_barrier(kLoad, 1, GROUP);
    }
    __builtin_amdgcn_sched_group_barrier(kProduct, 4, GROUP);
}

template <int D, bool BF16, int WAVES, int TOKENS>
__global__ __launch_bounds__(64 * WAVES, D == 256 ? 1 : 2) void k_attend_many(AttendArgs a) {
    constexpr int ROWS = 32 * WAVES, THREADS = 64 * WAVES, SUBS = TOKENS / 16;
    constexpr int N = TOKENS * D / 16 / THREADS;         // 16-byte pieces of keys, and of values, that a thread stages
    typedef ManyTile<D, TOKENS> Tile;
    __shared__ Tile buffer[2];
    __shared__ Softmax softmax[ROWS];                    // (of the pass kScores)
    __shared__ uint32_t far;
    Place p;
    if (!find_place<ROWS>(a, p)) return;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6)), n = lane & 31, hi = lane >> 5;
    const uint32_t B = 1u << a.block_log2;
    uint32_t mode = kAll;
    for (uint32_t tile = p.tile;;) {
        const uint32_t row = tile * ROWS + wave * 32 + n, rows = p.n * a.group;
        const Reach reach = reach_of<ROWS>(a, p, tile);
        const bool done = !p.last || (uint64_t)(tile + 1) * ROWS >= rows;
        if (a.splits > 1 && reach.begin >= reach.end) {
            nothing_seen<ROWS>(a, p, tile, D);
            if (done) return;
            ++tile;
            continue;
        }
        half8_t q[D / 16];
        float back = 1.0f;
        {
            uint4_t w[D / 16];
            uint32_t most = 0;
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                w[s] = uint4_t{0, 0, 0, 0};
                if (row < rows) {
                    const uint16_t *src = static_cast<const uint16_t *>(a.q) + (uint64_t)(p.begin + row / a.group) * a.q_stride +
                                          (uint64_t)(p.h * a.group + row % a.group) * D + 16 * s + 8 * hi;
                    w[s] = *reinterpret_cast<const uint4_t *>(src);
                }
                most = max(most, piece_most(w[s]));
            }
            float factor = 1.0f;
            if constexpr (BF16) {
                most = max(most, (uint32_t)__shfl_xor((int)most, 32));
                factor = query_factor(most, back);
            }
#pragma unroll
            for (int s = 0; s < D / 16; ++s) q[s] = query_piece<BF16>(w[s], factor);
        }
        uint32_t from, to;
        row_sees(a, p, row, from, to);

        float16_t acc[D / 32];
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
            for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;
        float ref = kNone, weight = 0.0f;
        bool coarse = false;         // some row's reference, a finite one, is too large for an exponent to be made in one rounding

        // staging: what this thread brings of a tile
        // (a thread's places in a block are the same for all tiles, but for the half of a block of 128 tokens)
        uint32_t key_entry[N], value_entry = 0;
        uint4_t kw[N], vw[N];
        const uint32_t block_bytes = a.kv_heads * B * D;
        const int8_t *keys[N], *values[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t e = i * THREADS + tid;
            keys[i] = static_cast<const int8_t *>(a.k) + (uint64_t)p.h * B * D + (e / (D / 16) & (B - 1)) * D + 16 * (e % (D / 16));
            values[i] = static_cast<const int8_t *>(a.v) + (uint64_t)p.h * B * D + (uint64_t)(e / SUBS) * B + (16 * (tid % SUBS) & (B - 1));
        }
        Scale scale = {};
        auto ask_entries = [&](uint32_t t0, uint32_t from) {
#pragma unroll
            for (int i = 0; i < N; ++i) key_entry[i] = table_entry(a, p, t0 + (i * THREADS + tid) / (D / 16), reach.end, from);
            value_entry = table_entry(a, p, t0 + 16 * (tid % SUBS), reach.end, from);
        };
        auto ask = [&](uint32_t t0) {
            const uint32_t half = t0 & (B - 1);
#pragma unroll
            for (int i = 0; i < N; ++i) kw[i] = *reinterpret_cast<const uint4_t *>(keys[i] + ((uint64_t)id_of(a, key_entry[i]) * block_bytes + half * D));
            const uint64_t at = (uint64_t)id_of(a, value_entry) * block_bytes + half;
#pragma unroll
            for (int i = 0; i < N; ++i) vw[i] = *reinterpret_cast<const uint4_t *>(values[i] + at);
            if (tid < SUBS) scale = scale_at(a, p, value_entry);
        };
        auto put = [&](Tile &t) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t e = i * THREADS + tid;
                half4_t h[4];
                for (int j = 0; j < 4; ++j) h[j] = codes_to_half(kw[i][j]);
                _Float16 *to_k = &t.k[e / (D / 16)][16 * (e % (D / 16))];
                *reinterpret_cast<half8_t *>(to_k) = __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
                *reinterpret_cast<half8_t *>(to_k + 8) = __builtin_shufflevector(h[2], h[3], 0, 1, 2, 3, 4, 5, 6, 7);
                for (int j = 0; j < 4; ++j) h[j] = codes_to_half(vw[i][j]);
                _Float16 *to_v = &t.v[e / SUBS][16 * (e % SUBS)];
                *reinterpret_cast<half8_t *>(to_v) = __builtin_shufflevector(h[0], h[2], 0, 1, 2, 3, 4, 5, 6, 7);
                *reinterpret_cast<half8_t *>(to_v + 8) = __builtin_shufflevector(h[1], h[3], 0, 1, 2, 3, 4, 5, 6, 7);
            }
            if (tid < SUBS) {
                const Block b = block_of(scale, a.scale_log2, mode);
                t.factor[tid] = b.c;
                t.log_v[tid] = b.log_v;
                t.back_v[tid] = b.back_v;
                if (is_far(b.log_v)) far = 1;
            }
        };

        // What a tile brings is asked for a tile ahead and put into the other buffer when the present one is worked on.
        if (tid == 0) far = 0;       // (the threads that may set it are of this wave)
        if (reach.begin < reach.end) {
            ask_entries(reach.begin, reach.first);
            ask(reach.begin);
            ask_entries(reach.begin + TOKENS, TOKENS < 128 ? reach.first : 0);
            put(buffer[0]);
            ask(reach.begin + TOKENS);
            ask_entries(reach.begin + 2 * TOKENS, 0);
        }
        __syncthreads();
        uint32_t at = 0;
        for (uint32_t t0 = reach.begin; t0 < reach.end; t0 += TOKENS, at ^= 1) {
            const Tile &t = buffer[at];
#pragma unroll
            for (uint32_t part = 0; part < TOKENS; part += 64) {
                const uint32_t u0 = t0 + part;
                // (a wave whose rows all end before these tokens, or begin behind them, only helps to stage)
                if (!__ballot(from < u0 + 64 && to > u0)) continue;
                float16_t s[2];
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    for (int i = 0; i < 16; ++i) s[c][i] = 0.0f;
#pragma unroll
                    for (int e = 0; e < D / 16; ++e)
                        s[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const half8_t *>(&t.k[part + 32 * c + n][16 * e + 8 * hi]), q[e], s[c], 0, 0, 0);
                }
                loads_among_products<2 * D / 16, 0>();
                __builtin_amdgcn_s_setprio(0);
                const bool whole = __ballot(u0 < from || u0 + 64 > to) == 0;
                const float4_t ks = *reinterpret_cast<const float4_t *>(t.factor + part / 16);
                float4_t lv = *reinterpret_cast<const float4_t *>(t.log_v + part / 16);
                const float4_t bv = *reinterpret_cast<const float4_t *>(t.back_v + part / 16);
                if (!whole) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        for (int i = 0; i < 16; ++i) {
                            const uint32_t token = u0 + 32 * c + 8 * (i / 4) + 4 * hi + i % 4;
                            if (token < from || token >= to) s[c][i] = -INFINITY;
                        }
                }
                float factor[4], top = -INFINITY;
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    float m = s[b / 2][8 * (b & 1)];
                    for (int i = 1; i < 8; ++i) m = fmaxf(m, s[b / 2][8 * (b & 1) + i]);
                    factor[b] = BF16 ? ks[b] * back : ks[b];
                    // (-inf times a scale of 0 is a NaN, which the maximum passes over)
                    top = fmaxf(top, __builtin_fmaf(m, factor[b], lv[b]));
                }
                top = max_across_halves(top);
                if (coarse || __ballot(top > ref + (kRoom + kSlack))) {
                    const float now = fmaxf(ref, top - kRoom), down = pow2(ref - now);
                    ref = now;
                    weight *= down;
#pragma unroll
                    for (int d = 0; d < D / 32; ++d) acc[d] *= down;
                    coarse = __ballot(fabsf(ref) > kCoarse && fabsf(ref) < -kNone) != 0;
                    if (coarse) {                        // the reference is rounded: so is, in its row, what it is taken from
                        const bool here = fabsf(ref) > kCoarse;
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            for (int i = 0; i < 8; ++i) {
                                const float x = s[b / 2][8 * (b & 1) + i];
                                s[b / 2][8 * (b & 1) + i] = here ? __builtin_fmaf(x, factor[b], lv[b]) - ref : x;
                            }
                            factor[b] = here ? 1.0f : factor[b];
                            lv[b] = here ? ref : lv[b];
                        }
                    }
                }
                half8_t pw[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const float off = lv[b] - ref;
                    for (int i = 0; i < 8; ++i) s[b / 2][8 * (b & 1) + i] = pow2(__builtin_fmaf(s[b / 2][8 * (b & 1) + i], factor[b], off));
                }
                if (!whole) {                            // (a factor of 0 or NaN has made NaN of -inf)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        for (int i = 0; i < 16; ++i) {
                            const uint32_t token = u0 + 32 * c + 8 * (i / 4) + 4 * hi + i % 4;
                            if (token < from || token >= to) s[c][i] = 0.0f;
                        }
                }
                float sum[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const float16_t &e = s[b / 2];
                    const int o = 8 * (b & 1);
                    sum[b] = ((e[o] + e[o + 1]) + (e[o + 2] + e[o + 3])) + ((e[o + 4] + e[o + 5]) + (e[o + 6] + e[o + 7]));
                    for (int i = 0; i < 8; ++i) pw[b][i] = (_Float16)e[o + i];
                }
                // (a block that a row sees nothing of stays out, whatever its scale is)
                if (whole) {
                    for (int b = 0; b < 4; ++b) weight = __builtin_fmaf(sum[b], bv[b], weight);
                } else {
                    for (int b = 0; b < 4; ++b) weight += sum[b] == 0.0f ? 0.0f : sum[b] * bv[b];
                }
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int d = 0; d < D / 32; ++d)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const half8_t *>(&t.v[32 * d + n][part + 16 * u + 8 * hi]), pw[u], acc[d], 0, 0, 0);
                loads_among_products<4 * D / 32, 1>();
                __builtin_amdgcn_s_setprio(0);
            }
            if (t0 + TOKENS < reach.end) put(buffer[at ^ 1]);
            ask(t0 + 2 * TOKENS);
            ask_entries(t0 + 3 * TOKENS, 0);
            __syncthreads();
        }
        weight += __shfl_xor(weight, 32);
        if (is_lost(a, p, row)) weight = __builtin_nanf("");

        const bool again = mode == kAll && far;
        Softmax &mine = softmax[wave * 32 + n];          // (of this wave alone)
        if (mode == kScores) mine = Softmax{ref, weight};
        else if (!again && row < rows) {
            const AttendArgs a = args_again();
            const Ending end = ending(a, mode, ref, weight, mine);
            const uint64_t id = row_id(a, p, row);
#pragma unroll
            for (int d = 0; d < D / 32; ++d) acc[d] *= end.f;
            if (mode == kValues) {
#pragma unroll
                for (int d = 0; d < D / 32; ++d) acc[d] = acc[d] * end.h * end.h;
            }
            if (a.splits == 1) {
                uint16_t *dst = static_cast<uint16_t *>(a.out) + (uint64_t)(p.begin + row / a.group) * a.out_stride +
                                (uint64_t)(p.h * a.group + row % a.group) * D + 4 * hi;
#pragma unroll
                for (int d = 0; d < D / 32; ++d)
                    for (int b = 0; b < 4; ++b)
                        *reinterpret_cast<uint2_t *>(dst + 32 * d + 8 * b) =
                            uint2_t{narrow2<BF16>(acc[d][4 * b], acc[d][4 * b + 1]), narrow2<BF16>(acc[d][4 * b + 2], acc[d][4 * b + 3])};
                if (a.lse && hi == 0) a.lse[id] = end.total == 0.0f ? -INFINITY : (end.top + log2_of(end.total)) * 0.69314718055994530942f;
            } else {
                float *dst = a.parts + (id * a.splits + p.split) * D + 4 * hi;
#pragma unroll
                for (int d = 0; d < D / 32; ++d)
                    for (int b = 0; b < 4; ++b)
                        *reinterpret_cast<float4_t *>(dst + 32 * d + 8 * b) = float4_t{acc[d][4 * b], acc[d][4 * b + 1], acc[d][4 * b + 2], acc[d][4 * b + 3]};
                if (hi == 0) {
                    float *st = a.parts + a.part_rows * a.splits * D + (id * a.splits + p.split) * 2;
                    st[0] = end.top;
                    st[1] = end.total;
                }
            }
        }
        if (again || mode == kScores) {
            mode = again ? kScores : kValues;
        } else {
            if (done) return;
            mode = kAll;
            ++tile;
        }
        __syncthreads();
    }
}

// The pieces of a row along the cache, joined: WAVES waves for a row, D / 4 lanes of them for a piece, so that
// PIECES = 256 WAVES / D pieces are read at once.  Which lanes add which pieces, and in which order the lanes'
// sums are added, is fixed.
template <int D, bool BF16, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void k_attend_join(JoinArgs j) {
    const AttendArgs &a = j.a;
    constexpr uint32_t LANES = D / 4, PIECES = 64 * WAVES / LANES, ROWS = WAVES == 1 ? 4 : 1;
    __shared__ float4_t sums[WAVES > 1 ? WAVES : 1][LANES];
    __shared__ float totals[WAVES > 1 ? WAVES : 1], tops[WAVES > 1 ? WAVES : 1];
    const uint32_t tid = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint64_t id = (uint64_t)blockIdx.x * ROWS + (WAVES == 1 ? (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) : 0);
    // the rows of the first launch, then those of the launch for requests of few rows
    const uint64_t firsts = a.splits == 1 ? 0 : a.part_rows;
    const bool of_few = id >= firsts;
    if (of_few) id -= firsts;
    const uint64_t part_rows = of_few ? j.few_part_rows : a.part_rows;
    const uint32_t splits = of_few ? j.few_splits : a.splits;
    const float *all = of_few ? j.few_parts : a.parts;
    if (id >= part_rows || splits == 1) return;
    // What most rows have is asked for at once: the first pieces of each lane and their statistics.
    const uint32_t part = tid / LANES, piece = tid % LANES;
    const float *parts = all + id * splits * D + 4 * piece, *stats = all + part_rows * splits * D + id * splits * 2;
    constexpr int KEPT = 4;
    float4_t v[KEPT];
    float2_t st[KEPT];
#pragma unroll
    for (int u = 0; u < KEPT; ++u) {
        const uint32_t i = min(part + u * PIECES, splits - 1);
        st[u] = *reinterpret_cast<const float2_t *>(stats + 2 * i);
        v[u] = *reinterpret_cast<const float4_t *>(parts + (uint64_t)i * D);
    }
    // rows that no request has, or one of the other launch's, were not computed and are not written
    uint32_t token, head;
    if (of_few && j.slots_each) {
        const uint32_t each = j.slots_each * a.kv_heads, r = (uint32_t)(id / each), slot = (uint32_t)(id % each), row = slot / a.kv_heads;
        const uint32_t b = min((uint32_t)max(a.starts[r], 0), a.tokens), e = min((uint32_t)max(a.starts[r + 1], 0), a.tokens);
        const uint32_t rows = e > b ? (e - b) * a.group : 0;
        if (row >= rows || rows >= a.rows_from) return;
        token = b + row / a.group;
        head = slot % a.kv_heads * a.group + row % a.group;
    } else {
        token = (uint32_t)(id / a.q_heads);
        head = (uint32_t)(id % a.q_heads);
        uint32_t lo = 0, hi = a.requests;
        while (hi - lo > 1) {                            // a wave halves 64 times at once
            const uint32_t step = (hi - lo + 63) / 64, at = lo + lane * step;
            const uint64_t below = __ballot(at < hi && a.starts[at] <= (int32_t)token);
            const uint32_t last = 63 - (uint32_t)__builtin_clzll(below | 1);
            hi = min(hi, lo + (last + 1) * step);
            lo += last * step;
        }
        const int32_t b = max(a.starts[lo], 0), e = a.starts[lo + 1];
        if ((int32_t)token < b || (int32_t)token >= e) return;
        const uint32_t rows = (min((uint32_t)e, a.tokens) - (uint32_t)b) * a.group;
        if (of_few ? rows >= a.rows_from : rows < a.rows_from) return;
    }
    float top = kNone;
#pragma unroll
    for (int u = 0; u < KEPT; ++u) top = fmaxf(top, st[u][0]);
    for (uint32_t i = part + KEPT * PIECES; i < splits; i += PIECES) top = fmaxf(top, stats[2 * i]);
    for (uint32_t d = LANES; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, (int)d));
    if constexpr (WAVES > 1) {
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, tops[w]);
    }
    float total = 0.0f;
    float4_t y = {0, 0, 0, 0};
    auto add = [&](float2_t t, float4_t x) {
        if (t[1] == 0.0f) return;                        // nothing seen, and perhaps no sums written (NaN is not 0)
        const float f = pow2(t[0] - top);
        total = __builtin_fmaf(t[1], f, total);
        for (int e = 0; e < 4; ++e) y[e] = __builtin_fmaf(x[e], f, y[e]);
    };
#pragma unroll
    for (int u = 0; u < KEPT; ++u)
        if (part + u * PIECES < splits) add(st[u], v[u]);
    for (uint32_t i = part + KEPT * PIECES; i < splits; i += PIECES)
        add(*reinterpret_cast<const float2_t *>(stats + 2 * i), *reinterpret_cast<const float4_t *>(parts + (uint64_t)i * D));
    for (uint32_t d = LANES; d < 64; d <<= 1) {
        total += __shfl_xor(total, (int)d);
        for (int e = 0; e < 4; ++e) y[e] += __shfl_xor(y[e], (int)d);
    }
    if constexpr (WAVES > 1) {
        if (lane < LANES) sums[wave][lane] = y;
        if (lane == 0) totals[wave] = total;
        __syncthreads();
        if (tid >= LANES) return;
        y = sums[0][tid];
        total = totals[0];
        for (int w = 1; w < WAVES; ++w) { y += sums[w][tid]; total += totals[w]; }
    }
    if (tid >= LANES) return;
    const float f = total == 0.0f ? 0.0f : 1.0f / total;
    uint16_t *dst = static_cast<uint16_t *>(a.out) + (uint64_t)token * a.out_stride + (uint64_t)head * D + 4 * piece;
    *reinterpret_cast<uint2_t *>(dst) = uint2_t{narrow2<BF16>(y[0] * f, y[1] * f), narrow2<BF16>(y[2] * f, y[3] * f)};
    if (a.lse && tid == 0) a.lse[(uint64_t)token * a.q_heads + head] = total == 0.0f ? -INFINITY : (top + log2_of(total)) * 0.69314718055994530942f;
}

}  // namespace

// Rows of a kv head up to which a request is k_attend_few's.
uint32_t few_rows(const CacheShape &s) { return s.head_dim == 256 ? 32 : 64; }

// Which kernel, how many rows a workgroup, and into how many pieces the cache's length is cut.
//
// Rows: a request with at most 64 rows of a kv head goes to k_attend_few, whose time is the cache's bytes as long as
// they are read once or twice (32 requests of 8192 tokens, 64 heads on 8 of 128, 4 queries each: 130 us in one pass of
// 32 rows, 217 us by k_attend_many; 16 of 4096, 8 each: 50 us in two, and 58).  k_attend_many takes 256 rows a workgroup, 128 where a request has no more.
// Pieces: `slots` workgroups run at once.  Fewer units than that leave the device partly idle, so each is cut; a piece
// costs its start and its share of the join.  Each launch has its own number of pieces and its own parts: prompts beside
// single tokens of long requests stay whole, and only the rows of the second launch have pieces to be joined.
AttendLaunch attend_launch(const CacheShape &s, uint32_t requests, uint32_t tokens, uint32_t max_new, uint32_t max_length, uint32_t window) {
    AttendLaunch l = {};
    l.few_splits = 1;
    const uint64_t group = s.q_heads / s.kv_heads, most = max_new * group, few = few_rows(s);
    auto tile = [&](uint32_t rows) {
        l.rows = rows;
        const uint64_t each = (most + rows - 1) / rows, packed = tokens * group / rows + requests;
        // the same number for every request saves the search for a tile's request; where requests differ much it would
        // launch more workgroups than there are tiles
        l.tiles_each = each == 0 ? 1u : (uint32_t)(each * requests <= packed ? each : 0);
        l.tiles = (uint32_t)(l.tiles_each ? (uint64_t)l.tiles_each * requests : packed);
    };
    uint64_t slots;
    if (most <= few) {
        tile(most <= 16 || s.head_dim == 256 ? 16 : 32);
        slots = s.head_dim == 256 ? 256 : s.head_dim == 128 || l.rows == 32 ? 512 : 768;
    } else {
        tile(s.head_dim == 256 || most <= 128 ? 128 : 256);
        slots = s.head_dim == 256 || l.rows == 256 ? 256 : 512;
        // Single tokens beside prompts: where the requests have a quarter of the longest one's rows on average, or less, a
        // launch of its own takes those of few rows, and this one the others (one token each of 63 requests of 2000 tokens
        // and a prompt of 512, 64 heads on 8: 80 us, and 157 all by k_attend_many; 15 of 8000 and 2048, 32 on 8: 135 and
        // 251; 200 of 500 and 1000, 32 on 32: 284 and 514; 3 of 300 and 200, 32 on 8: 20 and 20).
        if (requests > 1 && tokens * group * 4 <= requests * most) l.few_tiles = (uint32_t)(few / (s.head_dim == 256 ? 16 : 32)) * requests;
    }
    uint64_t reach = max_length < 0x7FFFFFFFu ? max_length : 0x7FFFFFFFu;     // (no request is longer, and a piece's tokens are 32 bits)
    if (window && reach > (uint64_t)window + max_new) reach = (uint64_t)window + max_new;
    auto cut = [&](uint64_t units, uint64_t at_once, bool is_few, uint64_t at_least, uint32_t &splits, uint32_t &chunk) {
        const uint64_t least = is_few ? 256 : 128;       // a tile of each wave of k_attend_few, one of k_attend_many
        const uint64_t longest = reach <= 256 ? 1 : (reach + least - 1) / least;
        uint64_t n = at_once / (units ? units : 1);
        if (n > longest) n = longest;
        if (n < at_least) n = at_least;
        chunk = (uint32_t)(((reach + n - 1) / n + 127) / 128 * 128);
        if (chunk == 0) chunk = 128;                     // (reach 0)
        // (pieces of whole tiles may be fewer)
        splits = (uint32_t)((reach + chunk - 1) / chunk);
        if (splits == 0) splits = 1;
    };
    // One request of a batch may be far longer than the others: a piece of k_attend_few has no more than 8192 tokens (63
    // requests of 2000 tokens and one of 131072, 64 heads on 8: 225 us, and 766 in one piece; 64 requests of 32768 each
    // 738 and 718).  The same holds for k_attend_many beside single tokens, whose tiles end at once there, as long as the
    // other tiles leave the device partly idle (512 tokens after 32256 beside 62 of 2000: 690 us, and 998 in one piece).
    const uint64_t units = (uint64_t)l.tiles * s.kv_heads, pieces = (reach + 8191) / 8192;
    uint64_t at_least = 1;
    if (l.rows < 128) at_least = pieces;
    else if (l.few_tiles && tokens > requests) {
        const uint64_t others = ((uint64_t)(tokens - requests) * group + l.rows - 1) / l.rows * s.kv_heads;
        at_least = pieces < slots / others ? pieces : slots / others;
    }
    cut(units, slots, l.rows < 128, at_least ? at_least : 1, l.splits, l.chunk);
    l.part_rows = (uint64_t)tokens * s.q_heads;
    auto bytes = [&](uint64_t rows, uint32_t splits) { return splits == 1 ? 0 : rows * splits * (s.head_dim + 2u) * 4u; };
    l.workspace = bytes(l.part_rows, l.splits);
    if (l.few_tiles) {
        // (one tile a request has rows, where they are single tokens)
        cut((uint64_t)requests * s.kv_heads, s.head_dim == 256 ? 256 : 512, true, pieces, l.few_splits, l.few_chunk);
        // as many rows as requests of few rows can have, or as the call has, whichever is less
        l.few_part_rows = (uint64_t)requests * few * s.kv_heads;
        l.slots_each = (uint32_t)few;
        if (l.few_part_rows > l.part_rows) { l.few_part_rows = l.part_rows; l.slots_each = 0; }
        l.few_at = (l.workspace + 255) / 256 * 256;
        if (l.few_splits > 1) l.workspace = l.few_at + bytes(l.few_part_rows, l.few_splits);
    }
    // Requests of several lengths in many more workgroups than run at once: the longest begin first, so that the last
    // ones to end are short (64 requests of 1024 to 4096 tokens on 40 heads, 2560 workgroups: 306 us against 318; with
    // little more than one round the ranking costs more than it brings: 20 requests of 250 to 1000 tokens on 32 heads 29
    // against 25).  A wave ranks 64 requests.
    l.by_length = l.tiles_each && requests > 1 && requests <= 64 && units * l.splits >= 4 * slots;
    // Workgroups of few rows over 4 bits are done sooner, and the ranking, a microsecond of each, pays from 1024 tokens on, of 16
    // rows.  Two of them run on a CU at once (three with heads of 64), i and i + 256.  Where that is all there are, those after
    // the first 256 go by length from the other end, the shortest with the longest (64 requests of 1024 to 4096 tokens, 64 heads
    // on 8: 40 us, in the order given 44; of 500 to 2000 24.3 and 26.6, of 250 to 1000 17.1 and 16.9, of 125 to 500 13.5 and
    // 12.3); where there are more, all go from the longest on (32 requests of 1024 to 4096, 32 heads: 64.4 us, in the order given
    // 70.3; 40 of 375 to 1500 41.5 and 42.9; 60 of 250 to 1000 48.7 and 45.0).
    if (s.bits == 4 && l.rows <= 32 && l.tiles_each == 1 && requests > 1 && requests <= 64) {
        const bool pays = reach * l.rows > 16 * 1024;
        const uint64_t groups = units * l.splits, at_once = std::max<uint64_t>(slots, 512);
        const uint32_t turn = (uint32_t)(256 / (s.kv_heads * l.splits));
        l.by_length = pays && groups > at_once ? 1 : 0;
        if (pays && groups > 256 && groups <= at_once && turn >= 1 && turn < requests) l.by_length = turn + 1;
    }
    return l;
}

int launch_attend(const CacheShape &s, const AttendLaunch &l, const AttendArgs &args, void *stream) {
    AttendArgs a = args;
    if (l.few_tiles) a.rows_from = few_rows(s) + 1;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    // the workgroups of the three launches
    const uint64_t all = (uint64_t)l.tiles * l.splits * s.kv_heads, few = (uint64_t)l.few_tiles * l.few_splits * s.kv_heads;
    const uint64_t joined = (l.splits > 1 ? l.part_rows : 0) + (l.few_splits > 1 ? l.few_part_rows : 0);
    // (a wave reads a few pieces of a row one after the other; more of them want more waves)
    const bool one_wave = l.splits <= 16 && l.few_splits <= 16;
    if (!fits(all, l.rows == 256 ? 512 : 256) || !fits(few, 256) || !(one_wave ? fits((joined + 3) / 4, 256) : fits(joined, 512))) return kTooLarge;
    const uint32_t grid = (uint32_t)all;
    const JoinArgs j = {a, reinterpret_cast<float *>(reinterpret_cast<char *>(a.parts) + l.few_at), l.few_part_rows, l.few_splits, l.slots_each};
    if (s.bits == 4) launch_attend_four(s, l.rows, l.tiles_each == 1, grid, a, stream);
    else by_shape(s, [&](auto d, auto bf16) {
        if (l.rows == 16) k_attend_few<d(), bf16(), 1><<<grid, 256, 0, st>>>(a);
        else if (l.rows == 32) { if constexpr (d() != 256) k_attend_few<d(), bf16(), 2><<<grid, 256, 0, st>>>(a); }
        else if (l.rows == 128) k_attend_many<d(), bf16(), 4, 64><<<grid, 256, 0, st>>>(a);
        else if constexpr (d() != 256) k_attend_many<d(), bf16(), 8, 128><<<grid, 512, 0, st>>>(a);
    });
    if (hipError_t e = hipGetLastError()) return (int)e;
    if (l.few_tiles) {
        AttendArgs f = a;
        f.tiles = l.few_tiles;
        f.tiles_each = l.few_tiles / a.requests;
        f.by_length = 0;
        // (most requests have one tile: the workgroups of the others, which end at once, would take every other place)
        f.by_tile = 1;
        f.rows_from = 0;
        f.rows_to = few_rows(s);
        f.splits = l.few_splits;
        f.chunk = l.few_chunk;
        f.parts = j.few_parts;
        f.part_rows = l.few_part_rows;
        f.slots_each = l.slots_each;
        if (s.bits == 4) launch_attend_four(s, s.head_dim == 256 ? 16 : 32, true, (uint32_t)few, f, stream);
        else by_shape(s, [&](auto d, auto bf16) { k_attend_few<d(), bf16(), d() == 256 ? 1 : 2><<<(uint32_t)few, 256, 0, st>>>(f); });
        if (hipError_t e = hipGetLastError()) return (int)e;
    }
    if (joined == 0) return 0;
    by_shape(s, [&](auto d, auto bf16) {
        if (one_wave) k_attend_join<d(), bf16(), 1><<<(uint32_t)((joined + 3) / 4), 256, 0, st>>>(j);
        else k_attend_join<d(), bf16(), 8><<<(uint32_t)joined, 512, 0, st>>>(j);
    });
    return (int)hipGetLastError();
}

}  // namespace tsq
