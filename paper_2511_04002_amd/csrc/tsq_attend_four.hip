// Attention over a cache held in 4 bits (tsq_cache_attend).
//
//   out = sum_t w_t v_t / sum_t w_t,   w_t = exp(scale * (q . k_t))
// Keys and values are exact in the queries' own 16-bit type, scale included: the conversion instructions make two elements
// at a time, and what goes into the matrix instructions is what the cache stands for.  The reference m of a row's weights
// 2^(score - m) follows its largest score in steps, as it moves only when a score is more than 8 above what it was set for.
// The weights of binary16 values are halves, at most 2^15 and of 11 bits down to 2^-21 of the row's largest; those of
// bfloat16 values, whose range halves have not, are the sum of two bfloat16, 16 bits, at most 1.  The denominator adds the
// weights as they are before that rounding.
//
// Scores are computed transposed, S^T = K Q^T: a lane then has all its scores in one row of the softmax (a query), and the
// registers that hold P^T are, in the order they are in, an operand of O^T = V^T P^T.  Values lie token by token, as keys
// do, and their operand wants tokens side by side: of two tokens' registers, which hold two elements each, two byte
// permutations make one register for either element.
#include "tsq_attend.hpp"
#include "tsq_four.hpp"

namespace tsq {
namespace {

template <bool BF16> struct Softmaxes {
    static constexpr float room = BF16 ? -8.0f : 7.0f;   // the reference is set this far below the largest exponent ...
    static constexpr float slack = 8.0f;                 // ... and kept until one exceeds that by as much
};

__device__ __forceinline__ uint32_t byte_of(uint32_t w, uint32_t shift) { return __builtin_amdgcn_ubfe(w, shift, 8); }

// Products of 16 x 16 x 32 with binary32 sums.
template <bool BF16> __device__ __forceinline__ float4_t product(uint4_t x, uint4_t y, float4_t z) {
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), __builtin_bit_cast(bf16x8_t, y), z, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, x), __builtin_bit_cast(half8_t, y), z, 0, 0, 0);
}

// Few rows: 16 of a kv head's, or 32 (SETS = 2, which share the converted elements).  Each of four waves takes every fourth
// tile of 64 tokens straight from memory to registers and keeps a softmax of its own; they meet in LDS at the end.
// Lane (m = lane % 16, g = lane / 16).  The tokens of a tile: group g has 16g .. 16g + 15, all of one block.
//   S^T tile t (16 tokens x 16 rows): row 4g + i is token 16g + 4t + i, so that a lane's 16 scores (t, i) are the
//   16 tokens of its group; its row of the softmax is m.
//   Keys: operand row m is token 16 (m / 4) + 4t + m % 4; the lane's elements are g D/4 .. + D/4 - 1, eight a product.
//   Values: a lane has elements m D/16 .. + D/16 - 1 of its group's 16 tokens; row m of product j is element m D/16 + j.
template <int D, bool BF16, int SETS>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void k_attend_four_few(AttendArgs a) {
    constexpr int ROWS = 16 * SETS;
    constexpr int KW = D / 32;                           // words of a lane's keys of a token, and products of a score
    constexpr int KS = D == 256 ? 2 : 1;                 // scales of them
    constexpr int VE = D / 16;                           // elements of a lane's values of a token: 4, 8 or 16
    constexpr int VW = D == 256 ? 2 : 1;                 // words of them
    constexpr int GROUPS = D / 32;
    __shared__ float sums[4][16][132];
    __shared__ float stats[4][16][2];
    Place p;
    if (!find_place<ROWS>(a, p)) return;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
    const uint32_t B = 1u << a.block_log2;
    const uint8_t *all_k = static_cast<const uint8_t *>(a.k), *all_v = static_cast<const uint8_t *>(a.v);
    const uint8_t *all_ks = static_cast<const uint8_t *>(a.k_scale), *all_vs = static_cast<const uint8_t *>(a.v_scale);
    for (uint32_t tile = p.tile;; ++tile) {
        const uint32_t rows = p.n * a.group;
        const Reach reach = reach_of<ROWS>(a, p, tile);
        const bool done = !p.last || (uint64_t)(tile + 1) * ROWS >= rows;
        if (a.splits > 1 && reach.begin >= reach.end) {
            nothing_seen<ROWS>(a, p, tile, D);
            if (done) return;
            continue;
        }
        uint4_t q[SETS][KW];
        uint32_t from[SETS], to[SETS];
#pragma unroll
        for (int c = 0; c < SETS; ++c) {
            const uint32_t row = tile * ROWS + 16 * c + m;
            for (int j = 0; j < KW; ++j) {
                q[c][j] = uint4_t{0, 0, 0, 0};
                if (row < rows) {
                    const uint16_t *src = static_cast<const uint16_t *>(a.q) + (uint64_t)(p.begin + row / a.group) * a.q_stride +
                                          (uint64_t)(p.h * a.group + row % a.group) * D + g * (D / 4) + 8 * j;
                    q[c][j] = *reinterpret_cast<const uint4_t *>(src);
                }
            }
            row_sees(a, p, row, from[c], to[c]);
        }
        float4_t acc[SETS][VE];
        float ref[SETS], weight[SETS];
#pragma unroll
        for (int c = 0; c < SETS; ++c) {
            for (int j = 0; j < VE; ++j) acc[c][j] = float4_t{0, 0, 0, 0};
            ref[c] = kNone;
            weight[c] = 0.0f;
        }

        // Loads are always on their way: a tile's keys are asked for while the tile before it is worked on, its values
        // when that one's are used up, and its block numbers a tile earlier still.
        uint32_t kw[4][KW], vw[16][VW];
        uint4_t ks[KS], vs;
        bool bad = false;
        auto ask_keys = [&](uint32_t t0, uint32_t entry) {
            const uint32_t id = (uint32_t)__shfl((int)id_of(a, entry), (int)(m >> 2) << 4), place = (t0 + 16 * (m >> 2)) & (B - 1);
            const uint64_t head = (uint64_t)id * a.kv_heads + p.h;
            const uint8_t *keys = all_k + (head * B + place + (m & 3)) * (D / 2) + g * (D / 8);
            const uint8_t *scales = all_ks + (head * GROUPS + g * (D / 4) / 32) * B + place;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint8_t *at = keys + 4 * t * (D / 2);
                if constexpr (D == 64) {
                    const uint2_t w = *reinterpret_cast<const uint2_t *>(at);
                    kw[t][0] = w[0]; kw[t][1] = w[1];
                } else {
                    for (int x = 0; x < KW; x += 4) {
                        const uint4_t w = *reinterpret_cast<const uint4_t *>(at + 4 * x);
                        for (int i = 0; i < 4; ++i) kw[t][x + i] = w[i];
                    }
                }
            }
            for (int x = 0; x < KS; ++x) ks[x] = *reinterpret_cast<const uint4_t *>(scales + x * B);
            bad = is_bad(a, p, entry);
        };
        auto ask_values = [&](uint32_t t0, uint32_t entry) {
            const uint32_t place = (t0 + 16 * g) & (B - 1);
            const uint64_t head = (uint64_t)id_of(a, entry) * a.kv_heads + p.h;
            const uint8_t *values = all_v + (head * B + place) * (D / 2) + m * (D / 32);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if constexpr (D == 64) vw[i][0] = *reinterpret_cast<const uint16_t *>(values + i * (D / 2));
                else if constexpr (D == 128) vw[i][0] = *reinterpret_cast<const uint32_t *>(values + i * (D / 2));
                else {
                    const uint2_t w = *reinterpret_cast<const uint2_t *>(values + i * (D / 2));
                    vw[i][0] = w[0]; vw[i][1] = w[1];
                }
            }
            vs = *reinterpret_cast<const uint4_t *>(all_vs + (head * GROUPS + m * VE / 32) * B + place);
        };
        uint32_t t0 = reach.begin + 64 * wave, next = 0;
        if (t0 < reach.end) {
            const uint32_t entry = table_entry(a, p, t0 + 16 * g, reach.end);
            next = table_entry(a, p, t0 + 256 + 16 * g, reach.end);
            ask_keys(t0, entry);
            ask_values(t0, entry);
        }
        for (; t0 < reach.end; t0 += 256) {
            float4_t s[SETS][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                for (int c = 0; c < SETS; ++c) s[c][t] = float4_t{0, 0, 0, 0};
                float scale[KS];
                for (int x = 0; x < KS; ++x) scale[x] = four_scale(byte_of(ks[x][t], 8 * (m & 3)));
                for (int j = 0; j < KW; ++j) {
                    const uint4_t k = four_eight<BF16>(kw[t][j], scale[KS == 1 ? 0 : j / 4]);
                    for (int c = 0; c < SETS; ++c) s[c][t] = product<BF16>(k, q[c][j], s[c][t]);
                }
            }
            const float factor = bad ? __builtin_nanf("") : a.scale_log2;
            const uint32_t entry = next;
            ask_keys(t0 + 256, entry);
            next = table_entry(a, p, t0 + 512 + 16 * g, reach.end);
            // exponents, and the reference
            const uint32_t mine = t0 + 16 * g;
            uint4_t pw[SETS][2], rest[SETS][2];
#pragma unroll
            for (int c = 0; c < SETS; ++c) {
                const bool whole = __ballot(mine < from[c] || mine + 16 > to[c]) == 0;
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    for (int i = 0; i < 4; ++i) s[c][t][i] *= factor;
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
                constexpr float room = Softmaxes<BF16>::room, slack = Softmaxes<BF16>::slack;
                if (__ballot(top > ref[c] + (room + slack))) {
                    const float now = fmaxf(ref[c], top - room), down = pow2(ref[c] - now);
                    ref[c] = now;
                    weight[c] *= down;
                    for (int j = 0; j < VE; ++j) acc[c][j] *= down;
                }
                float sum = 0.0f;
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    for (int i = 0; i < 4; i += 2) {
                        const float e0 = pow2(s[c][t][i] - ref[c]), e1 = pow2(s[c][t][i + 1] - ref[c]);
                        sum += e0 + e1;
                        const uint32_t w = narrow2<BF16>(e0, e1);
                        pw[c][t / 2][2 * (t & 1) + i / 2] = w;
                        if constexpr (BF16) rest[c][t / 2][2 * (t & 1) + i / 2] = narrow2<true>(e0 - widen<true>(w & 0xFFFFu), e1 - widen<true>(w >> 16));
                    }
                weight[c] += sum;
            }
            // (no value that is not seen may bring NaN or infinity into a sum, whatever stands there: its scale is one of
            // those that are finite, and its weight is 0.  A token whose values are NaN has keys that are NaN, too)
            constexpr uint32_t highest = FourScales<BF16>::highest;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float scale[8];
                for (int e = 0; e < 8; ++e) scale[e] = four_scale(min(byte_of(vs[2 * u + e / 4], 8 * (e & 3)), highest));
                auto each = [&](auto pair) {             // two elements of the lane's: byte pair % 4 of word pair / 4
                    constexpr int P = pair();
                    uint4_t first, second;
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t x = four_pair<BF16, P % 4>(vw[8 * u + 2 * e][P / 4], scale[2 * e]);
                        const uint32_t y = four_pair<BF16, P % 4>(vw[8 * u + 2 * e + 1][P / 4], scale[2 * e + 1]);
                        first[e] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                        second[e] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                    }
                    for (int c = 0; c < SETS; ++c) {
                        acc[c][2 * P] = product<BF16>(first, pw[c][u], acc[c][2 * P]);
                        acc[c][2 * P + 1] = product<BF16>(second, pw[c][u], acc[c][2 * P + 1]);
                        if constexpr (BF16) {
                            acc[c][2 * P] = product<BF16>(first, rest[c][u], acc[c][2 * P]);
                            acc[c][2 * P + 1] = product<BF16>(second, rest[c][u], acc[c][2 * P + 1]);
                        }
                    }
                };
                each(std::integral_constant<int, 0>{});
                each(std::integral_constant<int, 1>{});
                if constexpr (VE >= 8) {
                    each(std::integral_constant<int, 2>{});
                    each(std::integral_constant<int, 3>{});
                }
                if constexpr (VE >= 16) {
                    each(std::integral_constant<int, 4>{});
                    each(std::integral_constant<int, 5>{});
                    each(std::integral_constant<int, 6>{});
                    each(std::integral_constant<int, 7>{});
                }
            }
            ask_values(t0 + 256, entry);
        }

        // the four waves' sums, at one reference
#pragma unroll
        for (int c = 0; c < SETS; ++c) {
            weight[c] += __shfl_xor(weight[c], 16);
            weight[c] += __shfl_xor(weight[c], 32);
            if (c) __syncthreads();
            if (g == 0) { stats[wave][m][0] = ref[c]; stats[wave][m][1] = weight[c]; }
            __syncthreads();
            const float all = fmaxf(fmaxf(stats[0][m][0], stats[1][m][0]), fmaxf(stats[2][m][0], stats[3][m][0]));
            const float mine = pow2(ref[c] - all);
            const uint32_t out_row = threadIdx.x >> 4, piece = threadIdx.x & 15, o = tile * ROWS + 16 * c + out_row;
            float total = 0.0f, top = fmaxf(fmaxf(stats[0][out_row][0], stats[1][out_row][0]), fmaxf(stats[2][out_row][0], stats[3][out_row][0]));
            for (int w = 0; w < 4; ++w) total += stats[w][out_row][1] * pow2(stats[w][out_row][0] - top);
            if (is_lost(a, p, o)) total = __builtin_nanf("");
            const float back = a.splits > 1 ? 1.0f : total == 0.0f ? 0.0f : 1.0f / total;
            const uint64_t id = a.splits == 1 ? row_id(a, p, o) : part_row(a, p, o);
            for (int part = 0; part < (D + 127) / 128; ++part) {
                constexpr int N = D < 128 ? D : 128;     // elements at a time
                if (part) __syncthreads();
                // a lane's elements (4g + i) VE + j, those of heads of 256 in two halves
                if (D <= 128 || (int)(g >> 1) == part) {
                    float *dst = &sums[wave][m][D <= 128 ? 4 * g * VE : 4 * (g & 1) * VE];
                    for (int i = 0; i < 4; ++i)
                        for (int j = 0; j < VE; j += 4)
                            *reinterpret_cast<float4_t *>(dst + i * VE + j) = float4_t{acc[c][j][i], acc[c][j + 1][i], acc[c][j + 2][i], acc[c][j + 3][i]} * mine;
                }
                __syncthreads();
                if (piece * 8 < N && o < rows) {
                    float y[8];
                    for (int i = 0; i < 8; ++i) {
                        y[i] = sums[0][out_row][8 * piece + i] + sums[1][out_row][8 * piece + i] + sums[2][out_row][8 * piece + i] + sums[3][out_row][8 * piece + i];
                        y[i] *= back;
                    }
                    if (a.splits == 1) {
                        uint4_t w;
                        for (int i = 0; i < 4; ++i) w[i] = narrow2<BF16>(y[2 * i], y[2 * i + 1]);
                        uint16_t *dst = static_cast<uint16_t *>(a.out) + (uint64_t)(p.begin + o / a.group) * a.out_stride +
                                        (uint64_t)(p.h * a.group + o % a.group) * D + part * 128 + piece * 8;
                        *reinterpret_cast<uint4_t *>(dst) = w;
                    } else {
                        float *dst = a.parts + (id * a.splits + p.split) * D + part * 128 + piece * 8;
                        *reinterpret_cast<float4_t *>(dst) = float4_t{y[0], y[1], y[2], y[3]};
                        *reinterpret_cast<float4_t *>(dst + 4) = float4_t{y[4], y[5], y[6], y[7]};
                    }
                }
            }
            if (piece == 0 && o < rows) {
                if (a.splits > 1) {
                    float *dst = a.parts + a.part_rows * a.splits * D + (id * a.splits + p.split) * 2;
                    dst[0] = top;
                    dst[1] = total;
                } else if (a.lse) {
                    a.lse[id] = total == 0.0f ? -INFINITY : (top + log2_of(total)) * 0.69314718055994530942f;
                }
            }
        }
        if (done) return;
        __syncthreads();
    }
}

}  // namespace

void launch_attend_four(const CacheShape &s, uint32_t rows, uint32_t grid, const AttendArgs &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    by_shape(s, [&](auto d, auto bf16) {
        if (rows == 16) k_attend_four_few<d(), bf16(), 1><<<grid, 256, 0, st>>>(a);
        else if constexpr (d() != 256) k_attend_four_few<d(), bf16(), 2><<<grid, 256, 0, st>>>(a);
    });
}

}  // namespace tsq
