// Attention over a cache held in 4 bits (tsq_cache_attend).
//
//   out = sum_t w_t v_t / sum_t w_t,   w_t = exp(scale * (q . k_t))
// Keys and values are exact in the queries' own 16-bit type, scale included: the conversion instructions make two elements
// at a time, and what goes into the matrix instructions is what the cache stands for.  The reference m of a row's weights
// 2^(score - m) follows its largest score in steps, as it moves only when a score is more than 8 above what it was set for.
// Weights are halves, at most 2^15, of 11 bits down to 2^-21 of the row's largest, and values are converted to halves,
// exactly, whichever type the cache is of.  Values of bfloat16 that halves do not hold send their workgroup through all of
// its tokens a second time, with values in bfloat16 and weights the sum of two bfloat16, 16 bits, at most 1.  The
// denominator adds the weights as they are before that rounding.
//
// Scores are computed transposed, S^T = K Q^T: a lane then has all its scores in one row of the softmax (a query), and the
// registers that hold P^T are, in the order they are in, an operand of O^T = V^T P^T.  Values lie token by token, as keys
// do, and their operand wants tokens side by side: few rows make one register for either element of two tokens' registers,
// which hold two elements each, by two byte permutations; many rows read it so from LDS.
#include "tsq_attend.hpp"
#include "tsq_four.hpp"

namespace tsq {
namespace {

constexpr float kCoarse = 0x1p22f;   // beyond this a reference's last bit is worth 1/2 or more: the difference of a score that
                                     // is not rounded and one that is would pass a half's range
template <bool BF16> struct Softmaxes {
    static constexpr float room = BF16 ? -8.0f : 7.0f;   // the reference is set this far below the largest exponent ...
    static constexpr float slack = 8.0f;                 // ... and kept until one exceeds that by as much
};

__device__ __forceinline__ uint32_t byte_of(uint32_t w, uint32_t shift) { return __builtin_amdgcn_ubfe(w, shift, 8); }

// Codes, with a streaming load where they are read once.
template <bool ONCE, typename T> __device__ __forceinline__ T codes_at(const uint8_t *at) {
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const T *>(at));
    else return *reinterpret_cast<const T *>(at);
}

// The larger of a lane's value and that of the lane 16 away.
__device__ __forceinline__ float max_across_sixteen(float x) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane16_swap(bits, bits, false, false);
    const uint32_t a = r[0], b = r[1];
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

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
// Memory bounds it where a call has enough tokens to keep two workgroups a CU busy: 64 requests of 1024 to 4096 tokens on 40 heads
// of 128 (949 MB) take 156 us, 6.1 TB/s, where a kernel that reads the same pieces and drops them takes 147 to 157; one request
// of 131072 tokens, 64 heads on 8, 31 us with the join of its pieces, 4.6 TB/s; a single token of 128, 5 us from launch to
// end.  With 32 rows the conversions and the softmax, which is made for each 16 rows, take as long as the loads: 32 requests of
// 2400 to 8200 tokens, up to 4 queries of 64 heads on 8 each, 43 us with the join, 39 by itself, 4.3 TB/s.
// Little is left of that where requests are many and short: 256 of 25 to 100 tokens on 40 heads are 20 rounds of workgroups, 106 us,
// in which one wave of four is busy.
// (16 bytes at a time: the second pass has no more than the type to go by)
struct alignas(16) FewShared {
    float sums[4][16][132], stats[4][16][2];
    uint32_t odd[4];                                     // of each wave: some value is one that the first pass does not take
    static_assert(sizeof sums[0][0] % 16 == 0);
};

// Scales that the first pass does not take.  Of bfloat16 values those that are not 108 to 139 (2^-19 to 2^12), of which halves
// hold the values: the bytes of a word less 108 are below 32 each.  (Where one is not, those above it may be off by its borrow, but it
// shows itself.)  Of binary16 those above the largest, 140, which is the mark alone: its lower seven bits and 115 pass 127.
// (A token each of 64 requests of 1024 to 4096 tokens, 40 heads of 128, all scales 104 to 107: 157 us, and 411 with the range of bfloat16.)
template <bool BF16> __device__ __forceinline__ uint32_t odd_scales(uint4_t s) {
    if constexpr (BF16) {
        constexpr uint32_t lowest = 0x6C6C6C6Cu;
        return ((s[0] - lowest) | (s[1] - lowest) | (s[2] - lowest) | (s[3] - lowest)) & 0xE0E0E0E0u;
    } else {
        static_assert(FourScales<false>::highest == 128 + 127 - 115);
        uint32_t odd = 0;
        for (int i = 0; i < 4; ++i) odd |= ((s[i] & 0x7F7F7F7Fu) + 0x73737373u) & s[i];
        return odd & 0x80808080u;
    }
}

// CAREFUL: the second pass, for values that halves do not hold (of bfloat16), or that are NaN and not seen by all rows.
// -> whether the second pass is wanted.
template <int D, bool BF16, int SETS, bool ONCE, bool CAREFUL>
__device__ __forceinline__ bool attend_four_few(const AttendArgs &a, FewShared &shared) {
    constexpr int ROWS = 16 * SETS;
    constexpr int KW = D / 32;                           // words of a lane's keys of a token, and products of a score
    constexpr int KS = D == 256 ? 2 : 1;                 // scales of them
    constexpr int VE = D / 16;                           // elements of a lane's values of a token: 4, 8 or 16
    constexpr int VW = D == 256 ? 2 : 1;                 // words of them
    constexpr int GROUPS = D / 32;
    constexpr bool VALUES_BF16 = BF16 && CAREFUL;
    auto &sums = shared.sums;
    auto &stats = shared.stats;
    Place p;
    if (!find_place<ROWS, true>(a, p)) return false;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
    const uint32_t B = 1u << a.block_log2;
    uint32_t again = 0;
    const uint8_t *all_k = static_cast<const uint8_t *>(a.k), *all_v = static_cast<const uint8_t *>(a.v);
    const uint8_t *all_ks = static_cast<const uint8_t *>(a.k_scale), *all_vs = static_cast<const uint8_t *>(a.v_scale);
    for (uint32_t tile = p.tile;; ++tile) {
        const uint32_t rows = p.n * a.group;
        const Reach reach = reach_of<ROWS, true>(a, p, tile);
        const bool done = !p.last || (uint64_t)(tile + 1) * ROWS >= rows;
        if (a.splits > 1 && reach.begin >= reach.end) {
            nothing_seen<ROWS>(a, p, tile, D);
            if (done) return again != 0;
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
            to[c] = min(to[c], 0x7FFFFFFFu);
        }
        float4_t acc[SETS][VE];
        float ref[SETS], weight[SETS];
        bool coarse[SETS];           // (see k_attend_four_many)
        uint32_t odd = 0;
#pragma unroll
        for (int c = 0; c < SETS; ++c) {
            for (int j = 0; j < VE; ++j) acc[c][j] = float4_t{0, 0, 0, 0};
            ref[c] = kNone;
            weight[c] = 0.0f;
            coarse[c] = false;
        }

        // Loads are always on their way: a tile's keys are asked for while the tile before it is worked on, its values
        // when that one's are used up, and its block numbers a tile earlier still.
        uint32_t kw[4][KW], vw[16][VW];
        uint4_t ks[KS], vs;
        bool bad = false;
        auto ask_keys = [&](uint32_t t0, uint32_t id) {
            const uint32_t key_id = (uint32_t)__shfl((int)id, (int)(m >> 2) << 4), place = (t0 + 16 * (m >> 2)) & (B - 1);
            const uint64_t head = (uint64_t)key_id * a.kv_heads + p.h;
            const uint8_t *keys = all_k + (head * B + place + (m & 3)) * (D / 2) + g * (D / 8);
            const uint8_t *scales = all_ks + (head * GROUPS + g * (D / 4) / 32) * B + place;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint8_t *at = keys + 4 * t * (D / 2);
                if constexpr (D == 64) {
                    const uint2_t w = codes_at<ONCE, uint2_t>(at);
                    kw[t][0] = w[0]; kw[t][1] = w[1];
                } else {
                    for (int x = 0; x < KW; x += 4) {
                        const uint4_t w = codes_at<ONCE, uint4_t>(at + 4 * x);
                        for (int i = 0; i < 4; ++i) kw[t][x + i] = w[i];
                    }
                }
            }
            for (int x = 0; x < KS; ++x) ks[x] = *reinterpret_cast<const uint4_t *>(scales + x * B);
        };
        auto ask_values = [&](uint32_t t0, uint32_t id) {
            const uint32_t place = (t0 + 16 * g) & (B - 1);
            const uint64_t head = (uint64_t)id * a.kv_heads + p.h;
            const uint8_t *values = all_v + (head * B + place) * (D / 2) + m * (D / 32);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if constexpr (D == 64) vw[i][0] = codes_at<ONCE, uint16_t>(values + i * (D / 2));
                else if constexpr (D == 128) vw[i][0] = codes_at<ONCE, uint32_t>(values + i * (D / 2));
                else {
                    const uint2_t w = codes_at<ONCE, uint2_t>(values + i * (D / 2));
                    vw[i][0] = w[0]; vw[i][1] = w[1];
                }
            }
            vs = *reinterpret_cast<const uint4_t *>(all_vs + (head * GROUPS + m * VE / 32) * B + place);
        };
        uint32_t t0 = reach.begin + 64 * wave;
        if (t0 < reach.end) {
            const uint32_t first = table_entry(a, p, t0 + 16 * g, reach.end);
            uint32_t next = table_entry(a, p, t0 + 256 + 16 * g, reach.end);
            bad = is_bad(a, p, first);
            ask_keys(t0, id_of(a, first));
            ask_values(t0, id_of(a, first));
            do {                     // (not a loop that may be left out: its loads would be waited for along with the queries')
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
                const bool lost = bad;
                const float all_factor = lost ? __builtin_nanf("") : a.scale_log2;
                // (the entry is used up before the next one is asked for: a copy of it would wait for that)
                const uint32_t mine = t0 + 16 * g, id = id_of(a, next);
                bad = is_bad(a, p, next);
                next = table_entry(a, p, t0 + 512 + 16 * g, reach.end);
                ask_keys(t0 + 256, id);
                // weights, and the reference
                uint4_t pw[SETS][2], rest[SETS][2];
#pragma unroll
                for (int c = 0; c < SETS; ++c) {
                    float factor = all_factor;
                    if (coarse[c] || __ballot(mine < from[c] || mine + 16 > to[c])) {
                        const int first = (int)(from[c] - mine), behind = (int)(to[c] - mine);
#pragma unroll
                        for (int e = 0; e < 16; ++e) s[c][e / 4][e & 3] = e < first || e >= behind ? -INFINITY : s[c][e / 4][e & 3] * factor;
                        factor = 1.0f;
                    }
                    float top = -INFINITY;
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[c][t][i]);
                    top = max_across_halves(max_across_sixteen(top * factor));
                    constexpr float room = Softmaxes<VALUES_BF16>::room, slack = Softmaxes<VALUES_BF16>::slack;
                    if (__ballot(top > ref[c] + (room + slack))) {
                        const float now = fmaxf(ref[c], top - room), down = pow2(ref[c] - now);
                        ref[c] = now;
                        weight[c] *= down;
                        for (int j = 0; j < VE; ++j) acc[c][j] *= down;
                        if (!coarse[c] && __ballot(fabsf(now) > kCoarse && fabsf(now) < -kNone)) {       // from here on
                            coarse[c] = true;
#pragma unroll
                            for (int t = 0; t < 4; ++t)
                                for (int i = 0; i < 4; ++i) s[c][t][i] *= factor;
                            factor = 1.0f;
                        }
                    }
                    float sum = 0.0f;
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        for (int i = 0; i < 4; i += 2) {
                            const float e0 = pow2(__builtin_fmaf(s[c][t][i], factor, -ref[c])), e1 = pow2(__builtin_fmaf(s[c][t][i + 1], factor, -ref[c]));
                            sum += e0 + e1;
                            const uint32_t w = pack_two<VALUES_BF16>(e0, e1);
                            pw[c][t / 2][2 * (t & 1) + i / 2] = w;
                            if constexpr (VALUES_BF16) rest[c][t / 2][2 * (t & 1) + i / 2] = pack_two<true>(e0 - widen<true>(w & 0xFFFFu), e1 - widen<true>(w >> 16));
                        }
                    weight[c] += sum;
                }
                // No value that is not seen may bring NaN or infinity into a sum with a weight of 0.  (A token whose values are NaN
                // has keys that are NaN, too.)  Scales of tokens that no row of the tile sees, and of tokens in no block, may be
                // anything, and decide nothing.
                if (t0 + 64 > reach.end || t0 < reach.first || __ballot(lost)) {
                    const int first = lost ? 16 : (int)(reach.first - mine), behind = (int)(reach.end - mine);
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (e < first || e >= behind) vs[e / 4] = (vs[e / 4] & ~(0xFFu << 8 * (e & 3))) | 127u << 8 * (e & 3);
                }
                if constexpr (!CAREFUL) odd |= odd_scales<BF16>(vs);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float scale[8];
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t w = vs[2 * u + e / 4];
                        scale[e] = CAREFUL ? four_scale(min(w >> 8 * (e & 3) & 0xFFu, (uint32_t)FourScales<BF16>::highest)) :
                                   (e & 3) == 0 ? four_scale_at<0>(w) : (e & 3) == 1 ? four_scale_at<1>(w) : (e & 3) == 2 ? four_scale_at<2>(w) : four_scale_at<3>(w);
                    }
                    auto each = [&](auto pair) {         // two elements of the lane's: byte pair % 4 of word pair / 4
                        constexpr int P = pair();
                        uint4_t one, two;
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t x = four_pair<VALUES_BF16, P % 4>(vw[8 * u + 2 * e][P / 4], scale[2 * e]);
                            const uint32_t y = four_pair<VALUES_BF16, P % 4>(vw[8 * u + 2 * e + 1][P / 4], scale[2 * e + 1]);
                            one[e] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                            two[e] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                        }
                        for (int c = 0; c < SETS; ++c) {
                            acc[c][2 * P] = product<VALUES_BF16>(one, pw[c][u], acc[c][2 * P]);
                            acc[c][2 * P + 1] = product<VALUES_BF16>(two, pw[c][u], acc[c][2 * P + 1]);
                            if constexpr (VALUES_BF16) {
                                acc[c][2 * P] = product<true>(one, rest[c][u], acc[c][2 * P]);
                                acc[c][2 * P + 1] = product<true>(two, rest[c][u], acc[c][2 * P + 1]);
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
                ask_values(t0 + 256, id);
                t0 += 256;
                asm volatile("" ::: "memory");           // (the loads are to stay here: at the loop's head they would wait for the keys)
            } while (t0 < reach.end);
        }
        const bool any_odd = !CAREFUL && __ballot(odd != 0);
        if (!CAREFUL && lane == 0) shared.odd[wave] = any_odd;

        // the four waves' sums, at one reference
#pragma unroll
        for (int c = 0; c < SETS; ++c) {
            weight[c] += __shfl_xor(weight[c], 16);
            weight[c] += __shfl_xor(weight[c], 32);
            if (c) __syncthreads();
            if (g == 0) { stats[wave][m][0] = ref[c]; stats[wave][m][1] = weight[c]; }
            __syncthreads();
            if (!CAREFUL && c == 0) again |= shared.odd[0] | shared.odd[1] | shared.odd[2] | shared.odd[3];
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
                        for (int i = 0; i < 4; ++i) w[i] = pack_two<BF16>(y[2 * i], y[2 * i + 1]);
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
        if (done) return again != 0;
        __syncthreads();
    }
}

// The kernel's arguments, in a function that it calls at its end.
typedef const __attribute__((address_space(4))) void *KernelArgs;
__device__ __forceinline__ AttendArgs args_of(KernelArgs args) {
    struct Words { uint32_t w[sizeof(AttendArgs) / 4]; } words;
    const uint64_t bits = (uint64_t)args;
    const uint64_t from = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(bits >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)bits);
    for (uint32_t i = 0; i < sizeof(AttendArgs) / 4; ++i) words.w[i] = ((const __attribute__((address_space(4))) uint32_t *)from)[i];
    return __builtin_bit_cast(AttendArgs, words);
}

// All of a workgroup's tiles once more.  Not inlined, and the last thing that it does: what this pass keeps in registers would be
// taken from the first one's loop.
template <int D, bool BF16, int SETS>
__device__ __attribute__((noinline)) void attend_four_few_again(KernelArgs args, __attribute__((address_space(3))) FewShared *shared) {
    attend_four_few<D, BF16, SETS, false, true>(args_of(args), *(FewShared *)shared);
}

// (Two waves a SIMD, whose registers a second set would not fit with heads of 256; three with heads of 64.  64 requests of 1024 to 4096
// tokens: 16 heads on 8 of 256 77.7 us and 86.0 with one wave, 12 of 64 38.7 and 45.5 with two; heads of 128 lose by a third.)
template <int D, bool BF16, int SETS, bool ONCE>
__global__ __launch_bounds__(256, D == 64 && SETS == 1 ? 3 : 2) void k_attend_four_few(AttendArgs a) {
    __shared__ FewShared shared;
    if (__builtin_amdgcn_readfirstlane((int)attend_four_few<D, BF16, SETS, ONCE, false>(a, shared))) {
        __syncthreads();
        attend_four_few_again<D, BF16, SETS>((KernelArgs)__builtin_amdgcn_kernarg_segment_ptr(), (__attribute__((address_space(3))) FewShared *)&shared);
    }
}

// Many rows: 32 of a kv head's a wave, eight waves a workgroup (four, where a request has no more than 128 rows, and for
// heads of 256, whose sums and queries take the registers of two).  A tile of 128 tokens (64) goes through registers into
// LDS, converted, once for all rows; one barrier a tile is all that the waves wait for.  Keys and values lie there token by
// token; the values' operand, which wants tokens side by side, is read by the transposing loads: of 16 lanes, which
// point at four tokens' pieces of 16 elements, each gets one element of the four tokens.
// Lane (n = lane % 32, hi = lane / 32).  S^T in two 32 x 32 pieces: register i of a piece is token
// 8 (i / 4) + 4 hi + i % 4, row n.  P^T as an operand of 16 tokens: registers 8u .. 8u + 7, tokens 4 hi + (0..3) and
// 8 + 4 hi + (0..3) of the 16.
//
// Weights are halves.  Values of bfloat16 are converted to halves, too, as long as halves hold them exactly (all scales
// of 2^-23 to 2^13); a workgroup that meets others begins again with bfloat16 values and weights in two parts (SPLIT).
//
// The matrix instructions and the vector ones, which share a wave's issue, bound it; each is busy for half of the time: a prompt
// of 8192 tokens, 64 heads of 128 on 8, 983 to 1026 us, 1.07 to 1.12 PFLOP/s (840 on zeros, which cost no clock), where a product
// of two large matrices reaches 1.15 to 1.25; 448 rows over 1500 tokens, 20 heads of 64, six requests, 37 us.  Heads of 64 have
// half the products for the same exponentials: 8000 tokens on 20 heads, twice, 420 to 427 us, 0.78 PFLOP/s.
//
// Heads of 256 put a token's pieces of 16 bytes at other places within their 64, such that eight lanes that write at a time
// meet in no bank: a prompt of 4096 tokens on 16 heads, 214 us instead of 238 when that was done, 176 now.  (Heads of 128 do not notice, of 64 lose 3 % by
// it, and readers of values, who would meet nowhere with rows of D + 32, gain nothing by that.)
template <int D, int TOKENS>
struct alignas(16) FourTile {
    uint16_t k[TOKENS][D + 8];                           // (neighbours begin four banks apart ...
    uint16_t v[TOKENS][D + 16];                          // ... and eight)
    static_assert(sizeof k[0] % 16 == 0 && sizeof v[0] % 16 == 0, "rows are read and written 16 bytes at a time");
};
template <int D> __device__ constexpr uint32_t turned_by(uint32_t part) { return D == 256 ? part >> 1 & 3 : 0; }

// How a block's LOADS loads from LDS and PRODUCTS products are to be issued: the loads of some products, then the others behind the products.
// (Two for heads of 256, which have few registers left: a prompt of 4096 194 us, with four 206, with one 228; the others do not notice.)
template <int D, int LOADS, int PRODUCTS, int GROUP> __device__ __forceinline__ void loads_among_products() {
    constexpr int kLoad = 0x100, kProduct = 0x8, EACH = LOADS / PRODUCTS, AHEAD = D == 256 ? 2 : 4;
    __builtin_amdgcn_sched_group_barrier(kLoad, AHEAD * EACH, GROUP);
#pragma unroll
    for (int i = 0; i < PRODUCTS - AHEAD; ++i) {
        __builtin_amdgcn_sched_group_barrier(kProduct, 1, GROUP);
        __builtin_amdgcn_sched_group_barrier(kLoad, EACH, GROUP);
    }
    __builtin_amdgcn_sched_group_barrier(kProduct, AHEAD, GROUP);
}

// Products of 32 x 32 x 16.
template <bool BF16> __device__ __forceinline__ float16_t wide_product(uint4_t x, uint4_t y, float16_t z) {
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, x), __builtin_bit_cast(bf16x8_t, y), z, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, x), __builtin_bit_cast(half8_t, y), z, 0, 0, 0);
}

// Four tokens' elements of LDS, one element of each (see above).
__device__ __forceinline__ uint2_t transposed(const uint16_t *at) {
    typedef short short4_t __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(uint2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t *)at));
}

// A wave goes ahead of the other of its SIMD where it has products to issue (a prompt of 8192 on 64 heads of 128 1034 us, without 1089).
// Heads of 256 have one wave a SIMD, and lose by it the order in which the compiler would issue a tile (232 us, without 210).
template <int D> __device__ __forceinline__ void ahead(bool yes) {
    if constexpr (D != 256) {
        if (yes) __builtin_amdgcn_s_setprio(1);
        else __builtin_amdgcn_s_setprio(0);
    }
}

template <int D, bool BF16, int WAVES, int TOKENS, bool SPLIT>
__device__ __forceinline__ void attend_four_tile(const AttendArgs &a, const Place &p, uint32_t tile, const Reach &reach,
                                                 FourTile<D, TOKENS> *buffer, uint32_t *outside) {
    constexpr int ROWS = 32 * WAVES, THREADS = 64 * WAVES;
    constexpr int E = D == 64 ? 16 : 32, PT = D / E, GROUPS = D / 32;        // elements of a piece, pieces of a token
    constexpr int N = TOKENS * PT / THREADS;             // pieces of keys, and of values, that a thread stages
    constexpr bool VALUES_BF16 = BF16 && SPLIT;
    constexpr int SUB = SPLIT || TOKENS == 32 ? 32 : 64, C = SUB / 32;   // tokens whose scores a wave has at once
    typedef FourTile<D, TOKENS> Tile;
    typedef typename std::conditional<E == 16, uint2_t, uint4_t>::type Piece;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6)), n = lane & 31, hi = lane >> 5;
    const uint32_t B = 1u << a.block_log2;
    const uint32_t row = tile * ROWS + wave * 32 + n, rows = p.n * a.group;
    uint4_t q[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
        q[s] = uint4_t{0, 0, 0, 0};
        if (row < rows) {
            const uint16_t *src = static_cast<const uint16_t *>(a.q) + (uint64_t)(p.begin + row / a.group) * a.q_stride +
                                  (uint64_t)(p.h * a.group + row % a.group) * D + 16 * s + 8 * hi;
            q[s] = *reinterpret_cast<const uint4_t *>(src);
        }
    }
    uint32_t from, to;
    row_sees(a, p, row, from, to);
    if (tile * ROWS + wave * 32 >= rows) to = 0;         // (a wave without rows only helps to stage)

    float16_t acc[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;
    float ref = kNone, weight = 0.0f;
    bool coarse = false;             // some row's reference, a finite one, is too large for an exponent to be made in one rounding
    constexpr float room = Softmaxes<VALUES_BF16>::room, slack = Softmaxes<VALUES_BF16>::slack;

    // staging: what this thread brings of a tile, asked for a tile ahead, its table entries two
    uint32_t asked[N], entry[N];
    Piece kw[N], vw[N];
    uint32_t ks[N], vs[N];
    uint32_t code_at[N], scale_at[N];                    // of the thread's pieces in a block, for tiles that begin with one
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t e = i * THREADS + tid, place = e / PT & (B - 1), piece = e % PT;
        code_at[i] = place * (D / 2) + piece * (E / 2);
        scale_at[i] = piece * E / 32 * B + place;
    }
    const uint8_t *all_k = static_cast<const uint8_t *>(a.k) + (uint64_t)p.h * B * (D / 2), *all_v = static_cast<const uint8_t *>(a.v) + (uint64_t)p.h * B * (D / 2);
    const uint8_t *all_ks = static_cast<const uint8_t *>(a.k_scale) + (uint64_t)p.h * B * GROUPS, *all_vs = static_cast<const uint8_t *>(a.v_scale) + (uint64_t)p.h * B * GROUPS;
    auto ask_entries = [&](uint32_t t0) {
#pragma unroll
        for (int i = 0; i < N; ++i) entry[i] = table_entry(a, p, t0 + (i * THREADS + tid) / PT, reach.end);
    };
    auto ask = [&](uint32_t t0) {
        const uint32_t within = t0 & (B - 1);            // (of blocks longer than a tile)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t head = (uint64_t)id_of(a, entry[i]) * a.kv_heads * B;
            const uint64_t codes = head * (D / 2) + within * (D / 2) + code_at[i], scale = head * GROUPS + within + scale_at[i];
            kw[i] = *reinterpret_cast<const Piece *>(all_k + codes);
            vw[i] = *reinterpret_cast<const Piece *>(all_v + codes);
            ks[i] = all_ks[scale];
            vs[i] = all_vs[scale];
            asked[i] = entry[i];
        }
    };
    auto put = [&](Tile &t, uint32_t t0, uint32_t first) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t e = i * THREADS + tid, token = e / PT, at = e % PT * E;
            const bool lost = is_bad(a, p, asked[i]);
            const float k_scale = four_scale(lost ? kNotANumber : ks[i]);
            // (no value may bring NaN or infinity into a sum with a weight of 0: see k_attend_four_few)
            typedef FourScales<VALUES_BF16> Held;
            // (scales of tokens that no row of the tile sees, and of tokens in no block, may be anything, and decide nothing)
            if constexpr (BF16 && !SPLIT)
                if ((vs[i] < Held::lowest || vs[i] > Held::highest) && t0 + token >= first && t0 + token < reach.end && !lost) *outside = 1;
            const float v_scale = four_scale(min(vs[i], (uint32_t)Held::highest));
            const uint32_t turn = turned_by<D>(e % PT);
            for (int j = 0; j < E / 8; ++j) {
                *reinterpret_cast<uint4_t *>(&t.k[token][at + 8 * (j ^ turn)]) = four_eight<BF16>(kw[i][j], k_scale);
                *reinterpret_cast<uint4_t *>(&t.v[token][at + 8 * (j ^ turn)]) = four_eight<VALUES_BF16>(vw[i][j], v_scale);
            }
        }
    };
    if (reach.begin < reach.end) {
        uint32_t at = 0, t0 = reach.begin;
        // (the first token that some row sees is one of the first tile's)
        if (TOKENS < 128 && t0 + TOKENS <= reach.first && t0 + TOKENS < reach.end) t0 += TOKENS;
        ask_entries(t0);
        ask(t0);
        ask_entries(t0 + TOKENS);
        put(buffer[0], t0, reach.first);
        ask(t0 + TOKENS);
        ask_entries(t0 + 2 * TOKENS);
        __syncthreads();
        do {                         // (not a loop that may be left out: its loads would be waited for along with the queries')
            const Tile &t = buffer[at];
#pragma unroll SPLIT ? 1 : TOKENS / SUB
            for (uint32_t part = 0; part < TOKENS; part += SUB) {
                const uint32_t u0 = t0 + part;
                // (a wave whose rows all end before these tokens, or begin behind them, only helps to stage)
                if (!__ballot(from < u0 + SUB && to > u0)) continue;
                float16_t s[C];
                ahead<D>(true);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    for (int i = 0; i < 16; ++i) s[c][i] = 0.0f;
#pragma unroll
                    for (int e = 0; e < D / 16; ++e) {
                        constexpr int EACH = E / 16;     // products of a lane's piece
                        const uint32_t turn = turned_by<D>(e / EACH);
                        const uint16_t *at = &t.k[part + 32 * c + n][16 * (e ^ (turn >> 1)) + 8 * (hi ^ (turn & 1))];
                        s[c] = wide_product<BF16>(*reinterpret_cast<const uint4_t *>(at), q[e], s[c]);
                    }
                }
                loads_among_products<D, C * D / 16, C * D / 16, 0>();
                ahead<D>(false);
                const bool whole = __ballot(u0 < from || u0 + SUB > to) == 0;
                if (!whole) {
#pragma unroll
                    for (int c = 0; c < C; ++c)
                        for (int i = 0; i < 16; ++i) {
                            const uint32_t token = u0 + 32 * c + 8 * (i / 4) + 4 * hi + i % 4;
                            if (token < from || token >= to) s[c][i] = -INFINITY;
                        }
                }
                float top = -INFINITY;
#pragma unroll
                for (int c = 0; c < C; ++c)
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[c][i]);
                top = max_across_halves(top) * a.scale_log2;
                float factor = a.scale_log2;
                if (coarse || __ballot(top > ref + (room + slack))) {
                    const float now = fmaxf(ref, top - room), down = pow2(ref - now);
                    ref = now;
                    weight *= down;
#pragma unroll
                    for (int d = 0; d < D / 32; ++d) acc[d] *= down;
                    coarse = __ballot(fabsf(ref) > kCoarse && fabsf(ref) < -kNone) != 0;
                    if (coarse) {                            // the reference is rounded: so is what it is taken from
#pragma unroll
                        for (int c = 0; c < C; ++c)
                            for (int i = 0; i < 16; ++i) s[c][i] *= factor;
                        factor = 1.0f;
                    }
                }
                float sum[2 * C];
                uint4_t pw[2 * C], rest[2 * C];
#pragma unroll
                for (int u = 0; u < 2 * C; ++u) {
                    sum[u] = 0.0f;
                    for (int i = 0; i < 8; i += 2) {
                        const float e0 = pow2(__builtin_fmaf(s[u / 2][8 * (u & 1) + i], factor, -ref)), e1 = pow2(__builtin_fmaf(s[u / 2][8 * (u & 1) + i + 1], factor, -ref));
                        sum[u] += e0 + e1;
                        const uint32_t w = pack_two<VALUES_BF16>(e0, e1);
                        pw[u][i / 2] = w;
                        if constexpr (SPLIT) rest[u][i / 2] = pack_two<true>(e0 - widen<true>(w & 0xFFFFu), e1 - widen<true>(w >> 16));
                    }
                }
                for (int u = 1; u < 2 * C; ++u) sum[0] += sum[u];
                weight += sum[0];
                ahead<D>(true);
#pragma unroll
                for (int d = 0; d < D / 32; ++d)
#pragma unroll
                    for (int u = 0; u < 2 * C; ++u) {
                        // (eight elements of a token and 32: 4d + 2 (n / 16) + (lane % 4) / 2, turned as they were put)
                        const uint32_t nth = 2 * (n / 16) + (lane & 3) / 2;
                        const uint16_t *from_lds = &t.v[part + 16 * u + 4 * hi + (lane & 15) / 4][32 * d + 8 * (nth ^ turned_by<D>(d)) + 4 * (lane & 1)];
                        const uint2_t x = transposed(from_lds), y = transposed(from_lds + 8 * (D + 16));
                        const uint4_t v = {x[0], x[1], y[0], y[1]};
                        acc[d] = wide_product<VALUES_BF16>(v, pw[u], acc[d]);
                        if constexpr (SPLIT) acc[d] = wide_product<true>(v, rest[u], acc[d]);
                    }
                if constexpr (!SPLIT) loads_among_products<D, 4 * C * D / 32, 2 * C * D / 32, 1>();
                ahead<D>(false);
            }
            if (t0 + TOKENS < reach.end) put(buffer[at ^ 1], t0 + TOKENS, 0);
            ask(t0 + 2 * TOKENS);
            ask_entries(t0 + 3 * TOKENS);
            __syncthreads();
            t0 += TOKENS;
            at ^= 1;
        } while (t0 < reach.end);
    }
    weight += __shfl_xor(weight, 32);
    if (is_lost(a, p, row)) weight = __builtin_nanf("");
    if (row < rows) {
        const uint64_t id = row_id(a, p, row);
        if (a.splits == 1) {
            const float back = weight == 0.0f ? 0.0f : 1.0f / weight;
            uint16_t *dst = static_cast<uint16_t *>(a.out) + (uint64_t)(p.begin + row / a.group) * a.out_stride +
                            (uint64_t)(p.h * a.group + row % a.group) * D + 4 * hi;
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
                for (int b = 0; b < 4; ++b)
                    *reinterpret_cast<uint2_t *>(dst + 32 * d + 8 * b) = uint2_t{pack_two<BF16>(acc[d][4 * b] * back, acc[d][4 * b + 1] * back),
                                                                                 pack_two<BF16>(acc[d][4 * b + 2] * back, acc[d][4 * b + 3] * back)};
            if (a.lse && hi == 0) a.lse[id] = weight == 0.0f ? -INFINITY : (ref + log2_of(weight)) * 0.69314718055994530942f;
        } else {
            float *dst = a.parts + (id * a.splits + p.split) * D + 4 * hi;
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
                for (int b = 0; b < 4; ++b)
                    *reinterpret_cast<float4_t *>(dst + 32 * d + 8 * b) = float4_t{acc[d][4 * b], acc[d][4 * b + 1], acc[d][4 * b + 2], acc[d][4 * b + 3]};
            if (hi == 0) {
                float *st = a.parts + a.part_rows * a.splits * D + (id * a.splits + p.split) * 2;
                st[0] = ref;
                st[1] = weight;
            }
        }
    }
}

// A workgroup's tiles: one, or what is left of a request with more rows than were announced.
template <int D, bool BF16, int WAVES, int TOKENS, bool SPLIT>
__device__ __forceinline__ void attend_four_tiles(const AttendArgs &a, FourTile<D, TOKENS> *buffer, uint32_t *outside) {
    constexpr int ROWS = 32 * WAVES;
    Place p;
    if (!find_place<ROWS>(a, p)) return;
    for (uint32_t tile = p.tile;; ++tile) {
        const uint32_t rows = p.n * a.group;
        const Reach reach = reach_of<ROWS, true>(a, p, tile);
        const bool done = !p.last || (uint64_t)(tile + 1) * ROWS >= rows;
        if (a.splits > 1 && reach.begin >= reach.end) nothing_seen<ROWS>(a, p, tile, D);
        else attend_four_tile<D, BF16, WAVES, TOKENS, SPLIT>(a, p, tile, reach, buffer, outside);
        if (done) return;
        __syncthreads();
    }
}

// All of them once more.  Not inlined, and the last thing that a workgroup does: what this pass keeps in registers would be
// taken from the first one's loop, which then loads its operands one by one.
template <int D, int WAVES, int TOKENS>
__device__ __attribute__((noinline)) void attend_four_many_again(KernelArgs args, __attribute__((address_space(3))) FourTile<D, TOKENS> *buffer) {
    attend_four_tiles<D, true, WAVES, TOKENS, true>(args_of(args), (FourTile<D, TOKENS> *)buffer, nullptr);
}

template <int D, bool BF16, int WAVES, int TOKENS>
__global__ __launch_bounds__(64 * WAVES, D == 256 ? 1 : 2) void k_attend_four_many(AttendArgs a) {
    __shared__ FourTile<D, TOKENS> buffer[2];
    __shared__ uint32_t outside;     // (some value is one that halves do not hold)
    if constexpr (BF16) {
        if (threadIdx.x == 0) outside = 0;
        __syncthreads();
    }
    attend_four_tiles<D, BF16, WAVES, TOKENS, false>(a, buffer, &outside);
    if constexpr (BF16) {
        __syncthreads();
        if (__builtin_amdgcn_readfirstlane((int)outside))
            attend_four_many_again<D, WAVES, TOKENS>((KernelArgs)__builtin_amdgcn_kernarg_segment_ptr(),
                                                     (__attribute__((address_space(3))) FourTile<D, TOKENS> *)buffer);
    }
}

}  // namespace

void launch_attend_four(const CacheShape &s, uint32_t rows, bool once, uint32_t grid, const AttendArgs &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    by_shape(s, [&](auto d, auto bf16) {
        auto few = [&](auto sets) {
            // Streaming loads, not of heads of 64, whose pieces are less than half a line, and where a request has one tile: 64
            // requests of 1024 to 4096 tokens on 40 heads of 128 166 us against 180, on 8 of 256 73.7 against 77.5; but heads of 64
            // 55 against 39, and two tiles of 16 requests of 4096 on 8 heads, which read the cache twice, 43 against 39.
            if constexpr (d() != 64) {
                if (once) { k_attend_four_few<d(), bf16(), sets(), true><<<grid, 256, 0, st>>>(a); return; }
            }
            k_attend_four_few<d(), bf16(), sets(), false><<<grid, 256, 0, st>>>(a);
        };
        if (rows == 16) few(std::integral_constant<int, 1>{});
        else if (rows == 32) { if constexpr (d() != 256) few(std::integral_constant<int, 2>{}); }
        else if (rows == 128) k_attend_four_many<d(), bf16(), 4, 64><<<grid, 256, 0, st>>>(a);
        else if constexpr (d() != 256) k_attend_four_many<d(), bf16(), 8, 128><<<grid, 512, 0, st>>>(a);
    });
}

}  // namespace tsq
