// Append and gather of a cache in 4 bits (tsq_cache_append, tsq_cache_gather).
#include "tsq_four.hpp"

namespace tsq {
namespace {

// The largest magnitude of eight 16-bit elements, as bits.
__device__ __forceinline__ uint32_t most_of(uint4_t w) {
    uint32_t m = 0;
    for (int i = 0; i < 4; ++i) m = max(m, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
    return m;
}
// ... of four lanes that follow one another.
__device__ __forceinline__ uint32_t most_of_four(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));
}

// The byte of the least power of two that brings a magnitude to 7 or below: 7 and not 6, since the elements between are
// then no farther off than those between 4 and 6 are.  (Root mean square errors of normal data: 0.112 of its deviation with 7,
// 0.116 with 6, 0.144 with 4.)
template <bool BF16> __device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, widen<BF16>(most));
    const int e = (int)((bits + 0x1FFFFFu) >> 23) - 2;   // (a fraction above 1.75 moves on to the next exponent)
    typedef FourScales<BF16> S;
    return most == 0 ? 127u : (uint32_t)min(max(e, S::lowest), S::highest);
}

template <bool BF16> __device__ __forceinline__ uint32_t four_codes(uint4_t w, float scale) {
    uint32_t c = 0;
    if constexpr (BF16) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, (uint32_t)w[0]), scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, (uint32_t)w[1]), scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, (uint32_t)w[2]), scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, (uint32_t)w[3]), scale, 3);
    } else {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(half2_t, (uint32_t)w[0]), scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(half2_t, (uint32_t)w[1]), scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(half2_t, (uint32_t)w[2]), scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(half2_t, (uint32_t)w[3]), scale, 3);
    }
    return c;
}

// A lane has eight elements of a token's keys of a head, and the values' at the same place: D / 8 lanes a head, 512 / D
// heads a wave.  No token depends on another.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void k_append_four(AppendFourArgs a) {
    constexpr uint32_t LPH = D / 8, HEADS = 64 / LPH, GROUPS = D / 32;
    const uint32_t lane = threadIdx.x & 63, piece = lane % LPH, B = 1u << a.block_log2;
    const uint32_t at = (blockIdx.x * 4 + wave_in_group()) * HEADS + lane / LPH, token = at / a.kv_heads, h = at % a.kv_heads;
    const bool here = token < a.tokens;
    const uint32_t slot = here ? (uint32_t)a.slots[token] : ~0u, block = slot >> a.block_log2, place = slot & (B - 1);
    const bool stored = block < a.blocks;                // (a negative slot's is not)
    uint4_t k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
    if (stored) {
        k = *reinterpret_cast<const uint4_t *>(static_cast<const uint16_t *>(a.k) + token * a.k_stride + (uint64_t)h * D + 8 * piece);
        v = *reinterpret_cast<const uint4_t *>(static_cast<const uint16_t *>(a.v) + token * a.v_stride + (uint64_t)h * D + 8 * piece);
    }
    const uint32_t mk = most_of_four(most_of(k)), mv = most_of_four(most_of(v));
    const uint64_t odd = __ballot(max(mk, mv) >= (BF16 ? 0x7F80u : 0x7C00u));
    const bool bad = (odd >> (lane / LPH * LPH) & (~0ull >> (64 - LPH))) != 0;
    const uint32_t sk = scale_byte<BF16>(mk), sv = scale_byte<BF16>(mv);
    if (!stored) return;
    const uint64_t head = (uint64_t)block * a.kv_heads + h;
    const uint64_t codes = (head * B + place) * (D / 2) + 4 * piece, scale = (head * GROUPS + piece / 4) * B + place;
    *reinterpret_cast<uint32_t *>(a.k_codes + codes) = four_codes<BF16>(k, four_scale(sk));
    *reinterpret_cast<uint32_t *>(a.v_codes + codes) = four_codes<BF16>(v, four_scale(sv));
    if (piece % 4 == 0) {
        a.k_scale[scale] = (uint8_t)(bad ? kNotANumber : sk);
        a.v_scale[scale] = (uint8_t)(bad ? kNotANumber : sv);
    }
}

// 16 rows a wave, and a share of their heads: a lane has eight elements, D / 8 lanes a row of a head.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void k_gather_four(GatherArgs a) {
    constexpr uint32_t LPT = D / 8, TPI = 64 / LPT, LOADS = 16 / TPI, GROUPS = D / 32;
    const uint32_t lane = threadIdx.x & 63, B = a.block_tokens, piece = lane % LPT, sub = lane / LPT;
    const uint64_t begin = ((uint64_t)(blockIdx.x / a.waves_each) * 4 + wave_in_group()) * 16;
    if (begin >= a.tokens) return;
    const GatherRow row = gather_row(a, begin);
    int32_t block[LOADS];                                // -2: no request's row
    uint32_t place[LOADS];
#pragma unroll
    for (uint32_t t = 0; t < LOADS; ++t) {
        block[t] = __shfl(row.owned ? row.block : -2, (int)(TPI * t + sub));
        place[t] = (uint32_t)__shfl((int)row.place, (int)(TPI * t + sub));
    }
    for (uint32_t h = blockIdx.x % a.waves_each; h < a.kv_heads; h += a.waves_each) {
        uint32_t w[2][LOADS], s[2][LOADS];
#pragma unroll
        for (uint32_t t = 0; t < LOADS; ++t) {
            const uint64_t head = (uint64_t)max(block[t], 0) * a.kv_heads + h;
            const uint64_t codes = (head * B + place[t]) * (D / 2) + 4 * piece, scale = (head * GROUPS + piece / 4) * B + place[t];
            for (int x = 0; x < 2; ++x) {
                w[x][t] = *reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(a.codes[x]) + codes);
                s[x][t] = static_cast<const uint8_t *>(a.scale[x])[scale];
            }
        }
#pragma unroll
        for (uint32_t t = 0; t < LOADS; ++t) {
            if (block[t] == -2) continue;
            for (int x = 0; x < 2; ++x) {
                const uint4_t y = four_eight<BF16>(w[x][t], four_scale(block[t] < 0 ? kNotANumber : s[x][t]));
                uint16_t *out = static_cast<uint16_t *>(a.out[x]) + (begin + TPI * t + sub) * a.stride[x] + (uint64_t)h * D + 8 * piece;
                __builtin_nontemporal_store(y, reinterpret_cast<uint4_t *>(out));
            }
        }
    }
}

}  // namespace

int launch_append_four(const CacheShape &s, const AppendFourArgs &a, void *stream) {
    const uint32_t heads = 512 / s.head_dim;             // a wave
    uint32_t grid;
    if (int e = workgroups(((uint64_t)a.tokens * s.kv_heads + heads - 1) / heads, &grid)) return e;
    by_shape(s, [&](auto d, auto bf16) { k_append_four<d(), bf16()><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a); });
    return (int)hipGetLastError();
}

int launch_gather_four(const CacheShape &s, const GatherArgs &args, void *stream) {
    GatherArgs a = args;
    const uint64_t groups = ((uint64_t)a.tokens + 63) / 64;
    uint64_t each = (4096 + groups - 1) / groups;
    if (each > s.kv_heads) each = s.kv_heads;
    a.waves_each = (uint32_t)each;
    if (!fits(groups * each, 256)) return kTooLarge;
    by_shape(s, [&](auto d, auto bf16) { k_gather_four<d(), bf16()><<<(uint32_t)(groups * each), 256, 0, static_cast<hipStream_t>(stream)>>>(a); });
    return (int)hipGetLastError();
}

}  // namespace tsq
