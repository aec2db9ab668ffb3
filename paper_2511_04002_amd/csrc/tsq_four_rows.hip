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

// 16 rows of some heads a workgroup, as many as 512 elements are: rows are read and written one behind the other, the cache's
// tokens head after head, and between the two the codes go through LDS.  Both kernels write whole lines where their rows are
// tokens of a block that follow one another, 256 threads 4 KB of codes.
// Memory bounds both: 22090 rows of 8 heads of 128 (115 MB) are stored in 23.4 us, 4.9 TB/s, and read back in 21.3, 5.4 TB/s;
// 477 MB of ragged requests in 84 us, 5.7 TB/s, where a kernel that only reads and writes as much takes 84 to 88.  Straight
// through registers the first took 25.6 and the last, out of blocks of 64, 112.
constexpr uint32_t kElements = 512;
template <int D> struct FourRows {
    static constexpr uint32_t heads = kElements / D, pieces = D / 32, groups = D / 32;    // pieces: of 16 bytes, of a head's row
    uint8_t codes[2][16][kElements / 2 + 16], scales[2][16][kElements / 32 + 4];
};
// The head, row and piece that a thread has of the cache.
template <int D> struct FourPiece {
    uint32_t h, r, piece;
    __device__ __forceinline__ FourPiece() : h(threadIdx.x / (D / 32) / 16), r(threadIdx.x / (D / 32) % 16), piece(threadIdx.x % (D / 32)) {}
};

// A token does not depend on another.
template <int D, bool BF16, bool ONCE>
__global__ __launch_bounds__(256) void k_append_four(AppendFourArgs a, uint32_t groups_each) {
    typedef FourRows<D> Rows;
    constexpr uint32_t LPH = D / 8;                      // lanes with eight elements each of a head
    __shared__ __attribute__((aligned(16))) Rows rows;
    const uint32_t tid = threadIdx.x, lane = tid & 63, B = 1u << a.block_log2;
    const uint64_t begin = (uint64_t)(blockIdx.x / groups_each) * 16;
    const uint32_t h0 = blockIdx.x % groups_each * Rows::heads, heads = min(Rows::heads, a.kv_heads - h0);
    const uint32_t slot = begin + (lane & 15) < a.tokens ? (uint32_t)a.slots[begin + (lane & 15)] : ~0u;
    uint4_t x[2][4];
    const bool there = lane < heads * LPH;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t row = begin + 4 * i + (tid >> 6), at = (uint64_t)h0 * D + 8 * lane;
        x[0][i] = x[1][i] = uint4_t{0, 0, 0, 0};
        if (there && row < a.tokens) {
            const uint4_t *k = reinterpret_cast<const uint4_t *>(static_cast<const uint16_t *>(a.k) + row * a.k_stride + at);
            const uint4_t *v = reinterpret_cast<const uint4_t *>(static_cast<const uint16_t *>(a.v) + row * a.v_stride + at);
            x[0][i] = ONCE ? __builtin_nontemporal_load(k) : *k;
            x[1][i] = ONCE ? __builtin_nontemporal_load(v) : *v;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t r = 4 * i + (tid >> 6), mk = most_of_four(most_of(x[0][i])), mv = most_of_four(most_of(x[1][i]));
        const uint64_t odd = __ballot(max(mk, mv) >= (BF16 ? 0x7F80u : 0x7C00u));
        const bool bad = (odd >> (lane / LPH * LPH) & (~0ull >> (64 - LPH))) != 0;
        for (int y = 0; y < 2; ++y) {
            const uint32_t byte = scale_byte<BF16>(y ? mv : mk);
            *reinterpret_cast<uint32_t *>(&rows.codes[y][r][4 * lane]) = four_codes<BF16>(x[y][i], four_scale(byte));
            if (lane % 4 == 0) rows.scales[y][r][lane / 4] = (uint8_t)(bad ? kNotANumber : byte);
        }
    }
    __syncthreads();
    uint8_t *const codes[2] = {a.k_codes, a.v_codes}, *const scales[2] = {a.k_scale, a.v_scale};
    {
        const FourPiece<D> p;
        const uint32_t of_row = (uint32_t)__shfl((int)slot, (int)p.r), block = of_row >> a.block_log2, place = of_row & (B - 1);
        if (block < a.blocks && p.h < heads) {           // (a negative slot's is past all)
            const uint64_t head = (uint64_t)block * a.kv_heads + h0 + p.h;
            for (int y = 0; y < 2; ++y)
                *reinterpret_cast<uint4_t *>(codes[y] + (head * B + place) * (D / 2) + 16 * p.piece) =
                    *reinterpret_cast<const uint4_t *>(&rows.codes[y][p.r][p.h * (D / 2) + 16 * p.piece]);
        }
    }
    // scales: a group's of 16 rows side by side
    const uint32_t r = tid % 16, group = tid / 16, h = group / Rows::groups, block = slot >> a.block_log2, place = slot & (B - 1);
    if (block < a.blocks && h < heads) {
        const uint64_t head = (uint64_t)block * a.kv_heads + h0 + h;
        for (int y = 0; y < 2; ++y) scales[y][(head * Rows::groups + group % Rows::groups) * B + place] = rows.scales[y][r][group];
    }
}

template <int D, bool BF16>
__global__ __launch_bounds__(256) void k_gather_four(GatherArgs a) {
    typedef FourRows<D> Rows;
    __shared__ __attribute__((aligned(16))) Rows rows;
    const uint32_t tid = threadIdx.x, B = a.block_tokens;
    const uint64_t begin = (uint64_t)(blockIdx.x / a.waves_each) * 16;
    const uint32_t h0 = blockIdx.x % a.waves_each * Rows::heads, heads = min(Rows::heads, a.kv_heads - h0);
    const GatherRow row = gather_row(a, begin);
    {
        const FourPiece<D> p;
        const int32_t block = __shfl(row.block, (int)p.r);
        const uint32_t place = (uint32_t)__shfl((int)row.place, (int)p.r);
        const uint64_t head = (uint64_t)max(block, 0) * a.kv_heads + h0 + min(p.h, heads - 1);
        uint4_t w[2];
        uint32_t s[2];
        for (int x = 0; x < 2; ++x) {
            w[x] = *reinterpret_cast<const uint4_t *>(static_cast<const uint8_t *>(a.codes[x]) + (head * B + place) * (D / 2) + 16 * p.piece);
            s[x] = static_cast<const uint8_t *>(a.scale[x])[(head * Rows::groups + p.piece) * B + place];
        }
        for (int x = 0; x < 2; ++x) {
            *reinterpret_cast<uint4_t *>(&rows.codes[x][p.r][p.h * (D / 2) + 16 * p.piece]) = w[x];
            rows.scales[x][p.r][p.h * Rows::groups + p.piece] = (uint8_t)(block < 0 ? kNotANumber : s[x]);
        }
    }
    __syncthreads();
    const uint32_t owned = (uint32_t)__ballot(row.owned && (tid & 63) < 16), at = tid & 63;
    if (at >= heads * (D / 8)) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t r = 4 * i + (tid >> 6);
        if (!(owned >> r & 1)) continue;
        for (int x = 0; x < 2; ++x) {
            const uint4_t y = four_eight<BF16>(*reinterpret_cast<const uint32_t *>(&rows.codes[x][r][4 * at]), four_scale(rows.scales[x][r][at / 4]));
            uint16_t *out = static_cast<uint16_t *>(a.out[x]) + (begin + r) * a.stride[x] + (uint64_t)h0 * D + 8 * at;
            __builtin_nontemporal_store(y, reinterpret_cast<uint4_t *>(out));
        }
    }
}

// Workgroups of 16 rows; 0: too many in all.
uint32_t workgroups_each(const CacheShape &s, uint32_t tokens, uint32_t *grid) {
    const uint64_t groups = ((uint64_t)tokens + 15) / 16, each = ((uint64_t)s.kv_heads * s.head_dim + kElements - 1) / kElements;
    if (!fits(groups * each, 256)) return 0;
    *grid = (uint32_t)(groups * each);
    return (uint32_t)each;
}

}  // namespace

int launch_append_four(const CacheShape &s, const AppendFourArgs &a, void *stream) {
    uint32_t grid;
    const uint32_t each = workgroups_each(s, a.tokens, &grid);
    if (!each) return kTooLarge;
    // Streaming loads where the rows are more than a program has just made and the caches still hold: 22090 rows of 8 heads of 128
    // (90 MB) 23.6 us against 26.0, 30000 29.4 against 33.5; 3500 of 32 (57 MB) 18.0 against 16.7.
    const bool once = 4ull * a.tokens * s.kv_heads * s.head_dim >= 64ull << 20;
    by_shape(s, [&](auto d, auto bf16) {
        if (once) k_append_four<d(), bf16(), true><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a, each);
        else k_append_four<d(), bf16(), false><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a, each);
    });
    return (int)hipGetLastError();
}

int launch_gather_four(const CacheShape &s, const GatherArgs &args, void *stream) {
    GatherArgs a = args;
    uint32_t grid;
    a.waves_each = workgroups_each(s, a.tokens, &grid);
    if (!a.waves_each) return kTooLarge;
    by_shape(s, [&](auto d, auto bf16) { k_gather_four<d(), bf16()><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a); });
    return (int)hipGetLastError();
}

}  // namespace tsq
