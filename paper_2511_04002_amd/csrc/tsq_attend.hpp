// What the attention kernels of both caches (tsq_attend.hip: 8 bits, tsq_attend_four.hip: 4 bits) have in common: which
// rows a workgroup works on, which tokens they see, where results go.
#pragma once

#include <hip/hip_runtime.h>

#include "tsq_cache_internal.hpp"

namespace tsq {
namespace {

constexpr float kNone = -0x1.fffffep127f;      // reference of a row that has seen nothing: below any score

__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_of(float x) { return __builtin_amdgcn_logf(x); }

// The larger of a lane's value and that of the lane 32 away.
__device__ __forceinline__ float max_across_halves(float x) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
    const uint32_t a = r[0], b = r[1];                   // (a cast of an element itself would take the first)
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// What a workgroup works on: a row tile of a request (rows: query token and head of the group, the group fastest),
// a kv head, and a piece of the tile's reach along the cache.
struct Place {
    uint32_t h, split, r, tile;
    uint32_t begin, n;               // the request's rows of the call
    int32_t length;                  // as the caller gave it
    uint32_t seen;                   // tokens that the table can hold of them
    bool beyond, last;
};

template <int ROWS, bool TURNS = false>
__device__ __forceinline__ bool find_place(const AttendArgs &a, Place &p) {
    uint32_t x = blockIdx.x;
    p.h = x % a.kv_heads;
    x /= a.kv_heads;
    p.split = x % a.splits;
    x = a.tiles - 1 - x / a.splits;  // the tiles with the most tokens before them first
    uint32_t next;                   // tiles that the request has before the next one's begin
    if (a.tiles_each) {
        p.r = x / a.tiles_each;
        p.tile = x % a.tiles_each;
        next = a.tiles_each;
        if (a.by_tile) {
            p.r = x % a.requests;
            p.tile = a.tiles_each - 1 - x / a.requests;
        }
        if (a.by_length) {
            // the longest request first: p.r counts from the shortest here; each lane ranks one request
            const uint32_t lane = threadIdx.x & 63;
            // (its length and number in one word: they all differ, and lengths past 2^25 may change places)
            // (lanes without a request are above all)
            const uint32_t mine = lane < a.requests ? min((uint32_t)max(a.lengths[lane], 0), (1u << 25) - 1) << 6 | lane : ~0u;
            uint32_t below = 0;
            for (uint32_t j = 0; j < a.requests; j += 8)
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) below += (uint32_t)__builtin_amdgcn_readlane((int)mine, (int)(j + i)) < mine ? 1 : 0;
            // (or, where all of two rounds run at once, the second round's from the shortest on: a CU has one of each)
            if (TURNS && a.by_length > 1) {
                const uint32_t turn = a.by_length - 1, nth = a.requests - 1 - p.r;
                if (nth >= turn) p.r = nth - turn;
            }
            p.r = (uint32_t)__builtin_ctzll(__ballot(lane < a.requests && below == p.r));
        }
    } else {
        // request r begins at tile first(r) = rows before it / ROWS + r, which leaves it at least as many as it needs
        uint32_t lo = 0, hi = a.requests;
        const uint32_t lane = threadIdx.x & 63;
        auto first = [&](uint32_t r) {
            return (uint32_t)((uint64_t)min((uint32_t)max(a.starts[r], 0), a.tokens) * a.group / ROWS) + r;
        };
        while (hi - lo > 1) {        // a wave halves 64 times at once
            const uint32_t step = (hi - lo + 63) / 64, at = lo + lane * step;
            const uint64_t below = __ballot(at < hi && first(at) <= x);
            const uint32_t last = 63 - (uint32_t)__builtin_clzll(below | 1);
            hi = min(hi, lo + (last + 1) * step);
            lo += last * step;
        }
        p.r = lo;
        const uint32_t f = first(lo);
        p.tile = x - f;
        next = first(lo + 1) - f;
        if (x < f) return false;
    }
    const uint32_t b = min((uint32_t)max(a.starts[p.r], 0), a.tokens), e = min((uint32_t)max(a.starts[p.r + 1], 0), a.tokens);
    p.begin = b;
    p.n = e > b ? e - b : 0;
    p.length = max(a.lengths[p.r], 0);
    const uint64_t most = (uint64_t)a.max_blocks << a.block_log2;
    p.beyond = (uint64_t)p.length > most;
    p.seen = p.beyond ? (uint32_t)most : (uint32_t)p.length;
    p.last = p.tile + 1 == next;
    const uint32_t rows = p.n * a.group;
    return p.tile * (uint64_t)ROWS < rows && rows >= a.rows_from && rows <= a.rows_to;
}

// Tokens that any row of a tile sees, the part of them that a split has, and what a row sees.  EVEN: the pieces of a tile are
// alike, down to a quarter of a.chunk (or 256), instead of a.chunk each (32 requests of 2048 to 8192 tokens, 4 rows of 64 heads on 8 each, 47 us
// against 57: short ones have as many workgroups as long ones).
// (begin is a whole tile's; first: the first token that some row sees, up to 127 behind it)
struct Reach { uint32_t begin, end, first; };
template <int ROWS, bool EVEN = false>
__device__ __forceinline__ Reach reach_of(const AttendArgs &a, const Place &p, uint32_t tile) {
    const int64_t rows = (int64_t)p.n * a.group, first = (int64_t)tile * ROWS, last = min(first + ROWS, rows) - 1;
    const int64_t p0 = (int64_t)p.length - p.n + first / a.group, p1 = (int64_t)p.length - p.n + last / a.group;
    int64_t lo = a.window ? max(p0 - (int64_t)a.window + 1, (int64_t)0) : 0;
    int64_t hi = a.causal ? min(p1 + 1, (int64_t)p.seen) : (int64_t)p.seen;
    Reach w;
    w.first = (uint32_t)lo;
    lo &= ~(int64_t)127;             // (a whole tile's, and a block's)
    uint32_t chunk = a.chunk;
    if constexpr (EVEN)
        if (a.splits > 1) chunk = max((((uint32_t)max(hi - lo, (int64_t)0) + a.splits - 1) / a.splits + 127u) & ~127u, max(256u, a.chunk / 4 & ~127u));
    const int64_t begin = lo + (int64_t)p.split * chunk;
    if (p.split + 1 < a.splits) hi = min(hi, begin + chunk);
    w.begin = (uint32_t)min(begin, (int64_t)0x7FFFFFC0);
    w.end = hi > begin ? (uint32_t)hi : w.begin;
    return w;
}
__device__ __forceinline__ void row_sees(const AttendArgs &a, const Place &p, uint32_t row, uint32_t &from, uint32_t &to) {
    // (rows past the request's are computed along and not written: they ask for no mask)
    if (row >= p.n * a.group) { from = 0; to = ~0u; return; }
    const int64_t at = (int64_t)p.length - p.n + row / a.group;
    const int64_t lo = a.window ? max(at - (int64_t)a.window + 1, (int64_t)0) : 0;
    const int64_t hi = a.causal ? min(at + 1, (int64_t)p.seen) : (int64_t)p.seen;
    from = (uint32_t)lo;
    to = hi > lo ? (uint32_t)hi : 0u;
}

// A row of a request that is longer than its row of the table, and that sees anything of it: NaN, whatever it sees.  (Its
// window may lie past all that the table holds, so that the tokens which are looked at cannot tell.)
__device__ __forceinline__ bool is_lost(const AttendArgs &a, const Place &p, uint32_t row) {
    return p.beyond && (!a.causal || (int64_t)p.length - p.n + row / a.group >= 0);
}

// The table's entry for the 16 tokens from `token` on, as it is (past the end of a reach: its last one, so that what is
// asked for ahead of need is always there, and costs no new lines).  It is looked at when it is used, by id_of, so that
// nothing waits for it before.  (`from`: tokens before it are not looked up, but it is in their stead.  A reach begins up to
// 127 tokens before the first one that some row sees, and of blocks there the table may hold nothing, or others' by now.)
__device__ __forceinline__ uint32_t table_entry(const AttendArgs &a, const Place &p, uint32_t token, uint32_t end, uint32_t from = 0) {
    return (uint32_t)a.table[(uint64_t)p.r * a.max_blocks + (min(max(token, from), end - 1) >> a.block_log2)];
}
// A block's number, 0 for what is none; is_bad says which tokens are to come out as NaN for that.
__device__ __forceinline__ uint32_t id_of(const AttendArgs &a, uint32_t entry) { return entry < a.blocks ? entry : 0; }
__device__ __forceinline__ bool is_bad(const AttendArgs &a, const Place &p, uint32_t entry) { return entry >= a.blocks || p.beyond; }

// The kernel's arguments (its only parameter), read once more: what a tile's begin and end alone need then takes no scalar
// registers in its loop.  A few too many cost k_attend_many the order of its loads and products (7 % of its time), and
// k_attend_few with two sets vector registers that it has not (5 to 14 %).  Where there are enough, the first values serve:
// reading them again is 0.2 us of a single token's 5.
__device__ __forceinline__ AttendArgs args_again() {
    struct Words { uint32_t w[sizeof(AttendArgs) / 4]; } words;
    auto args = (const __attribute__((address_space(4))) uint32_t *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(args));
    for (uint32_t i = 0; i < sizeof(AttendArgs) / 4; ++i) words.w[i] = args[i];
    return __builtin_bit_cast(AttendArgs, words);
}

// Where a row's result goes.
__device__ __forceinline__ uint64_t row_id(const AttendArgs &a, const Place &p, uint32_t row) {
    return (uint64_t)(p.begin + row / a.group) * a.q_heads + p.h * a.group + row % a.group;
}

// ... and its row of the parts.
__device__ __forceinline__ uint64_t part_row(const AttendArgs &a, const Place &p, uint32_t row) {
    return a.slots_each ? ((uint64_t)p.r * a.slots_each + row) * a.kv_heads + p.h : row_id(a, p, row);
}

// A piece that lies behind a tile's reach: no row sees anything, and that is all that the join has to know (of a weight
// of NaN, too, whatever the sums are).
template <int ROWS>
__device__ __forceinline__ void nothing_seen(const AttendArgs &a, const Place &p, uint32_t tile, int head_dim) {
    const uint32_t row = tile * ROWS + threadIdx.x;
    if (threadIdx.x >= ROWS || row >= p.n * a.group) return;
    float *st = a.parts + a.part_rows * a.splits * head_dim + (part_row(a, p, row) * a.splits + p.split) * 2;
    st[0] = kNone;
    st[1] = is_lost(a, p, row) ? __builtin_nanf("") : 0.0f;
}

}  // namespace
}  // namespace tsq
