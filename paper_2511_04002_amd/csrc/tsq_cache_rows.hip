// Kernels of tsq_cache.h that work on rows: the schedule of blocks and slots, norm and rotation of queries and
// keys, append and gather.
#include <hip/hip_runtime.h>

#include "tsq_cache_internal.hpp"
#include "tsq.h"

namespace tsq {
namespace {

__device__ __forceinline__ uint32_t of_lane(uint32_t v, uint32_t l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, (int)l); }

constexpr uint32_t kScheduleThreads = 1024;
constexpr uint32_t kFewNew = 4;                          // new tokens that a request's own thread writes

// Sums that stay at 2^32 - 1 once they got there: what does not fit shows in them.
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Exclusive sums over the workgroup of three numbers a thread has; total[] receives the sums of all.
__device__ __forceinline__ void scan_three(uint32_t v[3], uint32_t (*wave_sum)[4], uint32_t total[3]) {
    const uint32_t lane = threadIdx.x & 63, wave = wave_in_group(), waves = blockDim.x / 64;
    uint32_t run[3] = {v[0], v[1], v[2]};
#pragma unroll
    for (uint32_t d = 1; d < 64; d <<= 1) {
        uint32_t o[3];
        for (int j = 0; j < 3; ++j) o[j] = (uint32_t)__shfl_up((int)run[j], d);
        for (int j = 0; j < 3; ++j) run[j] = lane >= d ? add_sat(run[j], o[j]) : run[j];
    }
    if (lane == 63)
        for (int j = 0; j < 3; ++j) wave_sum[wave][j] = run[j];
    __syncthreads();
    // the waves' sums, one a lane
    for (int j = 0; j < 3; ++j) {
        uint32_t s = lane < waves ? wave_sum[lane][j] : 0;
#pragma unroll
        for (uint32_t d = 1; d < 16; d <<= 1) {
            const uint32_t o = (uint32_t)__shfl_up((int)s, d);
            if (lane >= d) s = add_sat(s, o);
        }
        total[j] = of_lane(s, waves - 1);
        v[j] = run[j] - v[j] + (wave ? of_lane(s, wave - 1) : 0);
    }
}

// last r with first[r] <= i, of first[0 .. n] ascending from 0 and i < first[n]
__device__ __forceinline__ uint32_t owner(const uint32_t *first, uint32_t n, uint32_t i) {
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (first[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ uint32_t ring_at(uint32_t base, uint32_t k, uint32_t blocks) {
    const uint32_t i = base + k;                         // base < blocks, k <= blocks, blocks < 2^27
    return i >= blocks ? i - blocks : i;
}
__device__ __forceinline__ uint32_t ring_base(int64_t counter, uint32_t blocks) {
    const uint64_t c = (uint64_t)counter;
    return c >> 32 ? (uint32_t)(c % blocks) : (uint32_t)c % blocks;     // (a division of 64 bits takes ten times as long)
}

// What a step asks for a request: new rows, new blocks, blocks given back.  bad: 1 not an input of this call, 2 no
// room.
struct Wants { uint32_t len, held, rows, more, back; };
__device__ __forceinline__ Wants wants_of(const ScheduleArgs &a, uint32_t r, uint32_t &bad) {
    Wants w = {0, 0, 0, 0, 0};
    const int32_t len = a.lengths[r], n = a.fresh[r];
    const uint64_t most = (uint64_t)a.max_blocks << a.block_log2;
    if (len < 0 || (uint64_t)len > most || n < -1) { bad |= 1; return w; }
    w.len = (uint32_t)len;
    w.held = (w.len + a.block_tokens - 1) >> a.block_log2;
    if (n < 0) w.back = w.held;
    else if ((uint64_t)len + n > most || (uint32_t)n > a.capacity) bad |= 2;
    else {
        w.rows = (uint32_t)n;
        w.more = ((w.len + w.rows + a.block_tokens - 1) >> a.block_log2) - w.held;
    }
    return w;
}

// One launch, no workgroup waits for another: every workgroup sums up all requests by itself (a few KB from the
// caches) and writes its share of the tokens.  A slot is taken from the table where the request has the block
// already and from the ring where it is new, so no workgroup reads what another one writes.  In a step whose
// requests bring at most kFewNew tokens each, a request's thread writes them; otherwise a token's request is
// searched for in the sums.
//
// Latency is all there is: 512 requests, most with a token, some done, are 12.6 KB and 5.5 us; 32 prompts of 96000
// tokens together 0.8 MB and 8.5 us.  A call in a row with others costs 3.4 us whatever it does.
__global__ __launch_bounds__(kScheduleThreads) void k_schedule(ScheduleArgs a) {
    __shared__ uint32_t first_row[kMaxScheduleRequests + 1], first_new[kMaxScheduleRequests + 1], first_back[kMaxScheduleRequests + 1];
    __shared__ uint32_t wave_sum[kScheduleThreads / 64][4];
    __shared__ uint32_t flags;
    const uint32_t tid = threadIdx.x, threads = blockDim.x, B = a.block_tokens, lg = a.block_log2;
    const uint32_t each = (a.requests + threads - 1) / threads;
    if (tid == 0) flags = 0;
    __syncthreads();

    const int64_t taken = a.counters[0], returned = a.counters[1];
    uint32_t bad = 0;                                    // (4: some request brings more than kFewNew)
    if (taken < 0 || returned < taken || returned - taken > (int64_t)a.blocks) bad = 1;
    uint32_t at[3] = {0, 0, 0}, total[3];
    for (uint32_t j = 0; j < each; ++j) {
        const uint32_t r = tid * each + j;
        if (r >= a.requests) break;
        const Wants w = wants_of(a, r, bad);
        at[0] = add_sat(at[0], w.rows); at[1] = add_sat(at[1], w.more); at[2] = add_sat(at[2], w.back);
        if (w.rows > kFewNew) bad |= 4;
    }
    if (bad) atomicOr(&flags, bad);
    scan_three(at, wave_sum, total);                     // (its barrier also closes the writes of flags)
    uint32_t why = flags;
    if (total[0] > a.capacity || (int64_t)total[1] > returned - taken) why |= 2;
    // (a ring that would hold more blocks than there are: a block was given back twice)
    if (!(why & 1) && returned - taken + (int64_t)total[2] > (int64_t)a.blocks) why |= 1;

    const uint32_t first = blockIdx.x * threads + tid, step = gridDim.x * threads;
    if (why & 3) {
        if (blockIdx.x == 0) {
            for (uint32_t r = tid; r < a.requests; r += threads) a.lengths_out[r] = a.lengths[r];
            for (uint32_t r = tid; r <= a.requests; r += threads) a.starts[r] = 0;
            if (tid == 0) {
                a.counters_out[0] = taken;
                a.counters_out[1] = returned;
                a.status[0] = why & 1 ? TSQ_ERR_INVALID_ARG : TSQ_ERR_CAPACITY;
            }
        }
        for (uint32_t i = first; i < a.capacity; i += step) a.positions[i] = a.slots[i] = -1;
        return;
    }
    // from here on every sum is one: tokens <= capacity, blocks <= a.blocks
    const uint32_t head = ring_base(taken, a.blocks), tail = ring_base(returned, a.blocks);
    const bool few = !(why & 4);
    auto put = [&](uint32_t i, const Wants &w, uint32_t r, uint32_t t, uint32_t new_at) {
        const uint32_t nth = t >> lg;
        const int32_t block = nth < w.held ? a.table[(uint64_t)r * a.max_blocks + nth] : a.ring[ring_at(head, new_at + (nth - w.held), a.blocks)];
        a.positions[i] = (int32_t)t;
        // (an entry that is no block of the cache gives no slot)
        a.slots[i] = (uint32_t)block < a.blocks ? (int32_t)(((uint32_t)block << lg) + (t & (B - 1))) : -1;
    };
    uint32_t none = 0;
    for (uint32_t j = 0; j < each; ++j) {
        const uint32_t r = tid * each + j;
        if (r >= a.requests) break;
        const Wants w = wants_of(a, r, none);
        first_row[r] = at[0]; first_new[r] = at[1]; first_back[r] = at[2];
        if (blockIdx.x == 0) {
            a.starts[r] = (int32_t)at[0];
            a.lengths_out[r] = w.back || a.fresh[r] < 0 ? 0 : (int32_t)(w.len + w.rows);
            if (few)
                for (uint32_t i = 0; i < w.rows; ++i) put(at[0] + i, w, r, w.len + i, at[1]);
        }
        at[0] += w.rows; at[1] += w.more; at[2] += w.back;
    }
    if (tid == 0) {
        first_row[a.requests] = total[0]; first_new[a.requests] = total[1]; first_back[a.requests] = total[2];
        if (blockIdx.x == 0) {
            a.starts[a.requests] = (int32_t)total[0];
            a.counters_out[0] = taken + (int64_t)total[1];
            a.counters_out[1] = returned + (int64_t)total[2];
            a.status[0] = TSQ_OK;
        }
    }
    for (uint32_t i = total[0] + first; i < a.capacity; i += step) a.positions[i] = a.slots[i] = -1;
    if (few && total[1] + total[2] == 0) return;
    __syncthreads();
    if (!few)
        for (uint32_t i = first; i < total[0]; i += step) {
            const uint32_t r = owner(first_row, a.requests, i);
            Wants w;
            w.len = (uint32_t)a.lengths[r];
            w.held = (w.len + B - 1) >> lg;
            put(i, w, r, w.len + (i - first_row[r]), first_new[r]);
        }
    for (uint32_t k = first; k < total[1]; k += step) {
        const uint32_t r = owner(first_new, a.requests, k);
        const uint32_t held = ((uint32_t)a.lengths[r] + B - 1) >> lg;
        a.table[(uint64_t)r * a.max_blocks + held + (k - first_new[r])] = a.ring[ring_at(head, k, a.blocks)];
    }
    for (uint32_t k = first; k < total[2]; k += step) {
        const uint32_t r = owner(first_back, a.requests, k);
        a.ring[ring_at(tail, k, a.blocks)] = a.table[(uint64_t)r * a.max_blocks + (k - first_back[r])];
    }
}

// Norm and rotation.  A lane holds 16 elements of a head in two pieces of 8, chosen so that the pairs that turn
// together are the lane's own: D / 16 lanes a head, 1024 / D heads a wave.  The sum of squares, the product with the
// weight and the rotation stay in registers, in binary32; memory is read and written once, and bounds it: 8192 rows of
// 72 heads of 128 are 306 MB and 54 us, 5.7 TB/s where a copy reaches 6.2; by three axes (AXES, which choose each pair's row of
// angles) 59, and 63 with pairs dealt out in turn, whose lanes read the rows of all axes and choose.
template <int D, bool BF16, bool AXES, bool ONCE>
__global__ __launch_bounds__(256) void k_norm_rotate(NormRotateArgs a, uint32_t passes, uint32_t waves_each) {
    constexpr int LPH = D / 16, HEADS = 64 / LPH;
    const uint32_t lane = threadIdx.x & 63, wave = blockIdx.x * 4 + wave_in_group();
    const uint32_t token = wave / waves_each;
    if (token >= a.tokens) return;
    const int32_t position = a.positions[token];
    int32_t others[kMaxAxes - 1];                        // ... and on the axes after the first
    bool known = (uint32_t)position < a.angle_rows;
    if constexpr (AXES) {
        int32_t least = position;
        for (uint32_t x = 1; x < kMaxAxes; ++x) {
            others[x - 1] = x < a.axes ? a.positions[(uint64_t)x * a.tokens + token] : 0;
            least = min(least, others[x - 1]);
            known &= x >= a.axes || (uint32_t)others[x - 1] < a.angle_rows;
        }
        if (least < 0) return;
    } else if (position < 0) return;
    const uint32_t j = lane % LPH, sub = lane / LPH, turning = a.rotary / 16;
    uint32_t e0, e1;                                    // first elements of the lane's two pieces
    const bool turns = j < turning;
    if (a.neighbours || !turns) { e0 = 16 * j; e1 = 16 * j + 8; }
    else { e0 = 8 * j; e1 = 8 * j + a.rotary / 2; }
    float c[8], s[8];
    if (turns && known) {
        const float *row = a.angles + (uint64_t)position * a.rotary + 8 * j;
        bool together = true;
        if constexpr (AXES) {
            // the pairs' angles are those of their axes' rows; where a lane's eight have several axes, all rows are read and chosen from
            const uint2_t axis = *reinterpret_cast<const uint2_t *>(a.axis + 8 * j);
            auto place_on = [&](uint32_t x) { return x == 0 ? position : x == 1 ? others[0] : x == 2 ? others[1] : others[2]; };
            const uint32_t first = axis[0] & 0xFFu;
            together = axis[0] == axis[1] && axis[0] == first * 0x01010101u && first < a.axes;
            row = a.angles + (uint64_t)(uint32_t)place_on(first) * a.rotary + 8 * j;
            if (!together) {
                for (int i = 0; i < 8; ++i) c[i] = s[i] = __builtin_nanf("");
                for (uint32_t x = 0; x < kMaxAxes; ++x) {
                    if (x >= a.axes) break;
                    const float *at = a.angles + (uint64_t)(uint32_t)place_on(x) * a.rotary + 8 * j;
                    float4_t cs[2], sn[2];
                    for (int i = 0; i < 2; ++i) {
                        cs[i] = *reinterpret_cast<const float4_t *>(at + 4 * i);
                        sn[i] = *reinterpret_cast<const float4_t *>(at + a.rotary / 2 + 4 * i);
                    }
                    for (int i = 0; i < 8; ++i) {
                        const bool here = (axis[i / 4] >> 8 * (i % 4) & 0xFFu) == x;
                        c[i] = here ? cs[i / 4][i % 4] : c[i];
                        s[i] = here ? sn[i / 4][i % 4] : s[i];
                    }
                }
            }
        }
        if (together)
            for (int i = 0; i < 8; i += 4) {
                *reinterpret_cast<float4_t *>(c + i) = *reinterpret_cast<const float4_t *>(row + i);
                *reinterpret_cast<float4_t *>(s + i) = *reinterpret_cast<const float4_t *>(row + a.rotary / 2 + i);
            }
    } else {
        const float one = known ? 1.0f : __builtin_nanf("");
        for (int i = 0; i < 8; ++i) { c[i] = one; s[i] = one - one; }
    }
    const uint32_t heads = a.q_heads + a.kv_heads;
    for (uint32_t pass = wave % waves_each; pass < passes; pass += waves_each) {
        const uint32_t h = pass * HEADS + sub;
        const bool is_q = h < a.q_heads, here = h < heads;
        const uint64_t in_at = is_q ? (uint64_t)token * a.q_stride + (uint64_t)h * D : (uint64_t)token * a.k_stride + (uint64_t)(h - a.q_heads) * D;
        const uint64_t out_at = is_q ? (uint64_t)token * a.q_out_stride + (uint64_t)h * D : (uint64_t)token * a.k_out_stride + (uint64_t)(h - a.q_heads) * D;
        const uint16_t *in = static_cast<const uint16_t *>(is_q ? a.q : a.k) + in_at;
        float x[16];
        if (here) {
            const uint4_t *in0 = reinterpret_cast<const uint4_t *>(in + e0), *in1 = reinterpret_cast<const uint4_t *>(in + e1);
            const uint4_t p0 = ONCE ? __builtin_nontemporal_load(in0) : *in0, p1 = ONCE ? __builtin_nontemporal_load(in1) : *in1;
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = widen<BF16>(p0[i] & 0xFFFFu); x[2 * i + 1] = widen<BF16>(p0[i] >> 16);
                x[8 + 2 * i] = widen<BF16>(p1[i] & 0xFFFFu); x[9 + 2 * i] = widen<BF16>(p1[i] >> 16);
            }
        } else {
            for (int i = 0; i < 16; ++i) x[i] = 0.0f;
        }
        const uint16_t *weight = static_cast<const uint16_t *>(is_q ? a.q_weight : a.k_weight);
        float sum = 0.0f;
        for (int i = 0; i < 16; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
        for (int d = 1; d < LPH; d <<= 1) sum += __shfl_xor(sum, d);
        if (!here) continue;
        if (weight) {
            const float f = 1.0f / __builtin_sqrtf(sum * (1.0f / D) + a.eps);
            const uint4_t w0 = *reinterpret_cast<const uint4_t *>(weight + e0), w1 = *reinterpret_cast<const uint4_t *>(weight + e1);
            for (int i = 0; i < 4; ++i) {
                x[2 * i] *= f * widen<BF16>(w0[i] & 0xFFFFu); x[2 * i + 1] *= f * widen<BF16>(w0[i] >> 16);
                x[8 + 2 * i] *= f * widen<BF16>(w1[i] & 0xFFFFu); x[9 + 2 * i] *= f * widen<BF16>(w1[i] >> 16);
            }
        }
        float y[16];
        if (!turns) {                                   // (c is 1, or NaN past the angles' rows)
            for (int i = 0; i < 16; ++i) y[i] = x[i] * c[0];
        } else if (a.neighbours) {
            for (int i = 0; i < 8; ++i) {
                y[2 * i] = x[2 * i] * c[i] - x[2 * i + 1] * s[i];
                y[2 * i + 1] = x[2 * i + 1] * c[i] + x[2 * i] * s[i];
            }
        } else {
            for (int i = 0; i < 8; ++i) {
                y[i] = x[i] * c[i] - x[8 + i] * s[i];
                y[8 + i] = x[8 + i] * c[i] + x[i] * s[i];
            }
        }
        uint16_t *out = static_cast<uint16_t *>(is_q ? a.q_out : a.k_out) + out_at;
        uint4_t o0, o1;
        for (int i = 0; i < 4; ++i) {
            o0[i] = narrow2<BF16>(y[2 * i], y[2 * i + 1]);
            o1[i] = narrow2<BF16>(y[8 + 2 * i], y[9 + 2 * i]);
        }
        __builtin_nontemporal_store(o0, reinterpret_cast<uint4_t *>(out + e0));
        __builtin_nontemporal_store(o1, reinterpret_cast<uint4_t *>(out + e1));
    }
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    for (int d = 32; d > 0; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    return v;
}

// round(x * f), to even, in the low byte: the sum's last bit is worth 1, and below it stands the code in two's
// complement.  |x * f| is at most 127 and a few units of its last place here.  (Of a NaN, which only a scale of NaN
// goes with, it is some code.)
__device__ __forceinline__ uint32_t code_bits(float x, float f) { return __builtin_bit_cast(uint32_t, x * f + 12582912.0f); }
__device__ __forceinline__ uint32_t four_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u), 0x05040100u);
}
__device__ __forceinline__ uint32_t recode(uint32_t w, float factor) {
    return four_bytes(code_bits(code_at(w, 0), factor), code_bits(code_at(w, 1), factor), code_bits(code_at(w, 2), factor),
                      code_bits(code_at(w, 3), factor));
}

// Keeps the compiler from widening elements long before they are used, in twice the registers.
template <typename T> __device__ __forceinline__ void stay(T &v) { asm("" : "+v"(v)); }

// What a run does to a block's scale.  `most`: the bits of the largest magnitude among its elements (of NaN and
// infinity, which are larger than all others).
struct Scales { float now, inverse, factor; bool again; };
template <bool BF16> __device__ __forceinline__ Scales scales_of(uint32_t most, float before) {
    Scales s;
    float m = widen<BF16>(most) / 127.0f;
    if (m < 0x1p-126f) m = 0.0f;
    if (most >= (BF16 ? 0x7F80u : 0x7C00u) || before != before) s.now = __builtin_nanf("");
    else s.now = fmaxf(before, m);
    s.inverse = s.now > 0.0f ? 1.0f / s.now : 0.0f;
    s.again = before > 0.0f && s.now > before;
    s.factor = s.again ? before / s.now : 1.0f;
    return s;
}

// One run of tokens of one block, for one head, keys or values: rows x[0 .. n) go to places o .. o + n - 1.  A wave
// does it by itself: the largest magnitude first, then the block's scale, then the codes that are there if their
// scale changes, then the new ones.  It goes by 16 places of the block at a time; the elements of the first two
// such pieces stay in registers between the two steps, those of longer runs are read again.
//
// Keys lie token by token: a lane has 8 elements of a token, D / 8 lanes a token.
template <int D, bool BF16>
__device__ __forceinline__ void store_keys(const uint16_t *x, uint64_t stride, int8_t *codes, float *scale, uint32_t o, uint32_t n) {
    constexpr uint32_t LPT = D / 8, TPI = 64 / LPT, LOADS = 16 / TPI, KEPT = 2;
    const uint32_t lane = threadIdx.x & 63, piece = lane % LPT, sub = lane / LPT, end = o + n;
    const uint32_t first = o / 16, last = (end + 15) / 16;
    uint4_t w[KEPT][LOADS];
    auto ask = [&](uint4_t *to, uint32_t c) {
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) {
            const uint32_t place = 16 * c + TPI * i + sub;
            to[i] = uint4_t{0, 0, 0, 0};
            if (place >= o && place < end) to[i] = *reinterpret_cast<const uint4_t *>(x + (place - o) * stride + 8 * piece);
        }
    };
    uint32_t most = 0;
    auto look = [&](const uint4_t *from) {
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i)
            for (int j = 0; j < 4; ++j) most = max(most, max(from[i][j] & 0x7FFFu, (from[i][j] >> 16) & 0x7FFFu));
    };
#pragma unroll
    for (uint32_t b = 0; b < KEPT; ++b)
        if (first + b < last) ask(w[b], first + b);
    const float before = o ? *scale : 0.0f;
#pragma unroll
    for (uint32_t b = 0; b < KEPT; ++b)
        if (first + b < last) look(w[b]);
    for (uint32_t c = first + KEPT; c < last; ++c) {
        uint4_t v[LOADS];
        ask(v, c);
        look(v);
    }
    const Scales s = scales_of<BF16>(wave_max(most), before);
#pragma unroll
    for (uint32_t b = 0; b < KEPT; ++b)
        for (uint32_t i = 0; i < LOADS; ++i) stay(w[b][i]);
    if (lane == 0) *scale = s.now;
    if (s.again)
        for (uint32_t at = lane * 16; at < o * D; at += 1024) {
            uint4_t v = *reinterpret_cast<const uint4_t *>(codes + at);
            for (int i = 0; i < 4; ++i) v[i] = recode(v[i], s.factor);
            *reinterpret_cast<uint4_t *>(codes + at) = v;
        }
    auto put = [&](const uint4_t *from, uint32_t c) {
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) {
            const uint32_t place = 16 * c + TPI * i + sub;
            if (place < o || place >= end) continue;
            uint2_t q;
            for (int j = 0; j < 2; ++j) {
                const uint32_t a = from[i][2 * j], b = from[i][2 * j + 1];
                q[j] = four_bytes(code_bits(widen<BF16>(a & 0xFFFFu), s.inverse), code_bits(widen<BF16>(a >> 16), s.inverse),
                                  code_bits(widen<BF16>(b & 0xFFFFu), s.inverse), code_bits(widen<BF16>(b >> 16), s.inverse));
            }
            *reinterpret_cast<uint2_t *>(codes + (uint64_t)place * D + 8 * piece) = q;
        }
    };
#pragma unroll
    for (uint32_t b = 0; b < KEPT; ++b)
        if (first + b < last) put(w[b], first + b);
    for (uint32_t c = first + KEPT; c < last; ++c) {
        uint4_t v[LOADS];
        ask(v, c);
        put(v, c);
    }
}

// Values lie element by element, 16 places of one element side by side: a lane has D / 64 elements, of which it
// reads all 16 tokens and writes whole 16-byte pieces.
template <int D, bool BF16>
__device__ __forceinline__ void store_values(const uint16_t *x, uint64_t stride, int8_t *codes, float *scale, uint32_t B, uint32_t o, uint32_t n) {
    constexpr int E = D / 64;
    constexpr uint32_t KEPT = 2;
    const uint32_t lane = threadIdx.x & 63, end = o + n, first = o / 16, last = (end + 15) / 16;
    struct Row { uint32_t v[(E + 1) / 2]; };             // a token's elements of this lane
    Row w[KEPT][16];
    auto ask = [&](Row *to, uint32_t c) {
#pragma unroll
        for (uint32_t p = 0; p < 16; ++p) {
            const uint32_t place = 16 * c + p;
            to[p] = Row{};
            if (place < o || place >= end) continue;     // (the same for all lanes)
            const uint16_t *row = x + (uint64_t)(place - o) * stride + E * lane;
            if constexpr (E == 1) to[p].v[0] = row[0];
            else if constexpr (E == 2) to[p].v[0] = *reinterpret_cast<const uint32_t *>(row);
            else {
                const uint2_t q = *reinterpret_cast<const uint2_t *>(row);
                to[p].v[0] = q[0];
                to[p].v[1] = q[1];
            }
        }
    };
    uint32_t most = 0;
    auto look = [&](const Row *from) {
#pragma unroll
        for (int p = 0; p < 16; ++p)
            for (int e = 0; e < (E + 1) / 2; ++e) most = max(most, max(from[p].v[e] & 0x7FFFu, (from[p].v[e] >> 16) & 0x7FFFu));
    };
#pragma unroll
    for (uint32_t b = 0; b < KEPT; ++b)
        if (first + b < last) ask(w[b], first + b);
    const float before = o ? *scale : 0.0f;
#pragma unroll
    for (uint32_t b = 0; b < KEPT; ++b)
        if (first + b < last) look(w[b]);
    for (uint32_t c = first + KEPT; c < last; ++c) {
        Row v[16];
        ask(v, c);
        look(v);
    }
    const Scales s = scales_of<BF16>(wave_max(most), before);
#pragma unroll
    for (uint32_t b = 0; b < KEPT; ++b)
        for (int p = 0; p < 16; ++p)
            for (int e = 0; e < (E + 1) / 2; ++e) stay(w[b][p].v[e]);
    if (lane == 0) *scale = s.now;
    if (s.again)
        for (uint32_t c = 0; c < first; ++c)
            for (int e = 0; e < E; ++e) {
                uint4_t *at = reinterpret_cast<uint4_t *>(codes + (uint64_t)(E * lane + e) * B + 16 * c);
                uint4_t v = *at;
                for (int i = 0; i < 4; ++i) v[i] = recode(v[i], s.factor);
                *at = v;
            }
    if (n == 1 && !s.again) {
        // one token into a block whose scale stays: its bytes alone
        Row one = {};
        const uint16_t *row = x + E * lane;
        if constexpr (E == 1) one.v[0] = row[0];
        else if constexpr (E == 2) one.v[0] = *reinterpret_cast<const uint32_t *>(row);
        else { const uint2_t q = *reinterpret_cast<const uint2_t *>(row); one.v[0] = q[0]; one.v[1] = q[1]; }
#pragma unroll
        for (int e = 0; e < E; ++e)
            codes[(uint64_t)(E * lane + e) * B + o] = (int8_t)code_bits(widen<BF16>((one.v[e / 2] >> (16 * (e & 1))) & 0xFFFFu), s.inverse);
        return;
    }
    auto put = [&](const Row *from, uint32_t c) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            uint4_t *at = reinterpret_cast<uint4_t *>(codes + (uint64_t)(E * lane + e) * B + 16 * c);
            uint4_t old = {0, 0, 0, 0}, q;
            if (16 * c < o) {                            // places before the run
                old = *at;
                if (s.again)
                    for (int i = 0; i < 4; ++i) old[i] = recode(old[i], s.factor);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t b[4];
                for (int j = 0; j < 4; ++j) b[j] = code_bits(widen<BF16>((from[4 * i + j].v[e / 2] >> (16 * (e & 1))) & 0xFFFFu), s.inverse);
                q[i] = four_bytes(b[0], b[1], b[2], b[3]);
                const uint32_t place = 16 * c + 4 * i;   // bytes below the run's first place stay as they were
                if (place < o) {
                    const uint32_t keep = o - place >= 4 ? ~0u : (1u << (8 * (o - place))) - 1u;
                    q[i] = (q[i] & ~keep) | (old[i] & keep);
                }
            }
            *at = q;
        }
    };
#pragma unroll
    for (uint32_t b = 0; b < KEPT; ++b)
        if (first + b < last) put(w[b], first + b);
    for (uint32_t c = first + KEPT; c < last; ++c) {
        Row v[16];
        ask(v, c);
        put(v, c);
    }
}

// The largest of N lanes that follow one another (8, 16 or 32), in all of them.
template <int N> __device__ __forceinline__ uint32_t group_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));          // lane ^ 1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));          // lane ^ 2
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));         // the other four of eight
    if constexpr (N >= 16) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));  // ... eight of sixteen
    if constexpr (N == 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16));
    return v;
}

// A single token, as every request brings one in a step of decoding: D / 8 lanes a head, 512 / D heads at once, since
// one token's head is too little for a wave and a step's time is its waits, one after the other.  512 tokens on 40
// heads of 128: 22 us, with one head a wave 30.
template <int D, bool BF16, int WHICH>
__device__ __forceinline__ void store_single(const uint16_t *x, int8_t *codes, float *scale, uint32_t B, uint32_t o, uint32_t h0, uint32_t heads) {
    constexpr uint32_t LPT = D / 8;
    const uint32_t lane = threadIdx.x & 63, piece = lane % LPT, h = h0 + lane / LPT;
    const bool real = h < heads;
    uint4_t w = {0, 0, 0, 0};
    float before = 0.0f;
    if (real) {
        w = *reinterpret_cast<const uint4_t *>(x + (uint64_t)h * D + 8 * piece);
        if (o) before = scale[h];
    }
    uint32_t most = 0;
    for (int j = 0; j < 4; ++j) most = max(most, max(w[j] & 0x7FFFu, (w[j] >> 16) & 0x7FFFu));
    const Scales s = scales_of<BF16>(group_max<LPT>(most), before);
    if (!real) return;
    if (piece == 0) scale[h] = s.now;
    uint32_t q[8];
    for (int j = 0; j < 4; ++j) {
        q[2 * j] = code_bits(widen<BF16>(w[j] & 0xFFFFu), s.inverse);
        q[2 * j + 1] = code_bits(widen<BF16>(w[j] >> 16), s.inverse);
    }
    int8_t *mine = codes + (uint64_t)h * B * D;
    if constexpr (WHICH == 0) {
        if (s.again)
            for (uint32_t at = piece * 16; at < o * D; at += LPT * 16) {
                uint4_t v = *reinterpret_cast<const uint4_t *>(mine + at);
                for (int i = 0; i < 4; ++i) v[i] = recode(v[i], s.factor);
                *reinterpret_cast<uint4_t *>(mine + at) = v;
            }
        *reinterpret_cast<uint2_t *>(mine + (uint64_t)o * D + 8 * piece) = uint2_t{four_bytes(q[0], q[1], q[2], q[3]), four_bytes(q[4], q[5], q[6], q[7])};
    } else {
        mine += (uint64_t)(8 * piece) * B;               // the lane's elements
        if (!s.again) {
#pragma unroll
            for (int e = 0; e < 8; ++e) mine[e * B + o] = (int8_t)q[e];
            return;
        }
        for (uint32_t c = 0; c <= o; c += 16) {
            uint4_t v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const uint4_t *>(mine + e * B + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                for (uint32_t i = 0; i < 4; ++i) {
                    v[e][i] = recode(v[e][i], s.factor);
                    if (o - c < 16 && (o - c) / 4 == i) v[e][i] = (v[e][i] & ~(0xFFu << (8 * (o & 3)))) | (q[e] & 0xFFu) << (8 * (o & 3));
                }
                *reinterpret_cast<uint4_t *>(mine + e * B + c) = v[e];
            }
        }
    }
}

// A window of rows for waves_each waves: each finds the runs that begin in it, one row a lane, and takes its share of
// (run, head, keys or values).
//
// Of prompts, memory is the bound: 5600 rows of 32 heads of 128 are 138 MB and 29 us.  Of single tokens it is what the
// layout makes of them: the keys of a (token, head) are 128 bytes side by side, the values 128 bytes a block's tokens
// apart, so that as many lines of 128 bytes as a block has tokens are written in part.  512 tokens on 40 heads, 16 MB as
// they come, into blocks of 16, 32, 64 and 128 whose places are spread evenly: 25, 39, 67 and 102 us, with 16, 10, 6 and
// 3 % of the (token, head) pairs growing past their block's scale, whose codes are read and written again (blocks of
// 16 without: 22 us).
template <int D, bool BF16>
__global__ __launch_bounds__(256, D == 256 ? 3 : 4) void k_append(AppendArgs a) {
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t wave = (uint64_t)blockIdx.x * 4 + wave_in_group();
    const uint64_t begin = wave / a.waves_each * a.window;
    if (begin >= a.tokens) return;
    const uint32_t row = (uint32_t)begin + lane, B = a.block_tokens;
    int32_t slot = -1;
    if (lane < a.window && row < a.tokens) slot = a.slots[row];
    int32_t previous = __shfl_up(slot, 1);
    if (lane == 0) previous = row ? a.slots[row - 1] : -1;
    const bool real = slot >= 0 && ((uint32_t)slot >> a.block_log2) < a.blocks;
    const bool follows = real && ((uint32_t)slot & (B - 1)) && previous == slot - 1;
    const uint64_t leads = __ballot(real && !follows), goes = __ballot(follows);
    const uint32_t runs = (uint32_t)__builtin_popcountll(leads);
    // single tokens alone: none follows another, here or behind the window
    bool follows_on = false;
    if (lane == a.window - 1 && real && row + 1 < a.tokens) follows_on = a.slots[row + 1] == slot + 1 && ((uint32_t)slot + 1 & (B - 1));
    if (goes == 0 && __ballot(follows_on) == 0) {
        constexpr uint32_t AT_ONCE = 512 / D;
        const uint32_t groups = (a.kv_heads + AT_ONCE - 1) / AT_ONCE, each = groups * 2;
        uint64_t left = leads;
        uint32_t nth = 0;
        for (uint32_t u = (uint32_t)(wave % a.waves_each); u < runs * each; u += a.waves_each) {
            for (; nth < u / each; ++nth) left &= left - 1;
            const uint32_t l = (uint32_t)__builtin_ctzll(left), at = of_lane((uint32_t)slot, l), which = u % each & 1, h0 = u % each / 2 * AT_ONCE;
            const uint64_t block = at >> a.block_log2;
            if (which == 0)
                store_single<D, BF16, 0>(static_cast<const uint16_t *>(a.x[0]) + (begin + l) * a.stride[0], a.codes[0] + block * a.kv_heads * B * D,
                                         a.scale[0] + block * a.kv_heads, B, at & (B - 1), h0, a.kv_heads);
            else
                store_single<D, BF16, 1>(static_cast<const uint16_t *>(a.x[1]) + (begin + l) * a.stride[1], a.codes[1] + block * a.kv_heads * B * D,
                                         a.scale[1] + block * a.kv_heads, B, at & (B - 1), h0, a.kv_heads);
        }
        return;
    }
    const uint32_t each = a.kv_heads * 2;
    uint32_t nth = ~0u, o = 0, n = 0;
    uint64_t row0 = 0, block = 0;
    uint64_t left = leads;
    uint32_t passed = 0;                                 // leaders taken from `left`
    for (uint32_t u = (uint32_t)(wave % a.waves_each); u < runs * each; u += a.waves_each) {
        if (u / each != nth) {
            nth = u / each;
            uint32_t l = 0;
            for (; passed <= nth; ++passed) {
                l = (uint32_t)__builtin_ctzll(left);
                left &= left - 1;
            }
            const int32_t s = (int32_t)of_lane((uint32_t)slot, l);
            o = (uint32_t)s & (B - 1);
            block = (uint32_t)s >> a.block_log2;
            row0 = begin + l;
            // rows that follow in the window, then those behind it
            const uint64_t after = l == 63 ? 0 : ~(goes >> (l + 1));
            n = 1 + (l == 63 ? 0 : after ? (uint32_t)__builtin_ctzll(after) : 64u);
            if (l + n >= a.window) {
                n = a.window - l;
                const uint32_t most = min(B - o, (uint32_t)(a.tokens - row0));
                while (n < most) {
                    const uint32_t at = n + lane;
                    const uint64_t more = __ballot(at < most && a.slots[row0 + at] == s + (int32_t)at);
                    const uint32_t got = more == ~0ull ? 64 : (uint32_t)__builtin_ctzll(~more);
                    n += got;
                    if (got < 64) break;
                }
            }
        }
        const uint32_t h = u % each >> 1, which = u & 1;
        const uint64_t head = block * a.kv_heads + h;
        const uint16_t *x = static_cast<const uint16_t *>(which ? a.x[1] : a.x[0]) + row0 * (which ? a.stride[1] : a.stride[0]) + (uint64_t)h * D;
        if (which == 0) store_keys<D, BF16>(x, a.stride[0], a.codes[0] + head * B * D, a.scale[0] + head, o, n);
        else store_values<D, BF16>(x, a.stride[1], a.codes[1] + head * B * D, a.scale[1] + head, B, o, n);
    }
}

// Sixteen rows of the output for waves_each waves: row i's request, position and block by lane i, then a share of the
// heads each wave.
//
// Memory is the bound: 92000 rows of 8 heads of 128 from blocks of 64 tokens are 565 MB and 104 us, 126 where two such
// calls take turns (a part of one's data stays in the memory's cache otherwise): 5.4 and 4.5 TB/s where a copy reaches
// 6.1.  The keys alone take 45 us, the values alone 63, and 42 of those if they are only read: a wave reads 16 bytes out
// of each of 128 rows of 64 bytes, and the other waves of its workgroup the rest of the lines.  A request of 2048 rows of
// 32 heads, from blocks of 16, is 50 MB and 9 to 10 us.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void k_gather(GatherArgs a) {
    const int8_t *codes[2] = {static_cast<const int8_t *>(a.codes[0]), static_cast<const int8_t *>(a.codes[1])};
    const float *scales[2] = {static_cast<const float *>(a.scale[0]), static_cast<const float *>(a.scale[1])};
    const uint32_t lane = threadIdx.x & 63, B = a.block_tokens;
    // the four waves of a workgroup have the same heads of rows that follow one another: of blocks of more than 16
    // tokens they read neighbouring pieces of the same lines
    const uint64_t begin = ((uint64_t)(blockIdx.x / a.waves_each) * 4 + wave_in_group()) * 16;
    if (begin >= a.tokens) return;
    const GatherRow row = gather_row(a, begin);
    const uint32_t r = row.r, nth = row.nth, place = row.place;
    const int32_t block = row.block;
    const bool owned = row.owned;
    // keys: each row by itself, wherever it lies
    constexpr uint32_t LPT = D / 8, TPI = 64 / LPT, LOADS = 16 / TPI;
    constexpr int E = D / 64;
    const uint32_t piece = lane % LPT, sub = lane / LPT;
    uint32_t key_block[LOADS], key_place[LOADS];
#pragma unroll
    for (uint32_t t = 0; t < LOADS; ++t) {
        key_block[t] = (uint32_t)__shfl(owned ? block : -2, (int)(TPI * t + sub));
        key_place[t] = (uint32_t)__shfl((int)place, (int)(TPI * t + sub));
    }
    const uint32_t before_r = (uint32_t)__shfl_up((int)r, 1), before_n = (uint32_t)__shfl_up((int)nth, 1);
    const int before_owned = __shfl_up((int)owned, 1);
    const bool leads = owned && lane < 16 && (lane == 0 || !before_owned || before_r != r || before_n != nth);
    const uint32_t ours = (uint32_t)__ballot(owned && lane < 16), runs = (uint32_t)__ballot(leads);
    for (uint32_t h = blockIdx.x % a.waves_each; h < a.kv_heads; h += a.waves_each) {
        uint2_t kw[LOADS];
        float k_scale[LOADS];
#pragma unroll
        for (uint32_t t = 0; t < LOADS; ++t) {
            const uint64_t head = (uint64_t)((int32_t)key_block[t] < 0 ? 0 : key_block[t]) * a.kv_heads + h;
            kw[t] = *reinterpret_cast<const uint2_t *>(codes[0] + (head * B + key_place[t]) * D + 8 * piece);
            k_scale[t] = scales[0][head];
        }
        uint32_t left = runs;
        bool keys_done = false;
        do {
            // values: the rows of a run, which lie in one block at places that follow one another, 16 places of an
            // element side by side; what the first of them needs is asked for before the keys are written
            const uint32_t l = left ? (uint32_t)__builtin_ctz(left) : 0;
            const bool some = left != 0;
            left &= left - 1;
            const uint32_t reach = left ? (uint32_t)__builtin_ctz(left) : 16u;
            const uint32_t n = some ? min(reach - l, (uint32_t)__builtin_ctz(~(ours >> l))) : 0;
            const int32_t b = some ? (int32_t)of_lane((uint32_t)block, l) : -1;
            const uint32_t o = of_lane(place, l), first = o / 16 * 16;
            const uint64_t head = (uint64_t)max(b, 0) * a.kv_heads + h;
            const float v_scale = b < 0 ? __builtin_nanf("") : scales[1][head];
            const int8_t *values = codes[1] + (head * D + E * lane) * B + first;
            uint16_t *v_out = static_cast<uint16_t *>(a.out[1]) + (begin + l) * a.stride[1] + (uint64_t)h * D;
            uint4_t vw[E], vx[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                vw[e] = *reinterpret_cast<const uint4_t *>(values + e * B);
                if (first + 16 < o + n) vx[e] = *reinterpret_cast<const uint4_t *>(values + e * B + 16);
            }
            if (!keys_done) {
                keys_done = true;
#pragma unroll
                for (uint32_t t = 0; t < LOADS; ++t) {
                    if ((int32_t)key_block[t] == -2) continue;
                    const float scale = (int32_t)key_block[t] < 0 ? __builtin_nanf("") : k_scale[t];
                    uint4_t y;
                    for (int e = 0; e < 4; ++e)
                        y[e] = narrow2<BF16>(code_at(kw[t][e / 2], 2 * (e & 1)) * scale, code_at(kw[t][e / 2], 2 * (e & 1) + 1) * scale);
                    uint16_t *k_out = static_cast<uint16_t *>(a.out[0]) + (begin + TPI * t + sub) * a.stride[0] + (uint64_t)h * D + 8 * piece;
                    __builtin_nontemporal_store(y, reinterpret_cast<uint4_t *>(k_out));
                }
            }
            auto put = [&](const uint32_t *w, uint32_t byte, uint32_t t) {     // a token's elements: byte of each w[e]
                uint16_t *to = v_out + (uint64_t)t * a.stride[1] + E * lane;
                float y[E];
                for (int e = 0; e < E; ++e) y[e] = code_at(w[e], (int)byte) * v_scale;
                if constexpr (E == 1) __builtin_nontemporal_store((uint16_t)narrow<BF16>(y[0]), to);
                else if constexpr (E == 2) __builtin_nontemporal_store(narrow2<BF16>(y[0], y[1]), reinterpret_cast<uint32_t *>(to));
                else __builtin_nontemporal_store(uint2_t{narrow2<BF16>(y[0], y[1]), narrow2<BF16>(y[2], y[3])}, reinterpret_cast<uint2_t *>(to));
            };
            if (n == 16 && o == first) {
#pragma unroll
                for (uint32_t p = 0; p < 16; ++p) {
                    uint32_t w[E];
                    for (int e = 0; e < E; ++e) w[e] = vw[e][p / 4];
                    put(w, p & 3, p);
                }
            } else {
#pragma unroll 1
                for (uint32_t t = 0; t < n; ++t) {
                    const uint32_t p = o - first + t;    // place among the 32
                    uint32_t w[E];
                    for (int e = 0; e < E; ++e) {
                        const uint4_t v = p < 16 ? vw[e] : vx[e];
                        const uint32_t lower = p & 4 ? v[1] : v[0], upper = p & 4 ? v[3] : v[2];
                        w[e] = p & 8 ? upper : lower;
                    }
                    put(w, p & 3, t);
                }
            }
        } while (left);
    }
}

}  // namespace

int launch_schedule(const ScheduleArgs &a, void *stream) {
    // a thread a request or token while they are few; four tokens a thread where there are many
    const uint32_t most = a.requests > a.capacity ? a.requests : a.capacity;
    const uint32_t threads = most >= kScheduleThreads ? kScheduleThreads : (most + 63) / 64 * 64;
    // (requests have blocks to take and to give back, too: one workgroup for 64 of them, up to 16)
    uint32_t groups = (uint32_t)(((uint64_t)a.capacity + 4 * kScheduleThreads - 1) / (4 * kScheduleThreads));
    const uint32_t by_request = a.requests >= 1024 ? 16 : (a.requests + 63) / 64;
    if (groups < by_request) groups = by_request;
    k_schedule<<<groups < 256 ? groups : 256, threads, 0, static_cast<hipStream_t>(stream)>>>(a);
    return (int)hipGetLastError();
}

int launch_norm_rotate(const CacheShape &s, const NormRotateArgs &a, void *stream) {
    const uint32_t at_once = 1024 / s.head_dim, passes = (a.q_heads + a.kv_heads + at_once - 1) / at_once;
    uint32_t grid;
    // three passes a wave load the angles once for them (8192 rows of 72 heads of 128: 54 us against 61, nine passes a
    // wave 64; 2048 rows 13.6 against 16.0); a pass a wave while there are fewer waves than the device holds at once
    const uint32_t each = (uint64_t)a.tokens * passes <= 4096 ? passes : (passes + 2) / 3;
    if (int e = workgroups((uint64_t)a.tokens * each, &grid)) return e;
    by_shape(s, [&](auto d, auto bf16) {
        const hipStream_t st = static_cast<hipStream_t>(stream);
        // Streaming loads, which leave the caches to several axes' rows of angles, where the heads are more than the caches hold: 8192 rows
        // of 72 heads of 128 by three axes 58.9 us against 59.9, pairs dealt out in turn 62.5 against 66; 2048 rows of 40 13.0 against 10.8.
        if (a.axes == 0) k_norm_rotate<d(), bf16(), false, false><<<grid, 256, 0, st>>>(a, passes, each);
        else if (2ull * a.tokens * (a.q_heads + a.kv_heads) * d() >= 64ull << 20) k_norm_rotate<d(), bf16(), true, true><<<grid, 256, 0, st>>>(a, passes, each);
        else k_norm_rotate<d(), bf16(), true, false><<<grid, 256, 0, st>>>(a, passes, each);
    });
    return (int)hipGetLastError();
}

int launch_append(const CacheShape &s, const AppendArgs &args, void *stream) {
    AppendArgs a = args;
    // rows of a window: a block's worth, so that a long run's block begins in it, up to a wave's lanes
    a.window = s.block_tokens < 64 ? s.block_tokens : 64;
    const uint64_t windows = ((uint64_t)a.tokens + a.window - 1) / a.window;
    // as many waves as fill the device, if there is work for them: at most a run a row
    const uint64_t most = (uint64_t)(a.tokens < a.window ? a.tokens : a.window) * s.kv_heads * 2;
    uint64_t each = (16384 + windows - 1) / windows;
    if (each > most) each = most;
    a.waves_each = (uint32_t)each;
    uint32_t grid;
    if (int e = workgroups(windows * each, &grid)) return e;
    by_shape(s, [&](auto d, auto bf16) { k_append<d(), bf16()><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a); });
    return (int)hipGetLastError();
}

int launch_gather(const CacheShape &s, const GatherArgs &args, void *stream) {
    GatherArgs a = args;
    const uint64_t groups = ((uint64_t)a.tokens + 63) / 64;
    uint64_t each = (4096 + groups - 1) / groups;
    if (each > s.kv_heads) each = s.kv_heads;
    a.waves_each = (uint32_t)each;
    if (!fits(groups * each, 256)) return kTooLarge;
    by_shape(s, [&](auto d, auto bf16) { k_gather<d(), bf16()><<<(uint32_t)(groups * each), 256, 0, static_cast<hipStream_t>(stream)>>>(a); });
    return (int)hipGetLastError();
}

}  // namespace tsq
