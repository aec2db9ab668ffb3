// Kernels of tsq_cache.h that work on rows: the schedule of blocks and slots, norm and rotation of queries and
// keys, append and gather.
#include <hip/hip_runtime.h>

#include "tsq_cache_internal.hpp"
#include "tsq.h"

namespace tsq {
namespace {

constexpr int kScheduleThreads = 1024;
constexpr int kPerThread = kMaxScheduleRequests / kScheduleThreads;

// Exclusive sums over the workgroup of three 64-bit numbers a thread has; total[] receives the sums of all.
struct Three { uint64_t v[3]; };
__device__ Three scan_three(Three mine, uint64_t (*wave_sum)[3], uint64_t total[3]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Three run = mine;
    for (int d = 1; d < 64; d <<= 1)
        for (int j = 0; j < 3; ++j) {
            const uint64_t o = __shfl_up((unsigned long long)run.v[j], d);
            if (lane >= d) run.v[j] += o;
        }
    if (lane == 63)
        for (int j = 0; j < 3; ++j) wave_sum[wave][j] = run.v[j];
    __syncthreads();
    for (int j = 0; j < 3; ++j) {
        uint64_t before = 0, all = 0;
        for (int w = 0; w < kScheduleThreads / 64; ++w) {
            const uint64_t s = wave_sum[w][j];
            before += w < wave ? s : 0;
            all += s;
        }
        total[j] = all;
        run.v[j] = run.v[j] - mine.v[j] + before;
    }
    return run;
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

__device__ __forceinline__ uint32_t ring_at(uint64_t base, uint32_t k, uint32_t blocks) {
    const uint64_t i = base + k;                       // base < blocks, k <= blocks
    return (uint32_t)(i >= blocks ? i - blocks : i);
}

// One launch, no workgroup waits for another: every workgroup sums up all requests by itself (a few KB from the
// caches) and writes its share of the tokens.  A slot is taken from the table where the request has the block
// already and from the ring where it is new, so no workgroup reads what another one writes.
__global__ __launch_bounds__(kScheduleThreads) void k_schedule(ScheduleArgs a) {
    __shared__ uint32_t first_row[kMaxScheduleRequests + 1], first_new[kMaxScheduleRequests + 1], first_back[kMaxScheduleRequests + 1];
    __shared__ uint64_t wave_sum[kScheduleThreads / 64][3];
    __shared__ uint32_t flags;
    const uint32_t tid = threadIdx.x, B = a.block_tokens, lg = a.block_log2;
    if (tid == 0) flags = 0;
    __syncthreads();

    const int64_t taken = a.counters[0], returned = a.counters[1];
    uint32_t bad = 0;                                   // 1: not an input of this call, 2: no room
    if (taken < 0 || returned < taken || returned - taken > (int64_t)a.blocks) bad = 1;
    uint32_t rows[kPerThread], more[kPerThread], back[kPerThread];
    Three mine = {{0, 0, 0}};
    const uint64_t most = (uint64_t)a.max_blocks << lg;
    for (int j = 0; j < kPerThread; ++j) {
        const uint32_t r = tid * kPerThread + j;
        rows[j] = more[j] = back[j] = 0;
        if (r >= a.requests) continue;
        const int32_t len = a.lengths[r], n = a.fresh[r];
        if (len < 0 || (uint64_t)len > most || n < -1) { bad |= 1; continue; }
        const uint32_t held = ((uint32_t)len + B - 1) >> lg;
        if (n < 0) { back[j] = held; }
        else if ((uint64_t)len + n > most || (uint32_t)n > a.capacity) { bad |= 2; }
        else {
            rows[j] = (uint32_t)n;
            more[j] = (((uint32_t)len + (uint32_t)n + B - 1) >> lg) - held;
        }
        mine.v[0] += rows[j]; mine.v[1] += more[j]; mine.v[2] += back[j];
    }
    if (bad) atomicOr(&flags, bad);
    uint64_t total[3];
    const Three at = scan_three(mine, wave_sum, total);   // (its barrier also closes the writes of flags)
    uint32_t why = flags;
    if (total[0] > a.capacity || (int64_t)total[1] > returned - taken) why |= 2;
    // (a ring that would hold more blocks than there are: a block was given back twice)
    if (!(why & 1) && returned - taken + (int64_t)total[2] > (int64_t)a.blocks) why |= 1;

    const uint32_t first = blockIdx.x * kScheduleThreads + tid, step = gridDim.x * kScheduleThreads;
    if (why) {
        if (blockIdx.x == 0) {
            for (uint32_t r = tid; r < a.requests; r += kScheduleThreads) a.lengths_out[r] = a.lengths[r];
            for (uint32_t r = tid; r <= a.requests; r += kScheduleThreads) a.starts[r] = 0;
            if (tid == 0) {
                a.counters_out[0] = taken;
                a.counters_out[1] = returned;
                a.status[0] = why & 1 ? TSQ_ERR_INVALID_ARG : TSQ_ERR_CAPACITY;
            }
        }
        for (uint32_t i = first; i < a.capacity; i += step) a.positions[i] = a.slots[i] = -1;
        return;
    }
    // from here on every sum fits 32 bits: tokens <= capacity, blocks <= a.blocks
    uint64_t r0 = at.v[0], n0 = at.v[1], b0 = at.v[2];
    for (int j = 0; j < kPerThread; ++j) {
        const uint32_t r = tid * kPerThread + j;
        if (r < a.requests) {
            first_row[r] = (uint32_t)r0; first_new[r] = (uint32_t)n0; first_back[r] = (uint32_t)b0;
            if (blockIdx.x == 0) {
                a.starts[r] = (int32_t)r0;
                a.lengths_out[r] = a.fresh[r] < 0 ? 0 : a.lengths[r] + a.fresh[r];
            }
        }
        r0 += rows[j]; n0 += more[j]; b0 += back[j];
    }
    if (tid == 0) {
        first_row[a.requests] = (uint32_t)total[0]; first_new[a.requests] = (uint32_t)total[1]; first_back[a.requests] = (uint32_t)total[2];
        if (blockIdx.x == 0) {
            a.starts[a.requests] = (int32_t)total[0];
            a.counters_out[0] = taken + (int64_t)total[1];
            a.counters_out[1] = returned + (int64_t)total[2];
            a.status[0] = TSQ_OK;
        }
    }
    __syncthreads();
    const uint64_t head = (uint64_t)taken % a.blocks, tail = (uint64_t)returned % a.blocks;
    for (uint32_t i = first; i < a.capacity; i += step) {
        int32_t position = -1, slot = -1;
        if (i < total[0]) {
            const uint32_t r = owner(first_row, a.requests, i);
            const uint32_t len = (uint32_t)a.lengths[r], held = (len + B - 1) >> lg;
            const uint32_t t = len + (i - first_row[r]), nth = t >> lg;
            const int32_t block = nth < held ? a.table[(uint64_t)r * a.max_blocks + nth]
                                             : a.ring[ring_at(head, first_new[r] + (nth - held), a.blocks)];
            position = (int32_t)t;
            // (an entry that is no block of the cache gives no slot)
            slot = (uint32_t)block < a.blocks ? (int32_t)(((uint32_t)block << lg) + (t & (B - 1))) : -1;
        }
        a.positions[i] = position;
        a.slots[i] = slot;
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
// together are the lane's own: D / 16 lanes a head, 1024 / D heads a wave at a time.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void k_norm_rotate(NormRotateArgs a, uint32_t passes, uint32_t waves_each) {
    constexpr int LPH = D / 16, HEADS = 64 / LPH;
    const uint32_t lane = threadIdx.x & 63, wave = blockIdx.x * 4 + (threadIdx.x >> 6);
    const uint32_t token = wave / waves_each;
    if (token >= a.tokens) return;
    const int32_t position = a.positions[token];
    if (position < 0) return;
    const uint32_t j = lane % LPH, sub = lane / LPH, turning = a.rotary / 16;
    uint32_t e0, e1;                                    // first elements of the lane's two pieces
    const bool turns = j < turning;
    if (a.neighbours || !turns) { e0 = 16 * j; e1 = 16 * j + 8; }
    else { e0 = 8 * j; e1 = 8 * j + a.rotary / 2; }
    float c[8], s[8];
    if (turns && (uint32_t)position < a.angle_rows) {
        const float *row = a.angles + (uint64_t)position * a.rotary + 8 * j;
        for (int i = 0; i < 8; i += 4) {
            *reinterpret_cast<float4_t *>(c + i) = *reinterpret_cast<const float4_t *>(row + i);
            *reinterpret_cast<float4_t *>(s + i) = *reinterpret_cast<const float4_t *>(row + a.rotary / 2 + i);
        }
    } else {
        const float one = (uint32_t)position < a.angle_rows ? 1.0f : __builtin_nanf("");
        for (int i = 0; i < 8; ++i) { c[i] = one; s[i] = one - one; }
    }
    const uint32_t heads = a.q_heads + a.kv_heads, first_pass = wave % waves_each;
    for (uint32_t pass = first_pass; pass < passes; pass += waves_each) {
        const uint32_t h = pass * HEADS + sub;
        const bool is_q = h < a.q_heads, here = h < heads;
        const uint64_t in_at = is_q ? (uint64_t)token * a.q_stride + (uint64_t)h * D : (uint64_t)token * a.k_stride + (uint64_t)(h - a.q_heads) * D;
        const uint64_t out_at = is_q ? (uint64_t)token * a.q_out_stride + (uint64_t)h * D : (uint64_t)token * a.k_out_stride + (uint64_t)(h - a.q_heads) * D;
        const uint16_t *in = static_cast<const uint16_t *>(is_q ? a.q : a.k) + in_at;
        float x[16];
        if (here) {
            const uint4_t p0 = *reinterpret_cast<const uint4_t *>(in + e0), p1 = *reinterpret_cast<const uint4_t *>(in + e1);
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
        *reinterpret_cast<uint4_t *>(out + e0) = o0;
        *reinterpret_cast<uint4_t *>(out + e1) = o1;
    }
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    for (int d = 32; d > 0; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    return v;
}

// Four new codes, or four old ones at their new scale.
__device__ __forceinline__ uint32_t code_of(float x, float inverse) {
    // (NaN, which only a scale of NaN goes with, becomes some code)
    const float q = __builtin_rintf(x * inverse);
    return (uint32_t)(int32_t)fminf(fmaxf(q, -127.0f), 127.0f) & 0xFFu;
}
__device__ __forceinline__ uint32_t recode(uint32_t w, float factor) {
    uint32_t o = 0;
    for (int i = 0; i < 4; ++i) o |= code_of(code_at(w, i), factor) << (8 * i);
    return o;
}

// One run of tokens of one block, for one head, keys (WHICH = 0) or values (1): rows x[0 .. n) go to places
// o .. o + n - 1.  A wave does it by itself: the largest magnitude first (by the bits, so that a NaN or an
// infinity shows as the largest), then the block's scale, then the codes that are there if their scale changes,
// then the new ones.
template <int D, bool BF16, int WHICH>
__device__ void store_run(const uint16_t *x, uint64_t stride, int8_t *codes, float *scale, uint32_t B, uint32_t o, uint32_t n) {
    constexpr uint32_t LPT = D / 8, TPI = 64 / LPT;     // lanes a token, tokens at a time
    const uint32_t lane = threadIdx.x & 63, piece = lane % LPT, sub = lane / LPT;
    uint32_t most = 0;
    for (uint32_t t = sub; t < n; t += TPI) {
        const uint4_t w = *reinterpret_cast<const uint4_t *>(x + t * stride + 8 * piece);
        for (int i = 0; i < 4; ++i) most = max(most, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
    }
    most = wave_max(most);
    const float before = o ? *scale : 0.0f;
    float now = widen<BF16>(most) / 127.0f;
    if (now < 0x1p-126f) now = 0.0f;
    if (most >= (BF16 ? 0x7F80u : 0x7C00u) || before != before) now = __builtin_nanf("");
    else now = fmaxf(before, now);
    const float inverse = now > 0.0f ? 1.0f / now : 0.0f;
    const bool again = o && now > 0.0f && now != before;
    const float factor = again ? before / now : 1.0f;
    if (lane == 0) *scale = now;
    if constexpr (WHICH == 0) {
        if (again)
            for (uint32_t at = lane * 16; at < o * D; at += 1024) {
                uint4_t w = *reinterpret_cast<const uint4_t *>(codes + at);
                for (int i = 0; i < 4; ++i) w[i] = recode(w[i], factor);
                *reinterpret_cast<uint4_t *>(codes + at) = w;
            }
        for (uint32_t t = sub; t < n; t += TPI) {
            const uint4_t w = *reinterpret_cast<const uint4_t *>(x + t * stride + 8 * piece);
            uint2_t c = {0, 0};
            for (int i = 0; i < 4; ++i) {
                c[i / 2] |= code_of(widen<BF16>(w[i] & 0xFFFFu), inverse) << (16 * (i & 1));
                c[i / 2] |= code_of(widen<BF16>(w[i] >> 16), inverse) << (16 * (i & 1) + 8);
            }
            *reinterpret_cast<uint2_t *>(codes + (uint64_t)(o + t) * D + 8 * piece) = c;
        }
    } else {
        // 16 places of an element lie together: a lane makes them of its elements whole, 16 tokens at a time
        constexpr int E = D / 64;                       // elements of a lane, side by side
        for (uint32_t first = again ? 0 : o / 16 * 16; first < o + n; first += 16) {
            uint4_t w[E];
            for (int e = 0; e < E; ++e) {
                w[e] = uint4_t{0, 0, 0, 0};
                if (first < o) {
                    w[e] = *reinterpret_cast<const uint4_t *>(codes + (uint64_t)(E * lane + e) * B + first);
                    if (again)
                        for (int i = 0; i < 4; ++i) w[e][i] = recode(w[e][i], factor);
                }
            }
#pragma unroll
            for (uint32_t p = 0; p < 16; ++p) {
                const uint32_t t = first + p;
                if (t < o || t >= o + n) continue;
                const uint16_t *row = x + (uint64_t)(t - o) * stride + E * lane;
                uint32_t v[E];
                if constexpr (E == 1) v[0] = row[0];
                else if constexpr (E == 2) {
                    const uint32_t q = *reinterpret_cast<const uint32_t *>(row);
                    v[0] = q & 0xFFFFu; v[1] = q >> 16;
                } else {
                    const uint2_t q = *reinterpret_cast<const uint2_t *>(row);
                    v[0] = q[0] & 0xFFFFu; v[1] = q[0] >> 16; v[2] = q[1] & 0xFFFFu; v[3] = q[1] >> 16;
                }
                for (int e = 0; e < E; ++e)
                    w[e][p / 4] = (w[e][p / 4] & ~(0xFFu << (8 * (p & 3)))) | (code_of(widen<BF16>(v[e]), inverse) << (8 * (p & 3)));
            }
            for (int e = 0; e < E; ++e) *reinterpret_cast<uint4_t *>(codes + (uint64_t)(E * lane + e) * B + first) = w[e];
        }
    }
}

// A wave looks for the runs that begin among its rows, for one head, keys or values.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void k_append(AppendArgs a) {
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t unit = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const uint32_t which = (uint32_t)(unit & 1), h = (uint32_t)((unit >> 1) % a.kv_heads);
    const uint64_t seg = (unit >> 1) / a.kv_heads;
    const uint64_t begin = seg * a.segment;
    if (begin >= a.tokens) return;
    const uint32_t end = (uint32_t)min(begin + a.segment, (uint64_t)a.tokens);
    for (uint32_t i = (uint32_t)begin; i < end; ++i) {
        const int32_t slot = a.slots[i];
        if (slot < 0 || ((uint32_t)slot >> a.block_log2) >= a.blocks) continue;
        const uint32_t o = (uint32_t)slot & (a.block_tokens - 1);
        if (i > 0 && o > 0 && a.slots[i - 1] == slot - 1) continue;      // within a run that began before
        // rows that follow at the next places of the same block
        uint32_t n = 0;
        const uint32_t most = min(a.block_tokens - o, a.tokens - i);
        while (n < most) {
            const uint32_t at = n + lane;
            const uint64_t goes = __ballot(at < most && a.slots[i + at] == slot + (int32_t)at);
            const uint32_t got = goes == ~0ull ? 64 : (uint32_t)__builtin_ctzll(~goes);
            n += got;
            if (got < 64) break;
        }
        const uint64_t head = (uint64_t)((uint32_t)slot >> a.block_log2) * a.kv_heads + h;
        const uint64_t codes = head * a.block_tokens * D;
        if (which == 0)
            store_run<D, BF16, 0>(static_cast<const uint16_t *>(a.x[0]) + i * a.stride[0] + (uint64_t)h * D, a.stride[0],
                                  a.codes[0] + codes, a.scale[0] + head, a.block_tokens, o, n);
        else
            store_run<D, BF16, 1>(static_cast<const uint16_t *>(a.x[1]) + i * a.stride[1] + (uint64_t)h * D, a.stride[1],
                                  a.codes[1] + codes, a.scale[1] + head, a.block_tokens, o, n);
    }
}

// Sixteen rows of the output a wave, for one head, keys or values: row i's request, position and block by lane i,
// then the rows that lie in one block together.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void k_gather(GatherArgs a) {
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t unit = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const uint32_t which = (uint32_t)(unit & 1), h = (uint32_t)((unit >> 1) % a.kv_heads);
    const uint64_t begin = (unit >> 1) / a.kv_heads * 16;
    if (begin >= a.tokens) return;
    const uint32_t i = (uint32_t)begin + (lane & 15);
    // the last request that begins at or before the row; the row is its own if it ends behind it
    uint32_t lo = 0, hi = a.requests;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (a.starts[mid] <= (int32_t)i) lo = mid; else hi = mid;
    }
    const int32_t s0 = a.starts[lo], s1 = a.starts[lo + 1];
    const bool owned = i < a.tokens && s0 >= 0 && (int32_t)i >= s0 && (int32_t)i < s1;
    const int64_t position = (int64_t)a.lengths[lo] - s1 + (int32_t)i;
    const uint32_t nth = (uint32_t)((uint64_t)position >> a.block_log2);
    int32_t block = -1;
    if (owned && position >= 0 && ((uint64_t)position >> a.block_log2) < a.max_blocks) block = a.table[(uint64_t)lo * a.max_blocks + nth];
    if ((uint32_t)block >= a.blocks) block = -1;
    const uint32_t before_r = (uint32_t)__shfl_up((int)lo, 1), before_n = (uint32_t)__shfl_up((int)nth, 1);
    const int before_owned = __shfl_up((int)owned, 1);
    const bool leads = owned && lane < 16 && (lane == 0 || !before_owned || before_r != lo || before_n != nth);
    const uint32_t ours = (uint32_t)__ballot(owned && lane < 16);
    uint32_t left = (uint32_t)__ballot(leads);
    while (left) {
        const uint32_t l = (uint32_t)__builtin_ctz(left);
        left &= left - 1;
        // rows of the run: up to the next leader, as far as a request has them
        const uint32_t reach = left ? (uint32_t)__builtin_ctz(left) : 16u;
        uint32_t n = 0;
        while (l + n < reach && (ours >> (l + n) & 1)) ++n;
        const int32_t b = __shfl(block, (int)l);
        const uint32_t o = (uint32_t)__shfl((int)(uint32_t)position, (int)l) & (a.block_tokens - 1);
        const uint64_t row = begin + l;
        uint16_t *out = static_cast<uint16_t *>(a.out[which]) + row * a.stride[which] + (uint64_t)h * D;
        const uint64_t head = (uint64_t)max(b, 0) * a.kv_heads + h;
        const float scale = b < 0 ? __builtin_nanf("") : a.scale[which][head];
        const int8_t *codes = a.codes[which] + head * a.block_tokens * D;
        if (which == 0) {
            constexpr uint32_t LPT = D / 8, TPI = 64 / LPT;
            const uint32_t piece = lane % LPT;
            for (uint32_t t = lane / LPT; t < n; t += TPI) {
                const uint2_t w = *reinterpret_cast<const uint2_t *>(codes + (uint64_t)(o + t) * D + 8 * piece);
                uint4_t y;
                for (int e = 0; e < 4; ++e)
                    y[e] = narrow2<BF16>(code_at(w[e / 2], 2 * (e & 1)) * scale, code_at(w[e / 2], 2 * (e & 1) + 1) * scale);
                *reinterpret_cast<uint4_t *>(out + t * a.stride[0] + 8 * piece) = y;
            }
        } else {
            constexpr int E = D / 64;
            for (uint32_t first = o / 16 * 16; first < o + n; first += 16) {
                uint4_t w[E];
                for (int e = 0; e < E; ++e)
                    w[e] = *reinterpret_cast<const uint4_t *>(codes + (uint64_t)(E * lane + e) * a.block_tokens + first);
#pragma unroll
                for (uint32_t p = 0; p < 16; ++p) {
                    const uint32_t t = first + p;
                    if (t < o || t >= o + n) continue;
                    uint16_t *to = out + (uint64_t)(t - o) * a.stride[1] + E * lane;
                    float y[E];
                    for (int e = 0; e < E; ++e) y[e] = code_at(w[e][p / 4], p & 3) * scale;
                    if constexpr (E == 1) to[0] = (uint16_t)narrow<BF16>(y[0]);
                    else if constexpr (E == 2) *reinterpret_cast<uint32_t *>(to) = narrow2<BF16>(y[0], y[1]);
                    else *reinterpret_cast<uint2_t *>(to) = uint2_t{narrow2<BF16>(y[0], y[1]), narrow2<BF16>(y[2], y[3])};
                }
            }
        }
    }
}

// A grid of n waves in workgroups of four; 2^31 workgroups and more are refused.
int workgroups(uint64_t waves, uint32_t *out) {
    const uint64_t n = (waves + 3) / 4;
    if (n >= (1ull << 31)) return (int)hipErrorInvalidValue;
    *out = (uint32_t)n;
    return 0;
}

}  // namespace

int launch_schedule(const ScheduleArgs &a, void *stream) {
    const uint32_t groups = a.capacity <= 4 * kScheduleThreads ? 1 : (a.capacity + 4 * kScheduleThreads - 1) / (4 * kScheduleThreads);
    k_schedule<<<groups < 256 ? groups : 256, kScheduleThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
    return (int)hipGetLastError();
}

int launch_norm_rotate(const CacheShape &s, const NormRotateArgs &a, void *stream) {
    const uint32_t at_once = 1024 / s.head_dim, passes = (a.q_heads + a.kv_heads + at_once - 1) / at_once;
    uint32_t grid;
    const uint32_t each = passes;
    if (int e = workgroups((uint64_t)a.tokens * each, &grid)) return e;
    by_shape(s, [&](auto d, auto bf16) { k_norm_rotate<d(), bf16()><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a, passes, each); });
    return (int)hipGetLastError();
}

int launch_append(const CacheShape &s, const AppendArgs &a, void *stream) {
    uint32_t grid;
    if (int e = workgroups((((uint64_t)a.tokens + a.segment - 1) / a.segment) * a.kv_heads * 2, &grid)) return e;
    by_shape(s, [&](auto d, auto bf16) { k_append<d(), bf16()><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a); });
    return (int)hipGetLastError();
}

int launch_gather(const CacheShape &s, const GatherArgs &a, void *stream) {
    uint32_t grid;
    if (int e = workgroups((((uint64_t)a.tokens + 15) / 16) * a.kv_heads * 2, &grid)) return e;
    by_shape(s, [&](auto d, auto bf16) { k_gather<d(), bf16()><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a); });
    return (int)hipGetLastError();
}

}  // namespace tsq
