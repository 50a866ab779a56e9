// Gradients of attention over packed sequences for gfx950.
//
// With p = softmax(scale q k^T), dp = do v^T and delta = sum(do o) for each query, ds = p (dp - delta):
//     dq = scale ds k,   dk = scale ds^T q,   dv = p^T do.
// p comes from the scores and the forward pass's lse again.  Two kernels go over the pairs: one has 128 rows and all of their
// keys, for dq; the other 128 keys and all of their rows, for dk and dv.  So every sum is one workgroup's, in a fixed order, and no
// result is added up in memory; that costs 7 products of 2 D operations for each pair instead of the 5 that there are.
//
// Both are bound by the matrix cores and the power that they take: 3 and 4 products for each pair beside one exponential.  At 2 x
// 4429 tokens in 24 heads of 128 they run at 1050 and 1000 TFLOP/s of these products, busy 56% and 50% of the time at 1.8 GHz.
// Short sequences of 64 values keep neither unit busy (7 of up to 2048 tokens in 16 heads over 4, causal: matrix cores 34% and 27%,
// vector units 42% and 33% of the time): workgroups' begins and one round of them of unequal length.  A tile of rows begins with its
// rows of `out`, whose loads wait for each other.  p and ds enter their products in bf16, half a step of 2^-8 relative, as q, k, v and do have it; sums are fp32.
//
// Tried and not kept: 64 keys to a wave of the second kernel (spills); the first kernel's scores of 64 keys before their
// gradients, so that operands of neighbouring products are shared (spills 38 registers at D = 128, 2320 us for 1655); three
// waves to a SIMD for the first kernel at D = 64 (spills 22, 1480 us for 1320).
//
// Rows are those of the forward pass: row = token * group + head of the group; dk and dv sum over a group's heads as over
// tokens.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "attention.h"
#include "device.h"
#include "vec.h"

namespace orbit {

namespace {

__device__ __forceinline__ const uint16_t* at(const AttnHeads& t, int64_t token, int head) {
    return (const uint16_t*)t.p + token * t.token + head * t.head;
}

constexpr int kExactKeys = 512;

// dq of 128 rows, 32 to each wave, over their keys, 64 at a time in two buffers.  Transposed as in the forward pass: a lane has
// one query.
//
// delta comes from the output, which was rounded to its type: an error e that all of a row's ds share, and that reaches dq as
// e sum p k.  Beside many keys of many values that is small; else it was up to a third of the gradients' error.  The exact delta
// makes sum ds = 0, so that sum, taken in fp32 before ds is rounded, is e:
//   - heads of up to 64 values sum p k as well, a product more, and take e times it off at the end (of a tile in parts, where
//     they are joined).  Error of dq in bf16, as a
//     multiple of what its own rounding makes: 1.53 -> 1.47 at 40 values, 1.47 -> 1.44 at 64; forward and backward pass of 7
//     sequences of up to 2048 with 16 heads of 64: 198 -> 210 us.
//   - wider ones have no registers for it.  Tiles of up to kExactKeys keys sum p dp first, which is delta, in a pass of two
//     products more: 1.50 -> 1.44 at 400 keys of 96 values, for 233 -> 266 us of 16 sequences with 24 heads.  Longer ones are
//     left at 1.47 and less: for all of them it cost 970 -> 1100 us at 1163 keys of 128 values.
// The next kernel finds -delta, and -lse in units of the scores (-infinite where the row sees no key: its probabilities are zeros
// then), [key head][token * group + head of the group]: what its products begin from.
template <int DP>
__global__ __launch_bounds__(256, 2) void attention_row_grad_kernel(AttnGradParams p) {
    constexpr bool kSums = DP <= 64;
    __shared__ __attribute__((aligned(1024))) char lds[2][2][64 * kRowBytes<DP>];
    const Place place = place_of(blockIdx.x, p.kv_heads, p.count);
    if (place.tile >= p.count) return;
    const AttnTile t = p.tiles[place.tile];
    const int kv = place.head, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const TileLoads<DP, 64, 4> k(at(p.k, t.k_start, kv), p.k.token, t.k_len - 1, p.D, wave, lane);
    const TileLoads<DP, 64, 4> v(at(p.v, t.k_start, kv), p.v.token, t.k_len - 1, p.D, wave, lane);
    auto load = [&](int key, int buffer) {
        k.load(key, lds[buffer][0], p.D, lane);
        v.load(key, lds[buffer][1], p.D, lane);
    };
    const int row = 32 * wave + (lane & 31), rows = t.q_len * p.group;
    // keys of the tile's last row: of a part of a tile, those of the whole tile
    const int whole = seen_keys(p.causal, t.q_len, t.k_len, (min(t.first + kAttnRows, rows) - 1) / p.group);
    bool last = kSums || whole > kExactKeys;
    int begin = last ? t.begin : 0, end = last ? t.end : whole;
    if (begin < end) load(begin, 0);
    const Operands<DP> where(lane);
    const int r = min(t.first + row, rows - 1), token = r / p.group, head = kv * p.group + r % p.group;
    u32x4 q[DP / 16], g[DP / 16];
    load_operand<DP>(at(p.q, t.q_start + token, head), p.D, lane, q);
    load_operand<DP>(at(p.g, t.q_start + token, head), p.D, lane, g);
    const int64_t token_at = t.q_start + token;
    float delta = 0.f;
    {
        // half of a row's values: those that the lane has of do
        const int64_t from = token_at * p.o.token + head * p.o.head;
#pragma unroll
        for (int step = 0; step < DP / 16; ++step) {
            const int d = 16 * step + 8 * (lane >> 5);
            if (d >= p.D) continue;
            float o[8];
            if (p.o_f32) {
                const f32x4 lo = *(const f32x4*)((const float*)p.o.p + from + d), hi = *(const f32x4*)((const float*)p.o.p + from + d + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = lo[i], o[4 + i] = hi[i];
            } else {
                const u32x4 w = *(const u32x4*)((const uint16_t*)p.o.p + from + d);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[2 * i] = bf16_low(w[i]), o[2 * i + 1] = bf16_high(w[i]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) delta += bf16_low(g[step][i]) * o[2 * i] + bf16_high(g[step][i]) * o[2 * i + 1];
        }
        delta = -(delta + other_half(delta));
    }
    const float lse = p.lse[token_at * p.heads + head];
    const float lse2 = lse == -__builtin_inff() ? lse : -lse * kLog2e;
    const bool live = t.first + row < rows;
    f32x16 dq[DP / 32], mean[kSums ? DP / 32 : 1];
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[b][i] = mean[kSums ? b : 0][i] = 0.f;
    const int seen = seen_keys(p.causal, t.q_len, t.k_len, token), all = seen_keys(p.causal, t.q_len, t.k_len, t.first / p.group);
    float sum;
    for (;; last = true, begin = t.begin, end = t.end) {
        sum = 0.f;
        loads_done();
        __syncthreads();
        for (int key = begin; key < end;) {
#pragma unroll
            for (int buffer = 0; buffer < 2; ++buffer) {
                if (key >= end) break;
                if (key + 64 < end) load(key + 64, buffer ^ 1);
                const char *const kt = lds[buffer][0], *const vt = lds[buffer][1];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    f32x16 s, dp;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.f;
#pragma unroll
                    for (int step = 0; step < DP / 16; ++step) {
                        s = mfma32(where.rows_of(kt, n, step), q[step], s);
                        dp = mfma32(where.rows_of(vt, n, step), g[step], dp);
                    }
                    if (key + 64 > all) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const bool hidden = 32 * n + 8 * (i / 4) + 4 * (lane >> 5) + i % 4 >= seen - key;
                            s[i] = hidden ? -__builtin_inff() : s[i];
                            dp[i] = hidden ? 0.f : dp[i];
                        }
                    }
                    if (!kSums && !last) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum += exp2_fast(__builtin_fmaf(s[i], p.scale, lse2)) * dp[i];
                        continue;
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        s[i] = exp2_fast(__builtin_fmaf(s[i], p.scale, lse2));
                        dp[i] = s[i] * (dp[i] + delta);
                        if constexpr (kSums) sum += dp[i];
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const u32x4 ds = as_operand(dp, u), weights = as_operand(s, u);
#pragma unroll
                        for (int b = 0; b < DP / 32; ++b) {
                            const u32x4 keys = where.columns_of(kt, 2 * n + u, b);
                            dq[b] = mfma32(keys, ds, dq[b]);
                            if constexpr (kSums) mean[b] = mfma32(keys, weights, mean[b]);
                        }
                    }
                }
                loads_done();
                __syncthreads();
                key += 64;
            }
        }
        if (kSums || last) break;
        delta = -(sum + other_half(sum));
        if (t.begin < t.end) load(t.begin, 0);
    }
    if (kSums) sum += other_half(sum);
    if (kSums && t.slot < 0) {
        delta -= sum;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) dq[b][i] -= sum * mean[kSums ? b : 0][i];
    }
    // parts of a tile have the same delta: the first writes it
    if (live && lane < 32 && t.begin == 0) {
        const int64_t stat = ((int64_t)kv * p.q_tokens + t.q_start) * p.group + r;
        p.delta[stat] = delta;
        p.lse2[stat] = lse2 / p.scale;
    }
    if (t.slot < 0) return store_column<DP>(dq, p.out_scale, (uint16_t*)at(p.dq, t.q_start + token, head), p.D, lane, live);
    const int64_t part = (int64_t)t.slot * p.kv_heads + kv * kAttnRows + row;
    store_column_f32<DP>(dq, 1.f, p.part + part * DP, DP, lane, live);
    if constexpr (kSums) {
        store_column_f32<DP>(mean, 1.f, p.part2 + part * DP, DP, lane, live);
        if (live && lane < 32) p.part_sum[part] = sum;
    }
}

// Loads of 64 rows (token * group + head of the group) of one key head's queries by WAVES waves, as TileLoads.
template <int DP, int WAVES>
struct RowLoads {
    static constexpr int kChunks = kRowBytes<DP> / 16, kEach = 64 / kChunks, kLoads = 64 / kEach / WAVES;
    const char* rows;
    int64_t token;    // bytes
    uint32_t head;    // bytes
    int group, last;  // last: row
    uint32_t inverse; // 2^32 / group, rounded up: n * inverse >> 32 is n / group for n < 2^16
    __device__ __forceinline__ RowLoads(const uint16_t* t, int64_t token, int64_t head, int group, int last)
        : rows((const char*)t), token(2 * token), head((uint32_t)(2 * head)), group(group), last(last), inverse((uint32_t)(0xFFFFFFFFull / (uint32_t)group) + 1) {}
    __device__ __forceinline__ void load(int first, char* tile, int D, int wave, int lane) const {
        const uint32_t lds = lds_address(tile) + wave * kLoads * 1024;
        const int from = first / group, rest = first - from * group;   // scalar
        const char* const base = rows + from * token;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = (wave * kLoads + i) * kEach + lane / kChunks;
            const int c = swizzled<DP>(row, lane % kChunks);
            const uint32_t r = (uint32_t)(rest + min(row, last - first));
            const uint32_t ahead = group == 1 ? r : __umulhi(r, inverse);
            const uint32_t offset = ahead * (uint32_t)token + (r - ahead * group) * head + (8 * c >= D ? 0 : 16 * c);
            TileLoads<DP, 64, WAVES>::one(base, offset, lds + 1024 * i);
        }
    }
};

// dk and dv of 128 keys, 32 to each wave, over the rows that see them, 64 at a time in two buffers: q, do, lse2 and delta.  A lane
// has one key.  At D = 128 a wave's keys, values and sums take 192 of its 256 registers, so what follows from the lane is computed
// again where it is used (kept, it spilled 27).
template <int DP>
__global__ __launch_bounds__(256, 2) void attention_key_grad_kernel(AttnGradParams p) {
    constexpr int kTile = 64 * kRowBytes<DP>, kBuffer = 2 * kTile + 1024;
    extern __shared__ __attribute__((aligned(1024))) char key_lds[];
    const Place place = place_of(blockIdx.x, p.kv_heads, p.count);
    if (place.tile >= p.count) return;
    const AttnTile t = p.tiles[place.tile];
    const int kv = place.head, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = t.q_len * p.group, begin = t.begin * p.group, end = t.end * p.group;
    const RowLoads<DP, 4> q(at(p.q, t.q_start, kv * p.group), p.q.token, p.q.head, p.group, rows - 1);
    const RowLoads<DP, 4> g(at(p.g, t.q_start, kv * p.group), p.g.token, p.g.head, p.group, rows - 1);
    const int64_t stat = ((int64_t)kv * p.q_tokens + t.q_start) * p.group;
    const char* const stats = (const char*)((wave & 1 ? p.delta : p.lse2) + stat);
    auto load = [&](int row, int buffer) {
        char* const to = key_lds + buffer * kBuffer;
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));   // what is made of it is made again for each tile: the registers are taken
        q.load(row, to, p.D, wave, lane);
        g.load(row, to + kTile, p.D, wave, lane);
        if (wave < 2)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds_address(to) + 2 * kTile + 256 * wave),
                         "v"((uint32_t)(4 * min(lane, rows - 1 - row))), "s"(stats + 4 * (int64_t)row)
                         : "memory");
    };
    if (begin < end) load(begin, 0);
    Operands<DP> where = Operands<DP>(lane).further(lds_address(key_lds));
    const uint32_t stats_at = lds_address(key_lds) + 16 * (lane >> 5);
    const int key = t.first + 32 * wave + (lane & 31);
    const int64_t token = t.k_start + min(key, t.k_len - 1);
    u32x4 k[DP / 16], v[DP / 16];
    f32x16 dk[DP / 32], dv[DP / 32];
    load_operand<DP>(at(p.k, token, kv), p.D, lane, k);
    load_operand<DP>(at(p.v, token, kv), p.D, lane, v);
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[b][i] = dv[b][i] = 0.f;
    // the first row that sees all of the tile's keys
    const int shift = t.k_len - t.q_len;
    const int all = p.causal ? max(0, min(t.first + kAttnRows, t.k_len) - 1 - shift) * p.group : 0;
    loads_done();
    __syncthreads();
    for (int row = begin; row < end;) {
#pragma unroll
        for (int buffer = 0; buffer < 2; ++buffer) {
            if (row >= end) break;
            if (row + 64 < end) load(row + 64, buffer ^ 1);
            const uint32_t qt = buffer * kBuffer, gt = qt + kTile;   // from key_lds
#pragma unroll 1
            for (int n = 0; n < 2; ++n) {
                f32x16 s, dp;
                asm volatile("" : "+v"(where.row), "+v"(where.column));
                const Operands<DP> rows32 = where.further(n * 32 * kRowBytes<DP>);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t from = stats_at + 128 * n + gt + kTile + 32 * (i / 4);
                    s[i] = (*(const ORBIT_LDS f32x4*)(uintptr_t)from)[i % 4];
                    dp[i] = (*(const ORBIT_LDS f32x4*)(uintptr_t)(from + 256))[i % 4];
                }
#pragma unroll
                for (int step = 0; step < DP / 16; ++step) {
                    s = mfma32(rows32.rows_of(qt, 0, step), k[step], s);
                    dp = mfma32(rows32.rows_of(gt, 0, step), v[step], dp);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[i] = exp2_fast(s[i] * p.scale);
                    dp[i] *= s[i];
                }
                if (row < all || row + 64 > end) {
                    const int first = p.causal ? max(0, key - shift) * p.group : 0;   // that sees the lane's key
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int r = row + 32 * n + 8 * (i / 4) + 4 * (lane >> 5) + i % 4;
                        const bool live = r >= first && r < end;
                        s[i] = live ? s[i] : 0.f;
                        dp[i] = live ? dp[i] : 0.f;
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const u32x4 pb = as_operand(s, u), ds = as_operand(dp, u);
#pragma unroll
                    for (int b = 0; b < DP / 32; ++b) {
                        dv[b] = mfma32(rows32.columns_of(gt, u, b), pb, dv[b]);
                        dk[b] = mfma32(rows32.columns_of(qt, u, b), ds, dk[b]);
                    }
                }
            }
            loads_done();
            __syncthreads();
            row += 64;
        }
    }
    const bool live = key < t.k_len;
    if (t.slot >= 0) {
        const int64_t to = ((int64_t)t.slot * p.kv_heads + kv * kAttnRows + 32 * wave + (lane & 31)) * DP;
        store_column_f32<DP>(dk, 1.f, p.part + to, DP, lane, live);
        store_column_f32<DP>(dv, 1.f, p.part2 + to, DP, lane, live);
    } else {
        store_column<DP>(dk, p.out_scale, (uint16_t*)at(p.dk, token, kv), p.D, lane, live);
        store_column<DP>(dv, 1.f, (uint16_t*)at(p.dv, token, kv), p.D, lane, live);
    }
}

// Sums of the parts of tiles that several workgroups shared, in the order of their slots: DP / 8 lanes to a row or key.
template <int DP>
__global__ __launch_bounds__(256) void attention_grad_join_kernel(AttnGradParams p, bool keys) {
    constexpr int kLanes = DP / 8;
    const uint32_t place = blockIdx.x * 256 + threadIdx.x, id = place / kLanes, which_join = id / kAttnRows / (uint32_t)p.kv_heads;
    const int row = id % kAttnRows, kv = id / kAttnRows % (uint32_t)p.kv_heads, d = place % kLanes * 8;
    if (which_join >= (uint32_t)p.count) return;
    const AttnJoin j = p.joins[which_join];
    const int r = j.first + row;
    if (r >= (keys ? j.k_len : j.q_len * p.group) || d >= p.D) return;
    float first[8], all = 0.f;   // of the rows' parts: sum ds k, and sum ds
    const bool sums = DP <= 64 && !keys;
    if (sums) {
        for (int i = 0; i < j.count; ++i) all += p.part_sum[(int64_t)(j.slot + i * kAttnRows) * p.kv_heads + kv * kAttnRows + row];
        if (d == 0) p.delta[((int64_t)kv * p.q_tokens + j.q_start) * p.group + r] -= all;
    }
    for (int which = 0; which < (keys || sums ? 2 : 1); ++which) {
        const float* const part = which ? p.part2 : p.part;
        float sum[8] = {};
#pragma unroll 4
        for (int i = 0; i < j.count; ++i) {
            const float* const from = part + ((int64_t)(j.slot + i * kAttnRows) * p.kv_heads + kv * kAttnRows + row) * DP + d;
            const f32x4 lo = *(const f32x4*)from, hi = *(const f32x4*)(from + 4);
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[c] += lo[c], sum[4 + c] += hi[c];
        }
        if (sums) {
#pragma unroll
            for (int c = 0; c < 8; ++c) which ? sum[c] = first[c] - all * sum[c] : first[c] = sum[c];
            if (!which) continue;
        }
        const float factor = keys && which ? 1.f : p.out_scale;
        u32x4 w;
#pragma unroll
        for (int c = 0; c < 4; ++c) w[c] = pack_bf16(sum[2 * c] * factor, sum[2 * c + 1] * factor);
        const uint16_t* const to = keys ? at(which ? p.dv : p.dk, j.k_start + r, kv) : at(p.dq, j.q_start + r / p.group, kv * p.group + r % p.group);
        *(u32x4*)(to + d) = w;
    }
}

template <int DP>
hipError_t launch(const AttnGradParams& p, AttnGradStep step, hipStream_t stream) {
    const unsigned grid = (unsigned)places(p.count, p.kv_heads);
    switch (step) {
        case kAttnRowGrad:
            attention_row_grad_kernel<DP><<<grid, 256, 0, stream>>>(p);
            break;
        case kAttnKeyGrad: {
            constexpr int kBytes = 2 * (2 * 64 * kRowBytes<DP> + 1024);
            static std::atomic<uint64_t> raised{0};
            const hipError_t e = raise_lds_limit((const void*)attention_key_grad_kernel<DP>, kBytes, raised);
            if (e != hipSuccess) return e;
            attention_key_grad_kernel<DP><<<grid, 256, kBytes, stream>>>(p);
            break;
        }
        default:
            attention_grad_join_kernel<DP><<<(unsigned)(((int64_t)p.count * p.kv_heads * kAttnRows * (DP / 8) + 255) / 256), 256, 0, stream>>>(p, step == kAttnKeyJoin);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_grad(const AttnGradParams& p, AttnGradStep step, hipStream_t stream) {
    return with_padded_dim(p.D, [&](auto d) { return launch<decltype(d)::value>(p, step, stream); });
}

}  // namespace orbit
