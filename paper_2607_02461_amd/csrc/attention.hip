// Attention of packed sequences for gfx950: o = softmax(scale q k^T) v, row by row.
//
// One pass over a sequence's keys with the running maximum m and sum l of each query's softmax, in fp32 and in units of
// log2: p = 2^(s - m).  The result is rescaled by 2^(m_old - m_new) only where a score passes m by more than 8: until then p
// is at most 2^8, whose sums fp32 holds as well as those of values up to 1.  p enters the second product in bf16, half a step of
// 2^-8 relative, as q, k and v have it; l sums it unrounded.
//
// Bound by the matrix cores (4 D products and sums for each pair of a query and a key), with the exponentials beside them: 64
// keys x 32 queries take a wave 1024 cycles of MFMA and about 750 of VALU at D = 128, which overlap between the waves of a SIMD.
// Beside that they read 32 KB of LDS, 1400 of the card's 2048 cycles for the two waves of a SIMD.  What 4608 tokens in 24 heads of
// 128 (two sequences) reach, 1060 TFLOP/s of matrix products, is set by power: the matrix cores are busy 53% of the time at 1.65
// to 1.8 GHz, and the same call on zeros runs a third faster (1400).  Few queries are bound by HBM: each key and value is read once for
// each of its heads, 16 tokens over 4600 keys on average in 8 heads of 128 at 5.1 TB/s.
//
// Tried and not kept: 64 queries to a wave (its sums leave the registers, 520 TFLOP/s); sums of rounded probabilities by dot products
// (3% faster, but o off by 2^-6 where one key has it all); workgroups that take one tile after the other, which was to hide a tile's
// begin (32760 tokens over 512 keys 435 us for 420; with the next tile's first keys on their way during the last ones 439, with
// queries loaded by the compiler, which waits for all loads then); waves of different priorities (no difference).
//
// Rows: the queries of a group's heads lie together, row = token * group + head of the group, so that one tile of keys serves
// all heads that share it, and a single token of grouped heads fills as much of a tile as there is.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "attention.h"
#include "device.h"
#include "vec.h"

namespace orbit {

namespace {

constexpr float kSlack = 8.f;   // log2 of how far a score may pass the maximum that it is measured from

// A wave's 32 queries: operands, sums and softmax state of the lane's query
template <int DP>
struct Queries {
    u32x4 q[DP / 16];
    f32x16 o[DP / 32];
    float m, l;    // l: of the lane's keys, half of them
    __device__ __forceinline__ void clear() {
        m = kLowest, l = 0.f;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
    }
    // One tile of 32 NB keys; `seen`: keys of the tile that the query sees (all: no mask is applied)
    template <int NB>
    __device__ __forceinline__ void tile(const Operands<DP>& at, const char* k, const char* v, float scale, bool masked, int seen, int lane) {
        f32x16 s[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[n][i] = 0.f;
        // operands are read kAhead k-steps before their products: LDS takes longer than a pair of those
        constexpr int kSteps = DP / 16, kAhead = kSteps < 4 ? kSteps : 4;
        u32x4 a[kSteps][NB];
#pragma unroll
        for (int step = 0; step < kAhead; ++step)
#pragma unroll
            for (int n = 0; n < NB; ++n) a[step][n] = at.rows_of(k, n, step);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int step = 0; step < kSteps; ++step) {
#pragma unroll
            for (int n = 0; n < NB; ++n) s[n] = mfma32(a[step][n], q[step], s[n]);
            if (step + kAhead < kSteps) {
#pragma unroll
                for (int n = 0; n < NB; ++n) a[step + kAhead][n] = at.rows_of(k, n, step + kAhead);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        constexpr int kParts = 2 * NB * (DP / 32), kFirst = DP <= 64 ? (kParts < 4 ? kParts : 4) : 8;
        u32x4 c[kParts];
#pragma unroll
        for (int i = 0; i < kFirst; ++i) c[i] = at.columns_of(v, i / (DP / 32), i % (DP / 32));
        __builtin_amdgcn_sched_barrier(0);
        if (masked) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = 32 * n + 8 * (i / 4) + 4 * (lane >> 5) + i % 4;
                    s[n][i] = key < seen ? s[n][i] : -__builtin_inff();
                }
        }
        float most = s[0][0];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, s[n][i]);
        most = fmaxf(most, other_half(most));
        if (__any(most * scale > m + kSlack)) {
            const float next = fmaxf(m, most * scale), factor = exp2_fast(m - next);
            m = next;
            l *= factor;
#pragma unroll
            for (int b = 0; b < DP / 32; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[b][i] *= factor;
        }
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[n][i] = exp2_fast(__builtin_fmaf(s[n][i], scale, -m));
                sum[i % 4] += s[n][i];
            }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        u32x4 p;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const int u = i / (DP / 32), b = i % (DP / 32);
            if (b == 0) p = as_operand(s[u / 2], u % 2);
            o[b] = mfma32(c[i], p, o[b]);
            if (i + kFirst < kParts) c[i + kFirst] = at.columns_of(v, (i + kFirst) / (DP / 32), (i + kFirst) % (DP / 32));
        }
    }
};

__device__ __forceinline__ const uint16_t* at(const AttnHeads& t, int64_t token, int head) {
    return (const uint16_t*)t.p + token * t.token + head * t.head;
}

// The end of a row: its result and lse, or its part of them.  row: of the tile.
template <int DP, int ROWS>
__device__ __forceinline__ void finish(const AttnParams& p, const AttnTile& t, int kv, int row, Queries<DP>& mine, float l, int lane) {
    const int r = t.first + row;
    const bool live = r < t.q_len * p.group;
    if (t.slot >= 0) {
        const int64_t at = (int64_t)t.slot * p.kv_heads + kv * ROWS + row;
        store_column_f32<DP>(mine.o, 1.f, p.part + at * DP, DP, lane, live);
        if (live && lane < 32) *(f32x2*)(p.stat + 2 * at) = (f32x2){mine.m, l};
        return;
    }
    const int token = min(r / p.group, t.q_len - 1), head = kv * p.group + (r - r / p.group * p.group);
    const float inv = l == 0.f ? 0.f : 1.f / l;   // no key seen: zeros
    const int64_t to = (int64_t)(t.q_start + token) * p.o.token + head * p.o.head;
    if (p.out_f32)
        store_column_f32<DP>(mine.o, inv, (float*)p.o.p + to, p.D, lane, live);
    else
        store_column<DP>(mine.o, inv, (uint16_t*)p.o.p + to, p.D, lane, live);
    if (p.lse && live && lane < 32)
        p.lse[(int64_t)(t.q_start + token) * p.heads + head] = l == 0.f ? -__builtin_inff() : (mine.m + __builtin_log2f(l)) * kLn2;
}

// 32 rows to each wave; 64 keys at a time, shared, in two buffers.  Heads of up to 64 values have three waves to a SIMD, for which
// fewer of V's operands are read ahead: 2048 tokens in 16 heads over 4 of 64, 16 sequences, causal, 217 -> 195 us, whole 326 ->
// 302; 8 of 4096 in 16 heads 630 -> 593.  (These are workgroups of four waves; of those of eight a compute unit has one, two waves
// to a SIMD, in the same registers.)
template <int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DP <= 64 ? 3 : 2) void attention_kernel(AttnParams p) {
    __shared__ __attribute__((aligned(1024))) char lds[2][2][64 * kRowBytes<DP>];
    const Place place = place_of(blockIdx.x, p.kv_heads, p.count);
    if (place.tile >= p.count) return;
    const AttnTile t = p.tiles[place.tile];
    const int kv = place.head, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const TileLoads<DP, 64, WAVES> k(at(p.k, t.k_start, kv), p.k.token, t.k_len - 1, p.D, wave, lane);
    const TileLoads<DP, 64, WAVES> v(at(p.v, t.k_start, kv), p.v.token, t.k_len - 1, p.D, wave, lane);
    auto load = [&](int key, int buffer) {
        k.load(key, lds[buffer][0], p.D, lane);
        v.load(key, lds[buffer][1], p.D, lane);
    };
    if (t.begin < t.end) load(t.begin, 0);
    const Operands<DP> where(lane);
    Queries<DP> mine;
    const int row = 32 * wave + (lane & 31), rows = t.q_len * p.group;
    const int r = min(t.first + row, rows - 1), token = r / p.group;
    load_operand<DP>(at(p.q, t.q_start + token, kv * p.group + r % p.group), p.D, lane, mine.q);
    mine.clear();
    const int seen = seen_keys(p.causal, t.q_len, t.k_len, token);
    // keys that all of the tile's rows see
    const int all = seen_keys(p.causal, t.q_len, t.k_len, t.first / p.group);
    loads_done();
    __syncthreads();
    // in pairs, so that a buffer's place is part of the reads' instructions
    for (int key = t.begin; key < t.end;) {
#pragma unroll
        for (int buffer = 0; buffer < 2; ++buffer) {
            if (key >= t.end) break;
            if (key + 64 < t.end) load(key + 64, buffer ^ 1);
            mine.template tile<2>(where, lds[buffer][0], lds[buffer][1], p.scale, key + 64 > all, seen - key, lane);
            loads_done();
            __syncthreads();
            key += 64;
        }
    }
    finish<DP, 32 * WAVES>(p, t, kv, row, mine, mine.l + other_half(mine.l), lane);
}

// Up to 32 rows: the workgroup's four waves have the same ones and 32 keys each at a time, in buffers of their own, so they wait
// for their own loads alone.  A wave asks for its next tile before a tile's products, but does not multiply beside those loads:
// the compiler does not know that the queries have arrived and waits for all loads in front of the first product of each turn.
// What overlaps loads and products is the four waves, each at another place of its turn: 5.1 TB/s.
template <int DP>
__global__ __launch_bounds__(256) void attention_few_kernel(AttnParams p) {
    extern __shared__ __attribute__((aligned(1024))) char few_lds[];
    constexpr int kTile = 32 * kRowBytes<DP>;
    const Place place = place_of(blockIdx.x, p.kv_heads, p.count);
    if (place.tile >= p.count) return;
    const AttnTile t = p.tiles[place.tile];
    const int kv = place.head, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char* const own = few_lds + wave * 4 * kTile;   // [buffer][k, v]
    const TileLoads<DP, 32, 1> k(at(p.k, t.k_start, kv), p.k.token, t.k_len - 1, p.D, 0, lane);
    const TileLoads<DP, 32, 1> v(at(p.v, t.k_start, kv), p.v.token, t.k_len - 1, p.D, 0, lane);
    auto load = [&](int key, int buffer) {
        k.load(key, own + 2 * buffer * kTile, p.D, lane);
        v.load(key, own + (2 * buffer + 1) * kTile, p.D, lane);
    };
    constexpr int kLoads = 2 * kTile / 1024;   // of a wave for 32 keys
    int key = t.begin + 32 * wave;
    if (key < t.end) load(key, 0);
    const Operands<DP> where(lane);
    Queries<DP> mine;
    const int row = lane & 31, rows = t.q_len * p.group;
    const int r = min(t.first + row, rows - 1), token = r / p.group;
    load_operand<DP>(at(p.q, t.q_start + token, kv * p.group + r % p.group), p.D, lane, mine.q);
    mine.clear();
    const int seen = seen_keys(p.causal, t.q_len, t.k_len, token);
    const int all = seen_keys(p.causal, t.q_len, t.k_len, t.first / p.group);
    for (int buffer = 0; key < t.end; key += 128, buffer ^= 1) {
        if (key + 128 < t.end) {
            reads_done();
            load(key + 128, buffer ^ 1);
            loads_done<kLoads>();
        } else {
            loads_done();
        }
        mine.template tile<1>(where, own + 2 * buffer * kTile, own + (2 * buffer + 1) * kTile, p.scale, key + 32 > all, seen - key, lane);
    }
    // the waves' parts, joined by the first
    __syncthreads();
    float* const sums = (float*)few_lds;                         // [wave][register][lane]
    float* const stats = sums + 4 * DP / 2 * 64;                 // [wave][2][lane]
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[(wave * (DP / 2) + 16 * b + i) * 64 + lane] = mine.o[b][i];
    stats[(2 * wave) * 64 + lane] = mine.m;
    stats[(2 * wave + 1) * 64 + lane] = mine.l + other_half(mine.l);
    __syncthreads();
    if (wave) return;
    float m = kLowest, l = 0.f, factor[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, stats[2 * w * 64 + lane]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        factor[w] = exp2_fast(stats[2 * w * 64 + lane] - m);
        l += factor[w] * stats[(2 * w + 1) * 64 + lane];
    }
    mine.m = m;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) sum += factor[w] * sums[(w * (DP / 2) + 16 * b + i) * 64 + lane];
            mine.o[b][i] = sum;
        }
    finish<DP, kAttnFewRows>(p, t, kv, row, mine, l, lane);
}

// Rows whose keys several workgroups shared, in the order of their parts: DP / 8 lanes to a row, 8 values to a lane.
template <int DP>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnParams p) {
    constexpr int kLanes = DP / 8;
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, id = at / kLanes, which = id / kAttnWideRows / (uint32_t)p.kv_heads;
    const int row = id % kAttnWideRows, kv = id / kAttnWideRows % (uint32_t)p.kv_heads, d = at % kLanes * 8;
    if (which >= (uint32_t)p.count) return;
    const AttnJoin j = p.joins[which];
    const int r = j.first + row;
    if (row >= j.rows || r >= j.q_len * p.group) return;
    float m = kLowest, l = 0.f, o[8] = {};
    const int64_t first = (int64_t)j.slot * p.kv_heads + kv * j.rows + row, step = (int64_t)j.rows * p.kv_heads;
#pragma unroll 4
    for (int i = 0; i < j.count; ++i) m = fmaxf(m, p.stat[2 * (first + i * step)]);
#pragma unroll 4
    for (int i = 0; i < j.count; ++i) {
        const f32x2 stat = *(const f32x2*)(p.stat + 2 * (first + i * step));
        const float* const from = p.part + (first + i * step) * DP + d;
        const f32x4 lo = *(const f32x4*)from, hi = *(const f32x4*)(from + 4);
        const float factor = exp2_fast(stat.x - m);
        l += factor * stat.y;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] += factor * lo[c], o[4 + c] += factor * hi[c];
    }
    const int token = r / p.group, head = kv * p.group + r % p.group;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t to = (int64_t)(j.q_start + token) * p.o.token + head * p.o.head + d;
    if (p.lse && d == 0) p.lse[(int64_t)(j.q_start + token) * p.heads + head] = l == 0.f ? -__builtin_inff() : (m + __builtin_log2f(l)) * kLn2;
    if (d >= p.D) return;
    if (p.out_f32) {
        *(f32x4*)((float*)p.o.p + to) = (f32x4){o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
        *(f32x4*)((float*)p.o.p + to + 4) = (f32x4){o[4] * inv, o[5] * inv, o[6] * inv, o[7] * inv};
    } else {
        *(u32x4*)((uint16_t*)p.o.p + to) = (u32x4){pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv),
                                                  pack_bf16(o[4] * inv, o[5] * inv), pack_bf16(o[6] * inv, o[7] * inv)};
    }
}

template <int DP>
hipError_t launch(const AttnParams& p, AttnWay way, hipStream_t stream) {
    const unsigned grid = (unsigned)places(p.count, p.kv_heads);
    if (way != kAttnShared) {
        if (way == kAttnWide)
            attention_kernel<DP, 8><<<grid, 512, 0, stream>>>(p);
        else
            attention_kernel<DP, 4><<<grid, 256, 0, stream>>>(p);
        return hipGetLastError();
    }
    constexpr int kBytes = 4 * 4 * 32 * kRowBytes<DP>;   // the waves' buffers; their sums and states take less
    static std::atomic<uint64_t> raised{0};
    const hipError_t e = raise_lds_limit((const void*)attention_few_kernel<DP>, kBytes, raised);
    if (e != hipSuccess) return e;
    attention_few_kernel<DP><<<grid, 256, kBytes, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attention(const AttnParams& p, AttnWay way, hipStream_t stream) {
    return with_padded_dim(p.D, [&](auto d) { return launch<decltype(d)::value>(p, way, stream); });
}

hipError_t launch_attention_join(const AttnParams& p, hipStream_t stream) {
    return with_padded_dim(p.D, [&](auto d) {
        constexpr int DP = decltype(d)::value;
        attention_join_kernel<DP><<<(unsigned)(((int64_t)p.count * p.kv_heads * kAttnWideRows * (DP / 8) + 255) / 256), 256, 0, stream>>>(p);
        return hipGetLastError();
    });
}

}  // namespace orbit
