// Low-rank adapters of many requests beside the projection they share, forward and backward, for gfx950.
//
// Rows m of one request use one adapter a, of rank r <= R and scale s:
//     h = x A_a^T,  y = base + s h B_a^T                                    (A_a [R][K], B_a [N][R], bf16)
// and with g = dy B_a
//     dx = s g A_a,  dA_a = s sum over its rows of g^T x,  dB_a = s sum over its rows of dy^T h.
// At ranks up to 128 all of it is bound by the wide matrices x, base, y, dy and dx, which each kernel streams once (x and dy
// are read by two: by the shrink, and by the gradients):
//   shrink  h (or g): a wide matrix times a narrow one, contraction over the wide side
//   expand  y (or dx): a narrow matrix times a narrow one, added to the wide base on its way through the registers
//   grad    dA, dB: contraction over rows, of a wide matrix and a narrow one
// The matrix cores multiply bf16.  x, dy, A and B are bf16 and their products exact; h and g are fp32 sums and go into
// the next product as a sum of three bf16 values, which have all 24 bits of their fraction.  That costs MFMAs and no
// memory traffic.  (Two values lose 2^-17 of h: below a bf16 result's own rounding, but not where terms cancel.  They took
// the same time to 1% up to rank 32, 2% less at rank 64, and 187 for 199 us at rank 128: 9216 rows in bf16, 3072 -> 9216.)
//
// A tile is up to 64 rows of one adapter; the plan lists them.  An MFMA operand is 8 values in a row of the contraction for
// row (or column) lane % 16; loaded as such from rows 128 bytes or more apart, each lane's 16 bytes are a request of their
// own, 65 cycles to a wave's load against 18 for 1 KB in a row (measured in L2).  So wide rows, and narrow ones that
// several waves read, go through LDS, or lie in memory in the operands' order.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "device.h"
#include "vec.h"

namespace orbit {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// 16 bytes at any element: rows of odd length begin anywhere
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

__device__ __forceinline__ u32x4 load8(const uint16_t* p) { return *(const u32x4_any*)p; }

// The first n of 8 values, zeros after them; n may be below 1 or above 8
__device__ __forceinline__ u32x4 load8_part(const uint16_t* p, int64_t n) {
    if (n >= 8) return load8(p);
    u32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) v[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
    return v;
}

__device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// v - hi, and 0 where hi holds v already: of an infinity too
__device__ __forceinline__ float rest(float v, float hi) { return v == hi ? 0.f : v - hi; }

constexpr int kParts = 3;

// v as the sum of kParts bf16 values, the largest first; v becomes what is left.  Each is cut off after its 8 bits and
// not rounded: the next one has what follows, and a value above bf16's largest does not become an infinity.
__device__ __forceinline__ void split8(float* v, u32x4* part) {
#pragma unroll
    for (int k = 0; k < kParts; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = __builtin_amdgcn_perm(__float_as_uint(v[2 * i + 1]), __float_as_uint(v[2 * i]), 0x07060302u);
            part[k][i] = w;
            v[2 * i] = rest(v[2 * i], bf16_low(w));
            v[2 * i + 1] = rest(v[2 * i + 1], bf16_high(w));
        }
}

// 8 rows of 8 values become 8 columns
__device__ __forceinline__ void transpose8(u32x4 (&v)[8]) {
    u32x4 out[8];
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            out[c][i] = __builtin_amdgcn_perm(v[2 * i + 1][c / 2], v[2 * i][c / 2], c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = out[c];
}

constexpr int kWaves = 4;

// Where the sums of 16 rows and 32 r's begin, of a split of a tile: 64 lanes of 4 values twice, the order of an operand of
// the expansion in fp32.
__device__ __forceinline__ int64_t lora_sum(int split, int64_t tiles, int64_t tile, int rows, int c, int R) {
    const int wide = (R + 31) / 32;
    return (((split * tiles + tile) * 4 + rows) * wide + c) * 512;
}

// Where value (row of a tile, r) of part k lies in what the gradients' kernel reads, in the order of its operands: per 32
// rows, part and 16 r's, 64 lanes of 8 rows.
__device__ __forceinline__ int64_t lora_operand(int64_t tile, int row, int k, int r, int R) {
    const int64_t block = ((tile * 2 + row / 32) * kParts + k) * ((R + 15) / 16) + r / 16;
    return (block * 64 + row % 32 / 8 * 16 + r % 16) * 8 + row % 8;
}

// h partial sums (lora_sum) of rows x [M][K] and pool [adapter][R][K]: a workgroup takes a tile and a split of K, in
// chunks of 128 that all its waves bring to LDS, the loads of the next two on their way while one is multiplied.  Each wave
// takes 32 of a chunk's 128 for all rows, so that LDS is read once, and their sums are added at the end.  Bound by HBM:
// 33272 rows of 5120, rank 64, 100 us (3.4 TB/s); 9216 rows of 3072, rank 32, 17.5 us (3.2 TB/s).
template <int RF>
__global__ __launch_bounds__(64 * kWaves) void lora_shrink_kernel(LoraShrink p) {
    constexpr int kX = 64 * 16, kA = RF * 16 * 16;                    // pieces of 16 bytes: 16 to a row
    constexpr int kSumRow = RF * 16 + 4, kSums = kWaves * 16 * kSumRow / 4;
    __shared__ u32x4 lds[kX + kA > kSums ? kX + kA : kSums];          // at the end the waves' sums of 16 rows
    const LoraTile t = p.tiles[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, q = lane >> 4;

    f32x4 acc[4][RF];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int r = 0; r < RF; ++r) acc[m][r] = (f32x4){0, 0, 0, 0};
    if (t.rank > 0) {
        // this thread's piece of a row, and its rows tid / 16 + 16 j (the last one again beyond the tile's and the rank's)
        const int piece = tid & 15, line = tid >> 4;
        const uint16_t* x[4];
        const uint16_t* a[RF];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = p.x + ((int64_t)t.row + min(line + 16 * j, t.rows - 1)) * p.ldx + piece * 8;
#pragma unroll
        for (int j = 0; j < RF; ++j) a[j] = p.pool + ((int64_t)t.adapter * p.R + min(line + 16 * j, t.rank - 1)) * p.ldp + piece * 8;
        int64_t k = (int64_t)blockIdx.y * p.steps * 128;
        const int64_t end = max(k, min(k + (int64_t)p.steps * 128, p.K));
        u32x4 xv[2][4], av[2][RF];
        auto load = [&](int d, int64_t at) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) xv[d][j] = load8(x[j] + at);
#pragma unroll
            for (int j = 0; j < RF; ++j) av[d][j] = load8(a[j] + at);
        };
        auto stage = [&](int d) __attribute__((always_inline)) {
            // piece c of row r lies at c ^ r % 16: rows read at one piece fall on different banks
#pragma unroll
            for (int j = 0; j < 4; ++j) lds[(line + 16 * j) * 16 + (piece ^ line)] = xv[d][j];
#pragma unroll
            for (int j = 0; j < RF; ++j) lds[kX + (line + 16 * j) * 16 + (piece ^ line)] = line + 16 * j < t.rank ? av[d][j] : (u32x4){0, 0, 0, 0};
            __syncthreads();
        };
        const int mine = i * 16 + ((wave * 4 + q) ^ i);
        auto multiply = [&]() __attribute__((always_inline)) {
            u32x4 row[4], of_a[RF];
#pragma unroll
            for (int m = 0; m < 4; ++m) row[m] = lds[m * 256 + mine];
#pragma unroll
            for (int r = 0; r < RF; ++r) of_a[r] = lds[kX + r * 256 + mine];
            __builtin_amdgcn_sched_barrier(0);  // (the compiler would wait for every read)
#pragma unroll
            for (int r = 0; r < RF; ++r)
#pragma unroll
                for (int m = 0; m < 4; ++m) acc[m][r] = mfma(row[m], of_a[r], acc[m][r]);
            __syncthreads();
        };
        // every load in this loop comes whether it is needed or not (the last chunk's again), and nothing leaves the loop
        // halfway: after a branch around a load the compiler waits for all of them
        const int n = (int)((end - k) / 128);
        if (n > 0) {
            load(0, k);
            load(1, k + 128 * min(1, n - 1));
            int c = 0;
            for (; c < n - 1; c += 2) {
                stage(0);
                load(0, k + 128 * (int64_t)min(c + 2, n - 1));
                multiply();
                stage(1);
                load(1, k + 128 * (int64_t)min(c + 3, n - 1));
                multiply();
            }
            if (c < n) {
                stage(0);
                multiply();
            }
            k += 128 * (int64_t)n;
        }
        if (k < end) {
            // a partial chunk: the 128 that end with it, those before it cleared, or all there are of fewer than 128
            const int64_t at = max(end - 128, (int64_t)0);
            if (p.K >= 128) {
                load(0, at);
            } else {
                // the pool's rows are padded to 8 values
#pragma unroll
                for (int j = 0; j < 4; ++j) xv[0][j] = load8_part(x[j], end - piece * 8);
#pragma unroll
                for (int j = 0; j < RF; ++j) {
                    av[0][j] = (u32x4){0, 0, 0, 0};
                    if (piece * 8 < end) av[0][j] = *(const u32x4*)a[j];
                }
            }
            const int skip = (int)(k - at) - piece * 8;
            u32x4 keep;
#pragma unroll
            for (int j = 0; j < 4; ++j) keep[j] = (2 * j >= skip ? 0xFFFFu : 0u) | (2 * j + 1 >= skip ? 0xFFFF0000u : 0u);
#pragma unroll
            for (int j = 0; j < 4; ++j) xv[0][j] &= keep;
#pragma unroll
            for (int j = 0; j < RF; ++j) av[0][j] &= keep;
            stage(0);
            multiply();
        }
    }
    float* const sums = (float*)lds;
    const int columns = (p.R + 31) / 32 * 32;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        if (m * 16 >= t.rows) break;
        if (m) __syncthreads();
#pragma unroll
        for (int r = 0; r < RF; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) sums[(wave * 16 + q * 4 + j) * kSumRow + r * 16 + i] = acc[m][r][j];
        __syncthreads();
        float* const out = p.h + lora_sum(blockIdx.y, gridDim.x, blockIdx.x, m, 0, p.R);
        for (int e = tid; e < columns * 16; e += 64 * kWaves) {
            // value e % 4 of lane e / 4 % 64, in the half e / 256 % 2 of its 8, of 32 r's e / 512
            const int row = e / 4 % 16, r = e / 512 * 32 + e / 64 % 4 * 8 + e / 256 % 2 * 4 + e % 4;
            const float* const v = sums + row * kSumRow + r;
            // a row of x that is not finite times the rank's missing rows of A is nothing all the same
            out[e] = r < t.rank ? (v[0] + v[16 * kSumRow]) + (v[32 * kSumRow] + v[48 * kSumRow]) : 0.f;
        }
    }
}

// 16 bytes of a row of the wide output and of its base: the first n of their values, or all.  stream: a non-temporal store.
template <typename T>
struct Wide;

template <>
struct Wide<bf16_t> {
    static constexpr int kValues = 8;
    u32x4 w;
    __device__ __forceinline__ void load(const bf16_t* p) { w = load8((const uint16_t*)p); }
    __device__ __forceinline__ void load(const bf16_t* p, int64_t n) { w = load8_part((const uint16_t*)p, n); }
    __device__ __forceinline__ void clear() { w = (u32x4){0, 0, 0, 0}; }
    __device__ __forceinline__ void add(const f32x4* d) {
        const f32x4 a = d[0], b = d[1];
        w = (u32x4){pack_bf16(bf16_low(w[0]) + a[0], bf16_high(w[0]) + a[1]), pack_bf16(bf16_low(w[1]) + a[2], bf16_high(w[1]) + a[3]),
                    pack_bf16(bf16_low(w[2]) + b[0], bf16_high(w[2]) + b[1]), pack_bf16(bf16_low(w[3]) + b[2], bf16_high(w[3]) + b[3])};
    }
    __device__ __forceinline__ void store(bf16_t* p) const { *(u32x4_any*)p = w; }
    __device__ __forceinline__ void stream(bf16_t* p) const { __builtin_nontemporal_store(w, (u32x4_any*)p); }
    __device__ __forceinline__ void store(bf16_t* p, int64_t n) const {
        if (n >= 8) return store(p);
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) p[i].bits = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
    }
};

template <>
struct Wide<float> {
    static constexpr int kValues = 4;
    f32x4 w;
    __device__ __forceinline__ void load(const float* p) { w = *(const f32x4_any*)p; }
    __device__ __forceinline__ void load(const float* p, int64_t n) {
        if (n >= 4) return load(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = i < n ? p[i] : 0.f;
    }
    __device__ __forceinline__ void clear() { w = (f32x4){0, 0, 0, 0}; }
    __device__ __forceinline__ void add(const f32x4* d) { w += d[0]; }
    __device__ __forceinline__ void store(float* p) const { *(f32x4_any*)p = w; }
    __device__ __forceinline__ void stream(float* p) const { __builtin_nontemporal_store(w, (f32x4_any*)p); }
    __device__ __forceinline__ void store(float* p, int64_t n) const {
        if (n >= 4) return store(p);
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) p[i] = w[i];
    }
};

constexpr int kTimes = 4;  // rows to a lane in a strip of 16 rows of 256 bytes

// 16 rows of a tile of s h as operands of the expansion: the lane has row i and r = 32 c + 8 q .. + 7.
template <int RC>
__device__ __forceinline__ void load_h(const LoraExpand& p, const LoraTile& t, int tile, int rows, int lane, u32x4 (&h)[RC][kParts]) {
#pragma unroll
    for (int c = 0; c < RC; ++c) {
        f32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
        if (c * 32 < p.R) {
#pragma unroll 4
            for (int s = 0; s < p.splits; ++s) {
                const float* const from = p.h + lora_sum(s, p.count, tile, rows, c, p.R) + lane * 4;
                lo += *(const f32x4*)from;
                hi += *(const f32x4*)(from + 256);
            }
        }
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = lo[j] * t.scale, v[j + 4] = hi[j] * t.scale;
        split8(v, h[c]);
    }
}

// The same rows for what comes after the expansion: h itself [M][R], and s h in three parts in the order of lora_operand,
// for which they turn around in the wave's part of LDS.
__device__ __forceinline__ void copy_h(const LoraExpand& p, const LoraTile& t, int tile, int rows, int lane, float* turn, int stride) {
    const int i = lane & 15, q = lane >> 4;
    for (int c = 0; c * 32 < p.R; ++c) {
        f32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
        for (int s = 0; s < p.splits; ++s) {
            const float* const from = p.h + lora_sum(s, p.count, tile, rows, c, p.R) + lane * 4;
            lo += *(const f32x4*)from;
            hi += *(const f32x4*)(from + 256);
        }
        if (p.sum && rows * 16 + i < t.rows && c * 32 + q * 8 < p.R) {
            float* const to = p.sum + ((int64_t)t.row + rows * 16 + i) * p.R + c * 32 + q * 8;
            *(f32x4*)to = lo;
            *(f32x4*)(to + 4) = hi;
        }
        if (!p.turned || rows * 16 >= t.rows) continue;
        *(f32x4*)(turn + i * stride + q * 8) = lo * t.scale;
        *(f32x4*)(turn + i * stride + q * 8 + 4) = hi * t.scale;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        // lane: r = 16 (lane / 32) + lane % 16 of the 32, rows 8 (lane / 16 % 2) .. + 7 of the 16
        const int r = lane / 32 * 16 + i, first = lane / 16 % 2 * 8;
        float v[8];
        u32x4 part[kParts];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = turn[(first + j) * stride + r];
        split8(v, part);
        if (c * 32 + r < p.R) {
#pragma unroll
            for (int k = 0; k < kParts; ++k) *(u32x4*)(p.turned + lora_operand(tile, rows * 16 + first, k, c * 32 + r, p.R)) = part[k];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// y = base + s h B^T.  A workgroup takes a tile and p.columns columns of y in strips of 256 bytes, a wave 16 rows.  The
// strip's rows of the pool [adapter][N][R] are in LDS for all waves.  The MFMA's rows are columns of y and its columns
// rows of y, so a lane ends up with four values in a row of 16 rows; they turn around in the wave's own part of LDS, so
// that base and y are read and written in rows of 256 bytes (a copy of 9216 x 9216 bf16 values runs at 4.8 TB/s so, at
// 4.2 in 16 rows of 64 bytes).  The next strip's loads are on their way while this one is multiplied, and go out ahead of
// this one's stores, since loads and stores are waited for in the order of their issue.  Bound by HBM: 33272 x 13824
// values in fp32, rank 64, 666 us (5.5 TB/s); 9216 x 9216 in bf16, rank 32, 69 us (4.9 TB/s).
template <typename T, int RC, bool BASE>
__global__ __launch_bounds__(64 * kWaves) void lora_expand_kernel(LoraExpand p) {
    constexpr int kValues = Wide<T>::kValues, kStrip = 16 * kValues;
    constexpr int kPieces = kStrip * RC * 4 / (64 * kWaves);  // of 16 bytes of the pool to a thread
    constexpr int kRow = kStrip + 4;
    constexpr int kZero = kStrip * (RC * 4 + 1);              // the last piece is zero
    __shared__ __align__(16) float turn[kWaves * 16 * kRow];
    __shared__ u32x4 pool_lds[kZero + 1];
    // workgroups go to the eight dies in turn: all of a tile's go to one, whose L2 then has the tile's sums
    const int die = blockIdx.x % 8, at = blockIdx.x / 8, block = at % p.blocks, tile = at / p.blocks * 8 + die;
    if (tile >= p.count) return;
    const LoraTile t = p.tiles[tile];
    if (t.rank == 0 && p.base == p.y && p.ldb == p.ldy && !p.sum) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, q = lane >> 4;
    const int first = wave * 16;
    const int pieces = p.R / 8, stride = pieces | 1;  // of a pool row, in memory and, on all banks, in LDS
    const uint16_t* const pool = p.pool + (int64_t)max(t.adapter, 0) * p.N * p.R;
    int64_t n0 = (int64_t)block * p.columns;
    const int64_t end = min(n0 + p.columns, p.N);
    const int64_t last = n0 + (end - n0) / kStrip * kStrip - kStrip;  // the last whole strip (below n0: there is none)

    // of this thread: rows 16 wave + q + 4 j of the tile (its last one again beyond its rows), 16 bytes of their columns
    const int col = i * kValues;
    const T* base[kTimes];
    T* y[kTimes];
#pragma unroll
    for (int j = 0; j < kTimes; ++j) {
        const int64_t row = (int64_t)t.row + min(first + q + 4 * j, t.rows - 1);
        if (BASE) base[j] = (const T*)p.base + row * p.ldb + col;
        y[j] = (T*)p.y + row * p.ldy + col;
    }
    // and pieces of the strip's pool rows, which lie one behind the other in memory
    int slot[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        const int e = tid + 64 * kWaves * j, n = e / pieces;
        slot[j] = n < kStrip ? n * stride + e - n * pieces : -1;
    }
    Wide<T> wide[kTimes];
    u32x4 piece[kPieces];
    auto load_wide = [&](int64_t n) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kTimes; ++j) {
            if (BASE)
                wide[j].load(base[j] + n);
            else
                wide[j].clear();
        }
    };
    auto load_pool = [&](int64_t n) __attribute__((always_inline)) {
        const int64_t most = (p.N - n) * pieces - 1;
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
            piece[j] = *(const u32x4*)(pool + n * p.R + min((int64_t)(slot[j] < 0 ? 0 : tid + 64 * kWaves * j), most) * 8);
    };
    if (last >= n0) load_wide(n0);
    if (t.rank > 0) load_pool(n0);
    u32x4 h[RC][kParts];
    load_h<RC>(p, t, tile, wave, lane, h);
    if (block == 0 && (p.sum || p.turned)) copy_h(p, t, tile, wave, lane, turn + wave * 16 * kRow, kRow);

    // where the lane's operand pieces lie: those beyond R are the zero one
    if (tid == 0) pool_lds[kZero] = (u32x4){0, 0, 0, 0};
    int operand[RC], next[RC];
#pragma unroll
    for (int c = 0; c < RC; ++c) {
        const bool there = c * 4 + q < pieces;
        operand[c] = there ? i * stride + c * 4 + q : kZero;
        next[c] = there ? 16 * stride : 0;
    }
    float* const mine = turn + wave * 16 * kRow;
    auto stage = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            if (t.rank < p.R) {
                const int left = t.rank - (tid + 64 * kWaves * j) % pieces * 8;
#pragma unroll
                for (int e = 0; e < 4; ++e) piece[j][e] &= (2 * e < left ? 0xFFFFu : 0u) | (2 * e + 1 < left ? 0xFFFF0000u : 0u);
            }
            if (slot[j] >= 0) pool_lds[slot[j]] = piece[j];
        }
        __syncthreads();
    };
    // LDS reads go out in groups ahead of the products that take them, and products of different columns follow each
    // other: left alone, the compiler waits for every read and adds four products to one sum back to back
    auto add = [&]() __attribute__((always_inline)) {
        constexpr int kGroup = RC == 4 ? 2 : 4;  // of 16 columns
#pragma unroll
        for (int f0 = 0; f0 < kValues; f0 += kGroup) {
            u32x4 b[kGroup][RC];
            f32x4 acc[kGroup];
#pragma unroll
            for (int f = 0; f < kGroup; ++f) {
                acc[f] = (f32x4){0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < RC; ++c) b[f][c] = pool_lds[operand[c] + (f0 + f) * next[c]];
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int c = 0; c < RC; ++c)
#pragma unroll
                for (int k = kParts - 1; k >= 0; --k)
#pragma unroll
                    for (int f = 0; f < kGroup; ++f) acc[f] = mfma(b[f][c], h[c][k], acc[f]);
#pragma unroll
            for (int f = 0; f < kGroup; ++f) *(f32x4*)(mine + i * kRow + 16 * (f0 + f) + 4 * q) = acc[f];
        }
        // the wave's own rows of LDS: its accesses stay in order, and the compiler keeps them so
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        f32x4 delta[kTimes][kValues / 4];
#pragma unroll
        for (int j = 0; j < kTimes; ++j)
#pragma unroll
            for (int e = 0; e < kValues / 4; ++e) delta[j][e] = *(const f32x4*)(mine + (q + 4 * j) * kRow + col + 4 * e);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < kTimes; ++j) wide[j].add(delta[j]);
    };
    // a whole tile's strips have no test between their loads and stores, after which the compiler would wait for all
    auto strips = [&](auto whole, auto stream) __attribute__((always_inline)) {
        for (; n0 <= last; n0 += kStrip) {
            const int64_t then = min(n0 + kStrip, last);
            if (t.rank > 0) {
                stage();
                load_pool(n0 < last ? then : min(n0 + kStrip, p.N - 1));
                add();
            }
            Wide<T> out[kTimes];
#pragma unroll
            for (int j = 0; j < kTimes; ++j) out[j] = wide[j];
            load_wide(then);
#pragma unroll
            for (int j = 0; j < kTimes; ++j) {
                if (stream.value)
                    out[j].stream(y[j] + n0);
                else if (whole.value || first + q + 4 * j < t.rows)
                    out[j].store(y[j] + n0);
            }
            if (t.rank > 0) __syncthreads();
        }
    };
    if (t.rows < kLoraTileRows)
        strips(std::false_type{}, std::false_type{});
    else if (p.stream)
        strips(std::true_type{}, std::true_type{});
    else
        strips(std::true_type{}, std::false_type{});
    if (n0 < end) {
        // the last columns; their part of the pool is here or on its way
#pragma unroll
        for (int j = 0; j < kTimes; ++j)
            if (wide[j].clear(); BASE && n0 + col < p.N) wide[j].load(base[j] + n0, p.N - n0 - col);
        if (t.rank > 0) {
            stage();
            add();
        }
#pragma unroll
        for (int j = 0; j < kTimes; ++j)
            if (first + q + 4 * j < t.rows && n0 + col < p.N) wide[j].store(y[j] + n0, p.N - n0 - col);
    }
}

// Both products in one kernel for tiles of at most ROWS rows, the single tokens of many requests: bound by launches and
// latency, and by the pools, which every workgroup streams in rows of 1 KB.  A workgroup takes a tile and p.columns
// columns; its waves make h for themselves (A comes from L2 for all but the first), each for R / 8 rows of A, in fp32
// with the lanes along K; then 2^k >= R / 8 lanes share a row of B.  16 rows of 16 adapters of rank 16, 3072 -> 18432:
// 7.2 us for 13 MB, and 17 with the two kernels above and their launches.
constexpr int kRowWaves = 8, kAhead = 4;  // waves to a workgroup, and groups of rows of B that a wave has on their way

template <int LANES>
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
    for (int apart = 1; apart < LANES; apart *= 2) v += __shfl_xor(v, apart);
    return v;
}

__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, a), __builtin_bit_cast(bf16x2_t, b), c, false);
}

template <typename T>
__device__ __forceinline__ float wide_value(const T* p);
template <>
__device__ __forceinline__ float wide_value<bf16_t>(const bf16_t* p) { return bf16_low(p->bits); }
template <>
__device__ __forceinline__ float wide_value<float>(const float* p) { return *p; }
__device__ __forceinline__ void set_wide(bf16_t* p, float v) { p->bits = (uint16_t)pack_bf16(v, v); }
__device__ __forceinline__ void set_wide(float* p, float v) { *p = v; }

template <typename T, int RPW, int ROWS>
__global__ __launch_bounds__(64 * kRowWaves) void lora_rows_kernel(LoraRows p) {
    constexpr int kLanes = RPW, kGroups = 64 / kLanes;  // lanes to a row of B: 8 values of r each
    __shared__ float hs[ROWS][RPW * kRowWaves];
    const LoraTile t = p.tiles[blockIdx.x];
    if (t.rank == 0 && p.base == p.y && p.ldb == p.ldy && !p.h) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t adapter = max(t.adapter, 0);

    const int sub = lane & (kLanes - 1), group = lane / kLanes;
    const uint16_t* const b = p.b + adapter * p.N * p.R + min(sub * 8, p.R - 8);
    const int64_t end = min((int64_t)(blockIdx.y + 1) * p.columns, p.N);
    int64_t n0 = (int64_t)blockIdx.y * p.columns + wave * kAhead * kGroups;
    u32x4 bv[kAhead];
    float wide[kAhead][ROWS];
    auto load = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t n = min(n0 + u * kGroups + group, p.N - 1);
            bv[u] = *(const u32x4*)(b + n * p.R);
#pragma unroll
            for (int m = 0; m < ROWS; ++m) wide[u][m] = p.base ? wide_value((const T*)p.base + (t.row + min(m, t.rows - 1)) * p.ldb + n) : 0.f;
        }
    };
    load();

    float acc[RPW][ROWS];
#pragma unroll
    for (int r = 0; r < RPW; ++r)
#pragma unroll
        for (int m = 0; m < ROWS; ++m) acc[r][m] = 0.f;
    if (t.rank > 0) {
        constexpr int kBatch = RPW + ROWS <= 5 ? 3 : RPW + ROWS <= 12 ? 2 : 1;  // chunks of 512 whose loads go out together
        const uint16_t* x[ROWS];
        const uint16_t* a[RPW];
#pragma unroll
        for (int m = 0; m < ROWS; ++m) x[m] = p.x + (t.row + min(m, t.rows - 1)) * p.ldx;
#pragma unroll
        for (int r = 0; r < RPW; ++r) a[r] = p.a + (adapter * p.R + min(wave * RPW + r, t.rank - 1)) * p.K;
        for (int64_t k0 = 0; k0 < p.K; k0 += 512 * kBatch) {
            u32x4 xv[kBatch][ROWS], av[kBatch][RPW];
#pragma unroll
            for (int d = 0; d < kBatch; ++d) {
                const int64_t k = min(k0 + d * 512 + lane * 8, p.K - 8);
#pragma unroll
                for (int m = 0; m < ROWS; ++m) xv[d][m] = load8(x[m] + k);
#pragma unroll
                for (int r = 0; r < RPW; ++r) av[d][r] = *(const u32x4*)(a[r] + k);
            }
#pragma unroll
            for (int d = 0; d < kBatch; ++d) {
                const bool there = k0 + d * 512 + lane * 8 < p.K;
#pragma unroll
                for (int r = 0; r < RPW; ++r)
#pragma unroll
                    for (int m = 0; m < ROWS; ++m) {
                        float v = acc[r][m];
#pragma unroll
                        for (int e = 0; e < 4; ++e) v = dot2(av[d][r][e], xv[d][m][e], v);
                        acc[r][m] = there ? v : acc[r][m];
                    }
            }
        }
#pragma unroll
        for (int r = 0; r < RPW; ++r)
#pragma unroll
            for (int m = 0; m < ROWS; ++m) acc[r][m] = wave * RPW + r < t.rank ? sum_lanes<64>(acc[r][m]) : 0.f;
    }
#pragma unroll
    for (int r = 0; r < RPW; ++r)
#pragma unroll
        for (int m = 0; m < ROWS; ++m)
            if (lane == 0) hs[m][wave * RPW + r] = acc[r][m];
    __syncthreads();
    if (p.h && blockIdx.y == 0)
        for (int e = threadIdx.x; e < t.rows * p.R; e += 64 * kRowWaves) p.h[(int64_t)t.row * p.R + e] = hs[e / p.R][e % p.R];
    float h[ROWS][8];
#pragma unroll
    for (int m = 0; m < ROWS; ++m)
#pragma unroll
        for (int j = 0; j < 8; ++j) h[m][j] = sub * 8 + j < t.rank ? hs[m][sub * 8 + j] * t.scale : 0.f;

    while (n0 < end) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t n = n0 + u * kGroups + group;
            float v[ROWS];
#pragma unroll
            for (int m = 0; m < ROWS; ++m) v[m] = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // what lies beyond the rank need not be a number
                const float w = sub * 8 + j < t.rank ? (j & 1 ? bf16_high(bv[u][j / 2]) : bf16_low(bv[u][j / 2])) : 0.f;
#pragma unroll
                for (int m = 0; m < ROWS; ++m) v[m] += w * h[m][j];
            }
#pragma unroll
            for (int m = 0; m < ROWS; ++m) {
                const float y = wide[u][m] + sum_lanes<kLanes>(v[m]);
                if (sub == 0 && n < end && m < t.rows) set_wide((T*)p.y + (t.row + m) * p.ldy + n, y);
            }
        }
        n0 += kRowWaves * kAhead * kGroups;
        if (n0 < end) load();
    }
}

// What the backward pass reads the other way round: A [R][K] -> [K][R], B [N][R] -> [R][N padded to 8], and s h [M][R] as
// three bf16 parts in the order of lora_operand.  A thread turns a block of 8 x 8, and a workgroup is a wave: there are
// few, bound by latency, and more compute units have some (a training step of 9216 rows, 3072 -> 9216, rank 32: 204 us
// with workgroups of 256, 201.7 so; 230 where the kernels that use them turn them themselves).
__global__ __launch_bounds__(64) void lora_turn_kernel(LoraTurn p) {
    // (fewer than 2^31 blocks of 8 x 8 in all)
    const uint32_t r_blocks = p.R / 8, a_blocks = r_blocks * (uint32_t)(p.K / 8), b_blocks = r_blocks * (uint32_t)(p.ldn / 8);
    const uint32_t pools = (a_blocks + b_blocks) * p.adapters;
    uint32_t at = blockIdx.x * 64 + threadIdx.x;
    if (at < pools) {
        const uint32_t of = at / (a_blocks + b_blocks);
        at -= of * (a_blocks + b_blocks);
        const int64_t adapter = of;
        u32x4 v[8];
        if (at < a_blocks) {
            const int64_t k = at / r_blocks * 8, r = at % r_blocks * 8;
            const uint16_t* const from = p.a + (adapter * p.R + r) * p.K + k;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = *(const u32x4*)(from + j * p.K);
            transpose8(v);
            uint16_t* const to = p.at + (adapter * p.K + k) * p.R + r;
#pragma unroll
            for (int j = 0; j < 8; ++j) *(u32x4*)(to + j * p.R) = v[j];
        } else {
            at -= a_blocks;
            const uint32_t n_blocks = (uint32_t)(p.ldn / 8);
            const int64_t r = at / n_blocks * 8, n = at % n_blocks * 8;
            const uint16_t* const from = p.b + (adapter * p.N + n) * p.R + r;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = (u32x4){0, 0, 0, 0};
                if (n + j < p.N) v[j] = *(const u32x4*)(from + j * p.R);
            }
            transpose8(v);
            uint16_t* const to = p.bt + (adapter * p.R + r) * p.ldn + n;
#pragma unroll
            for (int j = 0; j < 8; ++j) *(u32x4*)(to + j * p.ldn) = v[j];
        }
        return;
    }
    at -= pools;
    const uint32_t tile = at / (8 * r_blocks);
    if (tile >= p.count) return;
    const LoraTile t = p.tiles[tile];
    const int in_tile = (int)(at - tile * 8 * r_blocks), first = in_tile % 8 * 8, r = in_tile / 8 * 8;
    if (first >= t.rows || t.rank == 0) return;
    float v[8][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float* const from = p.h + ((int64_t)t.row + min(first + j, t.rows - 1)) * p.R + r;
        const f32x4 lo = *(const f32x4*)from, hi = *(const f32x4*)(from + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e][j] = lo[e] * t.scale, v[e + 4][j] = hi[e] * t.scale;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        u32x4 part[kParts];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[e][j] = r + e < t.rank ? v[e][j] : 0.f;
        split8(v[e], part);
#pragma unroll
        for (int k = 0; k < kParts; ++k) *(u32x4*)(p.turned + lora_operand(tile, first, k, r + e, p.R)) = part[k];
    }
}

// Partial sums [split][R][width] over a split's rows of s narrow^T wide: of g and x (dA) in the first workgroups of a
// split, of h and dy (dB) in the rest.  A wave takes steps of 32 rows of 128 columns: a lane loads 8 rows of 8 columns,
// which transposed are 8 operands with the rows as contraction, each for columns 8 apart.  TOGETHER: the workgroup's waves
// take every fourth step of the same columns and add their sums in LDS; else they have columns of their own and store
// their sums themselves, which is faster where a wave has few steps.  Bound by HBM: 9216 rows, 3072 -> 9216, rank 32,
// 49 us (4.6 TB/s of x and dy).
template <int RF, bool TOGETHER>
__global__ __launch_bounds__(64 * kWaves) void lora_grad_kernel(LoraGrad p) {
    __shared__ float sums[TOGETHER ? RF * 16 : 1][128 + 4];
    const uint32_t index = blockIdx.x / (uint32_t)p.chunks;
    const int at_chunk = (int)(blockIdx.x - index * (uint32_t)p.chunks);
    const LoraSplit split = p.list[index];
    const bool second = at_chunk >= p.chunks_x;
    const LoraGradSide side = p.side[second];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, kg = lane >> 4;
    const int chunk = (at_chunk - (second ? p.chunks_x : 0)) * (TOGETHER ? 1 : kWaves) + (TOGETHER ? 0 : wave);
    if (!TOGETHER && (int64_t)chunk * 128 >= side.width) return;
    const int every = TOGETHER ? kWaves : 1;
    const int r0 = blockIdx.y * RF * 16;
    // a last chunk of fewer than 128 columns begins further left, among columns of the one before, which it leaves alone
    const int64_t n0 = min((int64_t)chunk * 128, max(side.width - 128, (int64_t)0)), col = n0 + c * 8;
    const int64_t left = side.width - col;
    const int skip = (int)((int64_t)chunk * 128 - n0);

    f32x4 acc[RF][8];
#pragma unroll
    for (int r = 0; r < RF; ++r)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[r][j] = (f32x4){0, 0, 0, 0};
    // two steps on their way; a load comes whether it is needed or not (the split's last step again), since after a branch
    // around one the compiler waits for all of them
    u32x4 z[2][8], part[2][RF][kParts];
    int mine[2], rows[2];  // the lane's first row of the step's tile, and the tile's rows
    auto load = [&](int d, int step, auto whole) __attribute__((always_inline)) {
        const LoraTile t = p.tiles[step / 2];
        mine[d] = (step & 1) * 32 + kg * 8;
        rows[d] = t.rows;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint16_t* const from = side.wide + ((int64_t)t.row + min(mine[d] + j, t.rows - 1)) * side.ld + col;
            z[d][j] = whole.value ? load8(from) : load8_part(from, left);
        }
#pragma unroll
        for (int r = 0; r < RF; ++r) {
            const int frag = min(r0 / 16 + r, (p.R - 1) / 16);
#pragma unroll
            for (int k = 0; k < kParts; ++k) part[d][r][k] = *(const u32x4*)(side.narrow + lora_operand(step / 2, (step & 1) * 32, k, frag * 16, p.R) + lane * 8);
        }
    };
    auto multiply = [&](int d, int step) __attribute__((always_inline)) {
        if ((step & 1) * 32 + 32 > rows[d]) {
            // rows beyond the tile are another's, or none
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (mine[d] + j >= rows[d]) z[d][j] = (u32x4){0, 0, 0, 0};
#pragma unroll
            for (int r = 0; r < RF; ++r)
#pragma unroll
                for (int k = 0; k < kParts; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        part[d][r][k][j] &= (mine[d] + 2 * j < rows[d] ? 0xFFFFu : 0u) | (mine[d] + 2 * j + 1 < rows[d] ? 0xFFFF0000u : 0u);
        }
        transpose8(z[d]);
#pragma unroll
        for (int r = 0; r < RF; ++r)
#pragma unroll
            for (int k = kParts - 1; k >= 0; --k)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[r][j] = mfma(part[d][r][k], z[d][j], acc[r][j]);
    };
    auto steps = [&](auto whole) __attribute__((always_inline)) {
        const int end = 2 * split.end;
        int step = 2 * split.begin + (TOGETHER ? wave : 0);
        if (step >= end) return;
        load(0, step, whole);
        load(1, min(step + every, end - 1), whole);
        for (; step < end; step += 2 * every) {
            multiply(0, step);
            load(0, min(step + 2 * every, end - 1), whole);
            if (step + every < end) multiply(1, step + every);
            load(1, min(step + 3 * every, end - 1), whole);
        }
    };
    if (side.width >= 128)
        steps(std::true_type{});
    else
        steps(std::false_type{});
    // a row of g or h beyond the rank is zero, and its sums are zero too where a value of x or dy is not finite
    const int rank = split.begin < split.end ? p.tiles[split.begin].rank : 0;
#pragma unroll
    for (int r = 0; r < RF; ++r)
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[r][j][k] = r0 + r * 16 + kg * 4 + k < rank ? acc[r][j][k] : 0.f;
    if (!TOGETHER) {
        // the lane has 8 columns in a row of rows q * 4 + k of each 16
#pragma unroll
        for (int r = 0; r < RF; ++r)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = r0 + r * 16 + kg * 4 + k;
                if (at >= p.R) continue;
                float* const to = side.part + ((int64_t)index * p.R + at) * side.width + col;
                if (left >= 8 && c * 8 >= skip) {
                    *(f32x4_any*)to = (f32x4){acc[r][0][k], acc[r][1][k], acc[r][2][k], acc[r][3][k]};
                    *(f32x4_any*)(to + 4) = (f32x4){acc[r][4][k], acc[r][5][k], acc[r][6][k], acc[r][7][k]};
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < left && c * 8 + j >= skip) to[j] = acc[r][j][k];
                }
            }
        return;
    }
    // the waves' sums, in order
    for (int w = 0; w < kWaves; ++w) {
        if (wave == w) {
#pragma unroll
            for (int r = 0; r < RF; ++r)
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float& to = sums[r * 16 + kg * 4 + k][c * 8 + j];
                        to = w ? to + acc[r][j][k] : acc[r][j][k];
                    }
        }
        __syncthreads();
    }
    if (p.direct && second) {
        // [width][R]
        for (int e = threadIdx.x; e < RF * 16 * 128; e += 64 * kWaves) {
            const int n = e / (RF * 16), r = e % (RF * 16);
            if (r0 + r < p.R && n0 + n < side.width && n >= skip) side.out[((int64_t)index * side.width + n0 + n) * p.R + r0 + r] = sums[r][n];
        }
        return;
    }
    float* const out = (p.direct ? side.out : side.part) + ((int64_t)index * p.R + r0) * side.width + n0;
    for (int e = threadIdx.x; e < RF * 16 * 128; e += 64 * kWaves) {
        const int r = e >> 7, n = e & 127;
        if (r0 + r < p.R && n0 + n < side.width && n >= skip) out[r * side.width + n] = sums[r][n];
    }
}

// Sums of an adapter's splits, in order (none: zeros): dA [R][K] as it lies, dB [R][N] turned to [N][R].  A thread takes
// 8 rows of r of one column, of four splits at a time (20480 rows, 3072 -> 3072, rank 16, a training step: 191 us, 195
// one after another and in workgroups of 256).
__global__ __launch_bounds__(64) void lora_grad_sum_kernel(LoraGrad p) {
    const int64_t adapter = blockIdx.z;
    const bool second = (int)blockIdx.x >= p.sum_blocks_x;
    const LoraGradSide side = p.side[second];
    const int64_t n = (int64_t)((int)blockIdx.x - (second ? p.sum_blocks_x : 0)) * 64 + threadIdx.x;
    const int r = blockIdx.y * 8;
    if (n >= side.width) return;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const int begin = p.first[adapter], end = p.first[adapter + 1];
#pragma unroll 4
    for (int s = begin; s < end; ++s) {
        const float* const from = side.part + ((int64_t)s * p.R + r) * side.width + n;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += from[j * side.width];
    }
    if (!second) {
        float* const to = side.out + (adapter * p.R + r) * side.width + n;
#pragma unroll
        for (int j = 0; j < 8; ++j) to[j * side.width] = v[j];
    } else {
        float* const to = side.out + (adapter * side.width + n) * p.R + r;
        *(f32x4*)to = (f32x4){v[0], v[1], v[2], v[3]};
        *(f32x4*)(to + 4) = (f32x4){v[4], v[5], v[6], v[7]};
    }
}

template <typename T>
void expand(const LoraExpand& p, dim3 grid, hipStream_t stream) {
    if (p.R <= 32)
        p.base ? lora_expand_kernel<T, 1, true><<<grid, 64 * kWaves, 0, stream>>>(p) : lora_expand_kernel<T, 1, false><<<grid, 64 * kWaves, 0, stream>>>(p);
    else if (p.R <= 64)
        p.base ? lora_expand_kernel<T, 2, true><<<grid, 64 * kWaves, 0, stream>>>(p) : lora_expand_kernel<T, 2, false><<<grid, 64 * kWaves, 0, stream>>>(p);
    else
        p.base ? lora_expand_kernel<T, 4, true><<<grid, 64 * kWaves, 0, stream>>>(p) : lora_expand_kernel<T, 4, false><<<grid, 64 * kWaves, 0, stream>>>(p);
}

template <typename T, int ROWS>
void rows(const LoraRows& p, dim3 grid, hipStream_t stream) {
    if (p.R <= 8)
        lora_rows_kernel<T, 1, ROWS><<<grid, 64 * kRowWaves, 0, stream>>>(p);
    else if (p.R <= 16)
        lora_rows_kernel<T, 2, ROWS><<<grid, 64 * kRowWaves, 0, stream>>>(p);
    else if (p.R <= 32)
        lora_rows_kernel<T, 4, ROWS><<<grid, 64 * kRowWaves, 0, stream>>>(p);
    else if (p.R <= 64)
        lora_rows_kernel<T, 8, ROWS><<<grid, 64 * kRowWaves, 0, stream>>>(p);
    else
        lora_rows_kernel<T, 16, ROWS><<<grid, 64 * kRowWaves, 0, stream>>>(p);
}

}  // namespace

int lora_splits(int tiles, int64_t K, int cus) {
    // halves of the K range until the workgroups are 2 to a compute unit, each keeping at least 6 chunks of 128: every
    // workgroup of the expansion reads all splits of its tile.  1024 rows 3072 -> 12288 of rank 32: 22.1 us, 25.9 with
    // splits down to one chunk, 29.4 with none below 24; 256 rows 13824 -> 5120 of rank 64: 20.6, 20.6 and 30.3.
    int splits = 1;
    while (splits < kLoraMaxSplits && (int64_t)tiles * splits < 2 * (int64_t)cus && K >= (int64_t)splits * 2 * 6 * 128) splits *= 2;
    return splits;
}

hipError_t launch_lora_shrink(LoraShrink p, int tiles, int splits, hipStream_t stream) {
    const int64_t steps = (p.K + 127) / 128;
    p.steps = (int)((steps + splits - 1) / splits);
    const dim3 grid(tiles, splits);
    if (p.R <= 16)
        lora_shrink_kernel<1><<<grid, 64 * kWaves, 0, stream>>>(p);
    else if (p.R <= 32)
        lora_shrink_kernel<2><<<grid, 64 * kWaves, 0, stream>>>(p);
    else if (p.R <= 64)
        lora_shrink_kernel<4><<<grid, 64 * kWaves, 0, stream>>>(p);
    else
        lora_shrink_kernel<8><<<grid, 64 * kWaves, 0, stream>>>(p);
    return hipGetLastError();
}

hipError_t launch_lora_expand(LoraExpand p, int tiles, bool f32, int cus, hipStream_t stream) {
    // 512 columns to a workgroup, fewer where that leaves less than 4 workgroups to a compute unit (2 or 8: the same to 1%).
    // 9216 rows, 9216 columns in bf16, rank 32: 86 us, 90 with 256 columns, 108 with 128, 87 with 1024; 33272 rows, 13824
    // columns in fp32, rank 64: 761, 768, 845 and 788.
    p.columns = 512;
    while (p.columns > 128 && tiles * ((p.N + p.columns - 1) / p.columns) < 4 * (int64_t)cus) p.columns /= 2;
    // a grid holds fewer than 2^32 threads: more columns to a workgroup where many short requests would pass that
    while ((tiles + 7) / 8 * 8 * ((p.N + p.columns - 1) / p.columns) >= ((int64_t)1 << 32) / (64 * kWaves)) p.columns *= 2;
    // Non-temporal stores leave the caches to what is read next (a training step with 170 MB of y 232 -> 213 us, a call with
    // 1.8 GB 841 -> 818, small ones the same), where rows are whole lines: 144 MB of rows of 13424 bytes took 69 us, 48 with
    // plain stores.
    const int size = f32 ? 4 : 2;
    p.stream = (uintptr_t)p.y % 128 == 0 && p.ldy * size % 128 == 0;
    p.count = tiles;
    p.blocks = (int)((p.N + p.columns - 1) / p.columns);
    const dim3 grid((unsigned)((tiles + 7) / 8 * 8 * p.blocks));
    f32 ? expand<float>(p, grid, stream) : expand<bf16_t>(p, grid, stream);
    return hipGetLastError();
}

hipError_t launch_lora_rows(LoraRows p, int tiles, int tile_rows, bool f32, int cus, hipStream_t stream) {
    // a workgroup to a compute unit, but no fewer columns than its waves take at once
    int lanes = 1;
    while (lanes * 8 < p.R) lanes *= 2;
    const int64_t once = kRowWaves * kAhead * (64 / lanes), most = (p.N + once - 1) / once;
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>(most, (cus + tiles - 1) / tiles));
    p.columns = (int)((most + blocks - 1) / blocks * once);
    const dim3 grid(tiles, (unsigned)((p.N + p.columns - 1) / p.columns));
    if (tile_rows <= 1)
        f32 ? rows<float, 1>(p, grid, stream) : rows<bf16_t, 1>(p, grid, stream);
    else
        f32 ? rows<float, kLoraFewRows>(p, grid, stream) : rows<bf16_t, kLoraFewRows>(p, grid, stream);
    return hipGetLastError();
}

hipError_t launch_lora_turn(const LoraTurn& p, hipStream_t stream) {
    const int64_t blocks = (int64_t)(p.R / 8) * ((p.K / 8 + p.ldn / 8) * p.adapters + 8 * p.count);
    lora_turn_kernel<<<(unsigned)((blocks + 63) / 64), 64, 0, stream>>>(p);
    return hipGetLastError();
}

hipError_t launch_lora_grad(LoraGrad p, int splits, int adapters, bool together, hipStream_t stream) {
    const int each = together ? 128 : 128 * kWaves;
    p.chunks_x = (int)((p.side[0].width + each - 1) / each);
    p.chunks = p.chunks_x + (int)((p.side[1].width + each - 1) / each);
    if (splits > 0) {
        const dim3 grid((unsigned)(p.chunks * splits), p.R > 64 ? 2 : 1);
        if (p.R <= 16)
            together ? lora_grad_kernel<1, true><<<grid, 64 * kWaves, 0, stream>>>(p) : lora_grad_kernel<1, false><<<grid, 64 * kWaves, 0, stream>>>(p);
        else if (p.R <= 32)
            together ? lora_grad_kernel<2, true><<<grid, 64 * kWaves, 0, stream>>>(p) : lora_grad_kernel<2, false><<<grid, 64 * kWaves, 0, stream>>>(p);
        else
            together ? lora_grad_kernel<4, true><<<grid, 64 * kWaves, 0, stream>>>(p) : lora_grad_kernel<4, false><<<grid, 64 * kWaves, 0, stream>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || p.direct) return e;
    }
    p.sum_blocks_x = (int)((p.side[0].width + 63) / 64);
    const int sums = p.sum_blocks_x + (int)((p.side[1].width + 63) / 64);
    lora_grad_sum_kernel<<<dim3(sums, p.R / 8, adapters), 64, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace orbit
