// Low-rank adapters of many requests beside the projection they share, forward and backward, for gfx950.
//
// Rows m of one request use one adapter a, of rank r <= R and scale s:
//     h = x A_a^T,  y = base + s h B_a^T                                    (A_a [R][K], B_a [N][R], bf16)
// and with g = dy B_a
//     dx = s g A_a,  dA_a = s sum over its rows of g^T x,  dB_a = s sum over its rows of dy^T h.
// At ranks up to 128 all of it is bound by the wide matrices x, base, y, dy and dx, each of which a kernel streams once:
//   shrink  h (or g): a wide matrix times a narrow one, contraction over the wide side
//   expand  y (or dx): a narrow matrix times a narrow one, added to the wide base on its way through the registers
//   grad    dA, dB: contraction over rows, of a wide matrix and a narrow one
// The matrix cores multiply bf16.  x, dy, A and B are bf16 and their products exact; h and g are fp32 sums and go into
// the next product as the sum of two bf16 values (16 bits of their fraction: 2^-17 of them is lost, where one bf16 would
// lose 2^-9), which costs a second MFMA and no memory traffic.
//
// A tile is up to 64 rows of one adapter; the plan lists them.  MFMA operands come straight from memory: a lane holds 8
// values in a row of the contraction for row (or column) lane % 16, so a wave's load covers 16 rows of 64 bytes.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "device.h"
#include "vec.h"

namespace orbit {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// 16 bytes of bf16 at any element: rows of odd length begin anywhere
struct __attribute__((packed, aligned(2))) Unaligned16 {
    u32x4 v;
};
struct __attribute__((packed, aligned(4))) Unaligned16f {
    f32x4 v;
};

__device__ __forceinline__ u32x4 load8(const uint16_t* p) { return ((const Unaligned16*)p)->v; }

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

// v as hi + lo, both bf16
__device__ __forceinline__ void split8(const float* v, u32x4& hi, u32x4& lo) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        hi[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        lo[i] = pack_bf16(rest(v[2 * i], bf16_low(hi[i])), rest(v[2 * i + 1], bf16_high(hi[i])));
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

// h partial sums [split][M][R] of rows x [M][K] and pool [adapter][R][K]: a workgroup takes 16 MT rows of a tile and a
// split of K, its waves a quarter of that each.
template <int MT, int RF>
__global__ __launch_bounds__(64 * kWaves) void lora_shrink_kernel(LoraShrink p) {
    constexpr int kSub = 4 / MT;
    __shared__ float part[kWaves][MT * 16][RF * 16 + (RF < 8 ? 1 : 0)];  // at most 64 KB
    const LoraTile t = p.tiles[blockIdx.x / kSub];
    const int first = (int)(blockIdx.x % kSub) * MT * 16;
    if (first >= t.rows) return;
    const int rows = min(t.rows - first, MT * 16);
    const int64_t row0 = t.row + first;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, kg = lane >> 4;

    f32x4 acc[MT][RF];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < RF; ++r) acc[m][r] = (f32x4){0, 0, 0, 0};
    if (t.rank > 0) {
        const uint16_t* x[MT];
        const uint16_t* a[RF];
        bool live[RF];
#pragma unroll
        for (int m = 0; m < MT; ++m) x[m] = p.x + (row0 + min(m * 16 + i, rows - 1)) * p.ldx + kg * 8;
#pragma unroll
        for (int r = 0; r < RF; ++r) {
            live[r] = r * 16 + i < t.rank;
            a[r] = p.pool + ((int64_t)t.adapter * p.R + (live[r] ? r * 16 + i : 0)) * p.ldp + kg * 8;
        }
        const int64_t begin = ((int64_t)blockIdx.y * kWaves + wave) * p.steps * 32;
        const int64_t end = min(begin + (int64_t)p.steps * 32, p.K);
        const int whole = (int)(max(end - begin, (int64_t)0) / 32);
        int64_t k = begin;
#pragma unroll 4
        for (int step = 0; step < whole; ++step, k += 32) {
            u32x4 xv[MT], av[RF];
#pragma unroll
            for (int m = 0; m < MT; ++m) xv[m] = load8(x[m] + k);
#pragma unroll
            for (int r = 0; r < RF; ++r) {
                av[r] = *(const u32x4*)(a[r] + k);
                if (!live[r]) av[r] = (u32x4){0, 0, 0, 0};
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < RF; ++r) acc[m][r] = mfma(xv[m], av[r], acc[m][r]);
        }
        if (k < end) {
            // the last, partial step; the pool's rows are padded to 8 values
            const int64_t left = end - k - kg * 8;
            u32x4 xv[MT], av[RF];
#pragma unroll
            for (int m = 0; m < MT; ++m) xv[m] = load8_part(x[m] + k, left);
#pragma unroll
            for (int r = 0; r < RF; ++r) {
                av[r] = (u32x4){0, 0, 0, 0};
                if (live[r] && left > 0) av[r] = *(const u32x4*)(a[r] + k);
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < RF; ++r) acc[m][r] = mfma(xv[m], av[r], acc[m][r]);
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < RF; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) part[wave][m * 16 + kg * 4 + j][r * 16 + i] = acc[m][r][j];
    __syncthreads();
    float* const out = p.h + ((int64_t)blockIdx.y * p.M + row0) * p.R;
    for (int e = threadIdx.x; e < rows * p.R; e += 64 * kWaves) {
        const int m = e / p.R, r = e - m * p.R;
        // a row of x that is not finite times the rank's missing rows of A is nothing all the same
        out[e] = r < t.rank ? (part[0][m][r] + part[1][m][r]) + (part[2][m][r] + part[3][m][r]) : 0.f;
    }
}

// Eight values of a row of the wide output or of its base.
template <typename T>
__device__ __forceinline__ void load_wide(const T* p, int64_t n, float* v);
template <>
__device__ __forceinline__ void load_wide<bf16_t>(const bf16_t* p, int64_t n, float* v) {
    const u32x4 w = load8_part((const uint16_t*)p, n);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16_low(w[i]), v[2 * i + 1] = bf16_high(w[i]);
}
template <>
__device__ __forceinline__ void load_wide<float>(const float* p, int64_t n, float* v) {
    if (n >= 8) {
        const f32x4 a = ((const Unaligned16f*)p)->v, b = ((const Unaligned16f*)(p + 4))->v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = a[i], v[i + 4] = b[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
    }
}

__device__ __forceinline__ void store_wide(bf16_t* p, int64_t n, const float* v) {
    const u32x4 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    if (n >= 8) {
        ((Unaligned16*)p)->v = w;
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) p[i].bits = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
    }
}
__device__ __forceinline__ void store_wide(float* p, int64_t n, const float* v) {
    if (n >= 8) {
        ((Unaligned16f*)p)->v = (f32x4){v[0], v[1], v[2], v[3]};
        ((Unaligned16f*)(p + 4))->v = (f32x4){v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) p[i] = v[i];
    }
}

// y = base + s h B^T for a tile's rows and `strips` strips of 64 columns to each wave.  The MFMA's rows are columns of y
// and its columns rows of y, so a lane ends up with values of one row; its fragments take the columns in the order that
// makes them 8 in a row.  The pool is [adapter][N][R].
template <typename T, int RC>
__global__ __launch_bounds__(64 * kWaves) void lora_expand_kernel(LoraExpand p) {
    const LoraTile t = p.tiles[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    if (t.rank == 0 && p.base == p.y && p.ldb == p.ldy) return;
    const int frags = (t.rows + 15) / 16;
    u32x4 hi[4][RC], lo[4][RC], mask[RC];
#pragma unroll
    for (int c = 0; c < RC; ++c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = c * 32 + q * 8 + 2 * j;
            mask[c][j] = (r < t.rank ? 0xFFFFu : 0u) | (r + 1 < t.rank ? 0xFFFF0000u : 0u);
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            if (m >= frags) break;
            const int row = min(m * 16 + i, t.rows - 1), r = c * 32 + q * 8;
            float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (r < p.R) {
                const float* from = p.h + ((int64_t)t.row + row) * p.R + r;
                for (int s = 0; s < p.splits; ++s, from += p.M * p.R) {
                    const f32x4 a = *(const f32x4*)from, b = *(const f32x4*)(from + 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] += a[j], v[j + 4] += b[j];
                }
                if (p.sum && blockIdx.y == 0 && wave == 0 && m * 16 + i < t.rows) {
                    float* const to = p.sum + ((int64_t)t.row + row) * p.R + r;
                    *(f32x4*)to = (f32x4){v[0], v[1], v[2], v[3]};
                    *(f32x4*)(to + 4) = (f32x4){v[4], v[5], v[6], v[7]};
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= t.scale;
            split8(v, hi[m][c], lo[m][c]);
        }
    }
    const uint16_t* const pool = p.pool + (int64_t)max(t.adapter, 0) * p.N * p.R;
    for (int s = 0; s < p.strips; ++s) {
        const int64_t n0 = (((int64_t)blockIdx.y * p.strips + s) * kWaves + wave) * 64;
        if (n0 >= p.N) break;
        // fragment f = 2 pair + half: its row i is column n0 + 32 pair + 8 (i / 4) + 4 half + i % 4
        f32x4 acc[4][4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            if (m >= frags) break;
            const int64_t row = t.row + min(m * 16 + i, t.rows - 1);
#pragma unroll
            for (int pair = 0; pair < 2; ++pair) {
                const int64_t n = n0 + 32 * pair + 8 * q;
                float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                if (p.base && n < p.N) load_wide<T>((const T*)p.base + row * p.ldb + n, p.N - n, v);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[m][2 * pair][j] = v[j], acc[m][2 * pair + 1][j] = v[j + 4];
            }
        }
        if (t.rank > 0) {
            u32x4 b[4][RC];
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const int64_t n = min(n0 + 32 * (f / 2) + 8 * (i / 4) + 4 * (f & 1) + i % 4, p.N - 1);
#pragma unroll
                for (int c = 0; c < RC; ++c) {
                    const int r = c * 32 + q * 8;
                    b[f][c] = *(const u32x4*)(pool + n * p.R + (r < p.R ? r : 0)) & mask[c];
                }
            }
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                if (m >= frags) break;
#pragma unroll
                for (int f = 0; f < 4; ++f)
#pragma unroll
                    for (int c = 0; c < RC; ++c) {
                        acc[m][f] = mfma(b[f][c], lo[m][c], acc[m][f]);
                        acc[m][f] = mfma(b[f][c], hi[m][c], acc[m][f]);
                    }
            }
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            if (m >= frags || m * 16 + i >= t.rows) break;
            const int64_t row = t.row + m * 16 + i;
#pragma unroll
            for (int pair = 0; pair < 2; ++pair) {
                const int64_t n = n0 + 32 * pair + 8 * q;
                float v[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = acc[m][2 * pair][j], v[j + 4] = acc[m][2 * pair + 1][j];
                if (n < p.N) store_wide((T*)p.y + row * p.ldy + n, p.N - n, v);
            }
        }
    }
}

// Pools with the other side contiguous, for the backward pass: A [R][K] -> [K][R], B [N][R] -> [R][N padded to 8].  A
// thread turns a block of 8 x 8.
__global__ __launch_bounds__(256) void lora_transpose_kernel(LoraTranspose p) {
    const int64_t a_blocks = (int64_t)(p.R / 8) * (p.K / 8), b_blocks = (int64_t)(p.R / 8) * (p.ldt / 8);
    int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t adapter = blockIdx.y;
    u32x4 v[8];
    if (at < a_blocks) {
        const int r = (int)(at % (p.R / 8)) * 8;
        const int64_t k = at / (p.R / 8) * 8;
        const uint16_t* const from = p.a + adapter * p.R * p.K + r * p.K + k;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = *(const u32x4*)(from + j * p.K);
        transpose8(v);
        uint16_t* const to = p.at + adapter * p.R * p.K + k * p.R + r;
#pragma unroll
        for (int j = 0; j < 8; ++j) *(u32x4*)(to + j * p.R) = v[j];
        return;
    }
    at -= a_blocks;
    if (at >= b_blocks) return;
    const int64_t n = at % (p.ldt / 8) * 8;
    const int r = (int)(at / (p.ldt / 8)) * 8;
    const uint16_t* const from = p.b + adapter * p.N * p.R + n * p.R + r;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[j] = (u32x4){0, 0, 0, 0};
        if (n + j < p.N) v[j] = *(const u32x4*)(from + j * p.R);
    }
    transpose8(v);
    uint16_t* const to = p.bt + (adapter * p.R + r) * p.ldt + n;
#pragma unroll
    for (int j = 0; j < 8; ++j) *(u32x4*)(to + j * p.ldt) = v[j];
}

// Partial sums [split][R][width] over a split's rows of s narrow^T wide: of g and x (dA) in the first workgroups of a
// split, of h and dy (dB) in the rest.  A wave takes every fourth step of 32 rows of 128 columns: a lane loads
// 8 rows of 8 columns, which transposed are 8 operands with the rows as contraction, each for columns 8 apart.
template <int RF>
__global__ __launch_bounds__(64 * kWaves) void lora_grad_kernel(LoraGrad p) {
    __shared__ float part[RF * 16][128 + 4];
    const uint32_t index = blockIdx.x / (uint32_t)p.chunks;
    const int at_chunk = (int)(blockIdx.x - index * (uint32_t)p.chunks);
    const LoraSplit split = p.list[index];
    const bool second = at_chunk >= p.chunks_x;
    const LoraGradSide side = p.side[second];
    const int chunk = at_chunk - (second ? p.chunks_x : 0);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, kg = lane >> 4;
    const int r0 = blockIdx.y * RF * 16;
    const int64_t col = (int64_t)chunk * 128 + c * 8;
    const int64_t left = side.width - col;

    f32x4 acc[RF][8];
#pragma unroll
    for (int r = 0; r < RF; ++r)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[r][j] = (f32x4){0, 0, 0, 0};
    for (int step = 2 * split.begin + wave; step < 2 * split.end; step += kWaves) {
        const LoraTile t = p.tiles[step / 2];
        const int first = (step & 1) * 32 + kg * 8;  // this lane's rows of the tile
        u32x4 z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            z[j] = (u32x4){0, 0, 0, 0};
            if (first + j < t.rows) z[j] = load8_part(side.wide + ((int64_t)t.row + first + j) * side.ld + col, left);
        }
        u32x4 hi[RF], lo[RF];
#pragma unroll
        for (int r = 0; r < RF; ++r) {
            const int at = r0 + r * 16 + c;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = 0.f;
                if (first + j < t.rows && at < t.rank) v[j] = side.narrow[((int64_t)t.row + first + j) * p.R + at] * t.scale;
            }
            split8(v, hi[r], lo[r]);
        }
        transpose8(z);
#pragma unroll
        for (int r = 0; r < RF; ++r)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                acc[r][j] = mfma(lo[r], z[j], acc[r][j]);
                acc[r][j] = mfma(hi[r], z[j], acc[r][j]);
            }
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
                        float& to = part[r * 16 + kg * 4 + k][c * 8 + j];
                        to = w ? to + acc[r][j][k] : acc[r][j][k];
                    }
        }
        __syncthreads();
    }
    float* const out = side.part + ((int64_t)index * p.R + r0) * side.width;
    for (int e = threadIdx.x; e < RF * 16 * 128; e += 64 * kWaves) {
        const int r = e >> 7, n = e & 127;
        if (r0 + r < p.R && (int64_t)chunk * 128 + n < side.width) out[r * side.width + (int64_t)chunk * 128 + n] = part[r][n];
    }
}

// Sums of an adapter's splits, in order (none: zeros): dA [R][K] as it lies, dB [R][N] turned to [N][R].  A thread takes
// 8 rows of r of one column.
__global__ __launch_bounds__(256) void lora_grad_sum_kernel(LoraGrad p) {
    const int64_t adapter = blockIdx.z;
    const bool second = (int)blockIdx.x >= p.sum_blocks_x;
    const LoraGradSide side = p.side[second];
    const int64_t n = (int64_t)((int)blockIdx.x - (second ? p.sum_blocks_x : 0)) * 256 + threadIdx.x;
    const int r = blockIdx.y * 8;
    if (n >= side.width) return;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const int begin = p.first[adapter], end = p.first[adapter + 1];
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

template <int MT>
void shrink(const LoraShrink& p, dim3 grid, hipStream_t stream) {
    if (p.R <= 16)
        lora_shrink_kernel<MT, 1><<<grid, 64 * kWaves, 0, stream>>>(p);
    else if (p.R <= 32)
        lora_shrink_kernel<MT, 2><<<grid, 64 * kWaves, 0, stream>>>(p);
    else if (p.R <= 64)
        lora_shrink_kernel<MT, 4><<<grid, 64 * kWaves, 0, stream>>>(p);
    else
        lora_shrink_kernel<MT, 8><<<grid, 64 * kWaves, 0, stream>>>(p);
}

template <typename T>
void expand(const LoraExpand& p, dim3 grid, hipStream_t stream) {
    if (p.R <= 32)
        lora_expand_kernel<T, 1><<<grid, 64 * kWaves, 0, stream>>>(p);
    else if (p.R <= 64)
        lora_expand_kernel<T, 2><<<grid, 64 * kWaves, 0, stream>>>(p);
    else
        lora_expand_kernel<T, 4><<<grid, 64 * kWaves, 0, stream>>>(p);
}

}  // namespace

int lora_splits(int tiles, int64_t K, int cus) {
    // halves of the K range until the waves of two-row-fragment workgroups are 8 to a compute unit, a wave keeping
    // at least 4 steps of 32
    int splits = 1;
    while (splits < kLoraMaxSplits && (int64_t)tiles * 2 * kWaves * splits < 8 * (int64_t)cus && K >= (int64_t)splits * 2 * kWaves * 4 * 32)
        splits *= 2;
    return splits;
}

hipError_t launch_lora_shrink(LoraShrink p, int tiles, int splits, hipStream_t stream) {
    const int64_t steps = (p.K + 31) / 32;
    p.steps = (int)((steps + splits * kWaves - 1) / (splits * kWaves));
    shrink<2>(p, dim3(tiles * 2, splits), stream);
    return hipGetLastError();
}

hipError_t launch_lora_expand(LoraExpand p, int tiles, bool f32, int cus, hipStream_t stream) {
    // four strips to a wave where that leaves 4 workgroups to a compute unit
    const int64_t blocks = (p.N + 64 * kWaves - 1) / (64 * kWaves);
    p.strips = (int)std::max<int64_t>(1, std::min<int64_t>(4, tiles * blocks / (4 * (int64_t)cus)));
    const dim3 grid(tiles, (unsigned)((blocks + p.strips - 1) / p.strips));
    f32 ? expand<float>(p, grid, stream) : expand<bf16_t>(p, grid, stream);
    return hipGetLastError();
}

hipError_t launch_lora_transpose(const LoraTranspose& p, int adapters, hipStream_t stream) {
    const int64_t blocks = (int64_t)(p.R / 8) * (p.K / 8 + p.ldt / 8);
    lora_transpose_kernel<<<dim3((unsigned)((blocks + 255) / 256), adapters), 256, 0, stream>>>(p);
    return hipGetLastError();
}

hipError_t launch_lora_grad(LoraGrad p, int splits, int adapters, hipStream_t stream) {
    p.chunks_x = (int)((p.side[0].width + 127) / 128);
    p.chunks = p.chunks_x + (int)((p.side[1].width + 127) / 128);
    if (splits > 0) {
        const dim3 grid((unsigned)(p.chunks * splits), p.R > 64 ? 2 : 1);
        if (p.R <= 16)
            lora_grad_kernel<1><<<grid, 64 * kWaves, 0, stream>>>(p);
        else if (p.R <= 32)
            lora_grad_kernel<2><<<grid, 64 * kWaves, 0, stream>>>(p);
        else
            lora_grad_kernel<4><<<grid, 64 * kWaves, 0, stream>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    p.sum_blocks_x = (int)((p.side[0].width + 255) / 256);
    const int sums = p.sum_blocks_x + (int)((p.side[1].width + 255) / 256);
    lora_grad_sum_kernel<<<dim3(sums, p.R / 8, adapters), 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace orbit
