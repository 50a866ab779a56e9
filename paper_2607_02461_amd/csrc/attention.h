// What the attention kernels share: tiles of rows in LDS, and the matrix cores' operands from them.
//
// The matrix cores multiply 32 x 16 by 16 x 32 bf16 values.  Lane l of a wave holds of either operand the 8 values 8 (l / 32) ..
// of row (or column) l % 32, and of the result column l % 32 at rows 8 a + 4 (l / 32) + c, register 4 a + c.  Scores are computed
// transposed, keys x queries, so that a lane holds one query's scores (of 16 keys of each 32): its maximum and its sum are
// sums over registers, and the probabilities are an operand of the next product as they lie, without a value changing its lane.
// That product's order of keys is then 8 a + 4 (l / 32) + c, in the other operand too: V (or K, Q, dO), whose values of one
// column it needs, is read from LDS by ds_read_b64_tr_b16, which turns 4 rows x 16 columns for 16 lanes.
//
// DP: the head size, padded to a multiple of 32 (of the products' columns).  A tile of rows lies in LDS as it does in memory, 128 or
// 256 bytes to a row, its 16-byte chunks in an order that differs from row to row (`swizzled`): both ways of reading find their
// rows in different banks (no conflict is counted).  Lanes load the chunks in that order (global_load_lds: lane i's 16 bytes go to
// the wave's place + 16 i).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "device.h"
#include "vec.h"

namespace orbit {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

#define ORBIT_LDS __attribute__((address_space(3)))

__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)(const ORBIT_LDS char*)p; }

constexpr float kLowest = -3.0e38f;   // stands for the largest of no scores
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ f32x16 mfma32(const u32x4& a, const u32x4& b, const f32x16& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// The other half-wave's value
__device__ __forceinline__ float other_half(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

template <int DP>
constexpr int kRowBytes = DP > 64 ? 256 : 128;   // of a row in LDS

// Chunk c of a row, as it lies in the tile.  16 rows in a row have one chunk in 16 places of the 256 bytes that LDS serves in a
// clock, and 4 rows that begin at a multiple of 4 have 64 bytes each in different ones.
template <int DP>
__device__ __forceinline__ int swizzled(int row, int c) {
    if (DP > 64) return c ^ ((row & 3) << 2 | (row >> 2 & 3));
    return c ^ ((row >> 1 & 1) << 2 | (row >> 2 & 3));
}

// A wave's share of tiles of ROWS rows of one tensor, of WAVES waves.  A load takes 64 chunks, lane by lane: the lanes' offsets from
// a tile's first row stay in registers and the row itself is a scalar.  (With 64-bit addresses for each load their products were
// 400 cycles of a tile's 1024.)  Columns behind D are other columns of the row: the other operand has zeros there.
//
// The loads are inline asm because the compiler, which cannot tell the buffers apart, would wait for them before the next read of
// LDS.  They have no output registers; loads_done() waits for them.  m0 is not in their list of clobbers because the compiler reserves
// it and warns of its name there; nothing else in these kernels may use it.
template <int DP, int ROWS, int WAVES>
struct TileLoads {
    static constexpr int kChunks = kRowBytes<DP> / 16, kEach = 64 / kChunks, kLoads = ROWS / kEach / WAVES;
    const char* rows;       // the sequence's first row
    int64_t stride;         // bytes
    uint32_t from[kLoads];  // bytes from a tile's first row
    uint32_t to;            // the wave's place in a tile
    int last;               // row of the sequence
    __device__ __forceinline__ TileLoads(const uint16_t* t, int64_t stride, int last, int D, int wave, int lane)
        : rows((const char*)t), stride(2 * stride), to(wave * kLoads * 1024), last(last) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) from[i] = (uint32_t)(row_of(i, lane) * this->stride) + column_of(i, lane, D);
    }
    __device__ __forceinline__ int row_of(int i, int lane) const { return (int)(to / 1024 + i) * kEach + lane / kChunks; }
    __device__ __forceinline__ uint32_t column_of(int i, int lane, int D) const {
        const int c = swizzled<DP>(row_of(i, lane), lane % kChunks);
        return 8 * c >= D ? 0 : 16 * c;
    }
    // rows first .. into the tile; those behind the last one are the last one
    __device__ __forceinline__ void load(int first, char* tile, int D, int lane) const {
        const uint32_t lds = lds_address(tile) + to;
        const char* const base = rows + first * stride;
        if (first + ROWS <= last + 1) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) one(base, from[i], lds + 1024 * i);
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                one(base, (uint32_t)(min(row_of(i, lane), last - first) * stride) + column_of(i, lane, D), lds + 1024 * i);
        }
    }
    static __device__ __forceinline__ void one(const char* base, uint32_t from, uint32_t lds) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(from), "s"(base) : "memory");
    }
};

// Waits until at most LEFT of the wave's loads are on their way (the builtin, so that the compiler knows that its own loads before
// a loop have arrived and does not wait for them in it)
template <int LEFT = 0>
__device__ __forceinline__ void loads_done() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (LEFT & 15) | (LEFT >> 4) << 14);
    asm volatile("" ::: "memory");
}

// Waits for the wave's reads of LDS: a tile may be loaded over another that the wave alone has read (where waves share it, a
// barrier does)
__device__ __forceinline__ void reads_done() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    asm volatile("" ::: "memory");
}

// Where a lane reads operands of a tile: rows of it (row l % 32 of 32, chunk l / 32 of each pair), and columns of it.  A chunk's
// place is an exclusive or of its number and the row's, so the other places are one such operation from the first.
template <int DP>
struct Operands {
    int row, column;   // bytes: of chunk l / 32 of the lane's row, and of the lane's 4 values in columns 0 .. 31 of rows 4 (l / 32) ..
    __device__ __forceinline__ explicit Operands(int lane) {
        const int r = lane & 31, half = lane >> 5, i = lane & 15, key = 4 * half + (i >> 2), d = 16 * (lane >> 4 & 1) + 4 * (i & 3);
        row = r * kRowBytes<DP> + 16 * swizzled<DP>(r, half);
        column = key * kRowBytes<DP> + 16 * swizzled<DP>(key, d / 8) + 2 * (d & 7);
    }
    // The same of tiles that lie `bytes` further in LDS, a multiple of a row's: an address then is an exclusive or and a constant
    __device__ __forceinline__ Operands further(uint32_t bytes) const {
        Operands other = *this;
        other.row += bytes;
        other.column += bytes;
        return other;
    }
    // rows 32 block .. of the tile, k-step s
    __device__ __forceinline__ u32x4 rows_of(uint32_t tile, int block, int s) const {
        return *(const ORBIT_LDS u32x4*)(uintptr_t)(tile + block * 32 * kRowBytes<DP> + (row ^ 32 * s));
    }
    __device__ __forceinline__ u32x4 rows_of(const char* tile, int block, int s) const { return rows_of(lds_address(tile), block, s); }
    // columns 32 b .., rows 16 step .. of the tile, 8 a + 4 (l / 32) .. of them
    __device__ __forceinline__ u32x4 columns_of(const char* tile, int step, int b) const { return columns_of(lds_address(tile), step, b); }
    __device__ __forceinline__ u32x4 columns_of(uint32_t tile, int step, int b) const {
        const uint32_t at = tile + step * 16 * kRowBytes<DP>;
        auto four = [&](int a) {
            return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                 (ORBIT_LDS s16x4*)(uintptr_t)(at + 8 * kRowBytes<DP> * a + (column ^ (64 * b | 32 * a)))));
        };
        const u32x2 lo = four(0), hi = four(1);
        return (u32x4){lo.x, lo.y, hi.x, hi.y};
    }
};

// Values 8 .. of a row of D for the lane's operand of each k-step, zeros behind D
template <int DP>
__device__ __forceinline__ void load_operand(const uint16_t* row, int D, int lane, u32x4 (&v)[DP / 16]) {
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        const int d = 16 * s + 8 * (lane >> 5);
        v[s] = d < D ? *(const u32x4*)(row + d) : (u32x4){0, 0, 0, 0};
    }
}

// Registers 8 u .. of a result as an operand of k-step u
__device__ __forceinline__ u32x4 as_operand(const f32x16& v, int u) {
    return (u32x4){pack_bf16(v[8 * u], v[8 * u + 1]), pack_bf16(v[8 * u + 2], v[8 * u + 3]), pack_bf16(v[8 * u + 4], v[8 * u + 5]),
                   pack_bf16(v[8 * u + 6], v[8 * u + 7])};
}

// A lane's column of a transposed result, [D x columns]: 32 b + 8 a + 4 (l / 32) + c, to the column's row of D values.  The
// half-waves trade registers, so that each lane stores 8 bf16 values in a row.
template <int DP>
__device__ __forceinline__ void store_column(const f32x16 (&v)[DP / 32], float factor, uint16_t* row, int D, int lane, bool live) {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int a = 0; a < 4; a += 2) {
            u32x2 x = {pack_bf16(v[b][4 * a] * factor, v[b][4 * a + 1] * factor), pack_bf16(v[b][4 * a + 2] * factor, v[b][4 * a + 3] * factor)};
            u32x2 y = {pack_bf16(v[b][4 * a + 4] * factor, v[b][4 * a + 5] * factor), pack_bf16(v[b][4 * a + 6] * factor, v[b][4 * a + 7] * factor)};
            const auto s = __builtin_amdgcn_permlane32_swap(x.x, y.x, false, false), t = __builtin_amdgcn_permlane32_swap(x.y, y.y, false, false);
            const int d = 32 * b + 8 * (a + (lane >> 5));
            if (live && d < D) *(u32x4*)(row + d) = (u32x4){s[0], t[0], s[1], t[1]};
        }
}

template <int DP>
__device__ __forceinline__ void store_column_f32(const f32x16 (&v)[DP / 32], float factor, float* row, int D, int lane, bool live) {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const int d = 32 * b + 8 * a + 4 * (lane >> 5);
            if (live && d < D)
                *(f32x4*)(row + d) = (f32x4){v[b][4 * a] * factor, v[b][4 * a + 1] * factor, v[b][4 * a + 2] * factor, v[b][4 * a + 3] * factor};
        }
}

// Keys of the sequence that a query sees
__device__ __forceinline__ int seen_keys(int causal, int q_len, int k_len, int token) {
    return causal ? max(0, min(k_len, token + 1 + k_len - q_len)) : k_len;
}

// Workgroups go round the 8 dies.  Those of one key head go to as few as they can, so that its keys and values stay in their
// L2: all on one die where the heads are a multiple of 8, on 8 / kv_heads dies where they are a divisor of it.
struct Place {
    int head, tile;   // tile: `tiles` or more where there is none
};

__device__ __forceinline__ Place place_of(uint32_t id, int kv_heads, int tiles) {
    const uint32_t die = id & 7, turn = id >> 3;
    if (kv_heads % 8 == 0) return {(int)(die + 8 * (turn / (uint32_t)tiles)), (int)(turn % (uint32_t)tiles)};
    if (8 % kv_heads == 0) return {(int)(die % (uint32_t)kv_heads), (int)(turn * (8 / kv_heads) + die / (uint32_t)kv_heads)};
    return {(int)(id % (uint32_t)kv_heads), (int)(id / (uint32_t)kv_heads)};
}

// Workgroups of a launch for that
inline int64_t places(int64_t tiles, int kv_heads) {
    return kv_heads % 8 && 8 % kv_heads == 0 ? 8 * ((tiles + 8 / kv_heads - 1) / (8 / kv_heads)) : tiles * kv_heads;
}

// The padded head size as a template parameter
template <typename F>
hipError_t with_padded_dim(int D, F f) {
    return D > 96 ? f(std::integral_constant<int, 128>()) : D > 64 ? f(std::integral_constant<int, 96>())
         : D > 32 ? f(std::integral_constant<int, 64>()) : f(std::integral_constant<int, 32>());
}

}  // namespace orbit
