// Layer norm of rows, with weights or modulated by a scale and a shift for each batch, forward and backward, for gfx950.
//
// With m the mean of a row's N values, s = mean((x - m)^2) + eps, r = 1 / sqrt(s) and n = (x - m) r:
//     y = n g + b,          g the weight, or 1 + scale
// and, with h = dy g,
//     dx = r (h - mean(h) - n mean(h n)),   dg = sum over rows of dy n,   db = sum over rows of dy.
// All of it streams its rows once and is bound by HBM: (size of x + size of y) N bytes a row forward, (2 size of x + size
// of dy) N backward: 32760 x 5120 in fp32, results and their gradients in bf16, 194 us (5.2 TB/s) and 295 us (5.7 TB/s), where a
// copy of 4 GiB runs at 4.75 TB/s.  (Non-temporal loads and stores: no difference from 50 MB to 1.7 GB.)
//
// A workgroup walks rows of one batch and keeps in registers what they share: its columns' gains and offsets, or its gains and
// the two gradients' sums.  (Read again for each row, a batch's fp32 scale and shift are twice the traffic of its bf16
// rows, from L2.)  The next row's loads are on their way while a row is reduced.
//
// Statistics: each wave has the mean and the sum of squared deviations of its own part of the row, and parts are joined as by
// Chan, Golub and LeVeque: sum of squares = sum_w (M2_w + n_w (m_w - m)^2).  No difference of large squares is taken, and a
// row costs one barrier.  sum h (x - m) is joined the same way, from sum_w h and sum_w h (x - m_w).
//
// A mean in fp32 is off by some steps of its last place, which a row that varies by no more than that shows whole: 5120 values of
// 3333.3 came out up to 0.9 from 0 at eps = 1e-6.  So a wave's mean is that quotient m' and the mean of the deviations from it,
// which is as small as they are, and waves' means meet as differences from the first one's.  Of bf16 values within a factor of 4
// sums of up to kNormMaxWidth < 2^14 are exact (10 bits above their last place), so one fma finds that mean: sum - n m'.  Of fp32
// values it is a sum of its own: 33272 x 5120 198.0 -> 199.3 us forward, 32760 x 5120 296 -> 296.5 backward, of bf16 values 8858 x
// 3072 20.4 -> 21.0 and 39.4 -> 39.6.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "device.h"
#include "vec.h"

namespace orbit {

namespace {

constexpr int kMostWaves = 16;

typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

// kPiece values in a row, at any element.  (Eight values of bf16 in 16 bytes: the backward pass of 32760 x 5120 took 345 us
// instead of 201, that of 2 x 4429 x 3072 55 instead of 46; forward 133 and 131.)
constexpr int kPiece = 4;

template <typename T>
struct Piece;

template <>
struct Piece<bf16_t> {
    u32x2 r;
    __device__ __forceinline__ void load(const bf16_t* p) { r = *(const u32x2_any*)p; }
    __device__ __forceinline__ void get(float* v) const { v[0] = bf16_low(r.x), v[1] = bf16_high(r.x), v[2] = bf16_low(r.y), v[3] = bf16_high(r.y); }
    static __device__ __forceinline__ void store(bf16_t* p, const float* v) { *(u32x2_any*)p = (u32x2){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}; }
};

template <>
struct Piece<float> {
    f32x4 r;
    __device__ __forceinline__ void load(const float* p) { r = *(const f32x4_any*)p; }
    __device__ __forceinline__ void get(float* v) const { v[0] = r.x, v[1] = r.y, v[2] = r.z, v[3] = r.w; }
    static __device__ __forceinline__ void store(float* p, const float* v) { *(f32x4_any*)p = (f32x4){v[0], v[1], v[2], v[3]}; }
};

__device__ __forceinline__ float value(const bf16_t* p) { return __uint_as_float((uint32_t)p->bits << 16); }
__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ void put(bf16_t* p, float v) { p->bits = (uint16_t)pack_bf16(v, 0.f); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }

// A thread's part of a row: C pieces of kPiece values, blockDim.x pieces apart.  With CUT (N is no multiple of kPiece) the piece
// that the row's end cuts begins further left, so that it is a whole one: its first values are its neighbour's and stay out of
// sums and stores; threads behind the end load it too, so that no branch holds up the next row's loads (32760 x 5118 344 -> 312 us
// backward in fp32).  (Value by value, one after the other and with a branch each, such a piece held up the whole wave: a backward
// pass of 32760 x 5120 370 us for 230, whose last pieces were idle and not even cut.)  A row of less than a piece is one thread's, value
// by value.
template <int C, bool CUT>
struct Columns {
    int at[C];     // first column
    int cut;       // values of the last piece that are its neighbour's
    bool within[C], last;   // whether the pieces are the row's, and the last one is
    int small;     // values of a row of less than a piece, or 0
    __device__ __forceinline__ Columns(int N) {
        small = CUT && C == 1 && N < kPiece ? N : 0;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            at[c] = (c * (int)blockDim.x + (int)threadIdx.x) * kPiece;
            within[c] = at[c] < N;
        }
        last = at[C - 1] < N;
        cut = 0;
        if (CUT && at[C - 1] + kPiece > N && !small) cut = last ? at[C - 1] + kPiece - N : 0, at[C - 1] = N - kPiece;
    }
    // whether value i of piece c is this thread's own
    __device__ __forceinline__ bool own(int c, int i) const { return have(c) && (!CUT || (C == 1 && small ? i < small : i >= skip(c))); }
    // Only the last piece can lie behind the row (`shape` gives the fewest).  Said with CUT: 32760 x 5118 930 -> 312 us backward and
    // 234 -> 199 forward in fp32.  Not without it, where a branch for each piece is faster: 32760 x 5120 294 us for 335 backward in
    // fp32, with as many rows on their way as there are else with 8 waves, though 8858 x 3072 in bf16 20.4 for 19.0 forward.
    __device__ __forceinline__ bool have(int c) const { return !CUT ? within[c] : c < C - 1 || last; }
    __device__ __forceinline__ int skip(int c) const { return c < C - 1 ? 0 : cut; }
};

// Pieces on their way from memory, and their values; values that the row does not have are zeros.
template <typename T, int C, bool CUT>
struct Part {
    Piece<T> piece[C];
    __device__ __forceinline__ void load(const T* row, const Columns<C, CUT>& k) {
        if (k.small) return;
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (CUT || k.have(c)) piece[c].load(row + k.at[c]);
    }
    __device__ __forceinline__ void get(const T* row, const Columns<C, CUT>& k, float (&v)[C][kPiece]) const {
        if (k.small) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < kPiece; ++i) v[c][i] = k.own(c, i) ? value(row + i) : 0.f;
            return;
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (k.have(c)) {
                piece[c].get(v[c]);
            } else {
#pragma unroll
                for (int i = 0; i < kPiece; ++i) v[c][i] = 0.f;
            }
        }
    }
    static __device__ __forceinline__ void store(T* row, const Columns<C, CUT>& k, const float (&v)[C][kPiece]) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (k.small) {
#pragma unroll
                for (int i = 0; i < kPiece; ++i)
                    if (k.own(c, i)) put(row + i, v[c][i]);
            } else if (CUT && k.skip(c)) {
                // the neighbour's values are its own: another wave's mean and deviations round otherwise
#pragma unroll
                for (int i = 1; i < kPiece; ++i)
                    if (i >= k.skip(c)) put(row + k.at[c] + i, v[c][i]);
            } else if (k.have(c)) {
                Piece<T>::store(row + k.at[c], v[c]);
            }
        }
    }
};

// A batch's weights of the thread's columns, `none` where there are none, and `add` to them where there are
template <typename T, int C, bool CUT>
__device__ __forceinline__ void load_weights(const T* w, float add, const Columns<C, CUT>& k, float (&v)[C][kPiece]) {
    Piece<T> piece[C];
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (k.have(c) && !k.small) piece[c].load(w + k.at[c]);
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[c][i] = k.small && k.own(c, i) ? value(w + i) : 0.f;
        if (k.have(c) && !k.small) piece[c].get(v[c]);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[c][i] += add;
    }
}

template <int C, bool CUT>
__device__ __forceinline__ void load_weights(const void* w, bool f32, int64_t first, float none, float add, const Columns<C, CUT>& k, float (&v)[C][kPiece]) {
    if (!w) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < kPiece; ++i) v[c][i] = none;
    } else if (f32) {
        load_weights<float, C, CUT>((const float*)w + first, add, k, v);
    } else {
        load_weights<bf16_t, C, CUT>((const bf16_t*)w + first, add, k, v);
    }
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}

// Sum over the wave, in all lanes: neighbours, pairs, mirrored halves and rows of 16, then across rows
__device__ __forceinline__ float wave_sum(float v) {
    v += dpp<0xB1>(v);    // quad_perm 1 0 3 2
    v += dpp<0x4E>(v);    // quad_perm 2 3 0 1
    v += dpp<0x141>(v);   // row_half_mirror
    v += dpp<0x140>(v);   // row_mirror
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Values of the row that wave w holds
template <int C>
__device__ __forceinline__ int wave_values(int w, int N) {
    int n = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) n += min(max(N - (c * (int)blockDim.x + 64 * w) * kPiece, 0), 64 * kPiece);
    return n;
}

// A wave's mean, as a quotient and the rest of it, the deviations from both in v's place and their sum of squares
template <typename T, int C, bool CUT>
__device__ __forceinline__ void wave_statistics(float (&v)[C][kPiece], const Columns<C, CUT>& k, float n, float inv_n, float* mean, float* rest, float* squares) {
    constexpr bool kExact = std::is_same<T, bf16_t>::value;
    float sum = 0.f, left = 0.f, sq = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < kPiece; ++i) sum += !CUT || k.own(c, i) ? v[c][i] : 0.f;
    sum = wave_sum(sum);
    *mean = n ? sum / n : 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            v[c][i] -= *mean;
            if (!kExact) left += k.own(c, i) ? v[c][i] : 0.f;
        }
    *rest = (kExact ? __builtin_fmaf(-n, *mean, sum) : wave_sum(left)) * inv_n;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            v[c][i] -= *rest;
            sq += k.own(c, i) ? v[c][i] * v[c][i] : 0.f;
        }
    *squares = wave_sum(sq);
}

struct Joined {
    float shift;   // the wave's mean less the row's
    float squares, sum, dot;
};

// What the waves found of a row, joined.  part[w]: its mean and the rest of it, squares, and backward sum h and sum h (x - m_w).
template <int Q>
__device__ __forceinline__ Joined join(const float (*part)[Q], const float* count, int waves, int wave, float inv_N) {
    const float first = part[0][0];
    float total = 0.f;
    for (int w = 0; w < waves; ++w) total += (part[w][0] - first + part[w][1]) * count[w];
    const float mean = total * inv_N;   // from `first`
    Joined j{part[wave][0] - first + part[wave][1] - mean, 0.f, 0.f, 0.f};
    for (int w = 0; w < waves; ++w) {
        const float d = part[w][0] - first + part[w][1] - mean;
        j.squares += part[w][2] + count[w] * d * d;
        if (Q == 5) {
            j.sum += part[w][Q - 2];
            j.dot += part[w][Q - 1] + d * part[w][Q - 2];
        }
    }
    return j;
}

template <typename T>
__device__ __forceinline__ T* row_of(const NormRows& t, int64_t b, int64_t l) {
    return (T*)t.p + b * t.batch + l * t.row;
}

// Workgroup p of group g: rows p, p + parts, ... of the group, which is a batch, or all batches' rows where they share their weights
template <typename TX, typename TY, int C, bool CUT>
__global__ __launch_bounds__(C > 2 ? 512 : 1024) void layer_norm_kernel(NormParams p) {
    __shared__ float part[2][kMostWaves][3];
    __shared__ float count[kMostWaves];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const Columns<C, CUT> k(p.N);
    const int n = wave_values<C>(wave, p.N);
    const float inv_N = 1.f / p.N, inv_n = n ? 1.f / n : 0.f;
    if ((threadIdx.x & 63) == 0) count[wave] = n;
    const int64_t g = blockIdx.x / (uint32_t)p.parts;
    int64_t row = blockIdx.x % (uint32_t)p.parts, b = g, l = row;
    auto locate = [&]() {
        if (p.joined) b = row / p.L, l = row - b * p.L;   // only of batches that do not follow each other row by row
        else l = row;
    };
    locate();
    Part<TX, C, CUT> next;
    next.load(row_of<const TX>(p.x, b, l), k);
    float gain[C][kPiece], offset[C][kPiece];
    load_weights<C, CUT>(p.w, p.w_f32, g * p.w_batch, 1.f, p.modulate ? 1.f : 0.f, k, gain);
    load_weights<C, CUT>(p.b, p.w_f32, g * p.b_batch, 0.f, 0.f, k, offset);
    for (int turn = 0; row < p.rows; turn ^= 1) {
        float v[C][kPiece];
        next.get(row_of<const TX>(p.x, b, l), k, v);
        TY* const y = row_of<TY>(p.y, b, l);
        row += p.parts;
        if (row < p.rows) {
            locate();
            next.load(row_of<const TX>(p.x, b, l), k);
        }
        float mean, rest, squares;
        wave_statistics<TX, C, CUT>(v, k, n, inv_n, &mean, &rest, &squares);
        if ((threadIdx.x & 63) == 0) part[turn][wave][0] = mean, part[turn][wave][1] = rest, part[turn][wave][2] = squares;
        __syncthreads();
        const Joined j = join<3>(part[turn], count, waves, wave, inv_N);
        const float r = rsqrtf(j.squares * inv_N + p.eps);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < kPiece; ++i) v[c][i] = (v[c][i] + j.shift) * r * gain[c][i] + offset[c][i];
        Part<TY, C, CUT>::store(y, k, v);
    }
}

template <typename TX, typename TG, int C, bool CUT>
__global__ __launch_bounds__(C > 2 ? 512 : 1024) void layer_norm_backward_kernel(NormParams p) {
    __shared__ float part[2][kMostWaves][5];
    __shared__ float count[kMostWaves];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const Columns<C, CUT> k(p.N);
    const int n = wave_values<C>(wave, p.N);
    const float inv_N = 1.f / p.N, inv_n = n ? 1.f / n : 0.f;
    if ((threadIdx.x & 63) == 0) count[wave] = n;
    const int64_t g = blockIdx.x / (uint32_t)p.parts;
    int64_t row = blockIdx.x % (uint32_t)p.parts, b = g, l = row;
    auto locate = [&]() {
        if (p.joined) b = row / p.L, l = row - b * p.L;   // only of batches that do not follow each other row by row
        else l = row;
    };
    Part<TX, C, CUT> next_x;
    Part<TG, C, CUT> next_g;
    if (row < p.rows) {
        locate();
        next_x.load(row_of<const TX>(p.x, b, l), k);
        next_g.load(row_of<const TG>(p.g, b, l), k);
    }
    float gain[C][kPiece], dw[C][kPiece], db[C][kPiece];
    load_weights<C, CUT>(p.w, p.w_f32, g * p.w_batch, 1.f, p.modulate ? 1.f : 0.f, k, gain);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < kPiece; ++i) dw[c][i] = db[c][i] = 0.f;
    for (int turn = 0; row < p.rows; turn ^= 1) {
        float v[C][kPiece], h[C][kPiece];
        next_x.get(row_of<const TX>(p.x, b, l), k, v);
        next_g.get(row_of<const TG>(p.g, b, l), k, h);
        TX* const y = row_of<TX>(p.y, b, l);
        row += p.parts;
        if (row < p.rows) {
            locate();
            next_x.load(row_of<const TX>(p.x, b, l), k);
            next_g.load(row_of<const TG>(p.g, b, l), k);
        }
        float mean, rest, squares, sum = 0.f, dot = 0.f;
        wave_statistics<TX, C, CUT>(v, k, n, inv_n, &mean, &rest, &squares);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                const float hg = k.own(c, i) ? h[c][i] * gain[c][i] : 0.f;
                sum += hg;
                dot += hg * v[c][i];
            }
        sum = wave_sum(sum);
        dot = wave_sum(dot);
        if ((threadIdx.x & 63) == 0) {
            part[turn][wave][0] = mean, part[turn][wave][1] = rest, part[turn][wave][2] = squares;
            part[turn][wave][3] = sum, part[turn][wave][4] = dot;
        }
        __syncthreads();
        const Joined j = join<5>(part[turn], count, waves, wave, inv_N);
        const float r = rsqrtf(j.squares * inv_N + p.eps);
        const float mean_h = j.sum * inv_N, mean_hn = r * (j.dot * inv_N);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                const float unit = (v[c][i] + j.shift) * r;
                db[c][i] += h[c][i];
                dw[c][i] += h[c][i] * unit;
                v[c][i] = r * (h[c][i] * gain[c][i] - mean_h - unit * mean_hn);
            }
        Part<TX, C, CUT>::store(y, k, v);
    }
    // [group][workgroup][2][N]
    float* const out = p.part + (int64_t)blockIdx.x * 2 * p.N;
    if (p.dw)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (k.own(c, i)) out[k.at[c] + i] = dw[c][i];
    if (p.db)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (k.own(c, i)) out[p.N + k.at[c] + i] = db[c][i];
}

// A group's gradients from its workgroups' sums, in a fixed order: 32 columns to a workgroup of 1024, 32 of its threads to a
// column.  blockIdx.y: weight or bias.
__global__ __launch_bounds__(1024) void layer_norm_sum_kernel(NormParams p) {
    __shared__ float part[32][33];
    float* const out = blockIdx.y ? p.db : p.dw;
    if (!out) return;
    const int col = threadIdx.x & 31, at = threadIdx.x >> 5, strips = (p.N + 31) / 32;
    const int64_t g = blockIdx.x / (uint32_t)strips;
    const int d = blockIdx.x % (uint32_t)strips * 32 + col;
    const float* const from = p.part + g * p.parts * 2 * (int64_t)p.N + (int64_t)blockIdx.y * p.N;
    float sum = 0.f;
    if (d < p.N) {
#pragma unroll 8
        for (int i = at; i < p.parts; i += 32) sum += from[(int64_t)i * 2 * p.N + d];
    }
    part[at][col] = sum;
    __syncthreads();
    for (int half = 16; half; half /= 2) {
        if (at < half) part[at][col] += part[at + half][col];
        __syncthreads();
    }
    if (at == 0 && d < p.N) out[g * p.N + d] = part[0][col];
}

constexpr int kMostPieces = 6;   // to a thread: kNormMaxWidth in 8 waves

// Waves that share a row, and pieces to a thread: the fewest of 1, 2, 3, 4 and 8 waves, which lie evenly on a compute unit's SIMDs
// (rows of 5120 fp32 values to bf16: 4 and 5 194 us, 5 and 4 242).  Where there are too few rows to fill the card, up to kMostWaves
// waves with up to 2 pieces, for latency.
struct Shape {
    int waves, pieces;
};

Shape shape(int N, int64_t rows, int cus) {
    const int groups = (N + 64 * kPiece - 1) / (64 * kPiece);   // of 64 pieces
    if (rows < 2 * (int64_t)cus && groups <= 2 * kMostWaves) {
        const int each = (groups + kMostWaves - 1) / kMostWaves;
        return {(groups + each - 1) / each, each};
    }
    int waves = 1;
    while (waves * kMostPieces < groups) waves = waves < 4 ? waves + 1 : 8;
    return {waves, (groups + waves - 1) / waves};
}

// The kernel's pieces as a template parameter.
template <typename F>
hipError_t with_pieces(int pieces, F f) {
    switch (pieces) {
        case 1: f(std::integral_constant<int, 1>()); break;
        case 2: f(std::integral_constant<int, 2>()); break;
        case 3: f(std::integral_constant<int, 3>()); break;
        case 4: f(std::integral_constant<int, 4>()); break;
        case 5: f(std::integral_constant<int, 5>()); break;
        case 6: f(std::integral_constant<int, 6>()); break;
        default: return hipErrorInvalidConfiguration;
    }
    return hipGetLastError();
}

template <typename TX, typename TY, bool CUT>
hipError_t launch_forward(NormParams p, int groups, int cus, hipStream_t stream) {
    const Shape s = shape(p.N, p.rows * groups, cus);
    return with_pieces(s.pieces, [&](auto c) {
        constexpr int C = decltype(c)::value;
        const int64_t resident = p.rows * groups <= cus ? 1 : resident_blocks((const void*)layer_norm_kernel<TX, TY, C, CUT>, 64 * s.waves, 0);
        p.parts = (int)std::min<int64_t>(p.rows, (resident * cus + groups - 1) / groups);
        layer_norm_kernel<TX, TY, C, CUT><<<(unsigned)(p.parts * groups), 64 * s.waves, 0, stream>>>(p);
    });
}

template <typename TX, typename TG, bool CUT>
hipError_t launch_backward(const NormParams& p, int groups, int cus, hipStream_t stream) {
    const Shape s = shape(p.N, p.rows * groups, cus);
    const hipError_t e = with_pieces(s.pieces, [&](auto c) {
        layer_norm_backward_kernel<TX, TG, decltype(c)::value, CUT><<<(unsigned)(p.parts * groups), 64 * s.waves, 0, stream>>>(p);
    });
    if (e != hipSuccess || (!p.dw && !p.db)) return e;
    layer_norm_sum_kernel<<<dim3((unsigned)((p.N + 31) / 32 * groups), 2), 1024, 0, stream>>>(p);
    return hipGetLastError();
}

template <typename TX, typename TO, bool BACK>
hipError_t launch(const NormParams& p, int groups, int cus, hipStream_t stream) {
    auto go = [&](auto cut) {
        constexpr bool CUT = decltype(cut)::value;
        if constexpr (BACK)
            return launch_backward<TX, TO, CUT>(p, groups, cus, stream);
        else
            return launch_forward<TX, TO, CUT>(p, groups, cus, stream);
    };
    return p.N % kPiece ? go(std::true_type()) : go(std::false_type());
}

template <bool BACK>
hipError_t launch(const NormParams& p, int groups, bool x_f32, bool o_f32, int cus, hipStream_t stream) {
    if (x_f32) return o_f32 ? launch<float, float, BACK>(p, groups, cus, stream) : launch<float, bf16_t, BACK>(p, groups, cus, stream);
    return o_f32 ? launch<bf16_t, float, BACK>(p, groups, cus, stream) : launch<bf16_t, bf16_t, BACK>(p, groups, cus, stream);
}

}  // namespace

hipError_t launch_layer_norm(const NormParams& p, int groups, bool x_f32, bool y_f32, int cus, hipStream_t stream) {
    return launch<false>(p, groups, x_f32, y_f32, cus, stream);
}

// 8 waves to a compute unit, 6 where x is fp32: more add to the sums that are written and read again, and have more rows on their
// way than the memory serves at once; fewer leave loads without cover.  us of 4, 6, 8, 12 and 16 waves:
//     x bf16, dy bf16, 32760 x 5120: 270 270 196 248 212    8858 x 3072: 54 45 43 51 57    65536 x 1024: 110 103 88 93 102
//     x fp32, dy bf16, 32760 x 5120: 293 293 333 347 346    8858 x 3072: 57 56 58 62 70    65536 x 2048: 282 242 259 276 299
int layer_norm_parts(int64_t rows, int groups, int64_t N, bool x_f32, int cus) {
    const int64_t most = std::max<int64_t>(1, (x_f32 ? 6 : 8) / shape((int)N, rows * groups, cus).waves) * cus;
    return (int)std::max<int64_t>(1, std::min(rows, (most + groups - 1) / groups));
}

hipError_t launch_layer_norm_backward(const NormParams& p, int groups, bool x_f32, bool g_f32, int cus, hipStream_t stream) {
    return launch<true>(p, groups, x_f32, g_f32, cus, stream);
}

}  // namespace orbit
