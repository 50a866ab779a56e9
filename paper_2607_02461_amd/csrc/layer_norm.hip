// Layer norm of rows, with weights or modulated by a scale and a shift for each batch, forward and backward, for gfx950.
//
// With m the mean of a row's N values, s = mean((x - m)^2) + eps, r = 1 / sqrt(s) and n = (x - m) r:
//     y = n g + b,          g the weight, or 1 + scale
// and, with h = dy g,
//     dx = r (h - mean(h) - n mean(h n)),   dg = sum over rows of dy n,   db = sum over rows of dy.
// All of it streams its rows once and is bound by HBM: (size of x + size of y) N bytes a row forward, (2 size of x + size
// of dy) N backward.
//
// A workgroup walks rows of one batch and keeps in registers what they share: its columns' gains and offsets, or its gains and
// the two gradients' sums.  (Read again for each row, a batch's fp32 scale and shift are twice the traffic of its bf16
// rows, from L2.)  The next row's loads are on their way while a row is reduced.
//
// Statistics: each wave has the mean and the sum of squared deviations of its own part of the row, two sums in registers, and
// parts are joined as by Chan, Golub and LeVeque: sum of squares = sum_w (M2_w + n_w (m_w - m)^2).  No difference of large
// squares is taken, and a row costs one barrier.  sum h (x - m) is joined the same way, from sum_w h and sum_w h (x - m_w).
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

// V values at any element: 8 of bf16 or 4 of either type are one access
template <typename T, int V>
struct Piece;

template <>
struct Piece<bf16_t, 8> {
    u32x4 r;
    __device__ __forceinline__ void load(const bf16_t* p, bool nt) { r = nt ? __builtin_nontemporal_load((const u32x4_any*)p) : *(const u32x4_any*)p; }
    __device__ __forceinline__ void get(float* v) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = bf16_low(r[i]), v[2 * i + 1] = bf16_high(r[i]);
    }
    static __device__ __forceinline__ void store(bf16_t* p, const float* v, bool nt) {
        const u32x4 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        if (nt)
            __builtin_nontemporal_store(w, (u32x4_any*)p);
        else
            *(u32x4_any*)p = w;
    }
};

template <>
struct Piece<bf16_t, 4> {
    u32x2 r;
    __device__ __forceinline__ void load(const bf16_t* p, bool nt) { r = nt ? __builtin_nontemporal_load((const u32x2_any*)p) : *(const u32x2_any*)p; }
    __device__ __forceinline__ void get(float* v) const { v[0] = bf16_low(r.x), v[1] = bf16_high(r.x), v[2] = bf16_low(r.y), v[3] = bf16_high(r.y); }
    static __device__ __forceinline__ void store(bf16_t* p, const float* v, bool nt) {
        const u32x2 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        if (nt)
            __builtin_nontemporal_store(w, (u32x2_any*)p);
        else
            *(u32x2_any*)p = w;
    }
};

template <>
struct Piece<float, 4> {
    f32x4 r;
    __device__ __forceinline__ void load(const float* p, bool nt) { r = nt ? __builtin_nontemporal_load((const f32x4_any*)p) : *(const f32x4_any*)p; }
    __device__ __forceinline__ void get(float* v) const { v[0] = r.x, v[1] = r.y, v[2] = r.z, v[3] = r.w; }
    static __device__ __forceinline__ void store(float* p, const float* v, bool nt) {
        const f32x4 w = {v[0], v[1], v[2], v[3]};
        if (nt)
            __builtin_nontemporal_store(w, (f32x4_any*)p);
        else
            *(f32x4_any*)p = w;
    }
};

// Values to an access: as many as both types have in 16 bytes
template <typename A, typename B>
constexpr int values_of() {
    return sizeof(A) + sizeof(B) == 4 ? 8 : 4;
}

__device__ __forceinline__ float value(const bf16_t* p) { return __uint_as_float((uint32_t)p->bits << 16); }
__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ void put(bf16_t* p, float v) { p->bits = (uint16_t)pack_bf16(v, 0.f); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }

// A thread's part of a row: C pieces of V values, T pieces apart.  The piece that the row's end cuts is read and written value
// by value (`cut`: the values that it has), those behind it not at all.
template <int V, int C>
struct Columns {
    int at[C];     // first column
    int have[C];   // values: V, fewer, or 0
    __device__ __forceinline__ Columns(int N) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            at[c] = (c * (int)blockDim.x + (int)threadIdx.x) * V;
            have[c] = min(max(N - at[c], 0), V);
        }
    }
};

// Pieces on their way from memory, and their values; values that the row does not have are zeros.
template <typename T, int V, int C, bool NT>
struct Part {
    Piece<T, V> piece[C];
    __device__ __forceinline__ void load(const T* row, const Columns<V, C>& k) {
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (k.have[c] == V) piece[c].load(row + k.at[c], NT);
    }
    __device__ __forceinline__ void get(const T* row, const Columns<V, C>& k, float (&v)[C][V]) const {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (k.have[c] == V) {
                piece[c].get(v[c]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) v[c][i] = i < k.have[c] ? value(row + k.at[c] + i) : 0.f;
            }
        }
    }
    static __device__ __forceinline__ void store(T* row, const Columns<V, C>& k, const float (&v)[C][V]) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (k.have[c] == V) {
                Piece<T, V>::store(row + k.at[c], v[c], NT);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i < k.have[c]) put(row + k.at[c] + i, v[c][i]);
            }
        }
    }
};

// A batch's weights of the thread's columns, `none` where there are none
template <int V, int C>
__device__ __forceinline__ void load_weights(const void* w, bool f32, int64_t first, float none, float add, const Columns<V, C>& k, float (&v)[C][V]) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[c][i] = none;
            if (w && i < k.have[c]) {
                const int64_t at = first + k.at[c] + i;
                v[c][i] = (f32 ? ((const float*)w)[at] : value((const bf16_t*)w + at)) + add;
            }
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
template <int V, int C>
__device__ __forceinline__ int wave_values(int w, int N) {
    int n = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) n += min(max(N - (c * (int)blockDim.x + 64 * w) * V, 0), 64 * V);
    return n;
}

// A wave's mean, the deviations from it in v's place (zeros for what the row does not have) and their sum of squares
template <int V, int C>
__device__ __forceinline__ void wave_statistics(float (&v)[C][V], const Columns<V, C>& k, float n, float* mean, float* squares) {
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) sum += v[c][i];
    *mean = n ? wave_sum(sum) / n : 0.f;   // a quotient: a row of equal values has that value for a mean
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[c][i] = i < k.have[c] ? v[c][i] - *mean : 0.f;
            sq += v[c][i] * v[c][i];
        }
    *squares = wave_sum(sq);
}

struct Joined {
    float shift;   // the wave's mean less the row's
    float squares, sum, dot;
};

// What the waves found of a row, joined.  part[w]: n_w times its mean, squares, and backward sum h and sum h (x - m_w).
template <int Q>
__device__ __forceinline__ Joined join(const float (*part)[Q], const float* count, int waves, int wave, float N) {
    float total = 0.f;
    for (int w = 0; w < waves; ++w) total += part[w][0] * count[w];
    const float mean = total / N;
    Joined j{part[wave][0] - mean, 0.f, 0.f, 0.f};
    for (int w = 0; w < waves; ++w) {
        const float d = part[w][0] - mean;
        j.squares += part[w][1] + count[w] * d * d;
        if (Q == 4) {
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
template <typename TX, typename TY, int C, bool NT>
__global__ __launch_bounds__((C * values_of<TX, TY>() > 8 ? 512 : 1024)) void layer_norm_kernel(NormParams p) {
    constexpr int V = values_of<TX, TY>();
    __shared__ float part[2][kMostWaves][2];
    __shared__ float count[kMostWaves];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const Columns<V, C> k(p.N);
    const int n = wave_values<V, C>(wave, p.N);
    const float inv_N = 1.f / p.N;
    if ((threadIdx.x & 63) == 0) count[wave] = n;
    const int64_t g = blockIdx.x / (uint32_t)p.parts;
    int64_t row = blockIdx.x % (uint32_t)p.parts, b = g, l = row;
    auto locate = [&]() {
        if (p.joined) b = row / p.L, l = row - b * p.L;
        else l = row;
    };
    locate();
    Part<TX, V, C, NT> next;
    next.load(row_of<const TX>(p.x, b, l), k);
    float gain[C][V], offset[C][V];
    load_weights<V, C>(p.w, p.w_f32, g * p.w_batch, 1.f, p.modulate ? 1.f : 0.f, k, gain);
    load_weights<V, C>(p.b, p.w_f32, g * p.b_batch, 0.f, 0.f, k, offset);
    for (int turn = 0; row < p.rows; turn ^= 1) {
        float v[C][V];
        next.get(row_of<const TX>(p.x, b, l), k, v);
        TY* const y = row_of<TY>(p.y, b, l);
        row += p.parts;
        if (row < p.rows) {
            locate();
            next.load(row_of<const TX>(p.x, b, l), k);
        }
        float mean, squares;
        wave_statistics<V, C>(v, k, n, &mean, &squares);
        if ((threadIdx.x & 63) == 0) part[turn][wave][0] = mean, part[turn][wave][1] = squares;
        __syncthreads();
        const Joined j = join<2>(part[turn], count, waves, wave, p.N);
        const float r = rsqrtf(j.squares * inv_N + p.eps);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] = (v[c][i] + j.shift) * r * gain[c][i] + offset[c][i];
        Part<TY, V, C, NT>::store(y, k, v);
    }
}

template <typename TX, typename TG, int C, bool NT>
__global__ __launch_bounds__((C * values_of<TX, TG>() > 8 ? 512 : 1024)) void layer_norm_backward_kernel(NormParams p) {
    constexpr int V = values_of<TX, TG>();
    __shared__ float part[2][kMostWaves][4];
    __shared__ float count[kMostWaves];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const Columns<V, C> k(p.N);
    const int n = wave_values<V, C>(wave, p.N);
    const float inv_N = 1.f / p.N;
    if ((threadIdx.x & 63) == 0) count[wave] = n;
    const int64_t g = blockIdx.x / (uint32_t)p.parts;
    int64_t row = blockIdx.x % (uint32_t)p.parts, b = g, l = row;
    auto locate = [&]() {
        if (p.joined) b = row / p.L, l = row - b * p.L;
        else l = row;
    };
    Part<TX, V, C, NT> next_x;
    Part<TG, V, C, NT> next_g;
    if (row < p.rows) {
        locate();
        next_x.load(row_of<const TX>(p.x, b, l), k);
        next_g.load(row_of<const TG>(p.g, b, l), k);
    }
    float gain[C][V], dw[C][V], db[C][V];
    load_weights<V, C>(p.w, p.w_f32, g * p.w_batch, 1.f, p.modulate ? 1.f : 0.f, k, gain);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) dw[c][i] = db[c][i] = 0.f;
    for (int turn = 0; row < p.rows; turn ^= 1) {
        float v[C][V], h[C][V];
        next_x.get(row_of<const TX>(p.x, b, l), k, v);
        next_g.get(row_of<const TG>(p.g, b, l), k, h);
        TX* const y = row_of<TX>(p.y, b, l);
        row += p.parts;
        if (row < p.rows) {
            locate();
            next_x.load(row_of<const TX>(p.x, b, l), k);
            next_g.load(row_of<const TG>(p.g, b, l), k);
        }
        float mean, squares, sum = 0.f, dot = 0.f;
        wave_statistics<V, C>(v, k, n, &mean, &squares);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float hg = h[c][i] * gain[c][i];
                sum += hg;
                dot += hg * v[c][i];
            }
        sum = wave_sum(sum);
        dot = wave_sum(dot);
        if ((threadIdx.x & 63) == 0) {
            part[turn][wave][0] = mean, part[turn][wave][1] = squares;
            part[turn][wave][2] = sum, part[turn][wave][3] = dot;
        }
        __syncthreads();
        const Joined j = join<4>(part[turn], count, waves, wave, p.N);
        const float r = rsqrtf(j.squares * inv_N + p.eps);
        const float mean_h = j.sum * inv_N, mean_hn = r * (j.dot * inv_N);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float unit = (v[c][i] + j.shift) * r;
                db[c][i] += h[c][i];
                if (i < k.have[c]) dw[c][i] += h[c][i] * unit;
                v[c][i] = r * (h[c][i] * gain[c][i] - mean_h - unit * mean_hn);
            }
        Part<TX, V, C, NT>::store(y, k, v);
    }
    // [group][workgroup][2][N]
    float* const out = p.part + (int64_t)blockIdx.x * 2 * p.N;
    if (p.dw)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < k.have[c]) out[k.at[c] + i] = dw[c][i];
    if (p.db)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < k.have[c]) out[p.N + k.at[c] + i] = db[c][i];
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

constexpr int kMostValues = 24;  // of a row to a thread: kNormMaxWidth in 512 threads

// Threads to a row, and pieces to a thread.  As few threads as hold a row with kMostValues each; where there are too few rows to
// fill the card, 8 values each in up to 1024, for latency.
struct Shape {
    int threads, pieces;
};

Shape shape(int64_t rows, int N, int V, int cus) {
    const int most = rows < 2 * (int64_t)cus && N <= 8 * 64 * kMostWaves ? 8 : kMostValues;
    int threads = 64;
    while (threads * most < N) threads *= 2;
    return {threads, (N + threads * V - 1) / (threads * V)};
}

// The kernel's pieces as a template parameter.  16-byte accesses of bf16 take 3 at most for kMostValues, of fp32 6.
template <int V, typename F>
hipError_t with_pieces(int pieces, F f) {
    switch (pieces) {
        case 1: f(std::integral_constant<int, 1>()); break;
        case 2: f(std::integral_constant<int, 2>()); break;
        case 3: f(std::integral_constant<int, 3>()); break;
        case 4: f(std::integral_constant<int, V == 4 ? 4 : 1>()); break;
        case 5: f(std::integral_constant<int, V == 4 ? 5 : 1>()); break;
        case 6: f(std::integral_constant<int, V == 4 ? 6 : 1>()); break;
        default: return hipErrorInvalidConfiguration;
    }
    return hipGetLastError();
}

template <typename TX, typename TY, bool NT>
hipError_t launch_forward(NormParams p, int groups, int cus, hipStream_t stream) {
    constexpr int V = values_of<TX, TY>();
    const Shape s = shape(p.rows * groups, p.N, V, cus);
    return with_pieces<V>(s.pieces, [&](auto c) {
        constexpr int C = decltype(c)::value;
        const int resident = resident_blocks((const void*)layer_norm_kernel<TX, TY, C, NT>, s.threads, 0);
        p.parts = (int)std::min<int64_t>(p.rows, ((int64_t)resident * cus + groups - 1) / groups);
        layer_norm_kernel<TX, TY, C, NT><<<(unsigned)(p.parts * groups), s.threads, 0, stream>>>(p);
    });
}

template <typename TX, typename TG, bool NT>
hipError_t launch_backward(const NormParams& p, int groups, int cus, hipStream_t stream) {
    constexpr int V = values_of<TX, TG>();
    const Shape s = shape(p.rows * groups, p.N, V, cus);
    const hipError_t e = with_pieces<V>(s.pieces, [&](auto c) {
        layer_norm_backward_kernel<TX, TG, decltype(c)::value, NT><<<(unsigned)(p.parts * groups), s.threads, 0, stream>>>(p);
    });
    if (e != hipSuccess || (!p.dw && !p.db)) return e;
    layer_norm_sum_kernel<<<dim3((unsigned)((p.N + 31) / 32 * groups), 2), 1024, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_layer_norm(const NormParams& p, int groups, bool x_f32, bool y_f32, int cus, hipStream_t stream) {
    if (p.stream) {
        if (x_f32) return y_f32 ? launch_forward<float, float, true>(p, groups, cus, stream) : launch_forward<float, bf16_t, true>(p, groups, cus, stream);
        return y_f32 ? launch_forward<bf16_t, float, true>(p, groups, cus, stream) : launch_forward<bf16_t, bf16_t, true>(p, groups, cus, stream);
    }
    if (x_f32) return y_f32 ? launch_forward<float, float, false>(p, groups, cus, stream) : launch_forward<float, bf16_t, false>(p, groups, cus, stream);
    return y_f32 ? launch_forward<bf16_t, float, false>(p, groups, cus, stream) : launch_forward<bf16_t, bf16_t, false>(p, groups, cus, stream);
}

int layer_norm_parts(int64_t rows, int groups, int cus) {
    const int64_t each = std::max<int64_t>(1, (2 * (int64_t)cus + groups - 1) / groups);
    return (int)std::max<int64_t>(1, std::min(rows, each));
}

hipError_t launch_layer_norm_backward(const NormParams& p, int groups, bool x_f32, bool g_f32, int cus, hipStream_t stream) {
    if (p.stream) {
        if (x_f32) return g_f32 ? launch_backward<float, float, true>(p, groups, cus, stream) : launch_backward<float, bf16_t, true>(p, groups, cus, stream);
        return g_f32 ? launch_backward<bf16_t, float, true>(p, groups, cus, stream) : launch_backward<bf16_t, bf16_t, true>(p, groups, cus, stream);
    }
    if (x_f32) return g_f32 ? launch_backward<float, float, false>(p, groups, cus, stream) : launch_backward<float, bf16_t, false>(p, groups, cus, stream);
    return g_f32 ? launch_backward<bf16_t, float, false>(p, groups, cus, stream) : launch_backward<bf16_t, bf16_t, false>(p, groups, cus, stream);
}

}  // namespace orbit
