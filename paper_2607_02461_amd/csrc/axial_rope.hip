// Rotary positions with several axes, alone and behind the RMS norms of queries and keys, for gfx950.
//
// A head of D values holds P = D_r / 2 pairs that are rotated and D - D_r values that are not.  Pair p belongs to
// one axis of the token's position (time, height, width) and turns by angle(p, position on that axis); cosines and
// sines come from a table per axis, made in 64 bits when the plan was.  With n = x / sqrt(mean(x^2) + eps) * w
// for the norm of one head (n = x without it), a pair (u, v) of n becomes (u cos - v sin, u sin + v cos).
//
// Backward: g = dy turned by the negative angles is the gradient of n, and with r = 1 / sqrt(mean(x^2) + eps)
//     dw = sum over rows of g x r,     dx = r (g w - x r^2 mean(g w x)).
// r comes from x again, which has to be read anyhow; both means come out of one pass over the row.
//
// All of it is bound by HBM: a value is read and written once and takes 3 to 16 operations.  So a head's row stays
// in registers, eight values (16 bytes of bf16) to a lane and D / 8 lanes to a head, a wave holds the same token's
// heads side by side and has the loads of up to kRows rows in flight before the first is used, and the cosines and
// sines of a lane's four pairs are fetched once for all of these rows.  (A token of more heads takes further waves, queries
// and keys take waves of their own, and each of them fetches them again, from a cache.)  Heads of 128, bytes read and written:
//   rotation, 32760 tokens of 40 heads in bf16                         108 us, 6.2 TB/s (a part stays in the last cache),
//     107 us where a pair's values are a half of the head apart
//   norms and rotation, 9216 tokens of 24 + 24 heads in bf16            47 us, 4.8 TB/s
//   the same, 32760 tokens of 40 + 40 heads, fp32 to bf16              372 us, 5.4 TB/s; fp32 to fp32 487, bf16 to fp32 361
//   its gradients, 8858 tokens of 24 + 24 heads in bf16            67 + 5 us, 4.9 TB/s; in fp32 122
// One token takes 4 to 6 us.  Heads of 80 or 96 leave 6 or 4 of 16 lanes idle: 9216 tokens of 24 + 24 of them take the
// norm's 18 million vector instructions of heads of 128, and 42 us for 142 and 170 MB where those take 47 for 226.
// The rotation alone (27 and 32 us; 40) keeps to the copy's rate, and so does the norm of 700 MB of heads of 80 (141 us).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "device.h"
#include "vec.h"

namespace orbit {

namespace {

constexpr int kRows = 6;       // head rows that a wave's lanes have in flight
constexpr int kBackRows = 3;   // the same for the backward pass, which reads two tensors, where heads are few
constexpr int kWaves = 4;      // waves to a workgroup
constexpr int kBackGroups = 8; // most workgroups of the backward pass to a compute unit
constexpr uint32_t kMostItems = 1u << 25;  // waves of one launch

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}

// The sum over aligned groups of `lanes` lanes (a power of two), in each of them.  Every lane is active.
__device__ __forceinline__ float group_sum(float v, int lanes) {
    if (lanes > 1) v = dpp_add<0xB1>(v);   // quad_perm [1,0,3,2]
    if (lanes > 2) v = dpp_add<0x4E>(v);   // quad_perm [2,3,0,1]
    if (lanes > 4) v = dpp_add<0x141>(v);  // row_half_mirror
    if (lanes > 8) v = dpp_add<0x140>(v);  // row_mirror
    if (lanes > 16) v += __shfl_xor(v, 16);
    if (lanes > 32) v += __shfl_xor(v, 32);
    return v;
}

// How a head's values lie in its lanes, eight to a lane, so that a load or store of the wave is whole lines: eight in a
// row of bf16 (kRow), or two fours, of pairs' first halves and their second ones (kHalves), or of the head's first half
// and its second one where values of 4 bytes are read or written (kApart).
enum { kRow, kHalves, kApart };

template <typename T, int LAY, bool NT>
struct Row8 {
    Vec4<T, NT> a, b;
    __device__ __forceinline__ void load(const T* p, int lo, int hi) { a.load(p + lo), b.load(p + hi); }
    __device__ __forceinline__ void get(float* f) const { a.get(f), b.get(f + 4); }
    static __device__ __forceinline__ void store(T* p, int lo, int hi, const float* f) {
        Vec4<T, NT>::store(p + lo, f);
        Vec4<T, NT>::store(p + hi, f + 4);
    }
};

template <bool NT>
struct Row8<bf16_t, kRow, NT> {
    Vec8<NT> v;
    __device__ __forceinline__ void load(const bf16_t* p, int lo, int) { v.load(p + lo); }
    __device__ __forceinline__ void get(float* f) const { v.get(f); }
    static __device__ __forceinline__ void store(bf16_t* p, int lo, int, const float* f) { Vec8<NT>::store(p + lo, f); }
};

// What a lane does in every row: where its two fours of values begin, and the first of its four pairs, or of the two
// pairs of either four.
template <int LAY>
struct Lane {
    int lo, hi, pair, pair_hi;
    bool live, turned, turned_hi;
    __device__ __forceinline__ Lane(const RopeParams& p, int lane) {
        int c = lane & (p.lanes - 1);
        live = c * 8 < p.D;
        if (!live) c = 0;  // loads what lane 0 of the group does, adds nothing to a sum and stores nothing
        if (LAY == kApart) {
            lo = 4 * c, hi = p.D / 2 + 4 * c;
            pair = 2 * c, pair_hi = p.D / 4 + 2 * c;
            turned = pair < p.pairs, turned_hi = pair_hi < p.pairs;
        } else {
            turned = turned_hi = 4 * c < p.pairs;
            pair = 4 * c, pair_hi = 4 * c + 2;
            if (LAY == kHalves) {
                // what is not turned lies behind the pairs, and in two halves too
                lo = 4 * c + (turned ? 0 : p.pairs);
                hi = lo + (turned ? p.pairs : p.D / 2 - p.pairs);
            } else {
                lo = 8 * c, hi = 8 * c + 4;
            }
        }
    }
};

__device__ __forceinline__ void load_weights(const RopeTensor& t, int lo, int hi, float* w) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = i < 4 ? lo + i : hi + i - 4;
        w[i] = !t.w ? 1.f : t.w_f32 ? ((const float*)t.w)[at] : bf16_low(((const uint16_t*)t.w)[at]);
    }
}

// Where the lane's four pairs find their cosines and sines for one token; -1 where a position lies outside its axis's
// table.
template <int LAY>
__device__ __forceinline__ void find_angles(const RopeParams& p, const Lane<LAY>& me, int64_t b, int64_t l, int* at) {
    const int32_t* pos = p.pos + b * p.pos_batch + l * p.axes;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int pair = min((i < 2 ? me.pair : me.pair_hi) + (i & 1), p.pairs - 1);
        int axis = 0, length = p.length[0], base = p.base[0], width = p.width[0];
        for (int a = 1; a < p.axes; ++a) {
            const bool mine = pair >= p.first[a];
            axis = mine ? a : axis;
            length = mine ? p.length[a] : length;
            base = mine ? p.base[a] : base;
            width = mine ? p.width[a] : width;
        }
        const int where = pos[axis];
        at[i] = (uint32_t)where < (uint32_t)length ? base + where * width + pair : -1;
    }
}

// Cosines and sines there; NaN at -1.
__device__ __forceinline__ void load_angles(const RopeParams& p, const int* at, float* cs, float* sn) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 v = ((const f32x2*)p.table)[max(at[i], 0)];
        cs[i] = at[i] < 0 ? __builtin_nanf("") : v.x;
        sn[i] = at[i] < 0 ? __builtin_nanf("") : v.y;
    }
}

template <int LAY>
__device__ __forceinline__ void turn(float* v, const float* cs, const float* sn, float sign, const Lane<LAY>& me) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = LAY == kHalves ? i : 2 * i, k = LAY == kHalves ? i + 4 : 2 * i + 1;
        const bool turned = i < 2 ? me.turned : me.turned_hi;
        const float s = sign * sn[i];
        const float a = v[j] * cs[i] - v[k] * s, b = v[j] * s + v[k] * cs[i];
        v[j] = turned ? a : v[j];
        v[k] = turned ? b : v[k];
    }
}

// One wave's work: tokens t.wave_tokens * group .. and of each the heads of one chunk.  Lane group j of the wave has
// token j / t.wave_heads of them and head j % t.wave_heads, then every t.wave_heads-th head after it.
struct Item {
    int64_t b, l;
    int head;
    bool live;
    __device__ __forceinline__ Item(const RopeParams& p, const RopeTensor& t, uint32_t item, int lane) {
        const uint32_t group = item / (uint32_t)t.chunks, chunk = item - group * (uint32_t)t.chunks;
        const int j = lane / p.lanes, k = j / t.wave_heads;
        uint32_t token = group * (uint32_t)t.wave_tokens + (uint32_t)k;
        live = token < p.tokens;
        token = live ? token : p.tokens - 1;
        b = token / p.L;
        l = token - (uint32_t)b * p.L;
        head = (int)chunk * t.rows * t.wave_heads + j - k * t.wave_heads;
    }
};

template <typename T>
__device__ __forceinline__ T* row_of(const HeadRows& r, const Item& it, int head) {
    return (T*)r.p + it.b * r.b + it.l * r.l + head * r.h;
}

template <typename TI, typename TO, bool NORM, int LAY, bool NT>
__global__ __launch_bounds__(64 * kWaves) void axial_rope_kernel(RopeParams p) {
    const RopeTensor& t = p.t[blockIdx.y];
    const int lane = threadIdx.x & 63;
    const uint32_t item = p.first_item + blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= t.items) return;
    const Lane<LAY> me(p, lane);
    const Item it(p, t, item, lane);
    int at[4];
    if (p.pairs) find_angles(p, me, it.b, it.l, at);
    Row8<TI, LAY, NT> x[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u)
        if (u < t.rows) x[u].load(row_of<const TI>(t.x, it, min(it.head + u * t.wave_heads, t.heads - 1)), me.lo, me.hi);
    float w[8], cs[4], sn[4];
    if (NORM) load_weights(t, me.lo, me.hi, w);
    if (p.pairs) load_angles(p, at, cs, sn);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        if (u >= t.rows) break;
        const int head = it.head + u * t.wave_heads;
        float v[8];
        x[u].get(v);
        if (NORM) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[i] * v[i];
            sum = group_sum(me.live ? sum : 0.f, p.lanes);
            const float r = rsqrtf(sum * p.inv_d + p.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= r * w[i];
        }
        if (p.pairs) turn(v, cs, sn, p.sign, me);
        if (me.live && it.live && head < t.heads) Row8<TO, LAY, NT>::store(row_of<TO>(t.y, it, head), me.lo, me.hi, v);
    }
}

// Persistent: the workgroup's sums of the weight's gradient stay in its lanes' registers, eight columns each, until
// its last row, and leave as one row of partial sums.  They are added in a fixed order, so the result does not
// depend on which workgroup ends first.
template <typename TX, typename TG, int LAY, bool NT, int ROWS>
__global__ __launch_bounds__(64 * kWaves) void qk_norm_rope_backward_kernel(RopeParams p) {
    __shared__ float part[kWaves][512];
    const RopeTensor& t = p.t[blockIdx.y];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Lane<LAY> me(p, lane);
    float w[8], dw[8];
    load_weights(t, me.lo, me.hi, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[i] = 0.f;
    for (uint32_t item = blockIdx.x * kWaves + wave; item < t.items; item += gridDim.x * kWaves) {
        const Item it(p, t, item, lane);
        int at[4];
        if (p.pairs) find_angles(p, me, it.b, it.l, at);
        Row8<TX, LAY, NT> x[ROWS];
        Row8<TG, LAY, NT> g[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            if (u < t.rows) {
                const int head = min(it.head + u * t.wave_heads, t.heads - 1);
                x[u].load(row_of<const TX>(t.x, it, head), me.lo, me.hi);
                g[u].load(row_of<const TG>(t.g, it, head), me.lo, me.hi);
            }
        }
        float cs[4], sn[4];
        if (p.pairs) load_angles(p, at, cs, sn);
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            if (u >= t.rows) break;
            const int head = it.head + u * t.wave_heads;
            const bool live = me.live && it.live && head < t.heads;
            float xv[8], gv[8];
            x[u].get(xv);
            g[u].get(gv);
            if (p.pairs) turn(gv, cs, sn, -1.f, me);
            float sum = 0.f, dot = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum += xv[i] * xv[i];
                dot += gv[i] * w[i] * xv[i];
            }
            sum = group_sum(me.live ? sum : 0.f, p.lanes);
            dot = group_sum(me.live ? dot : 0.f, p.lanes);
            const float r = rsqrtf(sum * p.inv_d + p.eps);
            const float m = r * r * (dot * p.inv_d);
            float dx[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dx[i] = r * (gv[i] * w[i] - xv[i] * m);
                if (live) dw[i] += gv[i] * (xv[i] * r);
            }
            if (live) Row8<TX, LAY, NT>::store(row_of<TX>(t.y, it, head), me.lo, me.hi, dx);
        }
    }
    if (!t.dw) return;
    // lane groups, then waves
#pragma unroll
    for (int i = 0; i < 8; ++i)
        for (int apart = p.lanes; apart < 64; apart *= 2) dw[i] += __shfl_xor(dw[i], apart);
    if (lane < p.lanes && me.live) {
#pragma unroll
        for (int i = 0; i < 8; ++i) part[wave][i < 4 ? me.lo + i : me.hi + i - 4] = dw[i];
    }
    __syncthreads();
    for (int d = threadIdx.x; d < p.D; d += 64 * kWaves)
        t.dw_part[(int64_t)blockIdx.x * p.D + d] = (part[0][d] + part[1][d]) + (part[2][d] + part[3][d]);
}

// Sums of the workgroups' rows: 16 columns to a workgroup of 1024, 64 of its threads to a column.
__global__ __launch_bounds__(1024) void norm_weight_grad_kernel(RopeParams p) {
    __shared__ float part[64][17];
    const RopeTensor& t = p.t[blockIdx.y];
    if (!t.dw) return;
    const int col = threadIdx.x & 15, row = threadIdx.x >> 4, d = blockIdx.x * 16 + col;
    float sum = 0.f;
    if (d < p.D) {
#pragma unroll 8
        for (int i = row; i < t.parts; i += 64) sum += t.dw_part[(int64_t)i * p.D + d];
    }
    part[row][col] = sum;
    __syncthreads();
    for (int half = 32; half; half /= 2) {
        if (row < half) part[row][col] += part[row + half][col];
        __syncthreads();
    }
    if (row == 0 && d < p.D) t.dw[d] = part[0][col];
}

// How a tensor's head rows go over the waves: as many of a token's heads side by side as fit, several tokens where
// it has fewer heads than that, and up to `most` rows a lane group after each other.
void divide(const RopeParams& p, RopeTensor& t, int most, int cus) {
    const int groups = 64 / p.lanes;
    int side = 1;
    while (side < groups && side < t.heads) side *= 2;
    t.wave_heads = side;
    t.wave_tokens = groups / side;
    const int steps = (t.heads + side - 1) / side;
    const int64_t token_groups = ((int64_t)p.tokens + t.wave_tokens - 1) / t.wave_tokens;
    t.chunks = (steps + most - 1) / most;
    // few tokens: fewer rows to a wave, until every SIMD has a wave
    while (t.chunks < steps && token_groups * t.chunks < 4 * (int64_t)cus) t.chunks = std::min(steps, 2 * t.chunks);
    t.rows = (steps + t.chunks - 1) / t.chunks;
    t.chunks = (steps + t.rows - 1) / t.rows;
    t.items = (uint32_t)(token_groups * t.chunks);
}

// Whether what a tensor has in one place is whole lines of 128 bytes: a head's row, or a token's heads where they lie
// together (with less than a row between them).
bool whole_lines(const HeadRows& r, int heads, int D, int size) {
    return D * size % 128 == 0 || (r.h < 2 * D && (int64_t)heads * D * size % 128 == 0);
}

// Non-temporal loads and stores where a call moves more than the memory-side cache keeps for the next kernel, in pieces
// of whole lines.  Measured plain / non-temporal, us: 100 MB 18.4 / 20.8, 227 MB 51.7 / 46.2, 340 MB 62.6 / 58, 671 MB
// 117 / 108; but in pieces of 64 bytes 66.8 / 75, and 24 heads of 80 that lie apart, [batch][head][token], 339 MB 77.5 / 92,
// 699 MB 141 / 170.  Where a piece begins in a line does not matter (24 heads of 80 from 16 bytes behind one on, 699 MB
// 130 / 131, their gradients 262 / 258), nor 16 bytes between heads (240 / 223).  size_g: of the gradients' values, or 0.
bool streams(const RopeParams& p, int size_x, int size_y, int size_g) {
    int64_t heads = 0;
    bool lines = !p.halves || p.pairs * std::min({size_x, size_y, size_g ? size_g : size_x}) >= 128;
    for (int i = 0; i < p.tensors; ++i) {
        const RopeTensor& t = p.t[i];
        heads += t.heads;
        lines = lines && whole_lines(t.x, t.heads, p.D, size_x) && whole_lines(t.y, t.heads, p.D, size_y) &&
                (!size_g || whole_lines(t.g, t.heads, p.D, size_g));
    }
    return lines && (int64_t)p.tokens * heads * p.D * (size_x + size_y + size_g) > (int64_t)160 << 20;
}

template <typename TI, typename TO, bool NORM>
void launch(const RopeParams& p, dim3 grid, hipStream_t stream) {
    constexpr int kPlain = sizeof(TI) + sizeof(TO) == 4 ? kRow : kApart;
    const bool nt = streams(p, sizeof(TI), sizeof(TO), 0);
    if (p.halves)
        nt ? axial_rope_kernel<TI, TO, NORM, kHalves, true><<<grid, 64 * kWaves, 0, stream>>>(p)
           : axial_rope_kernel<TI, TO, NORM, kHalves, false><<<grid, 64 * kWaves, 0, stream>>>(p);
    else
        nt ? axial_rope_kernel<TI, TO, NORM, kPlain, true><<<grid, 64 * kWaves, 0, stream>>>(p)
           : axial_rope_kernel<TI, TO, NORM, kPlain, false><<<grid, 64 * kWaves, 0, stream>>>(p);
}

template <typename TX, typename TG, int LAY, bool NT>
hipError_t launch_backward(RopeParams p, int cus, hipStream_t stream) {
    int steps = 0;
    for (int i = 0; i < p.tensors; ++i) {
        divide(p, p.t[i], kRows, cus);  // no tokens: no items, and the weights' gradients are sums of nothing
        steps = std::max(steps, p.t[i].rows);
    }
    // Six rows in flight where there are as many: 360 MB 134 -> 115 us; but three rows of the same registers' waves 46 -> 56.
    const bool many = steps > 4;
    const void* kernel = many ? (const void*)qk_norm_rope_backward_kernel<TX, TG, LAY, NT, kRows>
                              : (const void*)qk_norm_rope_backward_kernel<TX, TG, LAY, NT, kBackRows>;
    uint32_t items = 0;
    for (int i = 0; i < p.tensors; ++i) {
        divide(p, p.t[i], many ? kRows : kBackRows, cus);
        items = std::max(items, p.t[i].items);
    }
    // as many workgroups as are resident at once
    const int resident = std::min(resident_blocks(kernel, 64 * kWaves, 0), kBackGroups);
    const int groups = (int)std::min<int64_t>((items + kWaves - 1) / kWaves, (resident * cus + p.tensors - 1) / p.tensors);
    for (int i = 0; i < p.tensors; ++i) p.t[i].parts = groups;
    if (groups) {
        const dim3 grid(groups, p.tensors);
        if (many)
            qk_norm_rope_backward_kernel<TX, TG, LAY, NT, kRows><<<grid, 64 * kWaves, 0, stream>>>(p);
        else
            qk_norm_rope_backward_kernel<TX, TG, LAY, NT, kBackRows><<<grid, 64 * kWaves, 0, stream>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!p.t[0].dw && !p.t[1].dw) return hipSuccess;
    norm_weight_grad_kernel<<<dim3((p.D + 15) / 16, p.tensors), 1024, 0, stream>>>(p);
    return hipGetLastError();
}

template <typename TX, typename TG>
hipError_t launch_backward(const RopeParams& p, int cus, hipStream_t stream) {
    constexpr int kPlain = sizeof(TX) + sizeof(TG) == 4 ? kRow : kApart;
    const bool nt = streams(p, sizeof(TX), sizeof(TX), sizeof(TG));
    if (p.halves) return nt ? launch_backward<TX, TG, kHalves, true>(p, cus, stream) : launch_backward<TX, TG, kHalves, false>(p, cus, stream);
    return nt ? launch_backward<TX, TG, kPlain, true>(p, cus, stream) : launch_backward<TX, TG, kPlain, false>(p, cus, stream);
}

}  // namespace

hipError_t launch_axial_rope(RopeParams p, bool norm, bool in_f32, bool out_f32, int cus, hipStream_t stream) {
    uint32_t items = 0;
    for (int i = 0; i < p.tensors; ++i) {
        divide(p, p.t[i], kRows, cus);
        items = std::max(items, p.t[i].items);
    }
    // a grid holds fewer than 2^32 threads, which more than 2^26 items of a wave each pass
    for (p.first_item = 0; p.first_item < items; p.first_item += kMostItems) {
        const dim3 grid((std::min(items - p.first_item, kMostItems) + kWaves - 1) / kWaves, p.tensors);
        if (!norm)
            in_f32 ? launch<float, float, false>(p, grid, stream) : launch<bf16_t, bf16_t, false>(p, grid, stream);
        else if (in_f32)
            out_f32 ? launch<float, float, true>(p, grid, stream) : launch<float, bf16_t, true>(p, grid, stream);
        else
            out_f32 ? launch<bf16_t, float, true>(p, grid, stream) : launch<bf16_t, bf16_t, true>(p, grid, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int norm_rope_backward_groups(int cus) { return kBackGroups * cus; }

hipError_t launch_qk_norm_rope_backward(const RopeParams& p, bool x_f32, bool g_f32, int cus, hipStream_t stream) {
    if (x_f32) return g_f32 ? launch_backward<float, float>(p, cus, stream) : launch_backward<float, bf16_t>(p, cus, stream);
    return g_f32 ? launch_backward<bf16_t, float>(p, cus, stream) : launch_backward<bf16_t, bf16_t>(p, cus, stream);
}

}  // namespace orbit
