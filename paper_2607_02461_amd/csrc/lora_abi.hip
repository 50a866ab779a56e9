// Entry points of the low-rank adapters: plans, argument checks, workspaces, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "abi.h"
#include "device.h"
#include "internal.h"

using namespace orbit;

namespace {

constexpr int64_t kMaxRows = INT32_MAX;
constexpr int64_t kMaxTiles = (int64_t)1 << 22;  // workgroups of up to 512 threads, one to a tile, stay below 2^32 threads
constexpr int64_t kMaxWidth = (int64_t)1 << 21;
constexpr int32_t kMaxAdapters = 65535;

orbit_status lora_upload_dev(orbit_lora p, int dev) {
    std::lock_guard<std::mutex> lk(p->mu);
    if (p->dev_lists[dev]) return ORBIT_OK;
    void* d = nullptr;
    const orbit_status st = upload_copy("lora_plan upload", p->lists.data(), p->lists.size(), &d);
    p->dev_lists[dev] = (unsigned char*)d;
    return st;
}

// Tiles and splits of checked arguments.
void fill(orbit_lora p, int64_t segments, const int64_t* starts, const int32_t* adapters, int32_t n, const int32_t* ranks, const float* scales) {
    std::vector<LoraTile> tiles;
    std::vector<std::vector<LoraTile>> of(n + 1);
    auto add = [&](int64_t row, int64_t end, int32_t a) {
        const bool none = a < 0 || ranks[a] == 0;
        for (; row < end; row += kLoraTileRows) {
            LoraTile t{};
            t.row = (int32_t)row;
            t.rows = (int32_t)std::min<int64_t>(kLoraTileRows, end - row);
            t.adapter = none ? -1 : a;
            t.rank = none ? 0 : ranks[a];
            t.scale = none ? 0.f : scales[a];
            of[none ? n : a].push_back(t);
            p->tile_rows = std::max(p->tile_rows, t.rows);
        }
    };
    if (segments == 0 || starts[0] > 0) add(0, segments ? starts[0] : p->rows, -1);
    for (int64_t s = 0; s < segments; ++s) add(starts[s], s + 1 < segments ? starts[s + 1] : p->rows, adapters[s]);
    for (auto& list : of) tiles.insert(tiles.end(), list.begin(), list.end());
    p->tiles = (int64_t)tiles.size();
    for (int a = 0; a < n; ++a) p->most_tiles = std::max(p->most_tiles, (int32_t)of[a].size());

    std::vector<unsigned char>& blob = p->lists;
    auto append = [&](const void* data, size_t bytes) {
        const size_t at = (blob.size() + 15) / 16 * 16;
        blob.resize(std::max<size_t>(at + bytes, 16));
        if (bytes) std::memcpy(blob.data() + at, data, bytes);
        return at;
    };
    append(tiles.data(), tiles.size() * sizeof(LoraTile));
    for (int level = 0; level < kLoraLevels; ++level) {
        const bool whole = level == kLoraLevels - 1;
        const int step = 4 << level;
        std::vector<LoraSplit> list;
        std::vector<int32_t> first(1, 0);
        int32_t at = 0;
        for (int a = 0; a < n; ++a) {
            const int32_t end = at + (int32_t)of[a].size();
            if (whole)
                list.push_back({at, end});
            else
                for (int32_t t = at; t < end; t += step) list.push_back({t, std::min(t + step, end)});
            at = end;
            first.push_back((int32_t)list.size());
        }
        p->splits[level] = (int64_t)list.size();
        p->at_splits[level] = append(list.data(), list.size() * sizeof(LoraSplit));
        p->at_first[level] = append(first.data(), first.size() * sizeof(int32_t));
    }
}

size_t padded(int64_t bytes) { return ((size_t)bytes + 255) / 256 * 256; }

// Sizes of a call and its buffers in the workspace.
struct Layout {
    int splits = 1;         // of the shrink's contraction
    int level = 0;          // of the gradients' splits
    bool together = false, direct = false;
    size_t g = 0, g_turned = 0, h_turned = 0, at = 0, bt = 0, grad_x = 0, grad_y = 0, bytes = 0;
    int64_t ldn = 0;        // rows of the turned B
};

Layout forward_layout(orbit_lora p, int64_t K, int R, int cus) {
    Layout l;
    if (p->tile_rows <= kLoraFewRows) return l;
    l.splits = lora_splits((int)p->tiles, K, cus);
    l.bytes = padded(l.splits * lora_sum_bytes(p->tiles, R));
    return l;
}

Layout backward_layout(orbit_lora p, int64_t K, int64_t N, int R, int cus) {
    Layout l;
    const int64_t n = p->adapters;
    l.ldn = (N + 7) / 8 * 8;
    l.splits = lora_splits((int)p->tiles, N, cus);
    // Gradients: an adapter's rows in one go where no adapter has more than 4 tiles.  Else as many tiles to a split as
    // leave 2 splits and 128 columns to a compute unit; from 16 on a workgroup's waves share the columns and add up in
    // LDS, with fewer they have columns of their own (a training step of 9216 rows 3072 -> 9216, 16 tiles: 209 us sharing,
    // 226 else; 3072 -> 3072, 8 tiles: 128 and 120).
    const int64_t chunks = ((K + 127) / 128 + (N + 127) / 128) * (R > 64 ? 2 : 1);
    if (p->most_tiles <= 4) {
        l.level = kLoraLevels - 1;
        l.together = true;
    } else {
        l.level = kLoraLevels - 2;
        while (l.level > 0 && p->splits[l.level] * chunks < 2 * (int64_t)cus) --l.level;
        l.together = l.level > 1;
    }
    l.direct = l.level == kLoraLevels - 1;
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += padded(bytes);
        return here;
    };
    l.g = take(l.splits * lora_sum_bytes(p->tiles, R));
    l.g_turned = take(lora_operand_bytes(p->tiles, R));
    l.h_turned = take(lora_operand_bytes(p->tiles, R));
    l.at = take(n * K * R * 2);
    l.bt = take(n * R * l.ldn * 2);
    l.grad_x = take(l.direct ? 0 : p->splits[l.level] * R * K * (int64_t)sizeof(float));
    l.grad_y = take(l.direct ? 0 : p->splits[l.level] * R * N * (int64_t)sizeof(float));
    l.bytes = at;
    return l;
}

orbit_status check_sizes(const char* who, orbit_lora p, int64_t K, int64_t N, int32_t R) {
    if (!p) return fail(ORBIT_EINVAL, "%s: plan is NULL", who);
    if (K <= 0 || K % 8) return fail(ORBIT_EINVAL, "%s: K=%lld must be a positive multiple of 8", who, (long long)K);
    if (N < 1) return fail(ORBIT_EINVAL, "%s: N=%lld must be positive", who, (long long)N);
    if (R < 8 || R % 8 || R > kLoraMaxRank)
        return fail(ORBIT_EUNSUPPORTED, "%s: R=%d, a multiple of 8 up to %d is implemented", who, R, kLoraMaxRank);
    if (p->max_rank > R) return fail(ORBIT_EINVAL, "%s: the plan has an adapter of rank %d, above R=%d", who, p->max_rank, R);
    if (K > kMaxWidth || N > kMaxWidth)
        return fail(ORBIT_EUNSUPPORTED, "%s: K=%lld or N=%lld above %lld", who, (long long)K, (long long)N, (long long)kMaxWidth);
    return ORBIT_OK;
}

// An output at base's place has base's rows; the other wide inputs are read after an output's first values are written.
orbit_status check_places(const char* who, const char* name, const void* y, int64_t ldy, const void* base, int64_t ldb, int64_t rows,
                          const void* x, const void* dy) {
    if (!y) return ORBIT_OK;
    if (y == base && rows > 1 && ldy != ldb) return fail(ORBIT_EINVAL, "%s: %s lies on base with another row stride", who, name);
    if (y == x || y == dy) return fail(ORBIT_EINVAL, "%s: %s lies on an input other than base", who, name);
    return ORBIT_OK;
}

orbit_status lists_on(const char* who, orbit_lora p, int dev, const unsigned char** out) {
    std::lock_guard<std::mutex> lk(p->mu);
    if (!p->dev_lists[dev])
        return fail(ORBIT_EINVAL, "%s: the plan has no tables on device %d: create it with that device current, or call "
                                  "lora_plan_upload there first", who, dev);
    *out = p->dev_lists[dev];
    return ORBIT_OK;
}

}  // namespace

extern "C" {

orbit_status lora_plan(int64_t M, int64_t segments, const int64_t* starts, const int32_t* adapters, int32_t n_adapters, const int32_t* ranks,
                       const float* scales, orbit_lora* out) {
    const char* who = "lora_plan";
    clear_error();
    if (!out) return fail(ORBIT_EINVAL, "%s: out is NULL", who);
    *out = nullptr;
    if (M < 0 || segments < 0) return fail(ORBIT_EINVAL, "%s: negative M or number of segments", who);
    if (M > kMaxRows) return fail(ORBIT_EUNSUPPORTED, "%s: M=%lld above 2^31-1 rows", who, (long long)M);
    if (n_adapters < 1) return fail(ORBIT_EINVAL, "%s: %d adapters", who, n_adapters);
    if (n_adapters > kMaxAdapters) return fail(ORBIT_EUNSUPPORTED, "%s: more than %d adapters", who, kMaxAdapters);
    if (!ranks || !scales || (segments && (!starts || !adapters))) return fail(ORBIT_EINVAL, "%s: a list is NULL", who);
    int64_t tiles = segments ? starts[0] / kLoraTileRows + 1 : M / kLoraTileRows + 1;
    for (int64_t s = 0; s < segments; ++s) {
        const int64_t end = s + 1 < segments ? starts[s + 1] : M;
        if (starts[s] < 0 || starts[s] > end)
            return fail(ORBIT_EINVAL, "%s: segment %lld begins at row %lld and ends at %lld", who, (long long)s, (long long)starts[s], (long long)end);
        if (adapters[s] < -1 || adapters[s] >= n_adapters)
            return fail(ORBIT_EINVAL, "%s: segment %lld has adapter %d, -1..%d exist", who, (long long)s, adapters[s], n_adapters - 1);
        tiles += (end - starts[s] + kLoraTileRows - 1) / kLoraTileRows;
    }
    if (tiles > kMaxTiles) return fail(ORBIT_EUNSUPPORTED, "%s: more than %lld tiles of %d rows", who, (long long)kMaxTiles, kLoraTileRows);
    int32_t max_rank = 0;
    for (int a = 0; a < n_adapters; ++a) {
        if (ranks[a] < 0) return fail(ORBIT_EINVAL, "%s: adapter %d has rank %d", who, a, ranks[a]);
        if (ranks[a] > kLoraMaxRank) return fail(ORBIT_EUNSUPPORTED, "%s: adapter %d has rank %d, up to %d are implemented", who, a, ranks[a], kLoraMaxRank);
        if (!std::isfinite(scales[a])) return fail(ORBIT_EINVAL, "%s: the scale of adapter %d is not finite", who, a);
        max_rank = std::max(max_rank, ranks[a]);
    }
    orbit_lora p = new (std::nothrow) orbit_lora_s;
    if (!p) return fail(ORBIT_ENOMEM, "%s: out of host memory", who);
    p->rows = M;
    p->adapters = n_adapters;
    p->max_rank = max_rank;
    try {
        fill(p, segments, starts, adapters, n_adapters, ranks, scales);
    } catch (...) {
        delete p;
        return fail(ORBIT_ENOMEM, "%s: out of host memory", who);
    }
    int dev;
    orbit_status st = device_for_upload(&dev);
    if (st == ORBIT_OK && dev >= 0) st = lora_upload_dev(p, dev);
    if (st != ORBIT_OK) {
        delete p;
        return st;
    }
    *out = p;
    return ORBIT_OK;
}

orbit_status lora_plan_upload(orbit_lora p) {
    clear_error();
    if (!p) return fail(ORBIT_EINVAL, "lora_plan_upload: plan is NULL");
    int dev;
    DeviceInfo info;
    const orbit_status st = current_device(&dev, &info);
    return st != ORBIT_OK ? st : lora_upload_dev(p, dev);
}

void lora_plan_destroy(orbit_lora p) {
    if (!p) return;
    free_per_device(p->dev_lists);
    delete p;
}

orbit_status lora_add_workspace_size(orbit_lora p, int64_t K, int64_t N, int32_t R, int32_t backward, size_t* bytes) {
    const char* who = "lora_add_workspace_size";
    clear_error();
    if (!bytes) return fail(ORBIT_EINVAL, "%s: null output pointer", who);
    *bytes = 0;
    orbit_status st = check_sizes(who, p, K, N, R);
    if (st != ORBIT_OK) return st;
    int dev;
    DeviceInfo info;
    st = current_device(&dev, &info);
    if (st != ORBIT_OK) return st;
    *bytes = backward ? backward_layout(p, K, N, R, info.cus).bytes : forward_layout(p, K, R, info.cus).bytes;
    return ORBIT_OK;
}

orbit_status lora_add(orbit_lora p, const uint16_t* X, int64_t ldx, const uint16_t* A, const uint16_t* B, int64_t K, int64_t N, int32_t R,
                      const void* base, int64_t ldb, int32_t dtype, void* Y, int64_t ldy, float* h, void* workspace, size_t workspace_bytes,
                      void* stream) {
    const char* who = "lora_add";
    clear_error();
    orbit_status st = check_sizes(who, p, K, N, R);
    if (st != ORBIT_OK) return st;
    if (dtype != ORBIT_OUT_F32 && dtype != ORBIT_OUT_BF16) return fail(ORBIT_EINVAL, "%s: unknown type %d", who, dtype);
    if (ldx < K || ldy < N || (base && ldb < N)) return fail(ORBIT_EINVAL, "%s: a row stride is below the row's length", who);
    if (p->rows == 0) return ORBIT_OK;
    const int size = dtype == ORBIT_OUT_BF16 ? 2 : 4;
    if (!X || !A || !B || !Y) return fail(ORBIT_EINVAL, "%s: null device pointer", who);
    if (!aligned(X, 2) || !aligned(A, 16) || !aligned(B, 16) || !aligned(base, size) || !aligned(Y, size) || !aligned(h, 16))
        return fail(ORBIT_EINVAL, "%s: misaligned pointer (A, B and h need 16 bytes)", who);
    st = check_places(who, "Y", Y, ldy, base, ldb, p->rows, X, nullptr);
    if (st != ORBIT_OK) return st;
    int dev;
    DeviceInfo info;
    st = current_device(&dev, &info);
    if (st != ORBIT_OK) return st;
    const unsigned char* lists = nullptr;
    st = lists_on(who, p, dev, &lists);
    if (st != ORBIT_OK) return st;
    const Layout l = forward_layout(p, K, R, info.cus);
    if (l.bytes && (!workspace || !aligned(workspace, 16) || workspace_bytes < l.bytes))
        return fail(ORBIT_EINVAL, "%s: takes a workspace of %zu bytes, aligned to 16", who, l.bytes);
    if (p->tile_rows <= kLoraFewRows) {
        LoraRows r{};
        r.tiles = (const LoraTile*)lists;
        r.x = X;
        r.a = A;
        r.b = B;
        r.ldx = ldx;
        r.K = K;
        r.N = N;
        r.R = R;
        r.base = base;
        r.ldb = ldb;
        r.y = Y;
        r.ldy = ldy;
        r.h = h;
        const hipError_t e = launch_lora_rows(r, (int)p->tiles, p->tile_rows, dtype == ORBIT_OUT_F32, info.cus, (hipStream_t)stream);
        return e == hipSuccess ? ORBIT_OK : hip_fail(e, who);
    }
    LoraShrink s{};
    s.tiles = (const LoraTile*)lists;
    s.x = X;
    s.ldx = ldx;
    s.K = K;
    s.pool = A;
    s.ldp = K;
    s.R = R;
    s.h = (float*)workspace;
    hipError_t e = launch_lora_shrink(s, (int)p->tiles, l.splits, (hipStream_t)stream);
    if (e != hipSuccess) return hip_fail(e, who);
    LoraExpand x{};
    x.tiles = s.tiles;
    x.h = s.h;
    x.sum = h;
    x.splits = l.splits;
    x.R = R;
    x.N = N;
    x.pool = B;
    x.base = base;
    x.ldb = ldb;
    x.y = Y;
    x.ldy = ldy;
    e = launch_lora_expand(x, (int)p->tiles, dtype == ORBIT_OUT_F32, info.cus, (hipStream_t)stream);
    return e == hipSuccess ? ORBIT_OK : hip_fail(e, who);
}

orbit_status lora_add_backward(orbit_lora p, const uint16_t* dY, int64_t ldd, const uint16_t* X, int64_t ldx, const uint16_t* A, const uint16_t* B,
                               const float* h, int64_t K, int64_t N, int32_t R, const uint16_t* base, int64_t ldb, uint16_t* dX, int64_t lddx,
                               float* dA, float* dB, void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "lora_add_backward";
    clear_error();
    orbit_status st = check_sizes(who, p, K, N, R);
    if (st != ORBIT_OK) return st;
    if (ldd < N || ldx < K || lddx < K || (base && ldb < K)) return fail(ORBIT_EINVAL, "%s: a row stride is below the row's length", who);
    if (!A || !B || !dA || !dB || (p->rows && (!dY || !X || !h || !dX))) return fail(ORBIT_EINVAL, "%s: null device pointer", who);
    if (!aligned(dY, 2) || !aligned(X, 2) || !aligned(base, 2) || !aligned(dX, 2) || !aligned(A, 16) || !aligned(B, 16) || !aligned(h, 16) ||
        !aligned(dA, 16) || !aligned(dB, 16))
        return fail(ORBIT_EINVAL, "%s: misaligned pointer (A, B, h, dA and dB need 16 bytes)", who);
    st = check_places(who, "dX", dX, lddx, base, ldb, p->rows, X, dY);
    if (st != ORBIT_OK) return st;
    int dev;
    DeviceInfo info;
    st = current_device(&dev, &info);
    if (st != ORBIT_OK) return st;
    const unsigned char* lists = nullptr;
    st = lists_on(who, p, dev, &lists);
    if (st != ORBIT_OK) return st;
    const Layout l = backward_layout(p, K, N, R, info.cus);
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < l.bytes)
        return fail(ORBIT_EINVAL, "%s: takes a workspace of %zu bytes, aligned to 16", who, l.bytes);
    // launch grids hold fewer than 2^32 threads
    if (p->splits[l.level] * ((K + 127) / 128 + (N + 127) / 128) > (int64_t)1 << 23 ||
        (R / 8) * ((K / 8 + l.ldn / 8) * p->adapters + 8 * p->tiles) > (int64_t)1 << 31)
        return fail(ORBIT_EUNSUPPORTED, "%s: the launch grids are too large", who);
    unsigned char* const ws = (unsigned char*)workspace;
    hipStream_t hs = (hipStream_t)stream;
    hipError_t e;
    LoraGrad d{};
    if (p->rows) {
        LoraTurn t{};
        t.a = A;
        t.b = B;
        t.at = (uint16_t*)(ws + l.at);
        t.bt = (uint16_t*)(ws + l.bt);
        t.K = K;
        t.N = N;
        t.ldn = l.ldn;
        t.R = R;
        t.adapters = p->adapters;
        t.tiles = (const LoraTile*)lists;
        t.count = p->tiles;
        t.h = h;
        t.turned = (uint16_t*)(ws + l.h_turned);
        e = launch_lora_turn(t, hs);
        if (e != hipSuccess) return hip_fail(e, who);
        LoraShrink s{};
        s.tiles = t.tiles;
        s.x = dY;
        s.ldx = ldd;
        s.K = N;
        s.pool = t.bt;
        s.ldp = l.ldn;
        s.R = R;
        s.h = (float*)(ws + l.g);
        e = launch_lora_shrink(s, (int)p->tiles, l.splits, hs);
        if (e != hipSuccess) return hip_fail(e, who);
        LoraExpand x{};
        x.tiles = t.tiles;
        x.h = s.h;
        x.turned = (uint16_t*)(ws + l.g_turned);
        x.splits = l.splits;
        x.R = R;
        x.N = K;
        x.pool = t.at;
        x.base = base;
        x.ldb = ldb;
        x.y = dX;
        x.ldy = lddx;
        e = launch_lora_expand(x, (int)p->tiles, false, info.cus, hs);
        if (e != hipSuccess) return hip_fail(e, who);
        d.tiles = t.tiles;
    }
    d.list = (const LoraSplit*)(lists + p->at_splits[l.level]);
    d.first = (const int32_t*)(lists + p->at_first[l.level]);
    d.side[0] = {X, ldx, K, (const uint16_t*)(ws + l.g_turned), (float*)(ws + l.grad_x), dA};
    d.side[1] = {dY, ldd, N, (const uint16_t*)(ws + l.h_turned), (float*)(ws + l.grad_y), dB};
    d.R = R;
    d.direct = l.direct;
    e = launch_lora_grad(d, (int)p->splits[l.level], p->adapters, l.together, hs);
    return e == hipSuccess ? ORBIT_OK : hip_fail(e, who);
}

}  // extern "C"
