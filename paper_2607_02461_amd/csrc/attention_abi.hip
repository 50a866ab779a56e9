// Entry points of attention: plans, argument checks, workspaces, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <new>
#include <utility>

#include "abi.h"
#include "device.h"
#include "internal.h"

using namespace orbit;

namespace {

constexpr int64_t kMaxTokens = INT32_MAX;
constexpr int32_t kMaxHeads = 32767;
constexpr int64_t kMaxGroups = ((int64_t)1 << 24) - 8;   // workgroups of 256 threads to a launch
constexpr int64_t kMostParts = (int64_t)1 << 20;         // of divided tiles: a join has up to 2048 threads for each
constexpr int64_t kMaxStride = (int64_t)1 << 24;         // elements from a token to the next: a tile's rows lie within 2^32 bytes

struct Sequence {
    int64_t q_start, q_len, k_start, k_len;
};

// A list's tiles, with what each costs in units of the other side's tiles.
struct Work {
    AttnTile tile;
    int64_t cost;
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// What a list's tiles are divided for.
struct Card {
    int64_t slots;   // workgroups that are resident
    int64_t rows;    // of a tile
    int64_t step;    // keys (or queries) in a unit of cost
    double begin;    // units that a workgroup's begin and end take,
    double join;     // that a join's launch takes,
    double part;     // and that each part's sums take, written and read again
};

// Divides tiles along the other side where that is estimated to end earlier: where few long tiles leave the card partly idle.  Parts
// leave their sums in rows of their own, which a join adds up.  A list ends after as many rounds of its longest tile as there are,
// or after what each slot has and most of one, whichever is earlier.  The longest come first: workgroups start in the list's order,
// so the last to start are the shortest.
// Measured, us (D = 128, whole / in parts): forward 1024 tokens in 24 heads, causal, 22 / 30; in 4 heads, not causal, 21 / 17;
// single tokens over 2000 keys in 8 key heads, 4 sequences, 19 / 12.
// (Dividing the last, partial round of several as well, 1728 equal tiles on 512 slots for example, gained nothing, 502 and 504 us:
// the workgroups of that round run alone on their compute units and take half the time.)
void divide(std::vector<Work>& work, int64_t kv_heads, const Card& card, int64_t* slot_rows, std::vector<AttnJoin>* joins, std::vector<AttnTile>* out) {
    int64_t total = 0, longest = 0;
    for (const Work& w : work) total += w.cost, longest = std::max(longest, w.cost);
    const double share = (double)total * kv_heads / card.slots;
    auto ends = [&](int64_t count, int64_t most) {
        const double each = most + card.begin, rounds = (double)count * kv_heads / card.slots;
        return rounds <= 1.0 ? each : std::min(std::ceil(rounds) * each, share + rounds * card.begin + 0.8 * each);
    };
    auto parts_of = [](int64_t cost, int64_t part) { return std::max<int64_t>(1, (2 * cost + part) / (2 * part)); };
    int64_t part = INT64_MAX / 4;
    double best = ends((int64_t)work.size(), longest);
    for (int64_t size = (longest + 1) / 2; share < longest && size >= 2; size -= 1 + size / (work.size() > 4096 ? 4 : 16)) {
        int64_t count = 0, parts = 0, most = 0;
        for (const Work& w : work) {
            const int64_t n = parts_of(w.cost, size);
            count += n;
            if (n > 1) parts += n;
            most = std::max(most, ceil_div(w.cost, n));
        }
        if (count > (kMaxGroups - 8192) / kv_heads || parts > kMostParts / kv_heads) break;
        const double time = ends(count, most) + card.join + card.part * parts * kv_heads;
        if (time < best) best = time, part = size;
    }
    std::vector<Work> all;
    for (const Work& w : work) {
        const AttnTile& t = w.tile;
        const int64_t k = parts_of(w.cost, part);
        if (k == 1) {
            all.push_back(w);
            continue;
        }
        joins->push_back({t.q_start, t.q_len, t.k_start, t.k_len, t.first, (int32_t)*slot_rows, (int32_t)k, (int32_t)card.rows});
        for (int64_t j = 0; j < k; ++j) {
            Work piece = w;
            const int64_t from = w.cost * j / k, to = w.cost * (j + 1) / k;
            piece.cost = to - from;
            piece.tile.begin = (int32_t)(t.begin + from * card.step);
            piece.tile.end = (int32_t)std::min<int64_t>(t.end, t.begin + to * card.step);
            piece.tile.slot = (int32_t)*slot_rows;
            *slot_rows += card.rows;
            all.push_back(piece);
        }
    }
    std::stable_sort(all.begin(), all.end(), [](const Work& a, const Work& b) { return a.cost > b.cost; });
    for (const Work& w : all) out->push_back(w.tile);
}

// Lists of checked sequences.
void fill(orbit_attention p, const std::vector<Sequence>& sequences) {
    const int64_t group = p->heads / p->kv_heads, queries = std::max<int64_t>(1, 64 / group);   // of 64 rows
    std::vector<Work> whole, wide, few, every, keys;
    // Wide tiles load keys and values half as often, but a compute unit has one workgroup of them, whose begin and end nothing
    // else covers: 32760 tokens in 40 heads of 128 19.0 ms instead of 20.0, 4608 tokens 512 us instead of 502, over 512 keys
    // 442 us instead of 418.  (Measured at D = 128; the plan does not know D, and heads of up to 64 values go by the same rule.)
    int64_t wide_tiles = 0, wide_cost = 0;
    for (const Sequence& s : sequences) {
        const int64_t tiles = s.q_len * group > kAttnFewRows ? ceil_div(s.q_len * group, kAttnWideRows) : 0;
        wide_tiles += tiles;
        wide_cost += tiles * (p->causal ? (s.k_len + 1) / 2 : s.k_len);
    }
    const int64_t wide_groups = wide_tiles * p->kv_heads;
    const bool widely = wide_groups >= 2 * 256 && wide_groups < kMaxGroups / 2 && wide_cost >= 8192 * wide_tiles;
    for (const Sequence& s : sequences) {
        const int64_t rows = s.q_len * group;
        auto tiles = [&](std::vector<Work>& to, int64_t most, int64_t unit) {
            for (int64_t first = 0; first < rows; first += most) {
                const int64_t last = (std::min(first + most, rows) - 1) / group;   // the tile's last query
                const int64_t end = p->causal ? std::min(s.k_len, std::max<int64_t>(0, last + 1 + s.k_len - s.q_len)) : s.k_len;
                to.push_back({{(int32_t)s.q_start, (int32_t)s.q_len, (int32_t)s.k_start, (int32_t)s.k_len, (int32_t)first, 0, (int32_t)end, -1},
                              ceil_div(end, unit)});
            }
        };
        if (rows <= kAttnFewRows)
            tiles(few, kAttnFewRows, 128);
        else if (widely)
            tiles(wide, kAttnWideRows, 64);
        else
            tiles(whole, kAttnRows, 64);
        tiles(every, kAttnRows, 64);
        for (int64_t first = 0; first < s.k_len; first += kAttnRows) {
            // the first query that sees the tile's first key
            const int64_t begin = p->causal ? std::min(s.q_len, std::max<int64_t>(0, first - (s.k_len - s.q_len))) : 0;
            const AttnTile t{(int32_t)s.q_start, (int32_t)s.q_len, (int32_t)s.k_start, (int32_t)s.k_len, (int32_t)first, (int32_t)begin, (int32_t)s.q_len, -1};
            keys.push_back({t, ceil_div(s.q_len - begin, queries)});
        }
    }
    std::vector<AttnTile> list[kAttnLists];
    std::vector<AttnJoin> joins, row_joins, key_joins;
    // Resident on 256 compute units: two workgroups of four waves, one of eight, or one whose buffers take the LDS.  A unit takes 0.9
    // us forward (1.2 of few rows), 1.2 for the rows' gradients and 1.6 for the keys', a join 5 to 8 us, a part's 64 KB (16 of few
    // rows, 128 of keys) twice their time at 4.7 TB/s.  All of that is for D = 128: the plan does not know D.  Heads of up to 64 values
    // have three workgroups of four waves to a compute unit forward and for the keys' gradients, and units of about half the time.
    divide(whole, p->kv_heads, {512, kAttnRows, 64, 1.5, 6.0, 0.030}, &p->slots, &joins, &list[kAttnForward]);
    divide(wide, p->kv_heads, {256, kAttnWideRows, 64, 2.0, 6.0, 0.060}, &p->slots, &joins, &list[kAttnForwardWide]);
    divide(few, p->kv_heads, {256, kAttnFewRows, 128, 2.5, 3.0, 0.004}, &p->slots, &joins, &list[kAttnFew]);
    divide(every, p->kv_heads, {512, kAttnRows, 64, 1.5, 5.0, 0.023}, &p->row_slots, &row_joins, &list[kAttnRowGrads]);
    divide(keys, p->kv_heads, {512, kAttnRows, queries, 1.5, 4.0, 0.035}, &p->key_slots, &key_joins, &list[kAttnKeyGrads]);

    std::vector<unsigned char>& blob = p->lists;
    auto append = [&](int which, const void* data, size_t count, size_t size) {
        p->at[which] = (blob.size() + 15) / 16 * 16;
        p->count[which] = (int64_t)count;
        blob.resize(std::max<size_t>(p->at[which] + count * size, 16));
        if (count) std::memcpy(blob.data() + p->at[which], data, count * size);
    };
    for (int i : {kAttnForward, kAttnForwardWide, kAttnFew, kAttnRowGrads, kAttnKeyGrads}) append(i, list[i].data(), list[i].size(), sizeof(AttnTile));
    append(kAttnJoins, joins.data(), joins.size(), sizeof(AttnJoin));
    append(kAttnRowJoins, row_joins.data(), row_joins.size(), sizeof(AttnJoin));
    append(kAttnKeyJoins, key_joins.data(), key_joins.size(), sizeof(AttnJoin));
}

orbit_status upload_dev(orbit_attention p, int dev) {
    std::lock_guard<std::mutex> lk(p->mu);
    if (p->dev_lists[dev]) return ORBIT_OK;
    void* d = nullptr;
    const orbit_status st = upload_copy("attention_plan upload", p->lists.data(), p->lists.size(), &d);
    p->dev_lists[dev] = (unsigned char*)d;
    return st;
}

orbit_status lists_on(const char* who, orbit_attention p, int dev, const unsigned char** out) {
    std::lock_guard<std::mutex> lk(p->mu);
    if (!p->dev_lists[dev])
        return fail(ORBIT_EINVAL, "%s: the plan has no tables on device %d: create it with that device current, or call "
                                  "attention_plan_upload there first", who, dev);
    *out = p->dev_lists[dev];
    return ORBIT_OK;
}

// Whether two of the intervals (start, length) have a token in common
bool overlap(std::vector<std::pair<int64_t, int64_t>> v) {
    std::sort(v.begin(), v.end());
    int64_t end = 0;
    for (const auto& [start, length] : v) {
        if (length == 0) continue;
        if (start < end) return true;
        end = start + length;
    }
    return false;
}

orbit_status check_dim(const char* who, orbit_attention p, int64_t D) {
    if (!p) return fail(ORBIT_EINVAL, "%s: plan is NULL", who);
    if (D < 8 || D % 8 || D > kAttnMaxDim)
        return fail(ORBIT_EUNSUPPORTED, "%s: head size %lld, a multiple of 8 up to %d is implemented", who, (long long)D, kAttnMaxDim);
    return ORBIT_OK;
}

orbit_status check_heads(const char* who, const char* name, const orbit_heads* t, int64_t tokens, int32_t heads, int64_t D, bool f32,
                         bool output, AttnHeads* out) {
    if (!t) return fail(ORBIT_EINVAL, "%s: %s is NULL", who, name);
    if (t->heads != heads) return fail(ORBIT_EINVAL, "%s: %s has %d heads, the plan %d", who, name, t->heads, heads);
    if (t->dtype != ORBIT_OUT_BF16 && !(f32 && t->dtype == ORBIT_OUT_F32)) return fail(ORBIT_EINVAL, "%s: %s has type %d", who, name, t->dtype);
    const int unit = t->dtype == ORBIT_OUT_F32 ? 4 : 8;
    if (tokens == 0) return ORBIT_OK;
    if (!t->data) return fail(ORBIT_EINVAL, "%s: %s is a null device pointer", who, name);
    if (!aligned(t->data, 16) || (tokens > 1 && t->token % unit) || (heads > 1 && t->head % unit))
        return fail(ORBIT_EINVAL, "%s: %s must be aligned to 16 bytes, its strides too", who, name);
    if ((tokens > 1 && (t->token < 0 || t->token > kMaxStride)) || (heads > 1 && (t->head < 0 || t->head > ((int64_t)1 << 50) / heads)))
        return fail(ORBIT_EINVAL, "%s: %s has a stride out of range", who, name);
    out->p = t->data;
    out->token = tokens > 1 ? t->token : 0;
    out->head = heads > 1 ? t->head : 0;
    if (!output) return ORBIT_OK;
    // a token's heads lie together, or a head's tokens do
    const bool heads_apart = heads == 1 || out->head >= D, tokens_apart = tokens == 1 || out->token >= D;
    const bool nested = heads == 1 || tokens == 1 || out->token >= (heads - 1) * out->head + D || out->head >= (tokens - 1) * out->token + D;
    if (!heads_apart || !tokens_apart || !nested) return fail(ORBIT_EINVAL, "%s: %s's rows overlap", who, name);
    return ORBIT_OK;
}

size_t forward_bytes(orbit_attention p, int64_t D) { return (size_t)p->slots * p->kv_heads * (attention_part((int)D) + 2) * sizeof(float); }

// Of the backward pass: lse and delta of each row, then the parts of dq (with those of sum p k, and sum ds of each row, where D <= 64),
// whose place those of dk and dv take afterwards.
size_t stat_floats(orbit_attention p) { return ((size_t)p->heads * p->q_tokens + 63) / 64 * 64; }

size_t backward_bytes(orbit_attention p, int64_t D) {
    const int64_t part = attention_part((int)D), of_rows = p->row_slots * (part <= 64 ? 2 * part + 1 : part), of_keys = p->key_slots * 2 * part;
    return (2 * stat_floats(p) + (size_t)std::max(of_rows, of_keys) * p->kv_heads) * sizeof(float);
}

constexpr double kLog2e = 1.4426950408889634;

// `least`: backward, so that rows' sums in units of scores, -lse / scale, stay within fp32's range.
orbit_status check_scale(const char* who, float scale, float least) {
    if (!(scale > 0.f) || !std::isfinite(scale)) return fail(ORBIT_EINVAL, "%s: scale must be finite and above 0", who);
    if (scale * kLog2e > FLT_MAX || scale < least) return fail(ORBIT_EUNSUPPORTED, "%s: scale %g is beyond fp32's range of scores", who, scale);
    return ORBIT_OK;
}

constexpr float kLeastBackward = 0x1p-100f;

// The backward pass finds a tile's heads by 32-bit offsets
orbit_status check_group(const char* who, const char* name, const AttnHeads& t, int group) {
    if (group > 1 && t.head > ((int64_t)1 << 29) / group) return fail(ORBIT_EUNSUPPORTED, "%s: %s's heads lie more than 2^29 values apart", who, name);
    return ORBIT_OK;
}

}  // namespace

extern "C" {

orbit_status attention_plan(int64_t n, const int64_t* q_starts, const int64_t* q_lens, const int64_t* k_starts, const int64_t* k_lens, int32_t heads,
                            int32_t kv_heads, int32_t causal, orbit_attention* out) {
    const char* who = "attention_plan";
    clear_error();
    if (!out) return fail(ORBIT_EINVAL, "%s: out is NULL", who);
    *out = nullptr;
    if (n < 0) return fail(ORBIT_EINVAL, "%s: negative number of sequences", who);
    if (n && (!q_starts || !q_lens || !k_starts || !k_lens)) return fail(ORBIT_EINVAL, "%s: a list is NULL", who);
    if (heads < 1 || kv_heads < 1 || heads % kv_heads) return fail(ORBIT_EINVAL, "%s: %d heads over %d key heads", who, heads, kv_heads);
    if (heads > kMaxHeads) return fail(ORBIT_EUNSUPPORTED, "%s: more than %d heads", who, kMaxHeads);
    const int64_t group = heads / kv_heads;
    int64_t tiles = 0, q_tokens = 0, k_tokens = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (q_starts[i] < 0 || q_lens[i] < 0 || k_starts[i] < 0 || k_lens[i] < 0)
            return fail(ORBIT_EINVAL, "%s: sequence %lld has a negative start or length", who, (long long)i);
        if (q_starts[i] > kMaxTokens || q_lens[i] > kMaxTokens - q_starts[i] || k_starts[i] > kMaxTokens || k_lens[i] > kMaxTokens - k_starts[i] ||
            q_lens[i] > (kMaxTokens - kAttnWideRows) / group || k_lens[i] > kMaxTokens - kAttnWideRows)
            return fail(ORBIT_EUNSUPPORTED, "%s: sequence %lld passes 2^31 rows", who, (long long)i);
        // keys' tiles too, those of the backward pass
        tiles += ceil_div(q_lens[i] * group, kAttnRows) + ceil_div(k_lens[i], kAttnRows);
        if (tiles > (kMaxGroups - 8192) / kv_heads) return fail(ORBIT_EUNSUPPORTED, "%s: more tiles of rows than a launch takes", who);
        if (q_lens[i]) q_tokens = std::max(q_tokens, q_starts[i] + q_lens[i]);
        if (k_lens[i]) k_tokens = std::max(k_tokens, k_starts[i] + k_lens[i]);
    }
    orbit_attention p = new (std::nothrow) orbit_attention_s;
    if (!p) return fail(ORBIT_ENOMEM, "%s: out of host memory", who);
    p->heads = heads;
    p->kv_heads = kv_heads;
    p->causal = causal != 0;
    p->q_tokens = q_tokens;
    p->k_tokens = k_tokens;
    bool twice = false;
    try {
        std::vector<Sequence> s;
        std::vector<std::pair<int64_t, int64_t>> q, k;
        for (int64_t i = 0; i < n; ++i) {
            s.push_back({q_starts[i], q_lens[i], k_starts[i], k_lens[i]});
            q.push_back({q_starts[i], q_lens[i]});
            k.push_back({k_starts[i], k_lens[i]});
        }
        twice = overlap(q);
        p->shared_keys = overlap(k);
        if (!twice) fill(p, s);
    } catch (...) {
        delete p;
        return fail(ORBIT_ENOMEM, "%s: out of host memory", who);
    }
    if (twice) {
        delete p;
        return fail(ORBIT_EINVAL, "%s: two sequences have a query in common", who);
    }
    int dev;
    orbit_status st = device_for_upload(&dev);
    if (st == ORBIT_OK && dev >= 0) st = upload_dev(p, dev);
    if (st != ORBIT_OK) {
        delete p;
        return st;
    }
    *out = p;
    return ORBIT_OK;
}

orbit_status attention_plan_upload(orbit_attention p) {
    clear_error();
    if (!p) return fail(ORBIT_EINVAL, "attention_plan_upload: plan is NULL");
    int dev;
    DeviceInfo info;
    const orbit_status st = current_device(&dev, &info);
    return st != ORBIT_OK ? st : upload_dev(p, dev);
}

void attention_plan_destroy(orbit_attention p) {
    if (!p) return;
    free_per_device(p->dev_lists);
    delete p;
}

orbit_status attention_workspace_size(orbit_attention p, int64_t D, int32_t backward, size_t* bytes) {
    const char* who = "attention_workspace_size";
    clear_error();
    if (!bytes) return fail(ORBIT_EINVAL, "%s: null output pointer", who);
    *bytes = 0;
    const orbit_status st = check_dim(who, p, D);
    if (st == ORBIT_OK) *bytes = backward ? backward_bytes(p, D) : forward_bytes(p, D);
    return st;
}

orbit_status attention(orbit_attention p, const orbit_heads* q, const orbit_heads* k, const orbit_heads* v, const orbit_heads* out, int64_t D,
                       float scale, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "attention";
    clear_error();
    orbit_status st = check_dim(who, p, D);
    if (st != ORBIT_OK) return st;
    st = check_scale(who, scale, 0.f);
    if (st != ORBIT_OK) return st;
    if (p->q_tokens == 0) return ORBIT_OK;
    AttnParams a{};
    st = check_heads(who, "q", q, p->q_tokens, p->heads, D, false, false, &a.q);
    if (st == ORBIT_OK) st = check_heads(who, "k", k, p->k_tokens, p->kv_heads, D, false, false, &a.k);
    if (st == ORBIT_OK) st = check_heads(who, "v", v, p->k_tokens, p->kv_heads, D, false, false, &a.v);
    if (st == ORBIT_OK) st = check_heads(who, "out", out, p->q_tokens, p->heads, D, true, true, &a.o);
    if (st != ORBIT_OK) return st;
    if (a.o.p == a.q.p || a.o.p == a.k.p || a.o.p == a.v.p) return fail(ORBIT_EINVAL, "%s: out lies on an input", who);
    if (!aligned(lse, 4)) return fail(ORBIT_EINVAL, "%s: misaligned lse", who);
    const size_t bytes = forward_bytes(p, D);
    if (bytes && (!workspace || !aligned(workspace, 16) || workspace_bytes < bytes))
        return fail(ORBIT_EINVAL, "%s: takes a workspace of %zu bytes, aligned to 16", who, bytes);
    int dev;
    DeviceInfo info;
    st = current_device(&dev, &info);
    if (st != ORBIT_OK) return st;
    const unsigned char* lists = nullptr;
    st = lists_on(who, p, dev, &lists);
    if (st != ORBIT_OK) return st;
    a.heads = p->heads;
    a.kv_heads = p->kv_heads;
    a.group = p->heads / p->kv_heads;
    a.D = (int)D;
    a.causal = p->causal;
    a.scale = (float)(scale * kLog2e);
    a.out_f32 = out->dtype == ORBIT_OUT_F32;
    a.lse = lse;
    a.part = (float*)workspace;
    a.stat = a.part + p->slots * p->kv_heads * attention_part((int)D);
    const std::pair<int, AttnWay> ways[] = {{kAttnForwardWide, kAttnWide}, {kAttnForward, kAttnWhole}, {kAttnFew, kAttnShared}};
    for (const auto& [which, way] : ways) {
        a.tiles = (const AttnTile*)(lists + p->at[which]);
        a.count = (int)p->count[which];
        if (!a.count) continue;
        const hipError_t e = launch_attention(a, way, (hipStream_t)stream);
        if (e != hipSuccess) return hip_fail(e, who);
    }
    a.joins = (const AttnJoin*)(lists + p->at[kAttnJoins]);
    a.count = (int)p->count[kAttnJoins];
    if (!a.count) return ORBIT_OK;
    const hipError_t e = launch_attention_join(a, (hipStream_t)stream);
    return e == hipSuccess ? ORBIT_OK : hip_fail(e, who);
}

orbit_status attention_backward(orbit_attention p, const orbit_heads* dout, const orbit_heads* q, const orbit_heads* k, const orbit_heads* v,
                                const orbit_heads* out, const float* lse, const orbit_heads* dq, const orbit_heads* dk, const orbit_heads* dv, int64_t D,
                                float scale, void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "attention_backward";
    clear_error();
    orbit_status st = check_dim(who, p, D);
    if (st != ORBIT_OK) return st;
    st = check_scale(who, scale, kLeastBackward);
    if (st != ORBIT_OK) return st;
    if (p->shared_keys) return fail(ORBIT_EINVAL, "%s: two of the plan's sequences have a key in common", who);
    AttnGradParams a{};
    st = check_heads(who, "dout", dout, p->q_tokens, p->heads, D, false, false, &a.g);
    if (st == ORBIT_OK) st = check_heads(who, "q", q, p->q_tokens, p->heads, D, false, false, &a.q);
    if (st == ORBIT_OK) st = check_heads(who, "k", k, p->k_tokens, p->kv_heads, D, false, false, &a.k);
    if (st == ORBIT_OK) st = check_heads(who, "v", v, p->k_tokens, p->kv_heads, D, false, false, &a.v);
    if (st == ORBIT_OK) st = check_heads(who, "out", out, p->q_tokens, p->heads, D, true, false, &a.o);
    if (st == ORBIT_OK) st = check_heads(who, "dq", dq, p->q_tokens, p->heads, D, false, true, &a.dq);
    if (st == ORBIT_OK) st = check_heads(who, "dk", dk, p->k_tokens, p->kv_heads, D, false, true, &a.dk);
    if (st == ORBIT_OK) st = check_heads(who, "dv", dv, p->k_tokens, p->kv_heads, D, false, true, &a.dv);
    if (st != ORBIT_OK) return st;
    a.group = p->heads / p->kv_heads;
    st = check_group(who, "q", a.q, a.group);
    if (st == ORBIT_OK) st = check_group(who, "dout", a.g, a.group);
    if (st != ORBIT_OK) return st;
    const void* const inputs[] = {a.g.p, a.q.p, a.k.p, a.v.p, a.o.p};
    const void* const outputs[] = {a.dq.p, a.dk.p, a.dv.p};
    for (int i = 0; i < 3; ++i) {
        for (const void* other : inputs)
            if (outputs[i] && outputs[i] == other) return fail(ORBIT_EINVAL, "%s: a gradient lies on an input", who);
        if (outputs[i] && outputs[i] == outputs[(i + 1) % 3]) return fail(ORBIT_EINVAL, "%s: two gradients lie in one place", who);
    }
    if (p->q_tokens == 0 && p->k_tokens == 0) return ORBIT_OK;
    if (p->q_tokens && (!lse || !aligned(lse, 4))) return fail(ORBIT_EINVAL, "%s: lse is a null or misaligned device pointer", who);
    const size_t bytes = backward_bytes(p, D);
    if (bytes && (!workspace || !aligned(workspace, 16) || workspace_bytes < bytes))
        return fail(ORBIT_EINVAL, "%s: takes a workspace of %zu bytes, aligned to 16", who, bytes);
    int dev;
    DeviceInfo info;
    st = current_device(&dev, &info);
    if (st != ORBIT_OK) return st;
    const unsigned char* lists = nullptr;
    st = lists_on(who, p, dev, &lists);
    if (st != ORBIT_OK) return st;
    a.heads = p->heads;
    a.kv_heads = p->kv_heads;
    a.D = (int)D;
    a.causal = p->causal;
    a.o_f32 = out && out->dtype == ORBIT_OUT_F32;
    a.q_tokens = p->q_tokens;
    a.scale = (float)(scale * kLog2e);
    a.out_scale = scale;
    a.lse = lse;
    a.lse2 = (float*)workspace;
    a.delta = a.lse2 + stat_floats(p);
    a.part = a.delta + stat_floats(p);
    a.part_sum = a.part + 2 * p->row_slots * p->kv_heads * attention_part((int)D);
    const struct {
        AttnGradStep step;
        int list;
    } steps[] = {{kAttnRowGrad, kAttnRowGrads}, {kAttnRowJoin, kAttnRowJoins}, {kAttnKeyGrad, kAttnKeyGrads}, {kAttnKeyJoin, kAttnKeyJoins}};
    for (const auto& s : steps) {
        a.count = (int)p->count[s.list];
        a.tiles = (const AttnTile*)(lists + p->at[s.list]);
        a.joins = (const AttnJoin*)(lists + p->at[s.list]);
        if (a.count == 0) continue;
        const bool of_rows = s.step == kAttnRowGrad || s.step == kAttnRowJoin;
        a.part2 = a.part + (of_rows ? p->row_slots : p->key_slots) * p->kv_heads * attention_part((int)D);
        const hipError_t e = launch_attention_grad(a, s.step, (hipStream_t)stream);
        if (e != hipSuccess) return hip_fail(e, who);
    }
    return ORBIT_OK;
}

}  // extern "C"
