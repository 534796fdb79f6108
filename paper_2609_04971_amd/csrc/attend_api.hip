// Entry points of the attention over the cache (bkv_attend,
// bkv_attend_shared): argument checks, how the work is cut, the launches.
#include <math.h>
#include <string.h>

#include "attend.h"

namespace bkv {
namespace attend {

namespace {
constexpr size_t kAlign = 256;
inline size_t up(size_t x, size_t n) { return (x + n - 1) / n * n; }

constexpr int kCus = 256;
constexpr int kMinChunk = 128;      // keys: one group of 32 for each wave of a streaming item, two tiles
// Bytes of a unit's keys that one streaming item takes rather than splits and a
// join.  The second launch costs 2.5 us where calls are captured, but the host's
// time for it where they are launched one by one, so the two break even at
// about 96 and 160 KB: the limit lies between, and up to it neither loses more
// than a quarter (us captured / one by one, in one piece and split, 8 heads:
// bf16 D 128 256 tokens 6.3 / 7.5 and 7.8 / 9.9, 512 8.5 / 8.4 and 8.0 / 9.9, 640
// 10.1 / 9.8 and 8.5 / 9.8; D 64 768 7.5 / 7.5 and 7.5 / 10.1, 1024 8.8 / 8.7 and
// 7.9 / 9.9; fp32 D 64 256 6.5 / 7.4 and 7.6 / 9.8, 512 9.5 / 9.3 and 7.6 / 9.9; D
// 128 256 9.2 / 9.0 and 9.3 / 9.8, 384 11.6 / 11.5 and 9.5 / 10.3).
constexpr long long kWhole = 128 << 10;
constexpr int kFewRows = 32;        // rows per unit up to which keys are streamed and the logits kept for the mass

// Items of 32 rows and kMinChunk keys up to which a prefix of more rows is
// streamed all the same, in one launch with the sequences' own caches: its keys
// are read by every row block, but from L2, and the tiles' launch is spared.  Up
// to 480 items that is ahead nearly always, from 3360 on it is far behind; in
// between the number alone does not decide, by up to 14 % up to the limit (us, tiles
// and items: 24 13.7 11.0, 192 17.4 13.5, 256 18.8 14.4, 288 21.8 16.4, 320 18.5
// 18.9, 432 27.2 25.8, 480 21.0 17.8, 504 17.2 19.6, 576 21.9 22.8, 640 20.1 20.1,
// 704 22.9 21.8, 792 20.0 20.4, 1008 21.4 24.2, 1024 23.0 24.7, 1088 52.7 68.6, 1344
// 155 148, 3360 38 49).
constexpr long long kFewItems = 4 * kCus;

// Workgroups that sum the weights of many rows: where the blocks of keys alone
// are fewer, a block's rows are dealt out, since three fit a compute unit and a
// causal block's rows are fewer the later it is (us, a call of 4509 queries of
// 7 heads, 2 kv-heads, 72 blocks, for 512 workgroups 159, 768 151, 1024 147,
// 1536 152; 9 x 1510 of 4 heads, 108 blocks: 63, 61, 62, 68).
constexpr int kMassItems = 1024;
constexpr int kMassRows = 256;      // rows that make such a workgroup worth its own sums

// Splits of n keys at most, of `base` items each: what a workspace has room for.
int most_splits(long long base, int n) {
    constexpr int kMost = 256, kItems = 1024;
    const long long k = base > 0 ? kItems / base + 1 : 1, by_keys = (n + kMinChunk - 1) / kMinChunk;
    const long long least = k < by_keys ? k : by_keys;
    return (int)(least > kMost ? kMost : least > 1 ? least : 1);
}

// Splits of n keys, `base` items each, by what they cost in keys of one item
// that has a compute unit to itself: the rounds of items times their keys and
// what an item costs around them, and the partials' way through memory.
// Streaming items share their compute unit's bandwidth, so that a round is as
// many items as there are compute units; tile items share its matrix cores
// only in part: 2 or 3 of them at once take 1.7 or 2.4 times as long as one.
// us, splits as taken (*) and others, streaming: 8 heads x 65536 tokens 32* 49,
// 64 50, 96 53, 256 57; 192 x 4000 1 78, 3 78, 4* 67, 6 76; 160 x 6000 (ragged)
// 2 105, 3* 79, 7 74; 296 x 2000 fp32 1 143, 2 127, 3* 123, 4 119; tile: 112
// blocks of 500 x 7 queries against 24000 3 146, 4 119, 5 135, 9* 113, 19 138.
int best_splits(bool tile, long long base, int n, long long rows, int D) {
    constexpr float kRound[4] = {0.f, 1.f, 1.7f, 2.4f};
    constexpr float kJoinKeys = 43.f * 8.f / 4e6f;  // keys in the time that 8 bytes take at 4 TB/s
    const int resident = !tile ? 1 : D == 128 ? 2 : 3;
    const float around = tile ? 100.f : 64.f;
    const int most = most_splits(base, n);
    int best = 1;
    float least = 0.f;
    // one piece, or as many as 1 to 4 items per compute unit take: in between
    // a round is begun and not filled
    for (int j = 0; j <= 4; ++j) {
        const long long fills = j == 0 || base > j * kCus ? 1 : j * kCus / base;
        const int k = fills < most ? (int)fills : most;
        const long long items = base * k, full = items / (resident * kCus), rest = items % (resident * kCus);
        const float rounds = (float)full * kRound[resident] + kRound[(rest + kCus - 1) / kCus];
        const float cost = rounds * ((float)n / (float)k + around) + (k > 1 ? (float)rows * (float)(k * D) * kJoinKeys : 0.f);
        if (j == 0 || cost < least) {
            least = cost;
            best = k;
        }
    }
    return best;
}

// Splits of a causal prompt in tiles, whose row blocks see from n - T to n keys,
// longest first: what the compute units take for all of them, but no less than
// the longest one, and a join.  (us for 1, 2, 3, 4 splits: 7805 queries of 4
// heads 131 97 88 94, 4509 of 14 heads on 2 kv-heads 94 101 105 116, 1024 of 16
// on 4 against 4096 72 54 53 49; D 64: 2 x 3886 of 4 heads 47 41 36 38, 5 x 2226
// of 4 on 2 31 33 37 39.)
int prompt_splits(long long base, int n, int T, long long rows, int D) {
    const float resident = D == 128 ? 2.f : 3.f, round = D == 128 ? 1.7f : 2.4f, around = D == 128 ? 100.f : 64.f;
    const float join_us = D == 128 ? 43.f : 70.f;  // keys in a microsecond
    const int most = most_splits(base, n);
    int best = 1;
    float least = 0.f;
    for (int k = 1; k <= most && k <= 8; ++k) {
        const float each = ((float)n - 0.5f * (float)T) / (float)k + around, longest = (float)n / (float)k + around;
        const float bulk = (float)base * (float)k * each * round / (resident * kCus);
        const float join = k > 1 ? join_us * ((float)rows * (float)(k * D) * 2e-6f + 5.f) : 0.f;
        const float cost = (bulk > longest ? bulk : longest) + join;
        if (k == 1 || cost < least) {
            least = cost;
            best = k;
        }
    }
    return best;
}

// Splits of a segment of n keys that is streamed together with another: the
// items of both fill one another's last rounds, so that none has to be
// shorter than half of a compute unit's share of all keys.
int shared_splits(long long base, int n, long long all_keys) {
    const long long chunk = all_keys / (2 * kCus) > kMinChunk ? all_keys / (2 * kCus) : kMinChunk;
    const long long k = (n + chunk - 1) / chunk, most = most_splits(base, n);
    return (int)(k < 1 ? 1 : k < most ? k : most);
}

// Splits of n keys (at most those of the capacity) and their length.
void cut(int n, int ns, int* out_ns, int* chunk) {
    *chunk = n > 0 ? (int)up((size_t)((n + ns - 1) / ns), kMinChunk) : kMinChunk;
    *out_ns = n > 0 ? (n + *chunk - 1) / *chunk : 1;
}
}  // namespace

Plan make_plan(const bkv_dims& d, int T, bool causal, bool mass, int groups, int P, int P_cap) {
    Plan p;
    memset(&p, 0, sizeof p);
    const long long G = d.Hq / d.Hkv, R = G * T;
    const long long rows = (long long)d.B * d.Hq * T;
    const long long pre_rows = groups > 0 ? d.B / groups * R : 0;
    const bool tiles = d.dtype == BKV_BF16;
    p.own_tile = tiles && R > kFewRows;
    const long long pre_units = (long long)groups * d.Hkv, few_rb = (pre_rows + 31) / 32;
    const long long few_items = pre_units * few_rb * ((P + kMinChunk - 1) / kMinChunk);
    p.pre_tile = tiles && pre_rows > kFewRows && (p.own_tile || few_items > kFewItems);
    p.wide = (!p.own_tile && R > 16) || (!p.pre_tile && pre_rows > 16);
    const int own_rb = p.own_tile ? 128 : p.wide ? 32 : 16, pre_rb = p.pre_tile ? 128 : p.wide ? 32 : 16;
    p.own_nrb = (int)((R + own_rb - 1) / own_rb);
    p.pre_nrb = (int)((pre_rows + pre_rb - 1) / pre_rb);
    const long long own = (long long)d.B * d.Hkv * p.own_nrb, pre = (long long)groups * d.Hkv * p.pre_nrb;
    // room for every N and P within the capacities: P decides between the kernels
    // and so the size of the row blocks, and the splits are most with the fewest items
    const int widest = p.own_tile ? 128 : 32;
    p.ns_room = most_splits((long long)d.B * d.Hkv * ((R + widest - 1) / widest), d.N_cap);
    if (groups > 0) p.ns_room += most_splits(pre_units * ((pre_rows + 127) / 128), P_cap);
    int own_ns, pre_ns = 1;
    if (groups > 0 && P > 0 && !p.own_tile && !p.pre_tile) {  // one launch takes both
        const long long all = own * d.N + pre * P;
        own_ns = shared_splits(own, d.N, all);
        pre_ns = shared_splits(pre, P, all);
    } else {
        // a short cache goes in one piece: joining splits would be a launch of
        // its own.  Not by the mass: outputs do not depend on whether it is asked for
        const bool whole = groups == 0 && !p.own_tile &&
                           (long long)d.N * d.D * (d.dtype == BKV_BF16 ? 2 : 4) <= kWhole;
        const bool prompt = p.own_tile && causal && T <= d.N && T > d.N / 5;
        own_ns = whole    ? 1
                 : prompt ? prompt_splits(own, d.N, T, rows, d.D)
                          : best_splits(p.own_tile, own, d.N, rows, d.D);
        if (groups > 0 && P > 0) pre_ns = best_splits(p.pre_tile, pre, P, rows, d.D);
    }
    cut(d.N, own_ns, &p.own_ns, &p.own_chunk);
    if (groups > 0 && P > 0) cut(P, pre_ns, &p.pre_ns, &p.pre_chunk);
    p.keep = mass && R <= kFewRows;
    if (mass && !p.keep && tiles && R <= kRegRows)
        cut(d.N, best_splits(false, (long long)d.B * d.Hkv, d.N, 0, d.D), &p.mass_ns, &p.mass_chunk);
    size_t off = 0;
    p.part_o = off;
    if (p.ns_room > 1) off = up(off + sizeof(float) * (size_t)rows * p.ns_room * d.D, kAlign);
    p.part_ml = off;
    if (p.ns_room > 1) off = up(off + sizeof(float) * (size_t)rows * p.ns_room * 2, kAlign);
    p.row_lse2 = off;
    if (mass) off = up(off + sizeof(float) * (size_t)rows, kAlign);
    p.logits = off;
    // kept logits go to memory where other splits have a say in the normalisers or
    // LDS does not hold them; a decoding step of many heads needs no room for them
    const int most_chunk = (int)up((size_t)d.N_cap, kMinChunk);
    if (p.keep && (p.ns_room > 1 || stream_lds(R < 16 ? (int)R : 16, d.D, (int)R, most_chunk) > kLdsRoom))
        off = up(off + sizeof(float) * (size_t)rows * up((size_t)d.N_cap, 32), kAlign);
    // the sums of parts > 1 never pass 2 kMassItems blocks
    p.parts = 1;
    p.parts_at = off;
    const long long most = R / kMassRows;
    if (mass && !p.keep && most > 1) {
        const long long blocks = (long long)d.B * d.Hkv * ((d.N + kMassKeys - 1) / kMassKeys);
        const long long want = blocks < 1 ? 1 : (kMassItems + blocks - 1) / blocks;
        p.parts = (int)(want < most ? want : most);
        off = up(off + sizeof(float) * 2 * kMassItems * kMassKeys, kAlign);
    }
    p.end = off;
    return p;
}

}  // namespace attend
}  // namespace bkv

using namespace bkv;
using namespace bkv::attend;

namespace {

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Dimensions of a call; groups 0: no prefix.
bkv_status check_shape(const bkv_dims* d, int32_t T, int32_t groups, int32_t P, int32_t P_cap) {
    const bkv_status st = bkv_validate(d, BKV_OP_COMPACT);
    if (st != BKV_OK) return st;
    if (T < 0 || groups < 0 || (long long)d->B * d->Hq * T > 0x7fffffffLL) return BKV_ERR_SHAPE;
    if (groups > 0) {
        if (d->B % groups != 0 || P_cap < 1 || P < 0 || P > P_cap) return BKV_ERR_SHAPE;
        if ((long long)groups * d->Hkv * P_cap > 0x7fffffffLL) return BKV_ERR_SHAPE;
    }
    return BKV_OK;
}

bkv_status run(const bkv_dims* d, int32_t flags, const void* q, int32_t T, int32_t groups, const void* PK,
               const void* PV, int32_t P, int32_t P_cap, const int32_t* p_lens, const void* K, const void* V,
               const int32_t* lens, float scale, void* out, float* lse, float* mass, void* ws, size_t ws_bytes,
               hipStream_t stream) {
    if (flags & ~BKV_ATTEND_CAUSAL) return BKV_ERR_INVALID;
    const bkv_status st = check_shape(d, T, groups, P, P_cap);
    if (st != BKV_OK) return st;
    if (d->B == 0 || T == 0) return BKV_OK;
    if (!q || !out || !aligned(q) || !aligned(out)) return BKV_ERR_INVALID;
    if (d->N > 0 && (!K || !V || !aligned(K) || !aligned(V))) return BKV_ERR_INVALID;
    if (groups > 0 && P > 0 && (!PK || !PV || !aligned(PK) || !aligned(PV))) return BKV_ERR_INVALID;
    const float scale2 = (scale == 0.0f ? 1.0f / sqrtf((float)d->D) : scale) * 1.4426950408889634f;
    if (!(scale >= 0.0f) || isinf(scale2)) return BKV_ERR_INVALID;  // 0 times infinity would be a NaN
    const Plan p = make_plan(*d, T, flags & BKV_ATTEND_CAUSAL, mass != nullptr, groups, P, P_cap);
    if (p.end > 0 && (!ws || ws_bytes < p.end || !aligned(ws))) return BKV_ERR_WORKSPACE;
    if (p.own_ns + p.pre_ns > p.ns_room) return BKV_ERR_WORKSPACE;  // (the room covers every N and P)
    // what is written, then what is only read; of the last head the tokens that are there
    const size_t row = (size_t)d->D * (d->dtype == BKV_BF16 ? 2 : 4), queries = (size_t)d->B * d->Hq * T;
    auto tokens = [](size_t units, size_t n, size_t cap) { return n > 0 ? (units - 1) * cap + n : 0; };
    const size_t own_tokens = tokens((size_t)d->B * d->Hkv, d->N, d->N_cap);
    const size_t pre_tokens = groups > 0 ? tokens((size_t)groups * d->Hkv, P, P_cap) : 0;
    const Span spans[] = {{out, queries * row},        {lse, queries * sizeof(float)}, {mass, own_tokens * sizeof(float)},
                          {ws, p.end},                 {q, queries * row},             {K, own_tokens * row},
                          {V, own_tokens * row},       {PK, pre_tokens * row},         {PV, pre_tokens * row},
                          {lens, d->B * sizeof(int32_t)}, {p_lens, groups * sizeof(int32_t)}};
    if (!apart(spans, 11, 4)) return BKV_ERR_INVALID;
    char* w = static_cast<char*>(ws);
    Args a;
    memset(&a, 0, sizeof a);
    a.Hq = d->Hq;
    a.Hkv = d->Hkv;
    a.G = d->Hq / d->Hkv;
    a.T = T;
    a.R = a.G * T;
    a.D = d->D;
    a.N_cap = d->N_cap;
    a.rows = d->B * d->Hq * T;
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.mass = mass;
    a.scale2 = scale2;
    Segment& own = a.seg[1];
    own.K = K;
    own.V = V;
    own.lens = lens;
    own.n = d->N;
    own.cap = d->N_cap;
    own.units = d->B * d->Hkv;
    own.seqs = 1;
    own.rows = a.R;
    own.nrb = p.own_nrb;
    own.ns = p.own_ns;
    own.chunk = p.own_chunk;
    own.split0 = p.pre_ns;
    own.causal = (flags & BKV_ATTEND_CAUSAL) && T > 1;  // one query sees all of its cache either way
    Segment& pre = a.seg[0];
    pre.nrb = pre.ns = pre.seqs = 1;
    if (groups > 0 && P > 0) {
        pre.K = PK;
        pre.V = PV;
        pre.lens = p_lens;
        pre.n = P;
        pre.cap = P_cap;
        pre.units = groups * d->Hkv;
        pre.seqs = d->B / groups;
        pre.rows = pre.seqs * a.R;
        pre.nrb = p.pre_nrb;
        pre.ns = p.pre_ns;
        pre.chunk = p.pre_chunk;
    }
    const long long items0 = (long long)pre.units * pre.nrb * pre.ns;
    const long long items1 = (long long)own.units * own.nrb * own.ns;
    if (items0 + items1 > kMaxBlocks || (mass && !p.keep && mass_blocks(a, p.parts) > kMaxBlocks)) return BKV_ERR_SHAPE;
    a.ns = p.own_ns + p.pre_ns;
    a.part_o = reinterpret_cast<float*>(w + p.part_o);
    a.part_ml = reinterpret_cast<float*>(w + p.part_ml);
    a.row_lse2 = reinterpret_cast<float*>(w + p.row_lse2);
    a.logits = p.keep ? reinterpret_cast<float*>(w + p.logits) : nullptr;
    a.lstride = (int)up((size_t)d->N, 32);
    a.o_rows = a.R;
    if (!p.pre_tile && pre.units > 0 && pre.rows > a.o_rows) a.o_rows = pre.rows;
    if (a.o_rows > 16) a.o_rows = 16;
    a.keep = p.keep ? kKeepLds : kKeepNone;
    if (p.keep && stream_lds(a) > kLdsRoom) a.keep = kKeepStore;
    if (join_grid(a).blocks > kMaxBlocks) return BKV_ERR_SHAPE;
    if (p.pre_tile && launch_attend_tile(a, pre, stream) != hipSuccess) return BKV_ERR_HIP;
    if (p.own_tile && launch_attend_tile(a, own, stream) != hipSuccess) return BKV_ERR_HIP;
    if (!p.own_tile) {  // rows of the prefix are no fewer than a sequence's own
        a.items0 = p.pre_tile ? 0 : (int)items0;
        if (launch_attend_stream(a, d->dtype, p.wide, stream) != hipSuccess) return BKV_ERR_HIP;
    }
    if (launch_attend_join(a, d->dtype, stream) != hipSuccess) return BKV_ERR_HIP;
    if (p.mass_ns > 0 && d->N > 0) {
        if (launch_attend_row_mass(a, p.mass_ns, p.mass_chunk, stream) != hipSuccess) return BKV_ERR_HIP;
    } else if (mass && !p.keep && d->N > 0) {
        float* part = reinterpret_cast<float*>(w + p.parts_at);
        if (launch_attend_tile_mass(a, d->dtype, part, p.parts, stream) != hipSuccess) return BKV_ERR_HIP;
        if (p.parts > 1 && launch_attend_add_parts(a, part, p.parts, stream) != hipSuccess) return BKV_ERR_HIP;
    }
    return BKV_OK;
}

}  // namespace

extern "C" {

size_t bkv_attend_workspace_bytes(const bkv_dims* d, int32_t T, int32_t mass, int32_t groups, int32_t P_cap) {
    if (check_shape(d, T, groups, 0, P_cap) != BKV_OK || d->B == 0 || T == 0) return 0;
    return make_plan(*d, T, false, mass != 0, groups, 0, P_cap).end;
}

bkv_status bkv_attend(const bkv_dims* d, int32_t flags, const void* q, int32_t T, const void* K, const void* V,
                      const int32_t* lens, float scale, void* out, float* lse, float* mass, void* ws, size_t ws_bytes,
                      hipStream_t stream) {
    return run(d, flags, q, T, 0, nullptr, nullptr, 0, 0, nullptr, K, V, lens, scale, out, lse, mass, ws, ws_bytes,
               stream);
}

bkv_status bkv_attend_shared(const bkv_dims* d, int32_t flags, const void* q, int32_t T, int32_t groups, const void* PK,
                             const void* PV, int32_t P, int32_t P_cap, const int32_t* p_lens, const void* K,
                             const void* V, const int32_t* lens, float scale, void* out, float* lse, float* mass,
                             void* ws, size_t ws_bytes, hipStream_t stream) {
    if (groups < 1) return d ? BKV_ERR_SHAPE : BKV_ERR_INVALID;
    return run(d, flags, q, T, groups, PK, PV, P, P_cap, p_lens, K, V, lens, scale, out, lse, mass, ws, ws_bytes,
               stream);
}

}  // extern "C"
