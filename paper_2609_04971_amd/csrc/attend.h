// Shared by the attention kernels (attend.hip, attend_tile.hip): what a call
// reads and writes, how its work is cut, and the row arithmetic.
#pragma once

#include "device_common.h"
#include "internal.h"

namespace bkv {
namespace attend {

// Keys that many query rows attend to: one sequence's cache (own), or the
// prefix of a group of sequences.  A unit is one (sequence or group, kv-head)
// pair.  Its rows are those of seqs consecutive sequences, R = G*T each, in
// the order sequence, query, head of the kv-head's group; a unit's rows are
// cut into nrb row blocks and its keys into ns splits, and every (unit, row
// block, split) is one work item.
struct Segment {
    const void* K;
    const void* V;
    const int32_t* lens;  // valid keys of each sequence or group, or null: n of all
    int n, cap;           // keys at most; keys allocated, the unit stride of K and V
    int units, seqs, rows;
    int nrb, ns, chunk;
    int split0;           // its first partial of every row
    int causal;
};

struct Args {
    Segment seg[2];       // 0 the prefix (units 0 without one), 1 the sequences' own caches
    int items0;           // work items of seg[0]
    const void* q;
    void* out;
    float* lse;           // or null
    float* mass;          // or null
    float* part_o;        // [row][ns][D] unnormalised sums of exp2(l2 - m) v
    float* part_ml;       // [row][ns][2] m and z = sum of exp2(l2 - m)
    float* row_lse2;      // [B, Hq, T] log2-normalisers, +inf for a row that sees nothing
    float* logits;        // [own unit][R][lstride] l2 = l log2(e), -inf where not seen; null unless kept
    int lstride;
    int keep;             // Keep: whether and where an item keeps its logits
    int o_rows;           // rows of a 16-row tile that any item has
    int Hq, Hkv, G, T, R, D;
    int N_cap;
    int rows;             // B * Hq * T
    int ns;               // partials per row; 1: the outputs are written directly
    float scale2;         // scale * log2(e)
};

// How a call is cut.  N and P choose between kernels, row blocks, splits and
// parts; the workspace is laid out by what is most over all N <= N_cap and
// P <= P_cap, from the capacities alone, so that one serves them all.
struct Plan {
    bool own_tile, pre_tile;  // the tile kernel takes the segment
    bool wide;                // the streaming kernel takes 32 rows an item, else 16
    int own_nrb, pre_nrb;
    int own_ns, own_chunk, pre_ns, pre_chunk;
    int ns_room;              // partials of a row that the workspace holds
    bool keep;                // the logits are kept for the mass
    int mass_ns, mass_chunk;  // else, of rows that fit registers (mass_ns > 0): splits of the keys
    int parts;                // or: workgroups that share a block of keys
    size_t part_o, part_ml, row_lse2, logits, parts_at, end;
};
Plan make_plan(const bkv_dims& d, int T, bool causal, bool mass, int groups, int P, int P_cap);

// A row of a segment's unit: which query it is.
struct Row {
    int t;          // query, 0..T-1
    long long gr;   // row of the partials: (sequence, kv-head, query, head of the group)
    long long q;    // element offset of the query and of its output
    long long lse;  // offset of its normaliser
};
__device__ __forceinline__ Row decode_row(const Args& a, int unit, int seqs, int rr) {
    const int h = unit % a.Hkv, grp = unit / a.Hkv;
    const int b = grp * seqs + rr / a.R, r = rr % a.R;
    const int t = r / a.G, g = r - t * a.G;
    Row x;
    x.t = t;
    x.gr = ((long long)b * a.Hkv + h) * a.R + r;
    x.lse = ((long long)b * a.Hq + h * a.G + g) * a.T + t;
    x.q = x.lse * a.D;
    return x;
}

// The logits of the sequences' own tokens, for the mass: none kept; in LDS
// until the item ends (stores among the key loads would have to be waited for
// with them); written as they come, where they do not fit.
enum Keep { kKeepNone, kKeepLds, kKeepStore };
constexpr int kPadO = 4, kPadL = 16;  // floats that keep the rows of the LDS arrays apart
constexpr size_t kLdsRoom = 79 * 1024;  // two workgroups a compute unit
inline size_t stream_lds(int o_rows, int D, int kept_rows, int chunk) {
    return ((size_t)4 * o_rows * (D + kPadO) + (size_t)kept_rows * (chunk + kPadL)) * sizeof(float);
}
inline size_t stream_lds(const Args& a) {
    return stream_lds(a.o_rows, a.D, a.keep == kKeepLds ? a.R : 0, a.seg[1].chunk);
}

// Workgroups of 256 threads that one launch holds: its threads are counted in
// 32 bits.
constexpr long long kMaxBlocks = 0xffffffffLL / 256;

// Blocks of the join's launch.
constexpr int kFewSplits = 11;  // a row to some lanes, else to a workgroup
struct JoinGrid {
    bool few;
    int njoin, nchunk;
    long long blocks;
};
inline JoinGrid join_grid(const Args& a) {
    constexpr int kThreads = 256, kTokens = 1024;
    JoinGrid g;
    g.few = a.ns <= kFewSplits;
    const int rpb = g.few ? kThreads / (a.D / 4) : 1;
    g.njoin = a.ns > 1 ? (int)(((long long)a.rows + rpb - 1) / rpb) : 0;
    // (one split with its logits in LDS has added its weights itself)
    g.nchunk = a.keep && (a.ns > 1 || a.keep == kKeepStore) ? (a.seg[1].n + kTokens - 1) / kTokens : 0;
    g.blocks = g.njoin + (long long)a.seg[1].units * g.nchunk;
    return g;
}

// Length of a unit's keys: lens may hold anything, the keys read stay in [0, n).
__device__ __forceinline__ int unit_len(const Segment& sg, int unit, int Hkv) {
    return sg.lens ? min(max(sg.lens[unit / Hkv], 0), sg.n) : sg.n;
}

// The unit of an item of a launch whose units go round fastest.  Workgroups go
// round the eight XCDs, so that each works on few units at a time and keeps
// them in its L2; units of other lengths are dealt out anew every kTurns
// rounds, or an XCD would have the long ones all along (us, every 1, 2, 4, 8
// rounds and never: ragged prompts of 8 x 2048 queries of one kv-head 109 103
// 99 98 124, 2 x 4096 of eight 170 169 193 202 224; 8 x 200 against 8000 of
// four 257 284 286 286 292).
constexpr int kTurns = 2;
__device__ __forceinline__ int turning_unit(const Segment& sg, int item, int Hkv) {
    const int unit = item % sg.units;
    return sg.lens && sg.units > Hkv ? (unit + item / sg.units / kTurns) % sg.units : unit;
}

// What a row's sums come to.  z is 0 for a row that saw nothing and at least 1
// otherwise (or NaN, where it saw one, and then so are its results).
struct RowEnd {
    float inv;   // 1 / z, or 0
    float lse;   // natural log of the normaliser, -inf for nothing
    float lse2;  // its log2 for the weights, +inf for nothing: they come out 0
};
__device__ __forceinline__ RowEnd row_end(float m, float z) {
    const float l2 = m + log2f(z);
    return z == 0.f ? RowEnd{0.f, -INFINITY, INFINITY} : RowEnd{1.f / z, l2 * 0.6931471805599453f, l2};
}

// ---- rows of the weights' sums -------------------------------------------------------
// The kernels that sum the weights of many rows take a unit's rows as they lie
// (g T + t), `parts` workgroups to a block of kMassKeys keys, each a range of
// rows.  Key j of a causal cache is seen by the queries t >= j - lead.
constexpr int kMassKeys = 128;
// Rows of a bf16 cache that workgroups hold in registers instead: 128 of D 128
// do not fit (us, a call of 96 rows, registers and tiles: 128 heads of 4000 tokens
// 85 103, 16 of 16000 54 61, 512 of 600 57 64, 8 of 8000 29 29).
constexpr int kRegRows = 96;
inline long long mass_blocks(const Args& a, int parts) {
    return (long long)a.seg[1].units * parts * ((a.seg[1].n + kMassKeys - 1) / kMassKeys);
}

struct MassRows {
    int T, causal, lead, t0, full, end;  // t0: the first query that sees any key; full: from here on, all of them
    int first, first_t;
    __device__ __forceinline__ MassRows(const Args& a, int causal_, int len, int key0, int keys, int part, int parts) {
        T = a.T;
        causal = causal_;
        lead = len - a.T;
        t0 = causal ? max(0, key0 - lead) : 0;
        full = causal ? key0 + keys - 1 - lead : 0;
        end = (int)((long long)a.R * (part + 1) / parts);
        first = (int)((long long)a.R * part / parts);
        first_t = first % T;
        if (t0 >= T)
            first = end;  // no query sees these keys
        else
            skip(first, first_t);
    }
    // To the head's first query that sees anything.
    __device__ __forceinline__ void skip(int& r, int& t) const {
        if (t < t0) {
            r += t0 - t;
            t = t0;
        }
    }
    __device__ __forceinline__ void advance(int& r, int& t, int rows) const {
        r += rows;
        t += rows;
        if (t >= T) {
            t %= T;
            skip(r, t);
        }
    }
    // Whether some of the rows [r, r + rows), the first one query t, may not see
    // some key, or belong to a later head.
    __device__ __forceinline__ bool edge(int r, int t, int rows) const {
        return t < full || (causal && t + rows > T && r + T - t < end);
    }
    // Keys that row r sees.
    __device__ __forceinline__ int seen(int r) const { return lead + 1 + r % T; }
};

// Lowest running maximum: finite, so that exp2(-inf - m) is 0 and not NaN in
// a row that has seen nothing yet.
constexpr float kLowest = -3.402823466e38f;

}  // namespace attend

// Both segments in one launch (wide: 32 rows an item, else 16); a segment without units takes no part.
hipError_t launch_attend_stream(const attend::Args& a, int dtype, bool wide, hipStream_t s);
// One segment of a bf16 cache, 128 rows an item.
hipError_t launch_attend_tile(const attend::Args& a, const attend::Segment& sg, hipStream_t s);
// Joins the partials and, where the logits were kept, adds the weights to the mass.
hipError_t launch_attend_join(const attend::Args& a, int dtype, hipStream_t s);
// The weights' sums from the queries and keys, added to the mass: of at most kRegRows rows of a bf16 cache.
hipError_t launch_attend_row_mass(const attend::Args& a, int ns, int chunk, hipStream_t s);
// And of more rows, added to the mass, or, where parts > 1, to part [parts][units][n], whose sums the third adds.
hipError_t launch_attend_tile_mass(const attend::Args& a, int dtype, float* part, int parts, hipStream_t s);
hipError_t launch_attend_add_parts(const attend::Args& a, const float* part, int parts, hipStream_t s);

}  // namespace bkv
