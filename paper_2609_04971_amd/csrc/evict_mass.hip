// Eviction by accumulated attention weight for gfx950: each head keeps its
// first n_prefix and last W tokens and, of the others, the budget -
// n_prefix - W of largest mass (ties to the lower index); K, V and the
// masses themselves are compacted in place.
//
// One workgroup per head selects.  Masses are heavy-tailed (a few sinks hold
// most of the weight), so they are cut by their order-preserving bit pattern,
// which is about logarithmic: the candidates' range [lo, hi] is split into
// 4096 equal bins, a histogram in LDS finds the bin that holds the last one
// kept, and that bin becomes the range, 12 bits a round and at most three
// rounds.  Usually the first bin holds a few candidates, which one wave ranks
// directly; a bin that is taken whole, or whose masses are all equal, ends the
// search too.  What comes out is a (mass, token) pair: a candidate is kept if
// its mass is larger, or equal with a token at or below.
//
// Up to 32768 tokens a head's masses stay in registers (token tid + NT i), so
// they are read once and moved without a hazard; longer heads read them again
// on every pass.  Kept tokens are ranked from the ballots of runs of 64 tokens
// and one scan of the runs' counts.
//
// The rest is moving rows.  Order preserved, compact.hip does it.  Filling
// holes, the moves are a list, which the selecting workgroup works off itself
// where there are many heads (one's selection then overlaps another's copies)
// or few moves, and a second launch otherwise.
#include "device_common.h"
#include "internal.h"
#include "mx.h"

namespace bkv {
namespace {

constexpr int kBins = 4096;
constexpr int kPerMax = 32;    // tokens per thread in registers
constexpr int kLongThreads = 1024;  // threads per head, and few where heads are many and short
constexpr int kShortThreads = 256;
// Heads from which on a workgroup of kShortThreads selects and moves (us on
// masses that no eviction has seen, that and the other form, 4096 -> 3584 filling
// holes: 128 heads 34 28, 256 42 41, 384 57 65, 512 68 78, 2048 209 285; 8192 ->
// 7168: 256 76 70, 384 104 108, 768 176 194; in order both are the same but for 2 %).
constexpr int kManyHeads = 256, kManyLongHeads = 384;
// Bytes that move in a head at most, K and V, where that form is taken whatever
// the heads' number, as it spares a launch (us, the other form and that: 28 heads,
// 12 KB 18.9 17.9, 13 heads, 50 KB 17.3 16.0, 64 heads, 75 KB 19.0 19.4; 40 heads, 104
// KB 18.0 17.8, 8 heads, 100 KB 18.1 19.4, 16 heads, 140 KB 18.0 18.9).
constexpr long long kLittle = 96 << 10;
constexpr int kOwnMoves = kBins / 2;  // moves that the selecting workgroup's lists hold
constexpr int kCopyThreads = 256;
constexpr int kCopyMoves = 64;  // rows per copy item

enum Mode { kOrder, kFill, kFillCopy, kFillCopyMx };  // (the last of a 4-bit cache)

struct MassArgs {
    float* mass;
    int32_t* kept;
    // moves of the hole-filling layout, [P][max_moves], and their number [P]
    int32_t* mv_src;
    int32_t* mv_dst;
    int32_t* mv_val;
    int32_t* mv_n;
    // heads longer than the registers hold: [P][nruns] ballots and [P][nruns] counts
    unsigned long long* ballots;
    int32_t* runs;
    int nruns, max_moves;
    int N, N_cap, n_keep, W, n_prefix;
    int* hdr;  // the workspace's stamp
    int P, budget;
    // the rows, for workgroups that move them themselves
    char* K;
    char* V;
    size_t head_stride;  // bytes between heads
    int vec_shift;       // log2 of 16-byte vectors per row
    uint8_t* KS;         // a 4-bit cache's scales, N_cap rows a head
    uint8_t* VS;
    int scale_bytes;     // of a row, 2 or 4
};

// Exclusive scan of one int per thread over the workgroup; *total is the sum.
template <int NT>
__device__ __forceinline__ int block_scan(int v, int* buf, int* total) {
    constexpr int NW = NT / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    if (lane == 63) buf[wave] = x;
    __syncthreads();
    int before = x - v, all = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const int t = buf[w];
        if (w < wave) before += t;
        all += t;
    }
    *total = all;
    __syncthreads();
    return before;
}

// Exclusive scan of n counts in place.
template <int NT>
__device__ __forceinline__ void scan_runs(int* runs, int n, int* buf) {
    int base = 0;
    for (int i0 = 0; i0 < n; i0 += NT) {
        const int i = i0 + threadIdx.x;
        int total;
        const int before = block_scan<NT>(i < n ? runs[i] : 0, buf, &total);
        if (i < n) runs[i] = base + before;
        base += total;
    }
    __syncthreads();
}

// Rows src[m] -> dst[m] of K and V for moves [0, n): sources lie at or above
// the budget and destinations below it, so no move can read what another
// writes.  Threads [0, NT) of one workgroup, eight vectors each in flight.
template <int NT>
__device__ __forceinline__ void move_rows(char* K, char* V, const int* src, const int* dst, int n, int vec_shift) {
    if (n <= 0) return;
    const int vpr = 1 << vec_shift, total = n << (vec_shift + 1);  // K and V
    for (int e0 = threadIdx.x; e0 < total; e0 += 8 * NT) {
        dev::u32x4 b[8];
        dev::static_for<8>([&](auto kc) {
            const int e = min(e0 + decltype(kc)::value * NT, total - 1);
            const int r = e >> (vec_shift + 1), v = e & (2 * vpr - 1);  // a move's K row, then its V row
            const char* from = (v < vpr ? K : V) + ((size_t)src[r] << (vec_shift + 4)) + (v & (vpr - 1)) * 16;
            b[decltype(kc)::value] = __builtin_nontemporal_load(reinterpret_cast<const dev::u32x4*>(from));
        });
        dev::static_for<8>([&](auto kc) {
            const int e = e0 + decltype(kc)::value * NT;
            const int r = e >> (vec_shift + 1), v = e & (2 * vpr - 1);
            if (e < total) {
                char* to = (v < vpr ? K : V) + ((size_t)dst[r] << (vec_shift + 4)) + (v & (vpr - 1)) * 16;
                __builtin_nontemporal_store(b[decltype(kc)::value], reinterpret_cast<dev::u32x4*>(to));
            }
        });
    }
}

// The same moves of a 4-bit cache's scales, head h.  Four bytes here and there:
// 4608 heads of 4096 -> 3584 on masses that no eviction has seen take 246 us, 70 of
// them for these, whose stores meet parts of nearly every line.
template <int NT>
__device__ __forceinline__ void move_scales(const MassArgs& a, int h, const int* src, const int* dst, int n) {
    for (int e = threadIdx.x; e < 2 * n; e += NT) {
        uint8_t* head = (e & 1 ? a.VS : a.KS) + (size_t)h * a.N_cap * a.scale_bytes;
        const size_t from = src[e >> 1], to = dst[e >> 1];
        if (a.scale_bytes == 4)
            reinterpret_cast<uint32_t*>(head)[to] = reinterpret_cast<const uint32_t*>(head)[from];
        else
            reinterpret_cast<uint16_t*>(head)[to] = reinterpret_cast<const uint16_t*>(head)[from];
    }
}

// NT threads, PER tokens each in registers; PER 0: masses, ballots and counts
// stay in memory.
// Bound by its passes over the registers (search, ballots, moves), a compute
// unit's instructions: 64 heads of 32768 38 us, 2 of 22101 26; in the form that
// moves rows too, by those (4608 heads of 4096 -> 3584 on masses that no eviction
// has seen, 451 rows a head, 2.4 GB, 433 us, 5.5 TB/s; fewer rows move where the
// same tokens have been kept before).  Heads past the registers' length pass
// over memory in one workgroup each: 2 of 65000 90 us, 8 of them 104.
template <int NT, int PER, int MODE>
__global__ __launch_bounds__(NT) void mass_select_kernel(MassArgs a) {
    constexpr int NW = NT / 64, BPT = kBins / NT;
    __shared__ int hist[kBins];  // later the moves' two lists
    __shared__ unsigned long long s_ballots[PER ? PER * NW : 1];
    __shared__ int s_runs[PER ? PER * NW : 1];
    __shared__ int buf[NW];
    __shared__ unsigned s_min[NW], s_max[NW], s_cand[64];
    __shared__ int s_cand_j[64];
    __shared__ int s_bin, s_above, s_count, s_n, s_j, s_ok;
    __shared__ unsigned s_theta;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int h = blockIdx.x, N = a.N, n = a.n_keep;
    float* mass = a.mass + (size_t)h * a.N_cap;
    int32_t* kept = a.kept + (size_t)h * n;
    const int lo_t = a.n_prefix, hi_t = N - a.W;  // candidates [lo_t, hi_t)
    const int NI = PER ? PER : (N + NT - 1) / NT;
    unsigned long long* ballots = PER ? s_ballots : a.ballots + (size_t)h * a.nruns;
    int* runs = PER ? s_runs : a.runs + (size_t)h * a.nruns;

    float val[PER ? PER : 1];
    if constexpr (PER > 0) {
        dev::static_for<PER>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            val[i] = mass[min(tid + i * NT, N - 1)];
        });
    }
    if (tid == 0) {
        s_ok = dev::stamp_ok(a.hdr, a.P, a.budget);
        if (!s_ok) dev::raise_error(a.hdr, kErrStamp);
    }
    __syncthreads();
    if (!s_ok) return;  // nothing has been written
    // f(run, token, value) for every token of this thread, whole waves at a time
    auto each = [&](auto&& f) {
        if constexpr (PER > 0) {
            dev::static_for<PER>([&](auto ic) {
                constexpr int i = decltype(ic)::value;
                float v = val[i];
                asm volatile("" : "+v"(v));  // or every pass's keys would be kept in registers
                f(i * NW + wave, tid + i * NT, v);
            });
        } else {
            constexpr int kAhead = 8;  // loads in flight
            for (int i0 = 0; i0 < NI; i0 += kAhead) {
                float v[kAhead];
                dev::static_for<kAhead>([&](auto kc) { v[decltype(kc)::value] = mass[min(tid + (i0 + decltype(kc)::value) * NT, N - 1)]; });
                dev::static_for<kAhead>([&](auto kc) {
                    const int i = i0 + decltype(kc)::value;
                    if (i < NI) f(i * NW + wave, tid + i * NT, v[decltype(kc)::value]);
                });
            }
        }
    };
    const unsigned long long below = (1ull << lane) - 1ull;

    // the last candidate kept: mass order key theta, token last
    unsigned theta = 0xffffffffu;
    int last = -1;
    int take = n - a.n_prefix - a.W;  // places for candidates; 0: none but the forced tokens
    if (take > 0) {
        unsigned kmin = 0xffffffffu, kmax = 0u;
        each([&](int, int j, float v) {
            if (j >= lo_t && j < hi_t) {
                const unsigned u = dev::ord_key(v);
                kmin = min(kmin, u);
                kmax = max(kmax, u);
            }
        });
        kmin = dev::wave_min_u32(kmin);
        kmax = ~dev::wave_min_u32(~kmax);
        if (lane == 0) {
            s_min[wave] = kmin;
            s_max[wave] = kmax;
        }
        for (int i = tid; i < kBins; i += NT) hist[i] = 0;
        __syncthreads();
        unsigned lo = s_min[0], hi = s_max[0];
#pragma unroll
        for (int w = 1; w < NW; ++w) {
            lo = min(lo, s_min[w]);
            hi = max(hi, s_max[w]);
        }
        for (;;) {
            const unsigned span = hi - lo;
            if (span == 0) {  // the candidates left are equal: the first `take` of them in order
                theta = lo;
                each([&](int run, int j, float v) {
                    const unsigned long long eq = __ballot(j >= lo_t && j < hi_t && dev::ord_key(v) == theta);
                    if (lane == 0) runs[run] = __builtin_popcountll(eq);
                });
                __syncthreads();
                scan_runs<NT>(runs, NI * NW, buf);
                each([&](int run, int j, float v) {
                    const bool e = j >= lo_t && j < hi_t && dev::ord_key(v) == theta;
                    const unsigned long long eq = __ballot(e);
                    if (e && runs[run] + __builtin_popcountll(eq & below) == take - 1) s_j = j;
                });
                __syncthreads();
                last = s_j;
                break;
            }
            const int shift = max(0, 20 - __builtin_clz(span));  // bins 0..4095
            each([&](int, int j, float v) {
                const unsigned u = dev::ord_key(v);
                const bool in = j >= lo_t && j < hi_t && u >= lo && u <= hi;
                const int bin = in ? (int)((u - lo) >> shift) : -1;
                // the bin of the wave's first candidate is counted at once: equal masses (zeros) come in numbers
                const unsigned long long any = __ballot(in);
                if (any) {
                    const int first = __builtin_amdgcn_readlane(bin, __builtin_ctzll(any));
                    const unsigned long long same = __ballot(bin == first);
                    if (lane == 0) atomicAdd(&hist[first], __builtin_popcountll(same));
                    if (in && bin != first) atomicAdd(&hist[bin], 1);
                }
            });
            if (tid == 0) s_n = 0;
            __syncthreads();
            // the bin at which the count from the top reaches `take`; thread t
            // owns the bins from BPT (NT - 1 - t), the highest first
            const int b0 = BPT * (NT - 1 - tid);
            int c[BPT], mine = 0, total;
#pragma unroll
            for (int k = 0; k < BPT; ++k) {
                c[k] = hist[b0 + BPT - 1 - k];
                mine += c[k];
            }
            int above = block_scan<NT>(mine, buf, &total);
#pragma unroll
            for (int k = 0; k < BPT; ++k) {
                if (above < take && above + c[k] >= take) {
                    s_bin = b0 + BPT - 1 - k;
                    s_above = above;
                    s_count = c[k];
                }
                above += c[k];
            }
            __syncthreads();
            const int count = s_count;
            take -= s_above;
            lo += (unsigned)s_bin << shift;
            hi = lo + min(hi - lo, (1u << shift) - 1u);  // the last bin's end may lie past 2^32
            if (take == count) {  // the whole bin
                theta = lo;
                last = 0x7fffffff;
                break;
            }
            if (count <= 64) {  // one wave ranks them
                each([&](int, int j, float v) {
                    const unsigned u = dev::ord_key(v);
                    if (j >= lo_t && j < hi_t && u >= lo && u <= hi) {
                        const int at = atomicAdd(&s_n, 1);
                        s_cand[at] = u;
                        s_cand_j[at] = j;
                    }
                });
                __syncthreads();
                if (tid < count) {
                    const unsigned u = s_cand[tid];
                    const int j = s_cand_j[tid];
                    int rank = 0;
                    for (int k = 0; k < count; ++k) rank += s_cand[k] > u || (s_cand[k] == u && s_cand_j[k] < j);
                    if (rank == take - 1) {
                        s_theta = u;
                        s_j = j;
                    }
                }
                __syncthreads();
                theta = s_theta;
                last = s_j;
                break;
            }
            for (int i = tid; i < kBins; i += NT) hist[i] = 0;
            __syncthreads();
        }
    }
    // ballots of the kept tokens and their counts, run by run
    each([&](int run, int j, float v) {
        const unsigned u = dev::ord_key(v);
        const bool forced = j < lo_t || j >= hi_t;
        const unsigned long long k =
            __ballot(j < N && (forced || (last >= 0 && (u > theta || (u == theta && j <= last)))));
        if (lane == 0) {
            ballots[run] = k;
            runs[run] = __builtin_popcountll(k);
        }
    });
    __syncthreads();
    scan_runs<NT>(runs, NI * NW, buf);

    if constexpr (MODE == kOrder) {
        each([&](int run, int j, float v) {
            const unsigned long long k = ballots[run];
            const int rank = runs[run] + __builtin_popcountll(k & below);
            if (PER == 0) __syncthreads();  // rank <= j: what is written here, every thread has read
            if ((k >> lane) & 1) {
                kept[rank] = j;
                mass[rank] = v;
            }
        });
    } else {
        // kept rows from n on, in order, go to the holes below n, in order
        const int c = runs[n >> 6] + __builtin_popcountll(ballots[n >> 6] & ((1ull << (n & 63)) - 1ull));  // kept below n
        constexpr bool kOwn = MODE == kFillCopy || MODE == kFillCopyMx;
        int* src = kOwn ? hist : a.mv_src + (size_t)h * a.max_moves;
        int* dst = kOwn ? hist + kOwnMoves : a.mv_dst + (size_t)h * a.max_moves;
        // a moved mass waits in its move's slot of dst until its hole's thread takes it
        int* mv = kOwn ? dst : a.mv_val + (size_t)h * a.max_moves;
        each([&](int run, int j, float v) {
            const unsigned long long k = ballots[run];
            if (j >= n && ((k >> lane) & 1)) {
                const int m = runs[run] + __builtin_popcountll(k & below) - c;
                src[m] = j;
                mv[m] = __float_as_int(v);
            }
        });
        __syncthreads();
        each([&](int run, int j, float v) {
            if (j >= n) return;
            const unsigned long long k = ballots[run];
            int from = j;
            if (!((k >> lane) & 1)) {
                const int m = j - (runs[run] + __builtin_popcountll(k & below));
                from = src[m];
                mass[j] = __int_as_float(mv[m]);
                dst[m] = j;
            }
            kept[j] = from;
        });
        if (MODE == kFill && tid == 0) a.mv_n[h] = n - c;
        if constexpr (kOwn) {
            __syncthreads();
            move_rows<NT>(a.K + (size_t)h * a.head_stride, a.V + (size_t)h * a.head_stride, src, dst, n - c, a.vec_shift);
        }
        if constexpr (MODE == kFillCopyMx) move_scales<NT>(a, h, src, dst, n - c);
    }
    if (PER == 0) __syncthreads();  // every mass has been read
    for (int j = n + tid; j < N; j += NT) mass[j] = 0.f;  // the rows that the next tokens take
}

// N <= budget: everything stays.
__global__ void mass_identity_kernel(int32_t* kept, int n, long long total) {
    const long long i = (long long)blockIdx.x * kCopyThreads + threadIdx.x;
    if (i < total) kept[i] = (int)(i % n);
}

// The moves of the hole-filling layout where there are few heads: kCopyMoves
// of a head's list a workgroup.
template <bool MX>
__global__ __launch_bounds__(kCopyThreads) void mass_copy_kernel(MassArgs a, int nchunk) {
    if (!dev::stamp_ok(a.hdr, a.P, a.budget)) return;  // the lists were not written
    const int h = blockIdx.x / nchunk, m0 = (blockIdx.x - h * nchunk) * kCopyMoves;
    const size_t at = (size_t)h * a.max_moves + m0;
    move_rows<kCopyThreads>(a.K + (size_t)h * a.head_stride, a.V + (size_t)h * a.head_stride, a.mv_src + at,
                            a.mv_dst + at, min(kCopyMoves, a.mv_n[h] - m0), a.vec_shift);
    if (MX) move_scales<kCopyThreads>(a, h, a.mv_src + at, a.mv_dst + at, min(kCopyMoves, a.mv_n[h] - m0));
}

template <int NT, int PER>
hipError_t select(const MassArgs& a, int P, int mode, hipStream_t s) {
    const dim3 grid((unsigned)P), block(NT);
    if (mode == kOrder)
        hipLaunchKernelGGL((mass_select_kernel<NT, PER, kOrder>), grid, block, 0, s, a);
    else if constexpr (NT != kShortThreads)
        hipLaunchKernelGGL((mass_select_kernel<NT, PER, kFill>), grid, block, 0, s, a);
    else if (a.KS)
        hipLaunchKernelGGL((mass_select_kernel<NT, PER, kFillCopyMx>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((mass_select_kernel<NT, PER, kFillCopy>), grid, block, 0, s, a);
    return hipGetLastError();
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct MassLayout {
    size_t kept, src, dst, val, n, ballots, runs, end;
    int max_moves, nruns;
};

// Behind the control block; sized by the capacity, so that it serves every N.
// The block holds words of the split selection by score, unused here, as
// bkv_workspace_init clears the whole of it.
MassLayout mass_layout(const bkv_dims& d) {
    MassLayout m;
    const size_t P = (size_t)d.B * d.Hkv;
    bkv_dims full = d;
    full.N = d.N_cap;
    size_t off = up256(ws_layout(full).ctl_end);
    const int past = d.N_cap > d.budget ? d.N_cap - d.budget : 0;
    m.max_moves = past < d.budget ? past : d.budget;
    m.kept = off;
    off = up256(off + 4 * P * (size_t)(d.budget < d.N_cap ? d.budget : d.N_cap));
    m.src = off;
    off = up256(off + 4 * P * m.max_moves);
    m.dst = off;
    off = up256(off + 4 * P * m.max_moves);
    m.val = off;
    off = up256(off + 4 * P * m.max_moves);
    m.n = off;
    off = up256(off + 4 * P);
    m.nruns = d.N_cap > kPerMax * kLongThreads ? (d.N_cap + kLongThreads - 1) / kLongThreads * (kLongThreads / 64) : 0;
    m.ballots = off;
    off = up256(off + 8 * P * (size_t)m.nruns);
    m.runs = off;
    off = up256(off + 4 * P * (size_t)m.nruns);
    m.end = off;
    return m;
}

// K, V and, of a 4-bit cache, KS and VS.
bkv_status evict_run(const bkv_dims* d, int32_t flags, const bkv_mx_cache& c, bool four, float* mass, int32_t* kept, void* ws,
                     size_t ws_bytes, hipStream_t stream) {
    void *K = c.K, *V = c.V;
    if (flags & ~BKV_EVICT_FILL) return BKV_ERR_INVALID;
    const bkv_status st = bkv_validate(d, BKV_OP_COMPACT);
    if (st != BKV_OK) return st;
    if (d->B == 0 || d->N == 0) return BKV_OK;
    if (!K || !V || !mass || ((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) & 15u))
        return BKV_ERR_INVALID;
    if (four && !mx::whole(c)) return BKV_ERR_INVALID;
    // every launch's threads are counted in 32 bits
    if ((long long)d->B * d->Hkv > 0xffffffffLL / kLongThreads) return BKV_ERR_SHAPE;
    const MassLayout m = mass_layout(*d);
    if (!ws || ws_bytes < m.end || (reinterpret_cast<uintptr_t>(ws) & 15u)) return BKV_ERR_WORKSPACE;
    char* w = static_cast<char*>(ws);
    const int P = d->B * d->Hkv;
    const int n = d->N < d->budget ? d->N : d->budget;
    if (d->N <= d->budget && !kept) return BKV_OK;
    const int rb = four ? d->D / 2 : d->D * (d->dtype == BKV_BF16 ? 2 : 4), sb = four ? d->D / mx::kBlock : 0;
    const size_t tokens = (size_t)(P - 1) * d->N_cap + d->N;  // of the last head those that are there
    const Span k = {K, tokens * rb}, v = {V, tokens * rb};
    const Span spans[] = {{mass, tokens * sizeof(float)}, {kept, (size_t)P * n * sizeof(int32_t)}, {ws, m.end}, k, v,
                          {c.KS, tokens * sb}, {c.VS, tokens * sb}};
    if (!apart(spans, 7, 3)) return BKV_ERR_INVALID;
    if (four && !apart(spans + 3, 4, 4)) return BKV_ERR_INVALID;
    // K and V may be one array, whose rows then move once more to the same places,
    // or take turns, the tokens of one behind the other's in every head's rows
    const size_t head = (size_t)d->N_cap * rb, used = (size_t)d->N * rb;
    const uintptr_t k0 = reinterpret_cast<uintptr_t>(K), v0 = reinterpret_cast<uintptr_t>(V);
    const size_t off = (k0 < v0 ? v0 - k0 : k0 - v0) % head;
    if (K != V && overlap(k, v) && (off < used || head - off < used)) return BKV_ERR_INVALID;
    if (d->N <= d->budget) {
        const long long total = (long long)P * n;  // at most 2^31
        hipLaunchKernelGGL(mass_identity_kernel, dim3((unsigned)((total + kCopyThreads - 1) / kCopyThreads)),
                           dim3(kCopyThreads), 0, stream, kept, n, total);
        return hipGetLastError() == hipSuccess ? BKV_OK : BKV_ERR_HIP;
    }
    MassArgs a{};
    a.mass = mass;
    a.kept = kept ? kept : reinterpret_cast<int32_t*>(w + m.kept);
    a.mv_src = reinterpret_cast<int32_t*>(w + m.src);
    a.mv_dst = reinterpret_cast<int32_t*>(w + m.dst);
    a.mv_val = reinterpret_cast<int32_t*>(w + m.val);
    a.mv_n = reinterpret_cast<int32_t*>(w + m.n);
    a.ballots = reinterpret_cast<unsigned long long*>(w + m.ballots);
    a.runs = reinterpret_cast<int32_t*>(w + m.runs);
    a.nruns = m.nruns;
    a.max_moves = m.max_moves;
    a.N = d->N;
    a.N_cap = d->N_cap;
    a.n_keep = n;
    a.W = d->W;
    a.n_prefix = d->n_prefix;
    a.hdr = reinterpret_cast<int*>(w);
    a.P = P;
    a.budget = d->budget;
    a.K = static_cast<char*>(K);
    a.V = static_cast<char*>(V);
    a.head_stride = (size_t)d->N_cap * rb;
    for (a.vec_shift = 0; 16 << a.vec_shift < rb;) ++a.vec_shift;
    if (four) {
        a.KS = c.KS;
        a.VS = c.VS;
        a.scale_bytes = sb;
    }
    const bool fill = flags & BKV_EVICT_FILL;
    const int most = n < a.N - n ? n : a.N - n;  // moves of a head at most
    const int nchunk = (most + kCopyMoves - 1) / kCopyMoves;
    const bool few_moves = fill && a.N <= 16 * kShortThreads && 2LL * most * rb <= kLittle;
    const bool many = few_moves || (P >= (a.N <= 16 * kShortThreads ? kManyHeads : kManyLongHeads) &&
                                    a.N <= kPerMax * kShortThreads && (!fill || most <= kOwnMoves));
    if (fill && !many && (long long)P * nchunk > 0xffffffffLL / kCopyThreads) return BKV_ERR_SHAPE;
    const int mode = !fill ? kOrder : many ? kFillCopy : kFill;
    hipError_t e;
    if (many)
        e = a.N <= 16 * kShortThreads ? select<kShortThreads, 16>(a, P, mode, stream)
                                      : select<kShortThreads, kPerMax>(a, P, mode, stream);
    else if (a.N <= 8 * kLongThreads)
        e = select<kLongThreads, 8>(a, P, mode, stream);
    else if (a.N <= 16 * kLongThreads)  // every pass takes all of its registers: 2 heads of 12932 37 us, with 32 46
        e = select<kLongThreads, 16>(a, P, mode, stream);
    else if (a.N <= 24 * kLongThreads)
        e = select<kLongThreads, 24>(a, P, mode, stream);
    else if (a.N <= kPerMax * kLongThreads)
        e = select<kLongThreads, kPerMax>(a, P, mode, stream);
    else
        e = select<kLongThreads, 0>(a, P, mode, stream);
    if (e != hipSuccess) return BKV_ERR_HIP;
    if (mode == kOrder) {
        e = four ? launch_compact_mx(*d, ws_layout(*d), c, a.kept, ws, stream)
                 : launch_compact(*d, ws_layout(*d), K, V, a.kept, ws, stream);
        return e == hipSuccess ? BKV_OK : BKV_ERR_HIP;
    }
    const dim3 copies((unsigned)(P * nchunk));
    if (mode == kFill && four)
        hipLaunchKernelGGL(mass_copy_kernel<true>, copies, dim3(kCopyThreads), 0, stream, a, nchunk);
    else if (mode == kFill)
        hipLaunchKernelGGL(mass_copy_kernel<false>, copies, dim3(kCopyThreads), 0, stream, a, nchunk);
    return hipGetLastError() == hipSuccess ? BKV_OK : BKV_ERR_HIP;
}

}  // namespace
}  // namespace bkv

extern "C" {

size_t bkv_mass_workspace_bytes(const bkv_dims* d) {
    using namespace bkv;
    if (bkv_validate(d, BKV_OP_COMPACT) != BKV_OK) return 0;
    return mass_layout(*d).end;
}

bkv_status bkv_evict_mass(const bkv_dims* d, int32_t flags, void* K, void* V, float* mass, int32_t* kept, void* ws,
                          size_t ws_bytes, hipStream_t stream) {
    const bkv_mx_cache c = {static_cast<uint8_t*>(K), nullptr, static_cast<uint8_t*>(V), nullptr};
    return bkv::evict_run(d, flags, c, false, mass, kept, ws, ws_bytes, stream);
}

bkv_status bkv_evict_mass_mx(const bkv_dims* d, int32_t flags, const bkv_mx_cache* cache, float* mass, int32_t* kept, void* ws,
                             size_t ws_bytes, hipStream_t stream) {
    return bkv::evict_run(d, flags, cache ? *cache : bkv_mx_cache{}, true, mass, kept, ws, ws_bytes, stream);
}

}  // extern "C"
