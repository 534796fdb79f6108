// Eviction by accumulated attention weight for gfx950: each head keeps its
// first n_prefix and last W tokens and, of the others, the budget -
// n_prefix - W of largest mass (ties to the lower index); K, V and the
// masses themselves are compacted in place.
//
// One 1024-thread workgroup per head selects.  Masses are heavy-tailed (a
// few sinks hold most of the weight), so they are cut by their order-preserving
// bit pattern, which is about logarithmic: the candidates' range [lo, hi] is
// split into 4096 equal bins, a histogram in LDS finds the bin that holds the
// last one kept, and that bin becomes the range, 12 bits a round and at most
// three rounds.  A round ends the search when its bin is taken whole.  Up to
// 32768 tokens a head's masses stay in registers (token tid + 1024 i), so they
// are read once and moved without a hazard; longer heads read them again on
// every pass.  Kept tokens are ranked with ballots over runs of 64 tokens and
// one scan of the runs' counts.
#include "device_common.h"
#include "internal.h"

namespace bkv {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 4096;
constexpr int kPerMax = 32;  // tokens per thread in registers
constexpr int kCopyThreads = 256;
constexpr int kCopyMoves = 64;  // rows per copy item

struct MassArgs {
    float* mass;
    int32_t* kept;
    // moves of the hole-filling layout, [P][max_moves], and their number [P]
    int32_t* mv_src;
    int32_t* mv_dst;
    float* mv_val;
    int32_t* mv_n;
    int32_t* runs;  // [P][2][nruns], heads longer than the registers hold
    int nruns, max_moves;
    int N, N_cap, n_keep, W, n_prefix, fill;
};

// Exclusive scan of one int per thread over the workgroup; *total is the sum.
__device__ __forceinline__ int block_scan(int v, int* buf, int* total) {
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
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) before += all;
        all += buf[w];
    }
    *total = all;
    __syncthreads();
    return before;
}

__device__ __forceinline__ unsigned block_min(unsigned v, unsigned* buf) {
    v = dev::wave_min_u32(v);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    unsigned m = buf[0];
    for (int w = 1; w < kWaves; ++w) m = min(m, buf[w]);
    __syncthreads();
    return m;
}

// Exclusive scan of n counts in place.
__device__ __forceinline__ void scan_runs(int* runs, int n, int* buf) {
    int base = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        int total;
        const int before = block_scan(i < n ? runs[i] : 0, buf, &total);
        if (i < n) runs[i] = base + before;
        base += total;
    }
    __syncthreads();
}

// PER tokens per thread in registers; 0: read from memory on every pass.
template <int PER>
__global__ __launch_bounds__(kThreads) void mass_select_kernel(MassArgs a) {
    __shared__ int hist[kBins];
    __shared__ int s_runs[2][PER ? PER * kWaves : 1];
    __shared__ int buf[kWaves];
    __shared__ unsigned ubuf[kWaves];
    __shared__ int s_bin, s_above, s_count, s_c;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int h = blockIdx.x, N = a.N, n = a.n_keep;
    float* mass = a.mass + (size_t)h * a.N_cap;
    int32_t* kept = a.kept + (size_t)h * n;
    const int lo_t = a.n_prefix, hi_t = N - a.W;  // candidates [lo_t, hi_t)
    const int NI = PER ? PER : (N + kThreads - 1) / kThreads;
    const int nruns = NI * kWaves;
    int* runs_eq = PER ? s_runs[0] : a.runs + (size_t)h * 2 * a.nruns;
    int* runs_keep = PER ? s_runs[1] : runs_eq + a.nruns;

    float val[PER ? PER : 1];
    if constexpr (PER > 0) {
        dev::static_for<PER>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            val[i] = mass[min(tid + i * kThreads, N - 1)];
        });
    }
    // f(i, token, value) for every token of this thread, whole waves at a time
    auto each = [&](auto&& f) {
        if constexpr (PER > 0) {
            dev::static_for<PER>([&](auto ic) {
                constexpr int i = decltype(ic)::value;
                f(i, tid + i * kThreads, val[i]);
            });
        } else {
            for (int i = 0; i < NI; ++i) {
                const int j = tid + i * kThreads;
                f(i, j, mass[min(j, N - 1)]);
            }
        }
    };

    // the last candidate kept: its order key theta, and how many equal to it
    // are taken
    unsigned theta = 0xffffffffu;
    int take = n - a.n_prefix - a.W;  // > 0 places, or none but the forced ones
    bool ties = false;                // some equal to theta are left out
    if (take > 0) {
        unsigned kmin = 0xffffffffu, kmaxn = 0xffffffffu;
        each([&](int, int j, float v) {
            if (j >= lo_t && j < hi_t) {
                const unsigned u = dev::ord_key(v);
                kmin = min(kmin, u);
                kmaxn = min(kmaxn, ~u);
            }
        });
        unsigned lo = block_min(kmin, ubuf), hi = ~block_min(kmaxn, ubuf);
        for (;;) {
            const unsigned span = hi - lo;
            if (span == 0) {  // every candidate of the range is equal
                theta = lo;
                ties = true;
                break;
            }
            const int shift = max(0, 20 - __builtin_clz(span));  // bins 0..4095
            for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
            __syncthreads();
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
            __syncthreads();
            // the bin at which the count from the top reaches `take`
            const int b0 = 4 * (kThreads - 1 - tid);
            const int c3 = hist[b0 + 3], c2 = hist[b0 + 2], c1 = hist[b0 + 1], c0 = hist[b0];
            int total;
            int above = block_scan(c0 + c1 + c2 + c3, buf, &total);
            const int c[4] = {c3, c2, c1, c0};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (above < take && above + c[k] >= take) {
                    s_bin = b0 + 3 - k;
                    s_above = above;
                    s_count = c[k];
                }
                above += c[k];
            }
            __syncthreads();
            const int bin = s_bin, count = s_count;
            take -= s_above;
            __syncthreads();
            lo += (unsigned)bin << shift;
            if (take == count) {  // the whole bin
                theta = lo;
                break;
            }
            hi = min(hi, lo + ((1u << shift) - 1u));
        }
    }
    // kept: forced, above theta, or one of the first `take` equal to it
    // (without ties, everything from theta on)
    auto forced = [&](int j) { return j < lo_t || j >= hi_t; };
    const bool some = n > a.n_prefix + a.W;
    if (ties) {
        each([&](int i, int j, float v) {
            const unsigned long long eq = __ballot(j < N && !forced(j) && dev::ord_key(v) == theta);
            if (lane == 0) runs_eq[i * kWaves + wave] = __builtin_popcountll(eq);
        });
        __syncthreads();
        scan_runs(runs_eq, nruns, buf);
    }
    const unsigned long long below = (1ull << lane) - 1ull;
    auto is_kept = [&](int i, int j, float v) {
        const unsigned u = dev::ord_key(v);
        bool k = j < N && (forced(j) || (some && (ties ? u > theta : u >= theta)));
        if (ties) {
            const bool e = j < N && !forced(j) && u == theta;
            const unsigned long long eq = __ballot(e);
            if (e) k = runs_eq[i * kWaves + wave] + __builtin_popcountll(eq & below) < take;
        }
        return k;
    };
    each([&](int i, int j, float v) {
        const unsigned long long k = __ballot(is_kept(i, j, v));
        if (lane == 0) runs_keep[i * kWaves + wave] = __builtin_popcountll(k);
    });
    __syncthreads();
    scan_runs(runs_keep, nruns, buf);

    if (!a.fill) {
        // rank <= token, so a pass writes masses at or below the tokens it has read
        each([&](int i, int j, float v) {
            const bool k = is_kept(i, j, v);
            const int rank = runs_keep[i * kWaves + wave] + __builtin_popcountll(__ballot(k) & below);
            if (PER == 0) __syncthreads();
            if (k) {
                kept[rank] = j;
                mass[rank] = v;
            }
        });
    } else {
        // kept rows from n on, in order, go to the holes below n, in order
        int32_t* src = a.mv_src + (size_t)h * a.max_moves;
        int32_t* dst = a.mv_dst + (size_t)h * a.max_moves;
        float* mv = a.mv_val + (size_t)h * a.max_moves;
        each([&](int i, int j, float v) {
            const bool k = is_kept(i, j, v);
            const int rank = runs_keep[i * kWaves + wave] + __builtin_popcountll(__ballot(k) & below);
            if (j == n) s_c = rank;  // kept tokens below n (n < N)
        });
        __syncthreads();
        const int c = s_c;
        each([&](int i, int j, float v) {
            const bool k = is_kept(i, j, v);
            const int rank = runs_keep[i * kWaves + wave] + __builtin_popcountll(__ballot(k) & below);
            if (k && j >= n) {
                src[rank - c] = j;
                mv[rank - c] = v;
            }
        });
        __syncthreads();
        each([&](int i, int j, float v) {
            const bool k = is_kept(i, j, v);
            const int rank = runs_keep[i * kWaves + wave] + __builtin_popcountll(__ballot(k) & below);
            if (j < n) {
                int from = j;
                if (!k) {
                    const int m = j - rank;
                    from = src[m];
                    dst[m] = j;
                    mass[j] = mv[m];
                }
                kept[j] = from;
            }
        });
        if (tid == 0) a.mv_n[h] = n - c;
    }
    __syncthreads();
    for (int j = n + tid; j < N; j += kThreads) mass[j] = 0.f;  // the rows that the next tokens take
}

// N <= budget: everything stays.
__global__ void mass_identity_kernel(int32_t* kept, int n, long long total) {
    const long long i = (long long)blockIdx.x * kCopyThreads + threadIdx.x;
    if (i < total) kept[i] = (int)(i % n);
}

// The moves of the hole-filling layout: sources lie at or above n and
// destinations below it, so no move can read what another writes.
template <int RB>
__global__ __launch_bounds__(kCopyThreads) void mass_copy_kernel(char* K, char* V, MassArgs a, int nchunk,
                                                                 size_t head_stride) {
    constexpr int VPR = RB / 16;
    constexpr int NV = 2 * kCopyMoves * VPR / kCopyThreads;
    const int h = blockIdx.x / nchunk, m0 = (blockIdx.x - h * nchunk) * kCopyMoves;
    const int moves = min(kCopyMoves, a.mv_n[h] - m0);
    if (moves <= 0) return;
    const int32_t* src = a.mv_src + (size_t)h * a.max_moves + m0;
    const int32_t* dst = a.mv_dst + (size_t)h * a.max_moves + m0;
    char* Kh = K + (size_t)h * head_stride;
    char* Vh = V + (size_t)h * head_stride;
    dev::u32x4 b[NV];
    dev::static_for<NV>([&](auto kc) {
        constexpr int k = decltype(kc)::value;
        const int e = threadIdx.x + k * kCopyThreads;
        const int which = e / (kCopyMoves * VPR), r = e / VPR % kCopyMoves, v = e % VPR;
        if (r < moves)
            b[k] = __builtin_nontemporal_load(
                reinterpret_cast<const dev::u32x4*>((which ? Vh : Kh) + (size_t)src[r] * RB) + v);
    });
    dev::static_for<NV>([&](auto kc) {
        constexpr int k = decltype(kc)::value;
        const int e = threadIdx.x + k * kCopyThreads;
        const int which = e / (kCopyMoves * VPR), r = e / VPR % kCopyMoves, v = e % VPR;
        if (r < moves)
            __builtin_nontemporal_store(b[k],
                                        reinterpret_cast<dev::u32x4*>((which ? Vh : Kh) + (size_t)dst[r] * RB) + v);
    });
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct MassLayout {
    size_t kept, src, dst, val, n, runs, end;
    int max_moves, nruns;
};

// Behind the control block; sized by the capacity, so that it serves every N.
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
    m.nruns = d.N_cap > kPerMax * kThreads ? (d.N_cap + kThreads - 1) / kThreads * kWaves : 0;
    m.runs = off;
    off = up256(off + 4 * 2 * P * (size_t)m.nruns);
    m.end = off;
    return m;
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
    using namespace bkv;
    if (flags & ~BKV_EVICT_FILL) return BKV_ERR_INVALID;
    const bkv_status st = bkv_validate(d, BKV_OP_COMPACT);
    if (st != BKV_OK) return st;
    if (d->B == 0 || d->N == 0) return BKV_OK;
    if (!K || !V || !mass || ((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) & 15u))
        return BKV_ERR_INVALID;
    // every launch's threads are counted in 32 bits
    if ((long long)d->B * d->Hkv > 0xffffffffLL / kThreads) return BKV_ERR_SHAPE;
    const MassLayout m = mass_layout(*d);
    if (!ws || ws_bytes < m.end || (reinterpret_cast<uintptr_t>(ws) & 15u)) return BKV_ERR_WORKSPACE;
    char* w = static_cast<char*>(ws);
    const int P = d->B * d->Hkv;
    const int n = d->N < d->budget ? d->N : d->budget;
    if (d->N <= d->budget) {
        if (!kept) return BKV_OK;
        const long long total = (long long)P * n;  // at most 2^31
        hipLaunchKernelGGL(mass_identity_kernel, dim3((unsigned)((total + kCopyThreads - 1) / kCopyThreads)),
                           dim3(kCopyThreads), 0, stream, kept, n, total);
        return hipGetLastError() == hipSuccess ? BKV_OK : BKV_ERR_HIP;
    }
    MassArgs a;
    a.mass = mass;
    a.kept = kept ? kept : reinterpret_cast<int32_t*>(w + m.kept);
    a.mv_src = reinterpret_cast<int32_t*>(w + m.src);
    a.mv_dst = reinterpret_cast<int32_t*>(w + m.dst);
    a.mv_val = reinterpret_cast<float*>(w + m.val);
    a.mv_n = reinterpret_cast<int32_t*>(w + m.n);
    a.runs = reinterpret_cast<int32_t*>(w + m.runs);
    a.nruns = m.nruns;
    a.max_moves = m.max_moves;
    a.N = d->N;
    a.N_cap = d->N_cap;
    a.n_keep = n;
    a.W = d->W;
    a.n_prefix = d->n_prefix;
    a.fill = flags & BKV_EVICT_FILL;
    const int most = n < a.N - n ? n : a.N - n;
    const int nchunk = (most + kCopyMoves - 1) / kCopyMoves;
    if (a.fill && (long long)P * nchunk > 0xffffffffLL / kCopyThreads) return BKV_ERR_SHAPE;
    const dim3 grid((unsigned)P), block(kThreads);
    if (a.N <= 4 * kThreads)
        hipLaunchKernelGGL(mass_select_kernel<4>, grid, block, 0, stream, a);
    else if (a.N <= 16 * kThreads)
        hipLaunchKernelGGL(mass_select_kernel<16>, grid, block, 0, stream, a);
    else if (a.N <= kPerMax * kThreads)
        hipLaunchKernelGGL(mass_select_kernel<kPerMax>, grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL(mass_select_kernel<0>, grid, block, 0, stream, a);
    if (hipGetLastError() != hipSuccess) return BKV_ERR_HIP;
    if (!a.fill) {
        return launch_compact(*d, ws_layout(*d), K, V, a.kept, ws, stream) == hipSuccess ? BKV_OK : BKV_ERR_HIP;
    }
    const int rb = d->D * (d->dtype == BKV_BF16 ? 2 : 4);
    const size_t hs = (size_t)d->N_cap * rb;
    char* k = static_cast<char*>(K);
    char* v = static_cast<char*>(V);
    const dim3 cgrid((unsigned)(P * nchunk)), cblock(kCopyThreads);
    switch (rb) {
        case 128: hipLaunchKernelGGL(mass_copy_kernel<128>, cgrid, cblock, 0, stream, k, v, a, nchunk, hs); break;
        case 256: hipLaunchKernelGGL(mass_copy_kernel<256>, cgrid, cblock, 0, stream, k, v, a, nchunk, hs); break;
        default: hipLaunchKernelGGL(mass_copy_kernel<512>, cgrid, cblock, 0, stream, k, v, a, nchunk, hs); break;
    }
    return hipGetLastError() == hipSuccess ? BKV_OK : BKV_ERR_HIP;
}

}  // extern "C"
