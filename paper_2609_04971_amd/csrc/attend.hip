// Attention of the newest queries over the cache, for gfx950: the launches of the
// streaming kernel (attend_stream.h), the join of its partials, and the weights' sums.
#include "attend_stream.h"

namespace bkv {
namespace attend {
namespace {

// ---- joining the partials, and the weights of kept logits --------------------------
// One launch.  The first blocks join: the weights exp2(m_s - M) of a row's
// splits in lanes, their sums requested several splits at a time.  A split
// that saw nothing has z = 0 and weight 0; its sums are never used.  Bound by
// the partials' way through memory where there are many rows, which a row to
// D / 4 lanes takes at 3.8 TB/s (44520 rows of D 64 in two splits: 7.6 us, a
// wave a row 21.8).  Many splits come with few rows: four waves a row take
// them in turn.
// The other blocks add the kept logits' weights to the masses, four tokens a
// thread, rows in order, so that no sum depends on the launch:
//   mass_j += sum over the unit's rows of exp2(l2_rj - lse2_r).
// They take the rows' normalisers from the partials themselves.

// A row's results, coordinates [c, c + 4) of them; row gr of the partials.
template <class E, int D>
__device__ __forceinline__ void finish_row(const Args& a, long long gr, int c, f32x4 sum, float M, float Z) {
    const int r = (int)(gr % a.R);
    const long long bh = gr / a.R;
    const int t = r / a.G, g = r - t * a.G;
    const long long at = (bh * a.G + g) * a.T + t;  // (b Hkv + h) G + g is the query head
    const RowEnd end = row_end(M, Z);
    E::store4(static_cast<typename E::elem*>(a.out) + at * D + c, sum * end.inv);
    if (c == 0) {
        if (a.lse) a.lse[at] = end.lse;
        if (a.mass && !a.logits) a.row_lse2[at] = end.lse2;
    }
}

// Up to kFewSplits splits: a row to D / 4 lanes.
template <class E, int D>
__device__ __forceinline__ void join_few(const Args& a) {
    constexpr int LPR = D / 4, AHEAD = 4;
    static_assert(kFewSplits <= LPR, "a lane for every split");
    const int sub = threadIdx.x % LPR, ns = a.ns;
    const long long row = (long long)blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
    if (row >= a.rows) return;  // all lanes of a row at once
    const float* po = a.part_o + row * ns * D + 4 * sub;
    f32x4 v[AHEAD];
    auto load = [&](int s0) {
        dev::static_for<AHEAD>([&](auto kc) {
            constexpr int k = decltype(kc)::value;
            v[k] = *reinterpret_cast<const f32x4*>(po + (long long)min(s0 + k, ns - 1) * D);
        });
    };
    const float* ml = a.part_ml + 2 * (row * ns + min(sub, ns - 1));
    const float m = ml[0], z = sub < ns ? ml[1] : 0.f;
    load(0);
    float M = z != 0.f ? m : kLowest;
    for (int x = 1; x < LPR; x <<= 1) M = fmaxf(M, dev::shfl_xor_f(M, x));
    const float f = z != 0.f ? exp2_hw(m - M) : 0.f;
    float Z = f * z;
    for (int x = 1; x < LPR; x <<= 1) Z += dev::shfl_xor_f(Z, x);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < ns; s0 += AHEAD) {
        dev::static_for<AHEAD>([&](auto kc) {
            constexpr int k = decltype(kc)::value;
            const float w = s0 + k < ns ? __shfl(f, s0 + k, LPR) : 0.f;
            dev::static_for<4>([&](auto c) { sum[decltype(c)::value] += w != 0.f ? w * v[k][decltype(c)::value] : 0.f; });
        });
        if (s0 + AHEAD < ns) load(s0 + AHEAD);
    }
    finish_row<E, D>(a, row, 4 * sub, sum, M, Z);
}

// More: a row to a workgroup.
template <class E, int D>
__device__ __forceinline__ void join_many(const Args& a) {
    constexpr int PER = D / 64;
    __shared__ float s_sum[kWaves][D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long row = blockIdx.x;
    const float* ml = a.part_ml + 2 * row * a.ns;
    const float* po = a.part_o + row * a.ns * D + PER * lane;
    float M = kLowest;
    for (int s = lane; s < a.ns; s += 64)
        if (ml[2 * s + 1] != 0.f) M = fmaxf(M, ml[2 * s]);
    for (int x = 1; x < 64; x <<= 1) M = fmaxf(M, dev::shfl_xor_f(M, x));
    float Z = 0.f, sum[PER] = {};
    for (int s0 = 0; s0 < a.ns; s0 += 64) {
        const int s = s0 + lane;
        float f = 0.f;
        if (s < a.ns && ml[2 * s + 1] != 0.f) {
            f = exp2_hw(ml[2 * s] - M);
            Z += f * ml[2 * s + 1];
        }
        const int n = min(64, a.ns - s0);
        for (int i0 = wave; i0 < n; i0 += 8 * kWaves) {
            float v[8][PER];
            dev::static_for<8>([&](auto kc) {
                constexpr int k = decltype(kc)::value;
                const int i = s0 + min(i0 + k * kWaves, n - 1);
                dev::static_for<PER>([&](auto c) { v[k][decltype(c)::value] = po[(long long)i * D + decltype(c)::value]; });
            });
            dev::static_for<8>([&](auto kc) {
                constexpr int k = decltype(kc)::value;
                const int i = i0 + k * kWaves;
                const float w = i < n ? __shfl(f, i, 64) : 0.f;
                dev::static_for<PER>([&](auto c) {
                    constexpr int e = decltype(c)::value;
                    sum[e] += w != 0.f ? w * v[k][e] : 0.f;
                });
            });
        }
    }
    for (int x = 1; x < 64; x <<= 1) Z += dev::shfl_xor_f(Z, x);
    dev::static_for<PER>([&](auto c) { s_sum[wave][PER * lane + decltype(c)::value] = sum[decltype(c)::value]; });
    __syncthreads();
    const int c = 4 * threadIdx.x;
    if (c >= D) return;
    f32x4 all = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < kWaves; ++w)
        dev::static_for<4>([&](auto ic) { all[decltype(ic)::value] += s_sum[w][c + decltype(ic)::value]; });
    finish_row<E, D>(a, row, c, all, M, Z);
}

__device__ __forceinline__ void kept_mass(const Args& a, int item, int nchunk) {
    __shared__ float s_m[kThreads], s_z[kThreads], s_norm[kKeptRows];
    const int unit = item / nchunk, ch = item % nchunk;
    const Segment& sg = a.seg[1];
    const int len = unit_len(sg, unit, a.Hkv);
    if (ch * kThreads * 4 >= len) return;
    const long long row0 = (long long)unit * a.R;
    if (a.ns > 1) {  // eight threads a row
        const int r = threadIdx.x % kKeptRows;
        float m = kLowest, z = 0.f;
        if (r < a.R) {
            const float* ml = a.part_ml + 2 * (row0 + r) * a.ns;
            for (int s = threadIdx.x / kKeptRows; s < a.ns; s += kThreads / kKeptRows) {
                if (ml[2 * s + 1] == 0.f) continue;
                const float mn = fmaxf(m, ml[2 * s]);
                z = z * exp2_hw(m - mn) + ml[2 * s + 1] * exp2_hw(ml[2 * s] - mn);
                m = mn;
            }
        }
        s_m[threadIdx.x] = m;
        s_z[threadIdx.x] = z;
        __syncthreads();
        if (threadIdx.x < kKeptRows) {
            for (int w = 1; w < kThreads / kKeptRows; ++w) m = fmaxf(m, s_m[threadIdx.x + w * kKeptRows]);
            z = 0.f;
            for (int w = 0; w < kThreads / kKeptRows; ++w)
                z += s_z[threadIdx.x + w * kKeptRows] * exp2_hw(s_m[threadIdx.x + w * kKeptRows] - m);
            s_norm[threadIdx.x] = row_end(m, z).lse2;
        }
    } else if ((int)threadIdx.x < a.R) {
        const int t = threadIdx.x / a.G, g = threadIdx.x - t * a.G;
        s_norm[threadIdx.x] = a.row_lse2[row0 + g * a.T + t];
    }
    __syncthreads();
    const int j = (ch * kThreads + (int)threadIdx.x) * 4;
    if (j >= len) return;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    const float* l = a.logits + row0 * a.lstride + j;
#pragma unroll 4
    for (int r = 0; r < a.R; ++r) {
        add_weights(sum, *reinterpret_cast<const f32x4*>(l + (long long)r * a.lstride), s_norm[r]);
    }
    add_mass(a.mass + (long long)unit * a.N_cap + j, sum, len - j);
}

template <class E, int D, bool FEW>
__global__ __launch_bounds__(kThreads) void join_kernel(Args a, int njoin, int nchunk) {
    if ((int)blockIdx.x >= njoin)
        kept_mass(a, blockIdx.x - njoin, nchunk);
    else if (FEW)
        join_few<E, D>(a);
    else
        join_many<E, D>(a);
}
// The parts' sums, in order.
__global__ __launch_bounds__(kThreads) void add_parts_kernel(Args a, const float* part, int parts) {
    const Segment& sg = a.seg[1];
    const long long i = (long long)blockIdx.x * kThreads + threadIdx.x, n = (long long)sg.units * sg.n;
    if (i >= n) return;
    const int unit = (int)(i / sg.n), j = (int)(i - (long long)unit * sg.n);
    if (j >= unit_len(sg, unit, a.Hkv)) return;
    float v = 0.f;
#pragma unroll 4
    for (int p = 0; p < parts; ++p) v += part[p * n + i];
    a.mass[(long long)unit * a.N_cap + j] += v;
}

template <class E, int D>
hipError_t join(const Args& a, hipStream_t s) {
    const JoinGrid g = join_grid(a);
    if (g.blocks == 0) return hipSuccess;
    const dim3 grid((unsigned)g.blocks), block(kThreads);
    if (g.few)
        hipLaunchKernelGGL((join_kernel<E, D, true>), grid, block, 0, s, a, g.njoin, g.nchunk);
    else
        hipLaunchKernelGGL((join_kernel<E, D, false>), grid, block, 0, s, a, g.njoin, g.nchunk);
    return hipGetLastError();
}

}  // namespace
}  // namespace attend

hipError_t launch_attend_stream(const attend::Args& a, int dtype, bool wide, hipStream_t s) {
    using namespace attend;
    if (dtype == BKV_BF16) return a.D == 128 ? stream<Bf16<128>, 128>(a, wide, s) : stream<Bf16<64>, 64>(a, wide, s);
    return a.D == 128 ? stream<F32<128>, 128>(a, wide, s) : stream<F32<64>, 64>(a, wide, s);
}
hipError_t launch_attend_join(const attend::Args& a, int dtype, hipStream_t s) {
    using namespace attend;
    if (dtype == BKV_BF16) return a.D == 128 ? join<Bf16<128>, 128>(a, s) : join<Bf16<64>, 64>(a, s);
    return a.D == 128 ? join<F32<128>, 128>(a, s) : join<F32<64>, 64>(a, s);
}
hipError_t launch_attend_row_mass(const attend::Args& a, int ns, int chunk, hipStream_t s) {
    using namespace attend;
    return a.D == 128 ? row_mass<Bf16<128>, 128>(a, ns, chunk, s) : row_mass<Bf16<64>, 64>(a, ns, chunk, s);
}
hipError_t launch_attend_add_parts(const attend::Args& a, const float* part, int parts, hipStream_t s) {
    using namespace attend;
    const long long n = (long long)a.seg[1].units * a.seg[1].n;
    hipLaunchKernelGGL(add_parts_kernel, dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a, part,
                       parts);
    return hipGetLastError();
}

}  // namespace bkv
