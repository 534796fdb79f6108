// Rows into the 4-bit cache and out of it (bkv_store_mx, bkv_load_mx), gfx950.
//
// A block's byte comes from its largest magnitude, a maximum over the four
// lanes that hold its 32 coordinates, taken on the bits, which a NaN does not get
// lost in; its codes are those magnitudes over 2^e (exact) rounded to the nearest
// code, ties to the even one, which the conversion instruction does.  Both ways a thread takes eight coordinates of
// K and of V: bound by the bytes (36 x 8 heads of 4096 rows of D 128, 0.76 GB: 124
// us stored, 6.1 TB/s, 108 loaded, 7.1; one row of 4608 heads 3.3 each).
#include "internal.h"
#include "mx.h"

namespace bkv {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;               // coordinates of a thread
constexpr unsigned kMostBlocks = 1u << 20;  // the rest in turns

struct MxArgs {
    const void* in[2];   // K, V rows [B, Hkv, T, D], read (store)
    void* out[2];        // and written (load)
    uint8_t* codes[2];
    uint8_t* scales[2];
    const int32_t* at;   // or null
    int first, T, Hkv, N_cap;
    long long rows;      // B Hkv T
};

// Row of the cache that row r of the call belongs to, -1 outside of it.
__device__ __forceinline__ long long cache_row(const MxArgs& a, unsigned r) {
    const unsigned head = r / (unsigned)a.T, t = r - head * (unsigned)a.T;
    const long long pos = (long long)(a.at ? a.at[head / (unsigned)a.Hkv] : a.first) + t;
    return pos >= 0 && pos < a.N_cap ? (long long)head * a.N_cap + pos : -1;
}

template <int CTRL>
__device__ __forceinline__ unsigned dpp_max(unsigned v) {
    return max(v, (unsigned)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false));
}

// The eight coordinates at p as floats.
__device__ __forceinline__ void take(float (&x)[kPer], const uint16_t* p) {
    const dev::u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const dev::u32x4*>(p));
    dev::static_for<4>([&](auto c) {
        constexpr int i = decltype(c)::value;
        x[2 * i] = __uint_as_float(v[i] << 16);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    });
}
__device__ __forceinline__ void take(float (&x)[kPer], const float* p) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    dev::static_for<2>([&](auto c) {
        constexpr int i = decltype(c)::value;
        const f32x4 v = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p) + i);
        dev::static_for<4>([&](auto e) { x[4 * i + decltype(e)::value] = v[decltype(e)::value]; });
    });
}

template <class E, int D>
__global__ __launch_bounds__(kThreads) void store_kernel(MxArgs a) {
    constexpr int TPR = D / kPer;  // threads of a row, whole quads to a block
    const long long n = a.rows * TPR;
    for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long long)gridDim.x * kThreads) {
        const long long r = i / TPR;
        const int c = (int)(i % TPR);
        const long long to = cache_row(a, (unsigned)r);
        if (to < 0) continue;  // a row's threads together
        float x[2][kPer];
        dev::static_for<2>([&](auto sc) {
            constexpr int s = decltype(sc)::value;
            if (a.in[s]) take(x[s], static_cast<const E*>(a.in[s]) + r * D + c * kPer);
        });
        dev::static_for<2>([&](auto sc) {
            constexpr int s = decltype(sc)::value;
            if (!a.in[s]) return;
            unsigned top = 0;
            dev::static_for<kPer>([&](auto e) { top = max(top, __float_as_uint(x[s][decltype(e)::value]) & 0x7fffffffu); });
            top = dpp_max<0x4e>(dpp_max<0xb1>(top));  // the block's four lanes
            const unsigned byte = mx::scale_byte(top);
            unsigned w = 0;
            dev::static_for<4>([&](auto e) {
                constexpr int k = decltype(e)::value;
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[s][2 * k], x[s][2 * k + 1], mx::scale(byte), k);
            });
            if (byte == mx::kNan) w = 0;
            reinterpret_cast<unsigned*>(a.codes[s])[to * TPR + c] = w;
            if (c % 4 == 0) a.scales[s][to * (TPR / 4) + c / 4] = (uint8_t)byte;
        });
    }
}

__device__ __forceinline__ void put(uint16_t* p, unsigned w, float s) {
    __builtin_nontemporal_store(mx::eight_bf16(w, s), reinterpret_cast<dev::u32x4*>(p));
}
__device__ __forceinline__ void put(float* p, unsigned w, float s) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    const mx::f32x2 x0 = mx::pair_f32<0>(w, s), x1 = mx::pair_f32<1>(w, s), x2 = mx::pair_f32<2>(w, s),
                    x3 = mx::pair_f32<3>(w, s);
    __builtin_nontemporal_store(f32x4{x0[0], x0[1], x1[0], x1[1]}, reinterpret_cast<f32x4*>(p));
    __builtin_nontemporal_store(f32x4{x2[0], x2[1], x3[0], x3[1]}, reinterpret_cast<f32x4*>(p) + 1);
}

template <class E, int D>
__global__ __launch_bounds__(kThreads) void load_kernel(MxArgs a) {
    constexpr int TPR = D / kPer;
    const long long n = a.rows * TPR;
    for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long long)gridDim.x * kThreads) {
        const long long r = i / TPR;
        const int c = (int)(i % TPR);
        const long long from = cache_row(a, (unsigned)r);
        if (from < 0) continue;
        unsigned w[2] = {}, byte[2] = {};
        dev::static_for<2>([&](auto sc) {
            constexpr int s = decltype(sc)::value;
            if (!a.out[s]) return;
            w[s] = reinterpret_cast<const unsigned*>(a.codes[s])[from * TPR + c];
            byte[s] = a.scales[s][from * (TPR / 4) + c / 4];
        });
        dev::static_for<2>([&](auto sc) {
            constexpr int s = decltype(sc)::value;
            if (a.out[s]) put(static_cast<E*>(a.out[s]) + r * D + c * kPer, w[s], mx::scale(byte[s]));
        });
    }
}

template <bool STORE, class E, int D>
hipError_t launch(const MxArgs& a, hipStream_t s) {
    const long long blocks = (a.rows * (D / kPer) + kThreads - 1) / kThreads;
    const dim3 grid((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks));
    if (STORE)
        hipLaunchKernelGGL((store_kernel<E, D>), grid, dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((load_kernel<E, D>), grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Rows k, v (read where `store`, else written) and the cache's rows.
template <bool STORE>
bkv_status run(const bkv_dims* d, const void* k, const void* v, int32_t T, int32_t first, const int32_t* at,
               const bkv_mx_cache* cache, hipStream_t stream) {
    const bkv_status st = bkv_validate(d, BKV_OP_COMPACT);
    if (st != BKV_OK) return st;
    const long long heads = (long long)d->B * d->Hkv;
    if (T < 0 || heads * T > 0x7fffffffLL) return BKV_ERR_SHAPE;
    if (!at && (first < 0 || first > d->N_cap - T)) return BKV_ERR_SHAPE;
    if (d->B == 0 || T == 0) return BKV_OK;
    if (!cache || (!k && !v) || !aligned(k) || !aligned(v)) return BKV_ERR_INVALID;
    const void* rows[2] = {k, v};
    uint8_t* codes[2] = {cache->K, cache->V};
    uint8_t* scales[2] = {cache->KS, cache->VS};
    // what is written and what is read must not meet
    const size_t row = (size_t)d->D * (d->dtype == BKV_BF16 ? 2 : 4), n = (size_t)heads * T, cap = (size_t)heads * d->N_cap;
    Span plain[2], four[4];
    MxArgs a{};
    int np = 0, nf = 0;
    for (int s = 0; s < 2; ++s) {
        if (!rows[s]) continue;
        if (!codes[s] || !scales[s] || !aligned(codes[s]) || !aligned(scales[s])) return BKV_ERR_INVALID;
        plain[np++] = {rows[s], n * row};
        four[nf++] = {codes[s], cap * (size_t)(d->D / 2)};
        four[nf++] = {scales[s], cap * (size_t)(d->D / mx::kBlock)};
        a.in[s] = STORE ? rows[s] : nullptr;
        a.out[s] = STORE ? nullptr : const_cast<void*>(rows[s]);
        a.codes[s] = codes[s];
        a.scales[s] = scales[s];
    }
    Span spans[7];
    int m = 0;
    for (int i = 0; i < (STORE ? nf : np); ++i) spans[m++] = STORE ? four[i] : plain[i];
    const int written = m;
    for (int i = 0; i < (STORE ? np : nf); ++i) spans[m++] = STORE ? plain[i] : four[i];
    spans[m++] = {at, (size_t)d->B * sizeof(int32_t)};
    if (!apart(spans, m, written)) return BKV_ERR_INVALID;
    a.at = at;
    a.first = first;
    a.T = T;
    a.Hkv = d->Hkv;
    a.N_cap = d->N_cap;
    a.rows = heads * T;
    hipError_t e;
    if (d->dtype == BKV_BF16)
        e = d->D == 128 ? launch<STORE, uint16_t, 128>(a, stream) : launch<STORE, uint16_t, 64>(a, stream);
    else
        e = d->D == 128 ? launch<STORE, float, 128>(a, stream) : launch<STORE, float, 64>(a, stream);
    return e == hipSuccess ? BKV_OK : BKV_ERR_HIP;
}

}  // namespace
}  // namespace bkv

extern "C" {

bkv_status bkv_store_mx(const bkv_dims* d, const void* k, const void* v, int32_t T, int32_t first, const int32_t* at,
                        const bkv_mx_cache* cache, hipStream_t stream) {
    return bkv::run<true>(d, k, v, T, first, at, cache, stream);
}

bkv_status bkv_load_mx(const bkv_dims* d, const bkv_mx_cache* cache, int32_t T, int32_t first, const int32_t* at, void* k,
                       void* v, hipStream_t stream) {
    return bkv::run<false>(d, k, v, T, first, at, cache, stream);
}

}  // extern "C"
