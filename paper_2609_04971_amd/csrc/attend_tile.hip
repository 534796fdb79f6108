// Attention of many query rows of a bf16 cache for gfx950 (prompts, chunks,
// the samples of a shared prefix), and the sums of their weights.
//
// More rows than a few make the products the bound, so keys and values go
// through LDS once for 128 rows: a workgroup's four waves own 32 rows each and
// walk the same tiles of 64 keys, two tiles in LDS, the next one loaded
// straight into LDS while this one is computed.
//
// Products are transposed, on 32x32x16 MFMAs: S^T = K Q^T puts a row's logits
// into the two lanes row and row + 32 (h = lane / 32 holds keys 8 (i / 4) + 4 h
// + i % 4), which is the layout the B operand of out^T = V^T P^T takes if the
// contraction runs over the keys in that order: weights never leave their
// lane, and maxima cross lanes once per tile.  The A operand V^T reads V's
// rows through the transposing LDS read (4 keys of a coordinate per lane).
//
// Tiles lie in LDS row by row, the 16-byte chunks of row r permuted by
// chunk ^ f(r), f the bit reversal of r % 8: eight consecutive rows put one
// chunk into eight different bank groups (K), and the transposing read's four
// rows put a pair of chunks into four (V).
#include "attend.h"

namespace bkv {
namespace attend {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kKeys = 64;        // keys per tile
constexpr int kWaveRows = 32;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// The tiles loaded so far have landed in LDS for every wave, and every wave
// is done with the tiles read so far.  The wait is the wave's own: a barrier
// alone does not wait for loads into LDS.
__device__ __forceinline__ void turn() {
    dev::wait_all_memory();
    __syncthreads();
}

__device__ __forceinline__ int swz(int r) { return ((r & 1) << 2) | (r & 2) | ((r >> 2) & 1); }

template <int D>
struct Tile {
    static constexpr int CPR = D / 8;        // 16-byte chunks per row
    static constexpr int RPI = 64 / CPR;     // rows per load instruction
    static constexpr int NI = kKeys / RPI / kWaves;  // load instructions per wave and tile
    static constexpr int KK = D / 16;        // contraction steps of the logits
    static constexpr int DT = D / 32;        // 32-coordinate tiles of the outputs
    static constexpr int ELEMS = kKeys * D;
};

// One tile of rows [0, rows) at base into LDS; rows past them become zero.
template <int D>
__device__ __forceinline__ void load_tile(const uint16_t* base, int rows, uint16_t* stage, int wave, int lane) {
#if defined(__HIP_DEVICE_COMPILE__)
    using T = Tile<D>;
    const __amdgpu_buffer_rsrc_t rsrc =
        __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, max(0, min(rows, kKeys)) * D * 2, 0x00020000);
    dev::static_for<T::NI>([&](auto jc) {
        constexpr int jj = decltype(jc)::value;
        const int j = jj * kWaves + wave;
        const int r = j * T::RPI + lane / T::CPR;
        const int off = r * D * 2 + (((lane % T::CPR) ^ swz(r)) * 16);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(stage + j * 512), 16,
                                                 off, 0, 0, 0);
    });
#endif
}

// A operand of S^T: keys 32 kt + lane % 32, chunk 2 kk + h.
template <int D>
__device__ __forceinline__ bf16x8_t key_frag(const uint16_t* stage, int kt, int kk, int lane) {
    const int r = 32 * kt + (lane & 31), c = 2 * kk + (lane >> 5);
    return *reinterpret_cast<const bf16x8_t*>(stage + r * D + ((c ^ swz(r)) * 8));
}

// A operand of out^T: coordinates 32 dt + lane % 32, keys 16 c + 8 (j / 4) + 4 h + j % 4.
template <int D>
__device__ __forceinline__ bf16x8_t value_frag(const uint16_t* stage, int dt, int c, int lane) {
    s16x4 half[2];
    dev::static_for<2>([&](auto jc) {
        constexpr int jh = decltype(jc)::value;
        const int L = lane & 15, gg = lane >> 4;
        const int r = 16 * c + 8 * jh + 4 * (gg >> 1) + (L >> 2);
        const int chunk = 4 * dt + 2 * (gg & 1) + ((L & 3) >> 1);
        const uint16_t* p = stage + r * D + ((chunk ^ swz(r)) * 8) + (L & 1) * 4;
        half[jh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(const_cast<uint16_t*>(p)));
    });
    return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
}

// The larger of the lane's value and that of lane ^ 32.
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int D>
struct State {
    f32x16 o[D / 32];
    bf16x8_t q[D / 16];
    float m, z;
};

// A row's maximum follows the logits only once they pass it by this much
// (log2): rescaling the sums on every small rise cost more than weights of up
// to 2^8 do.
constexpr float kSlack = 8.f;

// One tile of keys [k0, k0 + 64) against the wave's rows.  edge: some row
// does not see some key (lim: keys that the lane's row sees).
template <int D>
__device__ __forceinline__ void tile_step(State<D>& st, const uint16_t* ks, const uint16_t* vs, int k0, int lim,
                                          bool edge, float scale2, int lane) {
    using T = Tile<D>;
    f32x16 s[2];
    dev::static_for<2>([&](auto tc) {
        constexpr int kt = decltype(tc)::value;
        f32x16 acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        dev::static_for<T::KK>([&](auto kc) {
            constexpr int kk = decltype(kc)::value;
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_frag<D>(ks, kt, kk, lane), st.q[kk], acc, 0, 0, 0);
        });
        s[kt] = acc;
    });
    if (edge) {
        const int h4 = 4 * (lane >> 5);
        dev::static_for<32>([&](auto ic) {
            constexpr int kt = decltype(ic)::value / 16, i = decltype(ic)::value % 16;
            if (k0 + 32 * kt + 8 * (i / 4) + h4 + i % 4 >= lim) s[kt][i] = -INFINITY;
        });
    }
    float top = s[0][0];
    dev::static_for<31>([&](auto ic) {
        constexpr int e = decltype(ic)::value + 1;
        top = fmaxf(top, s[e / 16][e % 16]);
    });
    top = max_halves(top) * scale2;
    if (__any(top > st.m + kSlack)) {
        const float mn = fmaxf(st.m, top), f = exp2_hw(st.m - mn);
        st.m = mn;
        st.z *= f;
        dev::static_for<T::DT>([&](auto dc) { st.o[decltype(dc)::value] *= f; });
    }
    bf16x8_t p[4];
    float z = 0.f;
    dev::static_for<32>([&](auto ic) {
        constexpr int kt = decltype(ic)::value / 16, i = decltype(ic)::value % 16;
        const float e = exp2_hw(__builtin_fmaf(s[kt][i], scale2, -st.m));
        z += e;
        p[2 * kt + i / 8][i % 8] = (__bf16)e;
    });
    st.z += z;
    dev::static_for<4>([&](auto cc) {
        constexpr int c = decltype(cc)::value;
        dev::static_for<T::DT>([&](auto dc) {
            constexpr int dt = decltype(dc)::value;
            st.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value_frag<D>(vs, dt, c, lane), p[c], st.o[dt], 0, 0, 0);
        });
    });
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void tile_kernel(Args a, Segment sg) {
    using T = Tile<D>;
    __shared__ __attribute__((aligned(16))) uint16_t k_a[T::ELEMS], v_a[T::ELEMS], k_b[T::ELEMS], v_b[T::ELEMS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5;
    // units fastest, so that an XCD's L2 keeps to few of them; causal row
    // blocks longest first
    int item = blockIdx.x;
    const int unit = item % sg.units;
    item /= sg.units;
    int rb, split;
    if (sg.causal) {
        split = item % sg.ns;
        rb = sg.nrb - 1 - item / sg.ns;
    } else {
        rb = item % sg.nrb;
        split = item / sg.nrb;
    }
    const int len = sg.lens ? min(max(sg.lens[unit / a.Hkv], 0), sg.n) : sg.n;
    const int r0 = rb * kWaves * kWaveRows;
    const int rr = r0 + wave * kWaveRows + (lane & 31);
    const bool valid = rr < sg.rows;
    const Row x = decode_row(a, unit, sg.seqs, valid ? rr : 0);
    State<D> st;
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + x.q + 8 * h;
    dev::static_for<T::KK>([&](auto kc) {
        constexpr int kk = decltype(kc)::value;
        st.q[kk] = valid ? *reinterpret_cast<const bf16x8_t*>(qp + 16 * kk) : bf16x8_t{};
    });
    dev::static_for<T::DT>([&](auto dc) { st.o[decltype(dc)::value] = f32x16{}; });
    st.m = kLowest;
    st.z = 0.f;
    // keys that the lane's row sees, and the fewest and most of the wave's rows and the workgroup's
    const int lim = valid ? (sg.causal ? max(0, len - a.T + 1 + x.t) : len) : 0x7fffffff;
    int least = lim, most = valid ? lim : 0;
    for (int o = 1; o < 32; o <<= 1) {
        least = min(least, dev::shfl_xor_i(least, o));
        most = max(most, dev::shfl_xor_i(most, o));
    }
    least = __builtin_amdgcn_readfirstlane(least);
    most = __builtin_amdgcn_readfirstlane(most);
    int all = len;
    if (sg.causal) {
        const int last_row = min(r0 + kWaves * kWaveRows, sg.rows) - 1;  // the largest t of the row block (seqs is 1)
        all = max(0, len - a.T + 1 + last_row / a.G);
    }
    const int k_lo = split * sg.chunk, k_hi = min(k_lo + sg.chunk, all);
    const uint16_t* K = static_cast<const uint16_t*>(sg.K) + (long long)unit * sg.cap * D;
    const uint16_t* V = static_cast<const uint16_t*>(sg.V) + (long long)unit * sg.cap * D;
    auto load = [&](int k0, uint16_t* ks, uint16_t* vs) {
        if (k0 < k_hi) {
            load_tile<D>(K + (long long)k0 * D, k_hi - k0, ks, wave, lane);
            load_tile<D>(V + (long long)k0 * D, k_hi - k0, vs, wave, lane);
        }
    };
    auto step = [&](int k0, const uint16_t* ks, const uint16_t* vs) {
        if (k0 < most)
            tile_step<D>(st, ks, vs, k0, min(lim, k_hi), k0 + kKeys > min(least, k_hi), a.scale2, lane);
    };
    load(k_lo, k_a, v_a);
    for (int k0 = k_lo; k0 < k_hi; k0 += 2 * kKeys) {
        turn();  // tile a has landed, tile b is free
        load(k0 + kKeys, k_b, v_b);
        step(k0, k_a, v_a);
        if (k0 + kKeys >= k_hi) break;
        turn();
        load(k0 + 2 * kKeys, k_a, v_a);
        step(k0 + kKeys, k_b, v_b);
    }
    if (!valid) return;
    const auto zr = __builtin_amdgcn_permlane32_swap(__float_as_uint(st.z), __float_as_uint(st.z), false, false);
    const float z = __uint_as_float(zr[0]) + __uint_as_float(zr[1]);
    if (a.ns > 1) {
        const long long at = x.gr * a.ns + sg.split0 + split;
        dev::static_for<T::DT * 4>([&](auto ic) {
            constexpr int dt = decltype(ic)::value / 4, i = decltype(ic)::value % 4;
            *reinterpret_cast<f32x4*>(a.part_o + at * D + 32 * dt + 8 * i + 4 * h) =
                f32x4{st.o[dt][4 * i], st.o[dt][4 * i + 1], st.o[dt][4 * i + 2], st.o[dt][4 * i + 3]};
        });
        if (h == 0) {
            a.part_ml[2 * at] = st.m;
            a.part_ml[2 * at + 1] = z;
        }
    } else {
        const float inv = z > 0.f ? 1.f / z : 0.f;
        uint16_t* out = static_cast<uint16_t*>(a.out) + x.q;
        dev::static_for<T::DT * 4>([&](auto ic) {
            constexpr int dt = decltype(ic)::value / 4, i = decltype(ic)::value % 4;
            typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
            *reinterpret_cast<bf16x4_t*>(out + 32 * dt + 8 * i + 4 * h) =
                bf16x4_t{(__bf16)(st.o[dt][4 * i] * inv), (__bf16)(st.o[dt][4 * i + 1] * inv),
                         (__bf16)(st.o[dt][4 * i + 2] * inv), (__bf16)(st.o[dt][4 * i + 3] * inv)};
        });
        if (h == 0) {
            const float l2 = st.m + log2f(z);
            if (a.lse) a.lse[x.lse] = z > 0.f ? l2 * 0.6931471805599453f : -INFINITY;
            if (a.mass) a.row_lse2[x.gr] = z > 0.f ? l2 : INFINITY;
        }
    }
}

// ---- the weights' sums -----------------------------------------------------------
// mass_j += sum over the unit's rows of exp2(l2_rj - lse2_r).  A workgroup
// holds 64 keys in operand registers (two waves of 32, twice) and walks the
// unit's rows in tiles of 64 through LDS; waves 0, 1 take a tile's first 32
// rows and 2, 3 the others.  A lane sums its 16 keys over its rows in order.
template <int D>
__device__ __forceinline__ void load_rows(const Args& a, const uint16_t* q, int r0, unsigned magic, uint16_t* stage,
                                          int wave, int lane) {
#if defined(__HIP_DEVICE_COMPILE__)
    using T = Tile<D>;
    // the unit's queries: row r = t G + g lies at (g T + t) D
    const __amdgpu_buffer_rsrc_t rsrc =
        __builtin_amdgcn_make_buffer_rsrc((void*)q, (short)0, a.R * D * 2, 0x00020000);
    dev::static_for<T::NI>([&](auto jc) {
        constexpr int jj = decltype(jc)::value;
        const int j = jj * kWaves + wave;
        const int i = j * T::RPI + lane / T::CPR, r = r0 + i;
        const int t = a.G == 1 ? r : (int)__umulhi((unsigned)r, magic), g = r - t * a.G;
        const int off = (g * a.T + t) * D * 2 + (((lane % T::CPR) ^ swz(i)) * 16);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(stage + j * 512), 16,
                                                 r < a.R ? off : 0x7fffffff, 0, 0, 0);
    });
#endif
}

template <int D>
__global__ __launch_bounds__(kThreads) void tile_mass_kernel(Args a, unsigned magic) {
    using T = Tile<D>;
    __shared__ __attribute__((aligned(16))) uint16_t q_a[T::ELEMS], q_b[T::ELEMS];
    __shared__ float s_sum[kKeys];
    const Segment& sg = a.seg[1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, kw = wave & 1, rw = wave >> 1;
    // chunks of keys slowest: the first ones are seen by the most rows
    const int unit = blockIdx.x % sg.units, k0 = blockIdx.x / sg.units * kKeys;
    const int len = sg.lens ? min(max(sg.lens[unit / a.Hkv], 0), sg.n) : sg.n;
    if (k0 >= len) return;
    const int key0 = k0 + 32 * kw;
    const uint16_t* K = static_cast<const uint16_t*>(sg.K) + (long long)unit * sg.cap * D;
    const uint16_t* kp = K + (long long)min(key0 + (lane & 31), len - 1) * D + 8 * h;
    bf16x8_t kr[T::KK];
    dev::static_for<T::KK>([&](auto kc) {
        constexpr int kk = decltype(kc)::value;
        kr[kk] = *reinterpret_cast<const bf16x8_t*>(kp + 16 * kk);
    });
    f32x16 sum = {};
    const int lead = len - a.T;  // key j is seen by queries t >= j - lead
    const int t0 = sg.causal ? min(max(0, k0 - lead), a.T) : 0;
    const int start = t0 * a.G / kKeys * kKeys;
    // rows from here on see all 64 keys
    const int full = sg.causal ? (int)min((long long)a.R, (long long)max(0, k0 + kKeys - 1 - lead) * a.G) : 0;
    const uint16_t* q = static_cast<const uint16_t*>(a.q) + (long long)unit * a.R * D;
    const float* norms = a.row_lse2 + (long long)unit * a.R;
    auto load = [&](int r, uint16_t* stage) {
        if (r < a.R) load_rows<D>(a, q, r, magic, stage, wave, lane);
    };
    auto norm_at = [&](int r) {
        const int i = r + 32 * rw + (lane & 31);
        return i < a.R ? norms[i] : INFINITY;
    };
    auto step = [&](int r, const uint16_t* stage, float norm) {
        f32x16 s = {};
        dev::static_for<T::KK>([&](auto kc) {
            constexpr int kk = decltype(kc)::value;
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kr[kk], key_frag<D>(stage, rw, kk, lane), s, 0, 0, 0);
        });
        if (r < full) {
            const int i = r + 32 * rw + (lane & 31);
            const int t = a.G == 1 ? i : (int)__umulhi((unsigned)i, magic);
            const int lim = lead + 1 + t;  // keys that the row sees
            dev::static_for<16>([&](auto ic) {
                constexpr int e = decltype(ic)::value;
                const float w = exp2_hw(__builtin_fmaf(s[e], a.scale2, -norm));
                sum[e] += key0 + 8 * (e / 4) + 4 * h + e % 4 < lim ? w : 0.f;
            });
        } else {
            dev::static_for<16>([&](auto ic) {
                constexpr int e = decltype(ic)::value;
                sum[e] += exp2_hw(__builtin_fmaf(s[e], a.scale2, -norm));
            });
        }
    };
    load(start, q_a);
    float norm = norm_at(start);
    for (int r = start; r < a.R; r += 2 * kKeys) {
        turn();
        load(r + kKeys, q_b);
        const float next = norm_at(r + kKeys);
        step(r, q_a, norm);
        if (r + kKeys >= a.R) break;
        turn();
        load(r + 2 * kKeys, q_a);
        norm = norm_at(r + 2 * kKeys);
        step(r + kKeys, q_b, next);
    }
    // over the 32 rows of the lanes, then the two row halves
    dev::static_for<16>([&](auto ic) {
        constexpr int e = decltype(ic)::value;
        float v = dev::row16_sum(sum[e]);
        v += dev::shfl_xor_f(v, 16);
        sum[e] = v;
    });
    if (rw == 1 && (lane & 31) == 0)
        dev::static_for<16>([&](auto ic) {
            constexpr int e = decltype(ic)::value;
            s_sum[32 * kw + 8 * (e / 4) + 4 * h + e % 4] = sum[e];
        });
    __syncthreads();
    if (rw == 0 && (lane & 31) == 0)
        dev::static_for<16>([&](auto ic) {
            constexpr int e = decltype(ic)::value;
            const int at = 32 * kw + 8 * (e / 4) + 4 * h + e % 4;
            if (k0 + at < len) a.mass[(long long)unit * a.N_cap + k0 + at] += sum[e] + s_sum[at];
        });
}

}  // namespace
}  // namespace attend

hipError_t launch_attend_tile(const attend::Args& a, const attend::Segment& sg, hipStream_t s) {
    using namespace attend;
    const long long items = (long long)sg.units * sg.nrb * sg.ns;
    if (items == 0) return hipSuccess;
    if (a.D == 128)
        hipLaunchKernelGGL(tile_kernel<128>, dim3((unsigned)items), dim3(kThreads), 0, s, a, sg);
    else
        hipLaunchKernelGGL(tile_kernel<64>, dim3((unsigned)items), dim3(kThreads), 0, s, a, sg);
    return hipGetLastError();
}

hipError_t launch_attend_tile_mass(const attend::Args& a, hipStream_t s) {
    using namespace attend;
    const Segment& sg = a.seg[1];
    if (sg.n == 0 || sg.units == 0) return hipSuccess;
    const unsigned items = (unsigned)sg.units * (unsigned)((sg.n + kKeys - 1) / kKeys);
    const unsigned magic = (unsigned)(((1ull << 32) + a.G - 1) / a.G);  // ceil(2^32 / G): r / G for r G < 2^32
    if (a.D == 128)
        hipLaunchKernelGGL(tile_mass_kernel<128>, dim3(items), dim3(kThreads), 0, s, a, magic);
    else
        hipLaunchKernelGGL(tile_mass_kernel<64>, dim3(items), dim3(kThreads), 0, s, a, magic);
    return hipGetLastError();
}

}  // namespace bkv
