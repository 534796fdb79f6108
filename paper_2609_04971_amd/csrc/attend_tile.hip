// Attention of many query rows of a bf16 cache for gfx950 (prompts, chunks,
// the samples of a shared prefix), and the sums of their weights (of fp32
// caches too).
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
// chunk ^ f(r).  LDS serves 256 bytes a cycle: 16 lanes of a 16-byte read (one
// chunk of 16 consecutive rows, K) or 32 lanes of an 8-byte one (four chunks
// of four rows, V).  f takes the low bits of r to the chunk's high bits, so
// that four rows put their four chunks into four different blocks of 64
// bytes, and is a permutation over 16 rows (over the 8 pairs of rows that
// share 256 bytes, bf16 of D = 64).
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
constexpr int kWaveRows = 32;

// Kinds of instructions for the scheduler.
constexpr int kSchedMfma = 0x8, kSchedLds = 0x100;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// The tiles loaded so far have landed in LDS for every wave, and every wave
// is done with the tiles read so far.  The wait is the wave's own: a barrier
// alone does not wait for loads into LDS.
__device__ __forceinline__ void turn() {
    dev::wait_all_memory();
    __syncthreads();
}

// Position of chunk c of row r is c ^ swz(r).
template <class E>
__device__ __forceinline__ int swz(int r) {
    if constexpr (E::CPR >= 16) return ((r & 3) << 2) | ((r >> 2) & 3);
    return ((r & 2) << 1) | ((r >> 2) & 3);
}

// ROWS rows of [0, rows) at base into LDS; rows past them become zero.
template <class E, int ROWS>
__device__ __forceinline__ void load_tile(const typename E::elem* base, int rows, typename E::elem* stage, int wave,
                                          int lane) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int RB = E::CPR * 16, RPI = 64 / E::CPR;  // bytes of a row, rows of a load instruction
    const __amdgpu_buffer_rsrc_t rsrc =
        __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, max(0, min(rows, ROWS)) * RB, 0x00020000);
    dev::static_for<ROWS / RPI / kWaves>([&](auto jc) {
        const int j = decltype(jc)::value * kWaves + wave;
        const int r = j * RPI + lane / E::CPR;
        const int off = r * RB + (((lane % E::CPR) ^ swz<E>(r)) * 16);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rsrc, (__attribute__((address_space(3))) void*)(reinterpret_cast<char*>(stage) + j * 1024), 16, off, 0, 0, 0);
    });
#endif
}

// Where a lane finds the operands that run over a row's coordinates: of row
// lane % 32, chunk 2 kk + h.  The swizzle depends on r % 16 alone, so that every
// read is one of these offsets and a constant.  Those of fp32's many chunks are
// one offset that 2 kk turns bits of.
template <class E>
struct RowAt {
    int k[E::kRowAts];
    __device__ __forceinline__ explicit RowAt(int lane) {
        const int r = lane & 31, h = lane >> 5;
        dev::static_for<E::kRowAts>([&](auto kc) {
            constexpr int kk = decltype(kc)::value;
            k[kk] = r * E::D + ((2 * kk + h) ^ swz<E>(r)) * E::EPC;
        });
    }
    __device__ __forceinline__ RowAt opaque() const {
        RowAt x = *this;  // or the turned offsets would be kept in registers
        if constexpr (E::kRowAts == 1) asm volatile("" : "+v"(x.k[0]));
        return x;
    }
    template <int KK>
    __device__ __forceinline__ typename E::frag frag(const typename E::elem* stage, std::integral_constant<int, KK>) const {
        const int off = E::kRowAts == 1 ? k[0] ^ (2 * KK * E::EPC) : k[KK % E::kRowAts];
        return *reinterpret_cast<const typename E::frag*>(stage + off);
    }
};

// ---- the two types -----------------------------------------------------------------
template <int D_>
struct Bf16 {
    static constexpr int D = D_;
    typedef uint16_t elem;
    typedef bf16x8_t frag;                  // a chunk's coordinates
    static constexpr int EPC = 8;           // of them
    static constexpr int CPR = D / 8;       // chunks of a row
    static constexpr int KK = D / 16;       // contraction steps of a row, a chunk each half
    static constexpr int kRowAts = KK;
    static constexpr int kKeys = 64;        // keys per tile
    static constexpr int kTiles = kKeys / 32;
    static constexpr int kMassResident = 3;  // workgroups that sum weights to a compute unit

    __device__ __forceinline__ static f32x16 dot(frag a, frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    struct Values { int v[D / 32][2]; };    // coordinates 32 dt + lane % 32, keys 4 h + L / 4 and 8 more
    __device__ __forceinline__ static Values values(int lane) {
        // lanes 4 i .. 4 i + 3 of a group of 16 read 16 coordinates of key i, and
        // lane i of the group ends up with coordinate i of the four keys
        Values o;
        const int L = lane & 15, gg = lane >> 4;
        dev::static_for<D / 16>([&](auto dc) {
            constexpr int dt = decltype(dc)::value / 2, jh = decltype(dc)::value % 2;
            const int r = 8 * jh + 4 * (gg >> 1) + (L >> 2);
            o.v[dt][jh] = r * D + ((4 * dt + 2 * (gg & 1) + ((L & 3) >> 1)) ^ swz<Bf16>(r)) * 8 + (L & 1) * 4;
        });
        return o;
    }
    // Keys 16 c + 8 (j / 4) + 4 h + j % 4 of a coordinate, j = 0..7.
    __device__ __forceinline__ static frag value_frag(const elem* stage, const int (&off)[2], int c) {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4*)(const_cast<uint16_t*>(stage + off[0] + 16 * c * D)));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4*)(const_cast<uint16_t*>(stage + off[1] + 16 * c * D)));
        return __builtin_bit_cast(frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // The weights go into the second product as one bf16 term, each off by at most
    // 2^-8 of itself: outputs are off by 2.2e-3 of their size (rms), 1.65e-3 of it
    // their own rounding.  The streaming kernel's two terms would leave only that,
    // but the products bound this kernel (us, one term and two: prompt of 2 x 4096
    // with weights 425 531, 500 queries against 24001 105 156, 5 drafted tokens 46
    // 50, 64 samples of a prompt 115 121).  Normalisers summed from the rounded
    // weights: 2.16e-3, at 440 and 119 us.
    struct Weights { frag p[4]; };
    template <int I>  // weight I % 16 of key tile I / 16
    __device__ __forceinline__ static void put(Weights& w, std::integral_constant<int, I>, float e) {
        w.p[I / 8][I % 8] = (__bf16)e;
    }
    __device__ __forceinline__ static void add_values(f32x16 (&o)[D / 32], const Weights& w, const Values& at,
                                                      const elem* vs) {
        constexpr int DT = D / 32;
        dev::static_for<4>([&](auto cc) {
            constexpr int c = decltype(cc)::value;
            dev::static_for<DT>([&](auto dc) {
                constexpr int dt = decltype(dc)::value;
                o[dt] = dot(value_frag(vs, at.v[dt], c), w.p[c], o[dt]);
            });
        });
        __builtin_amdgcn_sched_group_barrier(kSchedLds, 8, 1);
        dev::static_for<4 * DT - 4>([&](auto) {
            __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 1);
            __builtin_amdgcn_sched_group_barrier(kSchedLds, 2, 1);
        });
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, 4, 1);
    }
    // six key operands ahead of the products: without it the compiler reads
    // each one right before its product and waits for LDS every time
    __device__ __forceinline__ static void order_logits() {
        constexpr int N = kTiles * KK, AHEAD = 6;
        __builtin_amdgcn_sched_group_barrier(kSchedLds, AHEAD, 0);
        dev::static_for<N - AHEAD>([&](auto) {
            __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kSchedLds, 1, 0);
        });
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, AHEAD, 0);
    }
    __device__ __forceinline__ static void store4(elem* p, f32x4 x) {
        typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
        *reinterpret_cast<bf16x4_t*>(p) = bf16x4_t{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
    }
};

// fp32, for the weights' sums, on 32x32x2 products: a chunk is four steps.
template <int D_>
struct F32 {
    static constexpr int D = D_;
    typedef float elem;
    typedef f32x4 frag;
    static constexpr int EPC = 4;
    static constexpr int CPR = D / 4;
    static constexpr int KK = D / 8;
    static constexpr int kRowAts = 1;
    static constexpr int kMassResident = 2;

    __device__ __forceinline__ static f32x16 dot(frag a, frag b, f32x16 c) {
        dev::static_for<4>([&](auto ec) {
            constexpr int e = decltype(ec)::value;
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        });
        return c;
    }
};

// The larger of the lane's value and that of lane ^ 32.
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <class E>
struct State {
    f32x16 o[E::D / 32];
    typename E::frag q[E::KK];
    float m, z;
};

// New weights of a lane that call for another maximum.  A tile's weights of a
// row then never sum to more than 2 kMost (1 + 2^-8), so that the values' sums
// are finite where values times keys are below 2^128 / 32.1, as promised; it is
// no larger for that, and no smaller because the search costs where it is run
// (us, 2^24, 2^10 and 2^6: a ragged chunk 78 78 80, prompt 433 435 440, 500
// queries against 24001 108 108 109).
constexpr float kMost = 1024.f;

// One tile of keys [k0, k0 + kKeys) against the wave's rows.  edge: some row
// does not see some key (lim: keys that the lane's row sees).
template <class E>
__device__ __forceinline__ void tile_step(State<E>& st, const RowAt<E>& at, const typename E::Values& at_v,
                                          const typename E::elem* ks, const typename E::elem* vs, int k0, int lim,
                                          bool edge, float scale2, int lane) {
    constexpr int N = 16 * E::kTiles;
    f32x16 s[E::kTiles];
    const RowAt<E> at_k = at.opaque();
    dev::static_for<E::kTiles>([&](auto tc) {
        constexpr int kt = decltype(tc)::value;
        f32x16 acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        dev::static_for<E::KK>([&](auto kc) {
            constexpr int kk = decltype(kc)::value;
            acc = E::dot(at_k.frag(ks + 32 * kt * E::D, kc), st.q[kk], acc);
        });
        s[kt] = acc;
    });
    E::order_logits();
    if (edge) {
        const int h4 = 4 * (lane >> 5);
        dev::static_for<N>([&](auto ic) {
            constexpr int kt = decltype(ic)::value / 16, i = decltype(ic)::value % 16;
            if (k0 + 32 * kt + 8 * (i / 4) + h4 + i % 4 >= lim) s[kt][i] = -INFINITY;
        });
    }
    // The exponentials are taken against the running maximum as it stands: the
    // sums are floats, so a weight may be far above 1, and only where a lane's
    // new weights pass kMost (the first tile's, whose m is the lowest float,
    // always do) is the maximum looked for and everything brought down to it.
    // That spares the common tile the search and its wait for every logit.
    typename E::Weights p;
    float z;
    auto weights = [&]() __attribute__((always_inline)) {
        z = 0.f;
        dev::static_for<N>([&](auto ic) {
            constexpr int kt = decltype(ic)::value / 16, i = decltype(ic)::value % 16;
            const float e = exp2_hw(__builtin_fmaf(s[kt][i], scale2, -st.m));
            z += e;
            E::put(p, ic, e);
        });
    };
    weights();
    if (__any(!(z <= kMost))) {
        float top = s[0][0];
        dev::static_for<N - 1>([&](auto ic) {
            constexpr int e = decltype(ic)::value + 1;
            top = fmaxf(top, s[e / 16][e % 16]);
        });
        top = max_halves(top) * scale2;
        const float mn = fmaxf(st.m, top), f = exp2_hw(st.m - mn);
        st.m = mn;
        st.z *= f;
        dev::static_for<E::D / 32>([&](auto dc) { st.o[decltype(dc)::value] *= f; });
        weights();
    }
    st.z += z;
    E::add_values(st.o, p, at_v, vs);
}

// Bound by the chip's power where both products and exponentials run: 2 x 4096
// causal queries of 32 heads 265 us (1.03 PFLOP/s of what is seen; the library's
// product of 8192^3 1.21), and by the exponentials at D 64: 500 queries of 28
// heads against 24001 keys 100 us (850 TFLOP/s).  With 35 to 56 rows it reads
// keys and values at 4.8 to 6.0 TB/s.
template <class E>
__global__ __launch_bounds__(kThreads, 2) void tile_kernel(Args a, Segment sg) {
    using elem = typename E::elem;
    constexpr int D = E::D, DT = D / 32, kKeys = E::kKeys;
    __shared__ __attribute__((aligned(16))) elem k_a[kKeys * D], v_a[kKeys * D], k_b[kKeys * D], v_b[kKeys * D];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5;
    // units fastest, so that an XCD's L2 keeps to few of them; causal row
    // blocks longest first
    int item = blockIdx.x;
    const int unit = turning_unit(sg, item, a.Hkv);
    item /= sg.units;
    int rb, split;
    if (sg.causal) {
        split = item % sg.ns;
        rb = sg.nrb - 1 - item / sg.ns;
    } else {
        rb = item % sg.nrb;
        split = item / sg.nrb;
    }
    const int len = unit_len(sg, unit, a.Hkv);
    const int r0 = rb * kWaves * kWaveRows;
    const int rr = r0 + wave * kWaveRows + (lane & 31);
    const bool valid = rr < sg.rows;
    const Row x = decode_row(a, unit, sg.seqs, valid ? rr : 0);
    State<E> st;
    const elem* qp = static_cast<const elem*>(a.q) + x.q + E::EPC * h;
    dev::static_for<E::KK>([&](auto kc) {
        constexpr int kk = decltype(kc)::value;
        st.q[kk] = valid ? *reinterpret_cast<const typename E::frag*>(qp + 2 * E::EPC * kk) : typename E::frag{};
    });
    dev::static_for<DT>([&](auto dc) { st.o[decltype(dc)::value] = f32x16{}; });
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
    // a prompt's row blocks cut their own keys and ragged sequences theirs, so that
    // their splits are alike and none is empty; others share their tiles in L2
    int chunk = sg.chunk;
    const bool prompt = sg.causal && a.T > sg.n / 5;
    if (prompt || sg.lens) {
        const int each = ((prompt ? all : len) + sg.ns - 1) / sg.ns;
        chunk = __builtin_amdgcn_readfirstlane(max(128, (each + 63) / 64 * 64));
    }
    const int k_lo = split * chunk, k_hi = min(k_lo + chunk, all);
    const elem* K = static_cast<const elem*>(sg.K) + (long long)unit * sg.cap * D;
    const elem* V = static_cast<const elem*>(sg.V) + (long long)unit * sg.cap * D;
    auto load = [&](int k0, elem* ks, elem* vs) {
        if (k0 < k_hi) {
            load_tile<E, kKeys>(K + (long long)k0 * D, k_hi - k0, ks, wave, lane);
            load_tile<E, kKeys>(V + (long long)k0 * D, k_hi - k0, vs, wave, lane);
        }
    };
    const RowAt<E> at_k(lane);
    const typename E::Values at_v = E::values(lane);
    auto step = [&](int k0, const elem* ks, const elem* vs) {
        if (k0 < most)
            tile_step<E>(st, at_k, at_v, ks, vs, k0, min(lim, k_hi), k0 + kKeys > min(least, k_hi), a.scale2, lane);
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
        dev::static_for<DT * 4>([&](auto ic) {
            constexpr int dt = decltype(ic)::value / 4, i = decltype(ic)::value % 4;
            *reinterpret_cast<f32x4*>(a.part_o + at * D + 32 * dt + 8 * i + 4 * h) =
                f32x4{st.o[dt][4 * i], st.o[dt][4 * i + 1], st.o[dt][4 * i + 2], st.o[dt][4 * i + 3]};
        });
        if (h == 0) {
            a.part_ml[2 * at] = st.m;
            a.part_ml[2 * at + 1] = z;
        }
    } else {
        const RowEnd end = row_end(st.m, z);
        elem* out = static_cast<elem*>(a.out) + x.q;
        dev::static_for<DT * 4>([&](auto ic) {
            constexpr int dt = decltype(ic)::value / 4, i = decltype(ic)::value % 4;
            E::store4(out + 32 * dt + 8 * i + 4 * h,
                      f32x4{st.o[dt][4 * i], st.o[dt][4 * i + 1], st.o[dt][4 * i + 2], st.o[dt][4 * i + 3]} * end.inv);
        });
        if (h == 0) {
            if (a.lse) a.lse[x.lse] = end.lse;
            if (a.mass) a.row_lse2[x.lse] = end.lse2;
        }
    }
}

// ---- the weights' sums -----------------------------------------------------------
// mass_j += sum over the unit's rows of exp2(l2_rj - lse2_r).  A workgroup
// holds 128 keys in operand registers and walks the unit's rows in tiles of 64
// through LDS: waves 0, 1 take a tile's first 32 rows and 2, 3 the others,
// each for 64 of the keys.  S = Q K^T here: a lane's logits are of one key
// (lane % 32 of a tile) and rows 8 (i / 4) + 4 h + i % 4, so that a key's sum
// takes four registers and not the rows' lanes (a third workgroup a compute
// unit, and no sum over lanes at the end).  Bound by the exponentials and the
// products, which overlap in part: 2 x 4096 causal queries of 32 heads 161 us
// (850 TFLOP/s of what is seen), 340 queries of 32 heads against 21124 keys 85
// (690; with the rows in the lanes 112).  fp32: 300 queries of 28 heads
// against 16000 285 us (120 of the 154 TFLOP/s that its products reach; 409 with
// every wave loading rows of its own).
template <class E>
__global__ __launch_bounds__(kThreads, E::kMassResident) void tile_mass_kernel(Args a, float* part, int parts) {
    using elem = typename E::elem;
    constexpr int D = E::D, kRows = 64;  // rows per tile
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    __shared__ __attribute__((aligned(16))) elem q_a[kRows * D], q_b[kRows * D];
    __shared__ __attribute__((aligned(16))) float s_norm[2][kRows];  // of the tiles' rows
    __shared__ __attribute__((aligned(16))) int s_lim[2][kRows];     // keys that they see
    __shared__ float s_sum[kMassKeys];
    const Segment& sg = a.seg[1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, kw = wave & 1, rw = wave >> 1;
    // chunks of keys slowest: the first ones are seen by the most rows
    int item = blockIdx.x;
    const int unit = turning_unit(sg, item, a.Hkv);
    item /= sg.units;
    const int pt = item % parts, k0 = item / parts * kMassKeys;
    const int len = unit_len(sg, unit, a.Hkv);
    if (k0 >= len) return;
    const int key0 = k0 + 64 * kw;
    const elem* K = static_cast<const elem*>(sg.K) + (long long)unit * sg.cap * D;
    typename E::frag kr[2][E::KK];
    dev::static_for<2>([&](auto tc) {
        constexpr int kt = decltype(tc)::value;
        const elem* kp = K + (long long)min(key0 + 32 * kt + (lane & 31), len - 1) * D + E::EPC * h;
        dev::static_for<E::KK>([&](auto kc) {
            constexpr int kk = decltype(kc)::value;
            kr[kt][kk] = *reinterpret_cast<const typename E::frag*>(kp + 2 * E::EPC * kk);
        });
    });
    f32x4 sum[2] = {};
    const MassRows rows(a, sg.causal, len, k0, kMassKeys, pt, parts);
    int r = rows.first, t = rows.first_t;  // the tile's first row and its query
    auto load = [&](int row, elem* stage) {
        if (row < rows.end)
            load_tile<E, kRows>(static_cast<const elem*>(a.q) + ((long long)unit * a.R + row) * D, rows.end - row, stage,
                                wave, lane);
    };
    // wave 0 sees to the rows' normalisers: requested with a tile, put into LDS after the one before it
    const float* norms = a.row_lse2 + (long long)unit * a.R + lane;
    auto norm_at = [&](int row) { return wave == 0 && row + lane < rows.end ? norms[row] : INFINITY; };
    auto put = [&](int buf, int row, float norm) {
        if (wave == 0) {
            s_norm[buf][lane] = norm;
            s_lim[buf][lane] = sg.causal ? rows.seen(row + lane) : len;
        }
    };
    const RowAt<E> at(lane);
    auto step = [&](int row, int query, const elem* stage, int buf) {
        f32x16 s[2] = {};
        const RowAt<E> rows_at = at.opaque();
        dev::static_for<E::KK>([&](auto kc) {
            constexpr int kk = decltype(kc)::value;
            const typename E::frag q = rows_at.frag(stage + 32 * rw * D, kc);
            s[0] = E::dot(q, kr[0][kk], s[0]);
            s[1] = E::dot(q, kr[1][kk], s[1]);
        });
        const bool edge = rows.edge(row, query, kRows);
        dev::static_for<4>([&](auto jc) {
            constexpr int j = decltype(jc)::value;
            const f32x4 n = *reinterpret_cast<const f32x4*>(&s_norm[buf][32 * rw + 8 * j + 4 * h]);
            dev::static_for<8>([&](auto ic) {
                constexpr int kt = decltype(ic)::value / 4, i = decltype(ic)::value % 4;
                s[kt][4 * j + i] = exp2_hw(__builtin_fmaf(s[kt][4 * j + i], a.scale2, -n[i]));
            });
            if (edge) {
                const i32x4 lim = *reinterpret_cast<const i32x4*>(&s_lim[buf][32 * rw + 8 * j + 4 * h]);
                dev::static_for<8>([&](auto ic) {
                    constexpr int kt = decltype(ic)::value / 4, i = decltype(ic)::value % 4;
                    if (key0 + 32 * kt + (lane & 31) >= lim[i]) s[kt][4 * j + i] = 0.f;
                });
            }
            dev::static_for<8>([&](auto ic) {
                constexpr int kt = decltype(ic)::value / 4, i = decltype(ic)::value % 4;
                sum[kt][i] += s[kt][4 * j + i];
            });
        });
    };
    load(r, q_a);
    put(0, r, norm_at(r));
    while (r < rows.end) {
        const int ra = r, ta = t;
        rows.advance(r, t, kRows);
        turn();
        load(r, q_b);
        const float nb = norm_at(r);
        step(ra, ta, q_a, 0);
        if (r >= rows.end) break;
        put(1, r, nb);
        const int rb = r, tb = t;
        rows.advance(r, t, kRows);
        turn();
        load(r, q_a);
        const float na = norm_at(r);
        step(rb, tb, q_b, 1);
        put(0, r, na);
    }
    // over a key's four registers, two lanes and two row halves
    float v[2];
    dev::static_for<2>([&](auto tc) {
        constexpr int kt = decltype(tc)::value;
        v[kt] = (sum[kt][0] + sum[kt][1]) + (sum[kt][2] + sum[kt][3]);
        v[kt] += dev::shfl_xor_f(v[kt], 32);
    });
    const int i = 64 * kw + lane;  // the lane's key: half h takes tile h
    const float mine = h == 0 ? v[0] : v[1];
    if (rw == 1) s_sum[i] = mine;
    __syncthreads();
    if (rw == 1 || k0 + i >= len) return;
    if (parts > 1)
        part[((long long)pt * sg.units + unit) * sg.n + k0 + i] = mine + s_sum[i];
    else
        a.mass[(long long)unit * a.N_cap + k0 + i] += mine + s_sum[i];
}

}  // namespace
}  // namespace attend

hipError_t launch_attend_tile(const attend::Args& a, const attend::Segment& sg, hipStream_t s) {
    using namespace attend;
    const long long items = (long long)sg.units * sg.nrb * sg.ns;
    if (items == 0) return hipSuccess;
    if (a.D == 128)
        hipLaunchKernelGGL(tile_kernel<Bf16<128>>, dim3((unsigned)items), dim3(kThreads), 0, s, a, sg);
    else
        hipLaunchKernelGGL(tile_kernel<Bf16<64>>, dim3((unsigned)items), dim3(kThreads), 0, s, a, sg);
    return hipGetLastError();
}

hipError_t launch_attend_tile_mass(const attend::Args& a, int dtype, float* part, int parts, hipStream_t s) {
    using namespace attend;
    const dim3 grid((unsigned)mass_blocks(a, parts)), block(kThreads);
    if (dtype == BKV_BF16 && a.D == 128)
        hipLaunchKernelGGL(tile_mass_kernel<Bf16<128>>, grid, block, 0, s, a, part, parts);
    else if (dtype == BKV_BF16)
        hipLaunchKernelGGL(tile_mass_kernel<Bf16<64>>, grid, block, 0, s, a, part, parts);
    else if (a.D == 128)
        hipLaunchKernelGGL(tile_mass_kernel<F32<128>>, grid, block, 0, s, a, part, parts);
    else
        hipLaunchKernelGGL(tile_mass_kernel<F32<64>>, grid, block, 0, s, a, part, parts);
    return hipGetLastError();
}

}  // namespace bkv
