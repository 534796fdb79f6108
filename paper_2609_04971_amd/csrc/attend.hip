// Attention of the newest queries over the cache, for gfx950: the streaming
// kernel, the join of its partials, and the weights' sums.
//
// For a row (one query of one query head) with key logits l_j = scale q.k_j:
//   lse = log sum_j exp(l_j),  out = sum_j exp(l_j - lse) v_j
// over the keys it sees.  Everything is kept in log2 units, l2 = l log2(e),
// so that an exponential is one v_exp_f32.  A pass over some of the keys
// leaves m (their maximum), z = sum exp2(l2 - m) and o = sum exp2(l2 - m) v,
// and two such partials join by
//   M = max(m, m'), z <- z exp2(m - M) + z' exp2(m' - M), o likewise.
#include "attend.h"

namespace bkv {
namespace attend {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kWaves = 4;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- one group of keys through the matrix cores ---------------------------------
// Transposed products: S^T = K Q^T puts a row's logits into one lane column
// (lane % 16 is the row, 4 (lane / 16) + i the key), which is the layout the
// B operand of out^T = V^T P^T wants, so the weights never leave their lane.
// The A operand V^T needs the keys of one coordinate in one lane.  V is
// loaded by whole rows, D/16 consecutive coordinates a lane, and transposed
// in registers: coordinate dd of the lane's keys is a byte permute of two
// registers.  MFMA tile dd then holds the coordinates (D/16) m + dd, m the
// lane column, and lane 16 g + row ends up with D/4 consecutive coordinates
// of its row's sum.

template <int D>
struct Bf16 {
    typedef uint16_t elem;
    static constexpr int kKeys = 32;    // keys per group
    static constexpr int kTiles = 2;    // S tiles of 16 keys
    static constexpr int kKK = D / 32;  // 16-byte loads per lane and key tile
    static constexpr int kDV = D / 16;
    struct Q { dev::u32x4 v[kKK]; };
    struct K { dev::u32x4 v[kTiles][kKK]; };
    struct V { unsigned v[8][kDV / 2]; };

    // Which 16-byte chunk of a row (in elements) load kk of lane group g takes.
    __device__ static int chunk(int kk, int g) { return 32 * kk + 8 * g; }

    // Keys [k0, k0 + kKeys) of the head at base; rows past `last` repeat it, so
    // that nothing behind a sequence is read.  A whole group's addresses are a
    // uniform base and lane offsets that never change (off): no arithmetic.
    // Keys and values are read once, and go past the caches.
    struct Off { unsigned k, v; };
    __device__ static Off offsets(int lane) {
        const unsigned m = lane & 15, g = lane >> 4;
        return {m * D + 8 * g, 4 * g * D + kDV * m};
    }
    __device__ static void load_k(K& k, const elem* base, int k0, int last, Off off, int lane) {
        if (k0 + kKeys - 1 <= last) {
            const elem* p = base + (long long)k0 * D;
            dev::static_for<kTiles>([&](auto ac) {
                constexpr int a = decltype(ac)::value;
                dev::static_for<kKK>([&](auto c) {
                    constexpr int kk = decltype(c)::value;
                    k.v[a][kk] = __builtin_nontemporal_load(
                        reinterpret_cast<const dev::u32x4*>(p + 16 * a * D + 32 * kk + off.k));
                });
            });
        } else {
            const int m = lane & 15, g = lane >> 4;
            dev::static_for<kTiles>([&](auto ac) {
                constexpr int a = decltype(ac)::value;
                const elem* p = base + (long long)min(k0 + 16 * a + m, last) * D;
                dev::static_for<kKK>([&](auto c) {
                    constexpr int kk = decltype(c)::value;
                    k.v[a][kk] = *reinterpret_cast<const dev::u32x4*>(p + chunk(kk, g));
                });
            });
        }
    }
    __device__ static void load_v(V& v, const elem* base, int k0, int last, Off off, int lane) {
        if (k0 + kKeys - 1 <= last) {
            const elem* p = base + (long long)k0 * D;
            dev::static_for<8>([&](auto jc) {
                constexpr int j = decltype(jc)::value;
                take(v, decltype(jc){}, p + (16 * (j / 4) + j % 4) * D + off.v);
            });
        } else {
            const int m = lane & 15, g = lane >> 4;
            dev::static_for<8>([&](auto jc) {
                constexpr int j = decltype(jc)::value;
                take(v, decltype(jc){}, base + (long long)min(k0 + 16 * (j / 4) + 4 * g + j % 4, last) * D + kDV * m);
            });
        }
    }
    template <int J>
    __device__ static void take(V& v, std::integral_constant<int, J>, const elem* p) {
        if constexpr (kDV == 8) {
            const dev::u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const dev::u32x4*>(p));
            dev::static_for<4>([&](auto c) { v.v[J][decltype(c)::value] = x[decltype(c)::value]; });
        } else {
            const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
            dev::static_for<2>([&](auto c) { v.v[J][decltype(c)::value] = x[decltype(c)::value]; });
        }
    }
    __device__ static void logits(f32x4 (&s)[kTiles], const K& k, const Q& q) {
        dev::static_for<kTiles>([&](auto ac) {
            constexpr int a = decltype(ac)::value;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            dev::static_for<kKK>([&](auto c) {
                constexpr int kk = decltype(c)::value;
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k.v[a][kk]),
                                                              __builtin_bit_cast(bf16x8_t, q.v[kk]), acc, 0, 0, 0);
            });
            s[a] = acc;
        });
    }
    // o += V^T P^T.  The weights go in as two bf16 terms, high part and rest,
    // so that their rounding (2^-17) stays below the output's own: the
    // streaming kernel waits for memory, and the second product is free.
    template <int NR, int RT>
    __device__ static void values(f32x4 (&o)[RT][kDV], const V& v, const f32x4 (&p)[RT][kTiles]) {
        bf16x8_t hi[NR], lo[NR];
        dev::static_for<NR>([&](auto rc) {
            constexpr int rt = decltype(rc)::value;
            dev::static_for<8>([&](auto jc) {
                constexpr int j = decltype(jc)::value;
                const float x = p[rt][j / 4][j % 4];
                const __bf16 h = (__bf16)x;
                hi[rt][j] = h;
                lo[rt][j] = (__bf16)(x - (float)h);
            });
        });
        dev::static_for<kDV>([&](auto dc) {
            constexpr int dd = decltype(dc)::value;
            constexpr unsigned sel = dd % 2 ? 0x07060302u : 0x05040100u;  // a half of two registers
            dev::u32x4 t;
            dev::static_for<4>([&](auto c) {
                constexpr int i = decltype(c)::value;
                t[i] = __builtin_amdgcn_perm(v.v[2 * i + 1][dd / 2], v.v[2 * i][dd / 2], sel);
            });
            const bf16x8_t a = __builtin_bit_cast(bf16x8_t, t);
            dev::static_for<NR>([&](auto rc) {
                constexpr int rt = decltype(rc)::value;
                o[rt][dd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, hi[rt], o[rt][dd], 0, 0, 0);
                o[rt][dd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, lo[rt], o[rt][dd], 0, 0, 0);
            });
        });
    }
    __device__ static void store4(elem* p, f32x4 x) {
        typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
        *reinterpret_cast<bf16x4_t*>(p) = bf16x4_t{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
    }
};

template <int D>
struct F32 {
    typedef float elem;
    static constexpr int kKeys = 16;
    static constexpr int kTiles = 1;
    static constexpr int kKK = D / 16;
    static constexpr int kDV = D / 16;
    struct Q { f32x4 v[kKK]; };
    struct K { f32x4 v[1][kKK]; };
    struct V { f32x4 v[4][kDV / 4]; };

    __device__ static int chunk(int kk, int g) { return 16 * kk + 4 * g; }

    struct Off { unsigned k, v; };
    __device__ static Off offsets(int lane) {
        const unsigned m = lane & 15, g = lane >> 4;
        return {m * D + 4 * g, 4 * g * D + kDV * m};
    }
    __device__ static void load_k(K& k, const elem* base, int k0, int last, Off off, int lane) {
        const int m = lane & 15, g = lane >> 4;
        const elem* p = k0 + kKeys - 1 <= last ? base + (long long)k0 * D + off.k
                                               : base + (long long)min(k0 + m, last) * D + 4 * g;
        dev::static_for<kKK>([&](auto c) {
            constexpr int kk = decltype(c)::value;
            k.v[0][kk] = *reinterpret_cast<const f32x4*>(p + 16 * kk);
        });
    }
    __device__ static void load_v(V& v, const elem* base, int k0, int last, Off off, int lane) {
        if (k0 + kKeys - 1 <= last) {
            const elem* p = base + (long long)k0 * D;
            dev::static_for<kDV>([&](auto ic) {
                constexpr int j = decltype(ic)::value / (kDV / 4), i = decltype(ic)::value % (kDV / 4);
                v.v[j][i] = *reinterpret_cast<const f32x4*>(p + j * D + 4 * i + off.v);
            });
        } else {
            const int m = lane & 15, g = lane >> 4;
            dev::static_for<kDV>([&](auto ic) {
                constexpr int j = decltype(ic)::value / (kDV / 4), i = decltype(ic)::value % (kDV / 4);
                v.v[j][i] = *reinterpret_cast<const f32x4*>(base + (long long)min(k0 + 4 * g + j, last) * D + kDV * m + 4 * i);
            });
        }
    }
    __device__ static void logits(f32x4 (&s)[1], const K& k, const Q& q) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        dev::static_for<kKK>([&](auto c) {
            constexpr int kk = decltype(c)::value;
            dev::static_for<4>([&](auto jc) {
                constexpr int j = decltype(jc)::value;
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(k.v[0][kk][j], q.v[kk][j], acc, 0, 0, 0);
            });
        });
        s[0] = acc;
    }
    template <int NR, int RT>
    __device__ static void values(f32x4 (&o)[RT][kDV], const V& v, const f32x4 (&p)[RT][1]) {
        dev::static_for<4>([&](auto jc) {
            constexpr int j = decltype(jc)::value;
            dev::static_for<kDV>([&](auto dc) {
                constexpr int dd = decltype(dc)::value;
                dev::static_for<NR>([&](auto rc) {
                    constexpr int rt = decltype(rc)::value;
                    o[rt][dd] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.v[j][dd / 4][dd % 4], p[rt][0][j], o[rt][dd], 0,
                                                                     0, 0);
                });
            });
        });
    }
    __device__ static void store4(elem* p, f32x4 x) { *reinterpret_cast<f32x4*>(p) = x; }
};

// Keys that query t sees: the T queries are the newest tokens of the cache.
__device__ __forceinline__ int seen_by(const Args& a, const Segment& sg, int len, int t) {
    return sg.causal ? max(0, len - a.T + 1 + t) : len;
}

template <class E, int D>
__device__ __forceinline__ typename E::Q load_q(const Args& a, const Row& x, bool valid, int g) {
    typename E::Q q;
    const typename E::elem* p = static_cast<const typename E::elem*>(a.q) + x.q;
    dev::static_for<E::kKK>([&](auto c) {
        constexpr int kk = decltype(c)::value;
        typedef std::remove_reference_t<decltype(q.v[0])> V;
        q.v[kk] = valid ? *reinterpret_cast<const V*>(p + E::chunk(kk, g)) : V{};
    });
    return q;
}

constexpr int kKeptRows = 32;  // rows per unit of kept logits, at most

// Four tokens' weights of one row; what a row that sees nothing has (norm
// +inf) is 0.
__device__ __forceinline__ void add_weights(f32x4& sum, f32x4 l2, float norm) {
    dev::static_for<4>([&](auto c) { sum[decltype(c)::value] += exp2_hw(l2[decltype(c)::value] - norm); });
}

// mass[0..4) += sum, of which `n` are there.
__device__ __forceinline__ void add_mass(float* mass, f32x4 sum, int n) {
    if (n >= 4 && (reinterpret_cast<uintptr_t>(mass) & 15u) == 0) {
        *reinterpret_cast<f32x4*>(mass) += sum;
        return;
    }
    dev::static_for<4>([&](auto c) {
        if (decltype(c)::value < n) mass[decltype(c)::value] += sum[decltype(c)::value];
    });
}

// Pointers into LDS keep their address space, and an index is whole before it
// is added: an LDS address that wraps below its array's start on the way is
// none any more once it is widened.
typedef __attribute__((address_space(3))) float lds_float;
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;

// ---- streaming kernel ------------------------------------------------------------
// One work item: up to 16 RT rows of a unit against a chunk of its keys.  The
// four waves take key groups in turn, each with its own m, z and o, and join
// in LDS at the end.  What bounds it for few rows is the stream of K and V:
// no key passes through LDS, a wave's next keys are requested before this
// group's weights are computed and its next values after they are used, and
// rows that share a kv-head share every load.
// Measured, bf16 of D 128: 4608 units of 3584 tokens 1.31 ms (6.6 TB/s, where a
// probe with these loads alone reaches 7.0), 8 units of 65536 in 32 splits 44 us
// (6.1), 128 of 4224 in two 47 (6.0).  More rows (fp32 caches, prefixes of few
// items) come in row blocks and are bound by the products: fp32, 2048 causal
// queries of 32 heads 350 us (98 TFLOP/s of what is seen, products alone 154).
template <class E, int D, int RT>
__global__ __launch_bounds__(kThreads) void stream_kernel(Args a) {
    constexpr int KG = E::kKeys, NT = E::kTiles, DV = E::kDV;
    constexpr int DP = D + kPadO;  // padded row of the joined sums
    // the waves' sums, [wave][a.o_rows][DP], and with the logits kept in LDS
    // those of the item's keys, [R][chunk + kPadL]
    extern __shared__ __attribute__((aligned(16))) float dyn[];
    __shared__ float s_m[kWaves][16], s_z[kWaves][16], s_norm[kKeptRows];
    lds_float* const s_o = (lds_float*)dyn;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const bool own = (int)blockIdx.x >= a.items0;
    const Segment sg = own ? a.seg[1] : a.seg[0];
    int item = blockIdx.x - (own ? a.items0 : 0);
    // one row block: a unit's splits one after another.  Several (fp32 caches):
    // units fastest, so that an XCD's L2 keeps to few of them, and causal row
    // blocks longest first
    int unit, split, rb = 0;
    if (sg.nrb == 1) {
        split = item % sg.ns;
        unit = item / sg.ns;
    } else {
        unit = turning_unit(sg, item, a.Hkv);
        item /= sg.units;
        split = item % sg.ns;
        rb = item / sg.ns;
        if (sg.causal) rb = sg.nrb - 1 - rb;
    }
    const int len = unit_len(sg, unit, a.Hkv);
    const int r0 = rb * 16 * RT;

    typename E::Q q[RT];
    int lim[RT];  // keys the lane's row sees
    float m[RT], z[RT];
    f32x4 o[RT][DV];
    int most = 0;  // keys that any row of the item sees
    dev::static_for<RT>([&](auto rc) {
        constexpr int rt = decltype(rc)::value;
        const int rr = r0 + 16 * rt + col;
        const bool valid = rr < sg.rows;
        const Row x = decode_row(a, unit, sg.seqs, valid ? rr : 0);
        q[rt] = load_q<E, D>(a, x, valid, g);
        lim[rt] = valid ? seen_by(a, sg, len, x.t) : 0x7fffffff;  // a row that is none masks nothing
        most = max(most, valid ? lim[rt] : 0);
        m[rt] = kLowest;
        z[rt] = 0.f;
        dev::static_for<DV>([&](auto dc) { o[rt][decltype(dc)::value] = f32x4{0.f, 0.f, 0.f, 0.f}; });
    });
    int least = lim[0];
    dev::static_for<RT>([&](auto rc) { least = min(least, lim[decltype(rc)::value]); });
    for (int x = 1; x < 16; x <<= 1) {
        most = max(most, dev::shfl_xor_i(most, x));
        least = min(least, dev::shfl_xor_i(least, x));
    }
    most = __builtin_amdgcn_readfirstlane(most);  // (every lane has them)
    least = __builtin_amdgcn_readfirstlane(least);
    const int k_lo = split * sg.chunk;
    // with the logits kept, keys that no row sees are written too (as -inf)
    const int keep = own ? a.keep : kKeepNone;
    const int k_hi = min(k_lo + sg.chunk, keep ? len : most);
    const typename E::elem* K = static_cast<const typename E::elem*>(sg.K) + (long long)unit * sg.cap * D;
    const typename E::elem* V = static_cast<const typename E::elem*>(sg.V) + (long long)unit * sg.cap * D;
    lds_float* const s_l = s_o + kWaves * a.o_rows * DP;
    const int lds_stride = sg.chunk + kPadL;
    float* const glob = keep ? a.logits + (long long)unit * a.R * a.lstride : nullptr;

    // the keys, for the first NR row tiles
    auto walk = [&](auto nc) __attribute__((always_inline)) {
        constexpr int NR = decltype(nc)::value;
        int k0 = k_lo + KG * wave;
        if (k0 >= k_hi) return;
        const int last = k_hi - 1;  // rows past it repeat it: nothing behind a sequence is read
        typename E::K kr;
        typename E::V vr;
        const typename E::Off off = E::offsets(lane);
        E::load_k(kr, K, k0, last, off, lane);
        E::load_v(vr, V, k0, last, off, lane);
        for (; k0 < k_hi; k0 += KG * kWaves) {
            f32x4 p[RT][NT];
            dev::static_for<NR>([&](auto rc) {
                constexpr int rt = decltype(rc)::value;
                E::logits(p[rt], kr, q[rt]);
            });
            E::load_k(kr, K, k0 + KG * kWaves, last, off, lane);
            const bool edge = k0 + KG > min(least, k_hi);
            dev::static_for<NR>([&](auto rc) {
                constexpr int rt = decltype(rc)::value;
                float top = kLowest;
                dev::static_for<NT * 4>([&](auto ic) {
                    constexpr int ti = decltype(ic)::value / 4, i = decltype(ic)::value % 4;
                    float l = p[rt][ti][i] * a.scale2;
                    if (edge && k0 + 16 * ti + 4 * g + i >= min(lim[rt], k_hi)) l = -INFINITY;
                    p[rt][ti][i] = l;
                    top = fmaxf(top, l);
                });
                if (keep && 16 * rt + col < sg.rows)  // a kept unit is one row block
                    dev::static_for<NT>([&](auto tc) {
                        constexpr int ti = decltype(tc)::value;
                        const int at = k0 + 16 * ti + 4 * g;
                        if (keep == kKeepLds)
                            *(lds_f32x4*)(s_l + ((16 * rt + col) * lds_stride + (at - k_lo))) = p[rt][ti];
                        else
                            *reinterpret_cast<f32x4*>(glob + (long long)(16 * rt + col) * a.lstride + at) = p[rt][ti];
                    });
                top = fmaxf(top, dev::shfl_xor_f(top, 16));
                top = fmaxf(top, dev::shfl_xor_f(top, 32));
                if (__any(top > m[rt])) {
                    const float mn = fmaxf(m[rt], top), f = exp2_hw(m[rt] - mn);
                    m[rt] = mn;
                    z[rt] *= f;
                    dev::static_for<DV>([&](auto dc) { o[rt][decltype(dc)::value] *= f; });
                }
                dev::static_for<NT * 4>([&](auto ic) {
                    constexpr int ti = decltype(ic)::value / 4, i = decltype(ic)::value % 4;
                    const float e = exp2_hw(p[rt][ti][i] - m[rt]);
                    p[rt][ti][i] = e;
                    z[rt] += e;
                });
            });
            E::template values<NR>(o, vr, p);
            E::load_v(vr, V, k0 + KG * kWaves, last, off, lane);
        }
    };
    if constexpr (RT == 2) {
        if (sg.rows - r0 <= 16)
            walk(std::integral_constant<int, 1>{});
        else
            walk(std::integral_constant<int, 2>{});
    } else {
        walk(std::integral_constant<int, 1>{});
    }

    // join the waves, one row tile at a time
    dev::static_for<RT>([&](auto rc) {
        constexpr int rt = decltype(rc)::value;
        float zz = z[rt];
        zz += dev::shfl_xor_f(zz, 16);
        zz += dev::shfl_xor_f(zz, 32);
        if (g == 0) {
            s_m[wave][col] = m[rt];
            s_z[wave][col] = zz;
        }
        if (col < a.o_rows)
            dev::static_for<4>([&](auto ic) {
                constexpr int i = decltype(ic)::value;
                dev::static_for<DV / 4>([&](auto cc) {
                    constexpr int c = decltype(cc)::value;
                    *(lds_f32x4*)(s_o + ((wave * a.o_rows + col) * DP + DV * (4 * g + i) + 4 * c)) =
                        f32x4{o[rt][4 * c][i], o[rt][4 * c + 1][i], o[rt][4 * c + 2][i], o[rt][4 * c + 3][i]};
                });
            });
        __syncthreads();
        constexpr int VPR = D / 4;  // 16-byte vectors of a row
        for (int e = threadIdx.x; e < 16 * VPR; e += kThreads) {
            const int r = e / VPR, v = e % VPR;
            const int rr = r0 + 16 * rt + r;
            if (rr >= sg.rows) break;
            float M = s_m[0][r];
            for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][r]);
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            float Z = 0.f;
            for (int w = 0; w < kWaves; ++w) {
                const float f = exp2_hw(s_m[w][r] - M);
                Z += f * s_z[w][r];
                sum += f * *(const lds_f32x4*)(s_o + ((w * a.o_rows + r) * DP + 4 * v));
            }
            const Row x = decode_row(a, unit, sg.seqs, rr);
            if (a.ns > 1) {
                const long long at = x.gr * a.ns + sg.split0 + split;
                *reinterpret_cast<f32x4*>(a.part_o + at * D + 4 * v) = sum;
                if (v == 0) {
                    a.part_ml[2 * at] = M;
                    a.part_ml[2 * at + 1] = Z;
                }
            } else {
                const RowEnd end = row_end(M, Z);
                E::store4(static_cast<typename E::elem*>(a.out) + x.q + 4 * v, sum * end.inv);
                if (v == 0) {
                    if (a.lse) a.lse[x.lse] = end.lse;
                    if (a.mass) a.row_lse2[x.lse] = end.lse2;
                    if (keep) s_norm[16 * rt + r] = end.lse2;
                }
            }
        }
        __syncthreads();
    });
    if (keep != kKeepLds) return;
    // the kept logits: their weights, or on to the join where other splits
    // have a say in the normalisers
    for (int j = 4 * (int)threadIdx.x; j < k_hi - k_lo; j += 4 * kThreads) {
        if (a.ns > 1) {
            for (int r = 0; r < a.R; ++r)
                *reinterpret_cast<f32x4*>(glob + (long long)r * a.lstride + k_lo + j) =
                    *(const lds_f32x4*)(s_l + (r * lds_stride + j));
        } else {
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            for (int r = 0; r < a.R; ++r) add_weights(sum, *(const lds_f32x4*)(s_l + (r * lds_stride + j)), s_norm[r]);
            add_mass(a.mass + (long long)unit * a.N_cap + k_lo + j, sum, k_hi - k_lo - j);
        }
    }
}

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

// The same from the queries and keys, for more rows of a bf16 cache than the
// logits are kept of, as long as they fit registers: the unit's rows stay there
// and the keys are streamed past them, groups of 32 a wave in turn and
// the next group under way, so that the keys are read once at the rate of
// memory.  S = Q K^T, the transpose of the streaming kernel's: a lane's logits are of one
// key (lane % 16 of a tile) and rows 4 (lane / 16) + i, and a key's sum is the
// lane's own but for one add over the four lane groups.  Bound by the keys'
// reads and the chain of a wave: 54 heads of 48110 tokens and 56 rows 134 us
// (5.0 TB/s; blocks of keys in registers and the rows past them 593), 1504
// heads of 560 and 40 rows 50 (4.3 TB/s; 210).
template <int D, int RT>
__global__ __launch_bounds__(kThreads, 2) void row_mass_kernel(Args a, int chunk) {
    using E = Bf16<D>;
    __shared__ __attribute__((aligned(16))) float s_norm[16 * RT];
    __shared__ __attribute__((aligned(16))) int s_lim[16 * RT];  // keys that the row sees
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    const Segment& sg = a.seg[1];
    const int unit = turning_unit(sg, blockIdx.x, a.Hkv), split = blockIdx.x / sg.units;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int len = unit_len(sg, unit, a.Hkv);
    const int k_lo = split * chunk, k_hi = min(k_lo + chunk, len);
    if (k_lo >= k_hi) return;
    const uint16_t* K = static_cast<const uint16_t*>(sg.K) + (long long)unit * sg.cap * D;
    float* mass = a.mass + (long long)unit * a.N_cap;
    const typename E::Off off = E::offsets(lane);
    struct Group {
        typename E::K k;
        float old;  // the masses of the group's keys, in the first 32 lanes
    };
    auto load = [&](Group& x, int k0) __attribute__((always_inline)) {
        if (k0 < k_hi) {
            E::load_k(x.k, K, k0, len - 1, off, lane);
            x.old = mass[min(k0 + (lane & 31), k_hi - 1)];
        }
    };
    Group one, two;
    load(one, k_lo + E::kKeys * wave);
    const long long row0 = (long long)unit * a.R;
    const uint16_t* q = static_cast<const uint16_t*>(a.q) + row0 * D + 8 * g;
    typename E::Q y[RT];
    dev::static_for<RT>([&](auto rc) {
        constexpr int rt = decltype(rc)::value;
        const int r = 16 * rt + col;
        dev::static_for<E::kKK>([&](auto c) {
            constexpr int kk = decltype(c)::value;
            y[rt].v[kk] = r < a.R ? *reinterpret_cast<const dev::u32x4*>(q + (long long)r * D + 32 * kk) : dev::u32x4{};
        });
    });
    if ((int)threadIdx.x < 16 * RT) {
        const int r = threadIdx.x;
        s_norm[r] = r < a.R ? a.row_lse2[row0 + r] : INFINITY;
        s_lim[r] = sg.causal ? len - a.T + 1 + r % a.T : len;
    }
    __syncthreads();
    const int all = sg.causal ? len - a.T + 1 : len;  // keys that every row sees
    auto step = [&](const Group& x, int k0) __attribute__((always_inline)) {
        f32x4 sum[E::kTiles] = {};
        const bool edge = k0 + E::kKeys > all;
        asm volatile("" ::: "memory");  // or every row's normaliser would be kept in a register
        dev::static_for<RT>([&](auto rc) {
            constexpr int rt = decltype(rc)::value;
            const f32x4 n = *reinterpret_cast<const f32x4*>(s_norm + 16 * rt + 4 * g);
            f32x4 s[E::kTiles] = {};
            dev::static_for<E::kKK * E::kTiles>([&](auto c) {
                constexpr int kk = decltype(c)::value / E::kTiles, t = decltype(c)::value % E::kTiles;
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, y[rt].v[kk]),
                                                               __builtin_bit_cast(bf16x8_t, x.k.v[t][kk]), s[t], 0, 0, 0);
            });
            dev::static_for<E::kTiles>([&](auto tc) {
                constexpr int t = decltype(tc)::value;
                dev::static_for<4>([&](auto ic) {
                    constexpr int i = decltype(ic)::value;
                    s[t][i] = exp2_hw(__builtin_fmaf(s[t][i], a.scale2, -n[i]));
                });
            });
            if (edge) {
                const i32x4 lim = *reinterpret_cast<const i32x4*>(s_lim + 16 * rt + 4 * g);
                dev::static_for<E::kTiles * 4>([&](auto ic) {
                    constexpr int t = decltype(ic)::value / 4, i = decltype(ic)::value % 4;
                    if (k0 + 16 * t + col >= lim[i]) s[t][i] = 0.f;
                });
            }
            dev::static_for<E::kTiles>([&](auto tc) { sum[decltype(tc)::value] += s[decltype(tc)::value]; });
            if (rt % 2) __builtin_amdgcn_sched_barrier(0);
        });
        float v[E::kTiles];
        dev::static_for<E::kTiles>([&](auto tc) {
            constexpr int t = decltype(tc)::value;
            v[t] = (sum[t][0] + sum[t][1]) + (sum[t][2] + sum[t][3]);
            v[t] += dev::shfl_xor_f(v[t], 16);
            v[t] += dev::shfl_xor_f(v[t], 32);
        });
        if (lane < E::kKeys && k0 + lane < k_hi) mass[k0 + lane] = x.old + (g == 0 ? v[0] : v[1]);
    };
    constexpr int kStep = E::kKeys * kWaves;
    for (int k0 = k_lo + E::kKeys * wave; k0 < k_hi; k0 += 2 * kStep) {
        load(two, k0 + kStep);
        step(one, k0);
        if (k0 + kStep >= k_hi) break;
        load(one, k0 + 2 * kStep);
        step(two, k0 + kStep);
    }
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
hipError_t stream(const Args& a, bool wide, hipStream_t s) {
    const long long items = a.items0 + (long long)a.seg[1].units * a.seg[1].nrb * a.seg[1].ns;
    if (items == 0) return hipSuccess;
    if (wide)
        hipLaunchKernelGGL((stream_kernel<E, D, 2>), dim3((unsigned)items), dim3(kThreads), stream_lds(a), s, a);
    else
        hipLaunchKernelGGL((stream_kernel<E, D, 1>), dim3((unsigned)items), dim3(kThreads), stream_lds(a), s, a);
    return hipGetLastError();
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
    const dim3 grid((unsigned)(a.seg[1].units * ns)), block(kThreads);
    if (a.R <= 64) {
        if (a.D == 128)
            hipLaunchKernelGGL((row_mass_kernel<128, 4>), grid, block, 0, s, a, chunk);
        else
            hipLaunchKernelGGL((row_mass_kernel<64, 4>), grid, block, 0, s, a, chunk);
    } else {
        if (a.D == 128)
            hipLaunchKernelGGL((row_mass_kernel<128, 6>), grid, block, 0, s, a, chunk);
        else
            hipLaunchKernelGGL((row_mass_kernel<64, 6>), grid, block, 0, s, a, chunk);
    }
    return hipGetLastError();
}
hipError_t launch_attend_add_parts(const attend::Args& a, const float* part, int parts, hipStream_t s) {
    using namespace attend;
    const long long n = (long long)a.seg[1].units * a.seg[1].n;
    hipLaunchKernelGGL(add_parts_kernel, dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a, part,
                       parts);
    return hipGetLastError();
}

}  // namespace bkv
