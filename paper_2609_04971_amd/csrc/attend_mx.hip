// Attention over a 4-bit cache for gfx950: the streaming kernel's types and its
// launches, and the weights' sums of rows that stay in registers.
//
// A group's codes and bytes are what is streamed; they become bf16 operands in
// registers, exactly, and from there on the products are those of a plain bf16
// cache.  The contraction over a row's coordinates may run in any order that keys
// and queries share: lane group g takes the D/4 that follow one another from
// (D/4) g on, so that a lane's part of a key is one load and lies in one block.
// Few rows are bound by the bytes (4608 heads of 3584 tokens, 4 rows, 2.3 GB: 375
// us, 6.1 TB/s, where the loads alone take 368; one of 65536 tokens, 8 heads: 16.6),
// from about 16 rows on the products and conversions take as long (512 heads of
// 8000 tokens, 32 rows: 125 us, 557 MB; 4000 tokens, 40 rows: 70, 278 MB).
#include "attend_stream.h"
#include "mx.h"

namespace bkv {
namespace attend {
namespace {

// A lane's part of one key, kW words of codes, and of one value row, D/16
// coordinates.  A group's rows are read through a descriptor that ends behind the last key:
// what lies there reads as zeros (a value of 0), so that no row has to be clamped
// and all addresses are a uniform base and lane offsets that never change.
template <int D>
struct MxRows {
    static constexpr int kW = D / 32, kDV = D / 16;
    static constexpr int kCodes = mx::Row<D>::kCodes, kScales = mx::Row<D>::kScales;
    struct Key { unsigned c[kW], s; };
    struct Value { unsigned c, s; };
    struct Off { int kc, ks, vc, vs; };  // of key m and value row 4 g
    __device__ __forceinline__ static Off offsets(int lane) {
        const int m = lane & 15, g = lane >> 4;
        return {m * kCodes + kCodes / 4 * g, m * kScales + g * kScales / 4, 4 * g * kCodes + kDV / 2 * m,
                4 * g * kScales + m * kScales / 16};
    }
#if defined(__HIP_DEVICE_COMPILE__)
    // Rows [k0, k0 + rows), of which those up to `last` are there.
    struct Group {
        __amdgpu_buffer_rsrc_t c, s;
        __device__ __forceinline__ Group(mx::Src p, int k0, int rows, int last) {
            k0 = __builtin_amdgcn_readfirstlane(k0);  // (uniform as it is)
            const int n = __builtin_amdgcn_readfirstlane(max(0, min(rows, last + 1 - k0)));
            c = __builtin_amdgcn_make_buffer_rsrc((void*)(p.c + (long long)k0 * kCodes), (short)0, n * kCodes, 0x00020000);
            s = __builtin_amdgcn_make_buffer_rsrc((void*)(p.s + (long long)k0 * kScales), (short)0, n * kScales, 0x00020000);
        }
        __device__ __forceinline__ Key key(int row, Off o) const {
            Key k;
            if constexpr (kW == 4) {
                const dev::u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(c, o.kc + row * kCodes, 0, 0);
                dev::static_for<4>([&](auto i) { k.c[decltype(i)::value] = x[decltype(i)::value]; });
            } else {
                const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(c, o.kc + row * kCodes, 0, 0);
                dev::static_for<2>([&](auto i) { k.c[decltype(i)::value] = x[decltype(i)::value]; });
            }
            k.s = __builtin_amdgcn_raw_buffer_load_b8(s, o.ks + row * kScales, 0, 0);
            return k;
        }
        __device__ __forceinline__ Value value(int row, Off o) const {
            Value v;
            if constexpr (kDV == 8)
                v.c = __builtin_amdgcn_raw_buffer_load_b32(c, o.vc + row * kCodes, 0, 0);
            else
                v.c = __builtin_amdgcn_raw_buffer_load_b16(c, o.vc + row * kCodes, 0, 0);
            v.s = __builtin_amdgcn_raw_buffer_load_b8(s, o.vs + row * kScales, 0, 0);
            return v;
        }
    };
#endif
};

// bf16 queries.
template <int D>
struct Mx : Bf16<D> {
    using P = Bf16<D>;
    using R = MxRows<D>;
    static constexpr int kKeys = P::kKeys, kTiles = P::kTiles, kKK = P::kKK, kDV = P::kDV;
    struct K { typename R::Key k[kTiles]; };
    struct V { typename R::Value v[8]; };
    typedef mx::Src Src;
    __device__ static Src keys(const Args& a, const Segment& sg, long long row) { return mx::rows<D>(sg.K, a.KS, row); }
    __device__ static Src values_of(const Args& a, const Segment& sg, long long row) { return mx::rows<D>(sg.V, a.VS, row); }
    __device__ static int chunk(int kk, int g) { return D / 4 * g + 8 * kk; }
    using Off = typename R::Off;
    __device__ static Off offsets(int lane) { return R::offsets(lane); }
    __device__ static void load_k(K& k, Src p, int k0, int last, Off o, int) {
#if defined(__HIP_DEVICE_COMPILE__)
        const typename R::Group x(p, k0, kKeys, last);
        dev::static_for<kTiles>([&](auto ac) { k.k[decltype(ac)::value] = x.key(16 * decltype(ac)::value, o); });
#endif
    }
    __device__ static void load_v(V& v, Src p, int k0, int last, Off o, int) {
#if defined(__HIP_DEVICE_COMPILE__)
        const typename R::Group x(p, k0, kKeys, last);
        dev::static_for<8>([&](auto jc) {
            constexpr int j = decltype(jc)::value;
            v.v[j] = x.value(16 * (j / 4) + j % 4, o);
        });
#endif
    }
    __device__ static typename P::K plain(const K& k) {
        typename P::K x;
        dev::static_for<kTiles * kKK>([&](auto c) {
            constexpr int a = decltype(c)::value / kKK, kk = decltype(c)::value % kKK;
            const unsigned w = k.k[a].c[kk];
            const float s = mx::scale(k.k[a].s);
            x.v[a][kk] = mx::eight_bf16(w, s);
        });
        return x;
    }
    static constexpr bool kLazy = true;
    // The keys against the first NR row tiles; query(r): tile r's operands.
    template <int NR, int RT, class F>
    __device__ static void logits_rows(f32x4 (&s)[RT][kTiles], const K& k, F&& query) {
        const typename P::K x = plain(k);
        dev::static_for<NR>([&](auto rc) { P::logits(s[decltype(rc)::value], x, query(rc)); });
    }
    // next: the codes are operands now, and the next ones may be requested.
    template <int NR, int RT, class F>
    __device__ static void values(f32x4 (&o)[RT][kDV], const V& v, const f32x4 (&p)[RT][kTiles], F&& next) {
        const typename P::V x = plain_values(v);
        next(std::integral_constant<int, 0>{});
        products<NR>(o, x, p);
    }
    // (us, weights of three and four row tiles as one term and as two: 35 rows of 8 x 4
    // heads of up to 16001 tokens 26.3 29.5, 63 rows 36.9 43.0; 40 rows of 512 heads of
    // 4000 70 85)
    template <int NR, int RT>
    __device__ static void products(f32x4 (&o)[RT][kDV], const typename P::V& v, const f32x4 (&p)[RT][kTiles]) {
        P::template values<NR, RT, (RT > 2)>(o, v, p);
    }
    template <int H>
    __device__ static void load_half(V& v, Src p, int k0, int last, Off o, int lane) {
        load_v(v, p, k0, last, o, lane);
    }
    __device__ static typename P::V plain_values(const V& v) {
        typename P::V x;
        dev::static_for<8 * kDV / 2>([&](auto c) {
            constexpr int j = decltype(c)::value / (kDV / 2), i = decltype(c)::value % (kDV / 2);
            x.v[j][i] = mx::pair_bf16<i>(v.v[j].c, mx::scale(v.v[j].s));
        });
        return x;
    }
};

// fp32 queries.  What the cache holds is exact in bf16, so fp32 operands of the
// other side go through the bf16 products as three terms of eight bits each, cut
// off one after another: all 24 bits, at 16 / 3 times the rate of fp32 products (us,
// those and these: 512 heads of 4000 tokens, 4 rows 165 56, a prompt of 2048 of 32
// heads 306 104).
template <int D>
struct Mx3 : Mx<D> {
    using M = Mx<D>;
    using P = Bf16<D>;
    typedef float elem;
    static constexpr int kTerms = 3, kKK = M::kKK, kTiles = M::kTiles, kDV = M::kDV;
    struct Q { dev::u32x4 v[kTerms][kKK]; };
    __device__ static void query_terms(Q& q, const float* p, bool valid, int g) {
        dev::static_for<kKK>([&](auto c) {
            constexpr int kk = decltype(c)::value;
            const f32x4* from = reinterpret_cast<const f32x4*>(p + M::chunk(kk, g));
            f32x4 x[2] = {};
            if (valid) {
                x[0] = from[0];
                x[1] = from[1];
            }
            dev::static_for<kTerms * 4>([&](auto ic) {
                constexpr int t = decltype(ic)::value / 4, i = decltype(ic)::value % 4;
                float a = x[i / 2][2 * (i % 2)], b = x[i / 2][2 * (i % 2) + 1];
                q.v[t][kk][i] = mx::cut(a, b);
                x[i / 2][2 * (i % 2)] = a;
                x[i / 2][2 * (i % 2) + 1] = b;
            });
        });
    }
    template <int NR, int RT, class F>
    __device__ static void logits_rows(f32x4 (&s)[RT][kTiles], const typename M::K& k, F&& query) {
        const typename P::K x = M::plain(k);
        dev::static_for<NR>([&](auto rc) {
            constexpr int rt = decltype(rc)::value;
            const Q q = query(rc);
            f32x4 acc[kTiles] = {};
            dev::static_for<kTerms * kKK * kTiles>([&](auto c) {  // the smallest terms first
                constexpr int t = kTerms - 1 - decltype(c)::value / (kKK * kTiles), kk = decltype(c)::value / kTiles % kKK,
                              a = decltype(c)::value % kTiles;
                acc[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x.v[a][kk]),
                                                                 __builtin_bit_cast(bf16x8_t, q.v[t][kk]), acc[a], 0, 0, 0);
            });
            dev::static_for<kTiles>([&](auto ac) { s[rt][decltype(ac)::value] = acc[decltype(ac)::value]; });
        });
    }
    template <int NR, int RT, class F>
    __device__ static void values(f32x4 (&o)[RT][kDV], const typename M::V& v, const f32x4 (&p)[RT][kTiles], F&& next) {
        const typename P::V x = M::plain_values(v);
        next(std::integral_constant<int, 0>{});
        products<NR>(o, x, p);
    }
    template <int NR, int RT>
    __device__ static void products(f32x4 (&o)[RT][kDV], const typename P::V& v, const f32x4 (&p)[RT][kTiles]) {
        dev::u32x4 w[NR][kTerms];
        dev::static_for<NR * 4>([&](auto ic) {
            constexpr int rt = decltype(ic)::value / 4, i = decltype(ic)::value % 4;
            float a = p[rt][i / 2][2 * (i % 2)], b = p[rt][i / 2][2 * (i % 2) + 1];
            dev::static_for<kTerms>([&](auto tc) { w[rt][decltype(tc)::value][i] = mx::cut(a, b); });
        });
        dev::static_for<kDV>([&](auto dc) {
            constexpr int dd = decltype(dc)::value;
            const bf16x8_t a = P::template coordinate<dd>(v);
            dev::static_for<NR * kTerms>([&](auto rc) {
                constexpr int rt = decltype(rc)::value / kTerms, t = kTerms - 1 - decltype(rc)::value % kTerms;
                const bf16x8_t b = __builtin_bit_cast(bf16x8_t, w[rt][t]);
                o[rt][dd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, o[rt][dd], 0, 0, 0);
            });
        });
    }
    __device__ static void store4(elem* p, f32x4 x) { *reinterpret_cast<f32x4*>(p) = x; }
};

// One row tile's items take 64 keys at a time: a wave's requests under way are
// then 8.5 KB, and the search for maxima and the branches come half as often (us,
// 32 and 64 keys: 36 layers of 16 x 8 heads of 3584 tokens 478 439; two row tiles,
// whose registers then leave fewer waves, 125 128).
template <class M>
struct Wide : M {
    static constexpr int kKeys = 2 * M::kKeys, kTiles = 2 * M::kTiles, kDV = M::kDV;
    struct K { typename M::K h[2]; };
    struct V { typename M::V h[2]; };
    typedef mx::Src Src;
    using Off = typename M::Off;
    __device__ static void load_k(K& k, Src p, int k0, int last, Off o, int lane) {
        M::load_k(k.h[0], p, k0, last, o, lane);
        M::load_k(k.h[1], p, k0 + M::kKeys, last, o, lane);
    }
    __device__ static void load_v(V& v, Src p, int k0, int last, Off o, int lane) {
        load_half<0>(v, p, k0, last, o, lane);
        load_half<1>(v, p, k0, last, o, lane);
    }
    template <int H>
    __device__ static void load_half(V& v, Src p, int k0, int last, Off o, int lane) {
        M::load_v(v.h[H], p, k0 + H * M::kKeys, last, o, lane);
    }
    template <int NR, int RT, class F>
    __device__ static void logits_rows(f32x4 (&s)[RT][kTiles], const K& k, F&& query) {
        dev::static_for<2>([&](auto hc) {
            constexpr int h = decltype(hc)::value;
            f32x4 x[RT][M::kTiles];
            M::template logits_rows<NR>(x, k.h[h], query);
            dev::static_for<NR * M::kTiles>([&](auto c) {
                constexpr int r = decltype(c)::value / M::kTiles, t = decltype(c)::value % M::kTiles;
                s[r][M::kTiles * h + t] = x[r][t];
            });
        });
    }
    // next(h): half h's codes are operands now, and the next ones may be requested.
    template <int NR, int RT, class F>
    __device__ static void values(f32x4 (&o)[RT][kDV], const V& v, const f32x4 (&p)[RT][kTiles], F&& next) {
        dev::static_for<2>([&](auto hc) {
            constexpr int h = decltype(hc)::value;
            const auto plain = M::plain_values(v.h[h]);
            next(hc);
            f32x4 x[RT][M::kTiles];
            dev::static_for<NR * M::kTiles>([&](auto c) {
                constexpr int r = decltype(c)::value / M::kTiles, t = decltype(c)::value % M::kTiles;
                x[r][t] = p[r][M::kTiles * h + t];
            });
            M::template products<NR>(o, plain, x);
        });
    }
};

template <int D, bool WIN>
hipError_t stream_mx(const Args& a, int dtype, int rt, hipStream_t s) {
    if (dtype == BKV_F32) switch (rt) {
            case 1: return stream_rows<Wide<Mx3<D>>, D, 1, WIN>(a, s);
            case 2: return stream_rows<Mx3<D>, D, 2, WIN>(a, s);
            default: return stream_rows<Mx3<D>, D, 3, WIN>(a, s);
        }
    switch (rt) {
        case 1: return stream_rows<Wide<Mx<D>>, D, 1, WIN>(a, s);
        case 2: return stream_rows<Mx<D>, D, 2, WIN>(a, s);
        case 3: return stream_rows<Mx<D>, D, 3, WIN>(a, s);
        default: return stream_rows<Mx<D>, D, 4, WIN>(a, s);
    }
}

}  // namespace
}  // namespace attend

hipError_t launch_attend_stream_mx(const attend::Args& a, int dtype, int rt, hipStream_t s) {
    using namespace attend;
    if (a.window > 0) return a.D == 128 ? stream_mx<128, true>(a, dtype, rt, s) : stream_mx<64, true>(a, dtype, rt, s);
    return a.D == 128 ? stream_mx<128, false>(a, dtype, rt, s) : stream_mx<64, false>(a, dtype, rt, s);
}
hipError_t launch_attend_row_mass_mx(const attend::Args& a, int ns, int chunk, hipStream_t s) {
    using namespace attend;
    return a.D == 128 ? row_mass<Mx<128>, 128>(a, ns, chunk, s) : row_mass<Mx<64>, 64>(a, ns, chunk, s);
}

}  // namespace bkv
