// Attention of many query rows over a 4-bit cache for gfx950, and the sums of
// their weights: the tile kernels (attend_tile.h) with keys and values that become
// bf16 on their way.
//
// A tile's codes are requested before the tile in front of it is worked off and
// put into LDS as bf16 values after it, where the products find them as they do
// a plain cache's.  A thread takes whole blocks: 16 bytes of codes, 16
// conversions, four chunks of a row in LDS.  Threads are dealt to blocks so that
// the 16 lanes that LDS serves at once write 16 different positions of 16 bytes.
// Bound as on a plain cache, by the products, with a tenth for the conversions: 2 x
// 4096 causal queries of 32 heads 267 us a call, 294 traced, the sums 160.
#include "attend_tile.h"
#include "mx.h"

namespace bkv {
namespace attend {
namespace {

template <int D_>
struct Mx : Bf16<D_> {
    using P = Bf16<D_>;
    static constexpr int D = D_, kKeys = P::kKeys;
    static constexpr int kCodes = mx::Row<D>::kCodes, kScales = mx::Row<D>::kScales;
    typedef typename P::elem elem;
    typedef typename P::frag frag;
    typedef mx::Src Src;
    __device__ __forceinline__ static Src keys(const Args& a, const Segment& sg, long long row) {
        return mx::rows<D>(sg.K, a.KS, row);
    }
    __device__ __forceinline__ static Src values_of(const Args& a, const Segment& sg, long long row) {
        return mx::rows<D>(sg.V, a.VS, row);
    }
    // D 128: a block of the keys and one of the values a thread.  D 64: one block,
    // waves 0 and 1 the keys', 2 and 3 the values'.
    static constexpr int kStages = 1;
    struct Stage {
        static constexpr int kSides = kKeys * (D / mx::kBlock) / 128;  // of K and V that a thread takes blocks of
        dev::u32x4 c[kSides];
        unsigned s[kSides];
        // the thread's row of the tile, and its block of that row
        __device__ __forceinline__ static int row(int wave, int lane) {
            if constexpr (D == 128) return 16 * wave + 4 * ((lane >> 2) & 3) + (lane >> 4);
            return 32 * (wave & 1) + 16 * (lane >> 5) + 4 * ((lane >> 2) & 3) + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
        }
        __device__ __forceinline__ static int block(int lane) { return lane & (D / mx::kBlock - 1); }
        // rows at or past k_hi repeat the last one: nothing behind a sequence is read
        __device__ __forceinline__ void fetch(Src K, Src V, int k0, int k_hi, int wave, int lane) {
            const long long r = min(k0 + row(wave, lane), k_hi - 1);
            const int b = block(lane);
            dev::static_for<kSides>([&](auto ic) {
                constexpr int i = decltype(ic)::value;
                const bool values = kSides == 2 ? i == 1 : wave >= 2;
                const Src p = {values ? V.c : K.c, values ? V.s : K.s};
                c[i] = *reinterpret_cast<const dev::u32x4*>(p.c + r * kCodes + 16 * b);
                s[i] = p.s[r * kScales + b];
            });
        }
        __device__ __forceinline__ void commit(elem* ks, elem* vs, int wave, int lane) {
            // the four chunks' places, worked out anew for every tile: kept, as they are
            // for each of four arrays, they would cost 16 registers
            int r = row(wave, lane), b = 4 * block(lane);
            asm volatile("" : "+v"(r), "+v"(b));
            dev::static_for<kSides>([&](auto ic) {
                constexpr int i = decltype(ic)::value;
                elem* stage = (kSides == 2 ? i == 1 : wave >= 2) ? vs : ks;
                const float x = mx::scale(s[i]);
                dev::static_for<4>([&](auto jc) {
                    constexpr int j = decltype(jc)::value;
                    *reinterpret_cast<dev::u32x4*>(stage + r * D + ((b + j) ^ swz<P>(r)) * 8) = mx::eight_bf16(c[i][j], x);
                });
            });
        }
    };
    // Chunk 2 kk + h of a key: a word of codes.
    struct KeyAt {
        const unsigned* c;
        const uint8_t* s;
        int h;
        __device__ __forceinline__ KeyAt(Src K, int row, int h_)
            : c(reinterpret_cast<const unsigned*>(K.c + (long long)row * kCodes)), s(K.s + (long long)row * kScales), h(h_) {}
        template <int KK>
        __device__ __forceinline__ frag operator()(std::integral_constant<int, KK>) const {
            return __builtin_bit_cast(frag, mx::eight_bf16(c[2 * KK + h], mx::scale(s[KK / 2])));
        }
    };
};

// fp32 queries, for the weights' sums: three bf16 terms of a query's coordinates,
// cut off one after another as they come from LDS, against keys that are exact in
// bf16.  Two chunks of four floats make a step of 16 coordinates.  2048 causal
// queries of 32 heads: 81 us, 236 with fp32 products.
template <int D_>
struct Mx3 {
    static constexpr int D = D_;
    typedef float elem;
    typedef bf16x8_t frag;  // of a key
    static constexpr int EPC = 4, CPR = D / 4, KK = D / 16, kMassResident = 2;
    typedef mx::Src Src;
    __device__ __forceinline__ static Src keys(const Args& a, const Segment& sg, long long row) {
        return mx::rows<D>(sg.K, a.KS, row);
    }
    typedef typename Mx<D>::KeyAt KeyAt;
    struct Query { frag t[3]; };
    __device__ __forceinline__ static f32x16 dot(const Query& a, frag b, f32x16 c) {
        dev::static_for<3>([&](auto tc) {  // the smallest term first
            c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.t[2 - decltype(tc)::value], b, c, 0, 0, 0);
        });
        return c;
    }
};

}  // namespace

// Rows of floats: chunks 4 kk + 2 h and the next of row lane % 32.
template <int D_>
struct RowAt<Mx3<D_>> {
    using E = Mx3<D_>;
    int k;
    __device__ __forceinline__ explicit RowAt(int lane) {
        const int r = lane & 31, h = lane >> 5;
        k = r * E::D + ((2 * h) ^ swz<E>(r)) * E::EPC;
    }
    __device__ __forceinline__ RowAt opaque() const {
        RowAt x = *this;
        asm volatile("" : "+v"(x.k));
        return x;
    }
    template <int KK>
    __device__ __forceinline__ typename E::Query frag(const float* stage, std::integral_constant<int, KK>) const {
        f32x4 x[2];
        dev::static_for<2>([&](auto ec) {
            constexpr int e = decltype(ec)::value;
            x[e] = *reinterpret_cast<const f32x4*>(stage + (k ^ ((4 * KK + e) * E::EPC)));
        });
        typename E::Query q;
        dev::static_for<3>([&](auto tc) {
            dev::u32x4 w;
            dev::static_for<4>([&](auto ic) {
                constexpr int i = decltype(ic)::value;
                float a = x[i / 2][2 * (i % 2)], b = x[i / 2][2 * (i % 2) + 1];
                w[i] = mx::cut(a, b);
                x[i / 2][2 * (i % 2)] = a;
                x[i / 2][2 * (i % 2) + 1] = b;
            });
            q.t[decltype(tc)::value] = __builtin_bit_cast(bf16x8_t, w);
        });
        return q;
    }
};

}  // namespace attend

hipError_t launch_attend_tile_mx(const attend::Args& a, const attend::Segment& sg, hipStream_t s) {
    using namespace attend;
    return a.D == 128 ? tile<Mx<128>>(a, sg, s) : tile<Mx<64>>(a, sg, s);
}

hipError_t launch_attend_tile_mass_mx(const attend::Args& a, int dtype, float* part, int parts, hipStream_t s) {
    using namespace attend;
    if (dtype == BKV_BF16) return a.D == 128 ? tile_mass<Mx<128>>(a, part, parts, s) : tile_mass<Mx<64>>(a, part, parts, s);
    return a.D == 128 ? tile_mass<Mx3<128>>(a, part, parts, s) : tile_mass<Mx3<64>>(a, part, parts, s);
}

}  // namespace bkv
