// Attention over a paged cache in 4 bits: what a lane loads of a tile, and the products with it.
//
// A row of K elements is K / 2 bytes of codes and K / 32 scales.  Its four lanes take K / 4 adjacent elements each, whole words of eight codes, which one
// instruction a pair turns into the bf16 numbers that they stand for, exactly; the order of a row's elements is the same on both sides of
// the first product, so nothing is passed between lanes.  Values go through LDS as bf16.  fp32 queries and weights are sums of three bf16 numbers, which hold all their digits.
#include "osdn_decode.h"

namespace osdn {

template <typename IO, int W> struct Fp4Tile {
    using T = IO;
    using V = bf16;                                     // of the values in LDS
    static constexpr int K = W;
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int PER_CU = decode_mx_per_cu(K, BF);
    static constexpr int TT = DECODE_MX_TILE;
    static constexpr int SETS = TT / 16;
    static constexpr int EL = K / 4, WORDS = EL / 8;    // elements of a lane, words of codes
    static constexpr int SCALES = (EL + 31) / 32;
    static constexpr int PARTS = BF ? 1 : 3;            // bf16 numbers that make a query's element
    static constexpr int LDV = K + 8;

    struct Query {
        bf16x8 q[WORDS][PARTS];                         // (the smallest part first)
        __device__ __forceinline__ void load(const T *row, bool live, bool aligned, int lane) {
            const T *src = row + (lane >> 4) * EL;
#pragma unroll
            for (int s = 0; s < WORDS; ++s) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = 0.f;
                if (live) {
                    if (aligned) {
                        constexpr int N = 16 / sizeof(T);
#pragma unroll
                        for (int v = 0; v < 8 / N; ++v) {
                            const u32x4 raw = *reinterpret_cast<const u32x4 *>(src + 8 * s + N * v);
#pragma unroll
                            for (int e = 0; e < N; ++e) x[N * v + e] = vec_get<T>(raw, e);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = to_f32(src[8 * s + e]);
                    }
                }
#pragma unroll
                for (int u = PARTS - 1; u >= 0; --u)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t top = __builtin_bit_cast(uint32_t, x[e]) & 0xffff0000u;          // (cut off: the largest float stays finite)
                        q[s][u][e] = __builtin_bit_cast(bf16, (uint16_t)(top >> 16));
                        x[e] -= __builtin_bit_cast(float, top);
                    }
            }
        }
    };

    struct Codes { uint32_t word[WORDS]; uint32_t scale; };         // scale: a byte for each 32 elements
    const char *kc, *vc;
    const unsigned char *ks, *vs;
    int page[SETS];
    Codes k[SETS], v[SETS];
    static __device__ __forceinline__ int token(int tok, int i, int lo, int end, int lane) { return max(min(tok + 16 * i + (lane & 15), end - 1), lo); }
    __device__ __forceinline__ void begin(const DecodeArgs &a, int head, int lane) {
        const int g = lane >> 4;
        kc = static_cast<const char *>(a.cache_k.data) + head * a.cache_k.head + g * (EL / 2);
        vc = static_cast<const char *>(a.cache_v.data) + head * a.cache_v.head + g * (EL / 2);
        ks = static_cast<const unsigned char *>(a.scale_k.data) + head * a.scale_k.head + g * EL / 32;
        vs = static_cast<const unsigned char *>(a.scale_v.data) + head * a.scale_v.head + g * EL / 32;
    }
    __device__ __forceinline__ void ask(const DecodeArgs &a, const int *row, int tok, int lo, int end, int lane) {
#pragma unroll
        for (int i = 0; i < SETS; ++i) page[i] = row[min(token(tok, i, lo, end, lane) >> a.page_shift, a.max_pages - 1)];
    }
    static __device__ __forceinline__ Codes fetch(const char *codes, const unsigned char *scale) {
        Codes c;
        if constexpr (WORDS == 2) {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(codes);
            c.word[0] = x[0];
            c.word[1] = x[1];
        } else {
#pragma unroll
            for (int w = 0; w < WORDS; w += 4) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(codes + 4 * w);
#pragma unroll
                for (int e = 0; e < 4; ++e) c.word[w + e] = x[e];
            }
        }
        c.scale = SCALES == 1 ? *scale : *reinterpret_cast<const uint16_t *>(scale);
        return c;
    }
    __device__ __forceinline__ bool load(const DecodeArgs &a, int tok, int lo, int end, int lane) {
        bool bad = false;
#pragma unroll
        for (int i = 0; i < SETS; ++i) {
            const int slot = token(tok, i, lo, end, lane) & ((1 << a.page_shift) - 1);
            const bool ok = (unsigned)page[i] < (unsigned)a.n_pages;
            bad = bad || !ok;
            const long long g = ok ? page[i] : 0;
            k[i] = fetch(kc + g * a.cache_k.batch + slot * a.cache_k.token, ks + g * a.scale_k.batch + slot * a.scale_k.token);
            v[i] = fetch(vc + g * a.cache_v.batch + slot * a.cache_v.token, vs + g * a.scale_v.batch + slot * a.scale_v.token);
        }
        return bad;
    }
    static __device__ __forceinline__ bf16x8 values(const Codes &c, int w) { return fp4_values(c.word[w], fp4_scale(SCALES == 1 ? c.scale : w < 4 ? c.scale & 255u : c.scale >> 8)); }
    __device__ __forceinline__ f32x4 scores(int i, const Query &x) const {
        f32x4 p = {0.f, 0.f, 0.f, 0.f}, small = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            const bf16x8 kw = values(k[i], w);
#pragma unroll
            for (int u = 0; u + 1 < PARTS; ++u) small = Mfma<bf16>::mma(kw, x.q[w][u], small);
            p = Mfma<bf16>::mma(kw, x.q[w][PARTS - 1], p);
        }
        if constexpr (PARTS > 1) {
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] += small[r];
        }
        return p;
    }
    __device__ __forceinline__ void hide(int i, bool seen) {
#pragma unroll
        for (int w = 0; w < WORDS; ++w) v[i].word[w] = seen ? v[i].word[w] : 0u;
        v[i].scale = seen ? v[i].scale : 0x7f7fu;
    }
    __device__ __forceinline__ void put_values(int i, bf16 *row, int lane) const {
#pragma unroll
        for (int w = 0; w < WORDS; ++w) *reinterpret_cast<bf16x8 *>(row + (lane >> 4) * EL + 8 * w) = values(v[i], w);
    }
    static __device__ __forceinline__ void add_values(const bf16 *vs, const f32x4 (&p)[SETS], f32x4 (&o)[K / 16], int lane) {
        add_bf16_values<K, SETS, LDV, BF ? 2 : 3>(vs, p, o, lane);
    }
};
template <int K> using Fp4Bf16 = Fp4Tile<bf16, K>;
template <int K> using Fp4F32 = Fp4Tile<float, K>;

int launch_paged_decode_mx(const DecodeArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? decode_by_width<Fp4Bf16>(a, st) : decode_by_width<Fp4F32>(a, st); }

}  // namespace osdn
