// What a lane loads of a tile of the cache's rows, and the products with it: the rows' formats of the kernel of attention (osdn_decode.h).
#pragma once
#include "osdn_decode.h"

namespace osdn {

// ---- rows of the type of the queries (bf16, fp32) ----
// The rows of a tile that a lane loads, token 16 i + l % 16 of the tile, on their way: first their pages, then the rows.  In place of a token outside
// [lo, end) the nearest inside, that some other lane asks for too (266 sequences of one token, 16 heads, 10.7 us, with whatever
// stands there 20.3; 370 of 5 tokens, 8 heads, K = 256, 12.3 and 18.8; uneven 512 x 4096 x 4 388 and 393)
template <typename IO, int W, bool C = false> struct RowTile {
    using T = IO;
    using V = IO;                                       // of the values in LDS
    static constexpr int K = W;
    static constexpr bool CHOSEN = C, BY_SEQUENCE = false;      // CHOSEN: a table for each key head; BY_SEQUENCE: see by_sequence
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int PER_CU = decode_per_cu(K, BF);
    static constexpr int TT = decode_tile(K, BF);       // tokens: the depth of the second product's matrix instruction (fp32: four of them)
    static constexpr int SETS = TT / 16;                // 16-token products that make the scores
    static constexpr int VE = 16 / sizeof(T);           // elements of a 16-byte vector
    static constexpr int STEPS = K / (4 * VE);          // vectors of a row, per lane (four lanes share a row)
    static constexpr int LDV = K + VE;                  // row of the values in LDS: 16 rows of one column start on 16 different quads of banks

    // the queries as the matrix product wants them
    struct Query {
        u32x4 q[STEPS];
        __device__ __forceinline__ void load(const T *row, bool live, bool aligned, int lane) {
            const int g = lane >> 4;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                q[s] = u32x4{0u, 0u, 0u, 0u};
                if (live) {
                    const T *src = row + (4 * s + g) * VE;
                    if (aligned) {
                        q[s] = *reinterpret_cast<const u32x4 *>(src);
                    } else {
                        T v[VE];
#pragma unroll
                        for (int e = 0; e < VE; ++e) v[e] = src[e];
                        q[s] = __builtin_bit_cast(u32x4, v);
                    }
                }
            }
        }
    };

    static __device__ __forceinline__ void ask_arguments(const DecodeArgs &) {}
    const T *kc, *vc;
    int page[SETS];
    u32x4 k[SETS][STEPS], v[SETS][STEPS];
    static __device__ __forceinline__ int token(int tok, int i, int lo, int end, int lane) { return max(min(tok + 16 * i + (lane & 15), end - 1), lo); }
    __device__ __forceinline__ void begin(const DecodeArgs &a, int head, int lane) {
        kc = static_cast<const T *>(a.cache_k.data) + head * a.cache_k.head + (lane >> 4) * VE;
        vc = static_cast<const T *>(a.cache_v.data) + head * a.cache_v.head + (lane >> 4) * VE;
    }
    // pages of the tile at token tok, as far as the table goes (also where there is nothing to see)
    __device__ __forceinline__ void ask(const DecodeArgs &a, const int *row, int tok, int lo, int end, int lane) {
#pragma unroll
        for (int i = 0; i < SETS; ++i) page[i] = row[min(token(tok, i, lo, end, lane) >> a.page_shift, a.max_pages - 1)];
    }
    // the rows of a tile that has tokens to see; true: one has no page
    __device__ __forceinline__ bool load(const DecodeArgs &a, int tok, int lo, int end, int lane) {
        bool bad = false;
#pragma unroll
        for (int i = 0; i < SETS; ++i) {
            const int slot = token(tok, i, lo, end, lane) & ((1 << a.page_shift) - 1);
            const bool ok = (unsigned)page[i] < (unsigned)a.n_pages;
            bad = bad || !ok;
            const long long g = ok ? page[i] : 0;
            const T *kp = kc + g * a.cache_k.batch + slot * a.cache_k.token, *vp = vc + g * a.cache_v.batch + slot * a.cache_v.token;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) k[i][s] = *reinterpret_cast<const u32x4 *>(kp + 4 * VE * s);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) v[i][s] = *reinterpret_cast<const u32x4 *>(vp + 4 * VE * s);
        }
        return bad;
    }
    // the scores of 16 tokens, transposed: [r] is token 16 i + 4 g + r of head l % 16
    __device__ __forceinline__ f32x4 scores(int i, const Query &x) const {
        f32x4 p;
        if constexpr (BF) {
            p = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < STEPS; ++s) p = Mfma<bf16>::mma(__builtin_bit_cast(bf16x8, k[i][s]), __builtin_bit_cast(bf16x8, x.q[s]), p);
        } else {                // several sums of up to 32 products, then those: K = 256, scores of a spread of 4, o is 4.5e-7 off in norm, after one sum 1.9e-6
            constexpr int SUMS = K == 256 ? 8 : 4;
            f32x4 part[SUMS];
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f32x4 &to = part[(4 * s + e) % SUMS];
                    if (4 * s + e < SUMS) to = f32x4{0.f, 0.f, 0.f, 0.f};
                    to = Mfma<float>::mma(vec_get<float>(k[i][s], e), vec_get<float>(x.q[s], e), to);
                }
#pragma unroll
            for (int n = SUMS / 2; n > 0; n /= 2)
#pragma unroll
                for (int u = 0; u < n; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) part[u][r] += part[u + n][r];
            p = part[0];
        }
        return p;
    }
    // the values of a lane's token in the set i: zeros where it is not seen, and into its row in LDS
    __device__ __forceinline__ void hide(int i, bool seen) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][s][e] = seen ? v[i][s][e] : 0u;
    }
    __device__ __forceinline__ void put_values(int i, T *row, int lane) const {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) *reinterpret_cast<u32x4 *>(row + (4 * s + (lane >> 4)) * VE) = v[i][s];
    }
    static __device__ __forceinline__ void add_values(const T *vs, const f32x4 (&p)[SETS], f32x4 (&o)[K / 16], int lane) {
        if constexpr (BF) {
            add_bf16_values<K, SETS, LDV, 2>(vs, p, o, lane);
        } else {
            // (one address for all of them: K = 128, a row each, 162 or 164 registers, so three workgroups a CU; with one made of the lane for each 170 and two, 2000 x 200 x 4 179 us, so 153)
            const T *at = vs + 4 * (lane >> 4) * LDV + (lane & 15);
#pragma unroll
            for (int t = 0; t < K / 16; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[t] = Mfma<float>::mma(to_f32(at[r * LDV + 16 * t]), p[0][r], o[t]);
        }
    }
};

// ---- rows in 4 bits ----
// A row of K elements is K / 2 bytes of codes and K / 32 scales.  Its four lanes take K / 4 adjacent elements each, whole words of eight codes, which one
// instruction a pair turns into the bf16 numbers that they stand for, exactly; the order of a row's elements is the same on both sides of
// the first product, so nothing is passed between lanes.  Values go through LDS as bf16.  Bound by memory where there is enough: 573 MB of 512 sequences of 1 to 4096 tokens, four heads of 128,
// 114 us, 5.0 TB/s (in bf16 2.1 GB, 371); 142 MB of one sequence 32, its second kernel 4 of them; one of 1531 tokens 9.5, two launches.  fp32 queries and weights are sums of three bf16 numbers, which hold all their digits.
// REGULAR (fp4_regular): a row's place in all four arrays comes of one offset.  ONCE (decode_mx_once): the codes are loaded past the caches.
template <typename IO, int W, bool REGULAR, bool C = false, bool ONCE = false> struct Fp4Tile {
    using T = IO;
    using V = bf16;                                     // of the values in LDS
    static constexpr int K = W;
    static constexpr bool CHOSEN = C, BY_SEQUENCE = true;
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

    static __device__ __forceinline__ void ask_arguments(const DecodeArgs &a) { asm volatile("" ::"s"(a.scale_k.data), "s"(a.scale_v.head)); }
    struct Codes { uint32_t word[WORDS]; uint32_t scale; };         // scale: a byte for each 32 elements
    const char *kc, *vc;
    const unsigned char *ks, *vs;
    int page[SETS];
    Codes k[SETS], v[SETS];
    static __device__ __forceinline__ int token(int tok, int i, int lo, int end, int lane) { return max(min(tok + 16 * i + (lane & 15), end - 1), lo); }
    __device__ __forceinline__ void begin(const DecodeArgs &a, int head, int lane) {
        kc = static_cast<const char *>(a.cache_k.data) + head * a.cache_k.head;
        vc = static_cast<const char *>(a.cache_v.data) + head * a.cache_v.head;
        ks = static_cast<const unsigned char *>(a.scale_k.data) + head * a.scale_k.head;
        vs = static_cast<const unsigned char *>(a.scale_v.data) + head * a.scale_v.head;
    }
    __device__ __forceinline__ void ask(const DecodeArgs &a, const int *row, int tok, int lo, int end, int lane) {
#pragma unroll
        for (int i = 0; i < SETS; ++i) page[i] = row[min(token(tok, i, lo, end, lane) >> a.page_shift, a.max_pages - 1)];
    }
    static __device__ __forceinline__ Codes fetch(const char *codes, const unsigned char *scale) {
        Codes c;
        if constexpr (WORDS == 2) {
            const u32x2 *at = reinterpret_cast<const u32x2 *>(codes), x = ONCE ? __builtin_nontemporal_load(at) : *at;
            c.word[0] = x[0];
            c.word[1] = x[1];
        } else {
#pragma unroll
            for (int w = 0; w < WORDS; w += 4) {
                const u32x4 *at = reinterpret_cast<const u32x4 *>(codes + 4 * w), x = ONCE ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
                for (int e = 0; e < 4; ++e) c.word[w + e] = x[e];
            }
        }
        c.scale = SCALES == 1 ? *scale : *reinterpret_cast<const uint16_t *>(scale);
        return c;
    }
    __device__ __forceinline__ bool load(const DecodeArgs &a, int tok, int lo, int end, int lane) {
        bool bad = false;
        const unsigned g = lane >> 4;
#pragma unroll
        for (int i = 0; i < SETS; ++i) {
            const int slot = token(tok, i, lo, end, lane) & ((1 << a.page_shift) - 1);
            const bool ok = (unsigned)page[i] < (unsigned)a.n_pages;
            bad = bad || !ok;
            if constexpr (REGULAR) {
                const uint32_t in = __umul24(slot, (uint32_t)a.cache_k.token) + g * (EL / 2);
                const uint64_t off = (uint64_t)(ok ? (uint32_t)page[i] : 0u) * (uint32_t)a.cache_k.batch + in;
                k[i] = fetch(kc + off, ks + (off >> 4));
                v[i] = fetch(vc + off, vs + (off >> 4));
            } else {
                const long long p = ok ? page[i] : 0;
                k[i] = fetch(kc + p * a.cache_k.batch + slot * a.cache_k.token + g * (EL / 2), ks + p * a.scale_k.batch + slot * a.scale_k.token + g * EL / 32);
                v[i] = fetch(vc + p * a.cache_v.batch + slot * a.cache_v.token + g * (EL / 2), vs + p * a.scale_v.batch + slot * a.scale_v.token + g * EL / 32);
            }
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

}  // namespace osdn
