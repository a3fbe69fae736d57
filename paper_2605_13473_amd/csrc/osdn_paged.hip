// Attention over a paged cache whose rows are of the type of the queries (bf16, fp32): what a lane loads of a tile, and the products with it.
#include "osdn_decode.h"

namespace osdn {

// The rows of a tile that a lane loads, token 16 i + l % 16 of the tile, on their way: first their pages, then the rows.  In place of a token outside
// [lo, end) the nearest inside, that some other lane asks for too (266 sequences of one token, 16 heads, 10.7 us, with whatever
// stands there 20.3; 370 of 5 tokens, 8 heads, K = 256, 12.3 and 18.8; uneven 512 x 4096 x 4 388 and 393)
template <typename IO, int W> struct RowTile {
    using T = IO;
    using V = IO;                                       // of the values in LDS
    static constexpr int K = W;
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
            const int col = lane & 15, g = lane >> 4;
#pragma unroll
            for (int t = 0; t < K / 16; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[t] = Mfma<float>::mma(to_f32(vs[(4 * g + r) * LDV + 16 * t + col]), p[0][r], o[t]);
        }
    }
};
template <int K> using RowsBf16 = RowTile<bf16, K>;
template <int K> using RowsF32 = RowTile<float, K>;

int launch_paged_decode(const DecodeArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? decode_by_width<RowsBf16>(a, st) : decode_by_width<RowsF32>(a, st); }

}  // namespace osdn
