// Attention of one new token for each of B sequences over a paged cache of keys and values.
//
// For a query q of one head, the cached rows j of its key head that it sees (max(0, length - window) <= j < length):
//   s_j = scale <q, k_j>,  m = max_j s_j,  l = sum_j e^(s_j - m),  o = sum_j e^(s_j - m) v_j / l,  lse = m + log l
//
// Bound by memory: every visible key and value is read once, for all query heads that share it (up to 16 side by side: the columns
// of a 16 x 16 matrix product, so that one query head costs what 16 do, 6 % of the matrix cores' time).  A row is a sequence and a group of up to
// 16 query heads of one key head.  A workgroup takes R adjacent rows of a sequence over the same tokens, each by 4 / R of its
// wavefronts, which take the row's tiles in turn, with a running maximum and sum of their own, and join at its end (R = 4: nothing to join).
// The visible tokens of all groups of R rows make one list that is cut into even shares, one a workgroup, whatever the lengths; a share is
// a part of a group, or the end of one, whole ones and the beginning of the last.  Rows that a share does not hold whole go to a second
// kernel, which joins their parts in their order.
// 2.1 GB of keys and values of 512 sequences of 1 to 4096 tokens: 371 us, 5.8 TB/s (cut into pieces of 1024 tokens, a workgroup each, 22 more); 0.54 GB of
// one sequence 97 us, 5.5 TB/s; reading alone reaches 5.9.  (Calls among others.)  The second kernel takes 3 to 6 us; the fence that a join inside the
// first would take after every part costs more (900 and 180 us).
//
// A wavefront's tile is TT tokens.  Keys go from memory to registers as the matrix product wants them (lane l: token l % 16, 16 bytes);
// scores come out transposed, lane l with four tokens of head l % 16, which is how the second product (values transposed,
// times the weights) takes its weights: its order of tokens is the same on both sides, so no lane has to pass any on.  Values are
// transposed on their way through LDS.
#include "osdn_kernels.h"

#include <cfloat>

namespace osdn {

constexpr int DEC_T = DEC_THREADS, DEC_W = DEC_T / 64;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

__device__ __forceinline__ float max_xor16(float x) {
    float y = x;
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(x), "+v"(y));
    return fmaxf(x, y);
}
__device__ __forceinline__ float max_xor32(float x) {
    float y = x;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(x), "+v"(y));
    return fmaxf(x, y);
}

// Weights of the second product with bf16 values: each as the sum of two bf16 numbers, at most 2^-16 of it off.  The first is the bits of the float
// below it, cut off, so that neither is negative, and the second not zero where the weight is not: a value that is infinite makes the sum that.
// (From the exact value in norm, with two numbers and with one: 33 tokens, K = 128, 1.654e-3, which is the rounding of o alone, and 1.741e-3, 1531
// tokens 1.545e-3 and 1.589e-3.  us: 1531 tokens 10.25 and 10.14, uneven 64 x 8192 x 8 186.5 and 186.5, 512 x 4096 390.3 and 390.8.)
__device__ __forceinline__ void two_parts(const f32x4 &p, bf16x4 &high, bf16x4 &low) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float x = p[r];           // (a bit cast of p[r] itself takes element 0)
        const uint32_t top = __builtin_elementwise_sub_sat(__builtin_bit_cast(uint32_t, x), 1u) & 0xffff0000u;
        high[r] = __builtin_bit_cast(bf16, (uint16_t)(top >> 16));
        low[r] = (bf16)(x - __builtin_bit_cast(float, top));
    }
}

template <typename T, int K> struct DecodeTile {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int TT = decode_tile(K, BF);       // tokens: the depth of the second product's matrix instruction (fp32: four of them)
    static constexpr int SETS = TT / 16;                // 16-token products that make the scores
    static constexpr int VE = 16 / sizeof(T);           // elements of a 16-byte vector
    static constexpr int STEPS = K / (4 * VE);          // vectors of a row, per lane (four lanes share a row)
    static constexpr int LDV = K + VE;                  // row of the values in LDS: 16 rows of one column start on 16 different quads of banks
    static constexpr int OUT = K / 16;                  // 16-row tiles of the transposed result
};

// The rows of a tile that a lane loads, token 16 i + l % 16 of the tile, on their way: first their pages, then the rows.  In place of a token outside
// [lo, end) the nearest inside, that some other lane asks for too (266 sequences of one token, 16 heads, 10.7 us, with whatever
// stands there 20.3; 370 of 5 tokens, 8 heads, K = 256, 12.3 and 18.8; uneven 512 x 4096 x 4 388 and 393)
template <typename T, int K> struct TileLoads {
    using D = DecodeTile<T, K>;
    int page[D::SETS];
    u32x4 k[D::SETS][D::STEPS], v[D::SETS][D::STEPS];
    static __device__ __forceinline__ int token(int tok, int i, int lo, int end, int lane) { return max(min(tok + 16 * i + (lane & 15), end - 1), lo); }
    // pages of the tile at token tok, as far as the table goes (also where there is nothing to see)
    __device__ __forceinline__ void ask(const DecodeArgs &a, const int *row, int tok, int lo, int end, int lane) {
#pragma unroll
        for (int i = 0; i < D::SETS; ++i) page[i] = row[min(token(tok, i, lo, end, lane) >> a.page_shift, a.max_pages - 1)];
    }
    // the rows of a tile that has tokens to see; true: one has no page
    __device__ __forceinline__ bool load(const DecodeArgs &a, const T *kc, const T *vc, int tok, int lo, int end, int lane) {
        bool bad = false;
#pragma unroll
        for (int i = 0; i < D::SETS; ++i) {
            const int slot = token(tok, i, lo, end, lane) & ((1 << a.page_shift) - 1);
            const bool ok = (unsigned)page[i] < (unsigned)a.n_pages;
            bad = bad || !ok;
            const long long g = ok ? page[i] : 0;
            const T *kp = kc + g * a.cache_k.batch + slot * a.cache_k.token, *vp = vc + g * a.cache_v.batch + slot * a.cache_v.token;
#pragma unroll
            for (int s = 0; s < D::STEPS; ++s) k[i][s] = *reinterpret_cast<const u32x4 *>(kp + 4 * D::VE * s);
#pragma unroll
            for (int s = 0; s < D::STEPS; ++s) v[i][s] = *reinterpret_cast<const u32x4 *>(vp + 4 * D::VE * s);
        }
        return bad;
    }
};

// One use of each 64 bytes of the arguments: the scalar loads of all of them are on their way at once, where the compiler would place each ahead
// of its first use, one wait after the other (1531 tokens 9.27 us, so 9.09; fp32, 8 x 1000 tokens 14.1, so 13.4).
__device__ __forceinline__ void ask_arguments(const DecodeArgs &a) {
    asm volatile("" ::"s"(a.B), "s"(a.q.token), "s"(a.cache_k.data), "s"(a.cache_v.token), "s"(a.table_stride), "s"(a.part_ml));
}

__device__ __forceinline__ Seen seen_of(const DecodeArgs &a, int length, int seq) {
    return seen_tokens(length, seq, a.n_seqs, a.max_length, a.window, a.page_shift, a.max_pages);
}
// Units of UNIT tokens of each row of sequence b
template <int UNIT> __device__ __forceinline__ int units_of(const DecodeArgs &a, int b) {
    return seen_units(seen_of(a, a.lengths[b], a.seq ? a.seq[b] : b), UNIT);
}

// SHARED: even shares; else a workgroup takes one group of rows, whole (short ones, or many: no search and no second kernel)
template <typename T, int K, int R, bool SHARED>
__global__ __launch_bounds__(DEC_T, (decode_per_cu(K, sizeof(T) == 2))) void decode_kernel(DecodeArgs a) {
    using D = DecodeTile<T, K>;
    constexpr int TT = D::TT, VE = D::VE, STEPS = D::STEPS, LDV = D::LDV, OUT = D::OUT, LDO = K + 4, WPR = DEC_W / R, STRIDE = WPR * TT;
    constexpr size_t VALUES = TT * LDV * sizeof(T), SUMS = R < 4 ? 16 * LDO * 4 : 0;
    __shared__ __align__(16) char lds[DEC_W * (VALUES > SUMS ? VALUES : SUMS)];
    __shared__ float ml[R < 4 ? DEC_W : 1][2][16];
    __shared__ int found[2], sums[DEC_W];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    ask_arguments(a);
    const int groups = a.Hk * a.head_tiles / R, w = blockIdx.x;     // groups of rows of a sequence
    const int turn = wave % WPR;                                    // this wavefront's among those of its row
    // This workgroup's share: units [at, until), the first of them of sequence b, whose units start at `base`
    int b, base, at, until, total = 0;
    if constexpr (!SHARED) {
        b = w / (unsigned)groups;
        base = 0;
        const int u = units_of<STRIDE>(a, b);
        at = (w - b * groups) * u;
        until = at + u;
    } else {
        if (a.B == 1) {
            total = units_of<STRIDE>(a, 0) * groups;
            b = base = 0;
        } else {                        // where the share begins: a sum over the sequences before it, a run of them a thread
            const int run = (a.B + DEC_T - 1) / DEC_T, i0 = threadIdx.x * run, i1 = min(a.B, i0 + run);
            int mine = 0;
            for (int i = i0; i < i1; ++i) mine += units_of<STRIDE>(a, i);
            int upto = mine;
#pragma unroll
            for (int x = 1; x < 64; x <<= 1) {
                const int y = __shfl_up(upto, x, 64);
                if (lane >= x) upto += y;
            }
            if (lane == 63) sums[wave] = upto;
            __syncthreads();
            int before = upto - mine;
#pragma unroll
            for (int u = 0; u < DEC_W; ++u) {
                if (u < wave) before += sums[u];
                total += sums[u];
            }
            total = __builtin_amdgcn_readfirstlane(total) * groups;
            const int start = Shares(total, a.shares).begin(w);
            if (start >= before * groups && start < (before + mine) * groups) {
                int i = i0, u = units_of<STRIDE>(a, i);
                while (start >= (before + u) * groups) {
                    before += u;
                    u = units_of<STRIDE>(a, ++i);
                }
                found[0] = i;
                found[1] = before * groups;
            }
            __syncthreads();
            b = __builtin_amdgcn_readfirstlane(found[0]);
            base = __builtin_amdgcn_readfirstlane(found[1]);
        }
        const Shares share(total, a.shares);
        at = share.begin(w);
        until = share.begin(w + 1);
        if (at >= until) return;
    }
    const int share_begin = at;

    do {
        const int units = units_of<STRIDE>(a, b), group = (at - base) / units, u0 = at - base - group * units, u1 = min(units, u0 + until - at);
        const int kt = group * R + wave / WPR;                      // this wavefront's row
        const int kv = a.head_tiles == 1 ? kt : kt / a.head_tiles, h0 = kv * a.group + 16 * (kt - kv * a.head_tiles);
        const int heads = min(16, (kv + 1) * a.group - h0);
        const int seq = a.seq ? a.seq[b] : b;
        const Seen see = seen_of(a, a.lengths[b], seq);
        const int *row = a.table + (see.end > 0 ? seq * a.table_stride : 0);
        const int lo = see.lo, begin = seen_begin(see) + u0 * STRIDE, end = u1 == units ? see.end : begin + (u1 - u0) * STRIDE;
        TileLoads<T, K> x;
        x.ask(a, row, begin + turn * TT, lo, end, lane);
        // queries: lane l holds head l % 16
        u32x4 q[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            q[s] = u32x4{0u, 0u, 0u, 0u};
            if (col < heads) {
                const T *src = static_cast<const T *>(a.q.data) + b * a.q.batch + (h0 + col) * a.q.head + (4 * s + g) * VE;
                if (a.aligned) {
                    q[s] = *reinterpret_cast<const u32x4 *>(src);
                } else {
                    T v[VE];
#pragma unroll
                    for (int e = 0; e < VE; ++e) v[e] = src[e];
                    q[s] = __builtin_bit_cast(u32x4, v);
                }
            }
        }
        const T *kc = static_cast<const T *>(a.cache_k.data) + kv * a.cache_k.head + g * VE;
        const T *vc = static_cast<const T *>(a.cache_v.data) + kv * a.cache_v.head + g * VE;
        T *vs = reinterpret_cast<T *>(lds) + wave * TT * LDV;
        const float scale2 = a.scale * LOG2E;

        float m = -FLT_MAX, l = 0.f;        // finite: a score of minus infinity then weighs nothing, also where there is no other
        f32x4 o[OUT];
#pragma unroll
        for (int t = 0; t < OUT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        bool bad_page = false;

        // The rows of the next tile are asked for when this one's are in the matrix products' registers and in LDS, its pages a tile earlier
        int tok = begin + turn * TT;
        if (tok < end) {
            bad_page = x.load(a, kc, vc, tok, lo, end, lane);
            x.ask(a, row, tok + STRIDE, lo, end, lane);
        }
        while (tok < end) {
            // scores, transposed: p[i][r] is token 16 i + 4 g + r of head `col`
            f32x4 p[D::SETS];
            float top = m;
            const bool whole = tok >= lo && tok + TT <= end;
#pragma unroll
            for (int i = 0; i < D::SETS; ++i) {
                if constexpr (D::BF) {
                    p[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) p[i] = Mfma<bf16>::mma(__builtin_bit_cast(bf16x8, x.k[i][s]), __builtin_bit_cast(bf16x8, q[s]), p[i]);
                } else {                // several sums of up to 32 products, then those: K = 256, scores of a spread of 4, o is 4.5e-7 off in norm, after one sum 1.9e-6
                    constexpr int SUMS = K == 256 ? 8 : 4;
                    f32x4 part[SUMS];
#pragma unroll
                    for (int s = 0; s < STEPS; ++s)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            f32x4 &to = part[(4 * s + e) % SUMS];
                            if (4 * s + e < SUMS) to = f32x4{0.f, 0.f, 0.f, 0.f};
                            to = Mfma<float>::mma(vec_get<float>(x.k[i][s], e), vec_get<float>(q[s], e), to);
                        }
#pragma unroll
                    for (int n = SUMS / 2; n > 0; n /= 2)
#pragma unroll
                        for (int u = 0; u < n; ++u)
#pragma unroll
                            for (int r = 0; r < 4; ++r) part[u][r] += part[u + n][r];
                    p[i] = part[0];
                }
            }
            if (!whole) {               // what is not seen has no weight, and must not be infinite or NaN either
#pragma unroll
                for (int i = 0; i < D::SETS; ++i) {
                    const int j = tok + 16 * i + col;
                    const bool seen = j >= lo && j < end;
#pragma unroll
                    for (int s = 0; s < STEPS; ++s)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x.v[i][s][e] = seen ? x.v[i][s][e] : 0u;
                }
            }
#pragma unroll
            for (int i = 0; i < D::SETS; ++i)
#pragma unroll
                for (int s = 0; s < STEPS; ++s) *reinterpret_cast<u32x4 *>(vs + (16 * i + col) * LDV + (4 * s + g) * VE) = x.v[i][s];
            const int next = tok + STRIDE;
            if (next < end) {
                bad_page = x.load(a, kc, vc, next, lo, end, lane) || bad_page;
                x.ask(a, row, next + STRIDE, lo, end, lane);
            }
#pragma unroll
            for (int i = 0; i < D::SETS; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) p[i][r] *= scale2;
            if (!whole) {
#pragma unroll
                for (int i = 0; i < D::SETS; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int j = tok + 16 * i + 4 * g + r;
                        p[i][r] = j >= lo && j < end ? p[i][r] : -INFINITY;
                    }
            }
#pragma unroll
            for (int i = 0; i < D::SETS; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, p[i][r]);
            top = max_xor32(max_xor16(top));
            if (__any(top > m)) {
                const float f = __builtin_amdgcn_exp2f(m - top);
                l *= f;
#pragma unroll
                for (int t = 0; t < OUT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[t][r] *= f;
                m = top;
            }
#pragma unroll
            for (int i = 0; i < D::SETS; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    p[i][r] = __builtin_amdgcn_exp2f(p[i][r] - m);
                    l += p[i][r];
                }
            // o transposed += values transposed x weights
            if constexpr (D::BF) {
                typedef short v4s __attribute__((ext_vector_type(4)));
                typedef __attribute__((address_space(3))) v4s *lds_v4s;
                bf16x4 high[D::SETS], low[D::SETS];
#pragma unroll
                for (int i = 0; i < D::SETS; ++i) two_parts(p[i], high[i], low[i]);
#pragma unroll
                for (int t = 0; t < OUT; ++t) {
                    const bf16 *at = reinterpret_cast<const bf16 *>(vs) + (4 * g + (col >> 2)) * LDV + 16 * t + 4 * (col & 3);
                    const v4s a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(at));
                    if constexpr (D::SETS == 2) {
                        const v4s a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(at + 16 * LDV));
                        const bf16x8 values = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
                        o[t] = Mfma<bf16>::mma(values, __builtin_shufflevector(low[0], low[D::SETS - 1], 0, 1, 2, 3, 4, 5, 6, 7), o[t]);
                        o[t] = Mfma<bf16>::mma(values, __builtin_shufflevector(high[0], high[D::SETS - 1], 0, 1, 2, 3, 4, 5, 6, 7), o[t]);
                    } else {
                        o[t] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a0, __builtin_bit_cast(v4s, low[0]), o[t], 0, 0, 0);
                        o[t] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a0, __builtin_bit_cast(v4s, high[0]), o[t], 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int t = 0; t < OUT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[t] = Mfma<float>::mma(to_f32(vs[(4 * g + r) * LDV + 16 * t + col]), p[0][r], o[t]);
            }
            tok = next;
        }
        l = add_xor32(add_xor16(l));
        if (see.broken || __any(bad_page)) l = __builtin_nanf("");
        const bool alone = !SHARED || u1 - u0 == units;                     // (nothing to join)
        const int slot = part_slot(w, at == share_begin);
        if (SHARED && u0 == 0 && threadIdx.x == 0) {
            const int last = alone ? w : Shares(total, a.shares).owner(at + units - 1);
            a.info[((size_t)b * groups + group) * 2] = slot;
            a.info[((size_t)b * groups + group) * 2 + 1] = last - w + 1;
        }
        // four elements of head h of this wavefront's row from d on, whose maximum and sum are M and L
        auto leave = [&](int h, int d, f32x4 x, float M, float L) {
            if (alone) {
                const float inv = L == 0.f ? 0.f : 1.f / L;
                T *dst = static_cast<T *>(a.o.data) + b * a.o.batch + (h0 + h) * a.o.head + d;
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] *= inv;
                if (a.aligned) {
                    store4(dst, x);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) dst[r] = from_f32<T>(x[r]);
                }
                if (a.lse && d == 0) a.lse[(size_t)b * a.Hq + h0 + h] = L == 0.f ? -INFINITY : __builtin_fmaf(M, LN2, logf(L));
            } else {
                const size_t to = ((size_t)slot * R + wave / WPR) * a.part_heads + h;
                store4(a.part_o + to * K + d, x);
                if (d == 0) {
                    a.part_ml[to * 2] = M;
                    a.part_ml[to * 2 + 1] = L;
                }
            }
        };
        if constexpr (R == 4) {
            if (col < heads) {
#pragma unroll
                for (int t = 0; t < OUT; ++t) leave(col, 16 * t + 4 * g, o[t], m, l);
            }
        } else {                            // the wavefronts of a row join
            const int first = wave - turn;
            if (g == 0) { ml[wave][0][col] = m; ml[wave][1][col] = l; }
            __syncthreads();
            float M = ml[first][0][col];
#pragma unroll
            for (int u = 1; u < WPR; ++u) M = fmaxf(M, ml[first + u][0][col]);
            const float f = __builtin_amdgcn_exp2f(m - M);
            float *os = reinterpret_cast<float *>(lds) + wave * 16 * LDO;
#pragma unroll
            for (int t = 0; t < OUT; ++t) {
                f32x4 x = o[t];
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] *= f;
                *reinterpret_cast<f32x4 *>(os + col * LDO + 16 * t + 4 * g) = x;
            }
            __syncthreads();
            for (int i = turn * 64 + lane; i < heads * (K / 4); i += WPR * 64) {
                const int h = i / (K / 4), d = i % (K / 4) * 4;
                float top = ml[first][0][h], sum = 0.f;
#pragma unroll
                for (int u = 1; u < WPR; ++u) top = fmaxf(top, ml[first + u][0][h]);
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int u = 0; u < WPR; ++u) {
                    sum = __builtin_fmaf(ml[first + u][1][h], __builtin_amdgcn_exp2f(ml[first + u][0][h] - top), sum);
                    const f32x4 y = load4(reinterpret_cast<const float *>(lds) + ((first + u) * 16 + h) * LDO + d);
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] += y[r];
                }
                leave(h, d, x, top, sum);
            }
        }
        at += u1 - u0;
        if (at == base + groups * units) {
            base = at;
            ++b;
        }
        if (SHARED && R < 4 && at < until) __syncthreads();        // (the next row's values take the place of these sums)
    } while (SHARED && at < until);
}

// The parts of the query heads, joined in their order.  A wavefront (WG: a workgroup, its four wavefronts a quarter of the parts each) joins JC columns
// of one head: a lane four columns of every (64 / (JC / 4))-th part.
template <typename T, int K, int JC, bool WG>
__global__ __launch_bounds__(256) void decode_join_kernel(DecodeArgs a) {
    constexpr int QUADS = JC / 4, ROWS = 64 / QUADS, WAVES = WG ? 4 : 1;
    __shared__ float red[4][JC], sums[4];
    ask_arguments(a);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned item = WG ? blockIdx.x : blockIdx.x * 4 + wave;
    const unsigned bh = item / (K / JC);
    const int c0 = item % (K / JC) * JC + lane % QUADS * 4;
    if (!WG && bh >= (unsigned)a.B * a.Hq) return;
    const int b = bh / (unsigned)a.Hq, h = bh % (unsigned)a.Hq;
    // its row, the slot of the first part and how many there are: the parts after the first are each the first of their share
    const int kv = h / (unsigned)a.group, in = h - kv * a.group, hh = in & 15;
    const int kt = kv * a.head_tiles + (in >> 4), group = kt / (unsigned)a.row_group, r = kt - group * a.row_group;
    const int *info = a.info + ((size_t)b * (a.Hk * a.head_tiles / (unsigned)a.row_group) + group) * 2;
    const int first_slot = info[0], n = info[1];
    if (n <= 1) return;                 // decode_kernel has written it
    auto place = [&](int i) { return ((size_t)part_of_row(first_slot, i) * a.row_group + r) * a.part_heads + hh; };
    const float *ml = a.part_ml, *po = a.part_o + c0;
    // the first four of a lane's parts are on their way before the maximum is known
    constexpr int STEP = ROWS * WAVES, AHEAD = 4;
    const int first = (WG ? wave * ROWS : 0) + lane / QUADS;
    f32x4 ahead[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) ahead[u] = load4(po + place(min(first + u * STEP, n - 1)) * K);
    float M = -FLT_MAX;
    for (int i = lane; i < n; i += 64) M = fmaxf(M, ml[2 * place(i)]);
    M = max_xor32(max_xor16(M));
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) M = fmaxf(M, __shfl_xor(M, x, 64));
    float L = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](int i, const f32x4 &y) {
        const float f = __builtin_amdgcn_exp2f(ml[2 * place(i)] - M);
        L = __builtin_fmaf(ml[2 * place(i) + 1], f, L);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(y[e], f, x[e]);
    };
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        if (first + u * STEP < n) add(first + u * STEP, ahead[u]);
#pragma unroll 4
    for (int i = first + AHEAD * STEP; i < n; i += STEP) add(i, load4(po + place(i) * K));
#pragma unroll
    for (int s = QUADS; s < 64; s <<= 1) {
        L += __shfl_xor(L, s, 64);
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] += __shfl_xor(x[r], s, 64);
    }
    if constexpr (WG) {
        if (lane < QUADS) *reinterpret_cast<f32x4 *>(&red[wave][4 * lane]) = x;
        if (lane == 0) sums[wave] = L;
        __syncthreads();
        if (wave != 0) return;
        L = sums[0] + sums[1] + sums[2] + sums[3];
        x = load4(&red[0][lane % QUADS * 4]);
#pragma unroll
        for (int u = 1; u < 4; ++u) {
            const f32x4 y = load4(&red[u][lane % QUADS * 4]);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] += y[r];
        }
    }
    if (lane >= QUADS) return;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    T *dst = static_cast<T *>(a.o.data) + b * a.o.batch + h * a.o.head + c0;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] *= inv;
    if (a.aligned) {
        store4(dst, x);
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) dst[r] = from_f32<T>(x[r]);
    }
    if (a.lse && c0 == 0) a.lse[bh] = L == 0.f ? -INFINITY : __builtin_fmaf(M, LN2, logf(L));
}

namespace {
template <typename T, int K, bool SHARED> void decode_rows(const DecodeArgs &a, unsigned workgroups, hipStream_t st) {
    if (a.row_group == 4) hipLaunchKernelGGL((decode_kernel<T, K, 4, SHARED>), dim3(workgroups), dim3(DEC_T), 0, st, a);
    else if (a.row_group == 2) hipLaunchKernelGGL((decode_kernel<T, K, 2, SHARED>), dim3(workgroups), dim3(DEC_T), 0, st, a);
    else hipLaunchKernelGGL((decode_kernel<T, K, 1, SHARED>), dim3(workgroups), dim3(DEC_T), 0, st, a);
}
template <typename T, int K> void decode_of(const DecodeArgs &a, hipStream_t st) {
    const unsigned groups = (unsigned)a.B * a.Hk * a.head_tiles / a.row_group, heads = (unsigned)a.B * a.Hq, shares = (unsigned)a.shares;
    if (!shares) return decode_rows<T, K, false>(a, groups, st);
    decode_rows<T, K, true>(a, shares, st);
    // (many parts of few rows: a workgroup each, as the loads of a row are then what takes the time)
    if (shares > 16 * groups) hipLaunchKernelGGL((decode_join_kernel<T, K, 16, true>), dim3(heads * (K / 16)), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((decode_join_kernel<T, K, 64, false>), dim3((heads * (K / 64) + 3) / 4), dim3(256), 0, st, a);
}
}  // namespace

int launch_paged_decode(const DecodeArgs &a, bool bf16_io, hipStream_t st) {
    switch (a.K) {
        case 64: bf16_io ? decode_of<bf16, 64>(a, st) : decode_of<float, 64>(a, st); return 0;
        case 128: bf16_io ? decode_of<bf16, 128>(a, st) : decode_of<float, 128>(a, st); return 0;
        case 256: bf16_io ? decode_of<bf16, 256>(a, st) : decode_of<float, 256>(a, st); return 0;
        default: return -1;
    }
}

}  // namespace osdn
