// Norms of queries and keys for each head with the position rotation in the same pass, forward and backward, and the append of
// keys and values to a paged cache, which does the same to its rows on their way.
//
// A row x of K elements (one head of one token) becomes  z = R(p) (w . x r),  r = (m sum x^2 + eps)^(-1/2):
//   m = 1 (unit length), 1/K (unit mean square), or r = 1; w [K] or ones; R(p) turns the pairs (i, i + R/2) or (2i, 2i + 1) of the
//   first R elements by the angles of the token's position p, whose cosines and sines are row p of a table.
// Backward, with dy = R(-p) dz and g = w . dy:  dx = r (g - x r^2 m <g, x>),  dw = sum over rows of dy . x r.
//
// Bound by memory: a row is read once and written once (backward: two and one), everything between is in fp32 registers,
// and nothing is kept from the forward pass for the backward pass (r is formed again from the x that it reads anyway).
// A wavefront works on one token, so that the angles of its position are loaded once for its rows; 16 bytes per lane, K elements
// in K * sizeof(T) / 16 lanes, 64 lanes in as many rows as that makes (a block of rows).  bf16, K = 128: 4 x 4096 tokens of 16 + 16 rows, unit length,
// forward 44 us (6.1 TB/s, a part still in the last level cache), backward 78 us (5.2 TB/s: what a device copy reaches); 2 x 8192 of 32 + 8 with weights
// and rotation 61 and 110 us (4.6 of them the sum of dw); 65536 tokens of 16 + 4 + 4 appended 159 us (5.1 TB/s).  (Kernel times of a trace, medians,
// three sets of inputs in turn.)
#include "osdn_kernels.h"

namespace osdn {

constexpr int HEADS_T = 256;

template <typename T, int K> struct HeadRow {
    static constexpr int VE = 16 / sizeof(T);       // elements of a lane
    static constexpr int LANES = K / VE;            // lanes of a row
    static constexpr int ROWS = 64 / LANES;         // rows of a block
};

// 16 bytes of a row; VEC: at an address that is a multiple of 16, else element by element
template <typename T, bool VEC> __device__ __forceinline__ u32x4 load_row(const T *p) {
    if constexpr (VEC) {
        return *reinterpret_cast<const u32x4 *>(p);
    } else {
        T v[16 / sizeof(T)];
#pragma unroll
        for (int e = 0; e < (int)(16 / sizeof(T)); ++e) v[e] = p[e];
        return __builtin_bit_cast(u32x4, v);
    }
}
template <typename T, bool VEC, int VE> __device__ __forceinline__ void store_row(T *p, const float (&v)[VE]) {
    if constexpr (VEC) {
        store_vec_t(p, v);
    } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) p[e] = from_f32<T>(v[e]);
    }
}
template <typename T, int VE> __device__ __forceinline__ void unpack(const u32x4 &raw, float (&x)[VE]) {
#pragma unroll
    for (int e = 0; e < VE; ++e) x[e] = vec_get<T>(raw, e);
}
// sum over the LANES lanes of a row, every lane with the result
template <int LANES> __device__ __forceinline__ float row_sum(float x) {
    x += dpp_f32<0xB1>(x);         // quad_perm [1,0,3,2]
    x += dpp_f32<0x4E>(x);         // quad_perm [2,3,0,1]
    x += dpp_f32<0x141>(x);        // row_half_mirror
    if (LANES > 8) x += dpp_f32<0x140>(x);      // row_mirror
    if (LANES > 16) x = add_xor16(x);
    if (LANES > 32) x = add_xor32(x);
    return x;
}

// The caller's fp32 arrays are aligned as floats are
struct __attribute__((packed, aligned(4))) FloatQuad { float v[4]; };
template <int N> __device__ __forceinline__ void load_floats(float (&x)[N], const float *p) {
    static_assert(N % 2 == 0, "");
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const FloatQuad q = reinterpret_cast<const FloatQuad *>(p)[i];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * i + e] = q.v[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = p[e];
    }
}

// The pairs that turn: none, (i, i + R / 2) or (2i, 2i + 1)
enum { ROT_NONE = 0, ROT_HALF = 1, ROT_PAIRS = 2 };

// The rotation of a lane's elements: z = y c + partner s (transposed: y c - partner s).  Elements that do not turn: c = 1, partner = 0.
template <typename T, int K, int ROT> struct Turn {
    static constexpr int VE = HeadRow<T, K>::VE, LANES = HeadRow<T, K>::LANES;
    bool on;                        // the lane's elements turn
    int from;                       // the lane that holds their partners
    int i0;                         // the first one's pair
    float sign;
    __device__ __forceinline__ Turn(int R, int lane) {
        const int e0 = (lane & (LANES - 1)) * VE, half = R / 2;
        const bool low = e0 < half;
        on = e0 < R;
        from = ROT == ROT_PAIRS || !on ? lane : low ? lane + half / VE : lane - half / VE;
        i0 = !on ? 0 : ROT == ROT_PAIRS ? e0 / 2 : low ? e0 : e0 - half;
        sign = low ? -1.f : 1.f;
    }
    __device__ __forceinline__ void load(const float *row, int R, float (&c)[VE], float (&s)[VE]) const {
        constexpr int N = ROT == ROT_PAIRS ? VE / 2 : VE;
        float cs[N], sn[N];
        load_floats(cs, row + i0);
        load_floats(sn, row + R / 2 + i0);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            c[e] = on ? cs[ROT == ROT_PAIRS ? e / 2 : e] : 1.f;
            s[e] = ROT == ROT_PAIRS ? ((e & 1) ? sn[e / 2] : -sn[e / 2]) : sn[e] * sign;
        }
    }
    // the partners of a lane's elements (every lane of the wavefront calls it)
    __device__ __forceinline__ void partners(const u32x4 &raw, float (&x)[VE]) const {
        u32x4 o;
        if constexpr (ROT == ROT_PAIRS) {
#pragma unroll
            for (int w = 0; w < 4; ++w) o[w] = sizeof(T) == 2 ? (raw[w] >> 16) | (raw[w] << 16) : raw[w ^ 1];
        } else {
#pragma unroll
            for (int w = 0; w < 4; ++w) o[w] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * from, (int)raw[w]);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) o[w] = on ? o[w] : 0u;
        unpack<T>(o, x);
    }
    // what stands at the partners' places of a row that all lanes of a row hold (weights)
    __device__ __forceinline__ int partner_element(int lane, int e) const { return ROT == ROT_PAIRS ? (lane & (LANES - 1)) * VE + (e ^ 1) : (from & (LANES - 1)) * VE + e; }
};

// The weights of a lane's elements and of their partners, for queries (0) and keys (1); loaded once per wavefront
template <typename T, int K, int ROT> struct Weights {
    static constexpr int VE = HeadRow<T, K>::VE;
    float own[2][VE], partner[2][VE];
    __device__ __forceinline__ void load(const HeadsArgs &a, const Turn<T, K, ROT> &turn, int lane) {
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {
            const float *w = kind == 0 ? a.weight_q : a.weight_k;
            if (w) load_floats(own[kind], w + (lane & (HeadRow<T, K>::LANES - 1)) * VE);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                if (!w) own[kind][e] = 1.f;
                if constexpr (ROT == ROT_PAIRS) partner[kind][e ^ 1] = own[kind][e];
            }
            if constexpr (ROT == ROT_HALF) {
                if (w) load_floats(partner[kind], w + turn.partner_element(lane, 0));
                else {
#pragma unroll
                    for (int e = 0; e < VE; ++e) partner[kind][e] = 1.f;
                }
            }
        }
    }
};

template <typename T, bool VEC> __device__ __forceinline__ T *row_at(const HeadRows &r, int b, int t, int h) {
    return static_cast<T *>(r.data) + b * r.batch + t * r.token + h * r.head;
}

// ---- rows in 4 bits ----
// A block of 32 elements, VE of them a lane, becomes codes and a scale 2^e, e the least (from -120 to 125) with the largest element no more than 7 * 2^e: what lies
// between 6 and 7 is off by no more than what lies between 4 and 6 may be.  The codes are the nearest values, ties to the even code.
// Which code that is must not hang on a rounding before: values come as they are, keys in 64 bits.  There the lower word only says whether there is more
// than the upper one shows (its last bit, set if so), as no border of two codes has that many digits.
__device__ __forceinline__ int max_block(int x, int lanes) {
    auto with = [&](int y) { x = max(x, y); };
    with(__builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, true));         // quad_perm [1,0,3,2]
    with(__builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, true));         // quad_perm [2,3,0,1]
    if (lanes > 4) with(__builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true));     // row_half_mirror
    return x;
}
template <int VE> struct Fp4Block {
    uint32_t codes;
    int byte;
    __device__ __forceinline__ void scale_of(int exponent, bool beyond, bool finite) { byte = finite ? max(-120, min(125, exponent - 2 + beyond)) + 127 : 255; }
    __device__ __forceinline__ void encode(const float (&y)[VE]) {
        codes = 0;
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[0], y[1], 1.f, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[2], y[3], 1.f, 1);
        if constexpr (VE == 8) {
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[4], y[5], 1.f, 2);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[6], y[7], 1.f, 3);
        }
        if (byte == 255) codes = 0;
    }
    __device__ __forceinline__ explicit Fp4Block(const float (&x)[VE]) {
        int top = 0;
#pragma unroll
        for (int e = 0; e < VE; ++e) top = max(top, __builtin_bit_cast(int, x[e]) & 0x7fffffff);
        top = max_block(top, 32 / VE);
        scale_of((top >> 23) - 127, (top & 0x7fffff) > 0x600000, top < 0x7f800000);
        float y[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) y[e] = __builtin_ldexpf(x[e], 127 - byte);
        encode(y);
    }
    __device__ __forceinline__ explicit Fp4Block(const double (&x)[VE]) {
        int top = 0, upper[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const uint64_t bits = __builtin_bit_cast(uint64_t, x[e]);
            upper[e] = (int)(bits >> 32) | ((uint32_t)bits != 0);
            top = max(top, upper[e] & 0x7fffffff);
        }
        top = max_block(top, 32 / VE);
        scale_of((top >> 20) - 1023, (top & 0xfffff) > 0xc0000, top < 0x7ff00000);
        float y[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) y[e] = (float)__builtin_ldexp(__builtin_bit_cast(double, (uint64_t)(uint32_t)upper[e] << 32), 127 - byte);
        encode(y);
    }
    // e0: the lane's first element
    __device__ __forceinline__ void store(char *row, unsigned char *scale, int e0) const {
        if constexpr (VE == 8) *reinterpret_cast<uint32_t *>(row) = codes;
        else *reinterpret_cast<uint16_t *>(row) = (uint16_t)codes;
        if (e0 % 32 == 0) *scale = (unsigned char)byte;
    }
};
template <int LANES> __device__ __forceinline__ double row_sum(double x) {
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) x += __shfl_xor(x, d, 64);
    return x;
}
// A key's elements, normed, weighted and turned, in 64 bits
template <typename T, int K, int ROT>
__device__ __forceinline__ void key64(const HeadsArgs &a, const Turn<T, K, ROT> &turn, const Weights<T, K, ROT> &w, const u32x4 &raw,
                                      const float (&x)[HeadRow<T, K>::VE], const float (&c)[HeadRow<T, K>::VE], const float (&s)[HeadRow<T, K>::VE], bool off_table,
                                      double (&z)[HeadRow<T, K>::VE]) {
    constexpr int VE = HeadRow<T, K>::VE;
    double r = 1.0;
    if (a.norm != 0) {
        double ss = 0.0;
#pragma unroll
        for (int e = 0; e < VE; ++e) ss = __builtin_fma((double)x[e], (double)x[e], ss);
        const double d = __builtin_fma(row_sum<HeadRow<T, K>::LANES>(ss), (double)a.mean, (double)a.eps);
        r = __builtin_amdgcn_rsq(d);
#pragma unroll
        for (int i = 0; i < 2; ++i) r = __builtin_fma(r * 0.5, __builtin_fma(-d * r, r, 1.0), r);
        if (d == __builtin_inf()) r = 0.0;
    }
    if (off_table) r = __builtin_nan("");
#pragma unroll
    for (int e = 0; e < VE; ++e) z[e] = (double)x[e] * (r * (double)w.own[1][e]);
    if constexpr (ROT != ROT_NONE) {
        float y[VE];
        turn.partners(raw, y);
#pragma unroll
        for (int e = 0; e < VE; ++e) z[e] = __builtin_fma(z[e], (double)c[e], (double)y[e] * (r * (double)w.partner[1][e]) * (double)s[e]);
    }
}

// One use of each 64 bytes of the arguments, so that their loads are on their way at once (a token appended 3.79 us, so 3.58; 512 6.16, so 5.83)
template <bool APPEND> __device__ __forceinline__ void ask_arguments(const HeadsArgs &a) {
    asm volatile("" ::"s"(a.T), "s"(a.q.data), "s"(a.v.token), "s"(a.k_out.head));
    if constexpr (APPEND) asm volatile("" ::"s"(a.cache_k.head), "s"(a.table_stride));
}

// A wavefront walks (token, part of its blocks of rows) pairs in steps of the grid; it has the loads of NB blocks in flight at a time.
// APPEND: keys go to the cache, values follow them unchanged; MX: a cache in 4 bits, for which keys are computed in 64 bits (below).  AHEAD: the next blocks are asked for before these are written, as a wait for loads is one
// for the writes before them too (rule and figures: heads_ahead).
template <typename T, int K, bool VEC, int ROT, bool APPEND, bool AHEAD, bool MX = false>
__global__ __launch_bounds__(HEADS_T) void heads_fwd_kernel(HeadsArgs a) {
    using HR = HeadRow<T, K>;
    constexpr int VE = HR::VE, ROWS = HR::ROWS, NB = 2;
    const int lane = threadIdx.x & 63, sub = lane / HR::LANES, e0 = (lane % HR::LANES) * VE;
    ask_arguments<APPEND>(a);
    const Turn<T, K, ROT> turn(a.rotary_dim, lane);
    Weights<T, K, ROT> w;
    w.load(a, turn, lane);

    const unsigned items = (unsigned)a.tokens * (unsigned)a.parts, stride = gridDim.x * (HEADS_T / 64);
    for (unsigned item = __builtin_amdgcn_readfirstlane(blockIdx.x * (HEADS_T / 64) + (threadIdx.x >> 6)); item < items; item += stride) {
        const unsigned token = item / (unsigned)a.parts;
        const int part = item % (unsigned)a.parts, b = token / (unsigned)a.T, t = token % (unsigned)a.T;
        const int blk_end = min(a.blocks, (part + 1) * a.per_part);
        const int pos = a.positions ? a.positions[token] : t;
        const bool none = pos < 0;
        const bool off_table = ROT && pos >= a.rotary_rows;
        float c[VE], s[VE];
        if constexpr (ROT != ROT_NONE) turn.load(a.rotary + (size_t)(none || off_table ? 0 : pos) * a.rotary_dim, a.rotary_dim, c, s);
        using At = std::conditional_t<MX, char, T>;             // (rows in 4 bits: steps in bytes)
        At *page_k = nullptr, *page_v = nullptr;
        unsigned char *scale_k = nullptr, *scale_v = nullptr;
        if constexpr (APPEND) {
            const int seq = a.seq ? a.seq[token] : b, col = pos >> a.page_shift;
            if (!none && (unsigned)seq < (unsigned)a.n_seqs && col < a.max_pages) {
                const int page = a.table[seq * a.table_stride + col];
                const int slot = pos & ((1 << a.page_shift) - 1);
                if ((unsigned)page < (unsigned)a.n_pages) {
                    page_k = static_cast<At *>(a.cache_k.data) + page * a.cache_k.batch + slot * a.cache_k.token;
                    page_v = static_cast<At *>(a.cache_v.data) + page * a.cache_v.batch + slot * a.cache_v.token;
                    if constexpr (MX) {
                        scale_k = static_cast<unsigned char *>(a.scale_k.data) + page * a.scale_k.batch + slot * a.scale_k.token + e0 / 32;
                        scale_v = static_cast<unsigned char *>(a.scale_v.data) + page * a.scale_v.batch + slot * a.scale_v.token + e0 / 32;
                    }
                }
            }
        }
        const int first = part * a.per_part;
        u32x4 ahead[NB] = {};
        for (int blk0 = AHEAD ? first - NB : first; blk0 < blk_end; blk0 += NB) {
            u32x4 raw[NB];
            if constexpr (AHEAD) {
#pragma unroll
                for (int i = 0; i < NB; ++i) raw[i] = ahead[i];
            }
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int blk = blk0 + (AHEAD ? NB : 0) + i, kind = blk < a.q_blocks ? 0 : blk < a.q_blocks + a.k_blocks ? 1 : 2;
                const int h = (blk - (kind == 0 ? 0 : kind == 1 ? a.q_blocks : a.q_blocks + a.k_blocks)) * ROWS + sub;
                const HeadRows &src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
                u32x4 &to = AHEAD ? ahead[i] : raw[i];
                to = u32x4{0u, 0u, 0u, 0u};
                if (blk < blk_end && h < (kind == 0 ? a.Hq : a.Hk)) to = load_row<T, VEC>(row_at<const T, VEC>(src, b, t, h) + e0);
            }
            if (AHEAD && blk0 < first) continue;
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int blk = blk0 + i, kind = blk < a.q_blocks ? 0 : blk < a.q_blocks + a.k_blocks ? 1 : 2;
                const int h = (blk - (kind == 0 ? 0 : kind == 1 ? a.q_blocks : a.q_blocks + a.k_blocks)) * ROWS + sub;
                if (blk >= blk_end) break;
                const bool live = h < (kind == 0 ? a.Hq : a.Hk);
                if constexpr (APPEND && !MX) {
                    if (kind == 2) {
                        if (live && page_v) *reinterpret_cast<u32x4 *>(page_v + h * a.cache_v.head + e0) = raw[i];
                        continue;
                    }
                }
                float x[VE], z[VE];
                unpack<T>(raw[i], x);
                if constexpr (MX) {                     // (every lane of a block takes part)
                    if (kind == 2) {
                        const Fp4Block<VE> v(x);
                        if (live && page_v) v.store(page_v + h * a.cache_v.head + e0 / 2, scale_v + h * a.scale_v.head, e0);
                        continue;
                    }
                    if (kind == 1) {
                        double y[VE];
                        key64<T, K, ROT>(a, turn, w, raw[i], x, c, s, off_table, y);
                        const Fp4Block<VE> k(y);
                        if (live && page_k) k.store(page_k + h * a.cache_k.head + e0 / 2, scale_k + h * a.scale_k.head, e0);
                        continue;
                    }
                }
                float r = 1.f;
                if (a.norm != 0) {
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < VE; ++e) ss = __builtin_fmaf(x[e], x[e], ss);
                    r = rsqrtf(__builtin_fmaf(row_sum<HR::LANES>(ss), a.mean, a.eps));
                }
                if (off_table) r = __builtin_nanf("");
                if constexpr (ROT == ROT_NONE) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) z[e] = x[e] * (r * (kind == 0 ? w.own[0][e] : w.own[1][e]));
                } else {
                    float y[VE];
                    turn.partners(raw[i], y);
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        // (r first: where the sum of squares passes fp32 it is 0, and what it multiplies must not be infinite by then)
                        const float own = x[e] * (r * (kind == 0 ? w.own[0][e] : w.own[1][e])), other = y[e] * (r * (kind == 0 ? w.partner[0][e] : w.partner[1][e]));
                        z[e] = __builtin_fmaf(own, c[e], other * s[e]);
                    }
                }
                if (!live) continue;
                if (none) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) z[e] = 0.f;
                }
                if constexpr (APPEND && !MX) {
                    if (kind == 1) {
                        if (page_k) store_vec_t(page_k + h * a.cache_k.head + e0, z);
                        continue;
                    }
                }
                store_row<T, VEC, VE>(row_at<T, VEC>(kind == 0 ? a.q_out : a.k_out, b, t, h) + e0, z);
            }
        }
    }
}

// Backward: a wavefront walks (token, part) pairs in steps of the grid, so that its sums over rows of dw stay in registers until the end; the
// partial sums of a workgroup go to a row of `partial` [gridDim.x][2][K], which heads_dw_kernel adds up in a fixed order.
template <typename T, int K, bool VEC, int ROT>
__global__ __launch_bounds__(HEADS_T) void heads_bwd_kernel(HeadsArgs a) {
    using HR = HeadRow<T, K>;
    constexpr int VE = HR::VE, ROWS = HR::ROWS, WAVES = HEADS_T / 64, NB = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane / HR::LANES, e0 = (lane % HR::LANES) * VE;
    const Turn<T, K, ROT> turn(a.rotary_dim, lane);
    float w[2][VE], dw[2][VE];
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        const float *src = kind == 0 ? a.weight_q : a.weight_k;
        if (src) load_floats(w[kind], src + e0);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            if (!src) w[kind][e] = 1.f;
            dw[kind][e] = 0.f;
        }
    }

    const unsigned items = (unsigned)a.tokens * (unsigned)a.parts, stride = gridDim.x * WAVES;
    for (unsigned item = __builtin_amdgcn_readfirstlane(blockIdx.x * WAVES + wave); item < items; item += stride) {
        const unsigned token = item / (unsigned)a.parts;
        const int part = item % (unsigned)a.parts, b = token / (unsigned)a.T, t = token % (unsigned)a.T;
        const int blk_end = min(a.blocks, (part + 1) * a.per_part);
        const int pos = a.positions ? a.positions[token] : t;
        const bool none = pos < 0;
        const bool off_table = ROT && pos >= a.rotary_rows;
        float c[VE], s[VE];
        if constexpr (ROT != ROT_NONE) turn.load(a.rotary + (size_t)(none || off_table ? 0 : pos) * a.rotary_dim, a.rotary_dim, c, s);
        for (int blk0 = part * a.per_part; blk0 < blk_end; blk0 += NB) {
            u32x4 rx[NB], rz[NB];
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int blk = blk0 + i;
                const bool query = blk < a.q_blocks;
                const int h = (query ? blk : blk - a.q_blocks) * ROWS + sub;
                rx[i] = rz[i] = u32x4{0u, 0u, 0u, 0u};
                if (blk < blk_end && h < (query ? a.Hq : a.Hk)) {
                    rx[i] = load_row<T, VEC>(row_at<const T, VEC>(query ? a.q : a.k, b, t, h) + e0);
                    rz[i] = load_row<T, VEC>(row_at<const T, VEC>(query ? a.dq_out : a.dk_out, b, t, h) + e0);
                }
            }
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int blk = blk0 + i;
                const bool query = blk < a.q_blocks;
                const int h = (query ? blk : blk - a.q_blocks) * ROWS + sub;
                if (blk >= blk_end) break;
                const bool live = h < (query ? a.Hq : a.Hk);
                float x[VE], dy[VE], g[VE];
                unpack<T>(rx[i], x);
                unpack<T>(rz[i], dy);
                if constexpr (ROT != ROT_NONE) {
                    float y[VE];
                    turn.partners(rz[i], y);
#pragma unroll
                    for (int e = 0; e < VE; ++e) dy[e] = __builtin_fmaf(dy[e], c[e], -(y[e] * s[e]));
                }
                float r = 1.f, ss = 0.f, gx = 0.f;
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    g[e] = dy[e] * (query ? w[0][e] : w[1][e]);
                    ss = __builtin_fmaf(x[e], x[e], ss);
                    gx = __builtin_fmaf(g[e], x[e], gx);
                }
                if (a.norm != 0) {
                    r = rsqrtf(__builtin_fmaf(row_sum<HR::LANES>(ss), a.mean, a.eps));
                    gx = row_sum<HR::LANES>(gx) * (r * r * a.mean);
                    if (r == 0.f) gx = 0.f;             // (the sum of squares passes fp32, and so may this one: the row is zeros, and so is its gradient)
                }
                if (off_table) r = __builtin_nanf("");
                if (none || !live) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) g[e] = x[e] = dy[e] = 0.f;
                    gx = r = 0.f;
                }
                float dx[VE];
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    dx[e] = r * (a.norm != 0 ? __builtin_fmaf(-gx, x[e], g[e]) : g[e]);       // (without a norm x has no part in it, infinite or NaN)
                    const float term = dy[e] * r;
                    if (query) dw[0][e] = __builtin_fmaf(term, x[e], dw[0][e]);
                    else dw[1][e] = __builtin_fmaf(term, x[e], dw[1][e]);
                }
                if (live) store_row<T, VEC, VE>(row_at<T, VEC>(query ? a.dq : a.dk, b, t, h) + e0, dx);
            }
        }
    }
    if (!a.partial) return;
    // the rows of a block, then the wavefronts
    __shared__ float sums[WAVES][2][K];
#pragma unroll
    for (int kind = 0; kind < 2; ++kind)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            float v = dw[kind][e];
            if (HR::LANES <= 8) v += __shfl_xor(v, 8, 64);
            if (HR::LANES <= 16) v = add_xor16(v);
            if (HR::LANES <= 32) v = add_xor32(v);
            if (sub == 0) sums[wave][kind][e0 + e] = v;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * K; i += HEADS_T) {
        float v = 0.f;
#pragma unroll
        for (int u = 0; u < WAVES; ++u) v += (&sums[u][0][0])[i];
        a.partial[(size_t)blockIdx.x * 2 * K + i] = v;
    }
}

// dw = sum of the n rows of partial [n][2][K]: 16 columns a workgroup, its 64 groups of 16 lanes add up every 64th row
constexpr int DW_COLS = 16, DW_T = 1024, DW_ROWS = DW_T / DW_COLS;
__global__ __launch_bounds__(DW_T) void heads_dw_kernel(const float *partial, int n, int K, float *dwq, float *dwk) {
    __shared__ float s[DW_T / 64][DW_COLS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane % DW_COLS, c = blockIdx.x * DW_COLS + col;
    float v = 0.f;
#pragma unroll 8
    for (int i = threadIdx.x / DW_COLS; i < n; i += DW_ROWS) v += partial[(size_t)i * 2 * K + c];
    v = add_xor32(add_xor16(v));
    if (lane < DW_COLS) s[wave][col] = v;
    __syncthreads();
    if (wave != 0) return;
    v = (s[lane / DW_COLS][col] + s[lane / DW_COLS + 4][col]) + (s[lane / DW_COLS + 8][col] + s[lane / DW_COLS + 12][col]);
    v = add_xor32(add_xor16(v));
    float *dst = c < K ? dwq : dwk;
    if (lane < DW_COLS && dst) dst[c < K ? c : c - K] = v;
}

// Rows of a 4-bit cache as values: a wavefront takes blocks of rows (64 lanes of 8 elements) of a token
template <typename T, int K, bool VEC> __global__ __launch_bounds__(HEADS_T) void read_mx_kernel(HeadsArgs a) {
    constexpr int VE = 8, LANES = K / VE, ROWS = 64 / LANES, PER = 16 / sizeof(T);
    const int lane = threadIdx.x & 63, sub = lane / LANES, e0 = lane % LANES * VE;
    const unsigned items = (unsigned)a.tokens * (unsigned)a.parts, stride = gridDim.x * (HEADS_T / 64);
    for (unsigned item = __builtin_amdgcn_readfirstlane(blockIdx.x * (HEADS_T / 64) + (threadIdx.x >> 6)); item < items; item += stride) {
        const unsigned token = item / (unsigned)a.parts;
        const int part = item % (unsigned)a.parts, b = token / (unsigned)a.T, t = token % (unsigned)a.T;
        const int pos = a.positions[token], seq = a.seq ? a.seq[token] : b, col = max(pos, 0) >> a.page_shift, slot = pos & ((1 << a.page_shift) - 1);
        int page = -1;
        if (pos >= 0 && (unsigned)seq < (unsigned)a.n_seqs && col < a.max_pages) page = a.table[seq * a.table_stride + col];
        const bool there = (unsigned)page < (unsigned)a.n_pages;
        for (int blk = part * a.per_part; blk < min(a.blocks, (part + 1) * a.per_part); ++blk) {
            const bool value = blk >= a.k_blocks;
            const int h = (value ? blk - a.k_blocks : blk) * ROWS + sub;
            if (h >= a.Hk) continue;
            const HeadRows &row = value ? a.cache_v : a.cache_k, &scale = value ? a.scale_v : a.scale_k, &out = value ? a.v : a.k_out;
            float x[VE];
            if (there) {
                const uint32_t codes = *reinterpret_cast<const uint32_t *>(static_cast<const char *>(row.data) + page * row.batch + slot * row.token + h * row.head + e0 / 2);
                fp4_values(codes, fp4_scale(*(static_cast<const unsigned char *>(scale.data) + page * scale.batch + slot * scale.token + h * scale.head + e0 / 32)), x);
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) x[e] = pos < 0 ? 0.f : __builtin_nanf("");
            }
            T *to = row_at<T, VEC>(out, b, t, h) + e0;
#pragma unroll
            for (int v = 0; v < VE / PER; ++v) {
                float y[PER];
#pragma unroll
                for (int e = 0; e < PER; ++e) y[e] = x[v * PER + e];
                store_row<T, VEC, PER>(to + v * PER, y);
            }
        }
    }
}

namespace {
template <typename T, int K> int cut(HeadsArgs &a, bool backward) {
    const HeadsPlan h = heads_plan(a.tokens, a.Hq, a.Hk, K, sizeof(T) == 2, a.append, backward);
    a.q_blocks = h.q_blocks; a.k_blocks = h.k_blocks; a.blocks = h.blocks; a.parts = h.parts; a.per_part = h.per_part;
    return h.workgroups;
}
template <typename T, int K, bool VEC, int ROT> void fwd_of(HeadsArgs a, hipStream_t st) {
    const dim3 g((unsigned)cut<T, K>(a, false)), t(HEADS_T);
    if (!a.append) hipLaunchKernelGGL((heads_fwd_kernel<T, K, VEC, ROT, false, false>), g, t, 0, st, a);
    else if (a.mx) hipLaunchKernelGGL((heads_fwd_kernel<T, K, VEC, ROT, true, false, true>), g, t, 0, st, a);
    else if (VEC && heads_ahead(a.tokens, a.blocks)) hipLaunchKernelGGL((heads_fwd_kernel<T, K, VEC, ROT, true, VEC>), g, t, 0, st, a);
    else hipLaunchKernelGGL((heads_fwd_kernel<T, K, VEC, ROT, true, false>), g, t, 0, st, a);
}
template <typename T, int K, bool VEC, int ROT> void bwd_of(HeadsArgs a, hipStream_t st) {
    const int n = cut<T, K>(a, true);
    hipLaunchKernelGGL((heads_bwd_kernel<T, K, VEC, ROT>), dim3((unsigned)n), dim3(HEADS_T), 0, st, a);
    if (a.partial)
        hipLaunchKernelGGL(heads_dw_kernel, dim3(2 * K / DW_COLS), dim3(DW_T), 0, st, a.partial, n, K, a.dweight_q, a.dweight_k);
}
template <typename T, int K, bool VEC> void by_rotation(const HeadsArgs &a, bool backward, hipStream_t st) {
    if (!a.rotary) backward ? bwd_of<T, K, VEC, ROT_NONE>(a, st) : fwd_of<T, K, VEC, ROT_NONE>(a, st);
    else if (a.interleaved) backward ? bwd_of<T, K, VEC, ROT_PAIRS>(a, st) : fwd_of<T, K, VEC, ROT_PAIRS>(a, st);
    else backward ? bwd_of<T, K, VEC, ROT_HALF>(a, st) : fwd_of<T, K, VEC, ROT_HALF>(a, st);
}
template <typename T> int by_width(const HeadsArgs &a, bool backward, hipStream_t st) {
    auto go = [&](auto k) {
        a.aligned ? by_rotation<T, decltype(k)::value, true>(a, backward, st) : by_rotation<T, decltype(k)::value, false>(a, backward, st);
        return 0;
    };
    switch (a.K) {
        case 64: return go(std::integral_constant<int, 64>{});
        case 128: return go(std::integral_constant<int, 128>{});
        case 256: return go(std::integral_constant<int, 256>{});
        default: return -1;
    }
}
}  // namespace

namespace {
template <typename T> int read_of(HeadsArgs a, hipStream_t st) {
    const int rows = 64 * 8 / a.K;
    a.k_blocks = (a.Hk + rows - 1) / rows;
    a.blocks = 2 * a.k_blocks;
    a.per_part = heads_blocks_per_wave(a.tokens, a.blocks);
    a.parts = (a.blocks + a.per_part - 1) / a.per_part;
    const dim3 g((unsigned)heads_fwd_workgroups((long long)a.tokens * a.parts)), t(HEADS_T);
    auto go = [&](auto k) {
        if (a.aligned) hipLaunchKernelGGL((read_mx_kernel<T, decltype(k)::value, true>), g, t, 0, st, a);
        else hipLaunchKernelGGL((read_mx_kernel<T, decltype(k)::value, false>), g, t, 0, st, a);
        return 0;
    };
    switch (a.K) {
        case 64: return go(std::integral_constant<int, 64>{});
        case 128: return go(std::integral_constant<int, 128>{});
        case 256: return go(std::integral_constant<int, 256>{});
        default: return -1;
    }
}
}  // namespace

int launch_read_mx(const HeadsArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? read_of<bf16>(a, st) : read_of<float>(a, st); }
int launch_heads_fwd(const HeadsArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? by_width<bf16>(a, false, st) : by_width<float>(a, false, st); }
int launch_heads_bwd(const HeadsArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? by_width<bf16>(a, true, st) : by_width<float>(a, true, st); }

}  // namespace osdn
