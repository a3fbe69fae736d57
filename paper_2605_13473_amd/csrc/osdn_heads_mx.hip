// The append to a paged cache in 4 bits, and the way back from it.
//
// A wavefront takes 64 / LANES tokens next to each other, the lanes of a row one of them each, and walks the heads of their queries, keys and values: what does not depend on the head
// (position, page, angles, the rows' addresses) is found once for all of them, and the codes of adjacent tokens, which a cache that holds a page head
// after head has side by side, leave together.  Bound by memory: 65536 tokens of 16 + 4 + 4 heads of 128 in bf16 appended 147 us, 4.8 TB/s (a token a wavefront 205: 80 MB more are written,
// as rows of 64 and 4 bytes leave one by one), and read back 31 us, 5.6 TB/s (43).  (Append: calls in a loop; read back: the smallest of twelve launches in a kernel trace.)
#include "osdn_heads.h"

namespace osdn {

// A block of 32 elements, VE of them a lane, becomes codes and a scale 2^e, e the least (from -120 to 125) with the largest element no more than 7 * 2^e: what lies
// between 6 and 7 is off by no more than what lies between 4 and 6 may be.  The codes are the nearest values, ties to the even code.
// Which code that is must not hang on a rounding before.  Values come as they are.  Keys are computed in fp32 with a bound of their error, and where an element with
// its error either way could get another code or sign, or its block another scale, once more in 64 bits.  (All of them in 64 bits, a wavefront a token: 65536 tokens of 16 + 4 + 4 heads of 128
// in bf16 293 us, so 201.)  Of normed or rotated keys one block of rows in hundreds goes that way.  Keys of bf16 that come as they are mostly do: they have no error, but get its bound all
// the same, and one of their elements in ninety stands on a border of two codes.  The same tokens without norm and rotation take 143 us, as memory is what they wait for.
__device__ __forceinline__ int max_block(int x, int lanes) {
    auto with = [&](int y) { x = max(x, y); };
    with(__builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, true));         // quad_perm [1,0,3,2]
    with(__builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, true));         // quad_perm [2,3,0,1]
    if (lanes > 4) with(__builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true));     // row_half_mirror
    return x;
}
// the scale's byte for the largest element of a block, by its bits in fp32
__device__ __forceinline__ int fp4_byte(int top) { return top >= 0x7f800000 ? 255 : max(7, min(252, (top >> 23) - 2 + ((top & 0x7fffff) > 0x600000))); }
template <int VE> __device__ __forceinline__ int largest(const float (&x)[VE]) {
    int top = 0;
#pragma unroll
    for (int e = 0; e < VE; ++e) top = max(top, __builtin_bit_cast(int, x[e]) & 0x7fffffff);
    return top;
}
template <int VE> __device__ __forceinline__ uint32_t fp4_codes(const float (&x)[VE], int byte) {
    const float scale = fp4_scale(byte);
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
    if constexpr (VE == 8) {
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
    }
    return codes;
}
// e0: the lane's first element
template <int VE> __device__ __forceinline__ void store_fp4(uint32_t codes, int byte, char *row, unsigned char *scale, int e0) {
    if (byte == 255) codes = 0;
    if constexpr (VE == 8) *reinterpret_cast<uint32_t *>(row) = codes;
    else *reinterpret_cast<uint16_t *>(row) = (uint16_t)codes;
    if (e0 % 32 == 0) *scale = (unsigned char)byte;
}
template <int LANES> __device__ __forceinline__ double row_sum(double x) {
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) x += __shfl_xor(x, d, 64);
    return x;
}

// The weights of a lane's elements and of their partners
template <int VE> struct RowWeights { float own[VE], partner[VE]; };
template <typename T, int K, int ROT> __device__ __forceinline__ RowWeights<HeadRow<T, K>::VE> weights_of(const float *w, const Turn<T, K, ROT> &turn, int lane) {
    constexpr int VE = HeadRow<T, K>::VE;
    RowWeights<VE> r;
#pragma unroll
    for (int e = 0; e < VE; ++e) r.own[e] = r.partner[e] = 1.f;
    if (w) {
        load_floats(r.own, w + (lane & (HeadRow<T, K>::LANES - 1)) * VE);
        if constexpr (ROT == ROT_PAIRS) {
#pragma unroll
            for (int e = 0; e < VE; ++e) r.partner[e] = r.own[e ^ 1];
        }
        if constexpr (ROT == ROT_HALF) load_floats(r.partner, w + turn.partner_element(lane, 0));
    }
    return r;
}

// The lane's elements of a key in 64 bits, one after the other (side by side they would take the registers of another workgroup): x, and y at the partners' places.  The upper
// word of a number says all that a code asks for if its last bit is set where the lower word is not zero: no border of two codes has that many digits.
template <typename T, int K, int ROT>
__device__ __forceinline__ void key_in_64_bits(const HeadsArgs &a, const RowWeights<HeadRow<T, K>::VE> &w, const float (&x)[HeadRow<T, K>::VE], const float (&y)[HeadRow<T, K>::VE],
                                               const float (&c)[HeadRow<T, K>::VE], const float (&s)[HeadRow<T, K>::VE], bool off_table, uint32_t &codes, int &byte) {
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
    int top = 0, upper[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        auto wide = [](float v) {               // (here, not ahead of the loops around, where its registers would be held)
            asm volatile("" : "+v"(v));
            return (double)v;
        };
        double z = (double)x[e] * (r * wide(w.own[e]));
        if constexpr (ROT != ROT_NONE) z = __builtin_fma(z, wide(c[e]), (double)y[e] * (r * wide(w.partner[e])) * wide(s[e]));
        const uint64_t bits = __builtin_bit_cast(uint64_t, z);
        upper[e] = (int)((uint32_t)(bits >> 32) | (uint32_t)((uint32_t)bits != 0));
        top = max(top, upper[e] & 0x7fffffff);
        __builtin_amdgcn_sched_barrier(0);
    }
    top = max_block(top, 32 / VE);
    byte = top >= 0x7ff00000 ? 255 : max(-120, min(125, (top >> 20) - 1025 + ((top & 0xfffff) > 0xc0000))) + 127;
    codes = 0;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        const float v = (float)__builtin_ldexp(__builtin_bit_cast(double, (uint64_t)(uint32_t)upper[e] << 32), 127 - byte);
        codes |= (__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v, 0.f, 1.f, 0) & 15u) << (4 * e);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// How far an element of a key in fp32 is off, in parts of |own cosine| + |other sine|: the sum of squares is at most 15 roundings deep, of which half count in its root, which is two off
// by itself; the products with the weight, the row and the angle and the last sum are one each: 13.5 * 2^-24, and this is 32.
constexpr float KEY_OFF = 0x1p-19f;

// KEY: an element's error too.  The same steps as in heads_fwd_kernel, so that queries come out the same
template <typename T, int K, int ROT, bool KEY>
__device__ __forceinline__ bool row_ready(const HeadsArgs &a, const Turn<T, K, ROT> &turn, const RowWeights<HeadRow<T, K>::VE> &w, const u32x4 &raw, const float (&x)[HeadRow<T, K>::VE],
                                          const float (&c)[HeadRow<T, K>::VE], const float (&s)[HeadRow<T, K>::VE], bool off_table, float (&z)[HeadRow<T, K>::VE],
                                          float (&off)[HeadRow<T, K>::VE]) {
    using HR = HeadRow<T, K>;
    constexpr int VE = HR::VE;
    bool sure = true;                           // the sum of squares is far from where fp32 ends
    float r = 1.f;
    if (a.norm != 0) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < VE; ++e) ss = __builtin_fmaf(x[e], x[e], ss);
        const float d = __builtin_fmaf(row_sum<HR::LANES>(ss), a.mean, a.eps);
        r = rsqrtf(d);
        sure = d > 0x1p-60f && d < 0x1p100f;
    }
    if (off_table) r = __builtin_nanf("");
    if constexpr (ROT == ROT_NONE) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            z[e] = x[e] * (r * w.own[e]);
            if constexpr (KEY) off[e] = __builtin_fabsf(z[e]) * KEY_OFF;
        }
    } else {
        float y[VE];
        turn.partners(raw, y);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float own = x[e] * (r * w.own[e]), other = y[e] * (r * w.partner[e]);
            z[e] = __builtin_fmaf(own, c[e], other * s[e]);
            if constexpr (KEY) {                // (and where products are next to the smallest numbers no less than all of them)
                const float both = __builtin_fmaf(__builtin_fabsf(own), __builtin_fabsf(c[e]), __builtin_fabsf(other * s[e]));
                off[e] = __builtin_fmaf(both, KEY_OFF, __builtin_fminf(both, 0x1p-140f));
            }
        }
    }
    return sure;
}

// One use of each 64 bytes of the arguments: the scalar loads of all of them are on their way at once (one token appended and read 6.7 us, so 6.5; 512 8.95 and 8.75)
__device__ __forceinline__ void ask_arguments(const HeadsArgs &a) {
    asm volatile("" ::"s"(a.T), "s"(a.q.data), "s"(a.v.token), "s"(a.k_out.head), "s"(a.cache_k.head), "s"(a.table_stride), "s"(a.scale_k.data), "s"(a.scale_v.head));
}

template <typename T, int K, bool VEC, int ROT> __global__ __launch_bounds__(HEADS_T) void append_mx_kernel(HeadsArgs a) {
    ask_arguments(a);
    using HR = HeadRow<T, K>;
    constexpr int VE = HR::VE, ROWS = HR::ROWS, NB = sizeof(T) == 2 ? 4 : 2;
    const int lane = threadIdx.x & 63, sub = lane / HR::LANES, e0 = (lane % HR::LANES) * VE;
    const Turn<T, K, ROT> turn(a.rotary_dim, lane);
    const unsigned groups = ((unsigned)a.tokens + ROWS - 1) / ROWS, items = groups * (unsigned)a.parts, stride = gridDim.x * (HEADS_T / 64);
    for (unsigned item = __builtin_amdgcn_readfirstlane(blockIdx.x * (HEADS_T / 64) + (threadIdx.x >> 6)); item < items; item += stride) {
        const unsigned group = item / (unsigned)a.parts;
        const int part = item % (unsigned)a.parts, first = part * a.per_part, last = min(a.blocks, first + a.per_part);       // heads: queries, keys, values
        const bool live = group * ROWS + sub < (unsigned)a.tokens;
        const unsigned token = live ? group * ROWS + sub : (unsigned)a.tokens - 1, b = token / (unsigned)a.T, t = token - b * (unsigned)a.T;
        const int pos = a.positions[token], seq = a.seq ? a.seq[token] : (int)b;
        const bool none = pos < 0, off_table = ROT && pos >= a.rotary_rows;
        // the rows of heads [h0, h1) of this lane's token, NB at a time, the next ones asked for before these are made ready (65536 tokens of 16 + 4 + 4, NB = 1, 2 and 4 164, 161 and
        // 154 us; fp32, 8192 of 16 + 8 + 8, 45, 47, 51)
        auto rows = [&](const HeadRows &src, int h0, int h1, auto &&each) {
            if (h0 >= h1) return;
            const T *from = row_at<const T, VEC>(src, b, t, 0) + e0;
            u32x4 ahead[NB];
            auto ask = [&](int h) {
#pragma unroll
                for (int i = 0; i < NB; ++i) ahead[i] = load_row<T, VEC>(from + min(h + i, h1 - 1) * src.head);
            };
            ask(h0);
            for (int h = h0; h < h1; h += NB) {
                u32x4 raw[NB];
#pragma unroll
                for (int i = 0; i < NB; ++i) raw[i] = ahead[i];
                if (h + NB < h1) ask(h + NB);
#pragma unroll
                for (int i = 0; i < NB; ++i)
                    if (h + i < h1) {
                        float x[VE];
                        unpack<T>(raw[i], x);
                        each(h + i, raw[i], x);
                    }
            }
        };
        float c[VE], s[VE];
        if constexpr (ROT != ROT_NONE)
            if (first < a.Hq + a.Hk) turn.load(a.rotary + (size_t)(none || off_table ? 0 : pos) * a.rotary_dim, a.rotary_dim, c, s);
        if (first < a.Hq) {
            const RowWeights<VE> w = weights_of<T, K, ROT>(a.weight_q, turn, lane);
            T *to = row_at<T, VEC>(a.q_out, b, t, 0) + e0;
            rows(a.q, first, min(last, a.Hq), [&](int h, const u32x4 &raw, const float (&x)[VE]) {
                float z[VE], off[VE];
                row_ready<T, K, ROT, false>(a, turn, w, raw, x, c, s, off_table, z, off);
                if (!live) return;
                if (none) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) z[e] = 0.f;
                }
                store_row<T, VEC, VE>(to + h * a.q_out.head, z);
            });
        }
        if (last <= a.Hq) continue;
        // keys and values: their places in the cache
        char *page_k = nullptr, *page_v = nullptr;
        unsigned char *scale_k = nullptr, *scale_v = nullptr;
        {
            const int col = pos >> a.page_shift, slot = pos & ((1 << a.page_shift) - 1);
            if (live && !none && (unsigned)seq < (unsigned)a.n_seqs && col < a.max_pages) {
                const long long page = a.table[seq * a.table_stride + col];
                if ((unsigned long long)page < (unsigned long long)a.n_pages) {
                    page_k = static_cast<char *>(a.cache_k.data) + page * a.cache_k.batch + slot * a.cache_k.token + e0 / 2;
                    page_v = static_cast<char *>(a.cache_v.data) + page * a.cache_v.batch + slot * a.cache_v.token + e0 / 2;
                    scale_k = static_cast<unsigned char *>(a.scale_k.data) + page * a.scale_k.batch + slot * a.scale_k.token + e0 / 32;
                    scale_v = static_cast<unsigned char *>(a.scale_v.data) + page * a.scale_v.batch + slot * a.scale_v.token + e0 / 32;
                }
            }
        }
        if (first < a.Hq + a.Hk) {
            const RowWeights<VE> w = weights_of<T, K, ROT>(a.weight_k, turn, lane);
            // (the factor of a row is at least 2^-50 where its sum is far from where fp32 ends: times such a weight it has all its digits)
            uint32_t least_weight = ~0u;            // twice the bits of its magnitude, less one: of zero the largest
#pragma unroll
            for (int e = 0; e < VE; ++e) least_weight = min(least_weight, 2 * __builtin_bit_cast(uint32_t, w.own[e]) - 1u);
            const bool whole_digits = least_weight >= 2 * __builtin_bit_cast(uint32_t, 0x1p-60f) - 1u || a.norm == 0;
            rows(a.k, max(first, a.Hq) - a.Hq, min(last, a.Hq + a.Hk) - a.Hq, [&](int h, const u32x4 &raw, const float (&x)[VE]) {
                float z[VE], off[VE];
                bool sure = row_ready<T, K, ROT, true>(a, turn, w, raw, x, c, s, off_table, z, off) && whole_digits;
                // the elements as large and as small as they may be: the same byte, the same codes
                auto moved = [&](int e, float by) { return __builtin_copysignf(__builtin_fmaxf(__builtin_fmaf(off[e], by, __builtin_fabsf(z[e])), 0.f), z[e]); };
                float most = 0.f, least = 0.f;
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    most = __builtin_fmaxf(most, __builtin_fabsf(z[e]) + off[e]);
                    least = __builtin_fmaxf(least, __builtin_fabsf(z[e]) - off[e]);
                    // (not so of NaN; and what cancels below its error could have either sign)
                    sure = sure && off[e] < 0x1p100f && !(off[e] > 0.f && __builtin_fabsf(z[e]) <= off[e]);
                }
                int byte = fp4_byte(max_block(__builtin_bit_cast(int, most), 32 / VE));
                sure = sure && byte == fp4_byte(max_block(__builtin_bit_cast(int, least), 32 / VE));
                uint32_t codes = 0;
                const float scale = fp4_scale(byte);
#pragma unroll
                for (int e = 0; e < VE; e += 2) {
                    const uint32_t up = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, moved(e, 1.f), moved(e + 1, 1.f), scale, 0);
                    const uint32_t down = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, moved(e, -1.f), moved(e + 1, -1.f), scale, 0);
                    sure = sure && up == down;
                    codes |= (up & 255u) << (4 * e);
                }
                if (__any(!sure)) {
                    float y[VE];
                    if constexpr (ROT != ROT_NONE) turn.partners(raw, y);
                    key_in_64_bits<T, K, ROT>(a, w, x, y, c, s, off_table, codes, byte);
                }
                if (page_k) store_fp4<VE>(codes, byte, page_k + h * a.cache_k.head, scale_k + h * a.scale_k.head, e0);
            });
        }
        rows(a.v, max(first, a.Hq + a.Hk) - a.Hq - a.Hk, last - a.Hq - a.Hk, [&](int h, const u32x4 &, const float (&x)[VE]) {
            const int byte = fp4_byte(max_block(largest(x), 32 / VE));
            if (page_v) store_fp4<VE>(fp4_codes(x, byte), byte, page_v + h * a.cache_v.head, scale_v + h * a.scale_v.head, e0);
        });
    }
}

// Rows of the cache as values: a lane 8 elements of a row of each head
template <typename T, int K, bool VEC> __global__ __launch_bounds__(HEADS_T) void read_mx_kernel(HeadsArgs a) {
    ask_arguments(a);
    constexpr int VE = 8, LANES = K / VE, ROWS = 64 / LANES, PER = 16 / sizeof(T), NB = 4;
    const int lane = threadIdx.x & 63, sub = lane / LANES, e0 = lane % LANES * VE;
    const unsigned groups = ((unsigned)a.tokens + ROWS - 1) / ROWS, items = groups * (unsigned)a.parts, stride = gridDim.x * (HEADS_T / 64);
    for (unsigned item = __builtin_amdgcn_readfirstlane(blockIdx.x * (HEADS_T / 64) + (threadIdx.x >> 6)); item < items; item += stride) {
        const unsigned group = item / (unsigned)a.parts;
        const int part = item % (unsigned)a.parts, first = part * a.per_part, last = min(a.blocks, first + a.per_part);       // heads: keys, values
        const unsigned token = group * ROWS + sub;
        if (token >= (unsigned)a.tokens) continue;
        const unsigned b = token / (unsigned)a.T, t = token - b * (unsigned)a.T;
        const int pos = a.positions[token], seq = a.seq ? a.seq[token] : (int)b, col = max(pos, 0) >> a.page_shift, slot = pos & ((1 << a.page_shift) - 1);
        long long page = -1;
        if (pos >= 0 && (unsigned)seq < (unsigned)a.n_seqs && col < a.max_pages) page = a.table[seq * a.table_stride + col];
        const bool there = (unsigned long long)page < (unsigned long long)a.n_pages;
        const float missing = pos < 0 ? 0.f : __builtin_nanf("");
        auto rows = [&](const HeadRows &row, const HeadRows &scale, const HeadRows &out, int h0, int h1) {
            if (h0 >= h1) return;
            const char *codes = static_cast<const char *>(row.data) + (there ? page * row.batch + slot * row.token : 0) + e0 / 2;
            const unsigned char *bytes = static_cast<const unsigned char *>(scale.data) + (there ? page * scale.batch + slot * scale.token : 0) + e0 / 32;
            T *to = row_at<T, VEC>(out, b, t, 0) + e0;
            for (int h = h0; h < h1; h += NB) {
                uint32_t word[NB];
                unsigned byte[NB];
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    word[i] = *reinterpret_cast<const uint32_t *>(codes + min(h + i, h1 - 1) * row.head);
                    byte[i] = bytes[min(h + i, h1 - 1) * scale.head];
                }
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    if (h + i >= h1) break;
                    float x[VE];
                    fp4_values(word[i], fp4_scale(byte[i]), x);
#pragma unroll
                    for (int v = 0; v < VE / PER; ++v) {
                        float y[PER];
#pragma unroll
                        for (int e = 0; e < PER; ++e) y[e] = there ? x[v * PER + e] : missing;
                        store_row<T, VEC, PER>(to + (h + i) * out.head + v * PER, y);
                    }
                }
            }
        };
        rows(a.cache_k, a.scale_k, a.k_out, first, min(last, a.Hk));
        rows(a.cache_v, a.scale_v, a.v, max(first, a.Hk) - a.Hk, last - a.Hk);
    }
}

namespace {
template <typename F> int by_width(int K, F &&f) {
    switch (K) {
        case 64: f(std::integral_constant<int, 64>{}); return 0;
        case 128: f(std::integral_constant<int, 128>{}); return 0;
        case 256: f(std::integral_constant<int, 256>{}); return 0;
        default: return -1;
    }
}
// heads of a wavefront, and the workgroups; rows: of a wavefront, a token each
dim3 cut(HeadsArgs &a, int heads, int rows) {
    const long long groups = ((long long)a.tokens + rows - 1) / rows;
    a.blocks = heads;
    a.per_part = heads_mx_per_wave(groups, heads);
    a.parts = (heads + a.per_part - 1) / a.per_part;
    return dim3((unsigned)heads_fwd_workgroups(groups * a.parts));
}
template <typename T> int append_of(HeadsArgs a, hipStream_t st) {
    return by_width(a.K, [&](auto k) {
        constexpr int K = decltype(k)::value;
        const dim3 g = cut(a, a.Hq + 2 * a.Hk, HeadRow<T, K>::ROWS), t(HEADS_T);
        auto go = [&](auto vec, auto rot) { hipLaunchKernelGGL((append_mx_kernel<T, K, decltype(vec)::value, decltype(rot)::value>), g, t, 0, st, a); };
        auto turned = [&](auto vec) {
            if (!a.rotary) go(vec, std::integral_constant<int, ROT_NONE>{});
            else if (a.interleaved) go(vec, std::integral_constant<int, ROT_PAIRS>{});
            else go(vec, std::integral_constant<int, ROT_HALF>{});
        };
        a.aligned ? turned(std::true_type{}) : turned(std::false_type{});
    });
}
template <typename T> int read_of(HeadsArgs a, hipStream_t st) {
    return by_width(a.K, [&](auto k) {
        constexpr int K = decltype(k)::value;
        const dim3 g = cut(a, 2 * a.Hk, 64 * 8 / K), t(HEADS_T);
        if (a.aligned) hipLaunchKernelGGL((read_mx_kernel<T, K, true>), g, t, 0, st, a);
        else hipLaunchKernelGGL((read_mx_kernel<T, K, false>), g, t, 0, st, a);
    });
}
}  // namespace

int launch_append_mx(const HeadsArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? append_of<bf16>(a, st) : append_of<float>(a, st); }
int launch_read_mx(const HeadsArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? read_of<bf16>(a, st) : read_of<float>(a, st); }

}  // namespace osdn
