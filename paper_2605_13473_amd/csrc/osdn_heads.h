// Rows of queries, keys and values: what a lane holds of one, sums over it, the rotation of its pairs and its weights.
#pragma once
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

}  // namespace osdn
