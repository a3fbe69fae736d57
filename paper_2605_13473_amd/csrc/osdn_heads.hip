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

// One use of each 64 bytes of the arguments, so that their loads are on their way at once (a token appended 3.79 us, so 3.58; 512 6.16, so 5.83)
template <bool APPEND> __device__ __forceinline__ void ask_arguments(const HeadsArgs &a) {
    asm volatile("" ::"s"(a.T), "s"(a.q.data), "s"(a.v.token), "s"(a.k_out.head));
    if constexpr (APPEND) asm volatile("" ::"s"(a.cache_k.head), "s"(a.table_stride));
}

// A wavefront walks (token, part of its blocks of rows) pairs in steps of the grid; it has the loads of NB blocks in flight at a time.
// APPEND: keys go to the cache, values follow them unchanged.  AHEAD: the next blocks are asked for before these are written, as a wait for loads is one
// for the writes before them too (rule and figures: heads_ahead).
template <typename T, int K, bool VEC, int ROT, bool APPEND, bool AHEAD>
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
        T *page_k = nullptr, *page_v = nullptr;
        if constexpr (APPEND) {
            const int seq = a.seq ? a.seq[token] : b, col = pos >> a.page_shift;
            if (!none && (unsigned)seq < (unsigned)a.n_seqs && col < a.max_pages) {
                const int page = a.table[seq * a.table_stride + col];
                const int slot = pos & ((1 << a.page_shift) - 1);
                if ((unsigned)page < (unsigned)a.n_pages) {
                    page_k = static_cast<T *>(a.cache_k.data) + page * a.cache_k.batch + slot * a.cache_k.token;
                    page_v = static_cast<T *>(a.cache_v.data) + page * a.cache_v.batch + slot * a.cache_v.token;
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
                if (APPEND && kind == 2) {
                    if (live && page_v) *reinterpret_cast<u32x4 *>(page_v + h * a.cache_v.head + e0) = raw[i];
                    continue;
                }
                float x[VE], z[VE];
                unpack<T>(raw[i], x);
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
                if (APPEND && kind == 1) {
                    if (page_k) store_vec_t(page_k + h * a.cache_k.head + e0, z);
                } else {
                    store_row<T, VEC, VE>(row_at<T, VEC>(kind == 0 ? a.q_out : a.k_out, b, t, h) + e0, z);
                }
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

namespace {
template <typename T, int K> int cut(HeadsArgs &a, bool backward) {
    const HeadsPlan h = heads_plan(a.tokens, a.Hq, a.Hk, K, sizeof(T) == 2, a.append, backward);
    a.q_blocks = h.q_blocks; a.k_blocks = h.k_blocks; a.blocks = h.blocks; a.parts = h.parts; a.per_part = h.per_part;
    return h.workgroups;
}
template <typename T, int K, bool VEC, int ROT> void fwd_of(HeadsArgs a, hipStream_t st) {
    const dim3 g((unsigned)cut<T, K>(a, false)), t(HEADS_T);
    if (!a.append) hipLaunchKernelGGL((heads_fwd_kernel<T, K, VEC, ROT, false, false>), g, t, 0, st, a);
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

int launch_heads_fwd(const HeadsArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? by_width<bf16>(a, false, st) : by_width<float>(a, false, st); }
int launch_heads_bwd(const HeadsArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? by_width<bf16>(a, true, st) : by_width<float>(a, true, st); }

}  // namespace osdn
