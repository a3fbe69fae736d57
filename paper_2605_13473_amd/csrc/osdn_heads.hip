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
// in K * sizeof(T) / 16 lanes, 64 lanes in as many rows as that makes (a block of rows).
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

// The rotation of a lane's elements: z = x c + partner s (transposed: x c - partner s).  A lane that holds no pair leaves them alone.
template <typename T, int K> struct Turn {
    static constexpr int VE = HeadRow<T, K>::VE;
    float c[VE], s[VE];
    int from;                       // the lane that holds the partners, times 4 (adjacent pairs: this one)
    bool on;
    __device__ __forceinline__ void load(const float *row, int R, bool interleaved, int lane) {
        const int l = lane & (HeadRow<T, K>::LANES - 1), e0 = l * VE, half = R / 2;
        on = e0 < R;
        const bool low = e0 < half;
        const int i0 = !on ? 0 : interleaved ? e0 / 2 : low ? e0 : e0 - half;
        from = 4 * (!on || interleaved ? lane : low ? lane + half / VE : lane - half / VE);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const int i = i0 + (interleaved ? e / 2 : e);
            c[e] = row[i];
            const float sn = row[half + i];
            s[e] = (interleaved ? (e & 1) == 0 : low) ? -sn : sn;
        }
    }
    // the partners of a lane's elements (every lane of the wavefront calls it)
    __device__ __forceinline__ u32x4 partners(const u32x4 &raw, bool interleaved) const {
        u32x4 o;
        if (interleaved) {
#pragma unroll
            for (int w = 0; w < 4; ++w) o[w] = sizeof(T) == 2 ? (raw[w] >> 16) | (raw[w] << 16) : raw[w ^ 1];
        } else {
#pragma unroll
            for (int w = 0; w < 4; ++w) o[w] = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)raw[w]);
        }
        return o;
    }
};

// Where a token's rows are and what becomes of them: -1 none (its outputs are zero), else its position
__device__ __forceinline__ int token_position(const HeadsArgs &a, int t, size_t n) { return a.positions ? a.positions[n] : t; }

template <typename T, bool VEC> __device__ __forceinline__ T *row_at(const HeadRows &r, int b, int t, int h) {
    return static_cast<T *>(r.data) + b * r.batch + t * r.token + h * r.head;
}

// NB blocks of rows per wavefront.  APPEND: keys go to the cache, values follow them unchanged.
template <typename T, int K, bool VEC, bool ROT, int NB, bool APPEND>
__global__ __launch_bounds__(HEADS_T) void heads_fwd_kernel(HeadsArgs a) {
    using HR = HeadRow<T, K>;
    constexpr int VE = HR::VE, ROWS = HR::ROWS;
    const int lane = threadIdx.x & 63, sub = lane / HR::LANES, e0 = (lane % HR::LANES) * VE;
    const unsigned item = __builtin_amdgcn_readfirstlane(blockIdx.x * (HEADS_T / 64) + (threadIdx.x >> 6));
    const unsigned token = item / (unsigned)a.parts + blockIdx.y * (unsigned)a.tokens_y;
    const int part = item % (unsigned)a.parts;
    if (token >= (unsigned)a.tokens || item / (unsigned)a.parts >= (unsigned)a.tokens_y) return;
    const int b = token / (unsigned)a.T, t = token % (unsigned)a.T;

    // a block of rows: 0 queries, 1 keys, 2 values
    int kind[NB], h[NB];
    bool live[NB];
    u32x4 raw[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int blk = part * NB + i;
        kind[i] = blk < a.q_blocks ? 0 : blk < a.q_blocks + a.k_blocks ? 1 : 2;
        const int first = kind[i] == 0 ? 0 : kind[i] == 1 ? a.q_blocks : a.q_blocks + a.k_blocks;
        h[i] = (blk - first) * ROWS + sub;
        live[i] = blk < a.blocks && h[i] < (kind[i] == 0 ? a.Hq : a.Hk);
        const HeadRows &src = kind[i] == 0 ? a.q : kind[i] == 1 ? a.k : a.v;
        raw[i] = u32x4{0u, 0u, 0u, 0u};
        if (live[i]) raw[i] = load_row<T, VEC>(row_at<const T, VEC>(src, b, t, h[i]) + e0);
    }
    const int pos = token_position(a, t, token);
    const bool none = pos < 0;
    const bool off_table = ROT && pos >= a.rotary_rows;
    Turn<T, K> turn;
    if constexpr (ROT) turn.load(a.rotary + (size_t)(none || off_table ? 0 : pos) * a.rotary_dim, a.rotary_dim, a.interleaved, lane);
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
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        if (part * NB + i >= a.blocks) break;
        if (APPEND && kind[i] == 2) {
            if (live[i] && page_v) {
                T *dst = page_v + h[i] * a.cache_v.head + e0;
                *reinterpret_cast<u32x4 *>(dst) = raw[i];
            }
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
        const float *w = kind[i] == 0 ? a.weight_q : a.weight_k;
#pragma unroll
        for (int e = 0; e < VE; ++e) z[e] = x[e] * r;
        if (w) {
#pragma unroll
            for (int e = 0; e < VE; ++e) z[e] *= w[e0 + e];
        }
        if constexpr (ROT) {
            float y[VE];
            unpack<T>(turn.partners(raw[i], a.interleaved), y);
            const int from = a.interleaved ? e0 : (turn.from / 4 % HR::LANES) * VE;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                float yp = y[e] * r;
                if (w) yp *= w[from + (a.interleaved ? e ^ 1 : e)];
                const float turned = __builtin_fmaf(z[e], turn.c[e], yp * turn.s[e]);
                z[e] = turn.on ? turned : z[e];
            }
        }
        if (!live[i]) continue;
        if (none) {
#pragma unroll
            for (int e = 0; e < VE; ++e) z[e] = 0.f;
        }
        if (APPEND && kind[i] == 1) {
            if (page_k) store_vec_t(page_k + h[i] * a.cache_k.head + e0, z);
        } else {
            store_row<T, VEC, VE>(row_at<T, VEC>(kind[i] == 0 ? a.q_out : a.k_out, b, t, h[i]) + e0, z);
        }
    }
}

// Backward: a workgroup walks tokens in steps of the grid, so that the sums over rows of dw stay in registers until its end; its
// partial sums go to a row of `partial` [gridDim.x][2][K], which heads_dw_kernel adds up in a fixed order.
template <typename T, int K, bool VEC, bool ROT>
__global__ __launch_bounds__(HEADS_T) void heads_bwd_kernel(HeadsArgs a) {
    using HR = HeadRow<T, K>;
    constexpr int VE = HR::VE, ROWS = HR::ROWS, WAVES = HEADS_T / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane / HR::LANES, e0 = (lane % HR::LANES) * VE;
    float dw[2][VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) dw[0][e] = dw[1][e] = 0.f;

    for (unsigned token = __builtin_amdgcn_readfirstlane(blockIdx.x * WAVES + wave); token < (unsigned)a.tokens; token += gridDim.x * WAVES) {
        const int b = token / (unsigned)a.T, t = token % (unsigned)a.T;
        const int pos = token_position(a, t, token);
        const bool none = pos < 0;
        const bool off_table = ROT && pos >= a.rotary_rows;
        Turn<T, K> turn;
        if constexpr (ROT) turn.load(a.rotary + (size_t)(none || off_table ? 0 : pos) * a.rotary_dim, a.rotary_dim, a.interleaved, lane);
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {
            const HeadRows &xs = kind == 0 ? a.q : a.k, &zs = kind == 0 ? a.dq_out : a.dk_out, &ds = kind == 0 ? a.dq : a.dk;
            const int H = kind == 0 ? a.Hq : a.Hk;
            const float *w = kind == 0 ? a.weight_q : a.weight_k;
            for (int h0 = 0; h0 < H; h0 += ROWS) {
                const int h = h0 + sub;
                const bool live = h < H;
                u32x4 rx = {0u, 0u, 0u, 0u}, rz = {0u, 0u, 0u, 0u};
                if (live) {
                    rx = load_row<T, VEC>(row_at<const T, VEC>(xs, b, t, h) + e0);
                    rz = load_row<T, VEC>(row_at<const T, VEC>(zs, b, t, h) + e0);
                }
                float x[VE], dy[VE], g[VE];
                unpack<T>(rx, x);
                unpack<T>(rz, dy);
                if constexpr (ROT) {
                    float p[VE];
                    unpack<T>(turn.partners(rz, a.interleaved), p);
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        const float turned = __builtin_fmaf(dy[e], turn.c[e], -(p[e] * turn.s[e]));
                        dy[e] = turn.on ? turned : dy[e];
                    }
                }
                float r = 1.f, ss = 0.f, gx = 0.f;
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    g[e] = w ? dy[e] * w[e0 + e] : dy[e];
                    ss = __builtin_fmaf(x[e], x[e], ss);
                    gx = __builtin_fmaf(g[e], x[e], gx);
                }
                if (a.norm != 0) {
                    r = rsqrtf(__builtin_fmaf(row_sum<HR::LANES>(ss), a.mean, a.eps));
                    gx = row_sum<HR::LANES>(gx) * (r * r * a.mean);
                } else {
                    gx = 0.f;
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
                    dx[e] = r * __builtin_fmaf(-gx, x[e], g[e]);
                    dw[kind][e] = __builtin_fmaf(dy[e] * r, x[e], dw[kind][e]);
                }
                if (live) store_row<T, VEC, VE>(row_at<T, VEC>(ds, b, t, h) + e0, dx);
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
    __shared__ float s[DW_ROWS][DW_COLS + 1];
    const int col = threadIdx.x % DW_COLS, row = threadIdx.x / DW_COLS, c = blockIdx.x * DW_COLS + col;
    float v = 0.f;
    for (int i = row; i < n; i += DW_ROWS) v += partial[(size_t)i * 2 * K + c];
    s[row][col] = v;
    __syncthreads();
    if (row == 0) {
        v = 0.f;
        for (int i = 0; i < DW_ROWS; ++i) v += s[i][col];
        float *dst = c < K ? dwq : dwk;
        if (dst) dst[c < K ? c : c - K] = v;
    }
}

namespace {
template <typename T, int K, bool VEC, bool ROT> void fwd_parts(HeadsArgs &a, int nb, hipStream_t st) {
    auto go = [&](auto kernel, int n) {
        a.parts = (a.blocks + n - 1) / n;
        // (a grid has fewer than 2^32 threads along x: more tokens than that go along y)
        const long long most = (1ll << 25) / a.parts, rows = a.tokens < most ? a.tokens : most;
        a.tokens_y = (int)rows;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((rows * a.parts + HEADS_T / 64 - 1) / (HEADS_T / 64)), (unsigned)((a.tokens + rows - 1) / rows)), dim3(HEADS_T), 0, st, a);
    };
    if (a.append) {
        if (VEC && nb > 1) go(heads_fwd_kernel<T, K, VEC, ROT, VEC ? 4 : 1, true>, 4);
        else go(heads_fwd_kernel<T, K, VEC, ROT, 1, true>, 1);
    } else {
        if (VEC && nb > 1) go(heads_fwd_kernel<T, K, VEC, ROT, VEC ? 4 : 1, false>, 4);
        else go(heads_fwd_kernel<T, K, VEC, ROT, 1, false>, 1);
    }
}
template <typename T, int K> void set_blocks(HeadsArgs &a) {
    constexpr int ROWS = HeadRow<T, K>::ROWS;
    a.q_blocks = (a.Hq + ROWS - 1) / ROWS;
    a.k_blocks = (a.Hk + ROWS - 1) / ROWS;
    a.blocks = a.q_blocks + a.k_blocks * (a.append ? 2 : 1);
}
template <typename T, int K> void fwd_of(HeadsArgs &a, hipStream_t st) {
    set_blocks<T, K>(a);
    const int nb = heads_blocks_per_wave(a.tokens, a.blocks);
    if (a.aligned) a.rotary ? fwd_parts<T, K, true, true>(a, nb, st) : fwd_parts<T, K, true, false>(a, nb, st);
    else a.rotary ? fwd_parts<T, K, false, true>(a, nb, st) : fwd_parts<T, K, false, false>(a, nb, st);
}
template <typename T, int K> void bwd_of(HeadsArgs &a, hipStream_t st) {
    const dim3 g((unsigned)heads_bwd_workgroups(a.tokens)), t(HEADS_T);
    if (a.aligned) {
        if (a.rotary) hipLaunchKernelGGL((heads_bwd_kernel<T, K, true, true>), g, t, 0, st, a);
        else hipLaunchKernelGGL((heads_bwd_kernel<T, K, true, false>), g, t, 0, st, a);
    } else {
        if (a.rotary) hipLaunchKernelGGL((heads_bwd_kernel<T, K, false, true>), g, t, 0, st, a);
        else hipLaunchKernelGGL((heads_bwd_kernel<T, K, false, false>), g, t, 0, st, a);
    }
    if (a.partial)
        hipLaunchKernelGGL(heads_dw_kernel, dim3(2 * K / DW_COLS), dim3(DW_T), 0, st, a.partial, (int)g.x, K, a.dweight_q, a.dweight_k);
}
template <typename F> int by_width(int K, bool bf16_io, F &&f) {
    switch (K) {
        case 64: bf16_io ? f(bf16{}, std::integral_constant<int, 64>{}) : f(float{}, std::integral_constant<int, 64>{}); return 0;
        case 128: bf16_io ? f(bf16{}, std::integral_constant<int, 128>{}) : f(float{}, std::integral_constant<int, 128>{}); return 0;
        case 256: bf16_io ? f(bf16{}, std::integral_constant<int, 256>{}) : f(float{}, std::integral_constant<int, 256>{}); return 0;
        default: return -1;
    }
}
}  // namespace

int launch_heads_fwd(HeadsArgs a, bool bf16_io, hipStream_t st) {
    return by_width(a.K, bf16_io, [&](auto t, auto k) { fwd_of<decltype(t), decltype(k)::value>(a, st); });
}
int launch_heads_bwd(HeadsArgs a, bool bf16_io, hipStream_t st) {
    return by_width(a.K, bf16_io, [&](auto t, auto k) { bwd_of<decltype(t), decltype(k)::value>(a, st); });
}

}  // namespace osdn
