// The pages of a cache: which of them the tokens of a batch of requests go to, and which of them a query reads.
//
//  plan      request b of a batch brings f_b new tokens to a sequence that has c_b.  It needs ceil((c_b + f_b) / P) - ceil(c_b / P) pages of P tokens, which it
//            takes off a list of free ones; token j of the f_b stands at position c_b + j.  Running sums over the batch say who is served and where
//            each request's pages and tokens begin.
//  release   the pages of sequences that end go back onto the list.
//  bounds    for each page, head and element the smallest and the largest of its keys, lo and hi.
//  select    sum_i max(q_i lo_i, q_i hi_i) is no smaller than <q, k> for every key of a page.  Summed over the query heads that share the keys it is
//            <Q-, lo> + <Q+, hi>  with  Q- = sum of min(q, 0), Q+ = sum of max(q, 0):
//            one row of 2 K products per page and key head, however many query heads there are.  The pages of the largest sums are taken.
//
// plan and release are bound by the launch (a few KB); a workgroup of 16 wavefronts holds the running sums.  bounds is bound by the rows it reads, select by
// the bounds.  Sums of select are in 64 bits: the products of bf16 numbers are exact there and so, but for a spread of more than
// 2^25 between them, are their sums, so that which page wins does not hang on their order.
#include "osdn_kernels.h"
#include "osdn_plan.h"

namespace osdn {

constexpr int PLAN_T = 1024, PLAN_W = PLAN_T / 64;

__device__ __forceinline__ unsigned add_sat(unsigned a, unsigned b) { return __builtin_elementwise_add_sat(a, b); }

// Sums over the threads of a workgroup, each with its own and those before it; saturating.  `all`: the sum over all threads.
struct TwoSums { unsigned a, b; };
__device__ __forceinline__ TwoSums running_sums(TwoSums x, TwoSums &all, unsigned (&part)[PLAN_W][2], int lane, int wave) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const unsigned a = __shfl_up(x.a, d, 64), b = __shfl_up(x.b, d, 64);
        if (lane >= d) { x.a = add_sat(x.a, a); x.b = add_sat(x.b, b); }
    }
    __syncthreads();                    // (what stands in `part` has been read)
    if (lane == 63) { part[wave][0] = x.a; part[wave][1] = x.b; }
    __syncthreads();
    all = {0u, 0u};
    TwoSums before{0u, 0u};
#pragma unroll
    for (int w = 0; w < PLAN_W; ++w) {
        if (w == wave) before = all;
        all.a = add_sat(all.a, part[w][0]);
        all.b = add_sat(all.b, part[w][1]);
    }
    return {add_sat(x.a, before.a), add_sat(x.b, before.b)};
}

// Rows that two requests name: a bit for a row that is named, another for one that is named again
__device__ __forceinline__ void note_rows(unsigned *bits, int words, int n_seqs, int B, const int *seq, const int *asks) {
    for (int i = threadIdx.x; i < 2 * words; i += PLAN_T) bits[i] = 0u;
    __syncthreads();
    for (int b = threadIdx.x; b < B; b += PLAN_T) {
        const int s = seq[b];
        if ((unsigned)s >= (unsigned)n_seqs || asks[b] <= 0) continue;
        const unsigned bit = 1u << (s & 31);
        if (atomicOr(&bits[s >> 5], bit) & bit) atomicOr(&bits[words + (s >> 5)], bit);
    }
    __syncthreads();
}

struct Request { int row, first, need, cached, fresh; unsigned pages_before; };

// The pages of a request into its row of the table: its i-th is the (pages_before + i)-th from the top of the list
__device__ __forceinline__ int granted(const PlanArgs &a, int have, unsigned place) { return a.free_list[have - 1 - (int)place]; }

// What lanes [0, n) of the request of lane `src` do, for the requests of a wavefront one after the other
template <typename F> __device__ __forceinline__ void each_request(unsigned long long who, F &&f) {
    while (who) {
        const int src = __builtin_ctzll(who);
        who &= who - 1;
        f(src);
    }
}

// (a page that is not there has no slots)
__device__ __forceinline__ void leave_token(const PlanArgs &a, int at, int pos, int row, int page) {
    a.positions[at] = pos;
    a.rows[at] = row;
    if (a.slots) a.slots[at] = (unsigned)page < (unsigned)a.n_pages ? ((long long)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : -1;
}

// TOKENS: also the tokens' places (else plan_tokens_kernel, for many)
template <bool TOKENS> __global__ __launch_bounds__(PLAN_T) void plan_kernel(PlanArgs a) {
    extern __shared__ unsigned bits[];
    __shared__ unsigned part[PLAN_W][2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), words = (a.n_seqs + 31) / 32;
    const int P = 1 << a.page_shift;
    const long long capacity = (long long)a.max_pages << a.page_shift;
    const int have = max(0, min(*a.n_free, a.free_capacity));
    if (a.seq) note_rows(bits, words, a.n_seqs, a.B, a.seq, a.fresh);
    TwoSums asked{0u, 0u}, given{0u, 0u};           // of the requests before this round's: pages and tokens, asked for and given
    for (int b0 = 0; b0 < a.B; b0 += PLAN_T) {
        const int b = b0 + (int)threadIdx.x;
        Request r{};
        bool valid = false;
        if (b < a.B) {
            r.row = a.seq ? a.seq[b] : b;
            r.cached = a.cached[b];
            r.fresh = a.fresh[b];
            const bool known = (unsigned)r.row < (unsigned)a.n_seqs;
            const bool twice = a.seq && known && r.fresh > 0 && (bits[words + (r.row >> 5)] >> (r.row & 31) & 1u);
            valid = known && !twice && r.cached >= 0 && r.fresh >= 0 && (long long)r.cached + r.fresh <= capacity;
            if (!known || r.cached < 0) r.cached = 0;
            if (!valid) r.fresh = 0;
            r.first = (int)(((long long)r.cached + P - 1) >> a.page_shift);
            r.need = valid ? (int)(((long long)r.cached + r.fresh + P - 1) >> a.page_shift) - r.first : 0;
        }
        TwoSums all;
        TwoSums upto = running_sums({(unsigned)r.need, (unsigned)r.fresh}, all, part, lane, wave);
        const bool served = (r.need == 0 || add_sat(asked.a, upto.a) <= (unsigned)have) && (r.fresh == 0 || add_sat(asked.b, upto.b) <= (unsigned)a.N);
        asked = {add_sat(asked.a, all.a), add_sat(asked.b, all.b)};
        if (!served) r.need = r.fresh = 0;
        if (__syncthreads_or(!served)) upto = running_sums({(unsigned)r.need, (unsigned)r.fresh}, all, part, lane, wave);
        r.pages_before = given.a + upto.a - r.need;
        const int start = (int)(given.b + upto.b) - r.fresh;
        given = {given.a + all.a, given.b + all.b};
        if (b < a.B) {
            a.lengths[b] = r.cached + r.fresh;
            a.starts[b] = start;
            if (b == a.B - 1) a.starts[a.B] = start + r.fresh;
        }
        // pages: one or two by the request's lane, more by the whole wavefront
        int *row = a.table + (long long)r.row * a.table_stride;
        int page0 = -1;
        if (r.need > 0) page0 = granted(a, have, r.pages_before);
        if (r.need > 0 && r.need <= 2) {
            row[r.first] = page0;
            if (r.need == 2) row[r.first + 1] = granted(a, have, r.pages_before + 1);
        }
        each_request(__ballot(r.need > 2), [&](int src) {
            int *to = a.table + (long long)__shfl(r.row, src, 64) * a.table_stride + __shfl(r.first, src, 64);
            const int n = __shfl(r.need, src, 64);
            const unsigned from = __shfl(r.pages_before, src, 64);
            for (int i = lane; i < n; i += 64) to[i] = granted(a, have, from + i);
        });
        if constexpr (TOKENS) {
            if (r.fresh == 1) {
                const int col = r.cached >> a.page_shift, page = r.need ? page0 : a.slots ? row[col] : 0;
                leave_token(a, start, r.cached, r.row, page);
            }
            each_request(__ballot(r.fresh > 1), [&](int src) {
                const int R = __shfl(r.row, src, 64), n = __shfl(r.fresh, src, 64), c = __shfl(r.cached, src, 64), first = __shfl(r.first, src, 64), at = __shfl(start, src, 64);
                const unsigned from = __shfl(r.pages_before, src, 64);
                for (int i = lane; i < n; i += 64) {
                    const int pos = c + i, col = pos >> a.page_shift;
                    int page = 0;
                    if (a.slots) page = col < first ? a.table[(long long)R * a.table_stride + col] : granted(a, have, from + col - first);
                    leave_token(a, at + i, pos, R, page);
                }
            });
        }
    }
    if constexpr (TOKENS)
        for (int i = (int)given.b + (int)threadIdx.x; i < a.N; i += PLAN_T) leave_token(a, i, -1, -1, -1);
    if (threadIdx.x == 0) *a.n_free_out = have - (int)given.a;
}

// Places of many tokens, behind plan_kernel<false>: a token finds its request in the requests' starts
__global__ __launch_bounds__(256) void plan_tokens_kernel(PlanArgs a) {
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= a.N) return;
    if (j >= a.starts[a.B]) return leave_token(a, j, -1, -1, -1);
    int lo = 0, hi = a.B;                       // starts[lo] <= j < starts[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.starts[mid] <= j) lo = mid;
        else hi = mid;
    }
    const int row = a.seq ? a.seq[lo] : lo, pos = a.lengths[lo] - (a.starts[lo + 1] - j);
    const int page = a.slots ? a.table[(long long)row * a.table_stride + (pos >> a.page_shift)] : 0;
    leave_token(a, j, pos, row, page);
}

// The i-th page that is given back, of R in the order of the requests and of their pages, lands R - 1 - i above what the list holds, so that the next requests
// take them in that order again.  A wavefront takes a request: it counts its pages, and, once it is known how many come before them, moves them.
__global__ __launch_bounds__(PLAN_T) void release_kernel(PlanArgs a) {
    extern __shared__ unsigned bits[];
    __shared__ unsigned count[PLAN_T], before[PLAN_T], part[PLAN_W][2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), words = (a.n_seqs + 31) / 32;
    const int have = max(0, min(*a.n_free, a.free_capacity));
    if (a.seq) note_rows(bits, words, a.n_seqs, a.B, a.seq, a.cached);
    // columns of the table that request b holds; none where there is nothing to give back
    auto held = [&](int b, int &row) {
        row = a.seq ? a.seq[b] : b;
        const int n = a.cached[b];
        if ((unsigned)row >= (unsigned)a.n_seqs || n <= 0 || (a.seq && (bits[words + (row >> 5)] >> (row & 31) & 1u))) return 0;
        return (int)min((long long)a.max_pages, ((long long)n + (1 << a.page_shift) - 1) >> a.page_shift);
    };
    auto pages_of = [&](int b) {
        int row;
        const int cols = held(b, row);
        const int *from = a.table + (cols ? (long long)row * a.table_stride : 0);
        int n = 0;
        for (int i = 0; i < cols; i += 64) n += __builtin_popcountll(__ballot(i + lane < cols && (unsigned)from[min(i + lane, cols - 1)] < (unsigned)a.n_pages));
        return n;
    };
    auto count_round = [&](int b0) {
        __syncthreads();
        count[threadIdx.x] = 0;
        __syncthreads();
        for (int i = wave; i < PLAN_T && b0 + i < a.B; i += PLAN_W) {
            const int n = pages_of(b0 + i);
            if (lane == 0) count[i] = n;
        }
        __syncthreads();
    };
    unsigned total = 0;
    for (int b0 = 0; b0 < a.B; b0 += PLAN_T) {
        count_round(b0);
        TwoSums all;
        running_sums({count[threadIdx.x], 0u}, all, part, lane, wave);
        total += all.a;
    }
    unsigned done = 0;
    for (int b0 = 0; b0 < a.B; b0 += PLAN_T) {
        if (a.B > PLAN_T) count_round(b0);      // (else they are still there)
        TwoSums all;
        const TwoSums upto = running_sums({count[threadIdx.x], 0u}, all, part, lane, wave);
        before[threadIdx.x] = done + upto.a - count[threadIdx.x];
        __syncthreads();
        for (int i = wave; i < PLAN_T && b0 + i < a.B; i += PLAN_W) {
            int row;
            const int cols = held(b0 + i, row);
            int *from = a.table + (cols ? (long long)row * a.table_stride : 0);
            unsigned at = before[i];
            for (int c = 0; c < cols; c += 64) {
                const bool in = c + lane < cols;
                const int page = in ? from[c + lane] : -1;
                const bool there = (unsigned)page < (unsigned)a.n_pages;
                const unsigned long long who = __ballot(there);
                const long long to = (long long)have + total - 1 - (at + __builtin_popcountll(who & ((1ull << lane) - 1)));
                if (there && to < a.free_capacity) a.free_list[to] = page;
                if (in) from[c + lane] = -1;
                at += __builtin_popcountll(who);
            }
        }
        done += all.a;
    }
    if (threadIdx.x == 0) *a.n_free_out = (int)min((long long)a.free_capacity, (long long)have + total);
}

int launch_plan(const PlanArgs &a, hipStream_t st) {
    const size_t lds = a.seq ? (size_t)((a.n_seqs + 31) / 32) * 8 : 0;
    if (a.N <= PLAN_TOKENS_HERE) {
        hipLaunchKernelGGL(plan_kernel<true>, dim3(1), dim3(PLAN_T), lds, st, a);
    } else {
        hipLaunchKernelGGL(plan_kernel<false>, dim3(1), dim3(PLAN_T), lds, st, a);
        hipLaunchKernelGGL(plan_tokens_kernel, dim3(((unsigned)a.N + 255) / 256), dim3(256), 0, st, a);
    }
    return 0;
}
int launch_release(const PlanArgs &a, hipStream_t st) {
    const size_t lds = a.seq ? (size_t)((a.n_seqs + 31) / 32) * 8 : 0;
    hipLaunchKernelGGL(release_kernel, dim3(1), dim3(PLAN_T), lds, st, a);
    return 0;
}

// ---- bounds ------------------------------------------------------------------------------------

// A lane's 16 bytes of a row (4-bit rows: 8 elements) as floats
template <typename T, int K, bool MX> struct KeyRow {
    static constexpr int VE = MX ? 8 : 16 / (int)sizeof(T), LANES = K / VE;
    static __device__ __forceinline__ void load(const BoundsArgs &a, long long page, int slot, int h, int e0, float (&x)[VE]) {
        if constexpr (MX) {
            const char *codes = static_cast<const char *>(a.keys.data) + page * a.keys.batch + slot * a.keys.token + h * a.keys.head + e0 / 2;
            const unsigned char *scale = static_cast<const unsigned char *>(a.scales.data) + page * a.scales.batch + slot * a.scales.token + h * a.scales.head + e0 / 32;
            fp4_values(*reinterpret_cast<const uint32_t *>(codes), fp4_scale(*scale), x);
        } else {
            const u32x4 raw = *reinterpret_cast<const u32x4 *>(static_cast<const T *>(a.keys.data) + page * a.keys.batch + slot * a.keys.token + h * a.keys.head + e0);
#pragma unroll
            for (int e = 0; e < VE; ++e) x[e] = vec_get<T>(raw, e);
        }
    }
};
// (a NaN stays one)
__device__ __forceinline__ float least(float x, float y) { return __builtin_elementwise_minimum(x, y); }
__device__ __forceinline__ float greatest(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// A wavefront takes one page that got new tokens, for one head: its new rows, 64 / LANES at a time, and, where it had tokens before, its bounds.
template <typename T, int K, bool MX> __global__ __launch_bounds__(256) void bounds_kernel(BoundsArgs a) {
    using R = KeyRow<T, K, MX>;
    constexpr int VE = R::VE, ROWS = 64 / R::LANES;
    const int lane = threadIdx.x & 63, sub = lane / R::LANES, e0 = lane % R::LANES * VE;
    const long long item = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = (int)(item % a.Hk);
    const long long rest = item / a.Hk;
    const int nth = (int)(rest % a.touched);
    if (rest / a.touched >= a.B) return;
    const int b = (int)(rest / a.touched);
    const int from = max(0, a.cached[b]), end = (int)min((long long)a.lengths[b], (long long)from + a.max_new), row = a.seq ? a.seq[b] : b;
    const int col = (from >> a.page_shift) + nth;
    const long long begin = (long long)col << a.page_shift;
    if (begin >= end || from >= end || col >= a.max_pages || (unsigned)row >= (unsigned)a.n_seqs) return;
    const int page = a.table[(long long)row * a.table_stride + col];
    if ((unsigned)page >= (unsigned)a.n_pages) return;
    const int s0 = (int)(max((long long)from, begin) - begin), s1 = (int)min((long long)1 << a.page_shift, end - begin);
    T *out = static_cast<T *>(a.bounds) + ((long long)page * a.Hk + h) * 2 * K + e0;
    float lo[VE], hi[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
    if (s0 > 0) {                       // (tokens from before)
#pragma unroll
        for (int e = 0; e < VE; ++e) { lo[e] = to_f32(out[e]); hi[e] = to_f32(out[K + e]); }
    }
    for (int s = s0 + sub; s < s1; s += ROWS) {
        float x[VE];
        R::load(a, page, s, h, e0, x);
#pragma unroll
        for (int e = 0; e < VE; ++e) { lo[e] = least(lo[e], x[e]); hi[e] = greatest(hi[e], x[e]); }
    }
#pragma unroll
    for (int d = R::LANES; d < 64; d <<= 1)
#pragma unroll
        for (int e = 0; e < VE; ++e) { lo[e] = least(lo[e], __shfl_xor(lo[e], d, 64)); hi[e] = greatest(hi[e], __shfl_xor(hi[e], d, 64)); }
    if (sub == 0) {
#pragma unroll
        for (int e = 0; e < VE; ++e) { out[e] = from_f32<T>(lo[e]); out[K + e] = from_f32<T>(hi[e]); }
    }
}

// ---- select ------------------------------------------------------------------------------------

// Scores as 64-bit integers in the same order; what is not a number comes first of all, before infinity
__device__ __forceinline__ unsigned long long score_key(double s) {
    if (s != s) return ~0ull;
    const unsigned long long u = __builtin_bit_cast(unsigned long long, s + 0.0);           // (no negative zero)
    return u >> 63 ? ~u : u | 1ull << 63;
}

// The first lanes of a row of 2 K bounds hold the smallest, the rest the largest; a lane holds VPL vectors of VE.  A wavefront takes `HEADS` key heads next to
// each other and walks pages in steps.
template <typename T, int K> struct ScoreRow {
    static constexpr int VE = 16 / sizeof(T), ALL = 2 * K / VE, LANES = ALL < 64 ? ALL : 64, VPL = ALL / LANES, HEADS = 64 / LANES;
};
__device__ __forceinline__ double lane_sum(double x, int lanes) {
    for (int d = 1; d < lanes; d <<= 1) x += __shfl_xor(x, d, 64);
    return x;
}
__device__ __forceinline__ Seen pages_seen(const SelectArgs &a, int b) {
    return seen_tokens(a.lengths[b], a.seq ? a.seq[b] : b, a.n_seqs, a.max_length, 0, a.page_shift, a.max_pages);
}

template <typename T, int K> __global__ __launch_bounds__(256) void score_kernel(SelectArgs a) {
    using R = ScoreRow<T, K>;
    constexpr int VE = R::VE, VPL = R::VPL;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.y, h0 = (int)blockIdx.z * R::HEADS, h = h0 + lane / R::LANES;
    const Seen see = pages_seen(a, b);
    const int have = (see.end + (1 << a.page_shift) - 1) >> a.page_shift;
    if (have <= a.pages) return;                        // (all of them are taken)
    const int row = a.seq ? a.seq[b] : b, end = have - a.last;
    const int stride = gridDim.x * 4, hh = min(h, a.Hk - 1);
    // the weights of a lane's elements: sums of the negative (smallest) or positive (largest) parts of the queries
    double w[VPL][VE];
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
        const int at = (lane % R::LANES + v * R::LANES) * VE;
        const bool low = at < K;
#pragma unroll
        for (int e = 0; e < VE; ++e) w[v][e] = 0.0;
        for (int i = 0; i < a.group; ++i) {
            const T *q = static_cast<const T *>(a.q.data) + b * a.q.batch + (long long)(hh * a.group + i) * a.q.head + at % K;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float x = to_f32(q[e]);
                w[v][e] += (double)(low ? __builtin_elementwise_minimum(x, 0.f) : __builtin_elementwise_maximum(x, 0.f));
            }
        }
    }
    unsigned long long *keys = a.keys + ((long long)b * a.Hk + hh) * a.max_pages_seen;
    const int *table = a.table + (long long)row * a.table_stride;
    for (int p = a.first + blockIdx.x * 4 + wave; p < end; p += stride) {
        const int page = table[p];
        const bool there = (unsigned)page < (unsigned)a.n_pages;
        const T *from = static_cast<const T *>(a.bounds) + ((long long)(there ? page : 0) * a.Hk + hh) * 2 * K + lane % R::LANES * VE;
        double s = 0.0;
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            const u32x4 raw = *reinterpret_cast<const u32x4 *>(from + v * R::LANES * VE);
#pragma unroll
            for (int e = 0; e < VE; ++e) s = __builtin_fma(w[v][e], (double)vec_get<T>(raw, e), s);
        }
        s = lane_sum(s, R::LANES);
        if (lane % R::LANES == 0 && h < a.Hk) keys[p] = there ? score_key(s) : ~0ull;
    }
}

// A workgroup takes the pages of one sequence and key head.  The n-th largest key: the keys between the bounds known so far are counted in
// 2048 even bins, the bin that holds it gives the next bounds, until all of a bin is taken or it is one key wide.
constexpr int SEL_T = 1024, SEL_W = SEL_T / 64, SEL_BINS = 2048;
__global__ __launch_bounds__(SEL_T) void select_kernel(SelectArgs a) {
    __shared__ unsigned bins[SEL_BINS], part[SEL_W];
    __shared__ unsigned long long edge[SEL_W][2];
    __shared__ unsigned found[3];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = blockIdx.x / (unsigned)a.Hk, h = blockIdx.x % (unsigned)a.Hk;
    const Seen see = pages_seen(a, b);
    const int have = (see.end + (1 << a.page_shift) - 1) >> a.page_shift, row = a.seq ? a.seq[b] : b;
    int *out = a.chosen + (long long)blockIdx.x * a.pages;
    const int n = min(have, a.pages);
    if (threadIdx.x == 0) a.tokens[blockIdx.x] = see.broken ? 0x7fffffff : have ? ((n - 1) << a.page_shift) + ((see.end - 1) & ((1 << a.page_shift) - 1)) + 1 : 0;
    for (int i = n + threadIdx.x; i < a.pages; i += SEL_T) out[i] = -1;
    if (have == 0) return;
    const int *table = a.table + (long long)row * a.table_stride;
    auto leave = [&](int place, int p) {
        const int page = table[p];
        out[place] = (unsigned)page < (unsigned)a.n_pages ? page : -1;
    };
    if (have <= a.pages) {
        for (int i = threadIdx.x; i < have; i += SEL_T) leave(i, i);
        return;
    }
    for (int i = threadIdx.x; i < a.first; i += SEL_T) leave(i, i);
    for (int i = threadIdx.x; i < a.last; i += SEL_T) leave(a.pages - a.last + i, have - a.last + i);
    const unsigned long long *keys = a.keys + (long long)blockIdx.x * a.max_pages_seen;
    const int begin = a.first, end = have - a.last;
    unsigned need = a.pages - a.first - a.last;         // of the keys in [begin, end), which are more
    if (need == 0) return;
    unsigned long long lo = ~0ull, hi = 0;
    for (int i = begin + threadIdx.x; i < end; i += SEL_T) {
        const unsigned long long k = keys[i];
        lo = k < lo ? k : lo;
        hi = k > hi ? k : hi;
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const unsigned long long x = __shfl_xor(lo, d, 64), y = __shfl_xor(hi, d, 64);
        lo = x < lo ? x : lo;
        hi = y > hi ? y : hi;
    }
    if (lane == 0) { edge[wave][0] = lo; edge[wave][1] = hi; }
    __syncthreads();
    for (int w = 0; w < SEL_W; ++w) {
        lo = edge[w][0] < lo ? edge[w][0] : lo;
        hi = edge[w][1] > hi ? edge[w][1] : hi;
    }
    // keys of [lo, hi]; all above are taken; `need` of these are still to be taken
    for (;;) {
        const unsigned long long width = hi - lo;
        const int top = width ? 63 - __builtin_clzll(width) : 0, shift = top > 10 ? top - 10 : 0;
        for (int i = threadIdx.x; i < SEL_BINS; i += SEL_T) bins[i] = 0;
        __syncthreads();
        for (int i = begin + threadIdx.x; i < end; i += SEL_T) {
            const unsigned long long k = keys[i];
            if (k >= lo && k <= hi) atomicAdd(&bins[(k - lo) >> shift], 1u);
        }
        __syncthreads();
        // bins from the top: thread t holds bins 2047 - 2t and 2046 - 2t
        const unsigned c0 = bins[SEL_BINS - 1 - 2 * threadIdx.x], c1 = bins[SEL_BINS - 2 - 2 * threadIdx.x];
        unsigned upto = c0 + c1;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const unsigned y = __shfl_up(upto, d, 64);
            if (lane >= d) upto += y;
        }
        if (lane == 63) part[wave] = upto;
        __syncthreads();
        for (int w = 0; w < wave; ++w) upto += part[w];
        const unsigned above = upto - c0 - c1;
        if (above < need && above + c0 >= need) {
            found[0] = SEL_BINS - 1 - 2 * threadIdx.x; found[1] = need - above; found[2] = c0;
        } else if (above + c0 < need && upto >= need) {
            found[0] = SEL_BINS - 2 - 2 * threadIdx.x; found[1] = need - above - c0; found[2] = c1;
        }
        __syncthreads();
        need = found[1];
        const unsigned inside = found[2];
        lo += (unsigned long long)found[0] << shift;
        const unsigned long long far = lo + ((1ull << shift) - 1);
        hi = far < hi && far >= lo ? far : hi;
        if (inside == need || shift == 0) break;
        __syncthreads();
    }
    // taken: keys above hi, and the first `need` of [lo, hi] (all of them unless they are equal)
    unsigned placed = a.first, equal = 0;
    for (int i0 = begin; i0 < end; i0 += SEL_T) {
        const int i = i0 + threadIdx.x;
        const unsigned long long k = i < end ? keys[i] : 0;
        const bool above = i < end && k > hi, in = i < end && k >= lo && k <= hi;
        const unsigned long long ins = __ballot(in), below = (1ull << lane) - 1;
        __syncthreads();
        if (lane == 0) part[wave] = __builtin_popcountll(ins);
        __syncthreads();
        unsigned rank = equal + __builtin_popcountll(ins & below);
        for (int w = 0; w < SEL_W; ++w) {
            if (w < wave) rank += part[w];
            equal += part[w];
        }
        const bool take = above || (in && rank < need);
        const unsigned long long takes = __ballot(take);
        __syncthreads();
        if (lane == 0) part[wave] = __builtin_popcountll(takes);
        __syncthreads();
        unsigned place = placed + __builtin_popcountll(takes & below);
        for (int w = 0; w < SEL_W; ++w) {
            if (w < wave) place += part[w];
            placed += part[w];
        }
        if (take) leave(place, i);
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
template <typename T> int bounds_of(const BoundsArgs &a, bool mx, hipStream_t st) {
    const long long items = (long long)a.B * a.touched * a.Hk;
    const dim3 g((unsigned)((items + 3) / 4)), t(256);
    return by_width(a.K, [&](auto k) {
        if (mx) hipLaunchKernelGGL((bounds_kernel<T, decltype(k)::value, true>), g, t, 0, st, a);
        else hipLaunchKernelGGL((bounds_kernel<T, decltype(k)::value, false>), g, t, 0, st, a);
    });
}
template <typename T> int select_of(const SelectArgs &a, hipStream_t st) {
    int rc = 0;
    if (a.max_pages_seen > a.pages)
        rc = by_width(a.K, [&](auto k) {
            using R = ScoreRow<T, decltype(k)::value>;
            hipLaunchKernelGGL((score_kernel<T, decltype(k)::value>), dim3(select_chunks(a.B, a.Hk, R::HEADS, a.max_pages_seen), a.B, (a.Hk + R::HEADS - 1) / R::HEADS), dim3(256), 0, st, a);
        });
    if (rc == 0) hipLaunchKernelGGL(select_kernel, dim3((unsigned)a.B * a.Hk), dim3(SEL_T), 0, st, a);
    return rc;
}
}  // namespace

int launch_bounds(const BoundsArgs &a, bool bf16_io, bool mx, hipStream_t st) { return bf16_io ? bounds_of<bf16>(a, mx, st) : bounds_of<float>(a, mx, st); }
int launch_select(const SelectArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? select_of<bf16>(a, st) : select_of<float>(a, st); }

}  // namespace osdn
