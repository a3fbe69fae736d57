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
// plan and release are bound by latency: a launch, the lengths, the list, the table, one after the other (256 requests of a token 4.3 us, 96 prompts of 65536 tokens 6.3, whose positions,
// rows and slots are 1 MB; 64 sequences of 24 pages back 5.1).  A workgroup of 16 wavefronts holds the running sums, which every one of many makes for itself rather than wait for another's.
// bounds reads the new rows and the bounds of the pages that had some before (8 heads of one token 3.3 us, of 48 sequences in 4 bits 4.3).
// select is bound by the bounds that it reads where there are many: 4096 pages of 8 heads 13.7 us, of which the scores are 7.0 (17 MB), 384 rows of up to 512 pages 17.1 (44 MB, and half of
// the vector instructions' time), 256 of 4096 109 (537 MB, 4.9 TB/s).  Sums of select are in 64 bits: the products of bf16 numbers are exact there and so, but for a spread of more than
// 2^25 between them, are their sums, so that which page wins does not hang on their order.
// (The smallest of twelve launches in a kernel trace; 256 of 4096 pages: calls in a loop.)
#include "osdn_kernels.h"
#include "osdn_plan.h"

namespace osdn {

constexpr int PLAN_T = 1024, PLAN_W = PLAN_T / 64;

__device__ __forceinline__ unsigned add_sat(unsigned a, unsigned b) { return __builtin_elementwise_add_sat(a, b); }

// Sums over the lanes up to this one (SAT: that stop at the largest number)
template <bool SAT> __device__ __forceinline__ unsigned sum_upto(unsigned x) {
    auto with = [&](int y) { x = SAT ? add_sat(x, (unsigned)y) : x + (unsigned)y; };
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true));       // row_shr:1, 2, 4, 8
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));      // row_bcast:15 into rows 1 and 3
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));      // row_bcast:31 into rows 2 and 3
    return x;
}
// Sums over the threads of a workgroup, each with its own and those before it; saturating.  `all`: the sum over all threads.
struct TwoSums { unsigned a, b; };
__device__ __forceinline__ TwoSums running_sums(TwoSums x, TwoSums &all, unsigned (&part)[PLAN_W][2], int wave, int lane) {
    x = {sum_upto<true>(x.a), sum_upto<true>(x.b)};
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

// The page that the place-th from the top of the list is
__device__ __forceinline__ int granted(const PlanArgs &a, int have, unsigned place) { return a.free_list[have - 1 - (int)place]; }
// (a page that is not there has no slots)
__device__ __forceinline__ void leave_token(const PlanArgs &a, int at, int pos, int row, int page) {
    a.positions[at] = pos;
    a.rows[at] = row;
    if (a.slots) a.slots[at] = (unsigned)page < (unsigned)a.n_pages ? ((long long)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : -1;
}
// The last of n ascending numbers that is no larger than x (the first is); of equal ones the last
__device__ __forceinline__ int last_up_to(const int *v, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (v[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Every workgroup makes the running sums; the first leaves what there is for each request and grants the pages, each the tokens of its part of the token axis (`per` of
// them, 0: plan_tokens_kernel does).  A request of a token and of no more than two pages is its thread's; others are laid down in LDS, where every page and token finds its own.
__global__ __launch_bounds__(PLAN_T) void plan_kernel(PlanArgs a, int per) {
    extern __shared__ unsigned bits[];
    __shared__ unsigned part[PLAN_W][2];
    __shared__ int pages_at[PLAN_T], tokens_at[PLAN_T], first_of[PLAN_T], row_of[PLAN_T], cached_of[PLAN_T];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), words = (a.n_seqs + 31) / 32;
    const int P = 1 << a.page_shift, begin = min(a.N, (int)blockIdx.x * per), end = min(a.N, begin + per);
    const bool grants = blockIdx.x == 0;
    const long long capacity = min((long long)a.max_pages << a.page_shift, 0x7fffffffLL);
    const int have = max(0, min(*a.n_free, a.free_capacity));
    if (a.seq) note_rows(bits, words, a.n_seqs, a.B, a.seq, a.fresh);
    TwoSums asked{0u, 0u}, given{0u, 0u};           // of the requests before this round's: pages and tokens, asked for and given
    for (int b0 = 0; b0 < a.B; b0 += PLAN_T) {
        const int b = b0 + (int)threadIdx.x;
        int row = 0, cached = 0, fresh = 0, first = 0, need = 0;
        if (b < a.B) {
            row = a.seq ? a.seq[b] : b;
            cached = a.cached[b];
            fresh = a.fresh[b];
            const bool known = (unsigned)row < (unsigned)a.n_seqs;
            const bool twice = a.seq && known && fresh > 0 && (bits[words + (row >> 5)] >> (row & 31) & 1u);
            const bool valid = known && !twice && cached >= 0 && fresh >= 0 && (long long)cached + fresh <= capacity;
            if (!known || cached < 0) cached = 0;
            if (!valid) fresh = 0;
            first = (int)(((long long)cached + P - 1) >> a.page_shift);
            need = valid ? (int)(((long long)cached + fresh + P - 1) >> a.page_shift) - first : 0;
        }
        TwoSums all;
        TwoSums upto = running_sums({(unsigned)need, (unsigned)fresh}, all, part, wave, lane);
        const bool served = (need == 0 || add_sat(asked.a, upto.a) <= (unsigned)have) && (fresh == 0 || add_sat(asked.b, upto.b) <= (unsigned)a.N);
        asked = {add_sat(asked.a, all.a), add_sat(asked.b, all.b)};
        if (!served) need = fresh = 0;
        if (__syncthreads_or(!served)) upto = running_sums({(unsigned)need, (unsigned)fresh}, all, part, wave, lane);
        const unsigned place = given.a + upto.a - need;
        const int start = (int)(given.b + upto.b) - fresh;
        if (grants && b < a.B) {
            a.lengths[b] = cached + fresh;
            a.starts[b] = start;
            if (b == a.B - 1) a.starts[a.B] = start + fresh;
        }
        if (__syncthreads_or(need > 2 || (fresh > 1 && per > 0))) {
            const int n = min(PLAN_T, a.B - b0);
            pages_at[threadIdx.x] = (int)place;
            tokens_at[threadIdx.x] = start;
            first_of[threadIdx.x] = first;
            row_of[threadIdx.x] = row;
            cached_of[threadIdx.x] = cached;
            __syncthreads();
            if (grants)
                for (int i = (int)given.a + threadIdx.x; i < (int)(given.a + all.a); i += PLAN_T) {
                    const int r = last_up_to(pages_at, n, i);
                    a.table[(long long)row_of[r] * a.table_stride + first_of[r] + (i - pages_at[r])] = granted(a, have, i);
                }
            for (int i = max(begin, (int)given.b) + (int)threadIdx.x; i < min(end, (int)(given.b + all.b)); i += PLAN_T) {
                const int r = last_up_to(tokens_at, n, i), pos = cached_of[r] + (i - tokens_at[r]), col = pos >> a.page_shift;
                int page = 0;
                if (a.slots) page = col < first_of[r] ? a.table[(long long)row_of[r] * a.table_stride + col] : granted(a, have, pages_at[r] + (col - first_of[r]));
                leave_token(a, i, pos, row_of[r], page);
            }
            __syncthreads();
        } else {
            int *to = a.table + (long long)row * a.table_stride;
            const int page = need > 0 ? granted(a, have, place) : 0;
            if (grants && need > 0) {
                to[first] = page;
                if (need == 2) to[first + 1] = granted(a, have, place + 1);
            }
            if (fresh == 1 && start >= begin && start < end) leave_token(a, start, cached, row, need > 0 ? page : a.slots ? to[cached >> a.page_shift] : 0);
        }
        given = {given.a + all.a, given.b + all.b};
    }
    for (int i = max(begin, (int)given.b) + (int)threadIdx.x; i < end; i += PLAN_T) leave_token(a, i, -1, -1, -1);
    if (grants && threadIdx.x == 0) *a.n_free_out = have - (int)given.a;
}

// Places of many tokens, behind plan_kernel: where its outputs stand in the place of its inputs, which then no second workgroup may read beside the first
__global__ __launch_bounds__(256) void plan_tokens_kernel(PlanArgs a) {
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= a.N) return;
    if (j >= a.starts[a.B]) return leave_token(a, j, -1, -1, -1);
    const int b = last_up_to(a.starts, a.B, j), row = a.seq ? a.seq[b] : b, pos = a.lengths[b] - (a.starts[b + 1] - j);
    leave_token(a, j, pos, row, a.slots ? a.table[(long long)row * a.table_stride + (pos >> a.page_shift)] : 0);
}

// The i-th page that is given back, of R in the order of the requests and of their pages, lands R - 1 - i above what the list holds, so that the next requests
// take them in that order again.  All entries of the table that are given back make one list, of which a thread takes runs of RELEASE_RUN.
constexpr int RELEASE_RUN = 4;
__global__ __launch_bounds__(PLAN_T) void release_kernel(PlanArgs a) {
    extern __shared__ unsigned bits[];
    __shared__ unsigned part[PLAN_W][2];
    __shared__ int entries_at[PLAN_T], row_of[PLAN_T];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), words = (a.n_seqs + 31) / 32;
    const int have = max(0, min(*a.n_free, a.free_capacity));
    if (a.seq) note_rows(bits, words, a.n_seqs, a.B, a.seq, a.cached);
    // requests b0 .. of a round: how many entries come before each of theirs; all of the round's
    auto lay_down = [&](int b0) {
        const int b = b0 + (int)threadIdx.x;
        int row = 0, cols = 0;
        if (b < a.B) {
            row = a.seq ? a.seq[b] : b;
            const int n = a.cached[b];
            if ((unsigned)row < (unsigned)a.n_seqs && n > 0 && !(a.seq && (bits[words + (row >> 5)] >> (row & 31) & 1u)))
                cols = (int)min((long long)a.max_pages, ((long long)n + (1 << a.page_shift) - 1) >> a.page_shift);
        }
        TwoSums all;
        const TwoSums upto = running_sums({(unsigned)cols, 0u}, all, part, wave, lane);
        entries_at[threadIdx.x] = (int)upto.a - cols;
        row_of[threadIdx.x] = row;
        __syncthreads();
        return (int)all.a;
    };
    // the entries of a thread's run from i on
    auto entry = [&](int n, int i, long long &at) {
        const int r = last_up_to(entries_at, n, i);
        at = (long long)row_of[r] * a.table_stride + (i - entries_at[r]);
        return a.table[at];
    };
    // gives back the entries [0, count) of a round, `before` pages coming before theirs, of `total`; or, total < 0, only counts them (a round that is one run long does both)
    auto go = [&](int n, int count, unsigned before, long long total) {
        unsigned sum = 0;
        for (int i0 = 0; i0 < count; i0 += PLAN_T * RELEASE_RUN) {
            long long at[RELEASE_RUN];
            int page[RELEASE_RUN];
            unsigned mine = 0;
#pragma unroll
            for (int u = 0; u < RELEASE_RUN; ++u) {
                const int i = i0 + (int)threadIdx.x * RELEASE_RUN + u;
                at[u] = -1;
                page[u] = i < count ? entry(n, i, at[u]) : -1;
            }
#pragma unroll
            for (int u = 0; u < RELEASE_RUN; ++u) mine += (unsigned)page[u] < (unsigned)a.n_pages;
            TwoSums all;
            const TwoSums upto = running_sums({mine, 0u}, all, part, wave, lane);
            unsigned place = before + sum + upto.a - mine;
            sum += all.a;
            const long long of = total == 0 ? (long long)before + sum : total;          // (0: this run has all of them)
            if (total >= 0) {
#pragma unroll
                for (int u = 0; u < RELEASE_RUN; ++u) {
                    if (at[u] >= 0) a.table[at[u]] = -1;
                    if ((unsigned)page[u] < (unsigned)a.n_pages) {
                        const long long to = have + of - 1 - place++;
                        if (to < a.free_capacity) a.free_list[to] = page[u];
                    }
                }
            }
        }
        return sum;
    };
    unsigned total = 0;
    const int count = lay_down(0);
    if (a.B <= PLAN_T && count <= PLAN_T * RELEASE_RUN) {
        total = go(min(PLAN_T, a.B), count, 0, 0);
    } else {
        for (int pass = 0; pass < 2; ++pass) {
            unsigned before = 0;
            for (int b0 = 0; b0 < a.B; b0 += PLAN_T) {
                __syncthreads();
                const int c = lay_down(b0);
                before += go(min(PLAN_T, a.B - b0), c, before, pass == 0 ? -1 : (long long)total);
            }
            total = before;
            if (total == 0 && pass == 0) total = 1;         // (nothing to give back: entries are cleared all the same)
            if (pass == 1) total = before;
        }
    }
    if (threadIdx.x == 0) *a.n_free_out = (int)min((long long)a.free_capacity, (long long)have + total);
}

int launch_plan(const PlanArgs &a, hipStream_t st) {
    const size_t lds = a.seq ? (size_t)((a.n_seqs + 31) / 32) * 8 : 0;
    const bool over_itself = a.lengths == a.cached || a.lengths == a.fresh || a.n_free_out == a.n_free;
    const int workgroups = over_itself ? 1 : plan_workgroups(a.N), per = (a.N + workgroups - 1) / workgroups;
    if (!over_itself || a.N <= 4096) {
        hipLaunchKernelGGL(plan_kernel, dim3(workgroups), dim3(PLAN_T), lds, st, a, per);
    } else {
        hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(PLAN_T), lds, st, a, 0);
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

// A wavefront takes one page that got new tokens, for one head: its new rows, 64 / LANES at a time, and, where it had tokens before, its bounds.  (More pages than a launch has wavefronts:
// one after the other.)
template <typename T, int K, bool MX> __global__ __launch_bounds__(256) void bounds_kernel(BoundsArgs a) {
    using R = KeyRow<T, K, MX>;
    constexpr int VE = R::VE, ROWS = 64 / R::LANES, PER = 16 / sizeof(T);
    const int lane = threadIdx.x & 63, sub = lane / R::LANES, e0 = lane % R::LANES * VE;
    const long long items = (long long)a.B * a.touched * a.Hk;
    for (long long item = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); item < items; item += 4LL * gridDim.x) {
        const int h = (int)(item % a.Hk);
        const long long rest = item / a.Hk;
        const int nth = (int)(rest % a.touched);
        const int b = (int)(rest / a.touched);
        const int from = max(0, a.cached[b]), end = (int)min((long long)a.lengths[b], (long long)from + a.max_new), row = a.seq ? a.seq[b] : b;
        const int col = (from >> a.page_shift) + nth;
        const long long begin = (long long)col << a.page_shift;
        if (begin >= end || from >= end || col >= a.max_pages || (unsigned)row >= (unsigned)a.n_seqs) continue;
        const int page = a.table[(long long)row * a.table_stride + col];
        if ((unsigned)page >= (unsigned)a.n_pages) continue;
        const int s0 = (int)(max((long long)from, begin) - begin), s1 = (int)min((long long)1 << a.page_shift, end - begin);
        T *out = static_cast<T *>(a.bounds) + ((long long)page * a.Hk + h) * 2 * K + e0;
        float lo[VE], hi[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
        if (s0 > 0) {                       // (tokens from before)
            auto old = [&](const T *at, float (&x)[VE]) {
#pragma unroll
                for (int v = 0; v < VE / PER; ++v) {
                    const u32x4 raw = *reinterpret_cast<const u32x4 *>(at + v * PER);
#pragma unroll
                    for (int e = 0; e < PER; ++e) x[v * PER + e] = vec_get<T>(raw, e);
                }
            };
            old(out, lo);
            old(out + K, hi);
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
            auto leave = [&](T *at, const float (&x)[VE]) {
#pragma unroll
                for (int v = 0; v < VE / PER; ++v) {
                    float y[PER];
#pragma unroll
                    for (int e = 0; e < PER; ++e) y[e] = x[v * PER + e];
                    store_vec_t(at + v * PER, y);
                }
            };
            leave(out, lo);
            leave(out + K, hi);
        }
    }
}

// ---- select ------------------------------------------------------------------------------------

// Scores as 64-bit integers in the same order; what is not a number comes first of all, before infinity
__device__ __forceinline__ unsigned long long score_key(double s) {
    if (s != s) return ~0ull;
    const unsigned long long u = __builtin_bit_cast(unsigned long long, s + 0.0);           // (no negative zero)
    return u >> 63 ? ~u : u | 1ull << 63;
}

template <int CTRL> __device__ __forceinline__ int moved(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true); }
template <int CTRL> __device__ __forceinline__ double moved(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)moved<CTRL>((int)(u >> 32)) << 32 | (uint32_t)moved<CTRL>((int)(uint32_t)u));
}
// x and that of the lane 16 (32) away, added
template <int AWAY> __device__ __forceinline__ double with_lanes_away(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    uint32_t a = (uint32_t)u, b = (uint32_t)(u >> 32), c = a, d = b;
    if constexpr (AWAY == 16) asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\tv_permlane16_swap_b32 %2, %3" : "+v"(a), "+v"(c), "+v"(b), "+v"(d));
    else asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\tv_permlane32_swap_b32 %2, %3" : "+v"(a), "+v"(c), "+v"(b), "+v"(d));
    return __builtin_bit_cast(double, (uint64_t)b << 32 | a) + __builtin_bit_cast(double, (uint64_t)d << 32 | c);
}
// The largest of the lanes up to this one
__device__ __forceinline__ unsigned largest_upto(unsigned x) {
    auto with = [&](int y) { x = max(x, (unsigned)y); };
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));
    return x;
}

// The bounds of a page and head are a row of 2 K elements, the smallest first: 16 bytes a lane, VPL of them, in LANES lanes; a wavefront has ROWS of them side by side.
template <typename T, int K> struct ScoreRow {
    static constexpr int VE = 16 / sizeof(T), ALL = 2 * K / VE, LANES = ALL < 64 ? ALL : 64, VPL = ALL / LANES, ROWS = 64 / LANES;
    double w[VPL][VE];          // what a lane's elements are multiplied by: sums of the negative (smallest) or positive (largest) parts of the queries
    __device__ __forceinline__ void weights(const SelectArgs &a, int b, int h, int lane) {
#pragma unroll
        for (int v = 0; v < VPL; ++v)
#pragma unroll
            for (int e = 0; e < VE; ++e) w[v][e] = 0.0;
        for (int i0 = 0; i0 < a.group; i0 += 4) {               // (four heads on their way together)
            u32x4 raw[4][VPL];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const T *q = static_cast<const T *>(a.q.data) + b * a.q.batch + (long long)(h * a.group + min(i0 + i, a.group - 1)) * a.q.head;
#pragma unroll
                for (int v = 0; v < VPL; ++v) {
                    const T *at = q + (lane % LANES + v * LANES) * VE % K;
                    if (a.aligned) {
                        raw[i][v] = *reinterpret_cast<const u32x4 *>(at);
                    } else {
                        T x[VE];
#pragma unroll
                        for (int e = 0; e < VE; ++e) x[e] = at[e];
                        raw[i][v] = __builtin_bit_cast(u32x4, x);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i0 + i < a.group) {
#pragma unroll
                    for (int v = 0; v < VPL; ++v) {
                        const bool low = (lane % LANES + v * LANES) * VE < K;
#pragma unroll
                        for (int e = 0; e < VE; ++e) {
                            const float x = vec_get<T>(raw[i][v], e);
                            w[v][e] += (double)(low ? least(x, 0.f) : greatest(x, 0.f));
                        }
                    }
                }
        }
    }
    static __device__ __forceinline__ void ask(const SelectArgs &a, long long page, int h, int lane, u32x4 (&raw)[VPL]) {
        const T *from = static_cast<const T *>(a.bounds) + (page * a.Hk + h) * 2 * K + lane % LANES * VE;
#pragma unroll
        for (int v = 0; v < VPL; ++v) raw[v] = *reinterpret_cast<const u32x4 *>(from + v * LANES * VE);
    }
    __device__ __forceinline__ double sum(const u32x4 (&raw)[VPL]) const {
        double s = 0.0;
#pragma unroll
        for (int v = 0; v < VPL; ++v)
#pragma unroll
            for (int e = 0; e < VE; ++e) s = __builtin_fma(w[v][e], (double)vec_get<T>(raw[v], e), s);
        return s;
    }
    // the scores of four pages, of page u in the row's lanes that are u modulo 4 (a row has 16 lanes at least): the first two exchanges halve what there is to add
    __device__ __forceinline__ double scores(const u32x4 (&raw)[4][VPL], int lane) const {
        double s[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] = sum(raw[u]);
        const bool odd = lane & 1, upper = lane & 2;
        const double s01 = (odd ? s[1] : s[0]) + moved<0xB1>(odd ? s[0] : s[1]);            // quad_perm [1,0,3,2]
        const double s23 = (odd ? s[3] : s[2]) + moved<0xB1>(odd ? s[2] : s[3]);
        double x = (upper ? s23 : s01) + moved<0x4E>(upper ? s01 : s23);                    // quad_perm [2,3,0,1]
        x += moved<0x124>(x);                   // row_ror:4
        x += moved<0x128>(x);                   // row_ror:8
        if constexpr (LANES > 16) x = with_lanes_away<16>(x);
        if constexpr (LANES > 32) x = with_lanes_away<32>(x);
        return x;
    }
};
__device__ __forceinline__ Seen pages_seen(const SelectArgs &a, int b) {
    return seen_tokens(a.lengths[b], a.seq ? a.seq[b] : b, a.n_seqs, a.max_length, 0, a.page_shift, a.max_pages);
}
__device__ __forceinline__ int pages_of(const SelectArgs &a, const Seen &see) { return see.end > 0 ? ((see.end - 1) >> a.page_shift) + 1 : 0; }

// Keys of the pages p0 + l (l < 4 ROWS or, HEADS: 4) + stride i of a table's row, below p1, for one head (lanes of a wavefront: ROWS pages next to each other) or, HEADS, for ROWS heads next
// to each other.  The numbers of the pages of 16 steps (64 / (4 ROWS) if that is less) are on their way at once, the bounds of a step while those of the one before are summed.
template <typename T, int K, bool HEADS> struct PageSteps {
    static constexpr int SIDE = HEADS ? 1 : ScoreRow<T, K>::ROWS, STEP = 4 * SIDE, STEPS = 64 / STEP;
    static_assert(STEPS <= SELECT_STEPS, "the page counter's steps");
    // the lane STEP i + l: page l of step i from p on (what stands behind the last page is looked at, and left out in the end)
    static __device__ __forceinline__ int ask(const SelectArgs &a, const int *table, int p, int stride, int lane) {
        return table[min((long long)p + (long long)(lane / STEP) * stride + lane % STEP, (long long)a.max_pages - 1)];
    }
};
template <typename T, int K, bool HEADS, typename F>
__device__ __forceinline__ void score_pages(const SelectArgs &a, const ScoreRow<T, K> &r, const int *table, int h, int own, int p0, int p1, int stride, int lane, F &&leave) {
    using R = ScoreRow<T, K>;
    using P = PageSteps<T, K, HEADS>;
    constexpr int SIDE = P::SIDE, STEP = P::STEP, STEPS = P::STEPS;
    const int sub = HEADS ? 0 : lane / R::LANES;
    for (int p = p0; p < p1; p += STEPS * stride) {
        if (p > p0) own = P::ask(a, table, p, stride, lane);
        u32x4 raw[4][R::VPL];
        auto ask = [&](int i) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int page = __shfl(own, STEP * i + u * SIDE + sub, 64);
                R::ask(a, (unsigned)page < (unsigned)a.n_pages ? page : 0, h, lane, raw[u]);
            }
        };
        ask(0);
        for (int i = 0; i < STEPS && p + i * stride < p1; ++i) {
            u32x4 now[4][R::VPL];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < R::VPL; ++v) now[u][v] = raw[u][v];
            const int mine = __shfl(own, STEP * i + (lane & 3) * SIDE + sub, 64);
            if (i + 1 < STEPS && p + (i + 1) * stride < p1) ask(i + 1);
            const unsigned long long key = score_key(r.scores(now, lane));
            const int at = p + i * stride + (lane & 3) * SIDE + sub;
            if (at < p1 && lane % R::LANES < 4) leave(at, (unsigned)mine < (unsigned)a.n_pages ? key : ~0ull);
        }
    }
}

// Few rows of many pages: the keys by a launch of their own
template <typename T, int K> __global__ __launch_bounds__(256) void score_kernel(SelectArgs a) {
    using R = ScoreRow<T, K>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.y, h = (int)blockIdx.z * R::ROWS + lane / R::LANES, hh = min(h, a.Hk - 1), first = a.first + (int)(blockIdx.x * 4 + wave) * 4, stride = (int)gridDim.x * 16;
    // (what does not hang on the length is asked for beside it)
    const int row = a.seq ? a.seq[b] : b;
    const int *table = a.table + ((unsigned)row < (unsigned)a.n_seqs ? (long long)row * a.table_stride : 0);
    const int own = PageSteps<T, K, true>::ask(a, table, first, stride, lane);
    R r;
    r.weights(a, b, hh, lane);
    const int have = pages_of(a, pages_seen(a, b));
    if (have <= a.pages || first >= have - a.last) return;              // (all of them are taken)
    unsigned long long *keys = a.keys + ((long long)b * a.Hk + hh) * a.max_pages_seen;
    score_pages<T, K, true>(a, r, table, hh, own, first, have - a.last, stride, lane, [&](int p, unsigned long long key) {
        if (h < a.Hk) keys[p] = key;
    });
}

constexpr int SEL_T = 512, SEL_W = SEL_T / 64, SEL_BINS = 2048, SEL_RUN = SEL_BINS / SEL_T, SEL_LIST = 64;
// The n-th largest of a workgroup's keys, `need` of count: after it, taken are the keys above hi and the first `need` of those in [lo, hi].  The keys between the bounds known so far are
// counted in 2048 even bins, the bin that holds it gives the next bounds, until all of a bin is taken, it is one key wide, or few enough are in it to be compared
// with each other.  `each` calls its argument with every key of the thread.
struct Cut { unsigned long long lo, hi; unsigned need; };
struct CutSpace {
    unsigned bins[SEL_BINS], part[SEL_W], found[3], listed;
    unsigned edge[SEL_W][2];
    unsigned long long list[SEL_LIST];
};
template <typename F> __device__ __forceinline__ Cut cut_keys(CutSpace &c, unsigned need, int lane, int wave, F &&each) {
    unsigned least = 0, most = 0;               // of the upper words: the range starts at the least of them (kept as its complement) and ends with the largest
    each([&](unsigned long long k) {
        least = max(least, ~(unsigned)(k >> 32));
        most = max(most, (unsigned)(k >> 32));
    });
    least = largest_upto(least);
    most = largest_upto(most);
    if (lane == 63) { c.edge[wave][0] = least; c.edge[wave][1] = most; }
    for (int i = threadIdx.x; i < SEL_BINS; i += SEL_T) c.bins[i] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < SEL_W; ++w) {
        least = max(least, c.edge[w][0]);
        most = max(most, c.edge[w][1]);
    }
    least = __builtin_amdgcn_readfirstlane(least);
    most = __builtin_amdgcn_readfirstlane(most);
    unsigned long long lo = (unsigned long long)~least << 32, hi = (unsigned long long)most << 32 | 0xffffffffu;
    for (;;) {
        const unsigned long long width = hi - lo;
        const int top = width ? 63 - __builtin_clzll(width) : 0, shift = top > 10 ? top - 10 : 0;
        each([&](unsigned long long k) {
            if (k >= lo && k <= hi) atomicAdd(&c.bins[(k - lo) >> shift], 1u);
        });
        if (threadIdx.x == 0) c.listed = 0;
        __syncthreads();
        // bins from the top, a run of them a thread
        unsigned here[SEL_RUN], all = 0;
#pragma unroll
        for (int i = 0; i < SEL_RUN; ++i) {
            here[i] = c.bins[SEL_BINS - 1 - (SEL_RUN * threadIdx.x + i)];
            c.bins[SEL_BINS - 1 - (SEL_RUN * threadIdx.x + i)] = 0;
            all += here[i];
        }
        const unsigned upto = sum_upto<false>(all);
        if (lane == 63) c.part[wave] = upto;
        __syncthreads();
        unsigned above = upto - all;
#pragma unroll
        for (int w = 0; w < SEL_W; ++w) above += w < wave ? c.part[w] : 0u;
#pragma unroll
        for (int i = 0; i < SEL_RUN; ++i) {
            if (above < need && above + here[i] >= need) {
                c.found[0] = SEL_BINS - 1 - (SEL_RUN * threadIdx.x + i); c.found[1] = need - above; c.found[2] = here[i];
            }
            above += here[i];
        }
        __syncthreads();
        need = c.found[1];
        const unsigned inside = c.found[2];
        lo += (unsigned long long)c.found[0] << shift;
        const unsigned long long far = lo + ((1ull << shift) - 1);
        hi = far < hi && far >= lo ? far : hi;
        if (inside == need || shift == 0) return {lo, hi, need};
        if (inside <= SEL_LIST) {
            each([&](unsigned long long k) {
                if (k >= lo && k <= hi) c.list[atomicAdd(&c.listed, 1u)] = k;
            });
            __syncthreads();
            // (every wavefront does the same with all of them)
            const unsigned long long mine = lane < (int)inside ? c.list[lane] : 0;
            unsigned more = 0, alike = 0;
            for (unsigned i = 0; i < inside; ++i) {
                const unsigned long long k = c.list[i];
                more += k > mine;
                alike += k == mine;
            }
            const unsigned long long who = __ballot(lane < (int)inside && more < need && need <= more + alike);
            const int src = __builtin_ctzll(who);
            const unsigned long long key = __shfl(mine, src, 64);
            return {key, key, need - __shfl(more, src, 64)};
        }
        __syncthreads();
    }
}

// A workgroup takes one key head of a sequence: a run of EACH keys a thread (more pages than that: read again for every pass).  SCORE: it makes the keys itself, else score_kernel has.
template <typename T, int K, int EACH, bool SCORE> __global__ __launch_bounds__(SEL_T) void select_kernel(SelectArgs a) {
    __shared__ CutSpace space;
    __shared__ unsigned long long made[SCORE ? EACH * SEL_T : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), b = blockIdx.x / (unsigned)a.Hk, h = blockIdx.x % (unsigned)a.Hk;
    const int row = a.seq ? a.seq[b] : b;
    const int *table = a.table + ((unsigned)row < (unsigned)a.n_seqs ? (long long)row * a.table_stride : 0);
    using R = ScoreRow<T, K>;
    using P = PageSteps<T, K, false>;
    constexpr int STRIDE = SEL_W * P::STEP;
    [[maybe_unused]] int own = 0;
    [[maybe_unused]] R r;
    if constexpr (SCORE) {              // (what does not hang on the length is asked for beside it)
        own = P::ask(a, table, a.first + wave * P::STEP, STRIDE, lane);
        r.weights(a, b, h, lane);
    }
    const Seen see = pages_seen(a, b);
    const int have = pages_of(a, see), n = min(have, a.pages);
    int *out = a.chosen + (long long)blockIdx.x * a.pages;
    if (threadIdx.x == 0) a.tokens[blockIdx.x] = see.broken ? 0x7fffffff : have ? ((n - 1) << a.page_shift) + ((see.end - 1) & ((1 << a.page_shift) - 1)) + 1 : 0;
    for (int i = n + threadIdx.x; i < a.pages; i += SEL_T) out[i] = -1;
    if (have == 0) return;
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
    const unsigned need = a.pages - a.first - a.last;   // of the pages [begin, end), which are more
    if (need == 0) return;
    const int begin = a.first, end = have - a.last, count = end - begin;
    const unsigned long long *keys = a.keys + (long long)blockIdx.x * a.max_pages_seen + begin;
    if constexpr (SCORE) {
        score_pages<T, K, false>(a, r, table, h, own, begin + wave * P::STEP, end, STRIDE, lane, [&](int p, unsigned long long key) {
            made[p - begin] = key;
        });
        __syncthreads();
        keys = made;
    }
    const int run = (count + SEL_T - 1) / SEL_T, at = min((int)threadIdx.x * run, count), mine = min(run, count - at);
    unsigned long long k[EACH];
    const bool held = SCORE || run <= EACH;
    if (held) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) k[i] = i < mine ? keys[at + i] : 0;
    }
    auto each = [&](auto &&f) {
        if (held) {
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (i < mine) f(k[i]);
        } else {
            for (int i = 0; i < mine; ++i) f(keys[at + i]);
        }
    };
    const Cut cut = cut_keys(space, need, lane, wave, each);
    // of the pages before this thread's so many are above the cut and so many in it: as many of the first, and of the others up to cut.need, are taken
    unsigned above = 0, in = 0;
    each([&](unsigned long long x) {
        above += x > cut.hi;
        in += x >= cut.lo && x <= cut.hi;
    });
    unsigned a0 = sum_upto<false>(above), i0 = sum_upto<false>(in);
    __syncthreads();
    if (lane == 63) { space.part[wave] = a0; space.bins[wave] = i0; }
    __syncthreads();
    a0 -= above;
    i0 -= in;
#pragma unroll
    for (int w = 0; w < SEL_W; ++w) {
        a0 += w < wave ? space.part[w] : 0u;
        i0 += w < wave ? space.bins[w] : 0u;
    }
    int p = begin + at;
    each([&](unsigned long long x) {
        const bool up = x > cut.hi, inside = x >= cut.lo && x <= cut.hi;
        if (up || (inside && i0 < cut.need)) leave(a.first + a0 + min(i0, cut.need), p);
        a0 += up;
        i0 += inside;
        ++p;
    });
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
    const dim3 g(bounds_workgroups(items)), t(256);
    return by_width(a.K, [&](auto k) {
        if (mx) hipLaunchKernelGGL((bounds_kernel<T, decltype(k)::value, true>), g, t, 0, st, a);
        else hipLaunchKernelGGL((bounds_kernel<T, decltype(k)::value, false>), g, t, 0, st, a);
    });
}
template <typename T> int select_of(const SelectArgs &a, hipStream_t st) {
    return by_width(a.K, [&](auto k) {
        constexpr int K = decltype(k)::value;
        using R = ScoreRow<T, K>;
        const dim3 rows((unsigned)a.B * a.Hk), t(SEL_T);
        if (select_scores_itself(a.B * (long long)a.Hk, a.max_pages_seen, 2 * K * (int)sizeof(T))) {
            if (a.max_pages_seen <= 1024) hipLaunchKernelGGL((select_kernel<T, K, 1024 / SEL_T, true>), rows, t, 0, st, a);
            else hipLaunchKernelGGL((select_kernel<T, K, 4096 / SEL_T, true>), rows, t, 0, st, a);
            return;
        }
        if (a.max_pages_seen > a.pages)
            hipLaunchKernelGGL((score_kernel<T, K>), dim3(select_chunks(a.B, a.Hk, R::ROWS, a.max_pages_seen), a.B, (a.Hk + R::ROWS - 1) / R::ROWS), dim3(256), 0, st, a);
        if (a.max_pages_seen <= 4096) hipLaunchKernelGGL((select_kernel<T, 64, 4096 / SEL_T, false>), rows, t, 0, st, a);
        else hipLaunchKernelGGL((select_kernel<T, 64, 16384 / SEL_T, false>), rows, t, 0, st, a);
    });
}
}  // namespace

int launch_bounds(const BoundsArgs &a, bool bf16_io, bool mx, hipStream_t st) { return bf16_io ? bounds_of<bf16>(a, mx, st) : bounds_of<float>(a, mx, st); }
int launch_select(const SelectArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? select_of<bf16>(a, st) : select_of<float>(a, st); }

}  // namespace osdn
