// The rules by which osdn_fwd and osdn_bwd cut the work: segments of the sequence, pieces of a chain, the solved form of the
// reverse sweep, and the slices of the chain kernels.  Plain code without a device in it, so that the rules can be tested by themselves.
#pragma once
#include "../../include/osdn.h"

#include <cmath>

namespace osdn {

constexpr int NUM_CU = 256, NUM_XCD = 8;         // (workgroups are dealt to the XCDs in turn; each has its own L2)
constexpr int MAX_SEGMENTS = 16, MAX_PIECES = 512, MAX_PIECE_SWEEPS = 13;

// The chain kernels run V/VS workgroups (slices) per chain that all read the same tiles (-W, K~, P, ...): they are to share an XCD.
// Where the chains are not a multiple of the XCDs, narrow slices (VS = 16) are filled up to one with workgroups that end at once, if all still
// find a CU each; else the slices of a chain stand side by side on as many XCDs.  20 chains of 40 chunks, V = 128, us, side by
// side and filled up: forward 161 and 136, backward 222 and 189 (with slices of 32 203); of 128 chunks, forward 446 and 399; 28 chains of
// 128 chunks, forward 605 and 491; 12 of 64, V = 256, 181 and 163; fp32, 10 of 32, backward 336 and 328.  Not up to eight chains, which leave the L2s
// time (2 chains of 512 chunks, V = 256, forward 598 and 608, 6 of 64 with K = 64 118 and 122, 4 of 512 599 and 555), nor for slices of 32
// (50 chains of 64 chunks, forward 360 and 366, backward 521 and 527).
inline bool chains_filled_up(int nslices, long long chains, bool narrow) {
    return narrow && chains > NUM_XCD && (chains + NUM_XCD - 1) / NUM_XCD * nslices * NUM_XCD <= NUM_CU;
}
// How the workgroups of such a launch are laid out, with what a workgroup needs to find its slice: a multiplication in place of a division
// (reciprocal: the next above 2^32 / slices, exact below 2^27 workgroups), and nothing that it would have to wait for twice.
struct SliceMap { int slices, chains, share; unsigned reciprocal; };
inline SliceMap slice_map(int nslices, long long chains, bool narrow) {
    return {nslices, (int)chains, chains % NUM_XCD == 0 || chains_filled_up(nslices, chains, narrow), (unsigned)(((1ull << 32) + nslices - 1) / nslices)};
}
inline int chain_workgroups(const SliceMap &m) { return (m.share ? (m.chains + NUM_XCD - 1) / NUM_XCD * NUM_XCD : m.chains) * m.slices; }
// (constexpr: for the device too; a chain that there is not: nothing to do)
constexpr void chain_slice_of(int wg, const SliceMap &m, int &chain, int &slice) {
    const unsigned j = m.share ? (unsigned)wg / NUM_XCD : (unsigned)wg, c = (unsigned)(((unsigned long long)j * m.reciprocal) >> 32);
    slice = (int)(j - c * m.slices);
    chain = m.share ? (int)(wg % NUM_XCD + NUM_XCD * c) : (int)c;
}

// state_fwd_run_kernel with slices of 16: whether it asks for the lines of its operands ahead of its tiles (tiles: chunks of all chains).
// That pays where they come from HBM and the slices that share them share an L2: what the forward pass reads and writes around the chain
// kernel (-W, K~, T diag(beta), V, the checkpoint of S, E; three more with a gate per channel) is then more than the 256 MB
// of the last level cache hold beside the inputs.  Forward pass, us, without and with, K = V = 128 unless said, calls repeated: 16 chains of 64
// chunks (106 MB) 172.9 and 174.5, of 96 (160) 244.4 and 247.8, of 128 (213) 343 and 338, of 256 with retention 542 and 509; 24 of 48 (120)
// 178.7 and 180.6, of 128 (319) 456 and 451; V = 256: 16 of 64 (172) 180.8 and 182.7, of 128 (344) 331 and 324, 8 of 128 (172) 219.8 and 231.3, of
// 256 430 and 415; V = 64: 32 of 64 (147) 264.5 and 265.8, of 128 (295) 478 and 456, 8 of 512 (295) 945 and 890; K = V = 64: 8 of 512 (197)
// 707 and 729; V = 128: 16 of 512 (590) 747 and 738; a gate per channel: 16 of 64 (156) 207.9 and 209.9, 24 of 64 (233) 284 and 278, 16 of 128 (311)
// 413 and 393.  With the caches cleared between calls the line is the same (16 of 96 277 and 280, of 128 357 and 357; 8 of 512 773 and 722).  Slices
// on eight XCDs: 4 chains of 512 585 and 598, 2 of 512 431 and 463.
inline bool asks_ahead(const osdn_params *p, long long tiles, long long chains) {
    const long long K = p->K, V = p->V, kept = 2 * (64 * 64 + (p->gate_per_channel ? 5 : 2) * 64 * K + 2 * 64 * V + V * K);
    return slice_map(p->V / 16, chains, true).share && tiles * kept > 200ll << 20;
}

// Number of segments for a sequence of N chunks (params->segments > 0 overrides it; 1 = no
// pipelining).  A segment more shortens the stretch of phase 1 that runs with nothing beside it (the
// first segment of the forward pass, the last of the backward pass) and costs launches, cross-stream
// waits (25 us a call for the first) and partly filled rounds of workgroups.  Times below: one stream against the best
// of two to six segments, us, K = V = 128 in bf16.
//  - short sequences take one stream: forward up to 32 chunks (2 chains of 4 chunks 34 and 79, 64 of 16 106 and
//    127, 64 of 32 215 and 220; 64 of 48 319 and 304), backward up to 48 (2 of 4 53 and 117, 64 of 16
//    149 and 179, 8 of 32 116 and 159, 64 of 48 449 and 443, 128 of 48 773 and 755; 32 of 64 368 and 370).
//  - so do many chains, which fill the chip by themselves: 256 of 64 forward 1122 and 1182, backward 1779 and 1944;
//    from 128 chains on the forward pass takes two at most (128 of 128 1253, with four 1238, with six 1291).
//  - forward otherwise: about 16 chunks per segment, at most six segments (measured flat beyond).
//  - backward otherwise: a segment more costs more there, because every launch of the phase-2 chain kernel
//    meets a phase-1 chain kernel on the other stream and the two do not fit on one CU together:
//    when the workgroups of both (chain_wgs) outnumber the CUs, the count that balances the
//    exposed tail against that cost is about sqrt(N / 15) (2 at 64 chunks, 4 at 256); when they
//    all fit side by side, about 32 chunks per segment, at most four: of that count and the two
//    above it, the one whose segments fill whole rounds of bwd_post workgroups (one per chunk and
//    chain, post_round at a time) best; from 448 chunks on, where a segment is many rounds, seven.
//    16 chains, bf16, backward pass alone: 128 chunks 483, 503, 493, 517, 546, 575 us with 3 to 8 segments
//    (5 taken); 256 chunks, V = 256 989, 989, 1045, 1056, 1094, 1020 with 4 to 9 (5); 512 chunks 1603, 1593, 1604,
//    1599, 1623, 1769 with 4 to 8 and 12; chains that are swept, gates of 0.999, 512 chunks with 4 to 8, 10 and 12: 33 chains 2381,
//    2436, 2342, 2426, 2369, 2472, 2463; 48 2939, 2970, 2936, 2984, 2954, 3055, 3050; fp32, 8 chains 3653, 3647, 3616, 3704, 3810, 3675, 3867.
// Segments cut the chunk axis as a whole.  With packed sequences the sequential kernels of a
// segment only have the sequences that cross it to work on, one after the other segment by
// segment, so cutting pays only while one sequence makes up most of the axis; otherwise the
// many independent chains fill the chip by themselves and everything runs in one piece.
inline int segment_count(int forced, int N, int longest, long long chains, long long chain_wgs, bool backward, int post_round = 0) {
    if (forced <= 0 && (long long)longest * 4 < (long long)N * 3) return 1;
    int S = forced;
    if (forced <= 0) {
        if (N <= (backward ? 48 : 32) || chains >= NUM_CU) return 1;
        if (!backward) S = N / 16 > 6 ? 6 : N / 16;
        else if (chain_wgs > NUM_CU) S = (int)std::lround(std::sqrt(N / 15.0)) > 6 ? 6 : (int)std::lround(std::sqrt(N / 15.0));
        else {
            S = N >= 448 ? 7 : N / 32 > 4 ? 4 : N / 32;
            if (S < 2) S = 2;
            double best = 0.0;
            int pick = S;
            for (int c = S; N < 448 && c <= S + 2 && c <= N; ++c) {
                const int first = N / (2 * c) > 0 ? N / (2 * c) : 1;
                const double wgs = (double)(N - first) / (c - 1) * (double)chains;   // bwd_post workgroups of a segment
                const double fill = wgs / (std::ceil(wgs / post_round) * post_round);
                if (fill > best + 1e-9) { best = fill; pick = c; }
            }
            S = pick;
        }
        if (S < 2 || (!backward && chains * 2 >= NUM_CU)) S = 2;
    }
    if (S > MAX_SEGMENTS) S = MAX_SEGMENTS;
    if (S > N) S = N;
    return S < 1 ? 1 : S;
}
// first chunk of segment s.  Segment 0 is half as long as the others: it is the one that runs
// without a partner (phase 1 of it before anything of phase 2 can start in the forward pass,
// and after everything else in the backward pass).
// First chunk of segment s when every segment is r times as long as the one before.  Used by
// the forward pass when phase 2 is the slower of the two phases (many chains): phase 2 then
// starts early on a short segment and is never left waiting for phase 1, and the long last
// segment runs when phase 1 is already out of the way.
inline int seg_begin_grow(int N, int S, int s, double r) {
    if (s <= 0) return 0;
    if (s >= S) return N;
    const double f = (std::pow(r, s) - 1.0) / (std::pow(r, S) - 1.0);
    int b = (int)std::lround(N * f);
    if (b < s) b = s;                       // at least one chunk per segment
    if (b > N - (S - s)) b = N - (S - s);
    return b;
}
inline int seg_begin(int N, int S, int s) {
    if (s <= 0) return 0;
    if (s >= S) return N;
    const int first = N / (2 * S) > 0 ? N / (2 * S) : 1;
    return first + (int)((long long)(N - first) * (s - 1) / (S - 1));
}

// Phase 1 as sweeps over the whole sequence, for few long chains: one workgroup per chain leaves most
// of the chip idle and its walk over the chunks is most of the pass.  Every chain is cut into pieces
// (a workgroup per CU over all chains; two where a piece still has eight chunks and the kernel's registers let two onto a CU, at
// most 128: that shortens the walk more than two workgroups on a CU slow each other); a sweep runs all pieces side by
// side, each from its current start value, and leaves every piece as a composed map per
// coordinate; the next sweep walks those maps for its start values; a chain is settled when none
// of its start values moves any more.  Plain batches only.  params->p1_pieces forces a number of
// pieces per chain (-1: never), params->p1_piece_sweeps the sweep limit.
//
// Where the line lies (us per pass, sequential or in segments against pieces; K = V = 128 in bf16):
//  - forward, chains on an eighth of the CUs or fewer, from 24 chunks on: 16 chains of 24 108 and 90, with a retention
//    gate 121 and 109, of 32 136 and 97, 149 and 116, of 64 260 and 174 (pieces of 4 chunks; of 8: 221), 32 of
//    32 162 and 134; 16 chains of 16, with a gate, 90 and 94.
//  - not for more chains: how many sweeps the pieces need with a retention gate goes by how much it fades, two with gates of 0.999,
//    three to five with 0.9999 or 1, and with 33 to 64 chains only two pay (64 chains, segments and pieces, gates of 0.999, then of
//    1: forward of 32 chunks 226 and 214, 246 and 250, of 64 420 and 395, 426 and 468, of 128 761 and 697, 792 and 917, of 256 1336 and
//    1261, 1468 and 1947; backward of 64 572 and 564, 593 and 620, of 128 1025 and 1057, 1070 and 1170).
//  - how many pieces, forward without retention: 4 chains of 64 chunks 193 with 8 pieces, 144 with 16, 126 with 32; of 256 380 with
//    32, 337 with 64, 367 with 128; of 512 848, 721, 741; 2 of 1024 1600, 1270, 1152 and with 256 1238; 1 of 1024 1082 with 64, 959
//    with 128, 986 with 256.
//  - two workgroups a CU where they fit (us, one and two): forward, K = 128, one gate in bf16 (127 registers) 16 chains of 256 chunks
//    525 and 514, with gates of 1 739 and 686; where they do not, the pieces run in two rounds: one gate in fp32 (136) 1285 and 1311,
//    1526 and 1573; a gate per coordinate (159) 557 and 606, 774 and 825; backward (153 and more) 698 and 733, 807 and 844.
//  - backward, only with a retention gate (without, the solved form has the shorter chain), gates of 0.999, then of 1: 16 chains of
//    24 chunks 121 and 131, 133 and 131, of 32 144 and 141, 161 and 141, of 128 500 and 378, 569 and 408, of 512 1677 and 1341, 1897
//    and 1569; pieces of four chunks at least (16 chains of 32 chunks, gates of 0.999: pieces of two 131).
//    Not for long sequences of many chains, where segments keep phase 1 beside phase 2 (gates of 0.999, then of 1): 32 chains of 64
//    chunks 391 and 317, 431 and 347, of 128 710 and 577, 694 and 679, of 256 1216 and 1133, 1277 and 1352; with fp32 I/O and K = 128
//    16 chains of 96 959 and 910, 966 and 965, of 128 1232 and 1200, 1240 and 1268, of 256 2331 and 2344, 2336 and 2487.
//  - all this for eta up to what K allows (the sweeps over the pieces need the more the larger eta / K is, and beyond a limit do not
//    settle: 0.003 is within it by a factor of 2.1 and 1.07 for the forward pass, K = 128 and 64, of 11 and 5 for the
//    backward pass).  16 chains of 48 chunks, gates of 1, segments and pieces: forward, K = 128, eta 0.01 257 and 151, 0.03 312 and 206,
//    0.1 311 and 459; K = 64, 0.003 198 and 118, 0.01 235 and 143, 0.03 235 and 340; backward, K = 128, 0.03 266 and 222, 1 416 and
//    728, K = 64, 16 chains of 128 chunks 0.01 495 and 323, 0.1 672 and 976.  Beyond it only the forward pass of 64 chunks and more is
//    cut, into pieces of eight chunks.
inline void pieces_plan(const osdn_params *p, int N, long long chains, bool packed, bool retention, bool backward, int &pieces,
                        int &piece_chunks, int &sweeps) {
    pieces = 0; piece_chunks = 0;
    // sweeps needed without retention, measured: 4 at 64 and 128 chunks, then one more per
    // doubling (7 at 1024); the limit leaves two in hand
    sweeps = 7;                                  // (the last one only finds that nothing moved)
    for (int n = 128; n < N && sweeps < MAX_PIECE_SWEEPS; n *= 2) ++sweeps;
    if (packed || chains > MAX_PIECES / 2 || (backward && !retention)) return;
    const int forced = p->p1_pieces;              // 0: decide here; -1: never; n > 0: n pieces per chain
    int target, min_chunks;
    if (forced != 0) { target = forced > 0 ? forced : 0; min_chunks = 1; }
    else {
        if (chains * 8 > NUM_CU || N < 24) return;
        target = (int)(NUM_CU / chains);
        const bool gentle = p->eta <= (backward ? 2.5e-4f : 5e-5f) * p->K;
        if (backward && N > (chains > 16 ? 64 : p->io_dtype == OSDN_F32 && p->K == 128 && chains > 8 ? 96 : N)) return;
        if (!gentle) {
            if (backward || N < 64) return;
            min_chunks = 8;
        } else {
            const bool two = p->K == 64 || (!backward && (!retention || (p->io_dtype == OSDN_BF16 && !p->retention_per_channel)));
            if (two && N >= 16 * target) target *= 2;
            // (every workgroup walks the maps of all pieces of its chain, eight at a time; but pieces of more than eight chunks cost more than that walk)
            const int most = N <= 64 ? 16 : N <= 256 ? 32 : (N + 7) / 8;
            if (target > most) target = most;
            min_chunks = backward ? 4 : 2;
        }
    }
    if ((long long)target * chains > MAX_PIECES) target = (int)(MAX_PIECES / chains);
    if (target < 2) return;
    int len = (N + target - 1) / target;
    if (len < min_chunks) len = min_chunks;
    const int P = (N + len - 1) / len;
    if (P < 2) return;
    pieces = P; piece_chunks = len;
    if (p->p1_piece_sweeps >= 1) sweeps = p->p1_piece_sweeps;
}

// Slices of bwd_chain, 16 values or 32 (beside: a phase-1 chain runs on another stream; fp32 I/O at K = 128 always takes 16).
//  - bf16 takes 32 values beside a phase-1 chain: with 16 its workgroups hold twice the CUs, and what they
//    take from that chain, which bounds the pass there, costs more than the kernel gains.  With everything on one stream it takes 16 while the
//    workgroups find a CU each (training step, us, 32 and 16: 16 chains of 128 chunks, V = 256 848 and 836, of 24, V = 128 224 and
//    214, without retention of 32 245 and 234; 8 of 16 163 and 158; 2 of 300 799 and 697; 32 of 40 416 and 410), unless that puts the
//    slices of a chain on more XCDs than slices of 32 (backward pass: 21 chains of 32 chunks, V = 192 167 and 182).
//  - fp32 I/O at K = 64: 16 values while the
//    workgroups find a CU each (64 chains of 32 chunks, V = 64: training step 705 against 721 us; 16 chains of
//    128 chunks, V = 128: 1240 against 1400), above that 32, which read the shared tiles half as often
//    (256 chains of 16 chunks, V = 64: 1109 against 1155; 128 chains, V = 256: 1330 against 1404).
inline bool narrow_backward(const osdn_params *p, long long chains, bool beside) {
    const int slices = p->V / 16;
    if (p->io_dtype == OSDN_F32) return p->K == 128 || chains * slices <= NUM_CU;
    return !beside && chains * slices <= NUM_CU &&
           (chains <= NUM_XCD || chains % NUM_XCD == 0 || slices >= 2 * NUM_XCD || chains_filled_up(slices, chains, true));
}

// Without retention, chunks that never met the box can take the solved form of the reverse
// sweep: a dependent chain shorter than the sweeps' for 0.6 KB more memory traffic per
// token-head.  It pays while the phase-1 chain is what the pass waits for (us of the backward pass, sweeps and solved, V = K
// unless said; beta = sigmoid(N(0, 1)), then about 0.95, where a chunk takes three sweeps; the solved form knows neither):
//  - chains on at most an eighth of the CUs (K = 128, bf16: 32 of 64 chunks 430 and 380, 485 and 380; K = 64: 302 and 250);
//  - with bf16 I/O on a quarter, from 16 chunks on (48 chains, K = 128: 8 chunks 84 and 88, 16 129 and 134, with V = 64 121 and 119; 33 of 8
//    83 and 87, of 16 126 and 123; K = 64, 48 of 8 66 and 65, of 16 99 and 92; K = 64: 40 of 64 339 and 288, 64 of 32 201 and 191, of 64 395 and 352, of 128 639 and 701; K = 128:
//    40 of 64 476 and 443, 527 and 443; V = 64: 64 of 64 514 and 510, 569 and 508, of 128 916 and 1014), but for K = 128 with
//    V >= 128 beyond 48 chains, where the traffic of phase 2 fills the chip (48 of 64 507 and 500, 559 and 501; 64 of 32 319 and
//    328, 350 and 327; 64 of 64 611 and 636, 668 and 637; 64 of 128 1102 and 1200, 1163 and 1200).
// longest: chunks of the longest sequence
inline bool solved_plan(const osdn_params *p, long long chains, int longest, bool retention) {
    const bool bf = p->io_dtype == OSDN_BF16, quarter = bf && longest >= 16 && !(p->K == 128 && p->V >= 128 && chains > 48);
    if (retention) return !p->retention_per_channel && p->p1_solved > 0;       // (the form with a retention gate and any masks)
    return p->p1_solved > 0 || (p->p1_solved == 0 && chains * (quarter ? 4 : 8) <= NUM_CU);
}

// Whether no two rows of K elements of a batch [n[0], n[1], n[2]] stand in one another, by its steps: taken from the smallest on, each is at least
// the extent of what is inside it.  That holds for every slice, reordering and part of an array whose rows are apart; steps that only mesh
// (2 K and 3 K, twice each) are not told from those that meet.
inline bool rows_apart(const long long (&n)[3], const long long (&step)[3], int K) {
    unsigned __int128 extent = (unsigned)K, size[3];
    int axis[3], axes = 0;
    for (int i = 0; i < 3; ++i) {
        size[i] = step[i] < 0 ? -(__int128)step[i] : (__int128)step[i];
        if (n[i] <= 1) continue;
        int at = axes++;
        for (; at > 0 && size[axis[at - 1]] > size[i]; --at) axis[at] = axis[at - 1];
        axis[at] = i;
    }
    for (int i = 0; i < axes; ++i) {
        if (size[axis[i]] < extent) return false;
        extent += size[axis[i]] * (unsigned long long)(n[axis[i]] - 1);
    }
    return true;
}

// Blocks of rows (64 lanes of 16 bytes) of a token that one wavefront of heads_fwd_kernel takes: all of them where every CU then has sixteen wavefronts,
// else as many pairs as leave it sixteen (its loads go in pairs), and one by one below eight.  us, from eight wavefronts with any number and from
// sixteen: 1531 tokens of 8 blocks 8.5 and 7.5, 800 of 12 9.7 and 9.0, fp32 1500 of 8 8.6 and 7.7; 4000 of 2 one by one 8.4, as a pair 7.3.
inline int heads_blocks_per_wave(long long tokens, int blocks) {
    if (tokens * blocks < 2 * 8 * NUM_CU) return 1;
    const long long pairs = tokens * blocks / (2 * 16 * NUM_CU);
    return (int)(pairs < 1 ? 2 : 2 * pairs > blocks ? blocks : 2 * pairs);
}
// Whether an append asks for the next pair of blocks before it writes this one: where the memory and not a wavefront's wait bounds it.  us, one after the
// other and so: 65536 tokens of 6 blocks 176 and 164, 30000 86 and 81, fp32 3120 of 32 51.4 and 50.5; but 3158 of 10 18.8 and 19.4, 858 of 7 7.6 and 7.9.
// (Without the cache's rows it does not pay: 20000 of 2 17.8 and 18.6, 16384 of 10 69 and 70.)
inline bool heads_ahead(long long tokens, int blocks) { return tokens * blocks >= 256 * NUM_CU; }
// Workgroups (four wavefronts) for so many (token, part) pairs: 65536 tokens appended with up to 2048, 4096 and 16384 of them 175, 168 and 163 us
inline int heads_fwd_workgroups(long long items) { return (int)(items < 4 * 16384 ? (items + 3) / 4 : 16384); }
// Heads that a wavefront of append_mx_kernel (read_mx_kernel) takes of its tokens, of which there are `groups`: all where every CU then has sixteen wavefronts
inline int heads_mx_per_wave(long long groups, int heads) {
    const long long per = groups * heads / (16 * NUM_CU);
    return (int)(per < 1 ? 1 : per > heads ? heads : per);
}
// ... of heads_bwd_kernel, each with a row of partial sums: 2 x 8192 x (32 + 8) heads with 1024 and 2048 178 and 179 us (both passes), 4 x 2048 x (16 + 4) of 64 33 and 36
constexpr int HEADS_BWD_WGS = 1024;
inline int heads_bwd_workgroups(long long items) { return (int)(items < 4 * HEADS_BWD_WGS ? (items + 3) / 4 : HEADS_BWD_WGS); }
// Blocks of a token for one of its wavefronts: all where the tokens give every wavefront one, else as few as that takes (fours, as its loads go, from
// four on).  us, all and so: 27 tokens of 48 blocks 31.6 and 5.1, 502 of 20 19.7 and 10.8.
inline int heads_bwd_blocks_per_wave(long long tokens, int blocks) {
    const long long per = tokens * blocks / (4 * HEADS_BWD_WGS);
    return (int)(per < 1 ? 1 : per > blocks ? blocks : per < 4 ? per : per / 4 * 4);
}
// How a call is cut: the blocks of rows of a token's queries, of all its rows (`values`: those of the keys count twice), for one wavefront, and
// how many wavefronts that makes; the workgroups
struct HeadsPlan { int q_blocks, k_blocks, blocks, per_part, parts, workgroups; };
inline HeadsPlan heads_plan(long long tokens, int Hq, int Hk, int K, bool bf16, bool values, bool backward) {
    const int rows = 1024 / (K * (bf16 ? 2 : 4));
    HeadsPlan h{};
    h.q_blocks = (Hq + rows - 1) / rows;
    h.k_blocks = (Hk + rows - 1) / rows;
    h.blocks = h.q_blocks + h.k_blocks * (values ? 2 : 1);
    h.per_part = backward ? heads_bwd_blocks_per_wave(tokens, h.blocks) : heads_blocks_per_wave(tokens, h.blocks);
    h.parts = (h.blocks + h.per_part - 1) / h.per_part;
    h.workgroups = backward ? heads_bwd_workgroups(tokens * h.parts) : heads_fwd_workgroups(tokens * h.parts);
    return h;
}

// Attention over a paged cache: tokens that a sequence of at most max_length may see, counted from a multiple of the tile of 32
constexpr int DECODE_TILE = 32, DEC_THREADS = 256;
// Tokens of a wavefront's tile (wide rows: half, for the registers), and of a unit: a tile for each wavefront of a row, where a workgroup's four take R rows
constexpr int decode_tile(int K, bool bf16) { return bf16 && K <= 128 ? 32 : 16; }
// Workgroups that the registers of a CU hold
constexpr int decode_per_cu(int K, bool bf16) { return K == 64 ? 4 : K == 128 ? (bf16 ? 3 : 2) : bf16 ? 2 : 1; }
constexpr int decode_unit(int K, bool bf16, int R) { return DEC_THREADS / 64 / R * decode_tile(K, bf16); }
// ... over a cache in 4 bits
constexpr int DECODE_MX_TILE = 32;
constexpr int decode_mx_per_cu(int K, bool bf16) { return bf16 ? (K == 64 ? 4 : K == 128 ? 4 : 2) : K == 64 ? 4 : K == 128 ? 2 : 1; }
constexpr int decode_mx_unit(int R) { return DEC_THREADS / 64 / R * DECODE_MX_TILE; }
inline long long decode_span(int max_length, int window) {
    const long long seen = window > 0 && window < max_length ? (long long)window + DECODE_TILE - 1 : max_length;
    return seen < max_length ? seen : max_length;
}
// How a call is cut, for B sequences of `rows` rows (groups of up to 16 query heads of a key head) each: the rows that a workgroup takes together, the
// units of a sequence of max_length, and the shares (0: a row each, and no second kernel).  asked: > 0 shares, -1 a row each, 0 by these rules.
// us; "even": all lengths the same, "uneven": spread from 1 to the longest; four heads of the cache of K = 128 in bf16, head after head, unless said.
//  - a row each, against 512 shares, for rows of a few units, the more so for many rows: 1 x 300 tokens 9.3 and 10.3, 256 x 300 34.2 and 39.7, uneven
//    40 x 400 11.9 and 14.0, 512 x 450 54.5 and 57.9; but 1 x 500 12.0 and 10.3, 16 x 500 14.0 and 12.8, fp32 1 x 200 x 8 13.3 and 10.5.
//  - and for up to 1024 tokens where the rows fill the chip: uneven 200 x 700 38.8 and 42.8, fp32, K = 64, 512 x 1000 x 8 186 and 221; but not so many
//    where a token's heads stand side by side (uneven 200 x 1000 59 and 49, K = 64, 512 x 900 x 8 213 and 171) or in rows of 256 (uneven 200 x 700 x 2
//    48.7 and 40.3), and none where one workgroup is all that a CU holds (fp32, K = 256, uneven 300 x 500 x 2 95 and 81).
//  - of the former, four rows (or two) together, a wavefront each, where a row is no more than a tile and one by one they are more workgroups than
//    the chip holds, or four tiles and half as many again: one by one and so, times 8 heads: uneven 500 x 1 22.0 and 11.1, fp32, K = 256, 94 and 31;
//    300 x 20 17.5 and 11.7; 300 x 70 24.0 and 21.6; but 300 x 128 36.1 and 36.5, K = 256 100 x 250 46.8 and 48.6; 80 x 70 11 % more so, 50 x 16 6 %.
//  - of the latter, four rows (or two) together where the cache holds the heads of a token side by side, so that what is asked for at a time is not
//    each fourth or eighth 256 bytes of it, or where rows share their key head: one by one and so, uneven 64 x 8192 x 8 204 and 185, 512 x 4096 388 and
//    374, 1 x 131072 x 8 113 and 100, 16 x 4096 x 16 106 and 99, K = 64, uneven 64 x 4096 x 8 65 and 56.  Head after head, rows one by one do as well
//    with fewer parts to join (185 and 186, 378 and 384, 99 and 105), but for rows of 128 bytes (64 x 4096 x 8 57.5 and 54.5).
//  - two shares a CU, which start and end together whatever the lengths.  Rows one by one with 256, 512, 768 and 1024: uneven 512 x 4096 392, 379, 382,
//    383, 64 x 8192 x 8 199, 186, 187, 188; 16 x 4096 x 8, K = 256, 100, 104, 121, 106; fp32 115, 102, 119, 102; with 384 and 640, half a share a CU more
//    or less, 434 and 414 for the first.  Three for rows of 64 elements one by one (fp32, or bf16 alone: 64 x 4096 x 8 72.5, 63.5, 57.8, 62.7).
//    One for fp32 and K = 256, whose registers hold one workgroup (8 x 4096 63.5, 68.4, 74.0, 79.4), for four long rows of K = 128 in bf16 together (1 x 131072
//    x 8 99.8 and 102.8, 512 x 4096 374 and 378; but uneven 150 x 700 32.6 and 30.3, 512 x 1000 107 and 106), and for few rows, of which each share is a part to join (with 192, 256, 512 and 768, fp32 K = 64, 1 x 84732 x 1
//    18.7, 18.3, 20.3, 21.8, bf16 2 x 58831 x 2 16.2, 16.1, 18.8, 20.9, K = 128, 4 x 32768 x 1 25.5, 22.1, 22.8, 24.4; but 8 x 4096 x 4 18.4, 19.4, 18.2, 17.5).
//  - and not so many that the parts (an fp32 row of each query head) outweigh what a share reads: 8 x 8000 x 2 with 32 query heads each, 256 and 512
//    shares 31.6 and 35.3.
// Over a cache in 4 bits, whose rows are a quarter as long, what is the same for every row and every call weighs more, and so does the join (us, as above, four heads of
// K = 128 in bf16 unless said):
//  - a row each up to 768 tokens (K = 256: 384), where the second kernel costs more than what it makes shorter.  A row each and shares:
//        1 x 500 x 8             7.1   8.7        16 x 800              9.7  11.0        4 x 300, K = 256      8.8  11.9
//        1 x 1200 x 8           11.9   8.7                                               4 x 700, K = 256     12.7  12.5
//    up to 2048 where every CU has a row:
//        32 x 2000 x 8          18.7  21.8        uneven               17.9  25.5        32 x 3000 x 8 uneven 24.1  22.4
//    and to 3000 where it has two:
//        64 x 3000 x 8          42.6  51.5        uneven               31.5  37.4        512 x 3000            151   160
//        64 x 8192 x 8 uneven   75.3  65.8
//  - four rows together from two rows a CU on, as a share then begins fewer rows.  One by one and together:
//        512 x 4096 uneven       145   128        64 x 8192 x 8        76.5  65.8        1 x 131072 x 8       34.8  37.1 (all shares cut its rows)
//    of heads side by side, whose lines they then share, also from 32 rows and 64 MB on, with two shares a CU:
//        4 x 32000 x 8          62.7  44          K = 64               52.6  32          16 x 4096 x 8        33.4  26.9
//        50 x 8000 x 8           157   114        K = 64                137  80
//        16 x 8000 x 4          26.8  27.5        1 x 131072 x 8       42.7  43.6
//  - two shares a CU, four for rows of 64 elements and where there is about a row for each.  256, 512, 768 and 1024 shares:
//        64 x 4096 x 8, K = 64, uneven            34.4  27.4  26.7  25.5                  40 x 4000 x 8, K = 256   84.3  65.1  58.8  55.9
//        1 x 131072 x 8                           44.6  34.8  37.8  37.1                  16 x 8192 x 8            42.1  34.7  38.1  37.5
//    three from 192 rows of 128 on whose heads lie apart, the codes past the caches.  512, 768 and 1024 shares:
//        512 x 4096 uneven                         119   115.5 118.7                      64 x 4096 x 4            33.9  27.9  29.9
//        256 x 4096 x 8, fp32                      128   121   131                        64 x 8192 x 8            107   107.5 104
//        28 x 8192 x 8 even                       55.3  54.3  55.1                        uneven                   52.4  48.9  45.9 (here four would be better)
//        16 x 8192 x 8                            33.6  36.1  37.2                        512 x 4096 uneven, heads side by side   140.5  145  146
inline bool decode_mx_each(long long span, long long all, int K) {
    return span <= (all >= 2 * NUM_CU ? 3000 : all >= NUM_CU ? 2048 : K == 256 ? 384 : 768);
}
struct DecodePlan { int row_group, shares; long long units; };
// Rows of more than 64 MB, a quarter of the memory-side cache, from which a program that comes back to less of them soon would have them
constexpr bool decode_mx_large(long long rows, int K) { return rows * (K + K / 16) > 64LL << 20; }
// Whether a call over a cache in 4 bits loads its codes past the caches: rows of a head lie next to each other (K = 128: or are chosen ones), so that a load takes whole lines of 128 bytes which no
// other wants, and those that it may read are many (us, through the caches and past them: uneven 512 x 4096 x 4 heads 131 and 121, K = 64 84.1 and 79.7, 512 x 1000 x 4 59.8 and 57.2, K = 64
// 42.3 and 40.7, 64 x 4096 x 4 39.7 and 36.1, 4 x 32768 x 8 38.1 and 35.3, K = 64 29.5 and 28.6, 1 x 131072 x 8 38.2 and 37.5, K = 64 29.0 and 28.1; but 512 x 200 x 4, called again on
// what the memory-side cache holds, 18.7 and 21.0, 1 x 32768 x 8 16.4 and 17.0; heads side by side, whose lines wavefronts share, uneven 512 x 4096 x 4 142 and 148, K = 64 97.5 and
// 112; K = 256, half a line a load, 62.6 and 66.0.  Chosen pages of 48 x 8 heads, 32 of 64 tokens, side by side 51.4 and 47.6, apart 29.7 and 28.8, of 96 x 8, 128 of 16 tokens, 79.0 and 75.1,
// apart 46.0 and 41.4, K = 64 59.0 and 59.8, apart 32.6 and 31.0; of 300 x 2 side by side, one line for both, 112 and 115.)
constexpr bool decode_mx_once(long long rows, int K, long long token_step, bool chosen) {
    return K <= 128 && (token_step == K / 2 || (chosen && K == 128)) && decode_mx_large(rows, K);
}
inline DecodePlan decode_plan(int B, int rows, int max_length, int window, int K, bool bf16, int part_heads, bool heads_together, int asked, bool mx = false) {
    const long long span = decode_span(max_length, window), all = (long long)B * rows;
    const int tile = mx ? DECODE_MX_TILE : decode_tile(K, bf16), alone = mx ? decode_mx_unit(1) : decode_unit(K, bf16, 1), held = (mx ? decode_mx_per_cu(K, bf16) : decode_per_cu(K, bf16)) * NUM_CU;
    const bool beside = heads_together && rows % 2 == 0;
    const bool few_units = span <= (K == 64 ? 4 : bf16 ? 3 : 2) * alone || (span <= 4 * alone && all >= NUM_CU / 2);
    const bool full = all >= held && held > NUM_CU && span <= (beside || K == 256 ? 512 : 1024);
    const bool each = asked < 0 || (asked == 0 && (mx ? decode_mx_each(span, all, K) : few_units || full));
    const bool together = each ? (span <= tile && all > held) || (span <= 4 * tile && 2 * all > 3 * held) : mx ? all >= 2 * NUM_CU || (heads_together && K <= 128 && all >= 32 && decode_mx_large(all * span, K)) : beside || (K == 64 && bf16);
    DecodePlan p{};
    p.row_group = together && rows % 4 == 0 ? 4 : together && rows % 2 == 0 ? 2 : 1;
    const int unit = mx ? decode_mx_unit(p.row_group) : decode_unit(K, bf16, p.row_group);
    p.units = span < 1 ? 1 : (span + unit - 1) / unit;
    const long long groups = all / p.row_group;
    const int per_cu = mx ? (heads_together && p.row_group > 1 ? 2 : K == 128 && !heads_together && all >= 3 * NUM_CU / 4 ? 3 : K == 64 || (all >= NUM_CU && all < 2 * NUM_CU) ? 4 : 2) : all <= 16 || (K == 256 && !bf16) || (K == 128 && bf16 && p.row_group == 4 && span > 1024) ? 1 : K == 64 && p.row_group < 4 ? 3 : 2;
    const long long worth = groups * span / (16 * part_heads), most = per_cu * NUM_CU < worth ? per_cu * NUM_CU : worth > NUM_CU ? worth : NUM_CU;
    p.shares = each ? 0 : asked > 0 ? asked : (int)(groups * p.units < most ? groups * p.units : most);
    return p;
}

// Workgroups for the places of a batch's tokens, each of which makes the batch's running sums for itself (us, of 4096, 2048 and 1024 tokens each: 96 requests of 683 7.2, 6.1, 5.9, 2000 of 30
// 13.1, 11.5, 10.8, 32 of 128 6.3, 5.1, 4.7)
inline int plan_workgroups(int tokens) { return tokens <= 1024 ? 1 : (int)((tokens + 1023LL) / 1024 < NUM_CU ? (tokens + 1023LL) / 1024 : NUM_CU); }
// Rows of a page table that a call with an index of them may have (two bits each in LDS)
constexpr int PLAN_MAX_ROWS = 1 << 17;
// Selection of pages: whether a row's workgroup makes the scores itself, which saves a launch, or a launch of many workgroups does.  bytes: of a page's bounds.  (us, a launch of their own
// and so, pages of 512 bytes: 4 rows of 128 8.0 and 6.8, of 256 7.7 and 8.1, 8 of 4096 14.6 and 60; 64 rows of 256 9.4 and 8.9, of 512 12.1 and 12.2, of 768 14.3 and 16.4, of 1024 in fp32
// 14.8 and 16.2; 128 of 512 14.7 and 12.8, uneven 13.2 and 12.4; 256 of 1024 38.5 and 33.9, of 4096 124 and 109; uneven 384 of 512 19.1 and 18.0, 512 of 128 13.5 and 10.1.)
inline bool select_scores_itself(long long rows, int pages, int bytes) {
    return pages <= 4096 && (rows >= NUM_CU || (long long)pages * bytes <= (rows >= 64 ? 1 << 18 : 1 << 16));
}
// Workgroups (four wavefronts, a page and head each) for the bounds of pages: a launch has less than 2^32 threads
inline unsigned bounds_workgroups(long long items) { return (unsigned)(items < 4LL << 22 ? (items + 3) / 4 : 1 << 22); }
// Pages of a sequence that are counted, and that a query may choose: a step of the counter, SELECT_STEPS times 16 pages for each of up to 4 NUM_CU workgroups, then stays in 32 bits
constexpr int SELECT_MAX_PAGES = 1 << 30, SELECT_STEPS = 16;
// Workgroups (four wavefronts, four pages each at a time) for the scores of a sequence's pages of one group of key heads
inline unsigned select_chunks(int B, int Hk, int heads, int pages) {
    const long long others = (long long)B * ((Hk + heads - 1) / heads), want = (4 * NUM_CU + others - 1) / others, most = (pages + 15) / 16;
    return (unsigned)(want < most ? want : most);
}

// (constexpr, as what follows: for the device too)
// The tokens [lo, end) that a query of a sequence sees; none where `broken`: what the caller promised and did not keep makes the result NaN, and nothing
// outside the cache is read.  Without a token nothing is looked up, so the sequence is not asked for either.  Both lie in [0, max_length] whatever
// stands for the length, so that counting on from them by tiles stays in 32 bits.
struct Seen { int lo, end; bool broken; };
constexpr Seen seen_tokens(int length, int seq, int n_seqs, int max_length, int window, int page_shift, int max_pages) {
    const bool any = length > 0;
    const bool broken = any & (((unsigned)seq >= (unsigned)n_seqs) | (length > max_length) | ((length - any) >> page_shift >= max_pages));
    const int end = any & !broken ? length : 0;
    return Seen{(window > 0) & (end > window) ? end - window : 0, end, broken};
}
// Where the first unit of a row begins, and how many of `unit` tokens it has; one where there is nothing to see, so that its zeros (or NaN) are written
constexpr int seen_begin(const Seen &s) { return s.lo & ~(DECODE_TILE - 1); }
constexpr int seen_units(const Seen &s, int unit) { return s.end > 0 ? (s.end - seen_begin(s) + unit - 1) / unit : 1; }

// The even shares of n units among W workgroups: the first n % W have one more.  `owner`: the share that a unit falls to.
struct Shares {
    int q, rem;
    constexpr Shares(int n, int W) : q(n / W), rem(n % W) {}
    constexpr int begin(int w) const { return w * q + (w < rem ? w : rem); }
    constexpr int owner(int unit) const { return unit < rem * (q + 1) ? unit / (q + 1) : rem + (unit - rem * (q + 1)) / q; }
};
// Where share w leaves its part of a row that it does not hold whole: a share has at most two of those, its first row and its last.  A row's
// parts are those of its first share, which may be either, and of the ones behind it, which begin with it.
constexpr int part_slot(int w, bool first_of_share) { return 2 * w + (first_of_share ? 0 : 1); }
constexpr int part_of_row(int first_slot, int i) { return i == 0 ? first_slot : (first_slot & ~1) + 2 * i; }

}  // namespace osdn
