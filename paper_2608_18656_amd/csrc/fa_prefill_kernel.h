// fa_prefill_kernel.h -- prefill attention forward on gfx950 matrix cores: the
// kernel that fa_prefill.hip, fa_window.hip and fa_prefix.hip launch.
//
// Work split.  A workgroup owns NS (query head, 32-row block) slots that read
// the same key/value head: four, or eight (1 and 2 exist for the packing
// ablation).
// When the group size G = Hq/Hkv allows, up to four of the slots
// are query heads of one key/value group at the same rows -- the GPU form of
// the inter-head packing of Sec. 4.1.1 and the GQA reuse of Sec. 4.1.2 (iv):
// every K/V tile staged in LDS serves all slots of the workgroup, and slots
// of different heads share one causal extent; the other slots are
// consecutive row blocks.  Every wave handles 32 rows and 32 keys of each
// tile.  At D = 64 a slot has two waves (64-key tiles; wave kh takes keys
// 32 kh .. 32 kh + 31) whose states are merged through LDS at the end; at
// D = 128 one wave (32-key tiles).
//
// Per wave and tile, the blocked streaming softmax (Alg. 2 state carry over
// the per-key recurrence of Alg. 1):
//   S^T = K Q^T        32x32x16 MFMA; A = 32 K rows from LDS, B = the wave's
//                      32 query rows, kept in registers for the whole kernel
//   softmax            scores stay in the MFMA result registers; lane l owns
//                      query row l%32 (a row maximum needs one exchange with
//                      lane l^32); scale and log2(e) fold into one
//                      multiply-add ahead of exp2; weights packed to fp16
//   O^T += V^T P^T     32x32x16 fp16 MFMA; P straight from the score registers,
//                      V^T operands read from the row-major V tile with the
//                      transposing LDS read
// Staging.  K tiles, and fp16 V tiles, go from memory to LDS directly (no
// registers, no LDS store instructions); bf16 V passes through registers to
// become fp16.  The transposing read (8 bytes a lane) delivers 249 bytes per
// clock and CU when the four rows that 32 lanes read lie in different quarters
// of the 64 banks, as much as the plain 16-byte read (255), and 64 to 128
// when they do not; LDS stores take 62 (4 bytes a lane) to 79 (16 bytes).  So
// the tiles are laid out for the reads, by swizzling the addresses that a
// lane loads from, and nothing is transposed in the copy.  Against a copy
// through registers that wrote V transposed with 4-byte stores, timed in turn:
// D = 128, 2 x 32/8 heads, 4096 rows, fp16, causal: 299 -> 276 us; D = 64,
// 16/1 heads, 16384 rows, fp16: 597 -> 581 us; 32/8 heads, 2048 rows, bf16:
// 30.3 -> 28.9 us.
// What bounds it.  Large grids run at the card's power limit (1.85 to 2.0 GHz;
// with zeros for data, at 2.35 GHz, D = 128 takes 184 us and the 16384-row
// call 447 us), so what saves energy per tile saves time.  At full clock a
// wave's 32 x 32 block at D = 64 costs about 440 of its SIMD's cycles from
// registers alone: 256 of MFMA, and 35 vector instructions of 4 cycles and 16
// exponentials of 8, which overlap with them only in part.
// The exponent base only moves when a tile's weights against the current base
// grow too large (see the softmax step below), so the accumulator rescale is
// skipped on most tiles; sum and accumulator always share the base, so the
// result is unchanged.
// A wave's steps run in order; latency is hidden by the other waves of the
// SIMD (four-slot layouts: two 8-wave workgroups per CU at D = 64, four waves
// per SIMD within 128 VGPRs; three 4-wave ones at D = 128, three waves per
// SIMD within 168 VGPRs; their barriers are independent).  With three LDS
// stages the tile two steps ahead is loaded during a step.  Matrix
// instructions are issued at raised wave priority.
// Masked scores are -inf and give exactly 0 (the exponent factor is kept
// strictly positive, also for scale = 0).  Keys past the end read as zero
// (buffer loads with the tensor's extent as the range) and are masked.
// Normalisation happens once, after the last tile.
#pragma once

#include <type_traits>

#include "fa_common.h"

namespace fa {
namespace {

constexpr int WR = 32;        // query rows per slot
constexpr int NSLOT = 4;      // slots per workgroup where nothing speaks for another number
constexpr float kMaxLaneSum = 4096.0f;   // largest 16-weight lane sum kept without a rescale

// What a launch attends to.
//   ALL     every key of the sequence, up to the row's own if causal
//   WINDOW  the `window` keys up to the row's own and the first `sinks` (causal):
//           tiles between the two parts are not visited, nor are a tile's keys
//           that a wave's rows do not see multiplied
//   PARTS   sequences that share a prefix, their keys in parts: workgroups of the
//           prefix, whose rows are those of all sequences, and workgroups of one
//           sequence's own keys, both a split of the keys.  The B Nq G rows of a
//           key/value head are numbered together (token t, head e of the group:
//           row t G + e).  Each leaves a partial result (accumulator, base, sum).
//   JOIN    the shared keys, then the sequence's own (paged: the table has both)
//   WINDOW_PARTS  WINDOW with each row block's tiles split over workgroups, which
//           leave partial results
enum { ALL = 0, WINDOW = 1, PARTS = 2, JOIN = 3, WINDOW_PARTS = 4 };

struct PrefillArgs {
    const void *q, *k, *v;
    void *o;
    float *lse;
    int B, Hq, Hkv, Nq, Nk;
    float c;          // max(|scale|, tiny) * log2(e), > 0
    unsigned qsign;   // 0x80008000 to negate q (scale < 0), else 0
    int G;            // query heads per key/value head
    int HW, lgHW;     // query heads per workgroup (1, 2, 4 or 8) and its logarithm
    int nmb;          // row blocks of 32 * (slots / HW) rows
    Divisor per_mb;   // workgroups per row block: B * Hkv * (G / HW)
    Divisor nhg;      // head groups per key/value head (G / HW)
    Divisor nkv;      // key/value heads
    int ranked;       // > 0: uneven sequences are taken by length, the first `ranked` of their row
                      // blocks longest first, the others shortest first
    Divisor per_seq;      // workgroups per sequence and row block: Hkv * (G / HW)
    Divisor row_blocks;   // nmb
    int first;        // row blocks taken longest first, the others shortest first
    const int *seqlens;   // valid keys per batch element (NULL: Nk for all)
    const int *block_table;   // paged K/V: page of each key block (see Problem)
    int page_size, max_pages, num_pages;
    // all but ALL
    Divisor page_div;     // page_size
    int window, sinks;    // WINDOW, WINDOW_PARTS: at most Nk each
    // PARTS, JOIN: k, v and Nk are the sequences' own keys (paged: of all)
    const void *k_prefix, *v_prefix;
    int prefix;           // keys of the prefix
    int own;              // keys that a sequence can have of its own
    int counted;          // keys of the prefix that the lengths count: prefix, or 0
    // PARTS
    int first_page;       // table entry of a sequence's own first page
    int causal, rows;     // rows: B Nq G
    int prefix_blocks;    // workgroups of the prefix, ahead of the others
    Divisor own_splits;   // of a sequence's own keys
    Divisor batch, tokens, group;   // B, Nq, G
    // PARTS, WINDOW_PARTS
    Divisor splits;       // of the prefix's keys, of a row block's tiles
    float *opart, *mpart, *lpart;   // [token][head][slots] partial results (PARTS: the prefix's, then the own ones)
    int slots;
};

// Tile shape per head size.  Every wave handles 32 query rows and 32 keys of
// a tile.  D = 64: two waves per slot (64-key tiles, key halves merged at the
// end), 8-wave workgroups of at most 128 VGPRs, two per CU (four waves per
// SIMD).  D = 128: the accumulator (64 VGPRs) and Q (32) leave no room for
// that, so one wave per slot (32-key tiles) and 4-wave workgroups, three per
// CU (three waves per SIMD, from independent workgroups; operands are read
// from LDS in small groups to fit 168 VGPRs).  Three LDS stages (two for
// one- and two-slot workgroups).
// NS, the slots per workgroup (all reading one key/value head, each staged
// tile serving all of them), is 4, or 8 for some large grids (eight_slots); 1
// and 2 exist for the packing ablation (fewer slots stage more per thread, so
// they hold fewer waves per SIMD).
template <int D, int NS = NSLOT> struct Cfg {
    static constexpr int NQ = D == 64 ? 2 : 1;       // waves per slot
    // waves per SIMD (what the registers allow; fewer slots stage more per thread)
    static constexpr int WPE = D == 64 ? (NS >= 4 ? 4 : NS == 2 ? 3 : 2) : (NS >= 4 ? 3 : NS == 2 ? 2 : 1);
    static constexpr int NWG = NS * NQ;              // waves per workgroup
    static constexpr int WPC = NWG >= 4 * WPE ? 1 : 4 * WPE / NWG;   // workgroups per CU (registers)
    static constexpr int BC = 32 * NQ;               // keys per tile
    static constexpr int NT = 64 * NWG;              // threads per workgroup
    static constexpr int NSTAGE = NS >= 4 ? 3 : 2;   // LDS tile stages (small workgroups: two, for room on the CU)
    static constexpr int AHEAD = NSTAGE - 1;         // a tile is loaded this many steps ahead
    static constexpr int KSZ = BC * D;               // K tile: BC rows of D elements, chunks swizzled
    static constexpr int VSZ = BC * D;               // V tile: the same shape
    static constexpr int STAGE = KSZ + VSZ;
    static constexpr int MERGE = NQ > 1 ? NS * (NQ / 2) * ((D / 32) * 16 + 2) * 64 : 0;  // floats
    static constexpr int WORDS = (NSTAGE * STAGE) > (2 * MERGE) ? NSTAGE * STAGE : 2 * MERGE;
    // Staging split: a tile is eight 1 KiB pieces of K and eight of V, 64
    // consecutive 16-byte chunks each.  A wave takes NP pieces of both, or in
    // a 16-wave workgroup one piece of one (waves 0 .. 7 V, 8 .. 15 K).
    static constexpr int PIECES = KSZ * 2 / 1024;
    static constexpr bool SPLIT = NWG > PIECES;
    static constexpr int NP = SPLIT ? 1 : PIECES / NWG;
    static_assert(PIECES == 8 && (SPLIT ? NWG == 2 * PIECES : PIECES % NWG == 0), "staging split");
};

// Valid keys that sequence b has of its own (PARTS, JOIN).
__device__ __forceinline__ int own_keys(const PrefillArgs &a, int b) {
    return a.seqlens ? min(max(min(max(a.seqlens[b], 0), a.prefix + a.own) - a.counted, 0), a.own) : a.own;
}

// Keys of the prefix that a row sees (PARTS): fewer than all where it lies in the
// prefix (causal), or its sequence is shorter.
__device__ __forceinline__ int prefix_keys(const PrefillArgs &a, int row) {
    const int t = a.group.div(row), b = a.tokens.div(t);
    int n = a.prefix + a.own;
    if (a.seqlens) n = min(min(max(a.seqlens[b], 0), n) + a.prefix - a.counted, n);
    if (a.causal) n += t - b * a.Nq + 1 - a.Nq;
    return min(max(n, 0), a.prefix);
}

template <typename TIN, typename TOUT, int D, int NS, bool CAUSAL, bool PAGED, int MODE = ALL>
__global__ __launch_bounds__((Cfg<D, NS>::NT)) __attribute__((amdgpu_waves_per_eu((Cfg<D, NS>::WPE), (Cfg<D, NS>::WPE)))) void prefill_kernel(PrefillArgs a) {
    using S = typename TIN::scalar;
    using V8 = typename TIN::vec8;
    using SM = Cfg<D, NS>;
    constexpr int NSLOT = NS;
    constexpr int NQ = SM::NQ, BC = SM::BC, NT = SM::NT, NSTAGE = SM::NSTAGE;
    constexpr int KSTEPS = D / 16;          // QK^T contraction steps
    constexpr int DT = D / 32;              // output column tiles
    constexpr int CPR = D / 8;              // 16-byte chunks per row
    constexpr bool IN_BF16 = __is_same(TIN, bf16_t), SEGMENTS = MODE == JOIN && !PAGED;
    constexpr bool WIN = MODE == WINDOW || MODE == WINDOW_PARTS, JUMPS = WIN || MODE == PARTS;   // JUMPS: not all tiles are visited

    __shared__ __attribute__((aligned(1024))) unsigned short smem[SM::WORDS];

    const int tid = threadIdx.x;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l = tid & 63, lq = l & 31, lh = l >> 5;
    const int kh = w / NSLOT, slot = w % NSLOT;   // kh: the wave's 32 keys of a tile
    const int RB = NSLOT >> a.lgHW;
    const int wg = blockIdx.x;
    const int bid = MODE == WINDOW_PARTS ? (int)a.splits.div(wg) : wg;
    // Row block of this workgroup.  Latest rows (most keys) first, so that
    // the short causal blocks fill the tail; when the whole grid is resident
    // at once, only one workgroup for every CU in that order and the others
    // shortest first, so that workgroups sharing a CU carry about the same
    // total work (one per CU rather than half of the grid, us: 32/8 heads,
    // D = 64, 1200 rows 21.9 -> 20.1; D = 128, 1100 rows 30.6 -> 29.0, 3000 rows
    // 93.5 -> 89.7).  With lengths of their own that differ, sequences are
    // taken by length and rows within them, in that same pattern: in the order
    // of the batch two workgroups of one sequence share a CU, and the CUs of the
    // long ones finish last (4 x 32/8 heads, 512 rows, 4096 to 1024 keys, D = 64
    // 68 -> 54; 16 such sequences 250 -> 210; 6 of 1024 rows, D = 128 288 -> 250).
    // About equal ones stay in the order of the batch, where workgroups that
    // share a CU share its L1 as well (4 x 4096 keys 83 against 86 by rank), and
    // so do those of short caches, where ranking (0.5 us, 1.5 for 40 and more
    // sequences, ahead of the first load) costs more than it gives (in the
    // order of the batch, which is by length, against ranked, D = 64: 43 x 8/8
    // heads, 32 rows, 256 keys 9.5 / 11.0, 512 12.6 / 13.8, 1024 17.6 / 18.6, but
    // in a random one 21.0 / 18.7; 12 x 32/4, 128 rows, 256 keys 11.9 / 12.1,
    // 512 14.8 / 14.1).  Over 110 batches of 512 to 6000 keys, with 20 to 40
    // keys a sequence, ranking costs 5 % where they come by length and gives 2 in
    // a random order; from 40 on it gives 1 and 5.
    const int q_ = a.per_mb.div(bid);
    int mb = q_ < a.first ? a.nmb - 1 - q_ : q_ - a.first;
    int rest = bid - q_ * a.per_mb.d;
    int b = -1, len = a.Nk;
    if ((MODE == ALL || MODE == WINDOW) && a.ranked > 0) {
        const Lengths lens(a.seqlens, a.B, l);
        if (lens.uneven()) {
            const int u = a.per_seq.div(bid);
            rest = bid - u * a.per_seq.d;
            const int j = u < a.ranked ? u : a.B * a.nmb - 1 - (u - a.ranked), r = a.row_blocks.div(j);
            mb = a.nmb - 1 - (j - r * a.nmb);
            b = lens.nth_longest(r);
        }
        if (b < 0) b = a.nkv.div(a.nhg.div(rest));
        len = lens.of(b);
    }
    const int bg = a.nhg.div(rest), hg = rest - bg * a.nhg.d;
    int b0 = a.nkv.div(bg), g = bg - b0 * a.nkv.d;
    // PARTS: the prefix's workgroups, or a sequence's: split, rows and their bounds
    bool own = false;
    int split = 0, nsplit = 1, part_row0 = 0, part_rows = 0;
    if constexpr (MODE == PARTS) {
        own = bid >= a.prefix_blocks;
        const int r = own ? bid - a.prefix_blocks : bid;
        const int u = own ? a.own_splits.div(r) : a.splits.div(r);
        nsplit = own ? a.own_splits.d : a.splits.d;
        split = r - u * nsplit;
        const int t = a.nkv.div(u);
        g = u - t * a.nkv.d;
        mb = own ? (int)a.batch.div(t) : t;
        b0 = own ? t - mb * (int)a.batch.d : 0;
        part_row0 = b0 * a.Nq * a.G;
        part_rows = own ? part_row0 + a.Nq * a.G : a.rows;
    }
    if ((MODE != ALL && MODE != WINDOW) || a.ranked == 0) {
        b = b0;
        if (MODE != PARTS && a.seqlens) len = a.seqlens[b];
    }
    const int G = a.G;
    const int hs = slot & (a.HW - 1), rs = slot >> a.lgHW;
    const int row0_wg = mb * (WR * RB) + part_row0;
    const int row0 = row0_wg + rs * WR;
    const int qi = row0 + lq;
    const int Nq = MODE == PARTS ? part_rows : a.Nq;
    const int tok = MODE == PARTS ? (int)a.group.div(min(qi, Nq - 1)) : 0;   // the row's token (PARTS)
    const int h = MODE == PARTS ? g * G + (min(qi, Nq - 1) - tok * G) : g * G + hg * a.HW + hs;
    // Valid keys of this batch element: with per-sequence lengths the K/V
    // tensors hold a.Nk rows per batch element of which the first seqlens[b]
    // are valid, and the queries are the sequence's last Nq positions.
    // PARTS: of the part: the sequence's own, or of the prefix, in pages, those that
    // some row of the workgroup sees: what lies behind the longest sequence is not
    // read, and may hold anything.  JOIN: of both.
    int valid = min(max(len, 0), a.Nk);
    if constexpr (MODE == PARTS) {
        valid = own ? own_keys(a, b0) : a.prefix;
        if (!own && a.counted) {   // (a contiguous prefix is every sequence's, whole)
            static_assert(WR * NSLOT == 128, "two rows a lane");
            const int row = row0_wg + l;
            int n = max(prefix_keys(a, min(row, Nq - 1)), prefix_keys(a, min(row + 64, Nq - 1)));
            if (__builtin_amdgcn_ballot_w64(n == a.prefix) == 0) {
#pragma unroll
                for (int x = 32; x > 0; x >>= 1) n = max(n, __shfl_xor(n, x));
                valid = n;
            }
        }
    }
    if constexpr (SEGMENTS) valid = a.prefix + own_keys(a, b);
    const int Nk = __builtin_amdgcn_readfirstlane(valid);
    const int off = Nk - Nq;

    // Key extents: workgroup, this slot, and keys every row of the slot sees.
    const int last_wg = min(row0_wg + WR * RB, Nq) - 1;
    const int kend_wg = CAUSAL ? min(Nk, last_wg + off + 1) : Nk;
    const bool live = row0 < Nq;
    int kfree_w = CAUSAL ? min(Nk, row0 + off + 1) : Nk;
    int ntiles = (kend_wg + BC - 1) / BC;
    // The tiles visited: the first `near` ones and those from near + gap on.
    // WINDOW: the sinks' and, from the first row's window on (first_key), the others.
    // The keys between count as not there, so that what they hold has no part in the
    // result: the view of the last sink's tile ends, and that of the window's first
    // tile begins, at the key itself.  That can be one tile, visited twice (gap -1).
    // Sinks that reach the window are no part of their own.
    // JOIN: the prefix's tiles are the first `near`, the own ones follow.
    int near = 0, gap = 0, first_key = 0, sinks = 0;   // sinks: in a part of their own
    int rlim = 0;   // PARTS: keys of the part that the lane's row sees
    int first = 0;   // WINDOW_PARTS: visited tiles ahead of the split's
    if constexpr (WIN) {
        first_key = max(row0_wg + off + 1 - a.window, 0);
        first_key = first_key > a.sinks ? first_key : 0;
        sinks = first_key > 0 ? a.sinks : 0;
        near = (sinks + BC - 1) / BC;
        gap = first_key / BC - near;
        ntiles = max(ntiles - gap, 0);
    }
    if constexpr (MODE == WINDOW_PARTS) {
        split = wg - bid * (int)a.splits.d;
        const int q = a.splits.div(ntiles), each = q + (q * (int)a.splits.d != ntiles);
        first = min(split * each, ntiles);
        ntiles = min(ntiles - first, each);
    }
    if constexpr (MODE == PARTS) {
        const int each = (ntiles + nsplit - 1) / nsplit;
        gap = min(split * each, ntiles);
        ntiles = min(ntiles - gap, each);
        rlim = Nk;
        if (own) {
            if (a.causal) rlim = min(Nk - a.Nq + (tok - (int)a.tokens.div(tok) * a.Nq) + 1, Nk);
        } else if (a.causal || a.counted) {   // rows that lie in the prefix, sequences shorter than it
            rlim = prefix_keys(a, min(qi, Nq - 1));
        }
        // some row does not see all of the part: every tile is masked
        if (__builtin_amdgcn_ballot_w64(rlim < Nk)) kfree_w = 0;
    }
    if constexpr (SEGMENTS) {
        near = (a.prefix + BC - 1) / BC;
        if (kend_wg > a.prefix) ntiles = near + (kend_wg - a.prefix + BC - 1) / BC;
    }

    // Q rows of this lane (B operand of S^T = K Q^T).
    V8 qf[KSTEPS];
    {
        const int qrow = min(qi, Nq - 1);
        const size_t qtok = MODE == PARTS ? (size_t)tok : (size_t)b * Nq + qrow;
        const S *qp = reinterpret_cast<const S *>(a.q) + (qtok * a.Hq + h) * D + 8 * lh;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            uint4_t u = ld16(qp + 16 * ks);
            u ^= a.qsign;
            qf[ks] = as_vec8<V8>(u);
        }
    }

    // Tile staging.  K, and fp16 V, go from memory to LDS directly (no
    // registers, no store instructions); bf16 V passes through registers,
    // where it becomes fp16.  A tile's rows lie in LDS without padding, row r's
    // 16-byte chunk c at chunk position c ^ kswz(r) (K) or c ^ vswz(r) (V), so
    // that 16 lanes reading one K chunk of 16 rows, and 32 lanes reading four
    // V rows' 64-byte segments, meet all 64 banks.  A lane's place in LDS is
    // fixed by the load (64 consecutive chunks per instruction), so the swizzle
    // is applied to the address it loads from.  Loads are buffer loads: the
    // tile's first key row is the (scalar) base and each lane keeps a fixed
    // byte offset; chunks past the end of the view become zeros.
    constexpr int NP = SM::NP;
    const bool dok = !SM::SPLIT || w >= SM::PIECES, dov = !SM::SPLIT || w < SM::PIECES;   // wave-uniform
    const size_t row_elems = (size_t)a.Hkv * D;      // elements between consecutive keys
    const int row_bytes = (int)(row_elems * sizeof(S));
    auto kswz = [](int r) { return D == 64 ? (r >> 1) & 7 : r & 15; };
    auto vswz = [](int r) { return D == 64 ? ((r >> 1) & 1) << 2 : (r & 3) << 2; };
    const int piece = SM::SPLIT ? w % SM::PIECES : w;    // first piece; the next ones NT / 64 further
    int koff[NP], voff[NP];                              // tile-relative byte offsets
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int q = 64 * (piece + (NT / 64) * j) + l, r = q / CPR, c = q % CPR;
        koff[j] = r * row_bytes + 16 * (c ^ kswz(r));
        voff[j] = r * row_bytes + 16 * (c ^ vswz(r));
    }
    // PARTS, paged WINDOW: bf16 V also goes to LDS directly, as it is, and becomes fp16 in
    // its place once it is there.  A paged window has no registers left to hold it during
    // a step (29 would spill); PARTS takes less time so where its grid is full (64 x 32/8
    // heads behind 8192 keys 43.5 us against 49.0 through registers; 8 x 8 rows 24.5
    // against 23.2).  Contiguous windows have them (32/8 heads, D = 128, 4096 rows, window
    // 1024 80.5 us against 82.7 by way of LDS), and so has JOIN (8 x 256 rows behind 4096 +
    // 512 keys 154.2 against 157.8).
    constexpr bool RAW = IN_BF16 && (MODE == PARTS || (WIN && PAGED)), VREG = IN_BF16 && !RAW;
    typedef uint4_t vregs_t[VREG ? NP : 1];
    vregs_t vr;   // bf16: the next tile's V chunks, in flight during a step
    // Scalar state of the next tile to load: the address of its first key row
    // in K and V, which advances by one tile per load, and its number.  The
    // buffer view of a tile ends after its last valid key (keys past it read
    // as zero): a full tile's extent for the first Nk / BC tiles, then that of
    // the remaining keys, if any (one tile's extent fits 31 bits: tile_fits).
    const bool prefix_first = SEGMENTS || (MODE == PARTS && !own);   // the first tile is one of the prefix
    const size_t head0 = ((size_t)(MODE == PARTS ? b0 : b) * a.Nk * a.Hkv + g) * D;
    const S *kbase = reinterpret_cast<const S *>(prefix_first ? a.k_prefix : a.k);
    const S *vbase = reinterpret_cast<const S *>(prefix_first ? a.v_prefix : a.v);
    const S *ktile = kbase + (PAGED ? 0 : prefix_first ? (size_t)g * D : head0);
    const S *vtile = vbase + (PAGED ? 0 : prefix_first ? (size_t)g * D : head0);
    const int tile_bytes = (BC - 1) * row_bytes + D * (int)sizeof(S);
    auto bytes_of = [&](int rows) { return rows > 0 ? (rows - 1) * row_bytes + D * (int)sizeof(S) : 0; };
    int full_tiles = SEGMENTS ? a.prefix / BC : Nk / BC - gap;   // (of those visited)
    int last_bytes = bytes_of(SEGMENTS ? a.prefix % BC : Nk % BC);
    int tload = JUMPS ? first : 0;   // tiles visited ahead of it
    // paged K/V: the pool of pages, at head g.  Tiles are loaded in order
    // and a page holds a whole number of tiles, so the page index and the
    // offset inside the page advance without a division.  The wave holds 64
    // table entries, one per lane, and the next 64, read with vector loads
    // through a view of this sequence's row of the table (entries past the row
    // read as zero): no scalar load (whose counter the LDS reads share) is in
    // flight during a step, and no wait for an entry stands between the loads
    // of two tiles, where it would wait for the tiles as well (with the entry
    // of the following page loaded alone, 5 x 32/4 heads, 61 rows, 7680 keys,
    // D = 64, pages of 64 took 115 us against 78 for contiguous keys).
    const int page0 = MODE == PARTS && own ? a.first_page : 0;
    const __amdgpu_buffer_rsrc_t trs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int *>(PAGED ? a.block_table + (size_t)(MODE == PARTS ? b0 : b) * a.max_pages + page0 : nullptr), (short)0,
        PAGED ? (a.max_pages - page0) * 4 : 0, 0x00020000);
    const size_t page_elems = (size_t)a.page_size * row_elems;
    int pidx = 0, poff = 0;   // page index and key offset of the next tile
    int tcur = 0, tnx = 0;    // lane i: table entries of pages 64 (pidx / 64) + i and 64 further
    if constexpr (PAGED) {
        tcur = __builtin_amdgcn_raw_buffer_load_b32(trs, 4 * l, 0, 0);
        tnx = __builtin_amdgcn_raw_buffer_load_b32(trs, 4 * (64 + l), 0, 0);
    }
    // past the tiles that are not visited: to tile t, from tile 0; paged: to key `key` of
    // page `page`
    auto go_to_page = [&](int page, int key) __attribute__((always_inline)) {
        pidx = page;
        poff = key;
        const int at = 4 * ((pidx & ~63) + l);
        tcur = __builtin_amdgcn_raw_buffer_load_b32(trs, at, 0, 0);
        tnx = __builtin_amdgcn_raw_buffer_load_b32(trs, at + 256, 0, 0);
        const int p = min(max(__builtin_amdgcn_readlane(tcur, pidx % 64), 0), a.num_pages - 1);
        const size_t e = (size_t)g * D + (size_t)p * page_elems + (size_t)poff * row_elems;
        ktile = kbase + e;
        vtile = vbase + e;
    };
    const int far_page = WIN && PAGED ? (int)a.page_div.div((unsigned)(near + gap) * BC) : 0;   // of the window's first tile
    const int far_key = WIN && PAGED ? (near + gap) * BC - far_page * a.page_size : 0;
    auto go_to = [&](int t) __attribute__((always_inline)) {
        if constexpr (PAGED) {
            const int page = a.page_div.div((unsigned)t * BC);
            go_to_page(page, t * BC - page * a.page_size);
        } else {
            ktile += (size_t)t * BC * row_elems;
            vtile += (size_t)t * BC * row_elems;
        }
    };
    const unsigned lds0 = lds_address(smem);
    // the next tile (they are loaded in order) into stage `stage`; bf16 V into vr
    auto gload_to = [&](vregs_t &vr, int stage) __attribute__((always_inline)) {
        if constexpr (SEGMENTS) {
            if (tload == near) {   // on to the sequence's own keys
                ktile = reinterpret_cast<const S *>(a.k) + head0;
                vtile = reinterpret_cast<const S *>(a.v) + head0;
                full_tiles = near + (Nk - a.prefix) / BC;
                last_bytes = bytes_of((Nk - a.prefix) % BC);
            }
        }
        if constexpr (PAGED) {
            // the tile's rows sit in one page (pages hold a multiple of 64
            // keys, tiles start at multiples of BC): at the start of a page
            // the address comes from the table (page numbers clamped into the
            // pool), within it the address advances by one tile per load
            if (poff == 0) {
                if (pidx > 0 && pidx % 64 == 0 && !JUMPS) {
                    tcur = tnx;
                    tnx = __builtin_amdgcn_raw_buffer_load_b32(trs, 4 * (pidx + 64 + l), 0, 0);
                }
                const int page = min(max(__builtin_amdgcn_readlane(tcur, pidx % 64), 0), a.num_pages - 1);
                const size_t t = (size_t)g * D + (size_t)page * page_elems;
                ktile = kbase + t;
                vtile = vbase + t;
            }
        }
        const int nrec = tload < full_tiles ? tile_bytes : last_bytes;
        const int at = tload++;
        const unsigned dst = lds0 + stage * (2 * SM::STAGE) + 1024 * piece;
        // once: nobody else reads these keys; the view without `ahead` bytes at its start
        // (offsets there wrap and read as zeros)
        auto issue = [&](auto once, int nrec, auto ahead) __attribute__((always_inline)) {
            constexpr bool ONCE = decltype(once)::value;
            if (dok) {
#pragma unroll
                for (int j = 0; j < NP; ++j)
                    load_lds16<ONCE>(ktile + ahead / (int)sizeof(S), nrec - ahead, dst + 1024 * (NT / 64) * j, koff[j] - ahead);
            }
            if (dov) {
                const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<S *>(vtile + ahead / (int)sizeof(S)), (short)0, nrec - ahead, 0x00020000);
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    if constexpr (VREG)
                        vr[j] = __builtin_bit_cast(uint4_t, __builtin_amdgcn_raw_buffer_load_b128(rv, voff[j] - ahead, 0, 0));
                    else
                        load_lds16<ONCE>(vtile + ahead / (int)sizeof(S), nrec - ahead, dst + 2 * SM::KSZ + 1024 * (NT / 64) * j, voff[j] - ahead);
                }
            }
        };
        constexpr std::integral_constant<int, 0> none{};
        if (WIN && (unsigned)(at + 1 - near) < 2) {   // WINDOW: the last sink's tile (a full one), the window's first
            const bool sink = at + 1 == near;
            int bytes = row_bytes;
            asm volatile("" : "+s"(bytes));   // what follows is computed here, and not held during the loop
            const int behind = (near * BC - sinks) * bytes, ahead = first_key % BC * bytes;
            const long long jump = (long long)gap * BC * (bytes / (int)sizeof(S));
            issue(std::false_type{}, nrec - (sink ? behind : 0), sink ? 0 : ahead);
            if (PAGED && sink) {
                go_to_page(far_page, far_key);
                return;
            }
            ktile += sink ? jump : 0;
            vtile += sink ? jump : 0;
        } else if (MODE == PARTS && own) {
            issue(std::true_type{}, nrec, none);
        } else {
            issue(std::false_type{}, nrec, none);
        }
        ktile += BC * (size_t)row_elems;
        vtile += BC * (size_t)row_elems;
        if constexpr (PAGED) {
            poff += BC;
            const bool cross = poff == a.page_size;   // wave-uniform
            poff = cross ? 0 : poff;
            pidx += cross ? 1 : 0;
            if constexpr (JUMPS) {
                if (cross && pidx % 64 == 0) {
                    tcur = tnx;
                    tnx = __builtin_amdgcn_raw_buffer_load_b32(trs, 4 * (pidx + 64 + l), 0, 0);
                }
            }
        }
    };
    // bf16 V of a loaded tile, as fp16, into its stage
    auto vstore_from = [&](const vregs_t &vr, unsigned short *stage) __attribute__((always_inline)) {
        if constexpr (IN_BF16) {
            if (dov) {
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    unsigned short *at = stage + SM::KSZ + 512 * (piece + (NT / 64) * j) + 8 * l;
                    st16(at, bf16x8_to_f16x8(RAW ? ld16(at) : vr[j]));
                }
            }
        }
    };

    float16_t oacc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt] = float16_t{};
    float m_run = -INFINITY;   // exponent base (log2 domain), same in lanes l and l^32
    float l_run = 0.f;         // this lane's part of the row sum
    float nbase = 0.f;         // -m_run, or 0 while the row has no base
    float lim = -INFINITY;     // largest lane sum kept without a rescale; below any sum while the row has no base

    // LDS offsets (elements) of the lane's operands.  K: chunk 2 kk + lh of row
    // 32 kh + lq.  V: the transposing read gives a lane four keys of one column;
    // lane i of each 16 addresses row i / 4 of four, columns 4 (i % 4) .. + 3 of
    // 16, and the group of 16 picks the column half; k-step j takes keys 16 j +
    // 4 lh .. + 3 and 16 j + 8 + 4 lh .. + 3, the order of the weights.
    const int k_row = (32 * kh + lq) * D, k_sw = 8 * (lh ^ kswz(lq));
    auto kat = [&](const unsigned short *stage, int kk) {
        return as_vec8<V8>(*reinterpret_cast<const uint4_t *>(stage + k_row + ((16 * kk) ^ k_sw)));
    };
    const int v_j = l & 15;
    const int v_row = SM::KSZ + (32 * kh + 4 * lh + (v_j >> 2)) * D + 16 * ((l >> 4) & 1) + 4 * (v_j & 3);
    const int v_sw = 8 * vswz(v_j >> 2);
    auto vat = [&](const unsigned short *stage, int dt, int j) {
        const _Float16 *p = reinterpret_cast<const _Float16 *>(stage) + v_row + ((32 * dt) ^ v_sw) + 16 * D * j;
        return cat_half8(lds_read_tr16(p), lds_read_tr16(p + 8 * D));
    };
    auto stage_at = [&](int r) { return smem + r * SM::STAGE; };

    // K operands of this wave's 32 keys of the tile held in `stage`
    auto kread = [&](const unsigned short *stage, V8 (&ka)[KSTEPS]) {
#pragma unroll
        for (int kk = 0; kk < KSTEPS; ++kk)
            ka[kk] = kat(stage, kk);
    };
    // S^T = K Q^T.  Matrix instructions are issued at raised wave priority:
    // the SIMD then starts a wave's next MFMA as soon as the matrix core is
    // free and fills the gaps with the other waves' vector work.
    auto qk = [&](const V8 (&ka)[KSTEPS]) {
        float16_t s = float16_t{};
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int kk = 0; kk < KSTEPS; ++kk) s = mfma32(ka[kk], qf[kk], s);
        __builtin_amdgcn_s_setprio(0);
        return s;
    };
    auto scores = [&](const unsigned short *stage) {
        V8 ka[KSTEPS];
        kread(stage, ka);
        return qk(ka);
    };

    // V^T operands of one tile for this wave (k-step order: dt, j)
    auto vread = [&](const unsigned short *stage, half8_t (&va)[KSTEPS]) {
#pragma unroll
        for (int kk = 0; kk < KSTEPS; ++kk)
            va[kk] = vat(stage, kk >> 1, kk & 1);
    };
    // O^T += V^T P^T with the weights of one tile (k-step j = keys 16 j .. 16 j
    // + 15 of the wave's half)
    auto pv = [&](const half8_t &p0, const half8_t &p1, const half8_t (&va)[KSTEPS]) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            oacc[dt] = mfma32(va[2 * dt], p0, oacc[dt]);
            oacc[dt] = mfma32(va[2 * dt + 1], p1, oacc[dt]);
        }
        __builtin_amdgcn_s_setprio(0);
    };

    // Grouped operand reads for D = 128: two k-steps per group, the next
    // group read from LDS while the current one multiplies, so that at most
    // four operand words are live instead of one per k-step (this keeps the
    // kernel within the 168 VGPRs of three waves per SIMD).
    auto scores_jit = [&](const unsigned short *stage) {
        float16_t s = float16_t{};
        V8 cur0, cur1, nxt0, nxt1;
        cur0 = kat(stage, 0);
        cur1 = kat(stage, 1);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int g = 0; g < KSTEPS / 2; ++g) {
            if (g + 1 < KSTEPS / 2) {
                nxt0 = kat(stage, 2 * (g + 1));
                nxt1 = kat(stage, 2 * (g + 1) + 1);
            }
            s = mfma32(cur0, qf[2 * g], s);
            s = mfma32(cur1, qf[2 * g + 1], s);
            __builtin_amdgcn_sched_barrier(0);
            cur0 = nxt0;
            cur1 = nxt1;
        }
        __builtin_amdgcn_s_setprio(0);
        return s;
    };
    auto pv_jit = [&](const half8_t &p0, const half8_t &p1, const unsigned short *stage) {
        half8_t cur0, cur1, nxt0, nxt1;
        cur0 = vat(stage, 0, 0);
        cur1 = vat(stage, 0, 1);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            if (dt + 1 < DT) {
                nxt0 = vat(stage, dt + 1, 0);
                nxt1 = vat(stage, dt + 1, 1);
            }
            oacc[dt] = mfma32(cur0, p0, oacc[dt]);
            oacc[dt] = mfma32(cur1, p1, oacc[dt]);
            __builtin_amdgcn_sched_barrier(0);
            cur0 = nxt0;
            cur1 = nxt1;
        }
        __builtin_amdgcn_s_setprio(0);
    };

    // hide keys of tile t, the v-th visited, that some row of the wave must not see
    auto mask = [&](float16_t &s, int t, int v) __attribute__((always_inline)) {
        int kw = t * BC + 32 * kh;        // first key of this wave's half
        int end = Nk;                     // keys from here on do not exist
        if constexpr (SEGMENTS) {
            if (t < near)
                end = a.prefix;
            else
                kw += a.prefix - near * BC;
        }
        if constexpr (WIN) {
            // the lane's row sees keys lo .. hi - 1, counted from the lane's first key,
            // and, where the sinks are no part of their own, those below `always`: a
            // bit for each key (two instructions a score, and no scalar registers)
            const bool sink = v < near;
            const int k0 = kw + 4 * lh, at = qi + off + 1;
            auto below = [](int n) { return (1u << min(max(n, 0), 31)) - 1; };   // (keys 0 .. 27)
            const unsigned seen = below(min(sink ? a.sinks : Nk, at) - k0) &
                                  (~below(sink ? 0 : at - a.window - k0) | below(near > 0 ? 0 : a.sinks - k0));
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const unsigned x = (unsigned)((int)(seen << (31 - 8 * (r >> 2) - (r & 3))) >> 31);
                const float f = s[r];   // (a bit cast of the vector's element itself reads the first one)
                s[r] = __builtin_bit_cast(float, (x & __builtin_bit_cast(unsigned, f)) | (~x & 0xff800000u));
            }
            return;
        }
        if (kw + 32 > (SEGMENTS ? min(kfree_w, end) : kfree_w)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int key = kw + 8 * (r >> 2) + 4 * lh + (r & 3);
                const bool vis = MODE == PARTS ? key < rlim : key < end && (!CAUSAL || key <= qi + off);
                s[r] = vis ? s[r] : -INFINITY;
            }
        }
    };

    // p = 2^(s c + nbase) for the 16 scores of the lane, packed to f16 in the
    // key order of the two PV k-steps
    // All but ALL: the 16 weights are summed before they are rounded, for a
    // log-sum-exp of fp32 accuracy (2 to 3 % of JOIN's time, none of WINDOW's and PARTS')
    float wsum = 0.f;
    auto exp_pack = [&](const float16_t &s, float nbase, half8_t &p0, half8_t &p1) {
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = exp2_fast(__builtin_fmaf(s[r], a.c, nbase));
        if constexpr (MODE != ALL)
            wsum = (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]))) +
                   (((p[8] + p[9]) + (p[10] + p[11])) + ((p[12] + p[13]) + (p[14] + p[15])));
        p0 = pack_f16x8(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7]);
        p1 = pack_f16x8(p[8], p[9], p[10], p[11], p[12], p[13], p[14], p[15]);
    };

    // row sum += the 16 f16 weights of the lane, in fp32 (dot products with (1, 1))
    auto add_sum = [&](float l, const half8_t &p0, const half8_t &p1) {
        if constexpr (MODE != ALL) return l + wsum;
        const half2_t one = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            l = __builtin_amdgcn_fdot2(half2_t{p0[2 * i], p0[2 * i + 1]}, one, l, false);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            l = __builtin_amdgcn_fdot2(half2_t{p1[2 * i], p1[2 * i + 1]}, one, l, false);
        return l;
    };
    // Online softmax of one tile.  The weights are first formed against the
    // current base and kept if the lane's 16 weights add at most 4096 to its
    // row sum (every weight then fits f16 with room to spare and no rescale is
    // due; the row maximum is never formed).  Only when some row outgrows its
    // base that far (or a row has no base yet) is the row maximum taken, the
    // accumulator and row sum rescaled to it and the weights recomputed.  The
    // row sum adds, in fp32, the f16 weights that also feed the matrix product.
    auto softmax = [&](const float16_t &s, half8_t &p0, half8_t &p1) {
        exp_pack(s, nbase, p0, p1);
        const float l_old = l_run;
        l_run = add_sum(l_run, p0, p1);
        const bool over = !(l_run <= l_old + lim);
        if (__builtin_amdgcn_ballot_w64(over) != 0) {
            float mx = max3(s[0], s[1], s[2]);
            mx = max3(mx, s[3], s[4]);
            mx = max3(mx, s[5], s[6]);
            mx = max3(mx, s[7], s[8]);
            mx = max3(mx, s[9], s[10]);
            mx = max3(mx, s[11], s[12]);
            mx = max3(mx, s[13], s[14]);
            mx = __builtin_fmaxf(mx, s[15]);
            mx = pair_max(mx);
            const float m_new = __builtin_fmaxf(m_run, mx * a.c);
            const float alpha = (m_new == -INFINITY) ? 1.f : exp2_fast(m_run - m_new);
            m_run = m_new;
            nbase = (m_new == -INFINITY) ? 0.f : -m_new;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) oacc[dt] *= alpha;
            exp_pack(s, nbase, p0, p1);
            l_run = add_sum(l_old * alpha, p0, p1);
            lim = (m_new == -INFINITY) ? -INFINITY : kMaxLaneSum;
        }
    };

    // Tile loop: one tile per step, in order -- scores, softmax, PV -- and one
    // barrier.  The latencies of a step are hidden by the waves of the other
    // workgroups on the CU, whose barriers are independent of this one's.
    // Tile i + AHEAD is loaded during step i, into the stage that tile i - 1
    // (two stages: the other one) has left.  With three stages the loads have
    // the whole next step as well: step i waits for tile i + 1's, and writes its
    // bf16 V, after its own scores.  With two, at its end.
    constexpr int AHEAD = SM::AHEAD;
    if constexpr (JUMPS) {
        const int t = first + (first >= near ? gap : 0);
        if (ntiles > 0 && t > 0) go_to(t);
    }
    if (ntiles > 0) {
        vregs_t v0;
        gload_to(v0, 0);
        if (AHEAD == 2 && ntiles > 1) gload_to(vr, 1);
        if (!RAW) vstore_from(v0, stage_at(0));
        if (AHEAD == 2 && ntiles > 1)
            lds_loads_done<SM::SPLIT ? NP : 2 * NP>();   // all but those of tile 1
        else
            lds_loads_done<0>();
        if (RAW) vstore_from(v0, stage_at(0));
    }
    lds_barrier();
    // JUMPS: of the steps, those on tiles that every row of the wave sees whole (clean0,
    // clean_n of them; no mask), and those on tiles that some row sees keys of (some0,
    // some_n; WINDOW: and the sinks').  As ranges, since a chain of scalar instructions
    // stands in a step's way where one workgroup has the CU, and so do scalar registers
    // that do not fit (against tests of every tile's keys, with the mask in bits, one
    // sequence, 32/8 heads, D = 128, fp16, 1100 rows, window of all keys 32.6 -> 29.0 us,
    // 275 16.1 -> 14.5; 4096 rows, bf16, 1024 87.2 -> 82.7; D = 64, 16384 rows 175.8 -> 166.0).
    int clean0 = 0, clean_n = 0, some0 = 0, some_n = 0;
    if constexpr (JUMPS) {
        auto from = [&](int key) { return key < 32 * kh ? 0 : (key - 32 * kh) / BC + 1; };   // tiles whose first key of the wave's is <= key
        const int end = from(kfree_w - 32) - gap;
        int top = ntiles;
        if constexpr (WIN) {
            const int passed = row0 + WR - 1 + off - a.window;   // the last key that the last row does not see any more
            clean0 = max(from(passed) - gap, near);
            some0 = near == 0 && a.sinks > 0 ? 0 : max(from(passed - (WR - 1) - 31) - gap, near);
            top = from(row0 + WR - 1 + off) - gap;
        }
        clean_n = live ? max(end - clean0, 0) : 0;
        some_n = live ? max(top - some0, 0) : 0;
        clean0 -= first;
        some0 -= first;
    }
    const int sink_steps = WIN && live ? near - first : 0;
    auto step = [&](int i, auto R) __attribute__((always_inline)) {   // R: stage of tile i (i % NSTAGE)
        constexpr int r = decltype(R)::value;
        // the next tile's loads are issued after the K operand reads (their
        // scalar set-up then overlaps the LDS latency, and at D = 128 their
        // registers are not live across the QK^T product)
        const bool clean = JUMPS && (unsigned)(i - clean0) < (unsigned)clean_n;
        const int t = first + i + (JUMPS && first + i >= near ? gap : 0);   // the tile
        bool some = true;   // (wave-uniform)
        if (PAGED && WIN && D == 128)
            some = live;   // (no scalar registers left for the ranges: with them, 3 to 6 spilled, 32/8 heads, bf16,
                           // pages of 64, window 1024 85.6 -> 88.3 us on 4096 rows, 4 x 256 rows, 512 22.5 -> 23.8)
        else if (JUMPS && !clean)
            some = (unsigned)(i - some0) < (unsigned)some_n || (WIN && i < sink_steps);
        const bool more = i + AHEAD < ntiles;
        auto stage_next = [&]() __attribute__((always_inline)) {
            if (AHEAD == 2 && i + 1 < ntiles) {
                lds_loads_done<0>();   // tile i + 1, loaded since the previous step
                vstore_from(vr, stage_at((r + 1) % NSTAGE));
            }
            if (more) gload_to(vr, (r + AHEAD) % NSTAGE);
        };
        auto scored = [&]() __attribute__((always_inline)) { return D == 128 ? scores_jit(stage_at(r)) : scores(stage_at(r)); };
        auto finish = [&](float16_t &s) __attribute__((always_inline)) {
            if (!clean) mask(s, t, first + i);
            half8_t p0, p1;
            half8_t va[KSTEPS];
            // D = 64: the V operands are read before the softmax, so that their
            // LDS latency is not on the step's critical path
            if constexpr (D == 64) vread(stage_at(r), va);
            softmax(s, p0, p1);
            if constexpr (D == 128) {
                pv_jit(p0, p1, stage_at(r));
            } else {
                pv(p0, p1, va);
            }
        };
        if constexpr (PAGED && WIN) {   // (one copy of the loads: what they hold in scalar registers leaves no room for two)
            float16_t s;
            if (some) s = scored();
            stage_next();
            if (some) finish(s);
        } else if (some) {
            float16_t s = scored();
            stage_next();
            finish(s);
        } else {
            stage_next();
        }
        if (AHEAD == 1) {
            if (more) vstore_from(vr, stage_at((r + AHEAD) % NSTAGE));
            lds_loads_done<0>();
        }
        lds_barrier();
    };
    for (int i = 0; i < ntiles; i += NSTAGE) {   // unrolled over the stages: their offsets are constants
        step(i, std::integral_constant<int, 0>{});
        if (i + 1 < ntiles) step(i + 1, std::integral_constant<int, 1>{});
        if constexpr (NSTAGE > 2) {
            if (i + 2 < ntiles) step(i + 2, std::integral_constant<int, 2>{});
        }
    }
    __syncthreads();   // the merge below reuses the stage memory

    // ---- merge the two key halves of each slot through LDS
    float *mf = reinterpret_cast<float *>(smem);
    constexpr int NV = DT * 16 + 2;
    float *mine = mf + (slot * NV) * 64 + l;
    if (NQ == 2 && kh == 1) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) mine[(dt * 16 + r) * 64] = oacc[dt][r];
        mine[(DT * 16) * 64] = m_run;
        mine[(DT * 16 + 1) * 64] = l_run;
    }
    if (NQ == 2) __syncthreads();
    if (kh != 0 || !live) return;
    if (NQ == 2) {
        const float m1 = mine[(DT * 16) * 64];
        const float l1 = mine[(DT * 16 + 1) * 64];
        const float M = __builtin_fmaxf(m_run, m1);
        const float a0 = (m_run == -INFINITY) ? 0.f : exp2_fast(m_run - M);
        const float a1 = (m1 == -INFINITY) ? 0.f : exp2_fast(m1 - M);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                oacc[dt][r] = a0 * oacc[dt][r] + a1 * mine[(dt * 16 + r) * 64];
        l_run = a0 * l_run + a1 * l1;
        m_run = M;
    }
    const float l_tot = pair_sum(l_run);
    if constexpr (MODE == PARTS || MODE == WINDOW_PARTS) {
        if (qi >= Nq) return;
        const size_t token = MODE == PARTS ? (size_t)tok : (size_t)b * Nq + qi;
        const size_t at = (token * a.Hq + h) * a.slots + split + (own ? (int)a.splits.d : 0);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<float4_t *>(a.opart + at * D + 32 * dt + 8 * i + 4 * lh) =
                    float4_t{oacc[dt][4 * i], oacc[dt][4 * i + 1], oacc[dt][4 * i + 2], oacc[dt][4 * i + 3]};
        if (lh == 0) {
            a.mpart[at] = m_run;
            a.lpart[at] = l_tot;
        }
        return;
    }
    // a row with no visible key (only with per-sequence lengths) gives 0 and
    // a log-sum-exp of -inf
    const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
    if (qi < Nq) {
        TOUT *op = reinterpret_cast<TOUT *>(a.o) + ((size_t)((size_t)b * Nq + qi) * a.Hq + h) * D;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            if constexpr (sizeof(TOUT) == 4) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<float4_t *>(op + 32 * dt + 8 * i + 4 * lh) =
                        float4_t{oacc[dt][4 * i] * inv, oacc[dt][4 * i + 1] * inv,
                                 oacc[dt][4 * i + 2] * inv, oacc[dt][4 * i + 3] * inv};
            } else {
                // a lane has half of each 8-column chunk, lane l ^ 32 the other:
                // of every two chunks the pair exchanges halves, so that each
                // stores one chunk of 16 bytes (8-byte stores of the halves took
                // 2960 cycles of a D = 128 workgroup's end, these 1800: 4 x 16/2
                // heads, 135 rows, fp16 9.35 -> 7.98 us; 333 rows, bf16 13.1 ->
                // 12.1; D = 64, 100 rows 7.3 -> 6.8)
                typedef TOUT t4 __attribute__((ext_vector_type(4)));
                typedef unsigned uint2_t __attribute__((ext_vector_type(2)));
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    uint2_t u[2];
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        t4 x;
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = from_f32<TOUT>(oacc[dt][4 * (i + n) + e] * inv);
                        u[n] = __builtin_bit_cast(uint2_t, x);
                    }
                    auto lo = __builtin_amdgcn_permlane32_swap(u[0][0], u[1][0], false, false);
                    auto hi = __builtin_amdgcn_permlane32_swap(u[0][1], u[1][1], false, false);
                    st16(op + 32 * dt + 8 * (i + lh), uint4_t{lo[0], hi[0], lo[1], hi[1]});
                }
            }
        }
        if (a.lse && lh == 0)
            a.lse[((size_t)b * a.Hq + h) * Nq + qi] = l_tot > 0.f ? (m_run + log2f(l_tot)) * kLn2 : -INFINITY;
    }
}

}  // namespace
}  // namespace fa
