// fa_prefix.hip -- attention of a batch whose sequences share a long prefix.
//
// softmax over prefix and suffix together is the sum of parts, each an
// accumulator, a base and a sum (the state that streaming softmax carries from
// key block to key block), so the parts can be taken apart:
//   prefix  all B Nq G query rows of a key/value head against the prefix's keys,
//           which are read once for every 128 rows instead of once a sequence
//   own     each sequence's rows against its own keys
//   merge   the parts by their bases, the final normalisation, the log-sum-exp
// Prefix and own parts are workgroups of one launch (prefill kernel, PARTS), cut
// into splits of the keys: the prefix's multiply while the others read.
// Where there are rows enough for full waves on a full chip, or few keys, every
// row takes the prefix's keys and its own in one pass (JOIN).
#include <algorithm>

#include "fa_checks.h"
#include "fa_internal.h"
#include "fa_prefill_kernel.h"

namespace fa {
namespace {

constexpr int CUS = 256;                 // compute units of the card
constexpr int MIN_TILES = 4;             // least tiles in a split of the prefix
constexpr int ROWS = WR * NSLOT;         // rows of a workgroup against the prefix

// Partial results of `slots` parts merged, D / 64 columns a lane.  A row's parts are
// taken by one wave, eight loads together, or dealt out to the four of the
// workgroup, whose results are merged through LDS (WPR; a chain of loads the
// fewer for the long lists that few rows have: 2 x 32/4 heads, 64 parts, 16.5 -> 13.7
// us a call).
constexpr int LONG_LIST = 16;   // most parts that one wave takes

template <typename TOUT, int D, int WPR>
__global__ __launch_bounds__(256) void merge_kernel(const float *__restrict__ opart, const float *__restrict__ mpart,
                                                    const float *__restrict__ lpart, void *o, float *lse, int slots,
                                                    int rows, int Hq, int Nq) {
    constexpr int N = D / 64;
    typedef float vec __attribute__((ext_vector_type(N)));
    typedef TOUT out __attribute__((ext_vector_type(N)));
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6, row = WPR == 1 ? blockIdx.x * 4 + w : blockIdx.x;
    if (row >= rows) return;
    const int each = (slots + WPR - 1) / WPR, first = WPR == 1 ? 0 : min(w * each, slots), end = min(first + each, slots);
    const float *mp = mpart + (size_t)row * slots, *lp = lpart + (size_t)row * slots;
    const float *op = opart + (size_t)row * slots * D + N * l;
    float M = -INFINITY, L = 0.f;
    vec acc = vec{};
    auto add = [&](const float (&m)[8], const float (&n)[8], const vec (&x)[8]) {
        float Mc = M;
#pragma unroll
        for (int j = 0; j < 8; ++j) Mc = __builtin_fmaxf(Mc, m[j]);
        const float alpha = M == -INFINITY ? 0.f : exp2_fast(M - Mc);
        L *= alpha;
        acc *= alpha;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float f = m[j] == -INFINITY ? 0.f : exp2_fast(m[j] - Mc);
            L = __builtin_fmaf(f, n[j], L);
#pragma unroll
            for (int c = 0; c < N; ++c) acc[c] = __builtin_fmaf(f, x[j][c], acc[c]);
        }
        M = Mc;
    };
    for (int s0 = first; s0 < end; s0 += 8) {
        float m[8], n[8];
        vec x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int s = min(s0 + j, end - 1);
            m[j] = s0 + j < end ? mp[s] : -INFINITY;
            n[j] = lp[s];
            x[j] = *reinterpret_cast<const vec *>(op + (size_t)s * D);
        }
        add(m, n, x);
    }
    if constexpr (WPR > 1) {
        __shared__ float part[WPR][D + 2];
        *reinterpret_cast<vec *>(&part[w][N * l]) = acc;
        if (l == 0) {
            part[w][D] = M;
            part[w][D + 1] = L;
        }
        __syncthreads();
        if (w > 0) return;
        float m[8], n[8];
        vec x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = j < WPR ? j : 0;
            m[j] = j < WPR ? part[i][D] : -INFINITY;
            n[j] = part[i][D + 1];
            x[j] = *reinterpret_cast<const vec *>(&part[i][N * l]);
        }
        M = -INFINITY;
        L = 0.f;
        acc = vec{};
        add(m, n, x);
    }
    // a row that sees no key gives 0 and -inf
    const float inv = L > 0.f ? 1.f / L : 0.f;
    out r;
#pragma unroll
    for (int n = 0; n < N; ++n) r[n] = from_f32<TOUT>(acc[n] * inv);
    *reinterpret_cast<out *>(reinterpret_cast<TOUT *>(o) + (size_t)row * D + N * l) = r;
    if (lse && l == 0) {
        const int t = row / Hq, h = row - t * Hq, b = t / Nq;
        lse[((size_t)b * Hq + h) * Nq + (t - b * Nq)] = L > 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
    }
}

// Parts or one pass, and the splits.
//
// Parts: splits of the prefix's keys and of a sequence's own.  Both kinds of
// workgroups take about the same number of tiles, so that all of them together
// fill the chip once, but at least MIN_TILES; the prefix's, whose four slots all
// multiply, count their tiles 5 / 4 at D = 128 (64 x 32/8 heads behind 8192 keys, 1024
// to 64 of their own: 48.6 us with 10 splits of the prefix, 46.3 with 12, 50.1 with
// 16).  More prefix workgroups than one wave on every SIMD only leave more partial
// results: without own keys, D = 128, 37.2 us with 43 splits (688 workgroups), 28.8
// with 16 (256); D = 64, 64 x 16/1 heads, 19.6 with 32, 18.4 with 16 (128 workgroups
// of eight waves).
//
// One pass has no partial results and no merge, but no splits either, and pads
// each sequence's rows to 32.  Both times are estimated from the tiles (us a
// tile with one, two and three workgroups on a CU, D = 128: 0.72, 1.13, 1.56; D = 64,
// two at most: 0.65, 1.0), a start and end, and the partial results' traffic at 5
// bytes a ns.  Over 55 calls of 1 to 128 rows the choice was the quicker one (us, one
// pass / parts; 32/8 heads, D = 128: 8 x 48 rows behind 4096 keys 96 / 65, x 128 98 /
// 123, 32 x 8 behind 1000 32 / 24, x 24 33 / 45; 2 x 48 behind 8000 184 / 35; 16 x 8,
// 32/4 heads, D = 64, behind 500 11 / 14).
struct Plan {
    int prefix, own;   // 0, 0: one pass
};

// Query heads per workgroup in one pass.
int pass_heads(int G) { return G % 4 == 0 ? 4 : G % 2 == 0 ? 2 : 1; }

// most: at least as many of both as any shorter prefix and suffix get.
Plan plan(int B, int Hq, int Hkv, int Nq, int Np, int Nk, int D, bool most) {
    const int BC = D == 64 ? Cfg<64>::BC : Cfg<128>::BC, wpc = D == 64 ? Cfg<64>::WPC : Cfg<128>::WPC;
    const long long G = Hq / Hkv, rows = B * G * Nq;
    const long long pu = (rows + ROWS - 1) / ROWS * Hkv, pt = ((long long)Np + BC - 1) / BC;
    const long long su = (G * Nq + ROWS - 1) / ROWS * Hkv * B, st = ((long long)Nk + BC - 1) / BC;
    const long long room = CUS * wpc;   // workgroups that the chip holds at once
    const int hw = pass_heads((int)G), pass_rows = WR * NSLOT / hw;
    const long long passes = ((long long)Nq + pass_rows - 1) / pass_rows * B * Hkv * (G / hw);
    if (Nq >= WR && passes >= room) return Plan{0, 0};   // full waves on a full chip

    const long long each = std::max((long long)MIN_TILES, (pu * pt + su * st + room - 1) / room);
    const long long weight = D == 64 ? 4 : 5;              // of a prefix tile, in quarters
    const long long top = (D == 64 ? CUS / 2 : CUS) / pu;   // splits that give every SIMD one wave
    auto least_tiles = [](long long tiles) { return (tiles + MIN_TILES - 1) / MIN_TILES; };
    long long prefix = std::min(least_tiles(pt), top), own = std::min(least_tiles(st), room / su + 1);
    if (!most) {
        prefix = std::min(prefix, (pt * weight / 4 + each - 1) / each);
        own = std::min(own, (st + each - 1) / each);   // (each >= su st / room)
    }
    auto count = [](long long n) { return n < 1 ? 1 : n > FA_MAX_SPLITS ? FA_MAX_SPLITS : (int)n; };
    const Plan parts{count(prefix), Nk > 0 ? count(own) : 0};
    if (most) return parts;

    const long long tile128[] = {0, 720, 1130, 1560}, tile64[] = {0, 650, 1000};   // ns, by workgroups on the CU
    const long long *tile = D == 64 ? tile64 : tile128;
    const long long rest = (passes % room + CUS - 1) / CUS;
    const long long pass_ns = 5000 + (pt + st) * (passes / room * tile[wpc] + tile[rest]);
    const long long longest = std::max((pt + parts.prefix - 1) / parts.prefix, parts.own ? (st + parts.own - 1) / parts.own : 0);
    const long long parts_ns = 11000 + std::max(longest * tile[1], (pu * pt + su * st) * tile[wpc] / room) +
                               rows * Hkv * (parts.prefix + parts.own) * (D + 2) * 8 / 5000;
    return pass_ns < parts_ns ? Plan{0, 0} : parts;
}

void common_args(const PrefixProblem &pp, PrefillArgs &a) {
    const Problem &p = pp.p;
    a.q = p.q; a.k = p.k; a.v = p.v; a.o = p.o; a.lse = p.lse;
    a.B = p.B; a.Hq = p.Hq; a.Hkv = p.Hkv; a.Nq = p.Nq; a.Nk = p.Nk;
    a.seqlens = p.seqlens;
    a.block_table = p.block_table;
    a.page_size = p.page_size;
    a.max_pages = p.max_pages;
    a.num_pages = p.num_pages;
    a.page_div = Divisor(p.block_table ? p.page_size : 1);
    a.c = __builtin_fmaxf(__builtin_fabsf(p.scale), 1e-30f) * kLog2e;
    a.qsign = p.scale < 0.f ? 0x80008000u : 0u;
    a.G = p.Hq / p.Hkv;
    a.nkv = Divisor(p.Hkv);
    a.ranked = 0;
    a.k_prefix = pp.k_prefix;
    a.v_prefix = pp.v_prefix;
    a.prefix = pp.Np;
    a.own = pp.own;
    a.counted = p.block_table ? pp.Np : 0;
}

template <typename TIN, int D>
hipError_t launch_parts(const PrefixProblem &pp, const Plan &n, float *ws, hipStream_t stream) {
    using SM = Cfg<D>;
    const Problem &p = pp.p;
    const int G = p.Hq / p.Hkv;
    const long long rows = (long long)p.B * p.Nq * G;   // of a key/value head
    PrefillArgs a;
    common_args(pp, a);
    a.slots = n.prefix + n.own;
    const size_t parts = (size_t)rows * p.Hkv * a.slots;
    a.opart = ws;
    a.mpart = ws + parts * D;
    a.lpart = a.mpart + parts;
    a.HW = 1;
    a.lgHW = 0;
    a.nmb = a.first = 0;
    a.nhg = a.per_mb = Divisor(1);
    a.causal = p.causal;
    a.rows = (int)rows;
    a.splits = Divisor(n.prefix);
    a.own_splits = Divisor(n.own > 0 ? n.own : 1);
    a.batch = Divisor(p.B);
    a.tokens = Divisor(p.Nq);
    a.group = Divisor(G);
    a.first_page = p.block_table ? pp.Np / p.page_size : 0;
    const long long shared = (rows + ROWS - 1) / ROWS * p.Hkv * n.prefix;
    const long long nblocks = shared + ((long long)p.Nq * G + ROWS - 1) / ROWS * p.B * p.Hkv * n.own;
    // (also the merge's, whose launch comes second: a wave or a workgroup a row)
    if (!grid_fits(nblocks, SM::NT) || !grid_fits(rows * p.Hkv, a.slots > LONG_LIST ? 256 : 64))
        return hipErrorInvalidConfiguration;
    a.prefix_blocks = (int)shared;
    if (p.block_table)
        hipLaunchKernelGGL((prefill_kernel<TIN, float, D, NSLOT, false, true, PARTS>), dim3((unsigned)nblocks),
                           dim3(SM::NT), 0, stream, a);
    else
        hipLaunchKernelGGL((prefill_kernel<TIN, float, D, NSLOT, false, false, PARTS>), dim3((unsigned)nblocks),
                           dim3(SM::NT), 0, stream, a);
    return hipGetLastError();
}

template <typename TIN, typename TOUT, int D>
hipError_t launch_join(const PrefixProblem &pp, hipStream_t stream) {
    using SM = Cfg<D>;
    const Problem &p = pp.p;
    PrefillArgs a;
    common_args(pp, a);
    const int G = a.G;
    a.HW = pass_heads(G);
    a.lgHW = a.HW == 4 ? 2 : a.HW == 2 ? 1 : 0;
    const int RB = NSLOT / a.HW;
    a.nmb = a.first = (p.Nq + WR * RB - 1) / (WR * RB);
    const long long nblocks = (long long)a.nmb * p.B * p.Hkv * (G / a.HW);
    if (!grid_fits(nblocks, SM::NT)) return hipErrorInvalidConfiguration;
    a.nhg = Divisor(G / a.HW);
    a.per_mb = Divisor((unsigned)p.B * p.Hkv * (G / a.HW));
    const dim3 grid((unsigned)nblocks), block(SM::NT);
    if (p.block_table && p.causal)
        hipLaunchKernelGGL((prefill_kernel<TIN, TOUT, D, NSLOT, true, true, JOIN>), grid, block, 0, stream, a);
    else if (p.block_table)
        hipLaunchKernelGGL((prefill_kernel<TIN, TOUT, D, NSLOT, false, true, JOIN>), grid, block, 0, stream, a);
    else if (p.causal)
        hipLaunchKernelGGL((prefill_kernel<TIN, TOUT, D, NSLOT, true, false, JOIN>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((prefill_kernel<TIN, TOUT, D, NSLOT, false, false, JOIN>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <typename TOUT, int D>
hipError_t launch_merge_t(const Problem &p, int slots, const float *ws, hipStream_t stream) {
    const long long rows = (long long)p.B * p.Nq * p.Hq;
    const size_t parts = (size_t)rows * slots;
    const float *m = ws + parts * D;
    if (slots > LONG_LIST)
        hipLaunchKernelGGL((merge_kernel<TOUT, D, 4>), dim3((unsigned)rows), dim3(256), 0, stream, ws, m, m + parts, p.o,
                           p.lse, slots, (int)rows, p.Hq, p.Nq);
    else
        hipLaunchKernelGGL((merge_kernel<TOUT, D, 1>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, ws, m,
                           m + parts, p.o, p.lse, slots, (int)rows, p.Hq, p.Nq);
    return hipGetLastError();
}

template <typename TOUT>
hipError_t launch_merge_d(const Problem &p, int slots, const float *ws, hipStream_t stream) {
    return p.D == 64 ? launch_merge_t<TOUT, 64>(p, slots, ws, stream) : launch_merge_t<TOUT, 128>(p, slots, ws, stream);
}

template <typename TIN, typename TOUT>
hipError_t launch_d(const PrefixProblem &pp, float *ws, hipStream_t stream) {
    const Problem &p = pp.p;
    const Plan n = plan(p.B, p.Hq, p.Hkv, p.Nq, pp.Np, pp.own, p.D, false);
    if (n.prefix == 0)
        return p.D == 64 ? launch_join<TIN, TOUT, 64>(pp, stream) : launch_join<TIN, TOUT, 128>(pp, stream);
    const hipError_t e = p.D == 64 ? launch_parts<TIN, 64>(pp, n, ws, stream) : launch_parts<TIN, 128>(pp, n, ws, stream);
    return e != hipSuccess ? e : launch_merge(p, n.prefix + n.own, ws, stream);
}

}  // namespace

hipError_t launch_merge(const Problem &p, int slots, const float *ws, hipStream_t stream) {
    if (p.out == FA_F32) return launch_merge_d<float>(p, slots, ws, stream);
    return p.in == FA_F16 ? launch_merge_d<_Float16>(p, slots, ws, stream) : launch_merge_d<__bf16>(p, slots, ws, stream);
}

size_t prefix_workspace_bytes(int B, int Hq, int Hkv, int Nq, int Np, int Nk, int D, bool most) {
    const Plan n = plan(B, Hq, Hkv, Nq, Np, Nk, D, most);
    return (size_t)B * Nq * Hq * (n.prefix + n.own) * (size_t)(D + 2) * sizeof(float);
}

hipError_t launch_prefix(const PrefixProblem &pp, void *workspace, hipStream_t stream) {
    const Problem &p = pp.p;
    float *ws = reinterpret_cast<float *>(workspace);
    if (p.in == FA_F16)
        return p.out == FA_F32 ? launch_d<f16_t, float>(pp, ws, stream) : launch_d<f16_t, _Float16>(pp, ws, stream);
    return p.out == FA_F32 ? launch_d<bf16_t, float>(pp, ws, stream) : launch_d<bf16_t, __bf16>(pp, ws, stream);
}

}  // namespace fa
