// fa_window.hip -- attention with a sliding window and first keys that stay
// visible, more than one query row a sequence: launches of the prefill kernel
// (fa_prefill_kernel.h) that visit the tiles of the window and of the sinks alone.
#include <algorithm>

#include "fa_internal.h"
#include "fa_prefill_kernel.h"

namespace fa {
namespace {

constexpr int CUS = 256;        // compute units of the card
constexpr int MIN_TILES = 4;    // least tiles in a split

// Cache from which an order by length pays, as in fa_prefill.hip, where the window
// leaves the lengths a difference (us, in the batch's order / ranked, window of 3/4, 1/2
// and 1/4 of the longest: 16 x 32/8 heads, 512 rows, 4096 to 1096 keys, D = 64 226 /
// 198, 184 / 167, 114.8 / 113.0; 40 x 64 rows, 2048 to 488 keys, D = 128 76.0 / 73.1,
// 59.5 / 60.0, 39.0 / 40.1).
constexpr int RANKED_KEYS = 512, RANKED_KEYS_EACH = 40;

int heads(int G) { return G % 4 == 0 ? 4 : G % 2 == 0 ? 2 : 1; }   // query heads per workgroup

// Splits of each row block's tiles.  A workgroup visits them one after the other,
// 0.72 us each (D = 64: 0.65) while its CU holds no other, so that few row blocks
// with long windows leave most of the chip waiting for them: then the tiles are
// split, to one wave on every SIMD, and the parts merged.  Both times are
// estimated as for a shared prefix (fa_prefix.hip).
int splits_of(int B, int Hq, int Hkv, int Nq, int Nk, int D, int window, int sinks, bool most) {
    const int G = Hq / Hkv, hw = heads(G), rows = WR * NSLOT / hw, BC = D == 64 ? Cfg<64>::BC : Cfg<128>::BC;
    const long long blocks = ((long long)Nq + rows - 1) / rows * B * Hkv * (G / hw);
    const long long top = (D == 64 ? CUS / 2 : CUS) / blocks;
    if (top < 2) return 1;
    const long long far = ((long long)window + std::min(rows, Nq)) / BC + 2 + ((long long)sinks + BC - 1) / BC;
    const long long tiles = std::min(((long long)Nk + BC - 1) / BC, far);
    const long long S = std::min({top, (tiles + MIN_TILES - 1) / MIN_TILES, (long long)FA_MAX_SPLITS});
    if (S < 2) return 1;
    if (most) return (int)S;
    const long long tile = D == 64 ? 650 : 720;   // ns
    const long long bytes = (long long)B * Nq * Hq * S * (D + 2) * 8;   // of partial results, written and read
    return 11000 + (tiles + S - 1) / S * tile + bytes / 5000 < 5000 + tiles * tile ? (int)S : 1;
}

template <typename TIN, typename TOUT, int D, int MODE>
hipError_t launch_mode(const PrefillArgs &a, bool paged, long long blocks, hipStream_t stream) {
    if (!grid_fits(blocks, Cfg<D>::NT)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks), block(Cfg<D>::NT);
    if (paged)
        hipLaunchKernelGGL((prefill_kernel<TIN, TOUT, D, NSLOT, true, true, MODE>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((prefill_kernel<TIN, TOUT, D, NSLOT, true, false, MODE>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <typename TIN, typename TOUT, int D>
hipError_t launch_t(const Problem &p, float *ws, hipStream_t stream) {
    PrefillArgs a;
    a.q = p.q; a.k = p.k; a.v = p.v; a.o = p.o; a.lse = p.lse;
    a.B = p.B; a.Hq = p.Hq; a.Hkv = p.Hkv; a.Nq = p.Nq; a.Nk = p.Nk;
    a.seqlens = p.seqlens;
    a.block_table = p.block_table;
    a.page_size = p.page_size;
    a.max_pages = p.max_pages;
    a.num_pages = p.num_pages;
    a.c = __builtin_fmaxf(__builtin_fabsf(p.scale), 1e-30f) * kLog2e;
    a.qsign = p.scale < 0.f ? 0x80008000u : 0u;
    const int G = p.Hq / p.Hkv;
    a.HW = heads(G);
    const int RB = NSLOT / a.HW;
    a.nmb = (p.Nq + WR * RB - 1) / (WR * RB);
    const long long blocks = (long long)a.nmb * p.B * p.Hkv * (G / a.HW);
    a.G = G;
    a.lgHW = a.HW == 4 ? 2 : a.HW == 2 ? 1 : 0;
    a.nhg = Divisor(G / a.HW);
    a.nkv = Divisor(p.Hkv);
    a.per_mb = Divisor((unsigned)p.B * p.Hkv * (G / a.HW));
    a.first = a.nmb;
    a.ranked = 0;
    a.row_blocks = Divisor(a.nmb);
    if (p.seqlens && p.B > 1 && p.B <= kMaxRanked && blocks > CUS && 2LL * p.window >= p.Nk && p.Nk >= RANKED_KEYS &&
        p.Nk >= RANKED_KEYS_EACH * (long long)p.B) {
        a.per_seq = Divisor(p.Hkv * (G / a.HW));
        a.ranked = blocks <= (long long)Cfg<D>::WPC * CUS ? (CUS + (int)a.per_seq.d - 1) / (int)a.per_seq.d : a.nmb * p.B;
    }
    a.page_div = Divisor(p.block_table ? p.page_size : 1);
    a.window = p.window;
    a.sinks = p.sinks;
    const int S = splits_of(p.B, p.Hq, p.Hkv, p.Nq, p.Nk, D, p.window, p.sinks, false);
    if (S == 1) return launch_mode<TIN, TOUT, D, WINDOW>(a, p.block_table, blocks, stream);
    a.splits = Divisor(S);
    a.slots = S;
    const size_t parts = (size_t)p.B * p.Nq * p.Hq * S;
    a.opart = ws;
    a.mpart = ws + parts * D;
    a.lpart = a.mpart + parts;
    const hipError_t e = launch_mode<TIN, float, D, WINDOW_PARTS>(a, p.block_table, blocks * S, stream);
    return e != hipSuccess ? e : launch_merge(p, S, ws, stream);
}

template <typename TIN, typename TOUT>
hipError_t launch_d(const Problem &p, float *ws, hipStream_t s) {
    return p.D == 64 ? launch_t<TIN, TOUT, 64>(p, ws, s) : launch_t<TIN, TOUT, 128>(p, ws, s);
}

}  // namespace

size_t window_workspace_bytes(int B, int Hq, int Hkv, int Nq, int Nk, int D, int window, int sinks, bool most) {
    const int S = splits_of(B, Hq, Hkv, Nq, Nk, D, window, sinks, most);
    return S == 1 ? 0 : (size_t)B * Nq * Hq * S * (size_t)(D + 2) * sizeof(float);
}

hipError_t launch_prefill_window(const Problem &p, void *workspace, hipStream_t stream) {
    float *ws = reinterpret_cast<float *>(workspace);
    if (p.in == FA_F16)
        return p.out == FA_F32 ? launch_d<f16_t, float>(p, ws, stream) : launch_d<f16_t, _Float16>(p, ws, stream);
    return p.out == FA_F32 ? launch_d<bf16_t, float>(p, ws, stream) : launch_d<bf16_t, __bf16>(p, ws, stream);
}

}  // namespace fa
