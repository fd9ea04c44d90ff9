// fa_prefill.hip -- launches of the prefill kernel (fa_prefill_kernel.h) for
// attention over all keys, causal or not: order, layout and packing of the workgroups.
#include <atomic>
#include <type_traits>

#include "fa_checks.h"
#include "fa_internal.h"
#include "fa_prefill_kernel.h"

namespace fa {
namespace {

constexpr int RANKED_KEYS = 512, RANKED_KEYS_EACH = 40;   // cache from which an order by length pays: keys, keys a sequence

// Compute units of the current device (cached per device; 0 if unknown).
int cu_count() {
    static std::atomic<int> cached[64] = {};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 0;
    int n = cached[dev].load(std::memory_order_relaxed);
    if (n == 0 && hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess)
        cached[dev].store(n, std::memory_order_relaxed);
    return n;
}

// Query heads per workgroup of `slots` slots: the most of one key/value group,
// up to 4, that fill the slots evenly.
int default_heads(int slots, int G) {
    int hw = 1;
    for (int c = 2; c <= (slots < 4 ? slots : 4); c *= 2)
        if (slots % c == 0 && G % c == 0) hw = c;
    return hw;
}

// Whether a D = 64 call takes eight slots per workgroup (one 16-wave workgroup
// per CU) where the caller leaves the choice, rather than four (two of 8
// waves).  Eight stage each tile half as often and run a full CU 4 to 5 %
// faster; four end more evenly, and one's start and end go under in the other's
// steps.  Calls whose workgroups all take about the same time, not causal or few
// rows against many keys, compare rounds: a last round that leaves four-slot
// workgroups alone on their CUs costs them 0.58 of a full one (4 against 8, us,
// 32/8 heads, bf16: 1056 rows 24.8 / 23.3; 1400 rows 28.9 / 26.9; 2048 rows 47.9 /
// 45.6; 2500 rows 77.8 / 92.9; 5920 rows 342.9 / 329.6; 8192 rows 631 / 605; 16/1
// heads, 3000 rows 54.0 / 48.1; fp16, 16384 rows 1245 / 1198; bf16, 9000 rows 417.6
// / 453.7; causal, 4 x 1024 rows against 4096 keys 141.7 / 134.2, 5 x 1000 against
// 5000 216 / 228), and a round's start and end cost eight the time of some 90
// keys more, 32 where there is one round (over 1600 calls of 16 to 6000 keys the
// choice is on average 0.1 % off the better one; without those keys 2.1, at most
// 42: 49 x 32/8, 57 rows 13.7 / 15.4; 62 x 32/8, 189 rows 47.7 / 63.7; 14 x 32/4,
// 67 rows 8.5 / 10.0; 7 x 32/8, 1406 rows 143.9 / 153.7).  A K/V that the memory
// side's 256 MB do not hold comes from HBM for every workgroup that reads it:
// eight where they are half as many, and two rounds or more (97 x 16/16 heads,
// 172 rows, 2228 keys 401 / 322; 84 x 16/16, 506 rows, 1233 keys 419 / 338; at 290
// to 330 MB -10 to +9 %; not for uneven lengths in order, 33 x 16/16, 439 rows,
// 2978 to 2233 keys 223 / 256).
// Square causal calls end on short workgroups in any case: eight from four full
// rounds and 7168 rows on, where four heads share a workgroup (32/8, 8192 rows
// 314 / 307; 2 x 32/8, 7200 rows 483 / 476; 16/1 16384, fp16 628 / 621; but 2 x
// 32/8, 4700 rows 220 / 228; 29 x 32/4, 290 rows 35.7 / 46.2; and 2 x 16/16 heads,
// 5000 rows 137 / 146).  Lengths of their own are not known here.  Where they are
// equal, eight gain as much (16 x 32/8 heads, 512 rows against 4096 keys 370 /
// 348; 32 x 16/2, 256 rows 205 / 184), and long uneven ones lose at most 1 % (the
// first call with 614 keys and more 180 / 181); short ones would lose up to 12 %
// (16 x 512 rows against up to 1024 keys 64.5 / 72.5, against 2048 99.8 / 104.1,
// where equal ones gain 1.4 %), and so would those of one round, whose long and
// short workgroups then no longer share CUs (4 x 512 rows against 2048 to 4096
// keys 62.7 / 69.2): eight from 2048 keys and two rounds on.
bool eight_slots(const Problem &p, bool causal) {
    if (p.D != 64 || p.hw > 0 || p.block_table) return false;
    const long long cus = cu_count();
    if (cus == 0) return false;
    const int G = p.Hq / p.Hkv;
    auto groups = [&](int slots) {
        const int hw = default_heads(slots, G), rows = WR * slots / hw;
        return ((long long)p.Nq + rows - 1) / rows * p.B * p.Hkv * (G / hw);
    };
    const long long four = groups(4), eight = groups(8);
    const bool square = causal && p.Nk < 4LL * p.Nq;
    const long long kv_bytes = 256LL * p.B * p.Hkv * p.Nk;
    if (!square && eight >= 2 * cus && four == 2 * eight && kv_bytes > 335000000 && (!p.seqlens || p.B > kMaxRanked))
        return true;
    if (p.seqlens && (p.Nk < 2048 || eight < 2 * cus)) return false;
    if (square) return G % 4 == 0 && four >= 8 * cus && p.Nk >= 7168;
    const long long rest = four % (2 * cus);
    const long long cost4 = four / (2 * cus) * 1000 + (rest == 0 ? 0 : rest <= cus ? 580 : 1000);
    return (eight + cus - 1) / cus * (955 + 1000 * (eight <= cus ? 32 : 90) / p.Nk) < cost4;
}

template <typename TIN, typename TOUT, int D, int NS, bool CAUSAL>
hipError_t launch_t(const Problem &p, hipStream_t stream) {
    using SM = Cfg<D, NS>;
    PrefillArgs a;
    a.q = p.q; a.k = p.k; a.v = p.v; a.o = p.o; a.lse = p.lse;
    a.B = p.B; a.Hq = p.Hq; a.Hkv = p.Hkv; a.Nq = p.Nq; a.Nk = p.Nk;
    a.seqlens = p.seqlens;
    a.block_table = p.block_table;
    a.page_size = p.page_size;
    a.max_pages = p.max_pages;
    a.num_pages = p.num_pages;
    // A zero scale keeps a tiny positive factor: every visible exponent is then
    // exactly 0 in fp32, and masked (-inf) scores still give 0.
    a.c = __builtin_fmaxf(__builtin_fabsf(p.scale), 1e-30f) * kLog2e;
    a.qsign = p.scale < 0.f ? 0x80008000u : 0u;
    const int G = p.Hq / p.Hkv;
    // query heads per workgroup: the requested packing, else the default
    a.HW = p.hw > 0 ? p.hw : default_heads(NS, G);
    const int RB = NS / a.HW;
    a.nmb = (p.Nq + WR * RB - 1) / (WR * RB);
    const long long nblocks = (long long)a.nmb * p.B * p.Hkv * (G / a.HW);
    if (nblocks <= 0) return hipSuccess;
    if (nblocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    a.G = G;
    a.lgHW = a.HW == 8 ? 3 : a.HW == 4 ? 2 : a.HW == 2 ? 1 : 0;
    a.nhg = Divisor(G / a.HW);
    a.nkv = Divisor(p.Hkv);
    a.per_mb = Divisor((unsigned)p.B * p.Hkv * (G / a.HW));   // <= nblocks
    const int cus = cu_count();
    const bool at_once = nblocks <= (long long)SM::WPC * cus;   // every workgroup is resident from the start
    a.first = p.causal && at_once ? (cus + (int)a.per_mb.d - 1) / (int)a.per_mb.d : a.nmb;
    a.ranked = 0;
    a.row_blocks = Divisor(a.nmb);
    if (p.seqlens && p.B > 1 && p.B <= kMaxRanked && nblocks > cus && p.Nk >= RANKED_KEYS &&
        p.Nk >= RANKED_KEYS_EACH * (long long)p.B) {
        const int per_seq = p.Hkv * (G / a.HW);
        a.per_seq = Divisor(per_seq);
        a.ranked = at_once ? (cus + per_seq - 1) / per_seq : a.nmb * p.B;
    }
    if constexpr (NS == NSLOT) {
        if (p.block_table) {
            hipLaunchKernelGGL((prefill_kernel<TIN, TOUT, D, NS, CAUSAL, true>), dim3((unsigned)nblocks),
                               dim3(SM::NT), 0, stream, a);
            return hipGetLastError();
        }
    } else if (p.block_table) {
        return hipErrorInvalidValue;   // paged K/V takes the default slots
    }
    hipLaunchKernelGGL((prefill_kernel<TIN, TOUT, D, NS, CAUSAL, false>), dim3((unsigned)nblocks),
                       dim3(SM::NT), 0, stream, a);
    return hipGetLastError();
}

template <typename TIN, typename TOUT, int D, bool CAUSAL>
hipError_t launch_s(const Problem &p, hipStream_t s) {
    switch (p.slots) {
    case 1: return launch_t<TIN, TOUT, D, 1, CAUSAL>(p, s);
    case 2: return launch_t<TIN, TOUT, D, 2, CAUSAL>(p, s);
    case 4: return launch_t<TIN, TOUT, D, 4, CAUSAL>(p, s);
    case 8: return launch_t<TIN, TOUT, D, 8, CAUSAL>(p, s);
    default:
        return eight_slots(p, CAUSAL) ? launch_t<TIN, TOUT, D, 8, CAUSAL>(p, s) : launch_t<TIN, TOUT, D, NSLOT, CAUSAL>(p, s);
    }
}

template <typename TIN, typename TOUT>
hipError_t launch_d(const Problem &p, hipStream_t s) {
    if (p.D == 64) return p.causal ? launch_s<TIN, TOUT, 64, true>(p, s)
                                   : launch_s<TIN, TOUT, 64, false>(p, s);
    return p.causal ? launch_s<TIN, TOUT, 128, true>(p, s) : launch_s<TIN, TOUT, 128, false>(p, s);
}

}  // namespace

bool prefill_supported(int Hkv, int D, fa_dtype_t in) {
    return (D == 64 || D == 128) && (in == FA_F16 || in == FA_BF16) && tile_fits(Hkv, D, D == 64 ? Cfg<64>::BC : Cfg<128>::BC);
}

hipError_t launch_prefill(const Problem &p, hipStream_t stream) {
    if (p.in == FA_F16)
        return p.out == FA_F32 ? launch_d<f16_t, float>(p, stream)
                               : launch_d<f16_t, _Float16>(p, stream);
    return p.out == FA_F32 ? launch_d<bf16_t, float>(p, stream) : launch_d<bf16_t, __bf16>(p, stream);
}

}  // namespace fa
