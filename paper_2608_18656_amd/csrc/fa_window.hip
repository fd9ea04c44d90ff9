// fa_window.hip -- attention with a sliding window and first keys that stay
// visible, more than one query row a sequence: launches of the prefill kernel
// (fa_prefill_kernel.h) that visit the tiles of the window and of the sinks alone.
#include "fa_internal.h"
#include "fa_prefill_kernel.h"

namespace fa {
namespace {

template <typename TIN, typename TOUT, int D>
hipError_t launch_t(const Problem &p, hipStream_t stream) {
    using SM = Cfg<D>;
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
    a.HW = G % 4 == 0 ? 4 : G % 2 == 0 ? 2 : 1;
    const int RB = NSLOT / a.HW;
    a.nmb = (p.Nq + WR * RB - 1) / (WR * RB);
    const long long nblocks = (long long)a.nmb * p.B * p.Hkv * (G / a.HW);
    if (nblocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    a.G = G;
    a.lgHW = a.HW == 4 ? 2 : a.HW == 2 ? 1 : 0;
    a.nhg = Divisor(G / a.HW);
    a.nkv = Divisor(p.Hkv);
    a.per_mb = Divisor((unsigned)p.B * p.Hkv * (G / a.HW));
    a.first = a.nmb;
    a.ranked = 0;
    a.page_div = Divisor(p.block_table ? p.page_size : 1);
    a.window = p.window;
    a.sinks = p.sinks;
    if (p.block_table)
        hipLaunchKernelGGL((prefill_kernel<TIN, TOUT, D, NSLOT, true, true, WINDOW>), dim3((unsigned)nblocks),
                           dim3(SM::NT), 0, stream, a);
    else
        hipLaunchKernelGGL((prefill_kernel<TIN, TOUT, D, NSLOT, true, false, WINDOW>), dim3((unsigned)nblocks),
                           dim3(SM::NT), 0, stream, a);
    return hipGetLastError();
}

template <typename TIN, typename TOUT>
hipError_t launch_d(const Problem &p, hipStream_t s) {
    return p.D == 64 ? launch_t<TIN, TOUT, 64>(p, s) : launch_t<TIN, TOUT, 128>(p, s);
}

}  // namespace

hipError_t launch_prefill_window(const Problem &p, hipStream_t stream) {
    if (p.in == FA_F16)
        return p.out == FA_F32 ? launch_d<f16_t, float>(p, stream) : launch_d<f16_t, _Float16>(p, stream);
    return p.out == FA_F32 ? launch_d<bf16_t, float>(p, stream) : launch_d<bf16_t, __bf16>(p, stream);
}

}  // namespace fa
