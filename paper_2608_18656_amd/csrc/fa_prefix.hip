// fa_prefix.hip -- attention of a batch whose sequences share a long prefix.
//
// softmax over prefix and suffix together is the sum of two parts, each an
// accumulator, a base and a sum (the state that streaming softmax carries from
// key block to key block), so the parts can be taken apart:
//   prefix  all B Nq G query rows of a key/value head against the prefix's keys,
//           which are read once for every 128 rows instead of once a sequence
//           (prefill kernel, PREFIX: 128 rows and a split of the keys a workgroup)
//   suffix  each sequence's rows against its own keys (one row: the split-KV
//           decode kernel; more: the prefill kernel, SUFFIX)
//   merge   the parts by their bases, the final normalisation, the log-sum-exp
#include "fa_checks.h"
#include "fa_internal.h"
#include "fa_prefill_kernel.h"

namespace fa {
namespace {

constexpr int CUS = 256;                 // compute units of the card
constexpr int MIN_TILES = 4;             // least tiles in a split of the prefix
constexpr int ROWS = WR * NSLOT;         // rows of a workgroup against the prefix

// One wave per row: partial results of `slots` parts merged, D / 64 columns a lane.
template <typename TOUT, int D>
__global__ __launch_bounds__(256) void merge_kernel(const float *__restrict__ opart, const float *__restrict__ mpart,
                                                    const float *__restrict__ lpart, void *o, float *lse, int slots,
                                                    int rows, int Hq, int Nq) {
    constexpr int N = D / 64;
    typedef float vec __attribute__((ext_vector_type(N)));
    typedef TOUT out __attribute__((ext_vector_type(N)));
    const int l = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const float *mp = mpart + (size_t)row * slots, *lp = lpart + (size_t)row * slots;
    const float *op = opart + (size_t)row * slots * D + N * l;
    float M = -INFINITY, L = 0.f;
    vec acc = vec{};
    for (int s0 = 0; s0 < slots; s0 += 8) {   // eight parts' loads together
        float m[8], w[8];
        vec x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int s = min(s0 + j, slots - 1);
            m[j] = s0 + j < slots ? mp[s] : -INFINITY;
            w[j] = lp[s];
            x[j] = *reinterpret_cast<const vec *>(op + (size_t)s * D);
        }
        float Mc = M;
#pragma unroll
        for (int j = 0; j < 8; ++j) Mc = __builtin_fmaxf(Mc, m[j]);
        const float alpha = M == -INFINITY ? 0.f : exp2_fast(M - Mc);
        L *= alpha;
        acc *= alpha;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float f = m[j] == -INFINITY ? 0.f : exp2_fast(m[j] - Mc);
            L = __builtin_fmaf(f, w[j], L);
#pragma unroll
            for (int n = 0; n < N; ++n) acc[n] = __builtin_fmaf(f, x[j][n], acc[n]);
        }
        M = Mc;
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

// Splits of the prefix, and partial results of a row's suffix.
struct Plan {
    int prefix, suffix;
};

int prefix_splits(long long rows, int Hkv, int Np, int D) {
    const int BC = D == 64 ? Cfg<64>::BC : Cfg<128>::BC, wpc = D == 64 ? Cfg<64>::WPC : Cfg<128>::WPC;
    const long long units = (rows + ROWS - 1) / ROWS * Hkv, tiles = ((long long)Np + BC - 1) / BC;
    long long S = (long long)CUS * wpc / units;
    if (S > tiles / MIN_TILES) S = tiles / MIN_TILES;
    if (S > FA_MAX_SPLITS) S = FA_MAX_SPLITS;
    return S < 1 ? 1 : (int)S;
}

Plan plan(int B, int Hq, int Hkv, int Nq, int Np, int Nk, int D, bool most) {
    Plan n;
    n.prefix = prefix_splits((long long)B * Nq * (Hq / Hkv), Hkv, Np, D);
    n.suffix = Nk < 1 ? 0 : Nq > 1 ? 1 : most ? decode_most_splits(B, Hq, Hkv, Nk, D) : decode_default_splits(B, Hq, Hkv, Nk, D);
    return n;
}

void common_args(const Problem &p, PrefillArgs &a) {
    a.q = p.q;
    a.o = p.o; a.lse = p.lse;
    a.B = p.B; a.Hq = p.Hq; a.Hkv = p.Hkv; a.Nq = p.Nq;
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
}

template <typename TIN, int D>
hipError_t launch_parts(const PrefixProblem &pp, const Plan &n, float *ws, hipStream_t stream) {
    using SM = Cfg<D>;
    const Problem &p = pp.p;
    const int G = p.Hq / p.Hkv, slots = n.prefix + n.suffix;
    const long long rows = (long long)p.B * p.Nq * G;   // of a key/value head
    const size_t parts = (size_t)rows * p.Hkv * slots;
    const int total = pp.Np + pp.suffix_rows;

    PrefillArgs a;
    common_args(p, a);
    a.opart = ws;
    a.mpart = ws + parts * D;
    a.lpart = a.mpart + parts;
    a.slots = slots;

    a.k = pp.k_prefix; a.v = pp.v_prefix;
    a.Nk = pp.Np;
    a.HW = 1;
    a.lgHW = 0;
    a.nmb = (int)((rows + ROWS - 1) / ROWS);
    a.first = a.nmb;
    a.nhg = Divisor(n.prefix);
    a.per_mb = Divisor((unsigned)p.Hkv * n.prefix);
    a.tokens = Divisor(p.Nq);
    a.group = Divisor(G);
    a.rows = (int)rows;
    a.splits = n.prefix;
    const int tiles = (pp.Np + SM::BC - 1) / SM::BC;
    a.per_split = (tiles + n.prefix - 1) / n.prefix;
    a.causal = p.causal;
    a.total = total;
    a.length0 = p.block_table ? 0 : pp.Np;
    a.slot0 = 0;
    const long long nblocks = (long long)a.nmb * p.Hkv * n.prefix;
    if (nblocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    if (p.block_table)
        hipLaunchKernelGGL((prefill_kernel<TIN, float, D, NSLOT, false, true, PREFIX>), dim3((unsigned)nblocks),
                           dim3(SM::NT), 0, stream, a);
    else
        hipLaunchKernelGGL((prefill_kernel<TIN, float, D, NSLOT, false, false, PREFIX>), dim3((unsigned)nblocks),
                           dim3(SM::NT), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || n.suffix == 0) return e;
    if (p.Nq == 1) return launch_decode_part(p, n.suffix, slots, n.prefix, p.block_table ? pp.Np : 0, ws, stream);

    a.k = p.k; a.v = p.v;
    a.Nk = pp.suffix_rows;
    a.HW = G % 4 == 0 ? 4 : G % 2 == 0 ? 2 : 1;
    a.lgHW = a.HW == 4 ? 2 : a.HW == 2 ? 1 : 0;
    const int RB = NSLOT / a.HW;
    a.nmb = (p.Nq + WR * RB - 1) / (WR * RB);
    a.first = a.nmb;
    const long long sblocks = (long long)a.nmb * p.B * p.Hkv * (G / a.HW);
    if (sblocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    a.nhg = Divisor(G / a.HW);
    a.per_mb = Divisor((unsigned)p.B * p.Hkv * (G / a.HW));
    a.length0 = p.block_table ? -pp.Np : 0;
    a.first_page = p.block_table ? pp.Np / p.page_size : 0;
    a.slot0 = n.prefix;
    const dim3 grid((unsigned)sblocks), block(SM::NT);
    if (p.block_table && p.causal)
        hipLaunchKernelGGL((prefill_kernel<TIN, float, D, NSLOT, true, true, SUFFIX>), grid, block, 0, stream, a);
    else if (p.block_table)
        hipLaunchKernelGGL((prefill_kernel<TIN, float, D, NSLOT, false, true, SUFFIX>), grid, block, 0, stream, a);
    else if (p.causal)
        hipLaunchKernelGGL((prefill_kernel<TIN, float, D, NSLOT, true, false, SUFFIX>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((prefill_kernel<TIN, float, D, NSLOT, false, false, SUFFIX>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <typename TOUT>
hipError_t launch_merge(const Problem &p, int slots, const float *ws, hipStream_t stream) {
    const long long rows = (long long)p.B * p.Nq * p.Hq;
    const size_t parts = (size_t)rows * slots;
    const float *m = ws + parts * p.D;
    const dim3 grid((unsigned)((rows + 3) / 4));
    if (p.D == 64)
        hipLaunchKernelGGL((merge_kernel<TOUT, 64>), grid, dim3(256), 0, stream, ws, m, m + parts, p.o, p.lse, slots,
                           (int)rows, p.Hq, p.Nq);
    else
        hipLaunchKernelGGL((merge_kernel<TOUT, 128>), grid, dim3(256), 0, stream, ws, m, m + parts, p.o, p.lse, slots,
                           (int)rows, p.Hq, p.Nq);
    return hipGetLastError();
}

}  // namespace

size_t prefix_workspace_bytes(int B, int Hq, int Hkv, int Nq, int Np, int Nk, int D, bool most) {
    const Plan n = plan(B, Hq, Hkv, Nq, Np, Nk, D, most);
    return (size_t)B * Nq * Hq * (n.prefix + n.suffix) * (size_t)(D + 2) * sizeof(float);
}

hipError_t launch_prefix(const PrefixProblem &pp, void *workspace, hipStream_t stream) {
    const Problem &p = pp.p;
    const Plan n = plan(p.B, p.Hq, p.Hkv, p.Nq, pp.Np, pp.suffix_rows, p.D, false);
    float *ws = reinterpret_cast<float *>(workspace);
    hipError_t e;
    if (p.in == FA_F16)
        e = p.D == 64 ? launch_parts<f16_t, 64>(pp, n, ws, stream) : launch_parts<f16_t, 128>(pp, n, ws, stream);
    else
        e = p.D == 64 ? launch_parts<bf16_t, 64>(pp, n, ws, stream) : launch_parts<bf16_t, 128>(pp, n, ws, stream);
    if (e != hipSuccess) return e;
    const int slots = n.prefix + n.suffix;
    if (p.out == FA_F32) return launch_merge<float>(p, slots, ws, stream);
    return p.in == FA_F16 ? launch_merge<_Float16>(p, slots, ws, stream) : launch_merge<__bf16>(p, slots, ws, stream);
}

}  // namespace fa
