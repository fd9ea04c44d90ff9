// fa_append.hip -- new keys and values into a K/V cache (contiguous or paged),
// keys and queries rotated by their positions on the way.
//
// A pair (a, b) of columns at position p becomes (a cos t - b sin t, a sin t +
// b cos t) with t = p * inv_freq[pair]; p is the token's row in the cache, or
// the position given for the pair's axis.  t is formed in 64 bits and reduced to
// a fraction of a turn there (p = 10^6 radians in 32 bits would be 0.03 off);
// sine, cosine and the rotation are 32-bit, rounded once to the element type.
//
// Work split.  A workgroup takes TB tokens: their angles, one per lane and
// pair, and their cache rows go through LDS, since all Hq + Hkv heads of a
// token share them.  Then a thread takes units of two 16-byte chunks of a head
// row, those whose columns rotate together (both halves of the rotated columns,
// or any two chunks where pairs are neighbours), so that it writes exactly what
// it has read, and a rotation in place needs no barrier.
// What bounds it: HBM for long prompts (8192 tokens, 32/8 heads, D = 128, fp16: 34.8 to
// 37.6 us, 5.4 to 5.8 TB/s read and written; a large copy reaches 5.0), the chain launch,
// lengths, table entry, store for a step of single tokens (64: 4.2 us).
#include "fa_common.h"
#include "fa_internal.h"

namespace fa {
namespace {

constexpr int NT = 256;           // threads per workgroup
constexpr int MAX_PAIRS = 128;    // D <= 256
// Bytes read and written up to which the inputs are read through the caches.  A
// projection leaves its result in the memory side's 256 MB, from where plain loads are
// quicker; a long prompt's does not stay there with what is written.  32/8 heads, D =
// 128, fp16, us with plain / non-temporal loads, right behind a kernel that writes the
// inputs: 73 MB 14.4 / 15.2, 88 16.7 / 16.6, 103 19.1 / 19.0, 131 23.1 / 23.4, 147 25.6 /
// 26.2, 172 31.7 / 29.2, 201 36.8 / 35.7; three sets in turn: 73 MB 14.9 / 18.7, 88 20.3
// / 20.2, 103 24.8 / 23.5, 131 31.9 / 27.7, 201 46.1 / 41.3.
constexpr long long HELD = 96 << 20;

struct AppendArgs {
    const void *q, *k, *v;
    void *qo, *kc, *vc;
    long long qs, ks, vs;         // elements between consecutive tokens of q, k, v
    const int *seqlens;
    int B, Hq, Hkv, N, Nk, D;
    const float *inv_freq;
    const int *positions;         // [axes][B][N], or NULL: the cache row
    int rot, interleaved;
    unsigned axis[MAX_PAIRS / 16];   // two bits per pair
    const int *block_table;
    Divisor page_size;
    int max_pages, num_pages;
    int tokens;                   // B N
    Divisor per_seq;              // N
    Divisor pairs;                // rot / 2, at least 1
    Divisor units, row_units;     // units per token and per head row
};

// Element types: fp32 and the 16-bit ones.
template <typename S> struct Chunk {
    static constexpr int E = 16 / sizeof(S);
    typedef S vec __attribute__((ext_vector_type(16 / sizeof(S))));
};

// 16 bytes of an input; ONCE: past the caches.
template <typename V, bool ONCE> __device__ __forceinline__ V load(const void *p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const V *>(p));
    else return *reinterpret_cast<const V *>(p);
}

// VEC: chunks hold whole pairs (interleaved) or whole chunks pair (halves);
// else single elements, any even number of rotated columns.
template <typename S, bool VEC, int TB, bool ONCE>
__global__ __launch_bounds__(NT) void append_kernel(AppendArgs a) {
    constexpr int E = Chunk<S>::E;
    typedef typename Chunk<S>::vec V;
    __shared__ float2 turn[TB * MAX_PAIRS];
    __shared__ long long dest[TB];   // the token's row in the caches, -1: none

    const int tid = threadIdx.x, t0 = blockIdx.x * TB;
    const int here = min(TB, a.tokens - t0), half = a.rot / 2;
    for (int e = tid; e < here * half; e += NT) {
        const int t = a.pairs.div(e), j = e - t * half;
        const int tok = t0 + t, b = a.per_seq.div(tok), i = tok - b * a.N;
        int p;
        if (a.positions) {
            const int ax = (a.axis[j >> 4] >> (2 * (j & 15))) & 3;
            p = a.positions[(size_t)ax * a.tokens + tok];
        } else {
            p = max(a.seqlens[b], 0) - a.N + i;
        }
        const double turns = (double)p * ((double)a.inv_freq[j] * 0.15915494309189535);
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        turn[t * MAX_PAIRS + j] = float2{c, s};
    }
    if (tid < here) {
        const int tok = t0 + tid, b = a.per_seq.div(tok), r = max(a.seqlens[b], 0) - a.N + (tok - b * a.N);
        long long at = -1;
        if (r >= 0 && r < a.Nk) {
            if (a.block_table) {
                const int pi = a.page_size.div(r), page = a.block_table[(size_t)b * a.max_pages + pi];
                if (page >= 0 && page < a.num_pages) at = (long long)page * a.page_size.d + (r - pi * (int)a.page_size.d);
            } else {
                at = (long long)b * a.Nk + r;
            }
        }
        dest[tid] = at;
    }
    __syncthreads();

    const int items = here * (int)a.units.d;
    for (int it = tid; it < items; it += NT) {
        const int t = a.units.div(it), ru = it - t * (int)a.units.d;
        const int row = a.row_units.div(ru), u = ru - row * (int)a.row_units.d;
        const size_t tok = (size_t)t0 + t;
        const S *src;
        S *dst;
        bool rotate = true;
        if (row < a.Hq) {
            src = reinterpret_cast<const S *>(a.q) + tok * a.qs + (size_t)row * a.D;
            dst = reinterpret_cast<S *>(a.qo) + (tok * a.Hq + row) * a.D;
        } else {
            const int g = row - a.Hq;
            rotate = g < a.Hkv;
            const int h = rotate ? g : g - a.Hkv;
            const long long at = dest[t];
            if (at < 0) continue;
            src = rotate ? reinterpret_cast<const S *>(a.k) + tok * a.ks : reinterpret_cast<const S *>(a.v) + tok * a.vs;
            src += (size_t)h * a.D;
            dst = reinterpret_cast<S *>(rotate ? a.kc : a.vc) + ((size_t)at * a.Hkv + h) * a.D;
        }
        const float2 *tp = turn + t * MAX_PAIRS;
        const int rot = rotate ? a.rot : 0;
        if constexpr (VEC) {
            const int chunks = a.D / E;
            if (rot > 0 && !a.interleaved) {
                const int hc = rot / (2 * E);   // chunks of a half
                if (u < hc) {
                    V x = load<V, ONCE>(src + E * u), y = load<V, ONCE>(src + E * (u + hc));
                    V xo, yo;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float2 w = tp[E * u + e];
                        const float f = (float)x[e], g = (float)y[e];
                        xo[e] = from_f32<S>(f * w.x - g * w.y);
                        yo[e] = from_f32<S>(f * w.y + g * w.x);
                    }
                    *reinterpret_cast<V *>(dst + E * u) = xo;
                    *reinterpret_cast<V *>(dst + E * (u + hc)) = yo;
                } else {   // the columns past the rotated ones
                    const int rest = chunks - 2 * hc, n = (rest + 1) / 2, c0 = 2 * hc + (u - hc), c1 = c0 + n;
                    const V x = load<V, ONCE>(src + E * c0);
                    if (c1 < chunks) *reinterpret_cast<V *>(dst + E * c1) = load<V, ONCE>(src + E * c1);
                    *reinterpret_cast<V *>(dst + E * c0) = x;
                }
            } else {
                const int c1 = u + (int)a.row_units.d;
                const bool two = c1 < chunks;
                V x[2];
                x[0] = load<V, ONCE>(src + E * u);
                if (two) x[1] = load<V, ONCE>(src + E * c1);
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const int c = n ? c1 : u;
                    if (n && !two) break;
                    if (E * c < rot) {
#pragma unroll
                        for (int e = 0; e < E; e += 2) {
                            const float2 w = tp[(E * c + e) / 2];
                            const float f = (float)x[n][e], g = (float)x[n][e + 1];
                            x[n][e] = from_f32<S>(f * w.x - g * w.y);
                            x[n][e + 1] = from_f32<S>(f * w.y + g * w.x);
                        }
                    }
                    *reinterpret_cast<V *>(dst + E * c) = x[n];
                }
            }
        } else {
            // unit u: a pair, or two of the columns past the rotated ones, element by
            // element (8192 tokens, 32/8 heads, fp16: 20 of 128 columns rotated 66.7 us, all
            // of them 43.6; 24 of 96 in halves 52.9, as neighbours in chunks 36.6)
            const int i0 = 2 * u < rot && !a.interleaved ? u : 2 * u, i1 = 2 * u < rot && !a.interleaved ? u + rot / 2 : 2 * u + 1;
            S x = src[i0], y = src[i1];
            if (2 * u < rot) {
                const float2 w = tp[u];
                const float f = (float)x, g = (float)y;
                x = from_f32<S>(f * w.x - g * w.y);
                y = from_f32<S>(f * w.y + g * w.x);
            }
            dst[i0] = x;
            dst[i1] = y;
        }
    }
}

template <typename S, bool VEC>
hipError_t launch_t(AppendArgs &a, hipStream_t s) {
    const int rows = a.Hq + 2 * a.Hkv;
    const int ru = VEC ? (a.D / Chunk<S>::E + 1) / 2 : a.D / 2;
    a.row_units = Divisor(ru);
    a.units = Divisor((unsigned)rows * ru);
    constexpr int TB = 4;
    const unsigned blocks = ((unsigned)a.tokens + TB - 1) / TB;
    const long long bytes = 2LL * a.tokens * rows * a.D * sizeof(S);   // read and written
    if (a.tokens <= 1024)   // a workgroup each
        hipLaunchKernelGGL((append_kernel<S, VEC, 1, false>), dim3((unsigned)a.tokens), dim3(NT), 0, s, a);
    else if (bytes <= HELD)
        hipLaunchKernelGGL((append_kernel<S, VEC, TB, false>), dim3(blocks), dim3(NT), 0, s, a);
    else
        hipLaunchKernelGGL((append_kernel<S, VEC, TB, true>), dim3(blocks), dim3(NT), 0, s, a);
    return hipGetLastError();
}

template <typename S>
hipError_t launch_s(AppendArgs &a, hipStream_t s) {
    constexpr int E = Chunk<S>::E;
    const bool vec = a.rot % (a.interleaved ? E : 2 * E) == 0;
    return vec ? launch_t<S, true>(a, s) : launch_t<S, false>(a, s);
}

}  // namespace

hipError_t launch_append(const AppendProblem &p, hipStream_t stream) {
    AppendArgs a;
    a.q = p.q; a.k = p.k; a.v = p.v;
    a.qo = p.q_out; a.kc = p.k_cache; a.vc = p.v_cache;
    a.qs = p.q_stride; a.ks = p.k_stride; a.vs = p.v_stride;
    a.seqlens = p.seqlens;
    a.B = p.B; a.Hq = p.q ? p.Hq : 0; a.Hkv = p.Hkv; a.N = p.N; a.Nk = p.Nk; a.D = p.D;
    a.rot = 0;
    a.interleaved = 0;
    a.inv_freq = nullptr;
    a.positions = nullptr;
    for (unsigned &w : a.axis) w = 0;
    if (p.rotary) {
        a.rot = p.rotary->rot_dim;
        a.interleaved = p.rotary->interleaved != 0;
        a.inv_freq = p.rotary->inv_freq;
        a.positions = p.rotary->positions;
        if (p.rotary->axes > 1)
            for (int j = 0; j < a.rot / 2; ++j) a.axis[j >> 4] |= (unsigned)p.rotary->pair_axis[j] << (2 * (j & 15));
    }
    a.pairs = Divisor(a.rot > 0 ? a.rot / 2 : 1);
    a.block_table = p.block_table;
    a.page_size = Divisor(p.block_table ? p.page_size : 1);
    a.max_pages = p.max_pages;
    a.num_pages = p.num_pages;
    a.tokens = p.B * p.N;
    a.per_seq = Divisor(p.N);
    switch (p.dtype) {
    case FA_F32: return launch_s<float>(a, stream);
    case FA_F16: return launch_s<_Float16>(a, stream);
    default: return launch_s<__bf16>(a, stream);
    }
}

}  // namespace fa
