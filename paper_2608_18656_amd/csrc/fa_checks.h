// fa_checks.h -- the host-side argument checks of the attention entry points
// (plain C++, no HIP: the library includes it, and a sanitizer build of the
// test suite compiles it with g++ alone).
#pragma once

#include <cmath>
#include <cstddef>
#include <cstdint>

#include "../../include/fa.h"

namespace fa {

inline size_t esize(fa_dtype_t t) { return t == FA_F32 ? 4 : 2; }

// Whether the byte ranges [a, a + na) and [b, b + nb) intersect.
inline bool overlaps(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

// r = a * b for positive a, b, refused (false) when the product would exceed
// INT64_MAX / 4 (element counts that later get multiplied by element sizes).
inline bool mul_ok(long long a, long long b, long long *r) {
    if (a > 0 && b > 0 && a > (long long)(INT64_MAX / 4) / b) return false;
    *r = a * b;
    return true;
}

// Whether the offsets within a tile of `rows` key rows of 16-bit elements fit
// the 31 bits that the prefill and decode kernels have for them: key rows of
// some 33 MiB (64 rows) or 66 MiB (32 rows) and more do not.
inline bool tile_fits(int Hkv, int D, int rows) {
    return (long long)(rows - 1) * Hkv * D * 2 + 2 * D <= 0x7fffffffLL;
}

// The argument checks of every attention entry point.  kv_rows: rows of
// Hkv * D elements that k and v each hold (-1: B * Nk, the contiguous layout).
inline fa_status_t validate_core(const void *q, const void *k, const void *v, const void *o,
                                 const float *lse, int B, int Hq, int Hkv, int Nq, int Nk, int D,
                                 int causal, float scale, fa_dtype_t in, fa_dtype_t out,
                                 long long kv_rows) {
    if (!q || !k || !v || !o) return FA_ERR_NULL;
    if (B < 1 || Hq < 1 || Hkv < 1 || Nq < 1 || Nk < 1 || D < 1) return FA_ERR_DIM;
    if (in != FA_F16 && in != FA_BF16 && in != FA_F32) return FA_ERR_DTYPE;
    if (out != in && out != FA_F32) return FA_ERR_DTYPE;
    if (Hq % Hkv != 0) return FA_ERR_GQA_RATIO;
    if (D % 8 != 0 || D > 256) return FA_ERR_HEAD_DIM;
    if (causal && Nq > Nk) return FA_ERR_CAUSAL_SHAPE;
    if (!std::isfinite(scale)) return FA_ERR_SCALE;
    long long nq, nk, t;
    if (kv_rows < 0) kv_rows = (long long)B * Nk;
    if (!mul_ok((long long)B * Nq, (long long)Hq * D, &nq) ||
        !mul_ok(kv_rows, (long long)Hkv * D, &nk) ||
        !mul_ok((long long)B * Hq, (long long)Nq, &t))
        return FA_ERR_DIM;
    const uintptr_t a16 = 15;
    if ((reinterpret_cast<uintptr_t>(q) & a16) || (reinterpret_cast<uintptr_t>(k) & a16) ||
        (reinterpret_cast<uintptr_t>(v) & a16) || (reinterpret_cast<uintptr_t>(o) & a16) ||
        (reinterpret_cast<uintptr_t>(lse) & 3))
        return FA_ERR_ALIGN;
    const size_t qb = (size_t)nq * esize(in), kb = (size_t)nk * esize(in);
    const size_t ob = (size_t)nq * esize(out), lb = (size_t)t * sizeof(float);
    if (overlaps(o, ob, q, qb) || overlaps(o, ob, k, kb) || overlaps(o, ob, v, kb))
        return FA_ERR_ALIAS;
    if (lse && (overlaps(lse, lb, q, qb) || overlaps(lse, lb, k, kb) ||
                overlaps(lse, lb, v, kb) || overlaps(lse, lb, o, ob)))
        return FA_ERR_ALIAS;
    return FA_OK;
}

inline bool misaligned(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// A range of memory that a call reads or writes.
struct Range {
    const void *p;
    size_t bytes;
};

// The argument checks of fa_kvcache_append (table NULL) and its paged form.
// cache_rows: rows of Hkv * D elements that each cache holds.  Strides are
// those in use (0 already replaced).
inline fa_status_t validate_append(const void *k, const void *v, const void *k_cache, const void *v_cache,
                                   const void *q, const void *q_out, const int *seqlens, int B, int Hq, int Hkv,
                                   int N, int D, long long qs, long long ks, long long vs, const fa_rotary_t *rotary,
                                   fa_dtype_t dtype, long long cache_rows, const int *table, int max_pages) {
    if (!k || !v || !k_cache || !v_cache || !seqlens || (q == nullptr) != (q_out == nullptr) ||
        (rotary && !rotary->inv_freq))
        return FA_ERR_NULL;
    if (B < 1 || Hkv < 1 || (q && Hq < 1) || N < 1 || cache_rows < 1 || D < 1) return FA_ERR_DIM;
    if (dtype != FA_F16 && dtype != FA_BF16 && dtype != FA_F32) return FA_ERR_DTYPE;
    if (q && Hq % Hkv != 0) return FA_ERR_GQA_RATIO;
    if (D % 8 != 0 || D > 256) return FA_ERR_HEAD_DIM;
    const long long heads = (q ? Hq : 0) + 2LL * Hkv, tokens = (long long)B * N;
    if (heads * D > (1LL << 28) || tokens > FA_MAX_APPEND_TOKENS) return FA_ERR_DIM;
    if ((q && qs < (long long)Hq * D) || ks < (long long)Hkv * D || vs < (long long)Hkv * D) return FA_ERR_DIM;
    long long nq = 0, nk, nv, nc;
    if ((q && !mul_ok(tokens, qs, &nq)) || !mul_ok(tokens, ks, &nk) || !mul_ok(tokens, vs, &nv) ||
        !mul_ok(cache_rows, (long long)Hkv * D, &nc))
        return FA_ERR_DIM;
    if (rotary) {
        if (rotary->rot_dim < 2 || rotary->rot_dim % 2 != 0 || rotary->rot_dim > D || rotary->axes < 1 ||
            rotary->axes > FA_MAX_AXES || (rotary->axes > 1 && !rotary->positions))
            return FA_ERR_ROTARY;
        if (rotary->axes > 1)
            for (int j = 0; j < rotary->rot_dim / 2; ++j)
                if (rotary->pair_axis[j] >= rotary->axes) return FA_ERR_ROTARY;
    }
    const long long e = (long long)esize(dtype);
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(k_cache, 16) || misaligned(v_cache, 16) ||
        misaligned(q, 16) || misaligned(q_out, 16) || misaligned(seqlens, 4) || misaligned(table, 4) ||
        (rotary && (misaligned(rotary->inv_freq, 4) || misaligned(rotary->positions, 4))) || (q && qs * e % 16 != 0) ||
        ks * e % 16 != 0 || vs * e % 16 != 0)
        return FA_ERR_ALIGN;
    const size_t dense = (size_t)tokens * Hq * D * e, cb = (size_t)(nc * e);
    const Range in[] = {{k, (size_t)((nk - ks + (long long)Hkv * D) * e)},
                        {v, (size_t)((nv - vs + (long long)Hkv * D) * e)},
                        {q, q ? (size_t)((nq - qs + (long long)Hq * D) * e) : 0},
                        {seqlens, (size_t)B * sizeof(int)},
                        {table, table ? (size_t)B * max_pages * sizeof(int) : 0},
                        {rotary ? rotary->inv_freq : nullptr, rotary ? (size_t)rotary->rot_dim / 2 * sizeof(float) : 0},
                        {rotary ? rotary->positions : nullptr,
                         rotary && rotary->positions ? (size_t)rotary->axes * tokens * sizeof(int) : 0}};
    const Range out[] = {{k_cache, cb}, {v_cache, cb}, {q_out, q ? dense : 0}};
    for (int i = 0; i < 3; ++i) {
        if (!out[i].bytes) continue;
        for (const Range &r : in) {
            if (!r.bytes || (i == 2 && r.p == q && q == q_out && qs == (long long)Hq * D)) continue;
            if (overlaps(out[i].p, out[i].bytes, r.p, r.bytes)) return FA_ERR_ALIAS;
        }
        for (int j = 0; j < i; ++j)
            if (overlaps(out[i].p, out[i].bytes, out[j].p, out[j].bytes)) return FA_ERR_ALIAS;
    }
    return FA_OK;
}

}  // namespace fa
