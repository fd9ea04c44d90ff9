// fa_api.hip -- the exported C entry points: argument validation, dispatch to
// the prefill / decode / generic / unfused kernels, and the decode workspace.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <exception>
#include <mutex>
#include <vector>

#include "../../include/fa.h"
#include "fa_checks.h"
#include "fa_internal.h"

namespace {

using fa::esize;
using fa::overlaps;
using fa::validate_core;

// Device workspace for the split-KV partial results.  Library-owned buffers
// are kept per (device, stream), so that calls on different streams never
// share one; a buffer that is outgrown is retired, not freed (an earlier call
// or a captured graph may still use it) until fa_release_workspace().  No
// buffer is allocated while the stream is being captured.  A caller-owned
// workspace set with fa_set_workspace() replaces them for its device.
struct OwnedWs {
    int dev;
    hipStream_t stream;
    void *ptr;
    size_t bytes;
};
struct Retired {
    int dev;
    void *ptr;
};
constexpr int kMaxDevices = 64;
struct UserWs {
    void *ptr = nullptr;
    size_t bytes = 0;
};
UserWs g_user[kMaxDevices];
std::vector<OwnedWs> g_owned;
std::vector<Retired> g_retired;
// Guards these, and is held by a call that uses one of the buffers until all of its
// kernels are enqueued: another host thread's call on the same stream must not come
// between the kernel that leaves partial results and the one that merges them, nor
// a release between the choice of a buffer and its use.
std::mutex g_ws_mu;

// need: what the call uses; room: what a new buffer holds (for shorter caches too).
// With g_ws_mu held.
fa_status_t get_workspace(size_t need, size_t room, hipStream_t stream, void **out, bool *user) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return FA_ERR_HIP;
    *user = g_user[dev].ptr != nullptr;
    if (*user) {
        if (g_user[dev].bytes < need) return FA_ERR_WORKSPACE;
        *out = g_user[dev].ptr;
        return FA_OK;
    }
    OwnedWs *cur = nullptr;
    for (OwnedWs &w : g_owned)
        if (w.dev == dev && w.stream == stream) cur = &w;
    if (cur && cur->bytes >= need) {
        *out = cur->ptr;
        return FA_OK;
    }
    // a new buffer is needed: never inside stream capture (the allocation
    // would invalidate it)
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(stream, &cs) != hipSuccess) {
        (void)hipGetLastError();
        return FA_ERR_WORKSPACE;
    }
    if (cs != hipStreamCaptureStatusNone) return FA_ERR_WORKSPACE;
    const size_t sz = room < ((size_t)1 << 20) ? ((size_t)1 << 20) : room;
    void *ptr = nullptr;
    // room in the list that grows first: no exception may leave a C entry.  (Not in
    // g_owned with cur, which points into it.)
    try {
        if (cur) g_retired.reserve(g_retired.size() + 1);
        else g_owned.reserve(g_owned.size() + 1);
    } catch (const std::exception &) {
        return FA_ERR_WORKSPACE;
    }
    if (hipMalloc(&ptr, sz) != hipSuccess) {
        (void)hipGetLastError();
        return FA_ERR_WORKSPACE;
    }
    if (cur) {
        g_retired.push_back(Retired{dev, cur->ptr});
        cur->ptr = ptr;
        cur->bytes = sz;
    } else {
        g_owned.push_back(OwnedWs{dev, stream, ptr, sz});
    }
    *out = ptr;
    return FA_OK;
}

// A caller-owned workspace passed with one call (the *_ws entry points).
struct CallWs {
    void *ptr;
    size_t bytes;
};

// Fixed device scratch of fa_fwd_splitkv_noalloc: the split-KV partial results
// of its calls live here (each GPU holds its own copy until the process
// ends).  Host code never passes `scratch` itself to a kernel (on the host
// that name is a stand-in, not a device address): the address of the
// device's copy is read once per device with hipGetSymbolAddress and kept.
constexpr size_t kScratchBytes = (size_t)32 << 20;
static __device__ __align__(256) unsigned char scratch[kScratchBytes];
void *g_scratch_ptr[kMaxDevices];
std::mutex g_scratch_mu;   // guards these, and is held until a call's kernels are enqueued

// Device address of the current device's scratch (read on the first call per
// device, with that device current).  With g_scratch_mu held.
fa_status_t scratch_address(void **out) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return FA_ERR_HIP;
    if (!g_scratch_ptr[dev]) {
        void *ptr = nullptr;
        if (hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch)) != hipSuccess || ptr == nullptr) {
            (void)hipGetLastError();
            return FA_ERR_HIP;
        }
        g_scratch_ptr[dev] = ptr;
    }
    *out = g_scratch_ptr[dev];
    return FA_OK;
}

// What a query sees, besides causal: with size > 0 the `size` keys up to its own and the first `sinks`.
struct Window {
    int size = 0, sinks = 0;
};

// Splits of a decode call, and the most of any shorter cache.  With a window they
// go by the keys that it leaves, as for a cache of that length: one split would save
// the merge's launch, and with it 2 to 3 us of the host's time a call, but costs the
// GPU more (32/8 heads, D = 64, one sequence, caches that nothing holds, us replayed
// from a graph / waited for, several splits against one: 512 keys, one by the model,
// 7.3 / 23.3; 640 7.4 / 24.2 against 8.2 / 25.1, 768 7.6 / 24.5 against 9.2 / 25.7, 1024
// 7.7 / 24.6 against 10.9 / 27.4; 16/1 heads, 640 6.7 / 23.1 against 6.5 / 23.1, 768 7.0 /
// 23.7 against 7.0 / 23.4, 1024 7.0 / 23.5 against 8.0 / 24.0).
int decode_splits(int B, int Hq, int Hkv, int Nk, int D, const Window &w, bool most) {
    long long keys = Nk;
    if (w.size > 0 && (long long)w.size + w.sinks < keys) keys = (long long)w.size + w.sinks;
    return most ? fa::decode_most_splits(B, Hq, Hkv, (int)keys, D) : fa::decode_default_splits(B, Hq, Hkv, (int)keys, D);
}

// Most keys of a call: the kernels count keys in ints, up to the end of the last tile of
// at most 128, a tile ahead, and a window's length behind a row of the 128 before a
// tile.  Without a window the decode kernel's chunks of 32 need only their own end, and
// pages, of 64 keys at least, stop 64 ahead of 2^31: enough for the 16-bit kernels' tiles.
constexpr int kMostKeys = 0x7fffffff - 255;
bool keys_fit(int Nk, bool decode, bool prefill, bool paged, bool windowed) {
    if (Nk <= kMostKeys) return true;
    if (windowed) return false;
    return paged ? decode || prefill : decode && Nk <= 0x7fffffff - 31;
}

struct Paging {
    const int *block_table = nullptr;
    int page_size = 0, max_pages = 0, num_pages = 0;
};

fa_status_t run(const void *q, const void *k, const void *v, void *o, float *lse, int B, int Hq,
                int Hkv, int Nq, int Nk, int D, int causal, float scale, void *stream,
                fa_dtype_t in, fa_dtype_t out, int splits_req, int hw_req = 0,
                const int *seqlens = nullptr, const Paging &pg = Paging(),
                const CallWs *cws = nullptr, int slots_req = 0, const Window &win = Window()) {
    const long long kv_rows = pg.block_table ? (long long)pg.num_pages * pg.page_size : -1;
    fa_status_t st = validate_core(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, in, out, kv_rows);
    if (st != FA_OK) return st;
    if (splits_req < 0 || splits_req > FA_MAX_SPLITS) return FA_ERR_SPLITS;
    const int slots = slots_req > 0 ? slots_req : 4;
    if (!(slots_req == 0 || slots_req == 1 || slots_req == 2 || slots_req == 4 || slots_req == 8) ||
        !(hw_req == 0 || hw_req == 1 || hw_req == 2 || hw_req == 4 || hw_req == 8) ||
        (hw_req > 0 && ((Hq / Hkv) % hw_req != 0 || slots % hw_req != 0)))
        return FA_ERR_PACKING;
    fa::Problem p{q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, in, out, hw_req, slots_req, seqlens,
                  pg.block_table, pg.page_size, pg.max_pages, pg.num_pages,
                  win.size < Nk ? win.size : Nk, win.sinks < Nk ? win.sinks : Nk};
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const bool decode = fa::decode_supported(Nq, Hkv, D, in), prefill = fa::prefill_supported(Hkv, D, in);
    const bool windowed = win.size > 0;
    if (!keys_fit(Nk, decode, prefill, pg.block_table != nullptr, windowed)) return FA_ERR_DIM;
    // partial results: bytes that the call uses, and that a new buffer holds
    int S = 1;
    size_t need = 0, room = 0;
    if (decode) {
        S = splits_req > 0 ? splits_req : decode_splits(B, Hq, Hkv, Nk, D, win, false);
        need = fa::decode_workspace_bytes(B, Hq, D, S);
        room = fa::decode_workspace_bytes(B, Hq, D, splits_req > 0 ? splits_req : decode_splits(B, Hq, Hkv, Nk, D, win, true));
    } else if (windowed && prefill) {
        need = fa::window_workspace_bytes(B, Hq, Hkv, Nq, Nk, D, p.window, p.sinks, false);
        room = fa::window_workspace_bytes(B, Hq, Hkv, Nq, Nk, D, p.window, p.sinks, true);
    }
    void *ws = nullptr;
    std::unique_lock<std::mutex> lock(g_ws_mu, std::defer_lock);
    if (need > 0) {
        bool user = false;
        if (cws) {   // this call's own workspace: checked here, never allocated
            if (!cws->ptr) return FA_ERR_NULL;
            if (reinterpret_cast<uintptr_t>(cws->ptr) & 15) return FA_ERR_ALIGN;
            if (cws->bytes < need) return FA_ERR_WORKSPACE;
            ws = cws->ptr;
            user = true;
        } else {
            lock.lock();
            st = get_workspace(need, room, s, &ws, &user);
            if (st != FA_OK) return st;
        }
        if (user) {   // a caller-owned workspace must not overlap the call's tensors
            const size_t qb = (size_t)B * Nq * Hq * D * esize(in);
            const size_t kb = (size_t)(kv_rows < 0 ? (long long)B * Nk : kv_rows) * Hkv * D * esize(in);
            const size_t ob = (size_t)B * Nq * Hq * D * esize(out), lb = (size_t)B * Hq * Nq * sizeof(float);
            if (overlaps(ws, need, q, qb) || overlaps(ws, need, k, kb) || overlaps(ws, need, v, kb) ||
                overlaps(ws, need, o, ob) || (lse && overlaps(ws, need, lse, lb)) ||
                (seqlens && overlaps(ws, need, seqlens, (size_t)B * sizeof(int))) ||
                (pg.block_table && overlaps(ws, need, pg.block_table, (size_t)B * pg.max_pages * sizeof(int))))
                return FA_ERR_ALIAS;
        }
    }
    const hipError_t e = decode ? fa::launch_decode(p, S, ws, s)
                         : prefill ? (windowed ? fa::launch_prefill_window(p, ws, s) : fa::launch_prefill(p, s))
                                   : (windowed ? fa::launch_generic_window(p, s) : fa::launch_generic(p, s));
    return e == hipSuccess ? FA_OK : FA_ERR_HIP;
}

}  // namespace

extern "C" {

const char *fa_status_string(fa_status_t s) {
    switch (s) {
    case FA_OK: return "FA_OK";
    case FA_ERR_NULL: return "FA_ERR_NULL: q, k, v or o is NULL";
    case FA_ERR_DIM: return "FA_ERR_DIM: a size is < 1 or the tensors are too large";
    case FA_ERR_GQA_RATIO: return "FA_ERR_GQA_RATIO: Hq is not a multiple of Hkv";
    case FA_ERR_HEAD_DIM: return "FA_ERR_HEAD_DIM: D must be a multiple of 8 and at most 256";
    case FA_ERR_CAUSAL_SHAPE: return "FA_ERR_CAUSAL_SHAPE: causal requires Nq <= Nk";
    case FA_ERR_SCALE: return "FA_ERR_SCALE: scale is NaN or infinite";
    case FA_ERR_ALIGN: return "FA_ERR_ALIGN: a tensor pointer is misaligned";
    case FA_ERR_ALIAS: return "FA_ERR_ALIAS: o or lse overlaps another tensor";
    case FA_ERR_DTYPE: return "FA_ERR_DTYPE: unsupported dtype combination";
    case FA_ERR_WORKSPACE:
        return "FA_ERR_WORKSPACE: workspace allocation failed or not allowed during stream capture, or a caller-owned workspace is too small";
    case FA_ERR_HIP: return "FA_ERR_HIP: HIP runtime or launch error";
    case FA_ERR_SPLITS: return "FA_ERR_SPLITS: num_splits out of range";
    case FA_ERR_PACKING:
        return "FA_ERR_PACKING: slots_per_workgroup must be 0, 1, 2, 4 or 8; heads_per_workgroup 0, 1, 2, 4 or "
               "8, dividing Hq / Hkv and the slots";
    case FA_ERR_ROTARY:
        return "FA_ERR_ROTARY: rot_dim must be even, 2 to D; axes 1 to 4, with positions if several, and pair_axis "
               "below axes";
    case FA_ERR_WINDOW: return "FA_ERR_WINDOW: window must be at least 1 and sinks not negative";
    }
    return "unknown fa_status_t";
}

int fa_version(void) { return (0 << 16) | (1 << 8) | 0; }

fa_status_t fa_validate(const void *q, const void *k, const void *v, const void *o,
                        const float *lse, int B, int Hq, int Hkv, int Nq, int Nk, int D,
                        int causal, float scale, fa_dtype_t in, fa_dtype_t out) {
    const fa_status_t st = validate_core(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, in, out, -1);
    if (st != FA_OK) return st;
    return keys_fit(Nk, fa::decode_supported(Nq, Hkv, D, in), fa::prefill_supported(Hkv, D, in), false, false) ? FA_OK
                                                                                                              : FA_ERR_DIM;
}

fa_status_t fa_fwd(const void *q, const void *k, const void *v, void *o, float *lse, int B,
                   int Hq, int Hkv, int Nq, int Nk, int D, int causal, float scale, void *stream,
                   fa_dtype_t in_dtype, fa_dtype_t out_dtype) {
    return run(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, in_dtype, out_dtype,
               0);
}

fa_status_t fa_fwd_f16(const void *q, const void *k, const void *v, void *o, float *lse, int B,
                       int Hq, int Hkv, int Nq, int Nk, int D, int causal, float scale,
                       void *stream) {
    return run(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, FA_F16, FA_F16, 0);
}

fa_status_t fa_fwd_bf16(const void *q, const void *k, const void *v, void *o, float *lse, int B,
                        int Hq, int Hkv, int Nq, int Nk, int D, int causal, float scale,
                        void *stream) {
    return run(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, FA_BF16, FA_BF16,
               0);
}

fa_status_t fa_fwd_f32(const void *q, const void *k, const void *v, void *o, float *lse, int B,
                       int Hq, int Hkv, int Nq, int Nk, int D, int causal, float scale,
                       void *stream) {
    return run(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, FA_F32, FA_F32, 0);
}

fa_status_t fa_fwd_splitkv(const void *q, const void *k, const void *v, void *o, float *lse,
                           int B, int Hq, int Hkv, int Nq, int Nk, int D, int causal, float scale,
                           void *stream, fa_dtype_t in_dtype, fa_dtype_t out_dtype,
                           int num_splits) {
    return run(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, in_dtype, out_dtype,
               num_splits);
}

fa_status_t fa_fwd_packed(const void *q, const void *k, const void *v, void *o, float *lse,
                          int B, int Hq, int Hkv, int Nq, int Nk, int D, int causal, float scale,
                          void *stream, fa_dtype_t in_dtype, fa_dtype_t out_dtype,
                          int heads_per_workgroup) {
    return run(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, in_dtype, out_dtype,
               0, heads_per_workgroup);
}

}  // extern "C"

namespace {

fa_status_t kvcache(const void *q, const void *k, const void *v, void *o, float *lse,
                    const int *seqlens_k, int B, int Hq, int Hkv, int Nq, int Nk, int D, int causal,
                    float scale, void *stream, fa_dtype_t in_dtype, fa_dtype_t out_dtype,
                    const CallWs *cws, const Window &win = Window()) {
    if (!seqlens_k) return FA_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(seqlens_k) & 3) return FA_ERR_ALIGN;
    if (B >= 1 && o && Hq >= 1 && Nq >= 1 && D >= 1) {
        const size_t ob = (size_t)B * Nq * Hq * D * esize(out_dtype);
        if (overlaps(o, ob, seqlens_k, (size_t)B * sizeof(int)) ||
            (lse && overlaps(lse, (size_t)B * Hq * Nq * sizeof(float), seqlens_k, (size_t)B * sizeof(int))))
            return FA_ERR_ALIAS;
    }
    return run(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, in_dtype, out_dtype, 0,
               0, seqlens_k, Paging(), cws, 0, win);
}

bool pages_ok(int B, int page_size, int max_pages, int num_pages) {
    return page_size >= 64 && page_size % 64 == 0 && max_pages >= 1 && num_pages >= 1 &&
           (long long)page_size * max_pages <= 0x7fffffffLL && (long long)B * max_pages <= 0x7fffffffLL;
}

fa_status_t append(const void *k, const void *v, void *k_cache, void *v_cache, const void *q, void *q_out,
                   const int *seqlens, int B, int Hq, int Hkv, int N, int Nk, int D, long long qs, long long ks,
                   long long vs, const fa_rotary_t *rotary, void *stream, fa_dtype_t dtype, const Paging &pg) {
    if (qs == 0) qs = (long long)Hq * D;
    if (ks == 0) ks = (long long)Hkv * D;
    if (vs == 0) vs = (long long)Hkv * D;
    const long long rows = pg.block_table ? (long long)pg.num_pages * pg.page_size : (long long)B * Nk;
    const fa_status_t st = fa::validate_append(k, v, k_cache, v_cache, q, q_out, seqlens, B, Hq, Hkv, N, D, qs, ks, vs,
                                               rotary, dtype, rows, pg.block_table, pg.max_pages);
    if (st != FA_OK) return st;
    const fa::AppendProblem p{k, v, k_cache, v_cache, q, q_out, seqlens, B, Hq, Hkv, N, Nk, D, qs, ks, vs, rotary,
                              dtype, pg.block_table, pg.page_size, pg.max_pages, pg.num_pages};
    return fa::launch_append(p, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? FA_OK : FA_ERR_HIP;
}

// Attention behind a shared prefix: the checks of both forms, then the launch.
// table NULL: k, v [B][Nk][Hkv][D] are the suffixes, else the pools, and Nk what a suffix can hold.
fa_status_t prefix(const void *q, const void *k_prefix, const void *v_prefix, const void *k, const void *v, void *o,
                   float *lse, const int *seqlens, int B, int Hq, int Hkv, int Nq, int Np, int Nk, int D, int causal,
                   float scale, void *stream, fa_dtype_t in, fa_dtype_t out, const Paging &pg, void *workspace,
                   size_t workspace_bytes) {
    if (!k_prefix || !v_prefix) return FA_ERR_NULL;
    const bool paged = pg.block_table != nullptr;
    const long long kv_rows = paged ? (long long)pg.num_pages * pg.page_size : (long long)B * Nk;
    if (Np < 1 || Nk < (paged ? 0 : 1) || (long long)Np + Nk > FA_MAX_PREFIX_KEYS) return FA_ERR_DIM;
    const long long tokens = (long long)B * Nq;
    if (B > 0 && Nq > 0 && Hq > 0 && (tokens > 0x7fffffffLL || tokens * Hq > 0x7fffffffLL)) return FA_ERR_DIM;
    fa_status_t st = validate_core(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk > 0 ? Nk : 1, D, 0, scale, in, out, kv_rows);
    if (st != FA_OK) return st;
    if (in == FA_F32) return FA_ERR_DTYPE;
    if (D != 64 && D != 128) return FA_ERR_HEAD_DIM;
    if (causal && Nq > Np + Nk) return FA_ERR_CAUSAL_SHAPE;
    long long t;
    if (!fa::mul_ok((long long)Np * Hkv, D, &t) || !fa::prefill_supported(Hkv, D, in)) return FA_ERR_DIM;
    if (fa::misaligned(k_prefix, 16) || fa::misaligned(v_prefix, 16) || fa::misaligned(seqlens, 4) ||
        fa::misaligned(pg.block_table, 4))
        return FA_ERR_ALIGN;
    const size_t qb = (size_t)B * Nq * Hq * D * esize(in), kb = (size_t)kv_rows * Hkv * D * esize(in);
    const size_t ob = (size_t)B * Nq * Hq * D * esize(out), lb = (size_t)B * Hq * Nq * sizeof(float);
    const size_t pb = paged ? kb : (size_t)Np * Hkv * D * esize(in);
    const fa::Range read[] = {{q, qb}, {k, kb}, {v, kb}, {k_prefix, pb}, {v_prefix, pb},
                              {seqlens, seqlens ? (size_t)B * sizeof(int) : 0},
                              {pg.block_table, paged ? (size_t)B * pg.max_pages * sizeof(int) : 0}};
    for (const fa::Range &r : read)
        if (r.bytes && (overlaps(o, ob, r.p, r.bytes) || (lse && overlaps(lse, lb, r.p, r.bytes)))) return FA_ERR_ALIAS;
    const size_t need = fa::prefix_workspace_bytes(B, Hq, Hkv, Nq, Np, Nk, D, false);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    bool user = workspace || workspace_bytes;
    std::unique_lock<std::mutex> lock(g_ws_mu, std::defer_lock);
    if (need == 0) {   // one pass: no workspace
        user = false;
    } else if (user) {
        if (!workspace) return FA_ERR_NULL;
        if (fa::misaligned(workspace, 16)) return FA_ERR_ALIGN;
        if (workspace_bytes < need) return FA_ERR_WORKSPACE;
    } else {
        lock.lock();
        st = get_workspace(need, fa::prefix_workspace_bytes(B, Hq, Hkv, Nq, Np, Nk, D, true), s, &workspace, &user);
        if (st != FA_OK) return st;
    }
    if (user) {
        for (const fa::Range &r : read)
            if (r.bytes && overlaps(workspace, need, r.p, r.bytes)) return FA_ERR_ALIAS;
        if (overlaps(workspace, need, o, ob) || (lse && overlaps(workspace, need, lse, lb))) return FA_ERR_ALIAS;
    }
    fa::PrefixProblem pp{fa::Problem{q, k, v, o, lse, B, Hq, Hkv, Nq, paged ? pg.page_size * pg.max_pages : Nk, D, causal,
                                     scale, in, out, 0, 0, seqlens, pg.block_table, pg.page_size, pg.max_pages,
                                     pg.num_pages},
                         k_prefix, v_prefix, Np, Nk};
    return fa::launch_prefix(pp, workspace, s) == hipSuccess ? FA_OK : FA_ERR_HIP;
}

fa_status_t kvcache_paged(const void *q, const void *k_pages, const void *v_pages, void *o,
                          float *lse, const int *seqlens_k, const int *block_table, int B, int Hq,
                          int Hkv, int Nq, int D, int page_size, int max_pages, int num_pages,
                          int causal, float scale, void *stream, fa_dtype_t in_dtype,
                          fa_dtype_t out_dtype, const CallWs *cws, const Window &win = Window()) {
    if (!seqlens_k || !block_table) return FA_ERR_NULL;
    if (!pages_ok(B, page_size, max_pages, num_pages)) return FA_ERR_DIM;
    if ((reinterpret_cast<uintptr_t>(seqlens_k) & 3) || (reinterpret_cast<uintptr_t>(block_table) & 3))
        return FA_ERR_ALIGN;
    const int Nk = page_size * max_pages;
    // fp16 / bf16 with D of 64 or 128 only
    if (in_dtype != FA_F16 && in_dtype != FA_BF16) {
        const fa_status_t st = validate_core(q, k_pages, v_pages, o, lse, B, Hq, Hkv, Nq, Nk, D, causal,
                                             scale, in_dtype, out_dtype, (long long)num_pages * page_size);
        return st != FA_OK ? st : FA_ERR_DTYPE;
    }
    if (D != 64 && D != 128) {
        const fa_status_t st = validate_core(q, k_pages, v_pages, o, lse, B, Hq, Hkv, Nq, Nk, D, causal,
                                             scale, in_dtype, out_dtype, (long long)num_pages * page_size);
        return st != FA_OK ? st : FA_ERR_HEAD_DIM;
    }
    if (B >= 1 && o && Hq >= 1 && Nq >= 1) {
        const size_t ob = (size_t)B * Nq * Hq * D * esize(out_dtype);
        const size_t lb = (size_t)B * Hq * Nq * sizeof(float);
        const size_t sb = (size_t)B * sizeof(int), tb = (size_t)B * max_pages * sizeof(int);
        if (overlaps(o, ob, seqlens_k, sb) || overlaps(o, ob, block_table, tb) ||
            (lse && (overlaps(lse, lb, seqlens_k, sb) || overlaps(lse, lb, block_table, tb))))
            return FA_ERR_ALIAS;
    }
    Paging pg;
    pg.block_table = block_table;
    pg.page_size = page_size;
    pg.max_pages = max_pages;
    pg.num_pages = num_pages;
    return run(q, k_pages, v_pages, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, in_dtype,
               out_dtype, 0, 0, seqlens_k, pg, cws, 0, win);
}

}  // namespace

extern "C" {

fa_status_t fa_fwd_slots(const void *q, const void *k, const void *v, void *o, float *lse, int B,
                         int Hq, int Hkv, int Nq, int Nk, int D, int causal, float scale, void *stream,
                         fa_dtype_t in_dtype, fa_dtype_t out_dtype, int slots_per_workgroup,
                         int heads_per_workgroup) {
    return run(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, in_dtype, out_dtype, 0,
               heads_per_workgroup, nullptr, Paging(), nullptr, slots_per_workgroup);
}

fa_status_t fa_fwd_kvcache(const void *q, const void *k, const void *v, void *o, float *lse,
                           const int *seqlens_k, int B, int Hq, int Hkv, int Nq, int Nk, int D,
                           int causal, float scale, void *stream, fa_dtype_t in_dtype,
                           fa_dtype_t out_dtype) {
    return kvcache(q, k, v, o, lse, seqlens_k, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, in_dtype,
                   out_dtype, nullptr);
}

fa_status_t fa_fwd_kvcache_paged(const void *q, const void *k_pages, const void *v_pages, void *o,
                                 float *lse, const int *seqlens_k, const int *block_table, int B,
                                 int Hq, int Hkv, int Nq, int D, int page_size, int max_pages,
                                 int num_pages, int causal, float scale, void *stream,
                                 fa_dtype_t in_dtype, fa_dtype_t out_dtype) {
    return kvcache_paged(q, k_pages, v_pages, o, lse, seqlens_k, block_table, B, Hq, Hkv, Nq, D,
                         page_size, max_pages, num_pages, causal, scale, stream, in_dtype, out_dtype,
                         nullptr);
}

fa_status_t fa_fwd_ws(const void *q, const void *k, const void *v, void *o, float *lse, int B,
                      int Hq, int Hkv, int Nq, int Nk, int D, int causal, float scale, void *stream,
                      fa_dtype_t in_dtype, fa_dtype_t out_dtype, int num_splits, void *workspace,
                      size_t workspace_bytes) {
    const CallWs cws{workspace, workspace_bytes};
    return run(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, in_dtype, out_dtype,
               num_splits, 0, nullptr, Paging(), &cws);
}

fa_status_t fa_fwd_splitkv_noalloc(const void *q, const void *k, const void *v, void *o, float *lse,
                                   int B, int Hq, int Hkv, int Nq, int Nk, int D, int causal,
                                   float scale, void *stream, fa_dtype_t in_dtype,
                                   fa_dtype_t out_dtype, int num_splits) {
    // the argument checks of fa_fwd_splitkv, then the size of the partial
    // results against the scratch, all before any HIP call
    fa_status_t st = validate_core(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, in_dtype,
                                   out_dtype, -1);
    if (st != FA_OK) return st;
    if (num_splits < 0 || num_splits > FA_MAX_SPLITS) return FA_ERR_SPLITS;
    CallWs cws{nullptr, 0};
    std::unique_lock<std::mutex> lock(g_scratch_mu, std::defer_lock);
    if (fa::decode_supported(Nq, Hkv, D, in_dtype)) {
        const int S = num_splits > 0 ? num_splits : fa::decode_default_splits(B, Hq, Hkv, Nk, D);
        if (fa::decode_workspace_bytes(B, Hq, D, S) > kScratchBytes) return FA_ERR_WORKSPACE;
        lock.lock();
        st = scratch_address(&cws.ptr);
        if (st != FA_OK) return st;
        cws.bytes = kScratchBytes;
    }
    return run(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, in_dtype, out_dtype,
               num_splits, 0, nullptr, Paging(), &cws);
}

fa_status_t fa_fwd_kvcache_ws(const void *q, const void *k, const void *v, void *o, float *lse,
                              const int *seqlens_k, int B, int Hq, int Hkv, int Nq, int Nk, int D,
                              int causal, float scale, void *stream, fa_dtype_t in_dtype,
                              fa_dtype_t out_dtype, void *workspace, size_t workspace_bytes) {
    const CallWs cws{workspace, workspace_bytes};
    return kvcache(q, k, v, o, lse, seqlens_k, B, Hq, Hkv, Nq, Nk, D, causal, scale, stream, in_dtype,
                   out_dtype, &cws);
}

fa_status_t fa_fwd_kvcache_paged_ws(const void *q, const void *k_pages, const void *v_pages, void *o,
                                    float *lse, const int *seqlens_k, const int *block_table, int B,
                                    int Hq, int Hkv, int Nq, int D, int page_size, int max_pages,
                                    int num_pages, int causal, float scale, void *stream,
                                    fa_dtype_t in_dtype, fa_dtype_t out_dtype, void *workspace,
                                    size_t workspace_bytes) {
    const CallWs cws{workspace, workspace_bytes};
    return kvcache_paged(q, k_pages, v_pages, o, lse, seqlens_k, block_table, B, Hq, Hkv, Nq, D,
                         page_size, max_pages, num_pages, causal, scale, stream, in_dtype, out_dtype,
                         &cws);
}

size_t fa_workspace_bytes(int B, int Hq, int Hkv, int Nq, int Nk, int D, fa_dtype_t in_dtype,
                          int num_splits) {
    if (B < 1 || Hq < 1 || Hkv < 1 || Nk < 1 || Hq % Hkv != 0) return 0;
    if (!fa::decode_supported(Nq, Hkv, D, in_dtype)) return 0;
    if (num_splits < 0 || num_splits > FA_MAX_SPLITS) return 0;
    // enough for every shorter cache as well: a program sizes its workspace once
    const int S = num_splits > 0 ? num_splits : fa::decode_most_splits(B, Hq, Hkv, Nk, D);
    return fa::decode_workspace_bytes(B, Hq, D, S);
}

fa_status_t fa_set_workspace(void *dev_ptr, size_t bytes) {
    if ((dev_ptr == nullptr) != (bytes == 0)) return FA_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(dev_ptr) & 15) return FA_ERR_ALIGN;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return FA_ERR_HIP;
    std::lock_guard<std::mutex> lk(g_ws_mu);
    g_user[dev].ptr = dev_ptr;
    g_user[dev].bytes = bytes;
    return FA_OK;
}

fa_status_t fa_q8_0_gemv(const void *w, const void *x, void *y, int M, int K, fa_dtype_t x_dtype,
                         fa_dtype_t y_dtype, void *stream) {
    if (!w || !x || !y) return FA_ERR_NULL;
    if (M < 1 || K < 32 || K % 32 != 0 || K > (1 << 30)) return FA_ERR_DIM;
    const bool xt_ok = x_dtype == FA_F16 || x_dtype == FA_BF16 || x_dtype == FA_F32;
    if (!xt_ok || !(y_dtype == x_dtype || y_dtype == FA_F32)) return FA_ERR_DTYPE;
    const size_t xe = esize(x_dtype), ye = esize(y_dtype);
    if ((reinterpret_cast<uintptr_t>(w) & 3) || (reinterpret_cast<uintptr_t>(x) & 15) ||
        (reinterpret_cast<uintptr_t>(y) & (ye - 1)))
        return FA_ERR_ALIGN;
    const size_t wb = (size_t)M * (size_t)(K / 32) * 34;
    if (overlaps(y, (size_t)M * ye, w, wb) || overlaps(y, (size_t)M * ye, x, (size_t)K * xe))
        return FA_ERR_ALIAS;
    const hipError_t e =
        fa::launch_q8_gemv(w, x, y, M, K, x_dtype, y_dtype, reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? FA_OK : FA_ERR_HIP;
}

fa_status_t fa_fwd_window(const void *q, const void *k, const void *v, void *o, float *lse, const int *seqlens_k,
                          int B, int Hq, int Hkv, int Nq, int Nk, int D, int window, int sinks, float scale,
                          void *stream, fa_dtype_t in_dtype, fa_dtype_t out_dtype, void *workspace,
                          size_t workspace_bytes) {
    if (window < 1 || sinks < 0) return FA_ERR_WINDOW;
    const CallWs cws{workspace, workspace_bytes}, *own = workspace || workspace_bytes ? &cws : nullptr;
    const Window win{window, sinks};
    if (seqlens_k)
        return kvcache(q, k, v, o, lse, seqlens_k, B, Hq, Hkv, Nq, Nk, D, 1, scale, stream, in_dtype, out_dtype, own,
                       win);
    return run(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, 1, scale, stream, in_dtype, out_dtype, 0, 0, nullptr, Paging(),
               own, 0, win);
}

fa_status_t fa_fwd_window_paged(const void *q, const void *k_pages, const void *v_pages, void *o, float *lse,
                                const int *seqlens_k, const int *block_table, int B, int Hq, int Hkv, int Nq, int D,
                                int page_size, int max_pages, int num_pages, int window, int sinks, float scale,
                                void *stream, fa_dtype_t in_dtype, fa_dtype_t out_dtype, void *workspace,
                                size_t workspace_bytes) {
    if (window < 1 || sinks < 0) return FA_ERR_WINDOW;
    const CallWs cws{workspace, workspace_bytes};
    return kvcache_paged(q, k_pages, v_pages, o, lse, seqlens_k, block_table, B, Hq, Hkv, Nq, D, page_size, max_pages,
                         num_pages, 1, scale, stream, in_dtype, out_dtype,
                         workspace || workspace_bytes ? &cws : nullptr, Window{window, sinks});
}

size_t fa_window_workspace_bytes(int B, int Hq, int Hkv, int Nq, int Nk, int D, int window, int sinks,
                                 fa_dtype_t in_dtype) {
    if (window < 1 || sinks < 0 || B < 1 || Hq < 1 || Hkv < 1 || Nq < 1 || Nk < 1 || Hq % Hkv != 0 ||
        (long long)B * Nq > 0x7fffffffLL)
        return 0;
    if (fa::decode_supported(Nq, Hkv, D, in_dtype))
        return fa::decode_workspace_bytes(B, Hq, D, decode_splits(B, Hq, Hkv, Nk, D, Window{window, sinks}, true));
    return fa::prefill_supported(Hkv, D, in_dtype)
               ? fa::window_workspace_bytes(B, Hq, Hkv, Nq, Nk, D, window, sinks, true) : 0;
}

fa_status_t fa_fwd_prefix(const void *q, const void *k_prefix, const void *v_prefix, const void *k, const void *v,
                          void *o, float *lse, const int *seqlens_k, int B, int Hq, int Hkv, int Nq, int Np, int Nk,
                          int D, int causal, float scale, void *stream, fa_dtype_t in_dtype, fa_dtype_t out_dtype,
                          void *workspace, size_t workspace_bytes) {
    return prefix(q, k_prefix, v_prefix, k, v, o, lse, seqlens_k, B, Hq, Hkv, Nq, Np, Nk, D, causal, scale, stream,
                  in_dtype, out_dtype, Paging(), workspace, workspace_bytes);
}

fa_status_t fa_fwd_prefix_paged(const void *q, const void *k_pages, const void *v_pages, void *o, float *lse,
                                const int *seqlens_k, const int *block_table, int B, int Hq, int Hkv, int Nq, int D,
                                int page_size, int max_pages, int num_pages, int prefix_len, int causal, float scale,
                                void *stream, fa_dtype_t in_dtype, fa_dtype_t out_dtype, void *workspace,
                                size_t workspace_bytes) {
    if (!seqlens_k || !block_table) return FA_ERR_NULL;
    if (!pages_ok(B, page_size, max_pages, num_pages)) return FA_ERR_DIM;
    if (prefix_len < page_size || prefix_len % page_size != 0 || prefix_len > page_size * max_pages) return FA_ERR_DIM;
    Paging pg;
    pg.block_table = block_table;
    pg.page_size = page_size;
    pg.max_pages = max_pages;
    pg.num_pages = num_pages;
    return prefix(q, k_pages, v_pages, k_pages, v_pages, o, lse, seqlens_k, B, Hq, Hkv, Nq, prefix_len,
                  page_size * max_pages - prefix_len, D, causal, scale, stream, in_dtype, out_dtype, pg, workspace,
                  workspace_bytes);
}

size_t fa_prefix_workspace_bytes(int B, int Hq, int Hkv, int Nq, int Np, int Nk, int D, fa_dtype_t in_dtype) {
    if (B < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || Nq < 1 || Np < 1 || Nk < 0 || (D != 64 && D != 128) ||
        (long long)Np + Nk > FA_MAX_PREFIX_KEYS || (in_dtype != FA_F16 && in_dtype != FA_BF16) ||
        (long long)B * Nq > 0x7fffffffLL || (long long)B * Nq * Hq > 0x7fffffffLL)
        return 0;
    return fa::prefix_workspace_bytes(B, Hq, Hkv, Nq, Np, Nk, D, true);
}

fa_status_t fa_kvcache_append(const void *k, const void *v, void *k_cache, void *v_cache, const void *q,
                              void *q_out, const int *seqlens_k, int B, int Hq, int Hkv, int Nq, int Nk, int D,
                              long long q_stride, long long k_stride, long long v_stride,
                              const fa_rotary_t *rotary, void *stream, fa_dtype_t dtype) {
    return append(k, v, k_cache, v_cache, q, q_out, seqlens_k, B, Hq, Hkv, Nq, Nk, D, q_stride, k_stride, v_stride,
                  rotary, stream, dtype, Paging());
}

fa_status_t fa_kvcache_append_paged(const void *k, const void *v, void *k_pages, void *v_pages, const void *q,
                                    void *q_out, const int *seqlens_k, const int *block_table, int B, int Hq,
                                    int Hkv, int Nq, int D, int page_size, int max_pages, int num_pages,
                                    long long q_stride, long long k_stride, long long v_stride,
                                    const fa_rotary_t *rotary, void *stream, fa_dtype_t dtype) {
    if (!block_table) return FA_ERR_NULL;
    if (!pages_ok(B, page_size, max_pages, num_pages)) return FA_ERR_DIM;
    Paging pg;
    pg.block_table = block_table;
    pg.page_size = page_size;
    pg.max_pages = max_pages;
    pg.num_pages = num_pages;
    return append(k, v, k_pages, v_pages, q, q_out, seqlens_k, B, Hq, Hkv, Nq, page_size * max_pages, D, q_stride,
                  k_stride, v_stride, rotary, stream, dtype, pg);
}

size_t fa_unfused_workspace_bytes(int B, int Hq, int Nq, int Nk) {
    return fa::unfused_workspace_bytes(B, Hq, Nq, Nk);
}

fa_status_t fa_fwd_unfused(const void *q, const void *k, const void *v, void *o, float *lse, int B,
                           int Hq, int Hkv, int Nq, int Nk, int D, int causal, float scale,
                           void *stream, fa_dtype_t in_dtype, fa_dtype_t out_dtype,
                           void *workspace, size_t workspace_bytes) {
    fa_status_t st = validate_core(q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, in_dtype,
                                   out_dtype, -1);
    if (st != FA_OK) return st;
    if (in_dtype == FA_F32) return FA_ERR_DTYPE;
    if (!fa::unfused_supported(D, in_dtype)) return FA_ERR_HEAD_DIM;
    if (Nk > (1 << 23)) return FA_ERR_DIM;   // 32-bit offsets within a 32-row block of scores
    if ((long long)B * Hq * Nq > 0x7fffffffLL) return FA_ERR_DIM;   // one softmax workgroup per row at most
    if (!workspace) return FA_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return FA_ERR_ALIGN;
    const size_t need = fa::unfused_workspace_bytes(B, Hq, Nq, Nk);
    if (need == 0) return FA_ERR_DIM;
    if (workspace_bytes < need) return FA_ERR_WORKSPACE;
    const size_t qb = (size_t)B * Nq * Hq * D * esize(in_dtype), kb = (size_t)B * Nk * Hkv * D * esize(in_dtype);
    const size_t ob = (size_t)B * Nq * Hq * D * esize(out_dtype), lb = (size_t)B * Hq * Nq * sizeof(float);
    if (overlaps(workspace, need, q, qb) || overlaps(workspace, need, k, kb) ||
        overlaps(workspace, need, v, kb) || overlaps(workspace, need, o, ob) ||
        (lse && overlaps(workspace, need, lse, lb)))
        return FA_ERR_ALIAS;
    fa::Problem p{q, k, v, o, lse, B, Hq, Hkv, Nq, Nk, D, causal, scale, in_dtype, out_dtype, 0, 0,
                  nullptr, nullptr, 0, 0, 0};
    const hipError_t e = fa::launch_unfused(p, workspace, reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? FA_OK : FA_ERR_HIP;
}

fa_status_t fa_release_workspace(void) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return FA_ERR_HIP;
    std::lock_guard<std::mutex> lk(g_ws_mu);
    bool any = false;
    for (const OwnedWs &w : g_owned) any = any || w.dev == dev;
    for (const Retired &r : g_retired) any = any || r.dev == dev;
    if (!any) return FA_OK;
    // calls queued on any stream may still use these buffers
    if (hipDeviceSynchronize() != hipSuccess) return FA_ERR_HIP;
    fa_status_t st = FA_OK;
    std::vector<OwnedWs> keep;
    for (const OwnedWs &w : g_owned) {
        if (w.dev != dev) keep.push_back(w);
        else if (hipFree(w.ptr) != hipSuccess) st = FA_ERR_HIP;
    }
    g_owned.swap(keep);
    std::vector<Retired> keep_r;
    for (const Retired &r : g_retired) {
        if (r.dev != dev) keep_r.push_back(r);
        else if (hipFree(r.ptr) != hipSuccess) st = FA_ERR_HIP;
    }
    g_retired.swap(keep_r);
    return st;
}

}  // extern "C"
