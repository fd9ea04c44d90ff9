// Several host threads call the library on one stream.  The launchers here stand for
// the two that a call enqueues, the kernel that leaves partial results in the
// workspace and the one that merges them: between the two no other call may use
// that workspace, nor may it be freed.  Host code only (fa_api.hip with the stand-in
// for the HIP runtime in host/).
#include <atomic>
#include <chrono>
#include <cstdio>
#include <map>
#include <mutex>
#include <set>
#include <thread>
#include <vector>

#include "../../paper_2608_18656_amd/csrc/fa_api.hip"

static std::mutex mu;
static std::map<const void *, const void *> partial;   // workspace -> output of the call whose partial results it holds
static std::set<const void *> alive;                   // allocated buffers
static const void *const fixed_buffers[2] = {reinterpret_cast<const void *>(uintptr_t{1} << 50), scratch};
static int bad = 0, calls = 0, refused = 0;
static std::atomic<uintptr_t> next{uintptr_t{1} << 40};

hipError_t hipGetDevice(int *dev) { return *dev = 0, hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) { return *s = hipStreamCaptureStatusNone, hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipMalloc(void **p, size_t bytes) {
    *p = reinterpret_cast<void *>(next.fetch_add((bytes + 4095) & ~(size_t)4095));
    std::lock_guard<std::mutex> lk(mu);
    alive.insert(*p);
    return hipSuccess;
}
hipError_t hipFree(void *p) {
    std::lock_guard<std::mutex> lk(mu);
    alive.erase(p);
    return hipSuccess;
}
hipError_t hipGetSymbolAddress(void **p, const void *symbol) { return *p = const_cast<void *>(symbol), hipSuccess; }

static hipError_t two_kernels(const void *out, const void *ws) {
    auto usable = [&] { return alive.count(ws) || ws == fixed_buffers[0] || ws == fixed_buffers[1]; };
    {
        std::lock_guard<std::mutex> lk(mu);
        ++calls;
        bad += !usable();
        partial[ws] = out;
    }
    std::this_thread::sleep_for(std::chrono::microseconds(300));
    std::lock_guard<std::mutex> lk(mu);
    bad += !usable() || partial[ws] != out;
    return hipSuccess;
}

namespace fa {
hipError_t launch_prefill(const Problem &, hipStream_t) { return hipSuccess; }
hipError_t launch_prefill_window(const Problem &p, void *ws, hipStream_t) { return two_kernels(p.o, ws); }
hipError_t launch_generic(const Problem &, hipStream_t) { return hipSuccess; }
hipError_t launch_generic_window(const Problem &, hipStream_t) { return hipSuccess; }
hipError_t launch_decode(const Problem &p, int, void *ws, hipStream_t) { return two_kernels(p.o, ws); }
hipError_t launch_unfused(const Problem &, void *, hipStream_t) { return hipSuccess; }
hipError_t launch_prefix(const PrefixProblem &p, void *ws, hipStream_t) { return two_kernels(p.p.o, ws); }
hipError_t launch_append(const AppendProblem &, hipStream_t) { return hipSuccess; }
hipError_t launch_q8_gemv(const void *, const void *, void *, int, int, fa_dtype_t, fa_dtype_t, hipStream_t) { return hipSuccess; }
bool decode_supported(int Nq, int, int, fa_dtype_t) { return Nq == 1; }
bool prefill_supported(int, int, fa_dtype_t) { return true; }
int decode_default_splits(int, int, int, int Nk, int) { return 2 + Nk % 7; }
int decode_most_splits(int, int, int, int, int) { return 9; }
size_t decode_workspace_bytes(int, int, int, int splits) { return (size_t)splits << 20; }
size_t prefix_workspace_bytes(int, int, int, int, int Np, int, int, bool) { return (size_t)(1 + Np % 5) << 20; }
size_t window_workspace_bytes(int, int, int, int, int Nk, int, int, int, bool) { return (size_t)(1 + Nk % 11) << 20; }
bool unfused_supported(int, fa_dtype_t) { return true; }
size_t unfused_workspace_bytes(long long, long long, long long, long long) { return 1; }
}  // namespace fa

static void caller(int id, int rounds, bool release) {
    auto at = [&](int i) { return reinterpret_cast<void *>((uintptr_t)(i + 1 + 16 * id) << 30); };
    const int *lens = static_cast<const int *>(at(6));
    for (int r = 0; r < rounds; ++r) {
        const int Nk = 500 + 13 * r + id;
        float *lse = static_cast<float *>(at(5));
        fa_status_t st[5] = {
            fa_fwd_kvcache(at(0), at(1), at(2), at(4), lse, lens, 2, 4, 2, 1, Nk, 64, 0, 0.125f, nullptr, FA_F16, FA_F16),
            fa_fwd_window(at(0), at(1), at(2), at(4), lse, lens, 2, 4, 2, 1, Nk, 64, 100, 4, 0.125f, nullptr, FA_F16, FA_F16, nullptr, 0),
            fa_fwd_window(at(0), at(1), at(2), at(4), lse, lens, 2, 4, 2, 9, Nk, 64, 100, 4, 0.125f, nullptr, FA_F16, FA_F16, nullptr, 0),
            fa_fwd_prefix(at(0), at(7), at(8), at(1), at(2), at(4), lse, lens, 2, 4, 2, 1, 99 + r, Nk, 64, 1, 0.125f, nullptr, FA_F16,
                          FA_F16, nullptr, 0),
            fa_fwd_splitkv_noalloc(at(0), at(1), at(2), at(4), lse, 2, 4, 2, 1, Nk, 64, 0, 0.125f, nullptr, FA_F16, FA_F16, 3)};
        if (release && r % 3 == 0 && fa_release_workspace() != FA_OK) st[0] = FA_ERR_HIP;
        std::lock_guard<std::mutex> lk(mu);
        for (fa_status_t s : st) refused += s != FA_OK;
    }
}

static void together(bool release) {
    std::vector<std::thread> threads;
    for (int id = 0; id < 4; ++id) threads.emplace_back(caller, id, 12, release && id == 0);
    for (std::thread &t : threads) t.join();
}

int main() {
    together(false);
    together(true);
    if (fa_set_workspace(const_cast<void *>(fixed_buffers[0]), (size_t)64 << 20) != FA_OK) return 2;
    together(false);
    std::printf("%d calls, %d refused, %d met another's workspace\n", calls, refused, bad);
    return bad || refused ? 1 : 0;
}
