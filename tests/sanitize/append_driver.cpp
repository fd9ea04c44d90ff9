// Exercises the argument checks of the cache append (validate_append) over a grid
// of sizes, strides, rotations and pointer patterns, including extreme and
// overflowing values; built with AddressSanitizer and UndefinedBehaviorSanitizer
// by the CPU test suite, which fails on any report.  Pointers are fake addresses,
// never dereferenced, but for the rotation description, which the checks read.
#include <climits>
#include <cstdint>
#include <cstdio>
#include <initializer_list>

#include "../../paper_2608_18656_amd/csrc/fa_checks.h"

static const void *P(uintptr_t x) { return reinterpret_cast<const void *>(x); }

int main() {
    const int sizes[] = {INT_MIN, -1, 0, 1, 2, 3, 8, 64, 255, 1 << 20, INT_MAX};
    const long long strides[] = {LLONG_MIN, -8, 0, 1, 64, 4096, 1LL << 40, LLONG_MAX};
    const uintptr_t bases[] = {0, 1u << 20, (uintptr_t)1 << 44, UINTPTR_MAX - 4095};
    const fa_dtype_t dts[] = {FA_F16, FA_BF16, FA_F32, (fa_dtype_t)7};
    long long n = 0, ok = 0;
    for (int B : sizes)
        for (int Hq : sizes)
            for (int Hkv : sizes)
                for (int N : sizes)
                    for (int D : {INT_MIN, 0, 8, 40, 64, 256, 264, INT_MAX})
                        for (long long s : strides) {
                            const unsigned mix = (unsigned)B * 7u + (unsigned)Hq * 5u + (unsigned)N * 3u + (unsigned)D;
                            const uintptr_t base = bases[mix % 4], step = (uintptr_t)1 << 40;
                            fa_rotary_t r = {};
                            r.inv_freq = reinterpret_cast<const float *>(base + 7 * step);
                            r.positions = mix % 3 ? reinterpret_cast<const int *>(base + 8 * step) : nullptr;
                            r.rot_dim = mix % 5 == 0 ? D : sizes[mix % 11];
                            r.axes = (int)(mix % 7) - 1;
                            for (int j = 0; j < FA_MAX_ROTARY_PAIRS; ++j) r.pair_axis[j] = (unsigned char)(j % (mix % 6 + 1));
                            const bool with_q = mix & 1;
                            const fa_status_t st = fa::validate_append(
                                P(base), P(base + step), P(base + 2 * step), P(base + 3 * step), with_q ? P(base + 4 * step) : nullptr,
                                with_q ? P(base + (mix % 9 ? 5 : 4) * step) : nullptr, reinterpret_cast<const int *>(base + 6 * step), B, Hq,
                                Hkv, N, D, s, strides[mix % 8], strides[(mix / 8) % 8], mix % 4 ? &r : nullptr, dts[mix % 4],
                                mix % 3 ? (long long)B * N : LLONG_MAX / 4, mix % 2 ? reinterpret_cast<const int *>(base + 9 * step) : nullptr, 3);
                            ++n;
                            ok += st == FA_OK;
                        }
    // known answers: dense and strided, in place, and a rotation of every column
    int bad = 0;
    auto at = [](int i) { return P((uintptr_t)(i + 1) << 30); };
    auto lens = reinterpret_cast<const int *>((uintptr_t)40 << 30);
    fa_rotary_t r = {};
    r.inv_freq = reinterpret_cast<const float *>((uintptr_t)41 << 30);
    r.rot_dim = 64;
    r.axes = 1;
    bad |= fa::validate_append(at(0), at(1), at(2), at(3), at(4), at(5), lens, 2, 4, 2, 3, 64, 256, 128, 128, &r, FA_F16, 100, nullptr, 0) != FA_OK;
    bad |= fa::validate_append(at(0), at(1), at(2), at(3), at(4), at(4), lens, 2, 4, 2, 3, 64, 256, 512, 512, &r, FA_F16, 100, nullptr, 0) != FA_OK;
    bad |= fa::validate_append(at(0), at(1), at(2), at(3), at(4), at(4), lens, 2, 4, 2, 3, 64, 512, 128, 128, &r, FA_F16, 100, nullptr, 0) != FA_ERR_ALIAS;
    bad |= fa::validate_append(at(0), at(1), at(2), at(3), at(4), at(5), lens, 2, 4, 2, 3, 64, 256, 128, 127, &r, FA_F16, 100, nullptr, 0) != FA_ERR_DIM;
    std::printf("checked %lld argument sets, %lld accepted\n", n, ok);
    return bad;
}
