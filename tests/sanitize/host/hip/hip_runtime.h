// What fa_api.hip needs of the HIP runtime, for a build of the host code alone
// (threads_driver.cpp defines the functions; nothing here reaches a GPU).
#pragma once

#include <cstddef>

typedef int hipError_t;
typedef void *hipStream_t;
typedef int hipStreamCaptureStatus;
constexpr hipError_t hipSuccess = 0;
constexpr hipStreamCaptureStatus hipStreamCaptureStatusNone = 0;
#define __device__
#define __align__(n) __attribute__((aligned(n)))
#define HIP_SYMBOL(x) x

hipError_t hipGetDevice(int *dev);
hipError_t hipGetLastError();
hipError_t hipStreamIsCapturing(hipStream_t s, hipStreamCaptureStatus *status);
hipError_t hipMalloc(void **p, size_t bytes);
hipError_t hipFree(void *p);
hipError_t hipDeviceSynchronize();
hipError_t hipGetSymbolAddress(void **p, const void *symbol);
