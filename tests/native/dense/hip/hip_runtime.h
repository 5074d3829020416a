// Just enough of the runtime's interface to compile csrc/dense.hip for the CPU: "device" memory is host memory, copies
// happen at once, and a switch says whether the stream is recording.
#pragma once

#include <cstddef>
#include <cstdint>
#include <cstdlib>
#include <cstring>

#define __host__
#define __device__

enum hipError_t { hipSuccess = 0, hipErrorInvalidValue = 1, hipErrorOutOfMemory = 2 };
enum hipMemcpyKind { hipMemcpyHostToDevice = 1, hipMemcpyDeviceToHost = 2 };
enum hipStreamCaptureStatus { hipStreamCaptureStatusNone = 0, hipStreamCaptureStatusActive = 1 };
using hipStream_t = void*;

inline bool stub_recording = false, stub_no_memory = false;
inline int stub_device = 0, stub_allocations = 0;

inline const char* hipGetErrorString(hipError_t) { return "stub"; }
inline hipError_t hipGetLastError() { return hipSuccess; }
inline hipError_t hipGetDevice(int* d) { *d = stub_device; return hipSuccess; }
inline hipError_t hipSetDevice(int d) { stub_device = d; return hipSuccess; }
inline hipError_t hipMalloc(void** p, size_t bytes) {
    if (stub_no_memory) return hipErrorOutOfMemory;
    *p = std::malloc(bytes);
    ++stub_allocations;
    return hipSuccess;
}
inline hipError_t hipFree(void* p) { std::free(p); --stub_allocations; return hipSuccess; }
inline hipError_t hipMemcpyAsync(void* to, const void* from, size_t n, hipMemcpyKind, hipStream_t) { std::memcpy(to, from, n); return hipSuccess; }
inline hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
inline hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
    *s = stub_recording ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
    return hipSuccess;
}
