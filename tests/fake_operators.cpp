// The HIP calls of the operators' host code and their kernels' launch wrappers, on host memory: what a call would have launched is written down.
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <string>

#include "../paper_2211_13939_amd/csrc/operator_kernels.h"
#include "../paper_2211_13939_amd/csrc/hostutil.h"

namespace {
std::string text;
int current = 0, launches = 0, last_rows = 0, last_n = 0, devices_seen = 0, requests_seen = 0, many_launches = 0;
std::string failing;
hipError_t call(const char* name) { return failing == name ? hipErrorUnknown : hipSuccess; }
}  // namespace

namespace tts {
int fail(int code, const char* fmt, ...)
{
    char b[512];
    va_list a;
    va_start(a, fmt);
    vsnprintf(b, sizeof(b), fmt, a);
    va_end(a);
    text = b;
    return code;
}
hipError_t launch_norm(const NormArgs& a, bool, bool, int, hipStream_t)
{
    ++launches;
    last_rows = a.rows;
    devices_seen = current;
    return call("launch");
}
hipError_t allow_linear8() { return call("allow"); }
hipError_t launch_linear8(const Linear8Args& a, bool, int, hipStream_t)
{
    ++launches;
    last_rows = a.rows;
    return call("launch");
}
size_t cross_parts_bytes() { return 4096; }
hipError_t allow_cross() { return call("allow"); }
static hipError_t launched(const CrossArgs& a)
{
    ++launches;
    last_n = a.n;
    last_rows = a.req[a.n - 1].q_row + a.req[a.n - 1].q_len;
    for (int i = 0; i < a.n; ++i) requests_seen += 1;
    return call("launch");
}
hipError_t launch_cross_few(CrossArgs& a, bool, int, hipStream_t) { return launched(a); }
hipError_t launch_cross_many(CrossArgs& a, int, hipStream_t)
{
    ++many_launches;
    return launched(a);
}
}  // namespace tts

extern "C" {
const char* tts_last_error() { return text.c_str(); }
void fake_reset() { text.clear(); failing.clear(); launches = last_rows = last_n = current = requests_seen = many_launches = 0; }
void fake_fail(const char* name) { failing = name; }
void fake_device(int d) { current = d; }
int fake_launches() { return launches; }
int fake_rows() { return last_rows; }
int fake_requests() { return last_n; }
int fake_requests_seen() { return requests_seen; }
int fake_many() { return many_launches; }
int fake_current() { return current; }
int fake_seen() { return devices_seen; }
hipError_t hipGetDevice(int* d) { *d = current; return call("hipGetDevice"); }
hipError_t hipSetDevice(int d) { current = d; return call("hipSetDevice"); }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "a failure"; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return call("hipDeviceGetAttribute"); }
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) { if (failing != "hipMemcpy") memcpy(d, s, n); return call("hipMemcpy"); }
hipError_t hipMemset(void* d, int v, size_t n) { memset(d, v, n); return hipSuccess; }
hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, hipMemcpyKind, hipStream_t) { memcpy(d, s, n); return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipPointerGetAttributes(hipPointerAttribute_t* a, const void*) { a->type = hipMemoryTypeDevice; a->device = 0; return call("hipPointerGetAttributes"); }
}
