// A HIP runtime without a GPU for tests of host code: every call succeeds, kernels are not run, and the calls that order work are written down.
// Streams are any addresses; two devices.  Loaded before the library under test, whose calls then come here.
#include <cstddef>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <string>

namespace {
std::string trace;
int device = 0;
uint64_t capturing = 0;                                       // bit i: stream i is being captured
char memory[64];
template <typename... A> void note(const char* format, A... a)
{
    char line[96];
    snprintf(line, sizeof line, format, a...);
    trace += line;
}
unsigned number(const void* p) { return (unsigned)(uintptr_t)p; }
struct Dim { unsigned x, y, z; };
struct Config { Dim grid, block; size_t shared; void* stream; } pushed;
}  // namespace

extern "C" {
const char* trace_text() { return trace.c_str(); }
void trace_clear() { trace.clear(); }
void trace_capture(unsigned stream, int on) { capturing = on ? capturing | uint64_t(1) << stream : capturing & ~(uint64_t(1) << stream); }

int hipGetDeviceCount(int* n) { *n = 2; return 0; }
int hipGetDevice(int* d) { *d = device; return 0; }
int hipSetDevice(int d) { device = d; return 0; }
int hipDeviceGetAttribute(int* v, int, int) { *v = 256; return 0; }
int hipDeviceSynchronize() { note("synchronize\n"); return 0; }
int hipFuncSetAttribute(const void*, int, int) { return 0; }
int hipMalloc(void** p, size_t) { *p = reinterpret_cast<void*>(uintptr_t(1) << 40); return 0; }
int hipFree(void*) { return 0; }
int hipGetLastError() { return 0; }
const char* hipGetErrorString(int) { return "an error"; }
int hipEventCreateWithFlags(void** e, unsigned) { *e = memory; return 0; }
int hipEventDestroy(void*) { return 0; }
int hipEventRecord(void*, void* s) { note("record %u\n", number(s)); return 0; }
int hipStreamWaitEvent(void* s, void*, unsigned) { note("wait %u\n", number(s)); return 0; }
int hipStreamSynchronize(void*) { return 0; }
int hipStreamIsCapturing(void* s, int* status) { *status = (int)(capturing >> number(s) & 1); return 0; }
int __hipPushCallConfiguration(Dim grid, Dim block, size_t shared, void* stream) { pushed = {grid, block, shared, stream}; return 0; }
int __hipPopCallConfiguration(Dim* grid, Dim* block, size_t* shared, void** stream)
{
    *grid = pushed.grid;
    *block = pushed.block;
    *shared = pushed.shared;
    *stream = pushed.stream;
    return 0;
}
int hipLaunchKernel(const void*, Dim, Dim, void**, size_t, void* s) { note("launch %u on %d\n", number(s), device); return 0; }
}
