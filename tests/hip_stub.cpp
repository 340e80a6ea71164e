// Stand-ins for the HIP calls that the cache's host code makes, so that it runs
// without a GPU: two devices, memory that is only counted, launches that are
// only written down.  Loaded with global symbols before the library.
#include <cstddef>
#include <cstdint>
#include <cstdlib>

extern "C" {

struct Dim { uint32_t x, y, z; };
struct Call {                       // one per call, in order
    int what;                       // kMalloc ..
    int device;                     // current at the call
    void* stream;
    uint64_t bytes;
    uint32_t grid, block;
};
enum { kMalloc = 1, kFree, kMemset, kMemcpy, kMemcpyAsync, kSync, kLaunch, kDeviceSync };

Call stub_calls[4096];
int stub_n = 0, stub_device = 0, stub_failed_set = 0;
// the word that kernels record errors in, and what a kernel on another stream
// adds to it as soon as it has been copied
int stub_word = 0, stub_late = 0;
static uintptr_t base = 0x10000000, top = 0x10000000;

static void note(int what, void* stream, uint64_t bytes, uint32_t grid = 0, uint32_t block = 0) {
    if (stub_n < 4096) stub_calls[stub_n++] = {what, stub_device, stream, bytes, grid, block};
}
static uintptr_t taken_at = 0;
static int taken = 0;
static void copied(void* dst, const void* src) {
    *(int*)dst = taken_at && (uintptr_t)src == taken_at ? taken : stub_word;
    stub_word |= stub_late;
    stub_late = 0;
}

int hipGetDevice(int* d) { *d = stub_device; return 0; }
int hipSetDevice(int d) { if (d < 0 || d > 1) return 101; stub_device = d; return 0; }
int hipMalloc(void** p, size_t n) {
    note(kMalloc, nullptr, n);
    base = top;
    *p = (void*)base;
    top += (n + 4095) / 4096 * 4096;
    return 0;
}
int hipFree(void*) { note(kFree, nullptr, 0); return 0; }
int hipMemset(void* p, int, size_t n) {
    note(kMemset, nullptr, n);
    if ((uintptr_t)p == base) stub_word = 0;
    return 0;
}
int hipMemcpy(void* dst, const void* src, size_t n, int) { note(kMemcpy, nullptr, n); copied(dst, src); return 0; }
int hipMemcpyAsync(void* dst, const void* src, size_t n, int, void* stream) {
    note(kMemcpyAsync, stream, n);
    copied(dst, src);
    return 0;
}
int hipDeviceSynchronize() { note(kDeviceSync, nullptr, 0); return 0; }
int hipStreamSynchronize(void* stream) { note(kSync, stream, 0); return 0; }
int hipGetLastError() { return 0; }
const char* hipGetErrorString(int) { return "stub"; }

static Dim grid_, block_;
static size_t shared_;
static void* stream_;
int __hipPushCallConfiguration(Dim g, Dim b, size_t n, void* s) { grid_ = g; block_ = b; shared_ = n; stream_ = s; return 0; }
int __hipPopCallConfiguration(Dim* g, Dim* b, size_t* n, void** s) { *g = grid_; *b = block_; *n = shared_; *s = stream_; return 0; }
int hipLaunchKernel(const void*, Dim g, Dim b, void** args, size_t, void* s) {
    note(kLaunch, s, 0, g.x, b.x);
    if (g.x == 1 && b.x == 1) {     // the one launch of one thread takes the error word
        taken_at = *(uintptr_t*)args[1];
        taken = stub_word;
        stub_word = 0;
    }
    return 0;
}

}  // extern "C"
