// A HIP runtime without a GPU, for tests of the library's host code: memory is host memory, a
// launch is recorded and not run, and two devices with different numbers of compute units can
// be told.  Allocations of the library through operator new can be made to fail.  Loaded
// before the library, its functions come first.
#include <cxxabi.h>
#include <dlfcn.h>
#include <stdlib.h>
#include <string.h>

#include <map>
#include <new>
#include <string>

namespace {
struct Dim3 { unsigned x, y, z; };
int device = 0, units[2] = {256, 256}, per_unit[2] = {3, 1};  // blocks of four and of eight wavefronts
int fail_after = -1;  // allocations that succeed before one fails; -1: all do
std::map<const void *, std::string> &names() {
    static auto *m = new std::map<const void *, std::string>;
    return *m;
}
std::string &log() {
    static auto *s = new std::string;
    return *s;
}
void record(const void *f, Dim3 g, Dim3 b, size_t lds) {
    int status = 0;
    char *plain = abi::__cxa_demangle(names()[f].c_str(), nullptr, nullptr, &status);
    log() += (status == 0 ? plain : names()[f].c_str());
    free(plain);
    for (unsigned v : {g.x, g.y, g.z, b.x, b.y, b.z, (unsigned)lds}) log() += "\t" + std::to_string(v);
    log() += "\n";
}
}  // namespace

void *operator new(size_t n) {
    if (fail_after >= 0) {
        Dl_info at;
        if (dladdr(__builtin_return_address(0), &at) && strstr(at.dli_fname, "libkvr") && fail_after-- == 0) throw std::bad_alloc();
    }
    void *p = malloc(n ? n : 1);
    if (!p) throw std::bad_alloc();
    return p;
}

extern "C" {
// for the tests
void host_units(int d, int n) { units[d] = n; }
void host_blocks(int four, int eight) { per_unit[0] = four; per_unit[1] = eight; }
void host_fail_after(int n) { fail_after = n; }
int host_failed() { return fail_after < 0; }
const char *host_log() { return log().c_str(); }
void host_clear() { log().clear(); }

// registration of kernels and device variables
void **__hipRegisterFatBinary(const void *) {
    static void *module;
    return &module;
}
void __hipRegisterFunction(void **, const void *f, char *, const char *name, unsigned, void *, void *, void *, void *, int *) {
    names()[f] = name;
}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipUnregisterFatBinary(void **) {}
int __hipPopCallConfiguration(Dim3 *, Dim3 *, size_t *, void **) { return 1; }

int hipGetDevice(int *d) { return *d = device, 0; }
int hipSetDevice(int d) { return device = d, 0; }
int hipDeviceGetAttribute(int *v, int, int d) { return *v = units[d], 0; }  // (the compute units are all that is asked for)
int hipOccupancyMaxActiveBlocksPerMultiprocessor(int *n, const void *, int threads, size_t) { return *n = per_unit[threads > 256], 0; }
int hipDeviceSynchronize() { return 0; }
int hipGetLastError() { return 0; }
const char *hipGetErrorString(int) { return "error"; }

int hipMalloc(void **p, size_t n) { return *p = aligned_alloc(256, (n + 255) / 256 * 256), 0; }
int hipFree(void *p) { return free(p), 0; }
int hipHostMalloc(void **p, size_t n, unsigned) { return hipMalloc(p, n); }
int hipHostFree(void *p) { return free(p), 0; }
int hipMemcpy(void *d, const void *s, size_t n, int) { return memcpy(d, s, n), 0; }
int hipMemcpyAsync(void *d, const void *s, size_t n, int, void *) {
    log() += "copy\n";
    return memcpy(d, s, n), 0;
}
int hipMemcpy2DAsync(void *, size_t, const void *, size_t, size_t, size_t, int, void *) {
    log() += "copy\n";
    return 0;
}
int hipGetSymbolAddress(void **p, const void *s) { return *p = const_cast<void *>(s), 0; }

int hipEventCreate(void **e) { return *e = malloc(1), 0; }
int hipEventCreateWithFlags(void **e, unsigned) { return hipEventCreate(e); }
int hipEventDestroy(void *e) { return free(e), 0; }
int hipEventElapsedTime(float *ms, void *, void *) { return *ms = 0.f, 0; }
int hipEventRecord(void *, void *) { return 0; }
int hipEventSynchronize(void *) { return 0; }
int hipStreamIsCapturing(void *, int *s) { return *s = 0, 0; }
int hipStreamSynchronize(void *) { return 0; }

int hipLaunchKernel(const void *f, Dim3 g, Dim3 b, void **, size_t lds, void *) { return record(f, g, b, lds), 0; }
int hipExtLaunchKernel(const void *f, Dim3 g, Dim3 b, void **, size_t lds, void *, void *, void *, int) { return record(f, g, b, lds), 0; }
}
