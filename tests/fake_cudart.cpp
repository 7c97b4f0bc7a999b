// The CUDA runtime calls that the host code of the language-model operators makes, without a GPU: every call succeeds and does nothing,
// except the one that a test has fail.  Built into the library in place of the runtime.
#include <cstddef>
#include <cstring>

namespace {
char fail_name[64];
int fail_at, calls_of_it, launches, after_failure, last_error;
bool failed;
int call(const char *name) {
    if (std::strcmp(name, fail_name) != 0 || ++calls_of_it != fail_at) return 0;
    failed = true;
    return last_error = 1;
}
int launch(const char *name) {
    if (failed) ++after_failure;
    ++launches;
    return call(name);
}
int encode(...) { return 0; }
}  // namespace

extern "C" {
void fake_reset(const char *name, int at) {
    std::strncpy(fail_name, name, sizeof(fail_name) - 1);
    fail_at = at;
    calls_of_it = launches = after_failure = 0;                              // (not last_error: the library has to have taken it)
    failed = false;
}
int fake_launches() { return launches; }
int fake_launches_after_failure() { return after_failure; }
int fake_failed() { return failed; }

void **__cudaRegisterFatBinary(void *) { static void *handle; return &handle; }
char __cudaInitModule(void **) { return 1; }
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
void __cudaRegisterFunction(void **, const char *, char *, const char *, int, void *, void *, void *, void *, int *) {}
unsigned __cudaPushCallConfiguration(...) { return 0; }
int __cudaPopCallConfiguration(void *grid, void *block, size_t *shared, void *stream) {
    const unsigned one[3] = {1, 1, 1};
    std::memcpy(grid, one, sizeof(one));
    std::memcpy(block, one, sizeof(one));
    *shared = 0;
    *static_cast<void **>(stream) = nullptr;
    return 0;
}
int cudaLaunchKernel(...) { return launch("cudaLaunchKernel"); }
int cudaLaunchKernelExC(...) { return launch("cudaLaunchKernelExC"); }
int cudaGetLastError() { const int e = last_error; last_error = 0; return e; }
int cudaGetDevice(int *dev) { *dev = 0; return call("cudaGetDevice"); }
int cudaSetDevice(int) { return call("cudaSetDevice"); }
int cudaDeviceGetAttribute(int *value, int, int) { *value = 148; return call("cudaDeviceGetAttribute"); }
int cudaFuncSetAttribute(...) { return call("cudaFuncSetAttribute"); }
int cudaOccupancyMaxActiveClusters(int *n, ...) { *n = 15; return call("cudaOccupancyMaxActiveClusters"); }
int cudaMemsetAsync(...) { return call("cudaMemsetAsync"); }
int cudaMemcpyAsync(...) { return call("cudaMemcpyAsync"); }
int cudaGetDriverEntryPoint(const char *, void **fn, unsigned long long, int *result) {
    *fn = reinterpret_cast<void *>(encode);
    *result = 0;
    return call("cudaGetDriverEntryPoint");
}
}
