/* Stands in for the CUDA runtime in a process that has no GPU: kernels are not run, launches are counted, and a launch is refused as the
 * runtime refuses it when a function's limit of dynamic shared memory is too small.  One device, limits as on sm_100. */
#include <cuda_runtime_api.h>
#include <pthread.h>

static pthread_mutex_t lock = PTHREAD_MUTEX_INITIALIZER;
static struct { const void* fn; int limit; } known[256];
static int launched, refused, attributes_fail;

void fake_attributes_fail(int yes) { attributes_fail = yes; }
int fake_launched(void) { return launched; }
int fake_refused(void) { return refused; }

static int* limit_of(const void* fn) {
    for (int i = 0; i < 256; ++i) {
        if (!known[i].fn) {
            known[i].fn = fn;
            known[i].limit = 48 * 1024;
        }
        if (known[i].fn == fn) return &known[i].limit;
    }
    return 0;
}
cudaError_t cudaGetDevice(int* device) { *device = 0; return cudaSuccess; }
cudaError_t cudaGetLastError(void) { return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* value, enum cudaDeviceAttr attr, int device) {
    (void)device;
    *value = attr == cudaDevAttrMultiProcessorCount ? 148 : attr == cudaDevAttrMaxSharedMemoryPerBlockOptin ? 227 * 1024 : 0;
    return cudaSuccess;
}
cudaError_t cudaFuncGetAttributes(struct cudaFuncAttributes* a, const void* fn) {
    (void)fn;
    *a = (struct cudaFuncAttributes){0};
    a->sharedSizeBytes = 12 * 1024;
    return attributes_fail ? cudaErrorMemoryAllocation : cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void* fn, enum cudaFuncAttribute attr, int value) {
    if (attributes_fail) return cudaErrorMemoryAllocation;
    if (attr != cudaFuncAttributeMaxDynamicSharedMemorySize || value < 0 || value > 227 * 1024) return cudaErrorInvalidValue;
    pthread_mutex_lock(&lock);
    int* limit = limit_of(fn);
    if (limit) *limit = value;
    pthread_mutex_unlock(&lock);
    return limit ? cudaSuccess : cudaErrorMemoryAllocation;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* config, const void* fn, void** args) {
    (void)args;
    pthread_mutex_lock(&lock);
    const int* limit = limit_of(fn);
    const int ok = limit && config->dynamicSmemBytes <= (size_t)*limit;
    launched += ok;
    refused += !ok;
    pthread_mutex_unlock(&lock);
    return ok ? cudaSuccess : cudaErrorInvalidValue;
}
