/* A stand-in for the calls of the CUDA runtime that the library makes, loaded in front of it (LD_PRELOAD) where there is
 * no GPU: two devices, memory on the host, launches that are only counted and, to whoever asks, have not finished.
 * What the host side does can then be looked at. */
#include <stdlib.h>
#include <string.h>

static int current, launches, launch_device = -1;

int pretend_launches(void) { return launches; }
int pretend_launch_device(void) { return launch_device; }      /* current at the last one */

int cudaGetDevice(int* device) { *device = current; return 0; }
int cudaSetDevice(int device) {
  if (device < 0 || device > 1) return 101;                    /* cudaErrorInvalidDevice */
  current = device;
  return 0;
}
int cudaDeviceGetAttribute(int* value, int attr, int device) { (void)attr; (void)device; *value = 8; return 0; }
int cudaFuncSetAttribute(const void* f, int attr, int value) { (void)f; (void)attr; (void)value; return 0; }
int cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int* n, const void* f, int block, size_t smem, unsigned flags) {
  (void)f; (void)block; (void)smem; (void)flags;
  *n = 1;
  return 0;
}
int cudaOccupancyMaxActiveBlocksPerMultiprocessor(int* n, const void* f, int block, size_t smem) {
  return cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(n, f, block, smem, 0);
}
int cudaOccupancyMaxActiveClusters(int* n, const void* f, const void* config) { (void)f; (void)config; *n = 1; return 0; }
int cudaMalloc(void** p, size_t n) { *p = malloc(n ? n : 1); return *p ? 0 : 2; }
int cudaFree(void* p) { free(p); return 0; }
int cudaMemset(void* p, int v, size_t n) { memset(p, v, n); return 0; }
int cudaMemcpy(void* d, const void* s, size_t n, int kind) { (void)kind; memcpy(d, s, n); return 0; }
int cudaMemsetAsync(void* p, int v, size_t n, void* stream) { (void)p; (void)v; (void)n; (void)stream; return 0; }
int cudaStreamSynchronize(void* stream) { (void)stream; return 0; }
int cudaDeviceSynchronize(void) { return 0; }
int cudaStreamCreateWithFlags(void** stream, unsigned flags) { (void)flags; *stream = malloc(1); return 0; }
int cudaStreamDestroy(void* stream) { free(stream); return 0; }
int cudaStreamWaitEvent(void* stream, void* event, unsigned flags) { (void)stream; (void)event; (void)flags; return 0; }
int cudaEventCreateWithFlags(void** event, unsigned flags) { (void)flags; *event = malloc(1); return 0; }
int cudaEventDestroy(void* event) { free(event); return 0; }
int cudaEventRecord(void* event, void* stream) { (void)event; (void)stream; return 0; }
int cudaEventQuery(void* event) { (void)event; return 600; }   /* cudaErrorNotReady */
int cudaEventSynchronize(void* event) { (void)event; return 0; }
int cudaHostAlloc(void** p, size_t n, unsigned flags) { (void)flags; return cudaMalloc(p, n); }
int cudaFreeHost(void* p) { free(p); return 0; }
int cudaHostGetDevicePointer(void** d, void* h, unsigned flags) { (void)flags; *d = h; return 0; }
int cudaMemcpyAsync(void* d, const void* s, size_t n, int kind, void* stream) { (void)stream; return cudaMemcpy(d, s, n, kind); }
int cudaGetLastError(void) { return 0; }
const char* cudaGetErrorString(int e) { (void)e; return "made up"; }
int cudaLaunchKernelExC(const void* config, const void* f, void** args) {
  (void)config; (void)f; (void)args;
  ++launches;
  launch_device = current;
  return 0;
}
