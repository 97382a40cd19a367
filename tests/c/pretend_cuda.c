/* A stand-in for the calls of the CUDA runtime that the operators without a service make, loaded in front of it
 * (LD_PRELOAD) where there is no GPU: two devices, memory on the host, launches that are only counted.  What the
 * host side does about devices can then be looked at. */
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
int cudaLaunchKernelExC(const void* config, const void* f, void** args) {
  (void)config; (void)f; (void)args;
  ++launches;
  launch_device = current;
  return 0;
}
