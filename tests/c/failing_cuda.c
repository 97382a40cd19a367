/* Loaded in front of pretend_cuda.c's library (LD_PRELOAD): the n-th call of the runtime that can fail, counted from
 * fail_cuda(n), does, once; what the launches and the copies of tables were is remembered.  The driver's encoder of tensor
 * maps is made up too. */
#define _GNU_SOURCE
#include <dlfcn.h>
#include <stddef.h>
#include <string.h>

static int left, seen, copies, launches, mallocs, stops;
static const void* copied_from;

void fail_cuda(int n) { left = n; seen = 0; }
int calls_seen(void) { return seen; }
int copies_seen(void) { return copies; }
const void* last_copy_from(void) { return copied_from; }        /* host memory of the last asynchronous copy */
int launches_seen(void) { return launches; }
int mallocs_seen(void) { return mallocs; }
int stops_seen(void) { return stops; }                          /* calls that wait for all that runs on the device */

static int fails(void) {
  ++seen;
  return left && --left == 0;
}

#define NEXT(name) static __typeof__(name)* next; if (!next) next = (__typeof__(name)*)dlsym(RTLD_NEXT, #name)

int cudaMalloc(void** p, size_t n) {
  NEXT(cudaMalloc);
  ++mallocs;
  return fails() ? 2 : next(p, n);                              /* cudaErrorMemoryAllocation */
}
int cudaHostAlloc(void** p, size_t n, unsigned flags) {
  NEXT(cudaHostAlloc);
  return fails() ? 2 : next(p, n, flags);
}
int cudaMemcpy(void* d, const void* s, size_t n, int kind) {
  NEXT(cudaMemcpy);
  ++stops;
  return fails() ? 999 : next(d, s, n, kind);
}
int cudaMemcpyAsync(void* d, const void* s, size_t n, int kind, void* stream) {
  (void)kind; (void)stream;
  if (fails()) return 999;
  ++copies;
  copied_from = s;
  memcpy(d, s, n);
  return 0;
}
int cudaStreamWaitEvent(void* stream, void* event, unsigned flags) {
  NEXT(cudaStreamWaitEvent);
  return fails() ? 999 : next(stream, event, flags);
}
int cudaEventRecord(void* event, void* stream) {
  NEXT(cudaEventRecord);
  return fails() ? 999 : next(event, stream);
}
int cudaEventCreateWithFlags(void** event, unsigned flags) {
  NEXT(cudaEventCreateWithFlags);
  return fails() ? 999 : next(event, flags);
}
int cudaLaunchKernelExC(const void* config, const void* f, void** args) {
  NEXT(cudaLaunchKernelExC);
  if (fails()) return 999;
  ++launches;
  return next(config, f, args);
}

int cudaFree(void* p) {
  NEXT(cudaFree);
  ++stops;
  return next(p);
}
int cudaDeviceSynchronize(void) {
  NEXT(cudaDeviceSynchronize);
  ++stops;
  return next();
}
int cudaStreamSynchronize(void* stream) {
  NEXT(cudaStreamSynchronize);
  if (!stream || stream == (void*)1 || stream == (void*)2) ++stops;       /* the default streams */
  return next(stream);
}

static int encode() { return 0; }
int cudaGetDriverEntryPointByVersion(const char* name, void** fn, unsigned version, unsigned long long flags, int* result) {
  (void)name; (void)version; (void)flags;
  *fn = (void*)encode;
  if (result) *result = 0;
  return 0;
}
int cudaGetDriverEntryPoint(const char* name, void** fn, unsigned long long flags, int* result) {
  return cudaGetDriverEntryPointByVersion(name, fn, 0, flags, result);
}
