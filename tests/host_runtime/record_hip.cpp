/*
 * A stand-in for the HIP runtime that records instead of running: what the library
 * allocates, frees and launches, by which thread, can then be looked at without a GPU.
 * Loaded with its symbols global before libsparselnr.so, which then binds to it.
 * Memory is address space only (nothing may touch it).
 */
#define __HIP_PLATFORM_AMD__ 1
#include <hip/hip_runtime_api.h>

#include <pthread.h>
#include <stdio.h>
#include <string.h>
#include <time.h>

#include <cstdlib>
#include <new>

#define API extern "C" __attribute__((visibility("default")))

enum { kLaunch = 0, kMalloc = 1, kFree = 2 };

typedef struct {
  int32_t kind, device;
  uint64_t thread;
  uint32_t grid[3], block[3];
  uint64_t lds, stream, ptr, bytes;  /* ptr, bytes: of an allocation */
  char name[256];                    /* of a kernel */
} record_event;

enum { kMostEvents = 1 << 16, kMostKernels = 4096 };
static record_event g_events[kMostEvents];
static int g_count;
static struct {
  const void *host;
  const char *name;
} g_kernels[kMostKernels];
static int g_kernel_count;
static uint64_t g_next = (uint64_t)1 << 40;
static int g_device;
static int g_wait_ms;
static pthread_mutex_t g_mu = PTHREAD_MUTEX_INITIALIZER;
static pthread_cond_t g_other = PTHREAD_COND_INITIALIZER;

API int record_count(void) { return g_count; }
API const record_event *record_get(int i) { return &g_events[i]; }
API void record_reset(void) { g_count = 0; }
static bool g_no_memory;
/* From here on allocations of C++ objects fail. */
API void record_no_memory(int on) { g_no_memory = on != 0; }
__attribute__((visibility("default"))) void *operator new(size_t n) {
  void *p = g_no_memory ? nullptr : malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
__attribute__((visibility("default"))) void operator delete(void *p) noexcept { free(p); }
__attribute__((visibility("default"))) void operator delete(void *p, size_t) noexcept { free(p); }

/* From here on a thread's launch returns only after another thread's, or after so long. */
API void record_wait(int ms) { g_wait_ms = ms; }

static record_event *add(int kind) { /* g_mu is held */
  static record_event spill;
  record_event *e = g_count < kMostEvents ? &g_events[g_count++] : &spill;
  memset(e, 0, sizeof *e);
  e->kind = kind;
  e->device = g_device;
  e->thread = (uint64_t)pthread_self();
  return e;
}

API hipError_t hipMalloc(void **ptr, size_t size) {
  pthread_mutex_lock(&g_mu);
  record_event *e = add(kMalloc);
  e->ptr = g_next;
  e->bytes = size;
  *ptr = (void *)(uintptr_t)g_next;
  g_next += (size + 4095) / 4096 * 4096 + 4096;
  pthread_mutex_unlock(&g_mu);
  return hipSuccess;
}

API hipError_t hipFree(void *ptr) {
  pthread_mutex_lock(&g_mu);
  add(kFree)->ptr = (uint64_t)(uintptr_t)ptr;
  pthread_mutex_unlock(&g_mu);
  return hipSuccess;
}

API hipError_t hipGetDevice(int *device) {
  *device = g_device;
  return hipSuccess;
}
API hipError_t hipSetDevice(int device) {
  g_device = device;
  return hipSuccess;
}
API hipError_t hipDeviceGetAttribute(int *value, hipDeviceAttribute_t attribute, int device) {
  (void)device;
  *value = attribute == hipDeviceAttributeMultiprocessorCount ? 256 : 160 * 1024;
  return hipSuccess;
}
API hipError_t hipDeviceSynchronize(void) { return hipSuccess; }
API hipError_t hipStreamSynchronize(hipStream_t stream) {
  (void)stream;
  return hipSuccess;
}
API hipError_t hipGetLastError(void) { return hipSuccess; }
API hipError_t hipMemcpyAsync(void *dst, const void *src, size_t n, hipMemcpyKind kind, hipStream_t stream) {
  (void)dst, (void)src, (void)n, (void)kind, (void)stream;
  return hipErrorNotSupported;
}
API hipError_t hipMemsetAsync(void *dst, int value, size_t n, hipStream_t stream) {
  (void)dst, (void)value, (void)n, (void)stream;
  return hipErrorNotSupported;
}
API hipError_t hipGetSymbolAddress(void **ptr, const void *symbol) {
  (void)symbol;
  *ptr = (void *)(uintptr_t)((uint64_t)1 << 39);
  return hipSuccess;
}
API hipError_t hipOccupancyMaxActiveBlocksPerMultiprocessor(int *blocks, const void *f, int size, size_t lds) {
  (void)f, (void)size, (void)lds;
  *blocks = 2;
  return hipSuccess;
}

/* What a kernel's host side calls: the launch's shape is pushed, popped and passed on. */
static thread_local struct {
  dim3 grid, block;
  size_t lds;
  hipStream_t stream;
} g_call;

API hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) {
  g_call.grid = grid, g_call.block = block, g_call.lds = lds, g_call.stream = stream;
  return hipSuccess;
}
API hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream) {
  *grid = g_call.grid, *block = g_call.block, *lds = g_call.lds, *stream = g_call.stream;
  return hipSuccess;
}

API hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **args, size_t lds, hipStream_t stream) {
  (void)args;
  pthread_mutex_lock(&g_mu);
  record_event *e = add(kLaunch);
  e->grid[0] = grid.x, e->grid[1] = grid.y, e->grid[2] = grid.z;
  e->block[0] = block.x, e->block[1] = block.y, e->block[2] = block.z;
  e->lds = lds;
  e->stream = (uint64_t)(uintptr_t)stream;
  for (int i = 0; i < g_kernel_count; ++i)
    if (g_kernels[i].host == f) snprintf(e->name, sizeof e->name, "%s", g_kernels[i].name);
  if (g_wait_ms) {
    static int turn;
    const int mine = ++turn;
    pthread_cond_broadcast(&g_other);
    struct timespec until;
    clock_gettime(CLOCK_REALTIME, &until);
    until.tv_nsec += (long)(g_wait_ms % 1000) * 1000000;
    until.tv_sec += g_wait_ms / 1000 + until.tv_nsec / 1000000000;
    until.tv_nsec %= 1000000000;
    while (turn == mine && pthread_cond_timedwait(&g_other, &g_mu, &until) == 0) {
    }
  }
  pthread_mutex_unlock(&g_mu);
  return hipSuccess;
}

API void **__hipRegisterFatBinary(const void *data) {
  static void *handle;
  (void)data;
  return &handle;
}
API void __hipUnregisterFatBinary(void **modules) { (void)modules; }
API void __hipRegisterFunction(void **modules, const void *host, char *device, const char *name, unsigned int limit,
                               void *tid, void *bid, dim3 *block, dim3 *grid, int *size) {
  (void)modules, (void)device, (void)limit, (void)tid, (void)bid, (void)block, (void)grid, (void)size;
  if (g_kernel_count < kMostKernels) {
    g_kernels[g_kernel_count].host = host;
    g_kernels[g_kernel_count++].name = name;
  }
}
API void __hipRegisterVar(void **modules, void *var, char *host, char *device, int external, size_t size, int constant,
                          int global) {
  (void)modules, (void)var, (void)host, (void)device, (void)external, (void)size, (void)constant, (void)global;
}
