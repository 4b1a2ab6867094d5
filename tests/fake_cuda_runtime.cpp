// A CUDA runtime that launches nothing, for the library's host code: a call can be made to
// fail, as can an allocation on the host, and the words that reach the device's plan of shared
// pages are kept in `plan`.
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include <new>

namespace {
struct Kernel {
  const void* host;
  const char* name;
};
Kernel kernels[4096];
int n_kernels, fail_name_at = -1, launches, last_error;
char fail_name[64];
int32_t plan[1 << 14];
int fail_new = -1;
}  // namespace

void* operator new(size_t n) {
  if (fail_new >= 0 && fail_new-- == 0) throw std::bad_alloc();
  if (void* p = malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }

extern "C" {
// The next launch but `after` of a kernel whose name holds `part` fails.
void fake_fail(const char* part, int after) {
  strncpy(fail_name, part, sizeof fail_name - 1);
  fail_name_at = after;
}
// The next allocation but `after` fails; returns what was left of that before.
int fake_no_memory(int after) {
  const int was = fail_new;
  fail_new = after;
  return was;
}
int fake_launches() { return launches; }
int32_t* fake_plan() { return plan; }

void* __cudaRegisterFatBinary(void*) { return plan; }
void __cudaRegisterFatBinaryEnd(void*) {}
void __cudaUnregisterFatBinary(void*) {}
void __cudaRegisterVar() {}
void __cudaRegisterFunction(void*, const char* host, char*, const char* name) {
  if (n_kernels < 4096) kernels[n_kernels++] = Kernel{host, name};
}
int __cudaGetKernel() { return 0; }
int __cudaLaunchKernel() { return 0; }
int __cudaPopCallConfiguration() { return 0; }
int cudaLaunchKernelExC(const void*, const void* func, void** args) {
  ++launches;
  const char* name = "";
  for (int i = 0; i < n_kernels; ++i)
    if (kernels[i].host == func) name = kernels[i].name;
  if (fail_name_at >= 0 && strstr(name, fail_name) && fail_name_at-- == 0) return last_error = 1;
  if (strstr(name, "plan_words_kernel")) {
    const int32_t* w = static_cast<const int32_t*>(args[1]);   // n, at, words
    memcpy(plan + w[1], w + 2, 4 * (size_t)w[0]);
  }
  return 0;
}
int cudaMemsetAsync(void*, int, size_t n, void*) {
  if (n >= 2048) memset(plan, 0, sizeof plan);           // the cache's state
  return 0;
}
int cudaMemcpyAsync() {
  if (fail_name_at >= 0 && !strcmp(fail_name, "copy") && fail_name_at-- == 0) return last_error = 1;
  return 0;
}
int cudaDeviceGetAttribute(int* v, int, int) { *v = 152; return 0; }
int cudaGetDevice(int* d) { *d = 0; return 0; }
int cudaStreamIsCapturing(void*, int* st) { *st = 0; return 0; }
int cudaGetSymbolAddress(void** p, const void*) { *p = plan; return 0; }
int cudaFuncSetAttribute() { return 0; }
int cudaFuncGetAttributes(void* a, const void*) { memset(a, 0x7f, 56); return 0; }   // (registers enough)
int cudaGetDriverEntryPointByVersion() { return 0; }
const char* cudaGetErrorString(int) { return "made to fail"; }
int cudaGetLastError() {
  const int e = last_error;
  last_error = 0;
  return e;
}
int cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags() { return 0; }
int cudaStreamSynchronize() { return 0; }
}
