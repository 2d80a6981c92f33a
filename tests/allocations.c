/* The calls that make a plan (allocations, and the copy of a list into one) without a device:
 * a plan can then be made on the CPU, to see what it chose and refuses.  Nothing may be
 * enqueued on it. */
#include <stddef.h>
#include <stdint.h>

int hipMalloc(void** p, size_t bytes) {
  (void)bytes;
  *p = (void*)(uintptr_t)((uint64_t)1 << 40);
  return 0;
}
int hipFree(void* p) {
  (void)p;
  return 0;
}
int hipMemcpyAsync(void* to, const void* from, size_t bytes, int kind, void* stream) {
  (void)to, (void)from, (void)bytes, (void)kind, (void)stream;
  return 0;
}
int hipStreamSynchronize(void* stream) {
  (void)stream;
  return 0;
}
