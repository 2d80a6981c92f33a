/* The device's allocation calls without a device: a plan can then be made on the CPU, to see
 * what it chose.  Nothing may be enqueued on it. */
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
