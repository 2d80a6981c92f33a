/* Kernel launches that are written down and not made (with allocations.c): which kernels a call
 * would run, and on how many workgroups, without a device. */
#include <stddef.h>
#include <stdint.h>

typedef struct {
  uint32_t x, y, z;
} dim3;
typedef struct {
  const void* host;
  const char* name;
} kernel;
typedef struct {
  const char* name;
  uint32_t grid[3], block[3];
} launch;

static kernel kernels[8192];
static launch launches[4096];
static int kernel_count, launch_count;

void __hipRegisterFunction(void** modules, const void* host, char* device, const char* name,
                           unsigned limit, void* tid, void* bid, void* block, void* grid,
                           int* size) {
  (void)modules, (void)device, (void)limit, (void)tid, (void)bid, (void)block, (void)grid;
  (void)size;
  if (kernel_count < 8192) kernels[kernel_count++] = (kernel){host, name};
}
static dim3 next_grid, next_block;
int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, void* stream) {
  (void)shared, (void)stream;
  next_grid = grid, next_block = block;
  return 0;
}
int __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, void** stream) {
  *grid = next_grid, *block = next_block, *shared = 0, *stream = NULL;
  return 0;
}
int hipLaunchKernel(const void* host, dim3 grid, dim3 block, void** args, size_t shared,
                    void* stream) {
  (void)args, (void)shared, (void)stream;
  if (launch_count == 4096) return 1;
  launch* l = &launches[launch_count++];
  *l = (launch){"", {grid.x, grid.y, grid.z}, {block.x, block.y, block.z}};
  for (int i = 0; i < kernel_count; ++i)
    if (kernels[i].host == host) l->name = kernels[i].name;
  return 0;
}
int hipGetLastError(void) { return 0; }

int launch_total(void) { return launch_count; }
void launch_forget(void) { launch_count = 0; }
const char* launch_name(int i) { return launches[i].name; }
uint32_t launch_grid(int i, int axis) { return launches[i].grid[axis]; }
