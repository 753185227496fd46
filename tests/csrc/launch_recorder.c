/* Takes the place of the HIP runtime's launch calls for a library loaded after this one (by
 * symbol precedence, in a process of its own): each launch is printed as one line, the kernel's
 * name, its grid and its workgroup, and nothing is launched.  No GPU. */
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>

typedef struct {
  uint32_t x, y, z;
} dim3;

enum { kMost = 4096 };
static const void* stubs[kMost];
static const char* names[kMost];
static int registered;
static dim3 grid, block;
static size_t shared;
static void* stream;
static void* fat_binary;

void** __hipRegisterFatBinary(const void* data) { return (void)data, &fat_binary; }
void __hipUnregisterFatBinary(void** modules) { (void)modules; }
void __hipRegisterVar(void** m, void* v, char* a, char* b, int e, size_t s, int c, int g) {
  (void)m, (void)v, (void)a, (void)b, (void)e, (void)s, (void)c, (void)g;
}
void __hipRegisterFunction(void** modules, const void* stub, char* device_function, const char* name, unsigned limit,
                           void* tid, void* bid, dim3* block_dim, dim3* grid_dim, int* size) {
  (void)modules, (void)device_function, (void)limit, (void)tid, (void)bid, (void)block_dim, (void)grid_dim, (void)size;
  if (registered < kMost) {
    stubs[registered] = stub;
    names[registered++] = name;
  }
}
int __hipPushCallConfiguration(dim3 g, dim3 b, size_t s, void* st) {
  grid = g;
  block = b;
  shared = s;
  stream = st;
  return 0;
}
int __hipPopCallConfiguration(dim3* g, dim3* b, size_t* s, void** st) {
  *g = grid;
  *b = block;
  *s = shared;
  *st = stream;
  return 0;
}
int hipGetLastError(void) { return 0; }
int hipLaunchKernel(const void* stub, dim3 g, dim3 b, void** args, size_t s, void* st) {
  (void)args, (void)s, (void)st;
  const char* name = "?";
  for (int i = 0; i < registered; ++i)
    if (stubs[i] == stub) name = names[i];
  printf("launch %s %u %u %u %u %u %u\n", name, g.x, g.y, g.z, b.x, b.y, b.z);
  return 0;
}
int recorder_print(const char* line) { return printf("%s\n", line), fflush(stdout); }
