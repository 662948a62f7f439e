/* Stands in for the HIP runtime's launches on a machine without a GPU: loaded
 * ahead of the library, it writes down every kernel the library launches
 * (name, grid, block, dynamic LDS) and every limit of dynamic LDS it raises, on
 * the device that record_device names.  Nothing runs. */
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

typedef struct { uint32_t x, y, z; } dim3;

static struct { const void *host; char *name; } *kernels;
static size_t n_kernels;
static char *record;
static size_t used, room;
static int device, refuse;
static struct { dim3 grid, block; size_t lds; void *stream; } pushed;

static const char *name_of(const void *host) {
  for (size_t i = 0; i < n_kernels; ++i)
    if (kernels[i].host == host) return kernels[i].name;
  return "?";
}

static void put(const char *line) {
  const size_t n = strlen(line);
  if (used + n + 1 > room) {
    room = 2 * (used + n + 1);
    record = realloc(record, room);
  }
  memcpy(record + used, line, n + 1);
  used += n;
}

/* for the test */
void record_device(int d) { device = d; }
void record_refuse(int yes) { refuse = yes; }
const char *record_take(void) {
  put("");
  used = 0;
  return record;
}

const char *record_kernels(void) {
  for (size_t i = 0; i < n_kernels; ++i) {
    put(kernels[i].name);
    put("\n");
  }
  return record_take();
}

/* for the library */
int hipGetDevice(int *d) {
  *d = device;
  return 0;
}
int hipGetLastError(void) { return 0; }
int hipFuncSetAttribute(const void *f, int what, int value) {
  char line[4096];
  snprintf(line, sizeof line, "limit %d %d %s\n", device, value, name_of(f));
  put(line);
  (void)what;
  return refuse ? 1 : 0;
}
int hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **args,
                    size_t lds, void *stream) {
  char line[4096];
  snprintf(line, sizeof line, "launch %u %u %u %u %u %u %zu %s\n", grid.x,
           grid.y, grid.z, block.x, block.y, block.z, lds, name_of(f));
  put(line);
  (void)args;
  (void)stream;
  return 0;
}
int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds,
                               void *stream) {
  pushed.grid = grid;
  pushed.block = block;
  pushed.lds = lds;
  pushed.stream = stream;
  return 0;
}
int __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds,
                              void **stream) {
  *grid = pushed.grid;
  *block = pushed.block;
  *lds = pushed.lds;
  *stream = pushed.stream;
  return 0;
}
void **__hipRegisterFatBinary(const void *data) {
  static void *handle;
  (void)data;
  return &handle;
}
void __hipUnregisterFatBinary(void **h) { (void)h; }
void __hipRegisterFunction(void **h, const void *host, char *dev,
                           const char *name, unsigned limit, void *a, void *b,
                           void *c, void *d, int *e) {
  kernels = realloc(kernels, (n_kernels + 1) * sizeof *kernels);
  kernels[n_kernels].host = host;
  kernels[n_kernels++].name = strdup(name);
  (void)h; (void)dev; (void)limit; (void)a; (void)b; (void)c; (void)d;
  (void)e;
}
void __hipRegisterVar(void **h, void *var, char *host, char *dev, int ext,
                      size_t size, int constant, int global) {
  (void)h; (void)var; (void)host; (void)dev; (void)ext; (void)size;
  (void)constant; (void)global;
}
