/* Stands in front of the HIP runtime and writes down what would be launched, so that what a call launches can be checked
 * without a GPU: loaded into a process before libgta.so, whose launches end here.  One line per event:
 *   attr <kernel> <bytes>                          dynamic LDS asked for
 *   launch <kernel> <grid x y z> <threads> <bytes>  dynamic LDS of the launch */
#include <stdint.h>
#include <stdio.h>
#include <string.h>

typedef struct { uint32_t x, y, z; } dim;

static struct { const void *fn; const char *name; } kernels[4096];
static int n_kernels;
static char text[1 << 22];
static size_t used;

const char *spy_text(void) { return text; }
void spy_clear(void) { text[used = 0] = 0; }

/* the library's kernels */
const char *spy_names(void) {
  static char all[1 << 20];
  size_t n = 0;
  for (int i = 0; i < n_kernels; ++i) n += snprintf(all + n, n < sizeof all ? sizeof all - n : 0, "%s ", kernels[i].name);
  return all;
}

static const char *name_of(const void *fn) {
  for (int i = 0; i < n_kernels; ++i)
    if (kernels[i].fn == fn) return kernels[i].name;
  return "?";
}

#define WRITE(...) do { int k_ = snprintf(text + used, sizeof text - used, __VA_ARGS__); if (k_ > 0 && used + k_ < sizeof text) used += k_; } while (0)

void **__hipRegisterFatBinary(const void *data) { (void)data; static void *module; return &module; }
void __hipUnregisterFatBinary(void **module) { (void)module; }
void __hipRegisterFunction(void **module, const void *fn, char *dev, const char *name, unsigned limit, void *a, void *b, void *c, void *d, int *w) {
  (void)module; (void)dev; (void)limit; (void)a; (void)b; (void)c; (void)d; (void)w;
  if (strstr(name, "gta") && n_kernels < 4096) { kernels[n_kernels].fn = fn; kernels[n_kernels++].name = name; }   /* (torch registers its own) */
}
void __hipRegisterVar(void **module, void *var, char *h, char *dev, int ext, size_t size, int constant, int global) {
  (void)module; (void)var; (void)h; (void)dev; (void)ext; (void)size; (void)constant; (void)global;
}

static dim grid_, block_;
static size_t lds_;
static void *stream_;
int __hipPushCallConfiguration(dim grid, dim block, size_t lds, void *stream) { grid_ = grid; block_ = block; lds_ = lds; stream_ = stream; return 0; }
int __hipPopCallConfiguration(dim *grid, dim *block, size_t *lds, void **stream) { *grid = grid_; *block = block_; *lds = lds_; *stream = stream_; return 0; }

int hipLaunchKernel(const void *fn, dim grid, dim block, void **args, size_t lds, void *stream) {
  (void)args; (void)stream;
  WRITE("launch %s %u %u %u %u %zu\n", name_of(fn), grid.x, grid.y, grid.z, block.x * block.y * block.z, lds);
  return 0;
}
int hipFuncSetAttribute(const void *fn, int attribute, int value) { (void)attribute; WRITE("attr %s %d\n", name_of(fn), value); return 0; }
int hipGetDevice(int *device) { *device = 0; return 0; }
int hipGetLastError(void) { return 0; }
const char *hipGetErrorString(int e) { (void)e; return ""; }
int hipGetSymbolAddress(void **at, const void *symbol) { (void)symbol; *at = (void *)4096; return 0; }
