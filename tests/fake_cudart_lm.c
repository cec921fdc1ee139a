/* What csrc/co3_embed.cu, co3_layernorm.cu and co3_token_loss.cu call of the runtime beside fake_cudart.c's part, on host memory and without a
 * device.  Launches are written down: grid, thread block, shared memory, and what the first argument begins with. */
#include <stdint.h>
#define cudaLaunchKernelExC unused_launch
#define cudaMalloc plain_malloc
#include "fake_cudart.c"
#undef cudaLaunchKernelExC
#undef cudaMalloc

typedef struct { unsigned grid[3], block[3]; size_t shared; void* stream; void* attrs; unsigned n_attrs; } launch_config;
typedef struct { unsigned grid[3], block[3]; unsigned long long shared; unsigned char arg[512]; } launch;
static launch seen[256];
static int n_seen, fail_malloc;
static size_t allocated_bytes;

int fake_seen(void) { return n_seen; }
void fake_forget(void) { n_seen = 0; }
launch* fake_launch(int i) { return &seen[i]; }
void fake_fail_malloc(int yes) { fail_malloc = yes; }
unsigned long long fake_allocated_bytes(void) { return allocated_bytes; }

int cudaMalloc(void** p, size_t n) {                    /* addresses without memory behind them but for the first megabyte: nothing runs on it */
    *p = NULL;
    if (fail_malloc) return 2;
    allocated_bytes = n;
    return plain_malloc(p, n < 1 << 20 ? n : 1 << 20);
}
int cudaLaunchKernelExC(const launch_config* c, const void* f, void** args) {
    (void)f;
    if (n_seen < 256) {
        launch* l = &seen[n_seen++];
        memcpy(l->grid, c->grid, sizeof(l->grid));
        memcpy(l->block, c->block, sizeof(l->block));
        l->shared = c->shared;
        memcpy(l->arg, args[0], 200);                   /* every argument structure has so many */
    }
    ++launches;
    return SUCCESS;
}
int cudaFuncSetAttribute(const void* f, int what, int value) { (void)f; (void)what; return value <= 232448 ? SUCCESS : 1; }
int cudaOccupancyMaxActiveBlocksPerMultiprocessor(int* n, const void* f, int threads, size_t shared) {
    (void)f;
    *n = (int)(2048 / threads);
    if (shared && *n > (int)(232448 / shared)) *n = (int)(232448 / shared);
    return SUCCESS;
}
/* Refuses what the driver's refuses: addresses, strides and boxes that are not whole 16 bytes. */
static int encode(void* map, int type, unsigned rank, void* at, const uint64_t* dims, const uint64_t* strides, const uint32_t* box, const uint32_t* step,
                  int interleave, int swizzle, int promotion, int fill) {
    (void)step; (void)interleave; (void)swizzle; (void)promotion; (void)fill;
    const unsigned width = type == 7 ? 4 : 2;           /* 32-bit floats, else 16 */
    if ((uintptr_t)at % 16 || rank < 2 || rank > 3) return 1;
    for (unsigned i = 0; i < rank; ++i) if (dims[i] < 1 || dims[i] > (1ull << 32) || box[i] < 1 || box[i] > 256) return 1;
    for (unsigned i = 0; i + 1 < rank; ++i) if (strides[i] % 16 || strides[i] >= 1ull << 40) return 1;
    if (box[0] * width % 16 || box[0] * width > 128) return 1;
    memset(map, 0, 128);
    return SUCCESS;
}
int cudaGetDriverEntryPointByVersion(const char* name, void** f, unsigned version, unsigned long long flags, int* found) {
    (void)name; (void)version; (void)flags;
    *f = (void*)encode;
    *found = 0;
    return SUCCESS;
}
