/* The part of the CUDA runtime that csrc/co3_optim.cu calls, on host memory and without a device: what an order of calls may do
 * that a GPU shows only now and then.  A copy from pageable host memory, and a fill, return before they have been carried out
 * (the runtime's documentation allows both); they are carried out when the null stream or the device is waited for, or before a
 * copy back to the host.  Kernels are counted and do nothing. */
#include <stddef.h>
#include <stdlib.h>
#include <string.h>

enum { SUCCESS = 0, HOST_TO_DEVICE = 1, DEVICE_TO_HOST = 2, MULTIPROCESSORS = 16 };

typedef struct { char *to, *from; int value; size_t n; } operation;
static operation waiting[64];
static int n_waiting, device, launches, calls;
static size_t written;                    /* bytes */
static long long* advanced;               /* see fake_advance */

static int add(void* to, const void* from, int value, size_t n) {
    operation* o = &waiting[n_waiting++];
    o->to = (char*)to;
    o->from = from ? (char*)memcpy(malloc(n ? n : 1), from, n) : NULL;
    o->value = value;
    o->n = n;
    written += n;
    return SUCCESS;
}
static int carry_out(void) {
    for (int i = 0; i < n_waiting; ++i) {
        operation* o = &waiting[i];
        if (o->from) { memcpy(o->to, o->from, o->n); free(o->from); }
        else memset(o->to, o->value, o->n);
    }
    n_waiting = 0;
    return SUCCESS;
}

/* ---- for the tests ---- */
int fake_waiting(void) { return n_waiting; }
static void* allocated;
void* fake_allocated(void) { return allocated; }           /* the last allocation of device memory */
int fake_launches(void) { return launches; }
int fake_calls(void) { return calls; }                     /* that wait or touch device memory */
long fake_written(void) { long n = (long)written; written = 0; return n; }
void fake_set_device(int d) { device = d; }
/* As if a step ended on the device just after the next copy to the host: one more at the beginning of what was copied. */
static int advance_next;
void fake_advance(void) { advance_next = 1; }

/* ---- the runtime's names ---- */
int cudaGetDevice(int* d) { *d = device; return SUCCESS; }
int cudaDeviceGetAttribute(int* v, int what, int d) { (void)d; *v = what == MULTIPROCESSORS ? 148 : 0; return SUCCESS; }
int cudaGetLastError(void) { return SUCCESS; }
int cudaMalloc(void** p, size_t n) { *p = NULL; if (posix_memalign(p, 256, n ? n : 256)) return 2; allocated = memset(*p, 0xA5, n); return SUCCESS; }
int cudaFree(void* p) { carry_out(); free(p); return SUCCESS; }
int cudaMemset(void* p, int value, size_t n) { ++calls; return add(p, NULL, value, n); }
int cudaMemcpy(void* to, const void* from, size_t n, int kind) {
    ++calls;
    if (kind == HOST_TO_DEVICE) return add(to, from, 0, n);
    carry_out();
    memcpy(to, from, n);
    if (advance_next) { advanced = (long long*)from; *advanced += 1; advance_next = 0; }
    return SUCCESS;
}
int cudaDeviceSynchronize(void) { ++calls; return carry_out(); }
int cudaStreamSynchronize(void* stream) { ++calls; return stream ? SUCCESS : carry_out(); }
int cudaLaunchKernel(const void* f, ...) { (void)f; ++launches; return SUCCESS; }
int cudaLaunchKernelExC(const void* config, const void* f, void** args) { (void)config; (void)f; (void)args; ++launches; return SUCCESS; }

/* what a compiled .cu file registers when it is loaded */
static void* no_module;
void** __cudaRegisterFatBinary(void* p) { (void)p; return &no_module; }
void __cudaRegisterFatBinaryEnd(void** m) { (void)m; }
void __cudaUnregisterFatBinary(void** m) { (void)m; }
void __cudaRegisterFunction(void** m, const char* f, char* g, const char* n, int t, void* a, void* b, void* c, void* d, int* e) {
    (void)m; (void)f; (void)g; (void)n; (void)t; (void)a; (void)b; (void)c; (void)d; (void)e;
}
unsigned __cudaPushCallConfiguration(void) { return 0; }
int __cudaPopCallConfiguration(void) { return SUCCESS; }
char __cudaInitModule(void** m) { (void)m; return 1; }
