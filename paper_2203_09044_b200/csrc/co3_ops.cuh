// What the kernels at the two ends of a language model share (co3_embed.cu, co3_layernorm.cu, co3_token_loss.cu): element types,
// arrays [users][tokens][dim], launches that begin ahead of the end of the kernel before.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <new>
#include <stdlib.h>
#include <string.h>
#include <type_traits>

#include "co3_internal.h"

namespace {

constexpr int OPS_MAX_USERS = (1 << 16) - 1;                           // blockIdx.y
constexpr int64_t OPS_MAX_ROWS = ((int64_t)1 << 31) - (1 << 16);      // tokens of all users: their numbers are 32-bit ones

// A kernel may start while the one before it on the stream still runs.  It waits for the end of the other, and for its writes, before it
// touches memory.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Element types: EACH of them fill 16 bytes.
struct OF32 {
    typedef float type;
    static constexpr int EACH = 4;
    static __device__ __forceinline__ float get(type x) { return x; }
    static __device__ __forceinline__ type put(float x) { return x; }
    static __device__ __forceinline__ void unpack(uint4 u, float* x) {
        x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 pack(const float* x) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};
struct OBf16 {
    typedef __nv_bfloat16 type;
    static constexpr int EACH = 8;
    static __device__ __forceinline__ float get(type x) { return __bfloat162float(x); }
    static __device__ __forceinline__ type put(float x) { return __float2bfloat16_rn(x); }
    static __device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b) { a = __uint_as_float(w << 16); b = __uint_as_float(w & 0xFFFF0000u); }
    static __device__ __forceinline__ uint32_t pack2(float a, float b) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
        return r;
    }
    static __device__ __forceinline__ void unpack(uint4 u, float* x) {
        unpack2(u.x, x[0], x[1]); unpack2(u.y, x[2], x[3]); unpack2(u.z, x[4], x[5]); unpack2(u.w, x[6], x[7]);
    }
    static __device__ __forceinline__ uint4 pack(const float* x) {
        return make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
    }
};
struct OF16 {
    typedef __half type;
    static constexpr int EACH = 8;
    static __device__ __forceinline__ float get(type x) { return __half2float(x); }
    static __device__ __forceinline__ type put(float x) { return __float2half_rn(x); }
    static __device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b) {
        const float2 f = __half22float2(*(const __half2*)&w);
        a = f.x; b = f.y;
    }
    static __device__ __forceinline__ uint32_t pack2(float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        return *(const uint32_t*)&h;
    }
    static __device__ __forceinline__ void unpack(uint4 u, float* x) {
        unpack2(u.x, x[0], x[1]); unpack2(u.y, x[2], x[3]); unpack2(u.z, x[4], x[5]); unpack2(u.w, x[6], x[7]);
    }
    static __device__ __forceinline__ uint4 pack(const float* x) {
        return make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
    }
};

__device__ __forceinline__ float load_as_f32(const void* p, int type, int64_t i) {
    if (type == CO3_F32) return ((const float*)p)[i];
    if (type == CO3_BF16) return __bfloat162float(((const __nv_bfloat16*)p)[i]);
    return __half2float(((const __half*)p)[i]);
}
__device__ __forceinline__ void store_as(void* p, int type, int64_t i, float x, bool add) {
    if (add) x += load_as_f32(p, type, i);
    if (type == CO3_F32) ((float*)p)[i] = x;
    else if (type == CO3_BF16) ((__nv_bfloat16*)p)[i] = __float2bfloat16_rn(x);
    else ((__half*)p)[i] = __float2half_rn(x);
}

// Two 32-bit numbers on which one instruction works.
struct Two {
    unsigned long long v;
    __device__ __forceinline__ Two() {}
    __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ void get(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
    __device__ __forceinline__ float sum() const { float a, b; get(a, b); return a + b; }
};
__device__ __forceinline__ Two operator+(Two a, Two b) { Two r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ Two operator*(Two a, Two b) { Two r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ Two fma(Two a, Two b, Two c) { Two r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }

__device__ __forceinline__ float warp_sum_f32(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

inline int type_width(int type) { return type == CO3_F32 ? 4 : 2; }
inline bool type_known(int type) { return type == CO3_F32 || type == CO3_BF16 || type == CO3_F16; }
inline bool aligned_to(const void* p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// Whether `count` things `stride` elements apart lie within reach: no sum of such distances passes 64 bits, in bytes neither.
inline bool stride_fine(int64_t count, int64_t stride) {
    const int64_t most = (int64_t)1 << 46;
    return stride >= 0 && stride <= (count > 2 ? most / (count - 1) : most);
}
// Whether an array [users][tokens][dim] that a call is given can be addressed, and, if `out`, whether no two of its elements share a place.
inline bool array_fine(const co3_array* a, int64_t users, int64_t tokens, int64_t dim, bool out) {
    if (!a || !type_known(a->type)) return false;
    if (users == 0 || tokens == 0 || dim == 0) return true;
    if (!a->data || !aligned_to(a->data, type_width(a->type))) return false;
    if (!stride_fine(users, a->user_stride) || !stride_fine(tokens, a->token_stride)) return false;
    if (out && tokens > 1 && a->token_stride < dim) return false;
    if (out && users > 1 && a->user_stride < (tokens - 1) * a->token_stride + dim &&
        !(tokens > 1 && a->user_stride >= dim && a->token_stride >= (users - 1) * a->user_stride + dim)) return false;      // or tokens outermost
    return true;
}
// ... and of a gradient of a weight: [users][n], each user's part in one piece.
inline bool grad_fine(const co3_param_grad* g, int64_t users, int64_t n) {
    if (!g || !type_known(g->type)) return false;
    if (users == 0 || n == 0) return true;
    return g->data && aligned_to(g->data, type_width(g->type)) && (users == 1 || (g->user_stride >= n && stride_fine(users, g->user_stride)));
}
// Whether every row of the array begins on a multiple of 16 bytes.
inline bool rows_aligned(const co3_array* a, int64_t users, int64_t tokens) {
    const int w = type_width(a->type);
    return aligned_to(a->data, 16) && (tokens <= 1 || a->token_stride * w % 16 == 0) && (users <= 1 || a->user_stride * w % 16 == 0);
}

inline bool device_is(int device) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return false; }
    return dev == device;
}

// See let_next_start.  cluster: thread blocks that share a cluster.
template <class... P, class... A>
int launch_early(int64_t* launches, void (*kernel)(P...), dim3 grid, int threads, int shared, int cluster, cudaStream_t st, const A&... args) {
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)shared;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) { (void)cudaGetLastError(); return CO3_ECUDA; }
    *launches += 1;
    return CO3_OK;
}

// Sticky flags and a count on the device, of calls that meet a token number that the vocabulary does not have, or a wait that ran out.
struct OpsStatus {
    unsigned long long bad_tokens;
    uint32_t flags;
    uint32_t pad_;
};
inline int read_status(int device, OpsStatus* at, uint32_t* flags, uint64_t* count, int clear) {
    if (!device_is(device)) return CO3_EINVAL;
    OpsStatus s;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&s, at, sizeof(s), cudaMemcpyDeviceToHost) != cudaSuccess ||
        (clear && (cudaMemset(at, 0, sizeof(s)) != cudaSuccess || cudaStreamSynchronize(nullptr) != cudaSuccess))) {
        (void)cudaGetLastError();
        return CO3_ECUDA;
    }
    if (flags) *flags = s.flags;
    if (count) *count = s.bad_tokens;
    return CO3_OK;
}

}  // namespace
