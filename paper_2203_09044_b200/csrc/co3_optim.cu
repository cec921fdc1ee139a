// The optimizer step that follows the averaged gradient: gradient norm with its clipping factor, and AdamW over
// many tensors at once with the two moments in 32 bits or in 8 (co3_grad_norm, co3_adamw_step, co3_adamw_values).
//
// Work is cut into blocks of 256 consecutive elements of one tensor, one block per warp at a time; the moments of
// tensor l start at a block of their own, so that element i of it has its moments at 256 * block0[l] + i whatever the
// alignment of its weights and gradient.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <new>
#include <stdlib.h>
#include <string.h>

#include "co3_internal.h"

namespace {

constexpr int BLK = 256;                      // elements of a block
constexpr int WARPS = 8;                      // warps of a thread block
constexpr int PER_LANE = BLK / 32;
constexpr int INLINE_TENSORS = 128;           // pointers of so many tensors travel with the launch itself
constexpr int TABLE_TENSORS = 1300;           // ... and of so many with one launch of the kernel that fills the device table
constexpr int MAX_TENSORS = 1 << 20;
constexpr int NORM_WARPS = 4736;              // warps that the norm aims for: 148 SMs x 32

struct Pointers {
    const void* grad;
    void* weight;
    void* copy;
};

struct Tensor {
    int64_t size, block0;
    float decay;
    int32_t pad_;
};

// What changes from step to step, on the device: a captured step can be replayed.
struct Scalars {
    long long steps;                          // taken so far
    double pow1, pow2;                        // beta1^steps, beta2^steps
    float inv_c1, rsqrt_c2;                   // 1 / (1 - beta1^(steps+1)), 1 / sqrt(1 - beta2^(steps+1)): the next step's
    uint32_t key;                             // ... and its key of the rounding counters
    uint32_t ticket, norm_ticket;
    uint32_t flags;
    unsigned long long skipped_elements, skipped_steps;
};

// Published multiply-and-shift mixing of 32 bits (two odd constants): any input bit reaches every output bit.
__host__ __device__ inline uint32_t mix32(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x046CA68Bu;
    return x ^ (x >> 16);
}

__host__ __device__ inline void next_scalars(Scalars& s, double beta1, double beta2, uint32_t seed) {
    s.inv_c1 = (float)(1.0 / (1.0 - s.pow1 * beta1));
    s.rsqrt_c2 = (float)(1.0 / sqrt(1.0 - s.pow2 * beta2));
    s.key = mix32(mix32(seed) + (uint32_t)(s.steps + 1));
}

// 32 bits for the element at `place` of the moment arrays.  For a fixed place this is a bijection of the key, so that each
// value of every group of bits is equally likely over the keys, which is what unbiased rounding needs.
__device__ __forceinline__ uint32_t counter_bits(uint32_t key, uint32_t place) {
    const uint32_t s = key + place * 0x9E3779B9u;
    return (s ^ (s >> 15)) * 0x2C1B3C6Du;
}
__device__ __forceinline__ uint32_t key_of(uint32_t key, int64_t place) { return key + (uint32_t)(place >> 32) * 0x632BE5ABu; }

__device__ __forceinline__ float pow2i(int e) {          // 2^e, -149 <= e <= 127
    return __uint_as_float(e >= -126 ? (uint32_t)(e + 127) << 23 : 1u << (e + 149));
}

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }

__device__ __forceinline__ float load_grad(const void* p, int64_t i, int type) {
    if (type == CO3_F32) return static_cast<const float*>(p)[i];
    if (type == CO3_BF16) return to_f32(static_cast<const __nv_bfloat16*>(p)[i]);
    return to_f32(static_cast<const __half*>(p)[i]);
}

// ---- 8-bit moments ---------------------------------------------------------------------------------------------------
// A code is a float with three mantissa bits.  Its exponent field counts octaves up to that of the largest magnitude of the
// block, which has field TOP (one octave is left above it for values rounded up), and that exponent is stored per block, as
// 32-bit floats hold theirs.  First moment: sign and four exponent bits, the (1,4,3) format of the conversion.  Second: five
// exponent bits, no sign (32 octaves: sixteen of its square root).  Scaled so that its grid lies at the lower end of the
// 32-bit floats, a code IS the upper bits of the float, subnormal codes included, and both directions are a product and a shift.
template <int TOP> struct Scale {
    static constexpr int LEAST = TOP + 3;                // smallest stored exponent: the grid stays within normal floats
    // 2^(top - TOP), as two factors since their product can leave the range
    static __device__ __forceinline__ float up1(int top) { return pow2i(top - 127); }
    static __device__ __forceinline__ float up2() { return pow2i(127 - TOP); }
    static __device__ __forceinline__ float down1(int top) { return pow2i(127 - top); }
    static __device__ __forceinline__ float down2() { return pow2i(TOP - 127); }
    static __device__ __forceinline__ float decode(uint32_t code, int top) {
        return __fmul_rn(__fmul_rn(__uint_as_float(code << 20), up2()), up1(top));
    }
    // rand: 20 bits.  x goes to the grid point above it with the probability that its distance from the one below has.
    static __device__ __forceinline__ uint32_t encode(float x, int top, uint32_t rand) {
        return (__float_as_uint(__fmul_rn(__fmul_rn(x, down1(top)), down2())) + rand) >> 20;
    }
};
using ScaleM = Scale<14>;
using ScaleV = Scale<30>;

__device__ __forceinline__ int warp_top(float x, int least) {     // exponent of the largest of the warp's non-negative x
    const uint32_t m = __reduce_max_sync(0xffffffffu, __float_as_uint(x));
    const int e = (int)(m >> 23);
    return e < least ? least : e;
}

// bf16 by the same stochastic rounding, with 16 bits of the counter; non-finite values as they are
__device__ __forceinline__ __nv_bfloat16 bf16_stochastic(float x, uint32_t rand) {
    const uint32_t b = __float_as_uint(x);
    if ((b & 0x7F800000u) == 0x7F800000u) return __float2bfloat16_rn(x);
    return __ushort_as_bfloat16((unsigned short)((b + (rand & 0xFFFFu)) >> 16));
}

struct StepArgs {
    const Tensor* tensors;
    const int32_t* owner;
    const Pointers* table;                    // device table, or null: the pointers are in `inline_ptr`
    int64_t n_blocks;
    void *m, *v;
    uint8_t *m_exp, *v_exp;
    const co3_grad_info* info;
    const float* d_lr;
    Scalars* sc;
    double beta1, beta2;
    float b1, a1, b2, a2, eps, lr;
    uint32_t seed;
    int grad_type, copy_type;
    Pointers inline_ptr[INLINE_TENSORS];
};

template <int BITS, bool W16>
__global__ void __launch_bounds__(32 * WARPS) adamw_kernel(const __grid_constant__ StepArgs a) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float inv_c1 = a.sc->inv_c1, rsqrt_c2 = a.sc->rsqrt_c2;
    const uint32_t step_key = a.sc->key;
    const bool skip = a.info && a.info->nonfinite != 0;
    const float factor = a.info ? a.info->factor : 1.0f;
    const float lr = a.d_lr ? *a.d_lr : a.lr;
    const float rate = lr * inv_c1;
    __syncthreads();                                      // every thread has read what the last block changes below
    uint32_t kept = 0;
    if (!skip) {
        for (int64_t b = (int64_t)blockIdx.x * WARPS + warp; b < a.n_blocks; b += (int64_t)gridDim.x * WARPS) {
            const int t = a.owner[b];
            const Tensor tn = a.tensors[t];
            const Pointers p = a.table ? a.table[t] : a.inline_ptr[t];
            const int64_t e0 = (b - tn.block0) * BLK, place = b * BLK;
            const int n = (int)(tn.size - e0 < BLK ? tn.size - e0 : BLK);
            const float decay = lr * tn.decay;
            const uint32_t key = key_of(step_key, place);
            float m[PER_LANE], v[PER_LANE];
            int m_top = 0, v_top = 0;
            if (BITS == 8) { m_top = a.m_exp[b]; v_top = a.v_exp[b]; }
            float m_max = 0.0f, v_max = 0.0f;
#pragma unroll
            for (int k = 0; k < PER_LANE; ++k) {
                const int i = lane + 32 * k;
                m[k] = v[k] = 0.0f;
                if (i >= n) continue;
                const float g = __fmul_rn(load_grad(p.grad, e0 + i, a.grad_type), factor);
                float w = W16 ? to_f32(static_cast<const __nv_bfloat16*>(p.weight)[e0 + i]) : static_cast<const float*>(p.weight)[e0 + i];
                float m0, v0;
                if (BITS == 8) {
                    const uint32_t c = static_cast<const uint8_t*>(a.m)[place + i];
                    m0 = ScaleM::decode(c & 127u, m_top);
                    if (c & 128u) m0 = -m0;
                    v0 = ScaleV::decode(static_cast<const uint8_t*>(a.v)[place + i], v_top);
                } else {
                    m0 = static_cast<const float*>(a.m)[place + i];
                    v0 = static_cast<const float*>(a.v)[place + i];
                }
                const float m1 = __fadd_rn(__fmul_rn(m0, a.b1), __fmul_rn(g, a.a1));
                const float v1 = __fadd_rn(__fmul_rn(v0, a.b2), __fmul_rn(__fmul_rn(g, g), a.a2));
                const bool fine = v1 < 0x1p126f;          // also false for NaN
                m[k] = fine ? m1 : m0;
                v[k] = fine ? v1 : v0;
                if (!fine) { ++kept; }
                else {
                    w = w - (w * decay + rate * m1 / (sqrtf(v1) * rsqrt_c2 + a.eps));
                    if (W16) static_cast<__nv_bfloat16*>(p.weight)[e0 + i] = bf16_stochastic(w, counter_bits(key, (uint32_t)(place + i)) >> 10);
                    else static_cast<float*>(p.weight)[e0 + i] = w;
                }
                if (a.copy_type == CO3_BF16) static_cast<__nv_bfloat16*>(p.copy)[e0 + i] = __float2bfloat16_rn(w);
                if (a.copy_type == CO3_F16) static_cast<__half*>(p.copy)[e0 + i] = __float2half_rn(w);
                if (BITS == 8) {
                    m_max = fmaxf(m_max, fabsf(m[k]));
                    v_max = fmaxf(v_max, v[k]);
                } else {
                    static_cast<float*>(a.m)[place + i] = m[k];
                    static_cast<float*>(a.v)[place + i] = v[k];
                }
            }
            if (BITS == 8) {
                m_top = warp_top(m_max, ScaleM::LEAST);
                v_top = warp_top(v_max, ScaleV::LEAST);
                if (lane == 0) { a.m_exp[b] = (uint8_t)m_top; a.v_exp[b] = (uint8_t)v_top; }
#pragma unroll
                for (int k = 0; k < PER_LANE; ++k) {
                    const int i = lane + 32 * k;
                    if (i >= n) continue;
                    const uint32_t r = counter_bits(key, (uint32_t)(place + i));
                    uint32_t c = ScaleM::encode(fabsf(m[k]), m_top, r & 0xFFFFFu);
                    if (m[k] < 0.0f) c |= 128u;
                    static_cast<uint8_t*>(a.m)[place + i] = (uint8_t)c;
                    c = ScaleV::encode(v[k], v_top, r >> 12);
                    if (c == 0 && v[k] > 0.0f) c = 1;
                    static_cast<uint8_t*>(a.v)[place + i] = (uint8_t)c;
                }
            }
        }
    }
    if (kept) {                                           // rare: elements left as they were
        atomicOr(&a.sc->flags, CO3_FLAG_NONFINITE);
        atomicAdd(&a.sc->skipped_elements, (unsigned long long)kept);
    }
    if (threadIdx.x == 0) {                               // the last block to come here prepares the next step
        __threadfence();
        if (atomicAdd(&a.sc->ticket, 1u) == gridDim.x - 1) {
            a.sc->ticket = 0;
            if (skip) {
                atomicOr(&a.sc->flags, CO3_FLAG_NONFINITE);
                a.sc->skipped_steps += 1;
            } else {
                Scalars s = *a.sc;
                s.steps += 1;
                s.pow1 *= a.beta1;
                s.pow2 *= a.beta2;
                next_scalars(s, a.beta1, a.beta2, a.seed);
                a.sc->steps = s.steps; a.sc->pow1 = s.pow1; a.sc->pow2 = s.pow2;
                a.sc->inv_c1 = s.inv_c1; a.sc->rsqrt_c2 = s.rsqrt_c2; a.sc->key = s.key;
            }
        }
    }
}

// ---- gradient norm ------------------------------------------------------------------------------------------------------
// Warp q takes the blocks q*K .. q*K + K-1 and leaves one partial sum for every tensor that it meets, at slot q + tensor
// (going on to the next warp or to the next tensor moves one slot on, so the slots are all different and those of a tensor
// lie side by side).  The thread block that finishes last adds them up, always in the same order.
struct NormArgs {
    const Tensor* tensors;
    const int32_t* owner;
    const Pointers* table;
    int64_t n_blocks;
    int n_tensors, per_warp, grad_type;
    float grad_scale, max_norm;
    double* slots;
    double* sums;                             // per tensor
    unsigned long long* bad;                  // per thread block
    float* tensor_norms;
    co3_grad_info* info;
    Scalars* sc;
    Pointers inline_ptr[INLINE_TENSORS];
};

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

template <typename T>
__device__ __forceinline__ T block_sum(T x, T* sh) {      // same value in every thread
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    __syncthreads();
    if (lane == 0) sh[warp] = x;
    __syncthreads();
    T s = 0;
    for (int w = 0; w < WARPS; ++w) s += sh[w];
    return s;
}

__global__ void __launch_bounds__(32 * WARPS) norm_kernel(const __grid_constant__ NormArgs a) {
    __shared__ double sh[WARPS];
    __shared__ unsigned long long sh_n[WARPS];
    __shared__ bool last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t q = (int64_t)blockIdx.x * WARPS + warp;
    const int64_t b0 = q * a.per_warp, b1 = b0 + a.per_warp < a.n_blocks ? b0 + a.per_warp : a.n_blocks;
    unsigned long long bad = 0;
    int t = -1;
    double s = 0.0;
    for (int64_t b = b0; b < b1; ++b) {
        const int tb = a.owner[b];
        if (tb != t) {
            if (t >= 0) { s = warp_sum(s); if (lane == 0) a.slots[q + t] = s; }
            t = tb;
            s = 0.0;
        }
        const Tensor tn = a.tensors[t];
        const void* g = (a.table ? a.table[t] : a.inline_ptr[t]).grad;
        const int64_t e0 = (b - tn.block0) * BLK;
        const int n = (int)(tn.size - e0 < BLK ? tn.size - e0 : BLK);
#pragma unroll
        for (int k = 0; k < PER_LANE; ++k) {
            const int i = lane + 32 * k;
            if (i >= n) continue;
            const float x = load_grad(g, e0 + i, a.grad_type);
            if (!(fabsf(x) < INFINITY)) { ++bad; continue; }
            const double d = (double)x;
            s = __fma_rn(d, d, s);
        }
    }
    if (t >= 0) { s = warp_sum(s); if (lane == 0) a.slots[q + t] = s; }
    bad = block_sum(bad, sh_n);
    if (threadIdx.x == 0) a.bad[blockIdx.x] = bad;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(&a.sc->norm_ticket, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();

    double total = 0.0;
    for (int t0 = 0; t0 < a.n_tensors; t0 += WARPS) {     // one tensor per warp
        const int u = t0 + warp;
        double x = 0.0;
        if (u < a.n_tensors && a.tensors[u].size > 0) {
            const int64_t f = a.tensors[u].block0, l = f + (a.tensors[u].size - 1) / BLK;
            for (int64_t k = f / a.per_warp + u + lane; k <= l / a.per_warp + u; k += 32) x += __ldcg(&a.slots[k]);
        }
        x = warp_sum(x);
        if (u < a.n_tensors && lane == 0) {
            a.sums[u] = x;
            if (a.tensor_norms) a.tensor_norms[u] = (float)(sqrt(x) * fabs((double)a.grad_scale));
        }
    }
    __syncthreads();
    for (int u = threadIdx.x; u < a.n_tensors; u += 32 * WARPS) total += a.sums[u];
    total = block_sum(total, sh);
    bad = 0;
    for (unsigned k = threadIdx.x; k < gridDim.x; k += 32 * WARPS) bad += __ldcg(&a.bad[k]);
    bad = block_sum(bad, sh_n);
    if (threadIdx.x == 0) {
        const double norm = sqrt(total) * fabs((double)a.grad_scale);
        double factor = a.grad_scale;
        if (a.max_norm > 0.0f && norm > (double)a.max_norm) factor *= (double)a.max_norm / norm;
        a.info->factor = (float)factor;
        a.info->norm = (float)norm;
        a.info->nonfinite = bad;
        a.sc->norm_ticket = 0;
    }
}

// ---- values of the 8-bit moments, and the tables ---------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }

template <typename T>
__global__ void __launch_bounds__(32 * WARPS) values_kernel(const uint8_t* m, const uint8_t* v, const uint8_t* m_exp, const uint8_t* v_exp,
                                                            int64_t n_blocks, T* m_out, T* v_out) {
    const int lane = threadIdx.x & 31;
    for (int64_t b = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5); b < n_blocks; b += (int64_t)gridDim.x * WARPS) {
        const int m_top = m_exp[b], v_top = v_exp[b];
#pragma unroll
        for (int k = 0; k < PER_LANE; ++k) {
            const int64_t i = b * BLK + lane + 32 * k;
            const uint32_t c = m[i];
            const float x = ScaleM::decode(c & 127u, m_top);
            m_out[i] = from_f32<T>(c & 128u ? -x : x);
            v_out[i] = from_f32<T>(ScaleV::decode(v[i], v_top));
        }
    }
}

__global__ void owner_kernel(const Tensor* tensors, int n_tensors, int32_t* owner, int64_t n_blocks) {
    for (int64_t b = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; b < n_blocks; b += (int64_t)gridDim.x * blockDim.x) {
        int lo = 0, hi = n_tensors - 1;                   // last tensor whose block0 is at or below b: never an empty one
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (tensors[mid].block0 <= b) lo = mid; else hi = mid - 1;
        }
        owner[b] = lo;
    }
}

struct TableArgs {
    Pointers ptr[TABLE_TENSORS];
};

__global__ void table_kernel(const __grid_constant__ TableArgs a, Pointers* table, int count) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < count) table[i] = a.ptr[i];
}

int width_of(int type) { return type == CO3_F32 ? 4 : 2; }

}  // namespace

struct co3_adamw {
    int n_tensors, weight_type, grad_type, copy_type, state_bits, device, num_sms, per_warp, norm_grid;
    double beta1, beta2, eps;
    uint32_t seed;
    int64_t n_blocks, n_elements;
    int64_t* sizes;
    void* slab;                               // one device allocation:
    Tensor* tensors;
    int32_t* owner;
    Pointers* table;                          // only with more than INLINE_TENSORS tensors
    Scalars* sc;
    double *slots, *sums;
    unsigned long long* bad;
    int64_t launches;
};

namespace {

int launched(co3_adamw* h, int n) {
    if (cudaGetLastError() != cudaSuccess) return CO3_ECUDA;
    h->launches += n;
    return CO3_OK;
}

bool on_device(const co3_adamw* h) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return false; }
    return dev == h->device;
}

// The pointers of the call, in the launch's own arguments or in the device table.  weights == null: gradients only.
int place_pointers(co3_adamw* h, const void* const* grads, void* const* weights, void* const* copies, Pointers* in_args, cudaStream_t st) {
    for (int t = 0; t < h->n_tensors; ++t) {
        if (h->sizes[t] == 0) continue;
        if (!grads[t] || ((uintptr_t)grads[t] & (uintptr_t)(width_of(h->grad_type) - 1))) return CO3_EINVAL;
        if (weights && (!weights[t] || ((uintptr_t)weights[t] & (uintptr_t)(width_of(h->weight_type) - 1)))) return CO3_EINVAL;
        if (copies && (!copies[t] || ((uintptr_t)copies[t] & 1))) return CO3_EINVAL;
    }
    auto one = [&](int t) { return Pointers{grads[t], weights ? weights[t] : nullptr, copies ? copies[t] : nullptr}; };
    if (h->n_tensors <= INLINE_TENSORS) {
        for (int t = 0; t < h->n_tensors; ++t) in_args[t] = one(t);
        return CO3_OK;
    }
    TableArgs* args = (TableArgs*)malloc(sizeof(TableArgs));
    if (!args) return CO3_ENOMEM;
    int rc = CO3_OK;
    for (int t0 = 0; t0 < h->n_tensors && rc == CO3_OK; t0 += TABLE_TENSORS) {
        const int count = h->n_tensors - t0 < TABLE_TENSORS ? h->n_tensors - t0 : TABLE_TENSORS;
        for (int i = 0; i < count; ++i) args->ptr[i] = one(t0 + i);
        table_kernel<<<(count + 255) / 256, 256, 0, st>>>(*args, h->table + t0, count);
        rc = launched(h, 1);
    }
    free(args);
    return rc;
}

template <int BITS, bool W16>
int launch_step(co3_adamw* h, const StepArgs& a, int grid, cudaStream_t st) {
    adamw_kernel<BITS, W16><<<grid, 32 * WARPS, 0, st>>>(a);
    return launched(h, 1);
}

}  // namespace

extern "C" void co3_adamw_destroy(co3_adamw* h) {
    if (!h) return;
    if (h->slab) cudaFree(h->slab);
    free(h->sizes);
    delete h;
}

extern "C" int co3_adamw_create(co3_adamw** out, const co3_adamw_config* cfg) {
    if (!out || !cfg) return CO3_EINVAL;
    *out = nullptr;
    const int n = cfg->n_tensors;
    if (n < 1 || n > MAX_TENSORS || !cfg->sizes || cfg->reserved) return CO3_EINVAL;
    if (cfg->weight_type != CO3_F32 && cfg->weight_type != CO3_BF16) return CO3_EINVAL;
    if (cfg->grad_type != CO3_F32 && cfg->grad_type != CO3_BF16 && cfg->grad_type != CO3_F16) return CO3_EINVAL;
    if (cfg->copy_type != CO3_NONE && cfg->copy_type != CO3_BF16 && cfg->copy_type != CO3_F16) return CO3_EINVAL;
    if (cfg->copy_type != CO3_NONE && cfg->weight_type != CO3_F32) return CO3_EINVAL;
    if (cfg->state_bits != 32 && cfg->state_bits != 8) return CO3_EINVAL;
    if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) return CO3_EINVAL;
    if (!(cfg->eps >= 0.0 && cfg->eps < INFINITY) || !(cfg->weight_decay >= 0.0 && cfg->weight_decay < INFINITY)) return CO3_EINVAL;
    int64_t blocks = 0, elements = 0;
    for (int t = 0; t < n; ++t) {
        if (cfg->sizes[t] < 0 || cfg->sizes[t] > ((int64_t)1 << 40)) return CO3_EINVAL;
        if (cfg->decay && !(cfg->decay[t] >= 0.0f && cfg->decay[t] < INFINITY)) return CO3_EINVAL;
        blocks += (cfg->sizes[t] + BLK - 1) / BLK;
        elements += cfg->sizes[t];
        if (blocks > 0x7FFFFFFFLL) return CO3_EINVAL;
    }
    co3_adamw* h = new (std::nothrow) co3_adamw();
    if (!h) return CO3_ENOMEM;
    memset(h, 0, sizeof(*h));
    h->n_tensors = n;
    h->weight_type = cfg->weight_type; h->grad_type = cfg->grad_type; h->copy_type = cfg->copy_type; h->state_bits = cfg->state_bits;
    h->beta1 = cfg->beta1; h->beta2 = cfg->beta2; h->eps = cfg->eps; h->seed = cfg->seed;
    h->n_blocks = blocks; h->n_elements = elements;
    int64_t per = blocks / NORM_WARPS;
    h->per_warp = (int)(per < 1 ? 1 : per > 64 ? 64 : per);
    const int64_t norm_warps = (blocks + h->per_warp - 1) / h->per_warp;
    h->norm_grid = (int)((norm_warps + WARPS - 1) / WARPS);
    if (h->norm_grid < 1) h->norm_grid = 1;
    h->sizes = (int64_t*)malloc(sizeof(int64_t) * (size_t)n);
    Tensor* host = (Tensor*)calloc((size_t)n, sizeof(Tensor));
    int rc = h->sizes && host ? CO3_OK : CO3_ENOMEM;
    if (rc == CO3_OK) {
        memcpy(h->sizes, cfg->sizes, sizeof(int64_t) * (size_t)n);
        int64_t b0 = 0;
        for (int t = 0; t < n; ++t) {
            host[t].size = cfg->sizes[t];
            host[t].block0 = b0;
            host[t].decay = cfg->decay ? cfg->decay[t] : (float)cfg->weight_decay;
            b0 += (cfg->sizes[t] + BLK - 1) / BLK;
        }
        if (cudaGetDevice(&h->device) != cudaSuccess || cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, h->device) != cudaSuccess || h->num_sms < 1) {
            (void)cudaGetLastError();
            rc = CO3_ECUDA;
        }
    }
    if (rc == CO3_OK) {                       // one allocation, its parts on 256-byte boundaries
        size_t at = 0;
        auto part = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
        const size_t o_sc = part(sizeof(Scalars)), o_t = part(sizeof(Tensor) * (size_t)n), o_own = part(4 * (size_t)blocks);
        const size_t o_tab = part(n > INLINE_TENSORS ? sizeof(Pointers) * (size_t)n : 0);
        const size_t o_slots = part(8 * (size_t)(norm_warps + n)), o_sums = part(8 * (size_t)n), o_bad = part(8 * (size_t)h->norm_grid);
        if (cudaMalloc(&h->slab, at) != cudaSuccess) { (void)cudaGetLastError(); h->slab = nullptr; rc = CO3_ENOMEM; }
        else {
            char* base = (char*)h->slab;
            h->sc = (Scalars*)(base + o_sc); h->tensors = (Tensor*)(base + o_t); h->owner = (int32_t*)(base + o_own);
            h->table = n > INLINE_TENSORS ? (Pointers*)(base + o_tab) : nullptr;
            h->slots = (double*)(base + o_slots); h->sums = (double*)(base + o_sums); h->bad = (unsigned long long*)(base + o_bad);
            Scalars s;
            memset(&s, 0, sizeof(s));
            s.pow1 = s.pow2 = 1.0;
            next_scalars(s, h->beta1, h->beta2, h->seed);
            bool ok = cudaMemcpy(h->sc, &s, sizeof(s), cudaMemcpyHostToDevice) == cudaSuccess &&
                      cudaMemcpy(h->tensors, host, sizeof(Tensor) * (size_t)n, cudaMemcpyHostToDevice) == cudaSuccess;
            if (ok && blocks) {
                const int64_t grid = (blocks + 255) / 256;
                owner_kernel<<<(int)(grid < 4096 ? grid : 4096), 256>>>(h->tensors, n, h->owner, blocks);
                ok = cudaGetLastError() == cudaSuccess && cudaStreamSynchronize(nullptr) == cudaSuccess;
            }
            if (!ok) { (void)cudaGetLastError(); rc = CO3_ECUDA; }
        }
    }
    free(host);
    if (rc != CO3_OK) { co3_adamw_destroy(h); return rc; }
    *out = h;
    return CO3_OK;
}

extern "C" int co3_adamw_sizes(const co3_adamw* h, int64_t* n_blocks, int64_t* n_elements) {
    if (!h) return CO3_EINVAL;
    if (n_blocks) *n_blocks = h->n_blocks;
    if (n_elements) *n_elements = h->n_elements;
    return CO3_OK;
}

extern "C" int co3_grad_norm(co3_adamw* h, const void* const* grads, float grad_scale, float max_norm, float* tensor_norms, co3_grad_info* info,
                             void* cuda_stream) {
    if (!h || !grads || !info || ((uintptr_t)info & 15) || ((uintptr_t)tensor_norms & 3)) return CO3_EINVAL;
    if (!(fabsf(grad_scale) < INFINITY) || !(max_norm < INFINITY)) return CO3_EINVAL;
    if (!on_device(h)) return CO3_EINVAL;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    NormArgs a;
    int rc = place_pointers(h, grads, nullptr, nullptr, a.inline_ptr, st);
    if (rc != CO3_OK) return rc;
    a.tensors = h->tensors; a.owner = h->owner; a.table = h->table; a.n_blocks = h->n_blocks; a.n_tensors = h->n_tensors;
    a.per_warp = h->per_warp; a.grad_type = h->grad_type; a.grad_scale = grad_scale; a.max_norm = max_norm;
    a.slots = h->slots; a.sums = h->sums; a.bad = h->bad; a.tensor_norms = tensor_norms; a.info = info; a.sc = h->sc;
    norm_kernel<<<h->norm_grid, 32 * WARPS, 0, st>>>(a);
    return launched(h, 1);
}

extern "C" int co3_adamw_step(co3_adamw* h, void* const* weights, const void* const* grads, void* const* copies, const co3_adamw_state* state,
                              double lr, const float* d_lr, const co3_grad_info* info, void* cuda_stream) {
    if (!h || !weights || !grads || !state || !(fabs(lr) < INFINITY)) return CO3_EINVAL;
    if ((copies != nullptr) != (h->copy_type != CO3_NONE)) return CO3_EINVAL;
    if (((uintptr_t)info & 15) || ((uintptr_t)d_lr & 3)) return CO3_EINVAL;
    if (h->n_blocks) {
        if (!state->m || !state->v || (((uintptr_t)state->m | (uintptr_t)state->v) & 31)) return CO3_EINVAL;
        if (h->state_bits == 8 && (!state->m_exp || !state->v_exp)) return CO3_EINVAL;
    }
    if (!on_device(h)) return CO3_EINVAL;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    StepArgs a;
    int rc = place_pointers(h, grads, weights, copies, a.inline_ptr, st);
    if (rc != CO3_OK) return rc;
    a.tensors = h->tensors; a.owner = h->owner; a.table = h->table; a.n_blocks = h->n_blocks;
    a.m = state->m; a.v = state->v; a.m_exp = (uint8_t*)state->m_exp; a.v_exp = (uint8_t*)state->v_exp;
    a.info = info; a.d_lr = d_lr; a.sc = h->sc; a.beta1 = h->beta1; a.beta2 = h->beta2;
    a.b1 = (float)h->beta1; a.a1 = (float)(1.0 - h->beta1); a.b2 = (float)h->beta2; a.a2 = (float)(1.0 - h->beta2);
    a.eps = (float)h->eps; a.lr = (float)lr; a.seed = h->seed; a.grad_type = h->grad_type; a.copy_type = h->copy_type;
    const int64_t need = (h->n_blocks + WARPS - 1) / WARPS, most = (int64_t)h->num_sms * 8;
    const int grid = (int)(need < 1 ? 1 : need < most ? need : most);
    const bool w16 = h->weight_type == CO3_BF16;
    if (h->state_bits == 32) return w16 ? launch_step<32, true>(h, a, grid, st) : launch_step<32, false>(h, a, grid, st);
    return w16 ? launch_step<8, true>(h, a, grid, st) : launch_step<8, false>(h, a, grid, st);
}

extern "C" int co3_adamw_values(co3_adamw* h, const co3_adamw_state* state, void* m_values, void* v_values, int32_t value_type, void* cuda_stream) {
    if (!h || !state || h->state_bits != 8 || (value_type != CO3_F32 && value_type != CO3_BF16)) return CO3_EINVAL;
    if (!on_device(h)) return CO3_EINVAL;
    if (!h->n_blocks) return CO3_OK;
    if (!state->m || !state->v || !state->m_exp || !state->v_exp || (((uintptr_t)state->m | (uintptr_t)state->v) & 31)) return CO3_EINVAL;
    if (!m_values || !v_values || (((uintptr_t)m_values | (uintptr_t)v_values) & 15)) return CO3_EINVAL;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int64_t need = (h->n_blocks + WARPS - 1) / WARPS, most = (int64_t)h->num_sms * 8;
    const int grid = (int)(need < most ? need : most);
    const uint8_t *m = (const uint8_t*)state->m, *v = (const uint8_t*)state->v;
    if (value_type == CO3_F32)
        values_kernel<float><<<grid, 32 * WARPS, 0, st>>>(m, v, state->m_exp, state->v_exp, h->n_blocks, (float*)m_values, (float*)v_values);
    else
        values_kernel<__nv_bfloat16><<<grid, 32 * WARPS, 0, st>>>(m, v, state->m_exp, state->v_exp, h->n_blocks, (__nv_bfloat16*)m_values, (__nv_bfloat16*)v_values);
    return launched(h, 1);
}

extern "C" int co3_adamw_status(co3_adamw* h, uint32_t* flags, uint64_t* skipped_elements, uint64_t* skipped_steps, int32_t clear) {
    if (!h) return CO3_EINVAL;
    Scalars s;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&s, h->sc, sizeof(s), cudaMemcpyDeviceToHost) != cudaSuccess) { (void)cudaGetLastError(); return CO3_ECUDA; }
    if (flags) *flags = s.flags;
    if (skipped_elements) *skipped_elements = s.skipped_elements;
    if (skipped_steps) *skipped_steps = s.skipped_steps;
    if (clear) {
        s.flags = 0;
        s.skipped_elements = s.skipped_steps = 0;
        if (cudaMemcpy(h->sc, &s, sizeof(s), cudaMemcpyHostToDevice) != cudaSuccess) { (void)cudaGetLastError(); return CO3_ECUDA; }
    }
    return CO3_OK;
}

extern "C" int co3_adamw_steps_export(co3_adamw* h, int64_t* steps) {
    if (!h || !steps) return CO3_EINVAL;
    Scalars s;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&s, h->sc, sizeof(s), cudaMemcpyDeviceToHost) != cudaSuccess) { (void)cudaGetLastError(); return CO3_ECUDA; }
    *steps = s.steps;
    return CO3_OK;
}

extern "C" int co3_adamw_steps_import(co3_adamw* h, int64_t steps) {
    if (!h || steps < 0) return CO3_EINVAL;
    Scalars s;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&s, h->sc, sizeof(s), cudaMemcpyDeviceToHost) != cudaSuccess) { (void)cudaGetLastError(); return CO3_ECUDA; }
    s.steps = steps;
    s.pow1 = pow(h->beta1, (double)steps);
    s.pow2 = pow(h->beta2, (double)steps);
    next_scalars(s, h->beta1, h->beta2, h->seed);
    if (cudaMemcpy(h->sc, &s, sizeof(s), cudaMemcpyHostToDevice) != cudaSuccess) { (void)cudaGetLastError(); return CO3_ECUDA; }
    return CO3_OK;
}

extern "C" int64_t co3_adamw_launch_count(const co3_adamw* h) { return h ? h->launches : 0; }
