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
#include <stddef.h>
#include <stdlib.h>
#include <string.h>

#include "co3_internal.h"

namespace {

constexpr int BLK = 256;                      // elements of a block
constexpr int WARPS = 8;                      // warps of a thread block
constexpr int PER_LANE = BLK / 32;
// Pointers of so many tensors travel with the launch itself, of more through a table that a launch before it fills.  As many as 4 KB of
// arguments hold: 9000 elements each, 32-bit moments, device time of a step with room for 32, 64, 128, 160: 62 tensors 5.9, 4.7, 4.7, 4.7 us;
// 100: 6.2, 6.2, 5.0, 4.9; 148: 8.2, 8.2, 8.2, 7.0; one tensor 3.2 in all four; on the host the table costs 5 us more.
constexpr int INLINE_TENSORS = 160;
constexpr int INLINE_GRADS = 384;             // ... of the norm, which takes one for each
constexpr int TABLE_FEW = 400, TABLE_MANY = 1300;   // ... and of so many with one launch of the kernel that fills the device table
constexpr int MAX_TENSORS = 1 << 20;
constexpr int NORM_PER_SM = 3;                // thread blocks of the norm on an SM (2^26 f32: 3 take 44 us, 4 with fewer registers 46)
constexpr int NORM_CTAS = NORM_PER_SM * 148;  // ... and in all at most, whatever the device, so that a sum does not depend on it

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
    float inv_c1, sqrt_c2;                    // 1 / (1 - beta1^(steps+1)), sqrt(1 - beta2^(steps+1)): the next step's
    uint32_t key;                             // ... and its key of the rounding counters
    // What thread blocks change as they end lies apart from what others read as they begin: the two dies keep lines of their own.
    alignas(256) uint32_t ticket;
    uint32_t norm_ticket, flags;
    unsigned long long skipped_elements, skipped_steps;
    unsigned long long nonfinite;             // of the gradients that the norm is reading
};

// Two rounds of xor-shift and odd multiplier, the form of C. Wellons' lowbias32 with the top bit of its second multiplier taken off, so
// that the products of a plain form stay within signed 64 bits.  Any input bit reaches every output bit, about as evenly.
__host__ __device__ inline uint32_t mix32(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x046CA68Bu;
    return x ^ (x >> 16);
}

__host__ __device__ inline void next_scalars(Scalars& s, double beta1, double beta2, uint32_t seed) {
    s.inv_c1 = (float)(1.0 / (1.0 - s.pow1 * beta1));
    s.sqrt_c2 = (float)sqrt(1.0 - s.pow2 * beta2);
    s.key = mix32(mix32(seed) + (uint32_t)(s.steps + 1));
}

// 32 bits for the element at `place` of the moment arrays.  For a fixed place this is a bijection of the key, so that each
// value of every group of bits is equally likely over the keys, which is what unbiased rounding needs.
__device__ __forceinline__ uint32_t counter_bits(uint32_t key, uint32_t place) {
    const uint32_t s = key + place * 0x9E3779B9u;
    return (s ^ (s >> 15)) * 0x2C1B3C6Du;
}
// The key that makes counter_bits(block_key(key, place), i) the bits of `place` + i, for whole blocks at `place`.
__device__ __forceinline__ uint32_t block_key(uint32_t key, int64_t place) {
    return key + (uint32_t)(place >> 32) * 0x632BE5ABu + (uint32_t)place * 0x9E3779B9u;
}

__device__ __forceinline__ float pow2i(int e) {          // 2^e, -149 <= e <= 127
    return __uint_as_float(e >= -126 ? (uint32_t)(e + 127) << 23 : 1u << (e + 149));
}

// A kernel of this file may start while the one before it on the stream still runs.  It then reads what was fixed when the handle
// was made, and waits for the end of the other, and for its writes, before anything else.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
// One more on a ticket, after all that the thread block has written or read before its last barrier, and before what follows.
__device__ __forceinline__ uint32_t take_ticket(uint32_t* ticket) {
    uint32_t old;
    asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(old) : "l"(ticket) : "memory");
    return old;
}
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Two 32-bit operations in one instruction.  (A product whose result goes into a sum may come out as one fused operation, with one
// rounding; where that matters it is written as a fused one itself.)
struct Pair {
    unsigned long long v;
    __device__ __forceinline__ Pair() {}
    explicit __host__ __device__ __forceinline__ Pair(unsigned long long bits) : v(bits) {}
    __device__ __forceinline__ Pair(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ void get(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ Pair operator*(Pair a, Pair b) { Pair r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ Pair operator+(Pair a, Pair b) { Pair r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

__device__ __forceinline__ uint4 load16(const void* p) {
    uint4 u;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
    return u;
}
// The same accesses to shared memory that cp.async has filled.
__device__ __forceinline__ uint4 stage16(uint32_t at) {
    uint4 u;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(at));
    return u;
}
__device__ __forceinline__ uint2 stage8(uint32_t at) {
    uint2 u;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(u.x), "=r"(u.y) : "r"(at));
    return u;
}
template <int BYTES> __device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" :: "r"(to), "l"(from) : "memory");
}
// A type of weights, gradients or copies: one element, and a lane's eight neighbouring ones, in one access if the array begins on a
// multiple of ALIGN + 1 bytes.
struct F32 {
    typedef float type;
    static __device__ __forceinline__ void unpack(const uint4* u, float* x) {
        const uint32_t w[8] = {u[0].x, u[0].y, u[0].z, u[0].w, u[1].x, u[1].y, u[1].z, u[1].w};
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(w[k]);
    }
    static constexpr uintptr_t ALIGN = 31;
    static __device__ __forceinline__ float to(float x) { return x; }
    struct Raw { float x[8]; };                           // eight elements as they lie in memory
    static __device__ __forceinline__ Raw load_raw(const float* p) { Raw r; load8(p, r.x); return r; }
    static __device__ __forceinline__ void unpack_raw(const Raw& r, float* x) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = r.x[k];
    }
    static __device__ __forceinline__ void load8(const float* p, float* x) {
        asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "l"(p));
    }
    static __device__ __forceinline__ void store16(float* p, const float* x) { store8(p, x); store8(p + 8, x + 8); }
    static __device__ __forceinline__ void store8(float* p, const float* x) {
        asm volatile("st.global.v8.f32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"
                     :: "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]), "l"(p) : "memory");
    }
};
struct Bf16 {
    typedef __nv_bfloat16 type;
    static constexpr uintptr_t ALIGN = 15;
    static __device__ __forceinline__ float to(type x) { return __bfloat162float(x); }
    typedef uint4 Raw;
    static __device__ __forceinline__ Raw load_raw(const type* p) { return load16(p); }
    static __device__ __forceinline__ void unpack_raw(const Raw& u, float* x) { unpack(&u, x); }
    static __device__ __forceinline__ void load8(const type* p, float* x) { unpack_raw(load_raw(p), x); }
    static __device__ __forceinline__ void unpack(const uint4* u, float* x) {
        const uint32_t w[4] = {u->x, u->y, u->z, u->w};
#pragma unroll
        for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(w[k] << 16); x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u); }
    }
    static __device__ __forceinline__ uint4 pack(const float* x) {
        __nv_bfloat162 h[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
        return *reinterpret_cast<const uint4*>(h);
    }
    static __device__ __forceinline__ void store16(type* p, const float* x) {
        const uint4 u = pack(x), w = pack(x + 8);
        asm volatile("st.global.v8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"
                     :: "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w), "l"(p) : "memory");
    }
    static __device__ __forceinline__ void store8(type* p, const float* x) { *reinterpret_cast<uint4*>(p) = pack(x); }
};
struct F16 {
    typedef __half type;
    static constexpr uintptr_t ALIGN = 15;
    static __device__ __forceinline__ float to(type x) { return __half2float(x); }
    typedef uint4 Raw;
    static __device__ __forceinline__ Raw load_raw(const type* p) { return load16(p); }
    static __device__ __forceinline__ void unpack_raw(const Raw& u, float* x) { unpack(&u, x); }
    static __device__ __forceinline__ void load8(const type* p, float* x) { unpack_raw(load_raw(p), x); }
    static __device__ __forceinline__ void unpack(const uint4* u, float* x) {
        const uint32_t w[4] = {u->x, u->y, u->z, u->w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
            x[2 * k] = f.x; x[2 * k + 1] = f.y;
        }
    }
    static __device__ __forceinline__ uint4 pack(const float* x) {
        __half2 h[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = __floats2half2_rn(x[2 * k], x[2 * k + 1]);
        return *reinterpret_cast<const uint4*>(h);
    }
    static __device__ __forceinline__ void store8(type* p, const float* x) { *reinterpret_cast<uint4*>(p) = pack(x); }
};

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
    // ... and as one, for stored exponents up to PLAIN (and 2^(TOP - top))
    static constexpr int PLAIN = 126 + TOP;
    static __device__ __forceinline__ float up(int top) { return __uint_as_float((uint32_t)(top + (127 - TOP)) << 23); }
    static __device__ __forceinline__ float down(int top) { return __uint_as_float((uint32_t)(TOP + 127 - top) << 23); }
    static __device__ __forceinline__ float decode(uint32_t code, int top) {
        return __fmul_rn(__fmul_rn(__uint_as_float(code << 20), up2()), up1(top));
    }
    // rand: 20 bits.  x goes to the grid point above it with the probability that its distance from the one below has.
    static __device__ __forceinline__ uint32_t encode(float x, int top, uint32_t rand) {
        return (__float_as_uint(__fmul_rn(__fmul_rn(x, down1(top)), down2())) + rand) >> 20;
    }
    // Eight codes of a lane, with the scale as one factor.
    template <bool SIGNED> static __device__ __forceinline__ void decode8(uint2 c, float up, float* x) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t word = k < 4 ? c.x : c.y;
            const int left = 24 - 8 * (k & 3);                                 // brings the code on top
            uint32_t f;
            if (SIGNED) f = (uint32_t)((int32_t)(word << left) >> 4) & 0x87F00000u;
            else f = (left ? word << (left - 4) : word >> 4) & 0x0FF00000u;
            x[k] = __uint_as_float(f);
        }
        const Pair scale(up, up);
#pragma unroll
        for (int k = 0; k < 8; k += 2) (Pair(x[k], x[k + 1]) * scale).get(x[k], x[k + 1]);
    }
    // Eight codes as floats that lack their block's scale, which is multiplied into the constant that they meet: the first moments' as
    // the e4m3 numbers that they are (but for the code that is no number there and never made here), the second's as upper bits.
    static __device__ __forceinline__ void first8(uint2 c, float* x) {
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            uint32_t h;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)((k < 4 ? c.x : c.y) >> (8 * (k & 3)))));
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
            x[k] = f.x; x[k + 1] = f.y;
        }
    }
    static __device__ __forceinline__ float first_scale(int top) { return __uint_as_float((uint32_t)(top - 7) << 23); }   // e4m3 has field 14 at 2^7
    static __device__ __forceinline__ void second8(uint2 c, float* x) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t word = k < 4 ? c.x : c.y;
            const int left = 20 - 8 * (k & 3);
            x[k] = __uint_as_float((left >= 0 ? word << (left & 31) : word >> 4) & 0x0FF00000u);
        }
    }
    // r: the counters; the first moment takes bits 0..19, the second 12..31.
    template <bool SIGNED> static __device__ __forceinline__ uint2 encode8(const float* x, float down, const uint32_t* r) {
        const Pair scale(down, down);
        float y[8];
        uint32_t z[8], pack[2];
#pragma unroll
        for (int k = 0; k < 8; k += 2) (Pair(x[k], x[k + 1]) * scale).get(y[k], y[k + 1]);
#pragma unroll
        for (int k = 0; k < 8; ++k) z[k] = __float_as_uint(y[k]) + (SIGNED ? r[k] & 0xFFFFFu : r[k] >> 12);
#pragma unroll
        for (int h = 0; h < 2; ++h) {                                          // upper halves: the code in bits 4 .. 11, the sign on top
            const uint32_t a = __byte_perm(z[4 * h], z[4 * h + 1], 0x7632), b = __byte_perm(z[4 * h + 2], z[4 * h + 3], 0x7632);
            pack[h] = __byte_perm(a >> 4, b >> 4, 0x6420);
            if (SIGNED) {
                uint32_t signs;                                                // of four, each through a whole byte
                asm("prmt.b32 %0, %1, %2, 0xFDB9;" : "=r"(signs) : "r"(a), "r"(b));
                pack[h] = (pack[h] & 0x7F7F7F7Fu) | (signs & 0x80808080u);
            }
        }
        if (!SIGNED && ((((pack[0] - 0x01010101u) & ~pack[0]) | ((pack[1] - 0x01010101u) & ~pack[1])) & 0x80808080u)) {
#pragma unroll
            for (int k = 0; k < 8; ++k)                                        // some code is zero: a positive value never is
                if (!(pack[k / 4] >> (8 * (k & 3)) & 0xFFu) && x[k] > 0.0f) pack[k / 4] |= 1u << (8 * (k & 3));
        }
        return make_uint2(pack[0], pack[1]);
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
    unsigned long long b1_pair, a1_pair, b2_pair, a2_pair;   // the first four, each twice
    unsigned long long minus_zero;            // twice -0: a product plus this is the product, rounded
    uint32_t seed;
    int copy_type, stretch;
    bool fast;                                // block_whole is as precise as block_any, see co3_adamw_step
    Pointers inline_ptr[INLINE_TENSORS];
};

static_assert(sizeof(StepArgs) <= 4096, "see INLINE_TENSORS");

struct Step {                                 // what is the same for all elements of a block
    float factor, decay;
    float rate, eps;                          // lr sqrt(1 - beta2^t) / (1 - beta1^t), eps sqrt(1 - beta2^t): the update is rate m / (sqrt(v) + eps)
};

enum Begin { ON_16, ON_4, ON_2 };             // the bytes that an array's beginning is a multiple of
struct Bases {                                // where a tensor's arrays would begin if it began with block 0
    uintptr_t weight, grad, copy;
    Begin weight_begin, copy_begin;           // for stores; ON_16 for whole accesses
    int weight_shift, grad_shift;             // for loads: bytes past a multiple of 16
};

// An element whose second moment is not below this (or is no number) is left as it was.  The bound keeps the exponents
// of 8-bit moments, and first moments with them, far from the end of the range.
constexpr float V_LIMIT = 0x1p126f;

__device__ __forceinline__ void moments(float& m, float& v, float g, const StepArgs& a) {
    m = __fadd_rn(__fmul_rn(m, a.b1), __fmul_rn(g, a.a1));
    v = __fadd_rn(__fmul_rn(v, a.b2), __fmul_rn(__fmul_rn(g, g), a.a2));
}

constexpr int STRETCH = 128;                  // blocks of a thread block at most
template <int BITS> constexpr int STEP_CTAS = BITS == 8 ? 4 : 3;                  // thread blocks of the step on an SM

// Root and quotient to two units in the last place: 2^-22 of the update, itself a small part of the weight.  (block_whole takes them by
// other instructions to the same bound, so that a weight's last bits may depend on which way its block went.)
__device__ __forceinline__ float new_weight(float w, float m, float v, const Step& s) {
    float root;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v));
    return w - __fmaf_rn(w, s.decay, __fdividef(m * s.rate, root + s.eps));
}

// The general way for one block: any alignment, any count, any values.  Lane i takes the elements i, i + 32, ...
template <int BITS, class W, class G>
__device__ __forceinline__ uint32_t block_any(const StepArgs& a, const Step& s, uint32_t key, const Bases& p, int b, int n, uint8_t* tops) {
    const int lane = threadIdx.x & 31;
    const int64_t place = (int64_t)b * BLK;
    typename W::type* pw = reinterpret_cast<typename W::type*>(p.weight) + place;
    const typename G::type* pg = reinterpret_cast<const typename G::type*>(p.grad) + place;
    float g[PER_LANE], w[PER_LANE], m[PER_LANE], v[PER_LANE];
    uint32_t kept = 0;
#pragma unroll
    for (int k = 0; k < PER_LANE; ++k) {
        const int i = lane + 32 * k;
        g[k] = i < n ? G::to(pg[i]) : 0.0f;
        w[k] = i < n ? W::to(pw[i]) : 0.0f;
        if (BITS == 32) {
            m[k] = i < n ? static_cast<const float*>(a.m)[place + i] : 0.0f;
            v[k] = i < n ? static_cast<const float*>(a.v)[place + i] : 0.0f;
        } else {
            const uint32_t c = static_cast<const uint8_t*>(a.m)[place + i];
            m[k] = ScaleM::decode(c & 127u, tops[0]);
            if (c & 128u) m[k] = -m[k];
            v[k] = ScaleV::decode(static_cast<const uint8_t*>(a.v)[place + i], tops[STRETCH]);
            if (i >= n) m[k] = v[k] = 0.0f;
        }
    }
    float m_max = 0.0f, v_max = 0.0f;
#pragma unroll
    for (int k = 0; k < PER_LANE; ++k) {
        const int i = lane + 32 * k;
        float m1 = m[k], v1 = v[k];
        moments(m1, v1, __fmul_rn(g[k], s.factor), a);
        if (v1 < V_LIMIT) {
            m[k] = m1;
            v[k] = v1;
            w[k] = new_weight(w[k], m1, v1, s);
            if (i < n) {
                if (sizeof(typename W::type) == 2) reinterpret_cast<__nv_bfloat16*>(pw)[i] = bf16_stochastic(w[k], counter_bits(key, (uint32_t)i) >> 10);
                else reinterpret_cast<float*>(pw)[i] = w[k];
            }
        } else {
            ++kept;
        }
        if (i < n) {
            if (a.copy_type == CO3_BF16) reinterpret_cast<__nv_bfloat16*>(p.copy)[place + i] = __float2bfloat16_rn(w[k]);
            if (a.copy_type == CO3_F16) reinterpret_cast<__half*>(p.copy)[place + i] = __float2half_rn(w[k]);
            if (BITS == 32) {
                static_cast<float*>(a.m)[place + i] = m[k];
                static_cast<float*>(a.v)[place + i] = v[k];
            }
        }
        m_max = fmaxf(m_max, fabsf(m[k]));
        v_max = fmaxf(v_max, v[k]);
    }
    if (BITS == 8) {
        const int m_top = warp_top(m_max, ScaleM::LEAST), v_top = warp_top(v_max, ScaleV::LEAST);
        __syncwarp();
        if (lane == 0) { tops[0] = (uint8_t)m_top; tops[STRETCH] = (uint8_t)v_top; }
#pragma unroll
        for (int k = 0; k < PER_LANE; ++k) {
            const int i = lane + 32 * k;
            const uint32_t r = counter_bits(key, (uint32_t)i);
            uint32_t c = ScaleM::encode(fabsf(m[k]), m_top, r & 0xFFFFFu);
            c |= __float_as_uint(m[k]) >> 24 & 128u;
            if (i < n) static_cast<uint8_t*>(a.m)[place + i] = (uint8_t)c;
            c = ScaleV::encode(v[k], v_top, r >> 12);
            if (c == 0 && v[k] > 0.0f) c = 1;
            if (i < n) static_cast<uint8_t*>(a.v)[place + i] = (uint8_t)c;
        }
    }
    // with a factor that is not finite every element is left out, but the places past n, 0 times it, are no numbers either
    return fabsf(s.factor) < INFINITY ? kept : (uint32_t)(n + 31 - lane) >> 5;
}

__device__ __forceinline__ float root_fast(float x) { float y; asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float inverse_fast(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

template <int BITS, bool ANY> constexpr bool STAGED = BITS == 8 || ANY;
// With 8-bit moments a block is little to load and much to compute: its loads are started one block ahead, into shared memory, where
// they take no registers.  With 32-bit ones weights and gradients go this way where they do not begin on 16 bytes (67M bf16: 235 us,
// 288 element by element).  A copy of the warp is 512 bytes in a row (with 32 bytes a lane in two copies of 16 each, sectors would
// be fetched twice), so lanes read what others copied and the warp meets before and after.
// Weights and gradients that do not begin on 16 bytes come with what else lies in their first and last 16 (which the tensor's first
// and last blocks, without neighbours in the tensor, leave to the general way), and are moved to their places when they are read.
template <int BITS, class W, class G, bool ANY> struct Stage {      // ANY: arrays may begin anywhere
    static constexpr int W_BYTES = sizeof(typename W::type) * BLK, G_BYTES = sizeof(typename G::type) * BLK;
    static constexpr int W_AT = G_BYTES + 16, M_AT = W_AT + W_BYTES + 16, BYTES = M_AT + (BITS == 8 ? 2 * BLK : 0);
    uint32_t base;                            // of the warp: gradient, weights (each with room for 16 bytes more), codes of 8-bit moments
    template <int N> static __device__ __forceinline__ void bring(uint32_t to, const char* from, int shift) {
        const int lane = threadIdx.x & 31;
        if (ANY) from -= shift;
#pragma unroll
        for (int k = 0; k < N; k += 512) copy_async<16>(to + 16 * lane + k, from + 16 * lane + k);
        if (ANY && shift && lane == 0) copy_async<16>(to + N, from + N);
    }
    __device__ __forceinline__ void start(const StepArgs& a, const Bases& p, int b) const {
        const int lane = threadIdx.x & 31;
        const int64_t at = (int64_t)b * BLK;
        bring<G_BYTES>(base, reinterpret_cast<const char*>(p.grad) + at * (int)sizeof(typename G::type), p.grad_shift);
        bring<W_BYTES>(base + W_AT, reinterpret_cast<const char*>(p.weight) + at * (int)sizeof(typename W::type), p.weight_shift);
        if (BITS == 8) {
            copy_async<8>(base + M_AT + 8 * lane, static_cast<const uint8_t*>(a.m) + at + 8 * lane);
            copy_async<8>(base + M_AT + BLK + 8 * lane, static_cast<const uint8_t*>(a.v) + at + 8 * lane);
        }
    }
    template <class T> static __device__ __forceinline__ void eight(uint32_t from, int shift, float* x) {
        constexpr int n = sizeof(typename T::type) / 2;                        // times 16 bytes
        from += 16 * n * (threadIdx.x & 31);
        uint4 u[n];
#pragma unroll
        for (int k = 0; k < n; ++k) u[k] = stage16(from + 16 * k);
        if (ANY && shift) {
            const uint4 more = stage16(from + 16 * n);
            uint32_t w[4 * n + 4], z[4 * n + 1];
            memcpy(w, u, 16 * n);
            memcpy(w + 4 * n, &more, 16);
            const int words = shift >> 2;                                      // the same in the whole warp
            if (words == 0) { for (int k = 0; k <= 4 * n; ++k) z[k] = w[k]; }
            else if (words == 1) { for (int k = 0; k <= 4 * n; ++k) z[k] = w[k + 1]; }
            else if (words == 2) { for (int k = 0; k <= 4 * n; ++k) z[k] = w[k + 2]; }
            else { for (int k = 0; k <= 4 * n; ++k) z[k] = w[k + 3]; }
            if (n == 1 && (shift & 2)) { for (int k = 0; k < 4; ++k) z[k] = __byte_perm(z[k], z[k + 1], 0x5432); }
            memcpy(u, z, 16 * n);
        }
        T::unpack(u, x);
    }
    __device__ __forceinline__ void take(const Bases& p, float* g, float* w) const {
        eight<G>(base, p.grad_shift, g);
        eight<W>(base + W_AT, p.weight_shift, w);
    }
    __device__ __forceinline__ uint2 codes(int which) const { return stage8(base + M_AT + which * BLK + 8 * (threadIdx.x & 31)); }
    // A lane's eight 32-bit (u[0], u[1]) or 16-bit (u[0]) elements to an array that does not begin on 16 bytes, by way of `part`, which
    // the warp has read.
    template <int N> static __device__ __forceinline__ void send(uint32_t part, const uint4* u, char* to, Begin begin) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int k = 0; k < N / 32; k += 16)
            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" :: "r"(part + N / 32 * lane + k), "r"(u[k / 16].x), "r"(u[k / 16].y), "r"(u[k / 16].z), "r"(u[k / 16].w) : "memory");
        __syncwarp();
        if (begin != ON_2) {
#pragma unroll
            for (int k = 0; k < N; k += 128) {
                uint32_t w;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(part + 4 * lane + k));
                *reinterpret_cast<uint32_t*>(to + 4 * lane + k) = w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; k += 64) {
                unsigned short w;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(part + 2 * lane + k));
                *reinterpret_cast<unsigned short*>(to + 2 * lane + k) = w;
            }
        }
        __syncwarp();
    }
};

// The usual way: a whole block.  Lane i takes the elements 8i .. 8i + 7, each aligned array in one access.
// Returns false, before anything is written, if a value needs the general way.
template <int BITS, class W, class G, bool ANY>
__device__ __forceinline__ bool block_whole(const StepArgs& a, const Step& s, uint32_t key, const Bases& p, int b, const Stage<BITS, W, G, ANY>& stage, uint8_t* tops) {
    constexpr bool W16 = sizeof(typename W::type) == 2;
    const int lane = threadIdx.x & 31;
    const int64_t at = (int64_t)b * BLK + PER_LANE * lane;
    typename W::type* pw = reinterpret_cast<typename W::type*>(p.weight) + at;
    float g[PER_LANE], w[PER_LANE], m[PER_LANE], v[PER_LANE];
    bool other = false;                                   // some value needs the general way
    float b1m = 0.0f, b2v = 0.0f;                         // beta1 and beta2 times the scales of 8-bit moments
    if (BITS == 32) {
        F32::load8(static_cast<const float*>(a.m) + at, m);
        F32::load8(static_cast<const float*>(a.v) + at, v);
    }
    if (!STAGED<BITS, ANY>) {
        G::load8(reinterpret_cast<const typename G::type*>(p.grad) + at, g);
        W::load8(pw, w);
    } else {
        stage.take(p, g, w);
    }
    if (BITS == 8) {
        const uint2 cm = stage.codes(0), cv = stage.codes(1);
        const int m_top = max((int)tops[0], ScaleM::LEAST), v_top = tops[STRETCH];       // (0 before the first step)
        other = m_top > ScaleM::PLAIN || v_top > ScaleV::PLAIN;
        ScaleM::first8(cm, m);
        ScaleV::second8(cv, v);
        b1m = a.b1 * ScaleM::first_scale(m_top);          // exact: see `fast` in co3_adamw_step
        b2v = a.b2 * ScaleV::up(v_top);
    }
    // The four products are formed as fused ones that add -0, for ptxas makes a fused one of a packed product and the sum
    // that takes it, and the moments are rounded after each.
    const Pair b1 = BITS == 8 ? Pair(b1m, b1m) : Pair(a.b1_pair), b2 = BITS == 8 ? Pair(b2v, b2v) : Pair(a.b2_pair);
    const Pair a1(a.a1_pair), a2(a.a2_pair), zero(a.minus_zero);
    const Pair factor(s.factor, s.factor), rate(s.rate, s.rate), decay(s.decay, s.decay), eps(s.eps, s.eps), minus(-1.0f, -1.0f);
    uint32_t v_max = 0;
    float m_max = 0.0f;
    Pair none(0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < PER_LANE; k += 2) {
        const Pair gf = Pair(g[k], g[k + 1]) * factor;
        const Pair m1 = fma(Pair(m[k], m[k + 1]), b1, zero) + fma(gf, a1, zero);
        const Pair v1 = fma(Pair(v[k], v[k + 1]), b2, zero) + fma(gf * gf, a2, zero);
        m1.get(m[k], m[k + 1]);
        v1.get(v[k], v[k + 1]);
        // as whole numbers: NaN of either sign is above the limit too
        v_max = __vimax3_u32(v_max, __float_as_uint(v[k]), __float_as_uint(v[k + 1]));
        if (BITS == 8) asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m_max) : "f"(m_max), "f"(m[k]), "f"(m[k + 1]));
        const Pair d = Pair(root_fast(v[k]), root_fast(v[k + 1])) + eps;
        float d0, d1;
        d.get(d0, d1);
        const Pair w0(w[k], w[k + 1]), upd = fma(w0, decay, m1 * rate * Pair(inverse_fast(d0), inverse_fast(d1))), w1 = fma(upd, minus, w0);
        w1.get(w[k], w[k + 1]);
        if (W16) none = fma(w1, Pair(0.0f, 0.0f), none);  // NaN once a weight is not finite
    }
    int m_top = 0, v_top = 0;
    if (W16) {
        float x, y;
        none.get(x, y);
        other = other || !(x + y == 0.0f);
    }
    if (BITS == 8) {
        v_max = __reduce_max_sync(0xffffffffu, v_max);
        v_top = max((int)(v_max >> 23), ScaleV::LEAST);
        m_top = warp_top(m_max, ScaleM::LEAST);
        other = other || v_max >= __float_as_uint(V_LIMIT) || m_top > ScaleM::PLAIN || v_top > ScaleV::PLAIN;
        if (__any_sync(0xffffffffu, other)) return false;
    } else if (__any_sync(0xffffffffu, other || v_max >= __float_as_uint(V_LIMIT))) {
        return false;
    }
    // The lanes have read the stage and the block's exponents, which are overwritten below: the votes above order no memory.
    if (STAGED<BITS, ANY>) __syncwarp();
    uint32_t r[PER_LANE];
    if (BITS == 8 || W16) {
#pragma unroll
        for (int k = 0; k < PER_LANE; ++k) r[k] = counter_bits(key, (uint32_t)(PER_LANE * lane + k));
    }
    if (W16) {
        uint32_t h[PER_LANE / 2];
#pragma unroll
        for (int k = 0; k < PER_LANE; k += 2)             // all finite: the sum's upper halves (bits 10..25 of the counter by a product: 3 us of 218)
            h[k / 2] = __byte_perm(__float_as_uint(w[k]) + __umulhi(r[k] << 6, 0x10000u), __float_as_uint(w[k + 1]) + __umulhi(r[k + 1] << 6, 0x10000u), 0x7632);
        const uint4 u = make_uint4(h[0], h[1], h[2], h[3]);
        if (!ANY || p.weight_begin == ON_16) *reinterpret_cast<uint4*>(pw) = u;
        else Stage<BITS, W, G, ANY>::template send<2 * BLK>(stage.base + Stage<BITS, W, G, ANY>::W_AT, &u, reinterpret_cast<char*>(pw - PER_LANE * lane), p.weight_begin);
    } else {
        // (eight floats in two accesses of 16 bytes where 32 in one are not possible would write each sector twice)
        if (!ANY || p.weight_begin == ON_16) {
            F32::store8(reinterpret_cast<float*>(pw), w);
        } else {
            uint4 u[2];
            memcpy(u, w, sizeof(u));
            Stage<BITS, W, G, ANY>::template send<4 * BLK>(stage.base + Stage<BITS, W, G, ANY>::W_AT, u, reinterpret_cast<char*>(pw - PER_LANE * lane), p.weight_begin);
        }
        if (a.copy_type != CO3_NONE) {
            if (!ANY || p.copy_begin == ON_16) {
                if (a.copy_type == CO3_BF16) Bf16::store8(reinterpret_cast<__nv_bfloat16*>(p.copy) + at, w);
                else F16::store8(reinterpret_cast<__half*>(p.copy) + at, w);
            } else {
                const uint4 u = a.copy_type == CO3_BF16 ? Bf16::pack(w) : F16::pack(w);
                Stage<BITS, W, G, ANY>::template send<2 * BLK>(stage.base + Stage<BITS, W, G, ANY>::W_AT, &u, reinterpret_cast<char*>(p.copy) + (int64_t)b * (2 * BLK), p.copy_begin);
            }
        }
    }
    if (BITS == 32) {
        F32::store8(static_cast<float*>(a.m) + at, m);
        F32::store8(static_cast<float*>(a.v) + at, v);
    } else {
        if (lane == 0) { tops[0] = (uint8_t)m_top; tops[STRETCH] = (uint8_t)v_top; }
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.m) + at) = ScaleM::encode8<true>(m, ScaleM::down(m_top), r);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.v) + at) = ScaleV::encode8<false>(v, ScaleV::down(v_top), r);
    }
    return true;
}

// The step.  Every element is read and written once; the moments' products and sums are the formula's in its order, so that no other
// order of blocks, and neither way through a block, changes a bit of them.
// 32-bit moments: 28 bytes an element (f32) against 40 instructions, so memory binds: 2^28 f32 in 1091 us, 6.9 TB/s, and 124M with bf16
// gradient and copy in 519 us, 6.7 TB/s, both above the copy rate of 6.55.  11.2M in 62 tensors: 52 us (5.9 TB/s; it begins and ends).
// 8-bit moments: 16 bytes (f32) or 10 (bf16) against 49 instructions, which leave the issue slots 81% busy: 2^28 f32 weights with bf16
// gradient and copy in 667 us, 6.4 TB/s; 124M bf16 in 203 us, 6.15 TB/s, and more under the power limit, which takes clocks away.
template <int BITS, class W, class G, bool ANY>
__global__ void __launch_bounds__(32 * WARPS, STEP_CTAS<BITS>) adamw_kernel(const __grid_constant__ StepArgs a) {
    __shared__ uint8_t tops[2 * STRETCH];                 // the block exponents of the first moments, then of the second
    extern __shared__ __align__(16) char stages[];        // two of each warp, taken in turn
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);     // so that addresses are formed once for the warp
    const int64_t begin = (int64_t)blockIdx.x * a.stretch;
    const int end = (int)min(begin + a.stretch, a.n_blocks), count = end - (int)begin;
    Step s;
    float tensor_decay = 0.0f;
    // of the tensor: block past its last, and its blocks that can go the usual way, from `usual` to below `past`
    int end_t = 0, usual = 0, past = 0;
    Bases p = {0, 0, 0, ON_16, ON_16, 0, 0};
    int t = 0;
    Tensor tn = {0, 0, 0.0f, 0};
    auto find = [&](int b) { t = a.owner[b]; tn = a.tensors[t]; };
    auto enter = [&] {
        const Pointers at = a.table ? a.table[t] : a.inline_ptr[t];
        const uintptr_t e = (uintptr_t)tn.block0 * BLK;
        auto begin_of = [](const void* q, uintptr_t least) { return !((uintptr_t)q & least) ? ON_16 : !((uintptr_t)q & 3) ? ON_4 : ON_2; };
        p = {(uintptr_t)at.weight - e * sizeof(typename W::type), (uintptr_t)at.grad - e * sizeof(typename G::type), (uintptr_t)at.copy - e * 2,
             begin_of(at.weight, W::ALIGN), begin_of(at.copy, 15), (int)((uintptr_t)at.weight & 15), (int)((uintptr_t)at.grad & 15)};
        end_t = (int)(tn.block0 + (tn.size + BLK - 1) / BLK);
        usual = (int)tn.block0;
        past = (int)(tn.block0 + tn.size / BLK);
        const bool aligned = p.weight_begin == ON_16 && p.copy_begin == ON_16 && !((uintptr_t)at.grad & (BITS == 8 ? 15 : G::ALIGN));
        if (ANY && (p.weight_shift || p.grad_shift)) {    // needs the tensor's neighbouring elements, up to 16 bytes of them
            usual += 1;
            past -= tn.size % BLK < 8;
        }
        if (!a.fast || (!ANY && !aligned)) past = 0;
        tensor_decay = tn.decay;
    };
    // a stretch of blocks per thread block, one after the other to its warps
    int b = (int)begin + warp;
    let_next_start();
    if (b < end) find(b);
    wait_for_previous();
    if (b < end) enter();
    const bool skip = a.info && a.info->nonfinite != 0;
    const float lr = a.d_lr ? *a.d_lr : a.lr;
    Stage<BITS, W, G, ANY> stage = {(uint32_t)__cvta_generic_to_shared(stages) + 2 * warp * Stage<BITS, W, G, ANY>::BYTES};
    uint32_t to_other = Stage<BITS, W, G, ANY>::BYTES;
    bool have = false;                                    // block b is on its way to `stage`
    if (STAGED<BITS, ANY>) {
        have = b >= usual && b < min(end, past) && !skip;
        if (have) stage.start(a, p, b);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    if (BITS == 8) {
        for (int i = threadIdx.x; i < 2 * STRETCH; i += 32 * WARPS)
            if ((i & (STRETCH - 1)) < count) tops[i] = (i < STRETCH ? a.m_exp : a.v_exp)[begin + (i & (STRETCH - 1))];
    }
    const float inv_c1 = a.sc->inv_c1, sqrt_c2 = a.sc->sqrt_c2;
    const uint32_t step_key = a.sc->key;
    s.factor = a.info ? a.info->factor : 1.0f;
    s.rate = lr * (inv_c1 * sqrt_c2);
    s.eps = a.eps * sqrt_c2;
    __syncthreads();                                      // every thread has read what the last block changes below
    uint32_t kept = 0;
    if (!skip) {
        for (; b < end; b += WARPS) {
            if (b >= end_t) { find(b); enter(); }
            s.decay = lr * tensor_decay;
            const uint32_t key = block_key(step_key, (int64_t)b * BLK);
            if (STAGED<BITS, ANY>) {
                if (!have && b >= usual && b < past) {
                    stage.start(a, p, b);
                    asm volatile("cp.async.commit_group;" ::: "memory");
                }
                have = b + WARPS >= usual && b + WARPS < min(end, past);
                if (have) Stage<BITS, W, G, ANY>{stage.base + to_other}.start(a, p, b + WARPS);
                asm volatile("cp.async.commit_group;" ::: "memory");
                asm volatile("cp.async.wait_group 1;" ::: "memory");
                __syncwarp();
            }
            if (b < usual || b >= past || !block_whole<BITS, W, G, ANY>(a, s, key, p, b, stage, tops + (b - (int)begin))) {
                const Tensor tn = a.tensors[a.owner[b]];
                const int64_t left = tn.size - (b - tn.block0) * BLK;
                kept += block_any<BITS, W, G>(a, s, key, p, b, left < BLK ? (int)left : BLK, tops + (b - (int)begin));
            }
            __syncwarp();                                 // every lane has taken its part before it is overwritten
            stage.base += to_other;
            to_other = 0u - to_other;
        }
    }
    if (BITS == 8 && !skip) {
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * STRETCH; i += 32 * WARPS)
            if ((i & (STRETCH - 1)) < count) (i < STRETCH ? a.m_exp : a.v_exp)[begin + (i & (STRETCH - 1))] = tops[i];
    }
    if (kept) {                                           // rare: elements left as they were
        atomicOr(&a.sc->flags, CO3_FLAG_NONFINITE);
        atomicAdd(&a.sc->skipped_elements, (unsigned long long)kept);
    }
    if (threadIdx.x == 0) {                               // the last block to come here prepares the next step
        if (take_ticket(&a.sc->ticket) == gridDim.x - 1) {
            a.sc->ticket = 0;
            if (skip) {
                atomicOr(&a.sc->flags, CO3_FLAG_NONFINITE);
                a.sc->skipped_steps += 1;
            } else {
                Scalars n = *a.sc;
                n.steps += 1;
                n.pow1 *= a.beta1;
                n.pow2 *= a.beta2;
                next_scalars(n, a.beta1, a.beta2, a.seed);
                a.sc->steps = n.steps; a.sc->pow1 = n.pow1; a.sc->pow2 = n.pow2;
                a.sc->inv_c1 = n.inv_c1; a.sc->sqrt_c2 = n.sqrt_c2; a.sc->key = n.key;
            }
        }
    }
}

// ---- gradient norm ------------------------------------------------------------------------------------------------------
// Thread block c takes the blocks c*K .. c*K + K-1 and leaves one partial sum for every tensor that it meets, at slot c + tensor:
// going on to the next thread block or to the next tensor moves at least one slot on, so the slots are all different, and those of
// a tensor lie side by side.  Slots that nothing maps to stay zero.  The thread block that finishes last adds them up, always in
// the same order.  Within a thread block, all warps share the blocks of a large piece of a tensor, in turn, so that together they
// read one stretch of memory (a stretch of its own for each warp: 94 us for 2^28 bf16, against 86); small pieces go to one warp each.
struct NormArgs {
    const Tensor* tensors;
    const int32_t* owner;
    const Pointers* table;
    int64_t n_blocks, per_cta;
    int n_tensors, n_slots;
    float grad_scale, max_norm;
    double* slots;
    float* tensor_norms;
    co3_grad_info* info;
    Scalars* sc;
    const void* inline_grad[INLINE_GRADS];
};

template <class G> constexpr int NORM_UNROLL = sizeof(typename G::type) == 2 ? 6 : 3;    // blocks whose loads a warp has in flight
constexpr int NORM_SHARED = 128;              // pieces of tensors that the warps of a thread block share, at most
constexpr int NORM_STAGE = 1024;              // slots that the last thread block brings into shared memory

template <typename T>
__device__ __forceinline__ T warp_sum(T x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

template <typename T>
__device__ __forceinline__ T block_sum(T x, T* sh) {      // same value in every thread
    x = warp_sum(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    T s = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) s += sh[w];
    return s;
}

// The square of a 32-bit float is exact in 64 bits: no range is lost, and the sum rounds at 2^-53.  The conversions (16 a clock on an
// SM) would bind with 16-bit elements: the squares of those are exact in 32 bits too, so that two of them are added there, with
// one rounding, where the largest of a lane's eight has a square well within the range (one that underflows beside it, below 2^-149
// against 2^-100, would not change the sum in 32 bits).  Which two are neighbours in a lane depends on how the gradient is loaded.
template <class G>
__device__ __forceinline__ void add_squares(const float* x, double& s0, double& s1, uint32_t& bad) {
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < PER_LANE; k += 2) top = __vimax3_u32(top, __float_as_uint(x[k]) & 0x7FFFFFFFu, __float_as_uint(x[k + 1]) & 0x7FFFFFFFu);
    if (sizeof(typename G::type) == 2 && top - 0x26800000u < 0x37000000u) {     // 2^-50 <= top < 2^60
#pragma unroll
        for (int k = 0; k < PER_LANE; k += 4) {
            s0 += (double)(x[k] * x[k] + x[k + 1] * x[k + 1]);
            s1 += (double)(x[k + 2] * x[k + 2] + x[k + 3] * x[k + 3]);
        }
    } else if (top < 0x7F800000u) {
        if (sizeof(typename G::type) == 2 && top == 0) return;
#pragma unroll
        for (int k = 0; k < PER_LANE; k += 2) {
            const double d0 = (double)x[k], d1 = (double)x[k + 1];
            s0 = __fma_rn(d0, d0, s0);
            s1 = __fma_rn(d1, d1, s1);
        }
    } else {
#pragma unroll
        for (int k = 0; k < PER_LANE; ++k) {
            if ((__float_as_uint(x[k]) & 0x7FFFFFFFu) >= 0x7F800000u) { ++bad; continue; }
            const double d = (double)x[k];
            s0 = __fma_rn(d, d, s0);
        }
    }
}

// A lane's part of a block, eight elements side by side or 32 apart.
template <class G, bool ALIGNED> struct Part {
    typename G::Raw raw;
    __device__ __forceinline__ void load(const typename G::type* g) { raw = G::load_raw(g + PER_LANE * (threadIdx.x & 31)); }
    __device__ __forceinline__ void get(float* x) const { G::unpack_raw(raw, x); }
};
template <class G> struct Part<G, false> {
    typename G::type raw[PER_LANE];
    __device__ __forceinline__ void load(const typename G::type* g) {
#pragma unroll
        for (int k = 0; k < PER_LANE; ++k) raw[k] = g[(threadIdx.x & 31) + 32 * k];
    }
    __device__ __forceinline__ void get(float* x) const {
#pragma unroll
        for (int k = 0; k < PER_LANE; ++k) x[k] = G::to(raw[k]);
    }
};

// The blocks of a tensor from `first` to below `end`, or every turns-th group of U of them.
template <class G, bool ALIGNED>
__device__ __forceinline__ double squares(const typename G::type* g, int64_t first, int64_t end, int turns, int64_t size, uint32_t& bad) {
    constexpr int U = ALIGNED ? NORM_UNROLL<G> : 2;       // 16-bit elements one by one take a register each
    double s0 = 0.0, s1 = 0.0;
    float x[PER_LANE];
    const int64_t whole = min(end, size / BLK);
    first += (turns > 1 ? (threadIdx.x >> 5) * U : 0);
    g += first * BLK;
    const int stride = U * turns;
    for (int left = (int)(whole - first); left > 0; left -= stride, g += (int64_t)stride * BLK) {
        Part<G, ALIGNED> part[U];
#pragma unroll
        for (int u = 0; u < U; ++u) if (u < left) part[u].load(g + u * BLK);
#pragma unroll
        for (int u = 0; u < U; ++u) if (u < left) { part[u].get(x); add_squares<G>(x, s0, s1, bad); }
    }
    return s0 + s1;
}

// A tensor's last block, not whole.
template <class G>
__device__ __forceinline__ double squares_end(const typename G::type* g, int64_t size, uint32_t& bad) {
    const int lane = threadIdx.x & 31, n = (int)(size % BLK);
    double s0 = 0.0, s1 = 0.0;
    float x[PER_LANE];
    g += size - n;
#pragma unroll
    for (int j = 0; j < PER_LANE; ++j) x[j] = lane + 32 * j < n ? G::to(g[lane + 32 * j]) : 0.0f;
    add_squares<G>(x, s0, s1, bad);
    return s0 + s1;
}

// Reads every gradient once.  2^28 bf16 in 87 us, 6.2 TB/s (in 290 tensors of very different sizes, each with its norm, 100 us);
// 2^26 f32 in 44 us; 11.2M f32 in 13 us, of which the bytes explain 7: the rest is the chain of the last sums (barrier, ticket,
// slots, barrier) after the last load, and the begin of the first.  Gradients that do not begin on 16 bytes (f32: 32) are loaded
// element by element: 2^28 bf16 in 122 us, 2^26 in 37 against 28; f32, four bytes a lane, 161 us for 2^28 against 155, 47 for 2^26.
template <class G>
__global__ void __launch_bounds__(32 * WARPS, NORM_PER_SM) norm_kernel(const __grid_constant__ NormArgs a) {
    __shared__ double sh[WARPS], stage[NORM_STAGE], shared_sum[NORM_SHARED][WARPS];
    __shared__ int shared_tensor[NORM_SHARED];
    __shared__ bool last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c0 = blockIdx.x * a.per_cta, c1 = min(c0 + a.per_cta, a.n_blocks);
    const int large = max(WARPS, (int)(a.per_cta / NORM_SHARED) + 1);           // so that at most NORM_SHARED pieces are large
    uint32_t bad = 0;
    int n_shared = 0, n_small = 0;
    int base = c0 < c1 ? a.owner[c0] : 0;
    bool more = c0 < c1;
    let_next_start();
    bool first = true;
    while (more || first) {
        // 32 tensors at a time, one to a lane
        int64_t block0 = 0, size = 0;
        if (more && base + lane < a.n_tensors) { block0 = a.tensors[base + lane].block0; size = a.tensors[base + lane].size; }
        if (first) wait_for_previous();
        first = false;
        const int64_t f = max(block0, c0), e = min(block0 + (size + BLK - 1) / BLK, c1);
        uint32_t pieces = __ballot_sync(0xffffffffu, more && size > 0 && f < e);
        for (; pieces; pieces &= pieces - 1) {
            const int who = __ffs(pieces) - 1, t = base + who;
            const int64_t b0 = __shfl_sync(0xffffffffu, block0, who), n = __shfl_sync(0xffffffffu, size, who);
            const int64_t from = __shfl_sync(0xffffffffu, f, who) - b0, to = __shfl_sync(0xffffffffu, e, who) - b0;
            const bool share = to - from >= large;
            if (!share && (n_small++ & (WARPS - 1)) != warp) continue;
            int64_t at = from, end = to;
            int turns = 1;
            if (share) {
                if (to - from >= 8 * WARPS) turns = WARPS;
                else { at = from + (to - from) * warp / WARPS; end = from + (to - from) * (warp + 1) / WARPS; }
            }
            const typename G::type* g = static_cast<const typename G::type*>(a.table ? a.table[t].grad : a.inline_grad[t]);
            double s = (uintptr_t)g & G::ALIGN ? squares<G, false>(g, at, end, turns, n, bad) : squares<G, true>(g, at, end, turns, n, bad);
            if (to * BLK > n && (!share || warp == WARPS - 1)) s += squares_end<G>(g, n, bad);
            s = warp_sum(s);
            if (lane == 0) {
                if (share) { shared_sum[n_shared][warp] = s; shared_tensor[n_shared] = t; }
                else a.slots[blockIdx.x + t] = s;
            }
            n_shared += share;
        }
        // done once a tensor reaches beyond this thread block's blocks, or none is left
        more = more && !__any_sync(0xffffffffu, size > 0 && block0 + (size + BLK - 1) / BLK >= c1) && base + 32 < a.n_tensors;
        base += 32;
    }
    if (bad) atomicAdd(&a.sc->nonfinite, (unsigned long long)bad);             // rare
    __syncthreads();
    if (threadIdx.x < n_shared) {
        double s = 0.0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) s += shared_sum[threadIdx.x][w];
        a.slots[blockIdx.x + shared_tensor[threadIdx.x]] = s;
    }
    __syncthreads();
    if (threadIdx.x == 0) last = take_ticket(&a.sc->norm_ticket) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;

    // The sums, and where each tensor's lie, on their way together.
    double total = 0.0;
    for (int k = threadIdx.x; k < a.n_slots; k += 32 * WARPS) {
        const double x = __ldcg(&a.slots[k]);
        total += x;
        if (k < NORM_STAGE) stage[k] = x;
    }
    auto range = [&](int t) {
        const Tensor tn = a.tensors[t];
        int2 k = {0, 0};
        if (tn.size > 0) {
            k.x = (int)(tn.block0 / a.per_cta) + t;
            k.y = (int)((tn.block0 + (tn.size - 1) / BLK) / a.per_cta) + t + 1;
        }
        return k;
    };
    const int mine = lane * WARPS + warp;                 // the tensors of a warp lie apart: neighbours may both have many slots
    int2 k = {0, 0};
    if (a.tensor_norms && mine < a.n_tensors) k = range(mine);
    total = block_sum(total, sh);
    if (threadIdx.x == 0) {
        const double norm = sqrt(total) * fabs((double)a.grad_scale);
        double factor = a.grad_scale;
        if (a.max_norm > 0.0f && norm > (double)a.max_norm) factor *= (double)a.max_norm / norm;
        a.info->factor = (float)factor;
        a.info->norm = (float)norm;
        a.info->nonfinite = __ldcg(&a.sc->nonfinite);
        a.sc->nonfinite = 0;
        a.sc->norm_ticket = 0;
    }
    if (!a.tensor_norms) return;
    auto slot = [&](int i) { return i < NORM_STAGE ? stage[i] : __ldcg(&a.slots[i]); };
    const double scale = fabs((double)a.grad_scale);
    for (int t0 = 0; t0 < a.n_tensors; t0 += 32 * WARPS) {
        // a lane per tensor; those with many slots are then added by the whole warp
        const int t = t0 + mine;
        if (t0) k = t < a.n_tensors ? range(t) : int2{0, 0};
        const bool many = k.y - k.x > 8;
        double x = 0.0;
        if (!many) for (int i = k.x; i < k.y; ++i) x += slot(i);
        for (uint32_t left = __ballot_sync(0xffffffffu, many); left; left &= left - 1) {
            const int who = __ffs(left) - 1, f = __shfl_sync(0xffffffffu, k.x, who), l = __shfl_sync(0xffffffffu, k.y, who);
            double y = 0.0;
            for (int i = f + lane; i < l; i += 32) y += slot(i);
            y = warp_sum(y);
            if (lane == who) x = y;
        }
        if (t < a.n_tensors) a.tensor_norms[t] = (float)(sqrt(x) * scale);
    }
}

// ---- values of the 8-bit moments, and the tables ---------------------------------------------------------------------------
// A warp takes two blocks, sixteen codes of a block to a lane, and stores 32 bytes at a time (124M: 111 us, 6.7 TB/s; one block
// and 16 bytes at a time 125 us).
template <class T, bool SECOND>
__device__ __forceinline__ void values16(uint4 c, int top, typename T::type* out) {
    // the second factor is 1 but for the largest exponents, which one factor cannot hold
    const int most = SECOND ? ScaleV::PLAIN : ScaleM::PLAIN, more = top > most ? top - most : 0;
    const float up = SECOND ? ScaleV::up(top - more) : ScaleM::up(top - more);
    float x[16];
    if (SECOND) { ScaleV::decode8<false>(make_uint2(c.x, c.y), up, x); ScaleV::decode8<false>(make_uint2(c.z, c.w), up, x + 8); }
    else { ScaleM::decode8<true>(make_uint2(c.x, c.y), up, x); ScaleM::decode8<true>(make_uint2(c.z, c.w), up, x + 8); }
    if (more) for (int k = 0; k < 16; ++k) x[k] *= pow2i(more);
    T::store16(out, x);
}

template <class T>
__global__ void __launch_bounds__(32 * WARPS) values_kernel(const uint8_t* m, const uint8_t* v, const uint8_t* m_exp, const uint8_t* v_exp,
                                                            int64_t n_blocks, typename T::type* m_out, typename T::type* v_out) {
    const int lane = threadIdx.x & 31;
    const int64_t b = 2 * ((int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5)) + (lane >> 4), at = b * BLK + 16 * (lane & 15);
    let_next_start();
    wait_for_previous();
    if (b >= n_blocks) return;
    const uint4 cm = load16(m + at), cv = load16(v + at);
    const int m_top = m_exp[b], v_top = v_exp[b];
    values16<T, false>(cm, m_top, m_out + at);
    values16<T, true>(cv, v_top, v_out + at);
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

template <int N> struct TableArgs {
    Pointers ptr[N];
};

template <int N> __global__ void table_kernel(const __grid_constant__ TableArgs<N> a, Pointers* table, int count) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    let_next_start();
    wait_for_previous();
    if (i < count) table[i] = a.ptr[i];
}

int width_of(int type) { return type == CO3_F32 ? 4 : 2; }

}  // namespace

struct co3_adamw {
    int n_tensors, weight_type, grad_type, copy_type, state_bits, device, num_sms, norm_grid, n_slots;
    double beta1, beta2, eps;
    uint32_t seed;
    int64_t n_blocks, n_elements, per_cta;
    int64_t* sizes;
    void* slab;                               // one device allocation:
    Tensor* tensors;
    int32_t* owner;
    Pointers* table;                          // only with more than INLINE_TENSORS tensors
    Scalars* sc;
    double* slots;
    int64_t launches;
};

namespace {

// See let_next_start.
template <class... P, class... A>
int launch(co3_adamw* h, void (*kernel)(P...), int grid, int threads, int shared, cudaStream_t st, const A&... args) {
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)shared;
    cfg.stream = st;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) { (void)cudaGetLastError(); return CO3_ECUDA; }
    h->launches += 1;
    return CO3_OK;
}

bool on_device(const co3_adamw* h) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return false; }
    return dev == h->device;
}

// To the device, and there when the call returns.  A copy from pageable memory alone may still be on its way then, and streams that do
// not wait for the null stream (PyTorch's) would not wait for it.
bool to_device(void* to, const void* from, size_t bytes) {
    return cudaMemcpy(to, from, bytes, cudaMemcpyHostToDevice) == cudaSuccess && cudaStreamSynchronize(nullptr) == cudaSuccess;
}

// Whether all pointers are there and aligned as their types.  weights == null: gradients only.
bool pointers_fine(const co3_adamw* h, const void* const* grads, void* const* weights, void* const* copies) {
    for (int t = 0; t < h->n_tensors; ++t) {
        if (h->sizes[t] == 0) continue;
        if (!grads[t] || ((uintptr_t)grads[t] & (uintptr_t)(width_of(h->grad_type) - 1))) return false;
        if (weights && (!weights[t] || ((uintptr_t)weights[t] & (uintptr_t)(width_of(h->weight_type) - 1)))) return false;
        if (copies && (!copies[t] || ((uintptr_t)copies[t] & 1))) return false;
    }
    return true;
}

// The pointers of the call to the device table.
int fill_table(co3_adamw* h, const void* const* grads, void* const* weights, void* const* copies, cudaStream_t st) {
    auto one = [&](int t) { return Pointers{grads[t], weights ? weights[t] : nullptr, copies ? copies[t] : nullptr}; };
    TableArgs<TABLE_MANY>* args = (TableArgs<TABLE_MANY>*)malloc(sizeof(TableArgs<TABLE_MANY>));
    if (!args) return CO3_ENOMEM;
    int rc = CO3_OK;
    for (int t0 = 0; t0 < h->n_tensors && rc == CO3_OK; t0 += TABLE_MANY) {
        const int count = h->n_tensors - t0 < TABLE_MANY ? h->n_tensors - t0 : TABLE_MANY;
        for (int i = 0; i < count; ++i) args->ptr[i] = one(t0 + i);
        if (count <= TABLE_FEW)               // the arguments of a launch are copied whole
            rc = launch(h, table_kernel<TABLE_FEW>, (count + 255) / 256, 256, 0, st, *(const TableArgs<TABLE_FEW>*)args, h->table + t0, count);
        else
            rc = launch(h, table_kernel<TABLE_MANY>, (count + 255) / 256, 256, 0, st, *args, h->table + t0, count);
    }
    free(args);
    return rc;
}

template <int BITS, class W, class G>
int launch_step_of(co3_adamw* h, const StepArgs& a, bool aligned, int grid, cudaStream_t st) {
    // The kernel that takes arrays from any beginning, for one array of 67M elements that needs it and for one that does not but stands
    // beside one that does, against the other kernel: 8-bit moments, bf16 138 and 123 us against 111, f32 174 and 168 against 166; 32-bit
    // ones, bf16 236 and 229 against 225, f32 284 and 278 against 277.
    if (!aligned) {
        constexpr int shared = 2 * WARPS * Stage<BITS, W, G, true>::BYTES;
        static_assert(shared + 2 * STRETCH <= 48 * 1024, "more needs to be asked for");
        return launch(h, adamw_kernel<BITS, W, G, true>, grid, 32 * WARPS, shared, st, a);
    }
    constexpr int shared = BITS == 8 ? 2 * WARPS * Stage<BITS, W, G, false>::BYTES : 0;
    return launch(h, adamw_kernel<BITS, W, G, false>, grid, 32 * WARPS, shared, st, a);
}

template <int BITS, class W>
int launch_step(co3_adamw* h, const StepArgs& a, bool aligned, int grid, cudaStream_t st) {
    if (h->grad_type == CO3_F32) return launch_step_of<BITS, W, F32>(h, a, aligned, grid, st);
    if (h->grad_type == CO3_BF16) return launch_step_of<BITS, W, Bf16>(h, a, aligned, grid, st);
    return launch_step_of<BITS, W, F16>(h, a, aligned, grid, st);
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
    // eps times a bias correction, which is sqrt(1 - beta2) at least, has to be a normal number of 32 bits where it is not 0, and no
    // denominator may pass 2^126, where the kernels' quotients end.
    if (!(cfg->eps == 0.0 || (cfg->eps * sqrt(1.0 - cfg->beta2) >= 0x1p-126 && cfg->eps <= 0x1p126))) return CO3_EINVAL;
    if (!(cfg->weight_decay >= 0.0 && (float)cfg->weight_decay < INFINITY)) return CO3_EINVAL;
    int64_t blocks = 0, elements = 0;
    for (int t = 0; t < n; ++t) {
        if (cfg->sizes[t] < 0 || cfg->sizes[t] > ((int64_t)1 << 40)) return CO3_EINVAL;
        if (cfg->decay && !(cfg->decay[t] >= 0.0f && cfg->decay[t] < INFINITY)) return CO3_EINVAL;
        blocks += (cfg->sizes[t] + BLK - 1) / BLK;
        elements += cfg->sizes[t];
        if (blocks > 0x7FFFFF00LL) return CO3_EINVAL;
    }
    co3_adamw* h = new (std::nothrow) co3_adamw();
    if (!h) return CO3_ENOMEM;
    memset(h, 0, sizeof(*h));
    h->n_tensors = n;
    h->weight_type = cfg->weight_type; h->grad_type = cfg->grad_type; h->copy_type = cfg->copy_type; h->state_bits = cfg->state_bits;
    h->beta1 = cfg->beta1; h->beta2 = cfg->beta2; h->eps = cfg->eps; h->seed = cfg->seed;
    h->n_blocks = blocks; h->n_elements = elements;
    h->per_cta = (blocks + NORM_CTAS - 1) / NORM_CTAS;
    if (h->per_cta < WARPS) h->per_cta = WARPS;
    h->norm_grid = (int)((blocks + h->per_cta - 1) / h->per_cta);
    if (h->norm_grid < 1) h->norm_grid = 1;
    h->n_slots = h->norm_grid + n;
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
        const size_t o_slots = part(8 * (size_t)h->n_slots);
        if (cudaMalloc(&h->slab, at) != cudaSuccess) { (void)cudaGetLastError(); h->slab = nullptr; rc = CO3_ENOMEM; }
        else {
            char* base = (char*)h->slab;
            h->sc = (Scalars*)(base + o_sc); h->tensors = (Tensor*)(base + o_t); h->owner = (int32_t*)(base + o_own);
            h->table = n > INLINE_TENSORS ? (Pointers*)(base + o_tab) : nullptr;
            h->slots = (double*)(base + o_slots);
            Scalars s;
            memset(&s, 0, sizeof(s));
            s.pow1 = s.pow2 = 1.0;
            next_scalars(s, h->beta1, h->beta2, h->seed);
            bool ok = cudaMemset(h->slots, 0, 8 * (size_t)h->n_slots) == cudaSuccess && cudaMemcpy(h->sc, &s, sizeof(s), cudaMemcpyHostToDevice) == cudaSuccess &&
                      cudaMemcpy(h->tensors, host, sizeof(Tensor) * (size_t)n, cudaMemcpyHostToDevice) == cudaSuccess;
            if (ok && blocks) {
                const int64_t grid = (blocks + 255) / 256;
                owner_kernel<<<(int)(grid < 4096 ? grid : 4096), 256>>>(h->tensors, n, h->owner, blocks);
                ok = cudaGetLastError() == cudaSuccess;
            }
            ok = ok && cudaStreamSynchronize(nullptr) == cudaSuccess;
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
    if (!(fabsf(grad_scale) < INFINITY) || isnan(max_norm)) return CO3_EINVAL;
    if (!on_device(h)) return CO3_EINVAL;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (!pointers_fine(h, grads, nullptr, nullptr)) return CO3_EINVAL;
    NormArgs a;
    a.table = nullptr;
    if (h->n_tensors <= INLINE_GRADS) {
        for (int t = 0; t < h->n_tensors; ++t) a.inline_grad[t] = grads[t];
    } else {
        a.table = h->table;
        const int rc = fill_table(h, grads, nullptr, nullptr, st);
        if (rc != CO3_OK) return rc;
    }
    a.tensors = h->tensors; a.owner = h->owner; a.n_blocks = h->n_blocks; a.per_cta = h->per_cta;
    a.n_tensors = h->n_tensors; a.n_slots = h->n_slots; a.grad_scale = grad_scale; a.max_norm = max_norm;
    a.slots = h->slots; a.tensor_norms = tensor_norms; a.info = info; a.sc = h->sc;
    const int threads = 32 * WARPS;
    if (h->grad_type == CO3_F32) return launch(h, norm_kernel<F32>, h->norm_grid, threads, 0, st, a);
    if (h->grad_type == CO3_BF16) return launch(h, norm_kernel<Bf16>, h->norm_grid, threads, 0, st, a);
    return launch(h, norm_kernel<F16>, h->norm_grid, threads, 0, st, a);
}

extern "C" int co3_adamw_step(co3_adamw* h, void* const* weights, const void* const* grads, void* const* copies, const co3_adamw_state* state,
                              double lr, const float* d_lr, const co3_grad_info* info, void* cuda_stream) {
    if (!h || !weights || !grads || !state || !(fabsf((float)lr) < INFINITY)) return CO3_EINVAL;
    if ((copies != nullptr) != (h->copy_type != CO3_NONE)) return CO3_EINVAL;
    if (((uintptr_t)info & 15) || ((uintptr_t)d_lr & 3)) return CO3_EINVAL;
    if (h->n_blocks) {
        if (!state->m || !state->v || (((uintptr_t)state->m | (uintptr_t)state->v) & 31)) return CO3_EINVAL;
        if (h->state_bits == 8 && (!state->m_exp || !state->v_exp)) return CO3_EINVAL;
    }
    if (!on_device(h)) return CO3_EINVAL;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (!pointers_fine(h, grads, weights, copies)) return CO3_EINVAL;
    StepArgs a;
    a.table = h->table;
    if (!h->table) {
        for (int t = 0; t < h->n_tensors; ++t) a.inline_ptr[t] = Pointers{grads[t], weights[t], copies ? copies[t] : nullptr};
    } else {
        const int rc = fill_table(h, grads, weights, copies, st);
        if (rc != CO3_OK) return rc;
    }
    a.tensors = h->tensors; a.owner = h->owner; a.n_blocks = h->n_blocks;
    a.m = state->m; a.v = state->v; a.m_exp = (uint8_t*)state->m_exp; a.v_exp = (uint8_t*)state->v_exp;
    a.info = info; a.d_lr = d_lr; a.sc = h->sc; a.beta1 = h->beta1; a.beta2 = h->beta2;
    a.b1 = (float)h->beta1; a.a1 = (float)(1.0 - h->beta1); a.b2 = (float)h->beta2; a.a2 = (float)(1.0 - h->beta2);
    auto twice = [](float x) { uint32_t u; memcpy(&u, &x, 4); return (unsigned long long)u << 32 | u; };
    a.b1_pair = twice(a.b1); a.a1_pair = twice(a.a1); a.b2_pair = twice(a.b2); a.a2_pair = twice(a.a2); a.minus_zero = twice(-0.0f);
    a.eps = (float)h->eps; a.lr = (float)lr; a.seed = h->seed; a.copy_type = h->copy_type;
    // block_whole takes roots of numbers below 2^-126 as 0.  Beside eps that is less than 2^-24 of the denominator if eps is above
    // 2^24 * 2^-63 / sqrt(1 - beta2) (6e-11 for beta2 = 0.999); a smaller eps takes the general way.
    // The scale of 8-bit moments (2^-117 at least) times beta1 has to stay a normal number.
    // What the general way costs where every block takes it (67M elements, eps = 1e-15 against 1e-8): 8-bit moments, bf16 309 us against
    // 111, f32 247 against 166; 32-bit ones, bf16 286 against 225, f32 293 against 277.
    a.fast = h->eps * sqrt(1.0 - h->beta2) >= 0x1p-39 && (h->state_bits == 32 || h->beta1 == 0.0 || h->beta1 >= 0x1p-9);
    // Blocks of one thread block.  32-bit moments: one warp takes as many as leave every place for a thread block four of them one
    // after the other, so that the SMs end together, and at most 4 (2^28 f32: 1, 2, 4, 8, 16 take 1214, 1115, 1097, 1114, 1125 us).
    // 8-bit moments: whole rounds over all places, of at most 128 blocks (11.2M f32: 24 blocks in four and a bit rounds 39.4 us, 99
    // in one 36.9; 2^28: 8, 16, 32, 64, 128 blocks 1493, 1186, 1083, 1044, 1023 us).  Their exponents are bytes side by side, and
    // a line of them that thread blocks on both dies write has each of them wait for the other.
    const int64_t places = (int64_t)h->num_sms * (h->state_bits == 8 ? STEP_CTAS<8> : STEP_CTAS<32>);
    if (h->state_bits == 8) {
        const int64_t rounds = (h->n_blocks + places * STRETCH - 1) / (places * STRETCH);
        const int64_t each = rounds ? (h->n_blocks + places * rounds - 1) / (places * rounds) : 0;
        a.stretch = (int)(each < WARPS ? WARPS : each);
    } else {
        const int64_t per_warp = h->n_blocks / (places * WARPS * 4);
        a.stretch = (int)(WARPS * (per_warp < 1 ? 1 : per_warp > 4 ? 4 : per_warp));
    }
    const int grid = h->n_blocks ? (int)((h->n_blocks + a.stretch - 1) / a.stretch) : 1;
    const bool w16 = h->weight_type == CO3_BF16;
    uintptr_t weight_bits = 0, grad_bits = 0, copy_bits = 0;
    for (int t = 0; t < h->n_tensors; ++t)
        if (h->sizes[t] >= BLK) {
            weight_bits |= (uintptr_t)weights[t];
            grad_bits |= (uintptr_t)grads[t];
            if (copies) copy_bits |= (uintptr_t)copies[t];
        }
    const uintptr_t grad_align = h->state_bits == 32 && h->grad_type == CO3_F32 ? F32::ALIGN : 15;    // 8-bit: copied 16 bytes at a time
    const bool aligned = !(weight_bits & (w16 ? Bf16::ALIGN : F32::ALIGN)) && !(grad_bits & grad_align) && !(copy_bits & 15);
    if (h->state_bits == 32) return w16 ? launch_step<32, Bf16>(h, a, aligned, grid, st) : launch_step<32, F32>(h, a, aligned, grid, st);
    return w16 ? launch_step<8, Bf16>(h, a, aligned, grid, st) : launch_step<8, F32>(h, a, aligned, grid, st);
}

extern "C" int co3_adamw_values(co3_adamw* h, const co3_adamw_state* state, void* m_values, void* v_values, int32_t value_type, void* cuda_stream) {
    if (!h || !state || h->state_bits != 8 || (value_type != CO3_F32 && value_type != CO3_BF16)) return CO3_EINVAL;
    if (!on_device(h)) return CO3_EINVAL;
    if (!h->n_blocks) return CO3_OK;
    if (!state->m || !state->v || !state->m_exp || !state->v_exp || (((uintptr_t)state->m | (uintptr_t)state->v) & 31)) return CO3_EINVAL;
    if (!m_values || !v_values || (((uintptr_t)m_values | (uintptr_t)v_values) & 31)) return CO3_EINVAL;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int grid = (int)((h->n_blocks + 2 * WARPS - 1) / (2 * WARPS));
    const uint8_t *m = (const uint8_t*)state->m, *v = (const uint8_t*)state->v;
    if (value_type == CO3_F32)
        return launch(h, values_kernel<F32>, grid, 32 * WARPS, 0, st, m, v, (const uint8_t*)state->m_exp, (const uint8_t*)state->v_exp, h->n_blocks,
                      (float*)m_values, (float*)v_values);
    return launch(h, values_kernel<Bf16>, grid, 32 * WARPS, 0, st, m, v, (const uint8_t*)state->m_exp, (const uint8_t*)state->v_exp, h->n_blocks,
                  (__nv_bfloat16*)m_values, (__nv_bfloat16*)v_values);
}

extern "C" int co3_adamw_status(co3_adamw* h, uint32_t* flags, uint64_t* skipped_elements, uint64_t* skipped_steps, int32_t clear) {
    if (!h || !on_device(h)) return CO3_EINVAL;
    Scalars s;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&s, h->sc, sizeof(s), cudaMemcpyDeviceToHost) != cudaSuccess) { (void)cudaGetLastError(); return CO3_ECUDA; }
    if (flags) *flags = s.flags;
    if (skipped_elements) *skipped_elements = s.skipped_elements;
    if (skipped_steps) *skipped_steps = s.skipped_steps;
    if (clear) {                              // these three, side by side, and nothing that a step of another thread may be changing
        constexpr size_t first = offsetof(Scalars, flags), past = offsetof(Scalars, skipped_steps) + sizeof(s.skipped_steps);
        if (cudaMemset((char*)h->sc + first, 0, past - first) != cudaSuccess || cudaStreamSynchronize(nullptr) != cudaSuccess) {
            (void)cudaGetLastError();
            return CO3_ECUDA;
        }
    }
    return CO3_OK;
}

extern "C" int co3_adamw_steps_export(co3_adamw* h, int64_t* steps) {
    if (!h || !steps || !on_device(h)) return CO3_EINVAL;
    Scalars s;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&s, h->sc, sizeof(s), cudaMemcpyDeviceToHost) != cudaSuccess) { (void)cudaGetLastError(); return CO3_ECUDA; }
    *steps = s.steps;
    return CO3_OK;
}

// beta^steps as the steps themselves would have left it, one product after the other, to the bit; after very many (0.1 s of them) the
// power.  A product that changes nothing is the last that counts: 0, or a subnormal number that rounding brings back to itself
// (2.5e-323 for 0.9), on which products are slow (2^26 steps with 0.9 and 0.999 took 5.7 s until this was looked for, 2 ms since).
static double power_of_steps(double beta, int64_t steps) {
    if (steps > (int64_t)1 << 26) return pow(beta, (double)steps);
    double p = 1.0;
    for (int64_t i = 0; i < steps; ++i) {
        const double q = p * beta;
        if (q == p) break;
        p = q;
    }
    return p;
}

extern "C" int co3_adamw_steps_import(co3_adamw* h, int64_t steps) {
    if (!h || steps < 0 || !on_device(h)) return CO3_EINVAL;
    if (cudaDeviceSynchronize() != cudaSuccess) { (void)cudaGetLastError(); return CO3_ECUDA; }
    Scalars s;
    s.steps = steps;
    s.pow1 = power_of_steps(h->beta1, steps);
    s.pow2 = power_of_steps(h->beta2, steps);
    next_scalars(s, h->beta1, h->beta2, h->seed);
    if (!to_device(h->sc, &s, offsetof(Scalars, key) + sizeof(s.key))) { (void)cudaGetLastError(); return CO3_ECUDA; }
    return CO3_OK;
}

extern "C" int64_t co3_adamw_launch_count(const co3_adamw* h) { return h ? h->launches : 0; }
