// Layer norm forward and backward, with the reduction of the weight's and the bias' gradient per user (co3_layernorm_*).
//
// A row is held in the registers of TPR threads, E elements each, so that one read of it serves mean, variance and result: two
// passes over registers, and the variance is that of differences.  Thread blocks stay and take row after row.  What bounds the kernels is memory,
// and what they need for it is bytes on their way: each thread copies its elements of the rows to come into shared memory of its own ahead
// of time, which costs no registers and, since nobody else reads them, no barrier.
#include "co3_ops.cuh"

namespace {

constexpr int LN_MAX_DIM = 16384;

struct LnForward {
    const void* x; const void* weight; const void* bias; void* y;
    float *mean, *rstd;
    int64_t xu, xt, yu, yt;                   // strides
    uint32_t tokens, users, step_users, step_tokens;      // of all groups together, from one row of a group to its next
    int dim, weight_type;
    float inv_dim, eps;
};
struct LnBackward {
    const void* dy; const void* x; const void* weight; void* dx;
    const float *mean, *rstd;
    int64_t gu, gt, xu, xt, du, dt;           // strides of dy, x, dx
    uint32_t tokens;
    int dim, weight_type, slices;             // thread blocks of a user
    float inv_dim;
    float* part;                              // [users][slices][2][dim]
    co3_param_grad dweight, dbias;            // data null where not wanted
};

// Sum over the TPR threads of a row of one value each, or of two; `turn` counts the reductions of these threads, `sh` is theirs alone.
__device__ __forceinline__ float over_warp(float x) { return warp_sum_f32(x); }
__device__ __forceinline__ Two over_warp(Two x) {
    float a, b;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        x.get(a, b);
        x = x + Two(__shfl_xor_sync(0xffffffffu, a, o), __shfl_xor_sync(0xffffffffu, b, o));
    }
    return x;
}
template <int TPR, class V> struct RowSum {
    static constexpr int W = TPR / 32, GROUPS_MOST = TPR >= 256 ? 1 : 8 / W;
    static constexpr int PITCH = (W * (int)sizeof(V) + 15) / 16 * 16 / (int)sizeof(V);        // a group's warps begin at 16 bytes
    V sums[2][GROUPS_MOST * PITCH];           // two: one barrier a reduction
};
template <int TPR, class V> __device__ __forceinline__ V row_sum(V x, RowSum<TPR, V>& sh, int& turn) {
    constexpr int W = TPR / 32;
    x = over_warp(x);
    if constexpr (W == 1) return x;
    else {
        const int group = threadIdx.x / TPR, warp = threadIdx.x % TPR / 32, lane = threadIdx.x & 31;
        V* const s = sh.sums[turn & 1] + group * RowSum<TPR, V>::PITCH;
        ++turn;
        if (lane == 0) s[warp] = x;
        asm volatile("bar.sync %0, %1;" :: "r"(1 + group), "n"(TPR) : "memory");
        if constexpr (W > 8) {
            V t = s[lane % W];
            if (W < 32 && lane >= W) { if constexpr (sizeof(V) == 4) t = 0.0f; else t = Two(0.0f, 0.0f); }
            return over_warp(t);
        } else {                              // 16 bytes at a time
            constexpr int EACH = 16 / sizeof(V);
            union { uint4 u[(W + EACH - 1) / EACH]; unsigned long long pair[(W + EACH - 1) / EACH * 2]; float one[(W + EACH - 1) / EACH * 4]; } all;
#pragma unroll
            for (int i = 0; i < (W + EACH - 1) / EACH; ++i) all.u[i] = ((const uint4*)s)[i];
            if constexpr (sizeof(V) == 4) {
                float t = all.one[0];
#pragma unroll
                for (int w = 1; w < W; ++w) t += all.one[w];
                return t;
            } else {
                Two t, o;
                t.v = all.pair[0];
#pragma unroll
                for (int w = 1; w < W; ++w) { o.v = all.pair[w]; t = t + o; }
                return t;
            }
        }
    }
}

// How rows are read: in whole 16 bytes; in words (f32 rows that begin anywhere, or of an odd length); element by element (16 bits, likewise: 65536 x
// 1001 bf16 78 us forward and 124 backward, x 1000 in whole 16 bytes 48 and 83).
enum Take { WHOLE, WORDS, SINGLES };

// The elements that a thread holds of a row: E / V pieces of V neighbours, piece c at column (c TPR + t) V.  AHEAD: rows that are on
// their way into shared memory while one is worked on (none element by element, where there is no such copy).
template <class T, int TAKE, int TPR, int E> struct Held {
    typedef typename T::type type;
    static constexpr int V = TAKE == WHOLE ? T::EACH : 1, N = E / V, BYTES = V * sizeof(type);
    static constexpr int THREADS = TPR >= 256 ? TPR : TPR == 32 && E >= 24 ? 128 : 256 / TPR * TPR, GROUPS = THREADS / TPR;
    static constexpr int ROW = N * THREADS * BYTES;       // of a thread block, one row a group
    static constexpr bool ASYNC = TAKE != SINGLES;
    static_assert(E % V == 0, "whole pieces");
    static __device__ __forceinline__ int column(int t, int c) { return (c * TPR + t) * V; }
    // Begins to copy the thread's elements into its places of the slot, or reads them.
    static __device__ __forceinline__ void send(uint8_t* slot, const type* row, int t, int dim) {
        if constexpr (TAKE == SINGLES) return;
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(slot) + threadIdx.x * BYTES;
#pragma unroll
        for (int c = 0; c < N; ++c)
            if (column(t, c) < dim) {
                if constexpr (TAKE == WHOLE) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + c * THREADS * BYTES), "l"(row + column(t, c)) : "memory");
                else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" :: "r"(to + c * THREADS * BYTES), "l"(row + column(t, c)) : "memory");
            }
    }
    // Pair j of the thread: elements 2j and 2j + 1, 0 beyond the row.
    static __device__ __forceinline__ void take(const uint8_t* slot, const type* row, int t, int dim, Two* x) {
        float f[E];
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const int at = column(t, c);
            if constexpr (TAKE == WHOLE) {
                const uint4 u = at < dim ? *(const uint4*)(slot + (c * THREADS + threadIdx.x) * BYTES) : make_uint4(0, 0, 0, 0);
                T::unpack(u, f + c * V);
            } else if constexpr (TAKE == WORDS) f[c] = at < dim ? *(const float*)(slot + (c * THREADS + threadIdx.x) * BYTES) : 0.0f;
            else f[c] = at < dim ? T::get(row[at]) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < E / 2; ++j) x[j] = Two(f[2 * j], f[2 * j + 1]);
    }
    static __device__ __forceinline__ void beyond(int t, int dim, float otherwise, Two* x) {
#pragma unroll
        for (int j = 0; j < E / 2; ++j) {
            float a, b;
            x[j].get(a, b);
            const bool in_a = column(t, 2 * j / V) + 2 * j % V < dim, in_b = column(t, (2 * j + 1) / V) + (2 * j + 1) % V < dim;
            x[j] = Two(in_a ? a : otherwise, in_b ? b : otherwise);
        }
    }
    static __device__ __forceinline__ void store(type* row, int t, int dim, const Two* x) {
        float f[E];
#pragma unroll
        for (int j = 0; j < E / 2; ++j) x[j].get(f[2 * j], f[2 * j + 1]);
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const int at = column(t, c);
            if (at < dim) {
                if constexpr (TAKE == WHOLE) *(uint4*)(row + at) = T::pack(f + c * V);
                else row[at] = T::put(f[c]);
            }
        }
    }
    // per-column values in 32 bits
    static __device__ __forceinline__ void param(const void* p, int type, float otherwise, int t, int dim, Two* w) {
        float f[E];
#pragma unroll
        for (int c = 0; c < N; ++c)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int at = column(t, c) + k;
                f[c * V + k] = at < dim ? (p ? load_as_f32(p, type, at) : otherwise) : 0.0f;
            }
#pragma unroll
        for (int j = 0; j < E / 2; ++j) w[j] = Two(f[2 * j], f[2 * j + 1]);
    }
};
// Sum of the products of pairs (of their sums, if `y` is null) in two chains.
template <int P> __device__ __forceinline__ float sum_of(const Two* x, const Two* y) {
    Two s[2] = {Two(0.0f, 0.0f), Two(0.0f, 0.0f)};
#pragma unroll
    for (int j = 0; j < P; ++j) s[j & 1] = y ? fma(x[j], y[j], s[j & 1]) : s[j & 1] + x[j];
    return (s[0] + s[1]).sum();
}
__device__ __forceinline__ void sent() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void arrived() { asm volatile("cp.async.wait_group %0;" :: "n"(LEFT) : "memory"); }

// Slots of shared memory for a thread block's rows of `arrays` arrays: those ahead and the one that is being read, in 192 KB at most.
template <class H> __host__ __device__ constexpr int ln_slots(int arrays) {
    const int most = sizeof(typename H::type) == 2 ? 4 : 3, fit = 192 * 1024 / (arrays * H::ROW);
    return H::ASYNC ? (fit < 1 ? 1 : fit < most ? fit : most) : 1;
}

// 65536 x 4096 bf16: 180 us, 6.0 TB/s (5.4 where the same output is written again at once); 65536 x 768 37 us, 5.4 TB/s; issue slots 64 % used.
template <class T, int TAKE, int TPR, int E>
__global__ void __launch_bounds__(Held<T, TAKE, TPR, E>::THREADS) ln_forward_kernel(const __grid_constant__ LnForward a) {
    typedef Held<T, TAKE, TPR, E> H;
    typedef typename T::type type;
    constexpr int SLOTS = ln_slots<H>(1);
    extern __shared__ uint4 room[];
    __shared__ __align__(16) RowSum<TPR, float> sh;
    int turn = 0;
    const int t = threadIdx.x % TPR;
    let_next_start();
    wait_for_previous();
    constexpr int P = E / 2;
    Two w[P], b[P];
    H::param(a.weight, a.weight_type, 1.0f, t, a.dim, w);
    H::param(a.bias, a.weight_type, 0.0f, t, a.dim, b);
    auto slot = [&](int i) { return (uint8_t*)room + i * H::ROW; };
    // rows of this group: the one that is worked on and the one that is sent for, as user and token, without a division for each
    struct At { uint32_t user, token; };
    auto next = [&](At& r) {
        r.user += a.step_users;
        r.token += a.step_tokens;
        if (r.token >= a.tokens) { r.token -= a.tokens; ++r.user; }
    };
    const uint32_t first = blockIdx.x * H::GROUPS + threadIdx.x / TPR;
    At at = {first / a.tokens, first % a.tokens}, coming = at;
    auto row_of = [&](const At& r) { return (const type*)a.x + r.user * a.xu + r.token * a.xt; };
    auto send = [&](int i) {
        if (coming.user < a.users) H::send(slot(i), row_of(coming), t, a.dim);
        sent();
        next(coming);
    };
#pragma unroll
    for (int i = 0; i < SLOTS - 1; ++i) send(i);
    for (int i = 0; at.user < a.users; i = i + 1 == SLOTS ? 0 : i + 1, next(at)) {
        Two x[P];
        if (SLOTS == 1) send(0);
        arrived<SLOTS >= 2 ? SLOTS - 2 : 0>();
        H::take(slot(i), row_of(at), t, a.dim, x);
        if (SLOTS > 1) send(i ? i - 1 : SLOTS - 1);
        const float mean = row_sum<TPR>(sum_of<P>(x, nullptr), sh, turn) * a.inv_dim;
        if (a.dim < TPR * E) H::beyond(t, a.dim, mean, x);            // their differences are 0
#pragma unroll
        for (int j = 0; j < P; ++j) x[j] = x[j] + Two(-mean, -mean);
        const float rstd = rsqrtf(fmaf(row_sum<TPR>(sum_of<P>(x, x), sh, turn), a.inv_dim, a.eps));       // to two units in the last place
#pragma unroll
        for (int j = 0; j < P; ++j) x[j] = fma(x[j] * Two(rstd, rstd), w[j], b[j]);
        H::store((type*)a.y + at.user * a.yu + at.token * a.yt, t, a.dim, x);
        if (t == 0) {
            const int64_t r = (int64_t)at.user * a.tokens + at.token;
            a.mean[r] = mean;
            a.rstd[r] = rstd;
        }
    }
}

// blockIdx.x: slice of the user blockIdx.y's rows.  The sums for weight and bias stay in registers over all rows of a slice; as many slices as the
// device holds at a time, so that the order of sums depends on sizes and types alone.  65536 x 4096 bf16: 300 us, 5.3 TB/s; f32 rows of 16 KB 132 us for
// 16384, 6.1 TB/s; 65536 x 768 bf16 62 us, 4.9 TB/s: the shorter the rows, the more of the time goes to the two sums over each.
template <class T, int TAKE, int TPR, int E>
__global__ void __launch_bounds__(Held<T, TAKE, TPR, E>::THREADS) ln_backward_kernel(const __grid_constant__ LnBackward a) {
    typedef Held<T, TAKE, TPR, E> H;
    typedef typename T::type type;
    constexpr int SLOTS = ln_slots<H>(2);
    extern __shared__ uint4 room[];
    __shared__ __align__(16) RowSum<TPR, Two> sh;
    int turn = 0;
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const uint32_t user = blockIdx.y;
    let_next_start();
    wait_for_previous();
    constexpr int P = E / 2;
    Two w[P], dw2[P], db2[P];
    H::param(a.weight, a.weight_type, 1.0f, t, a.dim, w);
#pragma unroll
    for (int j = 0; j < P; ++j) dw2[j] = db2[j] = Two(0.0f, 0.0f);
    const type* gy = (const type*)a.dy + user * a.gu;
    const type* xs = (const type*)a.x + user * a.xu;
    type* dx = (type*)a.dx + user * a.du;
    const float *means = a.mean + (int64_t)user * a.tokens, *rstds = a.rstd + (int64_t)user * a.tokens;
    const uint32_t step = a.slices * H::GROUPS;
    auto slot = [&](int i) { return (uint8_t*)room + i * 2 * H::ROW; };
    uint32_t r = blockIdx.x * H::GROUPS + group;
    uint64_t coming = r;
    auto send = [&](int i) {
        if (coming < a.tokens) {
            H::send(slot(i), gy + coming * a.gt, t, a.dim);
            H::send(slot(i) + H::ROW, xs + coming * a.xt, t, a.dim);
        }
        sent();
        coming += step;
    };
#pragma unroll
    for (int i = 0; i < SLOTS - 1; ++i) send(i);
    float next_mean = r < a.tokens ? means[r] : 0.0f, next_rstd = r < a.tokens ? rstds[r] : 0.0f;
    for (int i = 0; r < a.tokens; i = i + 1 == SLOTS ? 0 : i + 1) {
        Two g[P], x[P];
        if (SLOTS == 1) send(0);
        arrived<SLOTS >= 2 ? SLOTS - 2 : 0>();
        H::take(slot(i), gy + r * a.gt, t, a.dim, g);
        H::take(slot(i) + H::ROW, xs + r * a.xt, t, a.dim, x);
        if (SLOTS > 1) send(i ? i - 1 : SLOTS - 1);
        const float mean = next_mean, rstd = next_rstd;
        const bool more = a.tokens - r > step;
        if (more) { next_mean = means[r + step]; next_rstd = rstds[r + step]; }
#pragma unroll
        for (int j = 0; j < P; ++j) {
            x[j] = (x[j] + Two(-mean, -mean)) * Two(rstd, rstd);
            dw2[j] = fma(g[j], x[j], dw2[j]);
            db2[j] = db2[j] + g[j];
            g[j] = g[j] * w[j];               // 0 beyond the row
        }
        if (a.dx) {
            float c1, c2;
            (row_sum<TPR>(Two(sum_of<P>(g, nullptr), sum_of<P>(g, x)), sh, turn) * Two(-a.inv_dim, -a.inv_dim)).get(c1, c2);
#pragma unroll
            for (int j = 0; j < P; ++j) g[j] = (g[j] + fma(x[j], Two(c2, c2), Two(c1, c1))) * Two(rstd, rstd);
            H::store(dx + r * a.dt, t, a.dim, g);
        }
        if (!more) break;
        r += step;
    }
    if (!a.dweight.data && !a.dbias.data) return;
    float dw[E], db[E];
#pragma unroll
    for (int j = 0; j < P; ++j) { dw2[j].get(dw[2 * j], dw[2 * j + 1]); db2[j].get(db[2 * j], db[2 * j + 1]); }
    if (H::GROUPS > 1) {                      // the groups' sums, in their order
        __shared__ float sums[2][H::GROUPS > 1 ? TPR * E : 1];
        for (int k = 0; k < H::GROUPS; ++k) {
            if (group == k)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int at = i * TPR + t;
                    sums[0][at] = dw[i] = k ? sums[0][at] + dw[i] : dw[i];
                    sums[1][at] = db[i] = k ? sums[1][at] + db[i] : db[i];
                }
            __syncthreads();
        }
        if (group != H::GROUPS - 1) return;
    }
    float* part = a.part + ((int64_t)user * a.slices + blockIdx.x) * 2 * a.dim;
#pragma unroll
    for (int c = 0; c < H::N; ++c)
#pragma unroll
        for (int k = 0; k < H::V; ++k) {
            const int at = H::column(t, c) + k, i = c * H::V + k;
            if (at >= a.dim) continue;
            if (a.slices == 1) {
                if (a.dweight.data) store_as(a.dweight.data, a.dweight.type, user * a.dweight.user_stride + at, dw[i], a.dweight.accumulate);
                if (a.dbias.data) store_as(a.dbias.data, a.dbias.type, user * a.dbias.user_stride + at, db[i], a.dbias.accumulate);
            } else {
                part[at] = dw[i];
                part[a.dim + at] = db[i];
            }
        }
}

// The slices' sums: 32 columns, eight stretches of the slices, then those in their order.
__global__ void __launch_bounds__(256) ln_join_kernel(const float* part, int slices, int dim, co3_param_grad dweight, co3_param_grad dbias) {
    __shared__ float sh[8][32];
    const int lane = threadIdx.x & 31, g = threadIdx.x >> 5, column = blockIdx.x * 32 + lane;
    const int64_t user = blockIdx.y;
    let_next_start();
    wait_for_previous();
    float s = 0.0f;
    if (column < 2 * dim) {
        const float* p = part + user * slices * 2 * dim + column;
        const int each = (slices + 7) / 8, end = (g + 1) * each < slices ? (g + 1) * each : slices;
#pragma unroll 8
        for (int i = g * each; i < end; ++i) s += __ldcg(p + (int64_t)i * 2 * dim);
    }
    sh[g][lane] = s;
    __syncthreads();
    if (g || column >= 2 * dim) return;
    for (int k = 1; k < 8; ++k) s += sh[k][lane];
    const co3_param_grad& to = column < dim ? dweight : dbias;
    if (to.data) store_as(to.data, to.type, user * to.user_stride + (column < dim ? column : column - dim), s, to.accumulate);
}

// How a row of up to `dim` elements is held: threads, and elements of each.  Few threads have few of a reduction's steps for each element, and more
// elements in flight each; many leave more registers to the backward pass' sums.  Times in us for 16 elements a thread and for 8, forward and
// backward: 65536 x 768 bf16 (24 elements) 37 and 60, 63 and 107; 32768 x 2048 bf16 52 and 78, 82 and 103; f32 99 and 98, 140 and 169; 16384 x
// 4096 f32 100 and 87, 141 and 132; 32768 x 1001 f32 word by word 57 and 58, 110 and 93.
struct LnShape { int dim, tpr, e; };
template <class T, int TAKE> constexpr LnShape LN_SHAPES[8] = {
    {256, 32, 8}, {512, 32, 16}, {768, 32, 24}, {1024, 64, 16}, {2048, 128, 16}, {4096, 256, 16}, {8192, 512, 16}, {LN_MAX_DIM, 1024, 16}};
template <> constexpr LnShape LN_SHAPES<OF32, WHOLE>[8] = {
    {256, 32, 8}, {512, 32, 16}, {768, 32, 24}, {1024, 64, 16}, {2048, 128, 16}, {4096, 512, 8}, {8192, 512, 16}, {LN_MAX_DIM, 1024, 16}};
template <> constexpr LnShape LN_SHAPES<OF32, WORDS>[8] = {
    {256, 32, 8}, {512, 64, 8}, {768, 96, 8}, {1024, 128, 8}, {2048, 256, 8}, {4096, 512, 8}, {8192, 512, 16}, {LN_MAX_DIM, 1024, 16}};

}  // namespace

struct co3_layernorm {
    int64_t dim, launches;
    int users, device, sms;
    int places[3][3][2];                      // thread blocks that the device holds at a time, by type, way of reading, and direction
    double eps;
    float* part;
};

namespace {

template <class H> int64_t ln_slices(const co3_layernorm* h, int64_t tokens, int places) {
    const int64_t each = places / h->users, most = (tokens + 2 * H::GROUPS - 1) / (2 * H::GROUPS), n = each < most ? each : most;
    return n < 1 ? 1 : n;
}

// What is done with the kernels of a shape.
struct LnPrepare {                            // asks for their shared memory, and for how many thread blocks there is room
    co3_layernorm* h;
    int64_t scratch;                          // numbers
    template <class T, int TAKE, int TPR, int E> int run(int type) {
        typedef Held<T, TAKE, TPR, E> H;
        for (int back = 0; back < 2; ++back) {
            const void* kernel = back ? (const void*)ln_backward_kernel<T, TAKE, TPR, E> : (const void*)ln_forward_kernel<T, TAKE, TPR, E>;
            const int bytes = H::ASYNC ? ln_slots<H>(1 + back) * (1 + back) * H::ROW : 0;
            int n = 0;
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess ||
                cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, H::THREADS, bytes) != cudaSuccess || n < 1) return CO3_ECUDA;
            h->places[type][TAKE][back] = n * h->sms;
            const int64_t slices = ln_slices<H>(h, OPS_MAX_ROWS, n * h->sms);
            if (back && slices > 1 && h->users * slices * 2 * h->dim > scratch) scratch = h->users * slices * 2 * h->dim;
        }
        return CO3_OK;
    }
};
struct LnRunForward {
    co3_layernorm* h;
    LnForward a;
    cudaStream_t st;
    template <class T, int TAKE, int TPR, int E> int run(int type) {
        typedef Held<T, TAKE, TPR, E> H;
        const int64_t need = ((int64_t)a.tokens * a.users + H::GROUPS - 1) / H::GROUPS, places = h->places[type][TAKE][0];
        const uint32_t grid = (uint32_t)(need < places ? need : places);
        a.step_users = grid * H::GROUPS / a.tokens;
        a.step_tokens = grid * H::GROUPS % a.tokens;
        return launch_early(&h->launches, ln_forward_kernel<T, TAKE, TPR, E>, dim3(grid), H::THREADS,
                            H::ASYNC ? ln_slots<H>(1) * H::ROW : 0, 1, st, a);
    }
};
struct LnRunBackward {
    co3_layernorm* h;
    LnBackward a;
    cudaStream_t st;
    template <class T, int TAKE, int TPR, int E> int run(int type) {
        typedef Held<T, TAKE, TPR, E> H;
        a.slices = (int)ln_slices<H>(h, a.tokens, h->places[type][TAKE][1]);
        const int rc = launch_early(&h->launches, ln_backward_kernel<T, TAKE, TPR, E>, dim3((unsigned)a.slices, (unsigned)h->users), H::THREADS,
                                    H::ASYNC ? ln_slots<H>(2) * 2 * H::ROW : 0, 1, st, a);
        if (rc != CO3_OK || a.slices == 1 || (!a.dweight.data && !a.dbias.data)) return rc;
        return launch_early(&h->launches, ln_join_kernel, dim3((unsigned)((2 * h->dim + 31) / 32), (unsigned)h->users), 256, 0, 1, st, (const float*)h->part,
                            a.slices, a.dim, a.dweight, a.dbias);
    }
};
template <class T, int TAKE, int I, class W> int ln_with_shape(int64_t dim, int type, W& what) {
    constexpr LnShape S = LN_SHAPES<T, TAKE>[I];
    if (dim <= S.dim) return what.template run<T, TAKE, S.tpr, S.e>(type);
    if constexpr (I < 7) return ln_with_shape<T, TAKE, I + 1>(dim, type, what);
    else return CO3_EINVAL;
}
template <class W> int ln_with(int64_t dim, int type, int take, W& what) {
    if (type == CO3_F32) return take == WHOLE ? ln_with_shape<OF32, WHOLE, 0>(dim, type, what) : ln_with_shape<OF32, WORDS, 0>(dim, type, what);
    if (type == CO3_BF16) return take == WHOLE ? ln_with_shape<OBf16, WHOLE, 0>(dim, type, what) : ln_with_shape<OBf16, SINGLES, 0>(dim, type, what);
    return take == WHOLE ? ln_with_shape<OF16, WHOLE, 0>(dim, type, what) : ln_with_shape<OF16, SINGLES, 0>(dim, type, what);
}
// WHOLE, or what the type has for rows that begin anywhere.
int ln_take(int type, bool whole) { return whole ? WHOLE : type == CO3_F32 ? WORDS : SINGLES; }

}  // namespace

extern "C" void co3_layernorm_destroy(co3_layernorm* h) {
    if (!h) return;
    if (h->part) cudaFree(h->part);
    delete h;
}

extern "C" int co3_layernorm_create(co3_layernorm** out, int64_t dim, int32_t n_users, double eps) {
    if (!out) return CO3_EINVAL;
    *out = nullptr;
    if (dim < 1 || dim > LN_MAX_DIM || n_users < 1 || n_users > OPS_MAX_USERS) return CO3_EINVAL;
    if (!(eps >= 0.0 && (float)eps < INFINITY)) return CO3_EINVAL;
    co3_layernorm* h = new (std::nothrow) co3_layernorm();
    if (!h) return CO3_ENOMEM;
    memset(h, 0, sizeof(*h));
    h->dim = dim; h->users = n_users; h->eps = eps;
    int rc = CO3_OK;
    if (cudaGetDevice(&h->device) != cudaSuccess || cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, h->device) != cudaSuccess || h->sms < 1) rc = CO3_ECUDA;
    if (rc == CO3_OK) {
        LnPrepare p = {h, 0};
        for (int type = CO3_F32; type <= CO3_F16 && rc == CO3_OK; ++type)
            for (int whole = 0; whole < 2 && rc == CO3_OK; ++whole) rc = ln_with(dim, type, ln_take(type, whole != 0), p);
        // sums of the thread blocks of users whose rows go to more than one
        if (rc == CO3_OK && p.scratch && cudaMalloc(&h->part, (size_t)p.scratch * 4) != cudaSuccess) { h->part = nullptr; rc = CO3_ENOMEM; }
    }
    if (rc != CO3_OK) { (void)cudaGetLastError(); co3_layernorm_destroy(h); return rc; }
    *out = h;
    return CO3_OK;
}

extern "C" int co3_layernorm_forward(co3_layernorm* h, const co3_array* x, const void* weight, const void* bias, int32_t weight_type, int64_t n_tokens,
                                     const co3_array* y, float* mean, float* rstd, void* cuda_stream) {
    if (!h || n_tokens < 0 || n_tokens > OPS_MAX_ROWS / h->users) return CO3_EINVAL;
    if (!array_fine(x, h->users, n_tokens, h->dim, false) || !array_fine(y, h->users, n_tokens, h->dim, true) || x->type != y->type) return CO3_EINVAL;
    if ((weight || bias) && (!type_known(weight_type) || !aligned_to(weight, type_width(weight_type)) || !aligned_to(bias, type_width(weight_type)))) return CO3_EINVAL;
    if (!device_is(h->device)) return CO3_EINVAL;
    if (n_tokens == 0) return CO3_OK;
    if (!mean || !rstd || !aligned_to(mean, 4) || !aligned_to(rstd, 4)) return CO3_EINVAL;
    LnForward a;
    a.x = x->data; a.weight = weight; a.bias = bias; a.y = y->data; a.mean = mean; a.rstd = rstd;
    a.xu = x->user_stride; a.xt = x->token_stride; a.yu = y->user_stride; a.yt = y->token_stride;
    a.tokens = (uint32_t)n_tokens; a.users = (uint32_t)h->users;
    a.dim = (int)h->dim; a.weight_type = weight_type; a.inv_dim = (float)(1.0 / (double)h->dim); a.eps = (float)h->eps;
    const bool whole = h->dim * type_width(x->type) % 16 == 0 && rows_aligned(x, h->users, n_tokens) && rows_aligned(y, h->users, n_tokens);
    LnRunForward run = {h, a, (cudaStream_t)cuda_stream};
    return ln_with(h->dim, x->type, ln_take(x->type, whole), run);
}

extern "C" int co3_layernorm_backward(co3_layernorm* h, const co3_array* dy, const co3_array* x, const void* weight, int32_t weight_type, const float* mean,
                                      const float* rstd, int64_t n_tokens, const co3_array* dx, const co3_param_grad* dweight,
                                      const co3_param_grad* dbias, void* cuda_stream) {
    if (!h || n_tokens < 0 || n_tokens > OPS_MAX_ROWS / h->users) return CO3_EINVAL;
    if (!array_fine(x, h->users, n_tokens, h->dim, false) || !array_fine(dy, h->users, n_tokens, h->dim, false) || x->type != dy->type) return CO3_EINVAL;
    if (dx && (!array_fine(dx, h->users, n_tokens, h->dim, true) || dx->type != x->type)) return CO3_EINVAL;
    if (weight && (!type_known(weight_type) || !aligned_to(weight, type_width(weight_type)))) return CO3_EINVAL;
    if ((dweight && !grad_fine(dweight, h->users, h->dim)) || (dbias && !grad_fine(dbias, h->users, h->dim))) return CO3_EINVAL;
    if (!device_is(h->device)) return CO3_EINVAL;
    if (n_tokens && (!mean || !rstd || !aligned_to(mean, 4) || !aligned_to(rstd, 4))) return CO3_EINVAL;
    if (!dx && !dweight && !dbias) return CO3_OK;
    LnBackward a;
    memset(&a, 0, sizeof(a));
    a.dy = dy->data; a.x = x->data; a.weight = weight; a.dx = dx ? dx->data : nullptr; a.mean = mean; a.rstd = rstd;
    a.gu = dy->user_stride; a.gt = dy->token_stride; a.xu = x->user_stride; a.xt = x->token_stride;
    if (dx) { a.du = dx->user_stride; a.dt = dx->token_stride; }
    a.tokens = (uint32_t)n_tokens; a.dim = (int)h->dim; a.weight_type = weight_type;
    a.inv_dim = (float)(1.0 / (double)h->dim); a.part = h->part;
    if (dweight) a.dweight = *dweight;
    if (dbias) a.dbias = *dbias;
    const bool whole = h->dim * type_width(x->type) % 16 == 0 && rows_aligned(x, h->users, n_tokens) && rows_aligned(dy, h->users, n_tokens) &&
                       (!dx || rows_aligned(dx, h->users, n_tokens));
    LnRunBackward run = {h, a, (cudaStream_t)cuda_stream};
    return ln_with(h->dim, x->type, ln_take(x->type, whole), run);
}

extern "C" int64_t co3_layernorm_launch_count(const co3_layernorm* h) { return h ? h->launches : 0; }
