// Layer norm forward and backward, with the reduction of the weight's and the bias' gradient per user (co3_layernorm_*).
//
// A row is held in the registers of TPR threads, E elements each, so that one read of it serves mean, variance and result: two
// passes over registers, and the variance is that of differences.  Thread blocks stay and take row after row, with the weight in
// registers; the next row's loads are in flight while a row is worked on.
#include "co3_ops.cuh"

namespace {

constexpr int LN_MAX_DIM = 16384;

struct LnForward {
    const void* x; const void* weight; const void* bias; void* y;
    float *mean, *rstd;
    int64_t xu, xt, yu, yt;                   // strides
    uint32_t tokens, rows;
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

// Sum over the TPR threads of a row of K values each; `turn` counts the reductions of a thread block.
template <int TPR, int K> __device__ __forceinline__ void row_sum(float (&x)[K], float (*sh)[32][K], int& turn) {
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = warp_sum_f32(x[k]);
    if (TPR == 32) return;
    float(*s)[K] = sh[turn & 1];              // two buffers: one barrier a reduction
    ++turn;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) s[threadIdx.x >> 5][k] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float t = 0.0f;
        if (TPR / 32 <= 8) {
#pragma unroll
            for (int w = 0; w < TPR / 32; ++w) t += s[w][k];
        } else t = warp_sum_f32((threadIdx.x & 31) < TPR / 32 ? s[threadIdx.x & 31][k] : 0.0f);
        x[k] = t;
    }
}

// The elements that a thread holds of a row: E / V pieces of V neighbours, piece c at column (c TPR + t) V.  VEC: 16 bytes each,
// else one element, for rows that begin anywhere or have an odd length.
template <class T, bool VEC, int TPR, int E> struct Held {
    static constexpr int V = VEC ? T::EACH : 1, N = E / V;
    static_assert(E % V == 0, "whole pieces");
    static __device__ __forceinline__ int column(int t, int c) { return (c * TPR + t) * V; }
    typename std::conditional<VEC, uint4, typename T::type>::type raw[N];
    __device__ __forceinline__ void load(const void* row, int t, int dim) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const int at = column(t, c);
            if (at < dim) {
                if constexpr (VEC) raw[c] = __ldcs((const uint4*)((const typename T::type*)row + at));
                else raw[c] = ((const typename T::type*)row)[at];
            } else {
                if constexpr (VEC) raw[c] = make_uint4(0, 0, 0, 0);
                else raw[c] = T::put(0.0f);
            }
        }
    }
    __device__ __forceinline__ void values(float* x) const {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            if constexpr (VEC) T::unpack(raw[c], x + c * V);
            else x[c] = T::get(raw[c]);
        }
    }
    static __device__ __forceinline__ void store(void* row, int t, int dim, const float* x) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const int at = column(t, c);
            if (at < dim) {
                if constexpr (VEC) *(uint4*)((typename T::type*)row + at) = T::pack(x + c * V);
                else ((typename T::type*)row)[at] = T::put(x[c]);
            }
        }
    }
    // per-column values in 32 bits
    static __device__ __forceinline__ void param(const void* p, int type, float otherwise, int t, int dim, float* w) {
#pragma unroll
        for (int c = 0; c < N; ++c)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int at = column(t, c) + k;
                w[c * V + k] = at < dim ? (p ? load_as_f32(p, type, at) : otherwise) : 0.0f;
            }
    }
};

template <int TPR> constexpr int LN_THREADS = TPR == 32 ? 256 : TPR;

template <class T, bool VEC, int TPR, int E>
__global__ void __launch_bounds__(LN_THREADS<TPR>) ln_forward_kernel(const __grid_constant__ LnForward a) {
    typedef Held<T, VEC, TPR, E> H;
    constexpr int GROUPS = LN_THREADS<TPR> / TPR;
    __shared__ float sh[2][32][1];
    int turn = 0;
    const int t = threadIdx.x % TPR;
    let_next_start();
    wait_for_previous();
    float w[E], b[E];
    H::param(a.weight, a.weight_type, 1.0f, t, a.dim, w);
    H::param(a.bias, a.weight_type, 0.0f, t, a.dim, b);
    auto row_of = [&](uint32_t r) {
        const uint32_t u = r / a.tokens;
        return (const typename T::type*)a.x + u * a.xu + (r - u * a.tokens) * a.xt;
    };
    const uint32_t step = gridDim.x * GROUPS;
    uint32_t r = blockIdx.x * GROUPS + threadIdx.x / TPR;
    H next;
    if (r < a.rows) next.load(row_of(r), t, a.dim);
    for (; r < a.rows; r += step) {
        float x[E];
        next.values(x);
        if (a.rows - r > step) next.load(row_of(r + step), t, a.dim);
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < E; ++i) s[0] += x[i];
        row_sum<TPR, 1>(s, sh, turn);
        const float mean = s[0] * a.inv_dim;
        s[0] = 0.0f;
#pragma unroll
        for (int c = 0; c < H::N; ++c)
#pragma unroll
            for (int k = 0; k < H::V; ++k) {
                const int i = c * H::V + k;
                x[i] -= mean;
                if (H::column(t, c) < a.dim) s[0] = fmaf(x[i], x[i], s[0]);
            }
        row_sum<TPR, 1>(s, sh, turn);
        const float rstd = 1.0f / sqrtf(fmaf(s[0], a.inv_dim, a.eps));
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = fmaf(x[i] * rstd, w[i], b[i]);
        const uint32_t u = r / a.tokens, k = r - u * a.tokens;
        H::store((typename T::type*)a.y + u * a.yu + k * a.yt, t, a.dim, x);
        if (t == 0) { a.mean[r] = mean; a.rstd[r] = rstd; }
    }
}

// blockIdx.x: slice of the user blockIdx.y's rows.
template <class T, bool VEC, int TPR, int E>
__global__ void __launch_bounds__(LN_THREADS<TPR>) ln_backward_kernel(const __grid_constant__ LnBackward a) {
    typedef Held<T, VEC, TPR, E> H;
    constexpr int GROUPS = LN_THREADS<TPR> / TPR;
    __shared__ float sh[2][32][2];
    int turn = 0;
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const uint32_t user = blockIdx.y;
    let_next_start();
    wait_for_previous();
    float w[E], dw[E], db[E];
    H::param(a.weight, a.weight_type, 1.0f, t, a.dim, w);
#pragma unroll
    for (int i = 0; i < E; ++i) dw[i] = db[i] = 0.0f;
    const typename T::type* gy = (const typename T::type*)a.dy + user * a.gu;
    const typename T::type* xs = (const typename T::type*)a.x + user * a.xu;
    typename T::type* dx = (typename T::type*)a.dx + user * a.du;
    const float *means = a.mean + (int64_t)user * a.tokens, *rstds = a.rstd + (int64_t)user * a.tokens;
    const uint32_t step = a.slices * GROUPS;
    H ng, nx;
    float nm = 0.0f, nr = 0.0f;
    auto fetch = [&](uint32_t r) {
        ng.load(gy + r * a.gt, t, a.dim);
        nx.load(xs + r * a.xt, t, a.dim);
        nm = means[r];
        nr = rstds[r];
    };
    uint32_t r = blockIdx.x * GROUPS + group;
    if (r < a.tokens) fetch(r);
    for (; r < a.tokens; r += step) {
        float g[E], x[E];
        ng.values(g);
        nx.values(x);
        const float mean = nm, rstd = nr;
        if (a.tokens - r > step) fetch(r + step);
        float c[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < E; ++i) {
            x[i] = (x[i] - mean) * rstd;
            dw[i] = fmaf(g[i], x[i], dw[i]);
            db[i] += g[i];
            g[i] *= w[i];                     // 0 beyond the row
            c[0] += g[i];
            c[1] = fmaf(g[i], x[i], c[1]);
        }
        row_sum<TPR, 2>(c, sh, turn);
        if (a.dx) {
            const float c1 = c[0] * a.inv_dim, c2 = c[1] * a.inv_dim;
#pragma unroll
            for (int i = 0; i < E; ++i) g[i] = (g[i] - fmaf(x[i], c2, c1)) * rstd;
            H::store(dx + r * a.dt, t, a.dim, g);
        }
    }
    if (!a.dweight.data && !a.dbias.data) return;
    if (GROUPS > 1) {                         // the warps' sums, in their order
        __shared__ float sums[2][GROUPS > 1 ? 32 * E : 1];
        for (int k = 0; k < GROUPS; ++k) {
            if (group == k)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int at = i * 32 + t;
                    sums[0][at] = dw[i] = k ? sums[0][at] + dw[i] : dw[i];
                    sums[1][at] = db[i] = k ? sums[1][at] + db[i] : db[i];
                }
            __syncthreads();
        }
        if (group != GROUPS - 1) return;
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

// How a row of `dim` elements is held: the least that holds it.  One warp up to 1024 elements, several above.
struct LnShape { int tpr, e; };
inline LnShape ln_shape(int64_t dim) {
    if (dim <= 256) return {32, 8};
    if (dim <= 512) return {32, 16};
    if (dim <= 768) return {32, 24};
    if (dim <= 1024) return {32, 32};
    if (dim <= 2048) return {128, 16};
    if (dim <= 4096) return {256, 16};
    if (dim <= 8192) return {512, 16};
    return {1024, 16};
}
// Thread blocks on an SM.
inline int ln_per_sm(int tpr) { return tpr == 32 ? 2 : tpr == 128 ? 5 : tpr == 256 ? 3 : tpr == 512 ? 1 : 1; }

}  // namespace

struct co3_layernorm {
    int64_t dim, launches;
    int users, device, sms;
    double eps;
    float* part;
};

namespace {

int ln_slices(const co3_layernorm* h, int64_t tokens) {
    const LnShape s = ln_shape(h->dim);
    const int64_t groups = s.tpr == 32 ? 8 : 1, places = (int64_t)h->sms * ln_per_sm(s.tpr) / h->users, most = (tokens + 2 * groups - 1) / (2 * groups);
    const int64_t n = places < most ? places : most;
    return n < 1 ? 1 : (int)n;
}

template <class T, bool VEC, int TPR, int E> int ln_forward_of(co3_layernorm* h, const LnForward& a, cudaStream_t st) {
    const uint32_t groups = LN_THREADS<TPR> / TPR;
    const int64_t need = ((int64_t)a.rows + groups - 1) / groups, places = (int64_t)h->sms * (2048 / LN_THREADS<TPR>);
    return launch_early(&h->launches, ln_forward_kernel<T, VEC, TPR, E>, dim3((unsigned)(need < places ? need : places)), LN_THREADS<TPR>, 0, 1, st, a);
}
template <class T, bool VEC, int TPR, int E> int ln_backward_of(co3_layernorm* h, const LnBackward& a, cudaStream_t st) {
    return launch_early(&h->launches, ln_backward_kernel<T, VEC, TPR, E>, dim3((unsigned)a.slices, (unsigned)h->users), LN_THREADS<TPR>, 0, 1, st, a);
}
template <class T, bool VEC, class A> int ln_launch_as(co3_layernorm* h, const A& a, cudaStream_t st) {
    const LnShape s = ln_shape(h->dim);
#define CO3_LN(tpr_, e_) \
    if (s.tpr == tpr_ && s.e == e_) { \
        if constexpr (std::is_same<A, LnForward>::value) return ln_forward_of<T, VEC, tpr_, e_>(h, a, st); \
        else return ln_backward_of<T, VEC, tpr_, e_>(h, a, st); \
    }
    CO3_LN(32, 8) CO3_LN(32, 16) CO3_LN(32, 24) CO3_LN(32, 32) CO3_LN(128, 16) CO3_LN(256, 16) CO3_LN(512, 16) CO3_LN(1024, 16)
#undef CO3_LN
    return CO3_EINVAL;
}
template <class A> int ln_launch(co3_layernorm* h, int type, bool vec, const A& a, cudaStream_t st) {
    if (type == CO3_F32) return vec ? ln_launch_as<OF32, true>(h, a, st) : ln_launch_as<OF32, false>(h, a, st);
    if (type == CO3_BF16) return vec ? ln_launch_as<OBf16, true>(h, a, st) : ln_launch_as<OBf16, false>(h, a, st);
    return vec ? ln_launch_as<OF16, true>(h, a, st) : ln_launch_as<OF16, false>(h, a, st);
}

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
        // of users whose rows go to more than one thread block
        const int64_t slices = ln_slices(h, OPS_MAX_ROWS);
        if (slices > 1 && cudaMalloc(&h->part, (size_t)(n_users * slices * 2 * dim * 4)) != cudaSuccess) { h->part = nullptr; rc = CO3_ENOMEM; }
    }
    if (rc != CO3_OK) { (void)cudaGetLastError(); co3_layernorm_destroy(h); return rc; }
    *out = h;
    return CO3_OK;
}

extern "C" int co3_layernorm_forward(co3_layernorm* h, const co3_array* x, const void* weight, const void* bias, int32_t weight_type, int64_t n_tokens,
                                     const co3_array* y, float* mean, float* rstd, void* cuda_stream) {
    if (!h || n_tokens < 0 || n_tokens * h->users > OPS_MAX_ROWS) return CO3_EINVAL;
    if (!array_fine(x, h->users, n_tokens, h->dim, false) || !array_fine(y, h->users, n_tokens, h->dim, true) || x->type != y->type) return CO3_EINVAL;
    if ((weight || bias) && (!type_known(weight_type) || !aligned_to(weight, type_width(weight_type)) || !aligned_to(bias, type_width(weight_type)))) return CO3_EINVAL;
    if (!device_is(h->device)) return CO3_EINVAL;
    if (n_tokens == 0) return CO3_OK;
    if (!mean || !rstd || !aligned_to(mean, 4) || !aligned_to(rstd, 4)) return CO3_EINVAL;
    LnForward a;
    a.x = x->data; a.weight = weight; a.bias = bias; a.y = y->data; a.mean = mean; a.rstd = rstd;
    a.xu = x->user_stride; a.xt = x->token_stride; a.yu = y->user_stride; a.yt = y->token_stride;
    a.tokens = (uint32_t)n_tokens; a.rows = (uint32_t)(n_tokens * h->users);
    a.dim = (int)h->dim; a.weight_type = weight_type; a.inv_dim = (float)(1.0 / (double)h->dim); a.eps = (float)h->eps;
    const bool vec = h->dim * type_width(x->type) % 16 == 0 && rows_aligned(x, h->users, n_tokens) && rows_aligned(y, h->users, n_tokens);
    return ln_launch(h, x->type, vec, a, (cudaStream_t)cuda_stream);
}

extern "C" int co3_layernorm_backward(co3_layernorm* h, const co3_array* dy, const co3_array* x, const void* weight, int32_t weight_type, const float* mean,
                                      const float* rstd, int64_t n_tokens, const co3_array* dx, const co3_param_grad* dweight,
                                      const co3_param_grad* dbias, void* cuda_stream) {
    if (!h || n_tokens < 0 || n_tokens * h->users > OPS_MAX_ROWS) return CO3_EINVAL;
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
    a.tokens = (uint32_t)n_tokens; a.dim = (int)h->dim; a.weight_type = weight_type; a.slices = ln_slices(h, n_tokens);
    a.inv_dim = (float)(1.0 / (double)h->dim); a.part = h->part;
    if (dweight) a.dweight = *dweight;
    if (dbias) a.dbias = *dbias;
    const bool vec = h->dim * type_width(x->type) % 16 == 0 && rows_aligned(x, h->users, n_tokens) && rows_aligned(dy, h->users, n_tokens) &&
                     (!dx || rows_aligned(dx, h->users, n_tokens));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int rc = ln_launch(h, x->type, vec, a, st);
    if (rc != CO3_OK || a.slices == 1 || (!dweight && !dbias)) return rc;
    return launch_early(&h->launches, ln_join_kernel, dim3((unsigned)((2 * h->dim + 31) / 32), (unsigned)h->users), 256, 0, 1, st, (const float*)h->part,
                        a.slices, a.dim, a.dweight, a.dbias);
}

extern "C" int64_t co3_layernorm_launch_count(const co3_layernorm* h) { return h ? h->launches : 0; }
