// Embedding lookup, and its gradient by sorted tokens (co3_embed_*).
//
// Gradient, three kernels: (1) a cluster of thread blocks per user sorts the user's tokens with their places by radix, stably, while
// the other SMs write the zeros of the table's gradient; (2) warps take 32 sorted places and 256 columns each, add the rows of equal
// tokens in their order and write a token's row where its run ends within the 32; (3) what runs longer than that left is joined, in
// order again.  No sum depends on the order of an atomic.
#include "co3_ops.cuh"

namespace {

constexpr int SORT_THREADS = 1024, SORT_WARPS = 32, SORT_CLUSTER = 8;
constexpr int SORT_ALONE = 4096;              // tokens of a user that one thread block sorts by itself
constexpr int RUN = 32;                       // sorted places of a warp
constexpr int SLAB = 256;                     // columns of a warp: eight to a lane
constexpr int PIECE = 1024;                   // columns of a row that a warp looks up at a time
constexpr int JOIN_WARPS = 8;

struct Tokens {
    const void* data;
    int64_t user_stride, token_stride;
    int wide;
};
__device__ __forceinline__ int64_t token_at(const Tokens& k, int64_t user, int64_t t) {
    const int64_t at = user * k.user_stride + t * k.token_stride;
    return k.wide ? ((const int64_t*)k.data)[at] : (int64_t)((const int32_t*)k.data)[at];
}

// ---- lookup ---------------------------------------------------------------------------------------------------------------
struct LookupArgs {
    Tokens tokens;
    const void* table; void* out;
    int64_t ou, ot;
    int64_t items;
    uint32_t n_tokens, pieces;
    int64_t vocab;
    int dim;
    float scale;
    OpsStatus* status;
};

// Eight neighbours of an aligned row.
template <class T> __device__ __forceinline__ void load8(const typename T::type* p, float* x) {
    T::unpack(((const uint4*)p)[0], x);
    if (T::EACH == 4) T::unpack(((const uint4*)p)[1], x + 4);
}
template <class T> __device__ __forceinline__ void store8(typename T::type* p, const float* x) {
    ((uint4*)p)[0] = T::pack(x);
    if (T::EACH == 4) ((uint4*)p)[1] = T::pack(x + 4);
}

template <class A, class B, bool VEC>
__global__ void __launch_bounds__(256) lookup_kernel(const __grid_constant__ LookupArgs a) {
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    let_next_start();
    wait_for_previous();
    if (item >= a.items) return;
    const uint32_t row = (uint32_t)(item / a.pieces), piece = (uint32_t)(item - (int64_t)row * a.pieces);
    const uint32_t user = row / a.n_tokens, t = row - user * a.n_tokens;
    int64_t token = token_at(a.tokens, user, t);
    if (token >= a.vocab) {
        if (lane == 0 && piece == 0) { atomicAdd(&a.status->bad_tokens, 1ull); atomicOr(&a.status->flags, CO3_FLAG_TOKEN); }
        token = -1;
    }
    const typename A::type* from = (const typename A::type*)a.table + token * a.dim;
    typename B::type* to = (typename B::type*)a.out + user * a.ou + t * a.ot;
    if (VEC) {
        float x[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = (int)piece * PIECE + i * 256 + lane * 8;
#pragma unroll
            for (int k = 0; k < 8; ++k) x[i][k] = 0.0f;
            if (token >= 0 && at < a.dim) load8<A>(from + at, x[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = (int)piece * PIECE + i * 256 + lane * 8;
            if (token >= 0)
#pragma unroll
                for (int k = 0; k < 8; ++k) x[i][k] *= a.scale;
            if (at < a.dim) store8<B>(to + at, x[i]);
        }
    } else {
        const int end = a.dim < ((int)piece + 1) * PIECE ? a.dim : ((int)piece + 1) * PIECE;
#pragma unroll 8
        for (int at = (int)piece * PIECE + lane; at < end; at += 32) to[at] = B::put(token < 0 ? 0.0f : A::get(from[at]) * a.scale);
    }
}

// ---- sort, and zeros -------------------------------------------------------------------------------------------------------
struct SortArgs {
    Tokens tokens;
    int64_t vocab;
    uint32_t n_tokens, pitch;                 // of a user's part of the arrays
    int users, cluster, passes, digit_bits;
    uint32_t *key[2], *place[2];              // [users][pitch]; the sorted ones end in [passes & 1]
    uint32_t* n_valid;                        // [users]
    uint32_t* n_long;                         // runs that are longer than a warp's part: counted by the next kernel
    OpsStatus* status;
    uint8_t* zero;                            // null: nothing to fill
    int64_t zero_stride, zero_bytes;          // of a user
};

__device__ __forceinline__ uint32_t shared_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t peer_word(uint32_t at, uint32_t rank) {      // a word of another thread block of the cluster
    uint32_t far, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(far) : "r"(at), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(far) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Zeros for the users' parts, by all fill blocks together; a part may begin and end at any element.
__device__ void fill_zeros(const SortArgs& a, uint32_t block, uint32_t blocks) {
    constexpr int64_t CHUNK = 64 * 1024;
    const int64_t per_user = (a.zero_bytes + 15 + CHUNK - 1) / CHUNK, all = per_user * a.users;
    for (int64_t i = block; i < all; i += blocks) {
        const int64_t user = i / per_user, j = i - user * per_user;
        uint8_t* const begin = a.zero + user * a.zero_stride, *const end = begin + a.zero_bytes;
        uint8_t* const whole = (uint8_t*)((uintptr_t)begin & ~(uintptr_t)15);       // chunks count from here
        uint8_t *p = whole + j * CHUNK, *q = p + CHUNK;
        if (q > end) q = end;
        if (p < begin) {                      // the first chunk's bytes before the first whole 16
            uint8_t* const edge = whole + 16 < q ? whole + 16 : q;
            for (uint8_t* b = begin + 2 * threadIdx.x; b < edge; b += 2 * SORT_THREADS) *(uint16_t*)b = 0;
            p = whole + 16;
        }
        if (p >= q) continue;
        const int64_t words = (q - p) / 16;
        for (int64_t w = threadIdx.x; w < words; w += SORT_THREADS) ((uint4*)p)[w] = make_uint4(0, 0, 0, 0);
        for (uint8_t* b = p + words * 16 + 2 * threadIdx.x; b < q; b += 2 * SORT_THREADS) *(uint16_t*)b = 0;
    }
}

__global__ void __launch_bounds__(SORT_THREADS, 2) sort_kernel(const __grid_constant__ SortArgs a) {
    __shared__ uint32_t hist[SORT_WARPS][256];
    __shared__ uint32_t totals[256 + 1], base[256], warp_sums[8];
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t user = blockIdx.x / a.cluster, rank = blockIdx.x - user * a.cluster;
    let_next_start();
    wait_for_previous();
    if (user >= (uint32_t)a.users) {
        fill_zeros(a, blockIdx.x - a.users * a.cluster, gridDim.x - a.users * a.cluster);
        return;
    }
    if (blockIdx.x == 0 && tid == 0) *a.n_long = 0;
    const uint32_t n = a.n_tokens;
    const uint32_t per_block = ((n + a.cluster - 1) / a.cluster + 1023) / 1024 * 1024, per_warp = per_block / 32;
    const uint64_t first = (uint64_t)rank * per_block + (uint64_t)warp * per_warp;
    const uint32_t begin = first < n ? (uint32_t)first : n, end = first + per_warp < n ? (uint32_t)(first + per_warp) : n;
    const uint32_t bins = 1u << a.digit_bits;
    const uint32_t below = (1u << lane) - 1u;
    for (int pass = 0; pass < a.passes; ++pass) {
        const uint32_t *key_in = a.key[pass & 1] + (int64_t)user * a.pitch, *place_in = a.place[pass & 1] + (int64_t)user * a.pitch;
        uint32_t *key_out = a.key[~pass & 1] + (int64_t)user * a.pitch, *place_out = a.place[~pass & 1] + (int64_t)user * a.pitch;
        const int shift = pass * a.digit_bits;
        auto key_of = [&](uint32_t i) -> uint32_t {
            if (pass) return __ldcg(key_in + i);
            const int64_t token = token_at(a.tokens, user, i);
            return token < 0 || token >= a.vocab ? (uint32_t)a.vocab : (uint32_t)token;      // those that are none come last
        };
        for (uint32_t b = lane; b < bins; b += 32) hist[warp][b] = 0;
        if (tid == 0) totals[256] = 0;
        __syncthreads();
        uint32_t valid = 0;
        for (uint32_t i = begin; i < end; i += 32) {
            const bool here = i + lane < end;
            const uint32_t key = here ? key_of(i + lane) : 0, digit = here ? key >> shift & (bins - 1) : 256;
            const uint32_t same = __match_any_sync(0xffffffffu, digit);
            if (here && !(same & below)) hist[warp][digit] += __popc(same);
            if (pass == 0) {
                valid += __popc(__ballot_sync(0xffffffffu, here && key < (uint32_t)a.vocab));
                if (here && key == (uint32_t)a.vocab && token_at(a.tokens, user, i + lane) >= a.vocab) {
                    atomicAdd(&a.status->bad_tokens, 1ull);
                    atomicOr(&a.status->flags, CO3_FLAG_TOKEN);
                }
            }
            __syncwarp();
        }
        if (pass == 0 && lane == 0 && valid) atomicAdd(&totals[256], valid);
        __syncthreads();
        if (tid < bins) {                     // where each warp's part of a digit begins within the block's
            uint32_t s = 0;
#pragma unroll 8
            for (int w = 0; w < SORT_WARPS; ++w) { const uint32_t c = hist[w][tid]; hist[w][tid] = s; s += c; }
            totals[tid] = s;
        }
        if (a.cluster > 1) cluster_barrier();
        else __syncthreads();
        uint32_t all = 0, before = 0;
        if (tid < bins) {
            for (int r = 0; r < a.cluster; ++r) {
                const uint32_t c = a.cluster > 1 ? peer_word(shared_at(&totals[tid]), r) : totals[tid];
                if (r < (int)rank) before += c;
                all += c;
            }
        }
        if (pass == 0 && rank == 0 && tid == 256) {
            uint32_t s = 0;
            for (int r = 0; r < a.cluster; ++r) s += a.cluster > 1 ? peer_word(shared_at(&totals[256]), r) : totals[256];
            a.n_valid[user] = s;
        }
        uint32_t up = all;                    // places of the smaller digits, over all blocks
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, up, o); if ((int)lane >= o) up += v; }
        if (warp < 8 && lane == 31) warp_sums[warp] = up;
        __syncthreads();
        if (tid < bins) {
            for (uint32_t w = 0; w < warp; ++w) before += warp_sums[w];
            base[tid] = before + up - all;
        }
        __syncthreads();
        for (uint32_t i = begin; i < end; i += 32) {
            const bool here = i + lane < end;
            const uint32_t key = here ? key_of(i + lane) : 0, digit = here ? key >> shift & (bins - 1) : 256;
            const uint32_t same = __match_any_sync(0xffffffffu, digit);
            const uint32_t ahead = here ? hist[warp][digit] : 0;
            __syncwarp();
            if (here) {
                if (!(same & below)) hist[warp][digit] = ahead + __popc(same);
                const uint32_t to = base[digit] + ahead + __popc(same & below);
                __stcg(key_out + to, key);
                __stcg(place_out + to, pass ? __ldcg(place_in + i + lane) : i + lane);
            }
            __syncwarp();
        }
        if (a.cluster > 1) cluster_barrier();  // also: nobody reads another block's totals any more
        else __syncthreads();
    }
}

// ---- sums ------------------------------------------------------------------------------------------------------------------
struct SumArgs {
    const void* dout;
    int64_t gu, gt;
    const uint32_t *key, *place, *n_valid;
    uint32_t pitch, chunks;                   // of a user
    uint32_t* n_long;
    uint32_t* long_runs;                      // [users * chunks]: user * chunks + chunk in which a longer run begins
    float* part;                              // [users * chunks][2][dim]: of a run that began before the chunk, of one that goes on after it
    co3_param_grad to;
    int64_t items;
    int dim, slabs;
    float scale;
};

template <class T> __device__ __forceinline__ void put_sum(typename T::type* p, float x, bool add) {
    *p = T::put(add ? T::get(*p) + x : x);
}
// VEC: a lane has eight neighbouring columns, else every 32nd.
template <class B, bool VEC> __device__ __forceinline__ void put_sums(const SumArgs& a, int64_t user, uint32_t token, int column, const float* s) {
    typename B::type* p = (typename B::type*)a.to.data + user * a.to.user_stride + (int64_t)token * a.dim + column;
    if (VEC) {
        if (column >= a.dim) return;
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = 0.0f;
        if (a.to.accumulate) load8<B>(p, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = a.to.accumulate ? x[k] + s[k] * a.scale : s[k] * a.scale;
        store8<B>(p, x);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (column + 32 * k < a.dim) put_sum<B>(p + 32 * k, s[k] * a.scale, a.to.accumulate);
    }
}

template <class A, class B, bool VEC>
__global__ void __launch_bounds__(256) sum_kernel(const __grid_constant__ SumArgs a) {
    constexpr int AT_ONCE = 8;                // rows whose loads are in flight
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    let_next_start();
    wait_for_previous();
    if (item >= a.items) return;
    const uint32_t at = (uint32_t)(item / a.slabs);       // user * chunks + chunk
    const int slab = (int)(item - (int64_t)at * a.slabs);
    const uint32_t user = at / a.chunks, chunk = at - user * a.chunks, n = a.n_valid[user], i0 = chunk * RUN;
    if (i0 >= n) return;
    const int count = n - i0 < RUN ? (int)(n - i0) : RUN;
    const uint32_t* keys = a.key + (int64_t)user * a.pitch + i0;
    const uint32_t key = lane < count ? keys[lane] : 0xFFFFFFFFu, place = lane < count ? a.place[(int64_t)user * a.pitch + i0 + lane] : 0;
    const uint32_t before = i0 ? keys[-1] : 0xFFFFFFFFu, after = i0 + RUN < n ? keys[RUN] : 0xFFFFFFFFu;
    const int column = slab * SLAB + (VEC ? lane * 8 : lane);
    const typename A::type* rows = (const typename A::type*)a.dout + user * a.gu + column;
    float sum[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
    bool first = true;                        // still in the chunk's first run
    for (int e0 = 0; e0 < count; e0 += AT_ONCE) {
        float x[AT_ONCE][8];
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) {
#pragma unroll
            for (int k = 0; k < 8; ++k) x[e][k] = 0.0f;
            const uint32_t t = __shfl_sync(0xffffffffu, place, (e0 + e) & 31);
            if (e0 + e < count) {
                const typename A::type* row = rows + (int64_t)t * a.gt;
                if (VEC) { if (column < a.dim) load8<A>(row, x[e]); }
                else
#pragma unroll
                    for (int k = 0; k < 8; ++k) if (column + 32 * k < a.dim) x[e][k] = A::get(row[32 * k]);
            }
        }
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) {
            if (e0 + e >= count) break;
            const uint32_t mine = __shfl_sync(0xffffffffu, key, e0 + e);
            const uint32_t next = e0 + e + 1 < count ? __shfl_sync(0xffffffffu, key, (e0 + e + 1) & 31) : after;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += x[e][k];
            const bool last = e0 + e + 1 == count;
            if (next == mine && !last) continue;
            const bool began_before = first && mine == before, goes_on = last && next == mine;
            if (began_before || goes_on) {
                float* part = a.part + ((int64_t)at * 2 + (began_before ? 0 : 1)) * a.dim + column;
                if (VEC) { if (column < a.dim) store8<OF32>(part, sum); }
                else
#pragma unroll
                    for (int k = 0; k < 8; ++k) if (column + 32 * k < a.dim) part[32 * k] = sum[k];
                if (!began_before && slab == 0 && lane == 0) a.long_runs[atomicAdd(a.n_long, 1u)] = at;
            } else put_sums<B, VEC>(a, user, mine, column, sum);
            first = false;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
        }
    }
}

// The runs longer than a chunk, each by a thread block: its warps add a stretch of the chunks each, the stretches are added in order.
template <class B, bool VEC>
__global__ void __launch_bounds__(32 * JOIN_WARPS) join_kernel(const __grid_constant__ SumArgs a) {
    __shared__ float sh[JOIN_WARPS][SLAB];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    let_next_start();
    wait_for_previous();
    const int64_t items = (int64_t)*a.n_long * a.slabs;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t at = a.long_runs[item / a.slabs];
        const int slab = (int)(item % a.slabs);
        const uint32_t user = at / a.chunks, chunk = at - user * a.chunks, n = a.n_valid[user];
        const uint32_t* keys = a.key + (int64_t)user * a.pitch;
        const uint32_t token = keys[chunk * RUN + RUN - 1];
        uint32_t lo = (chunk + 1) * RUN, hi = n;          // the run ends before the first larger key
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (keys[mid] == token) lo = mid + 1; else hi = mid;
        }
        const uint32_t parts = (lo - 1) / RUN - chunk + 1, each = (parts + JOIN_WARPS - 1) / JOIN_WARPS;
        const uint32_t p0 = warp * each < parts ? warp * each : parts, p1 = p0 + each < parts ? p0 + each : parts;
        const int column = slab * SLAB + lane;
        float s[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] = 0.0f;
#pragma unroll 4
        for (uint32_t p = p0; p < p1; ++p) {
            const float* part = a.part + (((int64_t)at + p) * 2 + (p ? 0 : 1)) * a.dim + column;
#pragma unroll
            for (int k = 0; k < 8; ++k) if (column + 32 * k < a.dim) s[k] += part[32 * k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sh[warp][lane + 32 * k] = s[k];
        __syncthreads();
        if (warp == 0) {
            float x[8];
            const int c0 = VEC ? lane * 8 : lane, step = VEC ? 1 : 32;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                x[k] = sh[0][c0 + k * step];
                for (int w = 1; w < JOIN_WARPS; ++w) x[k] += sh[w][c0 + k * step];
            }
            put_sums<B, VEC>(a, user, token, slab * SLAB + c0, x);
        }
        __syncthreads();
    }
}

}  // namespace

struct co3_embed {
    int64_t vocab, dim, max_tokens, launches;
    int users, device, sms;
    uint32_t pitch, chunks;
    void* slab;
    OpsStatus* status;
    uint32_t *key[2], *place[2], *n_valid, *n_long, *long_runs;
    float* part;
};

extern "C" void co3_embed_destroy(co3_embed* h) {
    if (!h) return;
    if (h->slab) cudaFree(h->slab);
    delete h;
}

extern "C" int co3_embed_create(co3_embed** out, int64_t vocab, int64_t dim, int32_t n_users, int64_t max_tokens) {
    if (!out) return CO3_EINVAL;
    *out = nullptr;
    if (vocab < 1 || vocab >= (int64_t)1 << 31 || dim < 1 || dim >= ((int64_t)1 << 31) - PIECE || n_users < 1 || n_users > OPS_MAX_USERS) return CO3_EINVAL;
    if (vocab * dim > (int64_t)1 << 44 || max_tokens < 0 || max_tokens > OPS_MAX_ROWS / n_users) return CO3_EINVAL;
    co3_embed* h = new (std::nothrow) co3_embed();
    if (!h) return CO3_ENOMEM;
    memset(h, 0, sizeof(*h));
    h->vocab = vocab; h->dim = dim; h->users = n_users; h->max_tokens = max_tokens;
    h->pitch = (uint32_t)((max_tokens + 3) / 4 * 4);
    h->chunks = (uint32_t)((max_tokens + RUN - 1) / RUN);
    int rc = CO3_OK;
    if (cudaGetDevice(&h->device) != cudaSuccess || cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, h->device) != cudaSuccess || h->sms < 1) rc = CO3_ECUDA;
    if (rc == CO3_OK) {
        size_t at = 0;
        auto part = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
        const size_t words = 4 * (size_t)h->pitch * n_users, runs = (size_t)h->chunks * n_users;
        const size_t o_status = part(sizeof(OpsStatus)), o_key = part(words), o_key2 = part(words), o_place = part(words), o_place2 = part(words);
        const size_t o_valid = part(4 * (size_t)n_users), o_count = part(4), o_long = part(4 * runs), o_part = part(runs * 2 * dim * 4);
        if (cudaMalloc(&h->slab, at) != cudaSuccess) { h->slab = nullptr; rc = CO3_ENOMEM; }
        else {
            char* base = (char*)h->slab;
            h->status = (OpsStatus*)(base + o_status);
            h->key[0] = (uint32_t*)(base + o_key); h->key[1] = (uint32_t*)(base + o_key2);
            h->place[0] = (uint32_t*)(base + o_place); h->place[1] = (uint32_t*)(base + o_place2);
            h->n_valid = (uint32_t*)(base + o_valid); h->n_long = (uint32_t*)(base + o_count); h->long_runs = (uint32_t*)(base + o_long);
            h->part = (float*)(base + o_part);
            if (cudaMemset(h->status, 0, sizeof(OpsStatus)) != cudaSuccess || cudaStreamSynchronize(nullptr) != cudaSuccess) rc = CO3_ECUDA;
        }
    }
    if (rc != CO3_OK) { (void)cudaGetLastError(); co3_embed_destroy(h); return rc; }
    *out = h;
    return CO3_OK;
}

namespace {

bool embed_tokens_fine(const co3_embed* h, const co3_tokens* k, int64_t n) {
    if (!k || (k->type != CO3_I32 && k->type != CO3_I64) || k->top != 1) return false;
    if (n == 0) return true;
    const int64_t most = (int64_t)1 << 46;
    return k->data && aligned_to(k->data, k->type == CO3_I32 ? 4 : 8) && k->user_stride >= 0 && k->token_stride >= 0 && k->user_stride <= most && k->token_stride <= most;
}
Tokens tokens_of(const co3_tokens* k) { return Tokens{k->data, k->user_stride, k->token_stride, k->type == CO3_I64}; }

template <class A, class B> int lookup_of(co3_embed* h, bool vec, const LookupArgs& a, dim3 grid, cudaStream_t st) {
    return vec ? launch_early(&h->launches, lookup_kernel<A, B, true>, grid, 256, 0, 1, st, a)
               : launch_early(&h->launches, lookup_kernel<A, B, false>, grid, 256, 0, 1, st, a);
}
template <class A> int lookup_to(co3_embed* h, int type, bool vec, const LookupArgs& a, dim3 grid, cudaStream_t st) {
    if (type == CO3_F32) return lookup_of<A, OF32>(h, vec, a, grid, st);
    if (type == CO3_BF16) return lookup_of<A, OBf16>(h, vec, a, grid, st);
    return lookup_of<A, OF16>(h, vec, a, grid, st);
}
template <class A, class B> int sums_of(co3_embed* h, bool vec, const SumArgs& a, cudaStream_t st) {
    const dim3 grid((unsigned)((a.items + 7) / 8));
    const int64_t runs = (int64_t)h->users * a.chunks * a.slabs, places = (int64_t)h->sms * 4;
    const dim3 joins((unsigned)(runs < places ? runs : places));
    int rc = vec ? launch_early(&h->launches, sum_kernel<A, B, true>, grid, 256, 0, 1, st, a)
                 : launch_early(&h->launches, sum_kernel<A, B, false>, grid, 256, 0, 1, st, a);
    if (rc != CO3_OK || a.chunks == 1) return rc;         // a run within one chunk needs no join
    return vec ? launch_early(&h->launches, join_kernel<B, true>, joins, 32 * JOIN_WARPS, 0, 1, st, a)
               : launch_early(&h->launches, join_kernel<B, false>, joins, 32 * JOIN_WARPS, 0, 1, st, a);
}
template <class A> int sums_to(co3_embed* h, bool vec, const SumArgs& a, cudaStream_t st) {
    if (a.to.type == CO3_F32) return sums_of<A, OF32>(h, vec, a, st);
    if (a.to.type == CO3_BF16) return sums_of<A, OBf16>(h, vec, a, st);
    return sums_of<A, OF16>(h, vec, a, st);
}

}  // namespace

extern "C" int co3_embed_forward(co3_embed* h, const co3_tokens* tokens, int64_t n_tokens, const void* table, int32_t table_type, float scale,
                                 const co3_array* out, void* cuda_stream) {
    if (!h || n_tokens < 0 || n_tokens > h->max_tokens || !embed_tokens_fine(h, tokens, n_tokens) || !(fabsf(scale) < INFINITY)) return CO3_EINVAL;
    if (!type_known(table_type) || !table || !aligned_to(table, type_width(table_type)) || !array_fine(out, h->users, n_tokens, h->dim, true)) return CO3_EINVAL;
    if (!device_is(h->device)) return CO3_EINVAL;
    if (n_tokens == 0) return CO3_OK;
    LookupArgs a;
    a.tokens = tokens_of(tokens); a.table = table; a.out = out->data; a.ou = out->user_stride; a.ot = out->token_stride;
    a.n_tokens = (uint32_t)n_tokens; a.pieces = (uint32_t)((h->dim + PIECE - 1) / PIECE); a.items = n_tokens * h->users * a.pieces;
    a.vocab = h->vocab; a.dim = (int)h->dim; a.scale = scale; a.status = h->status;
    if ((a.items + 7) / 8 > 0x7FFFFFFF) return CO3_ELIMIT;
    const dim3 grid((unsigned)((a.items + 7) / 8));
    const bool vec = h->dim % 8 == 0 && aligned_to(table, 16) && rows_aligned(out, h->users, n_tokens);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (table_type == CO3_F32) return lookup_to<OF32>(h, out->type, vec, a, grid, st);
    if (table_type == CO3_BF16) return lookup_to<OBf16>(h, out->type, vec, a, grid, st);
    return lookup_to<OF16>(h, out->type, vec, a, grid, st);
}

extern "C" int co3_embed_backward(co3_embed* h, const co3_array* dout, const co3_tokens* tokens, int64_t n_tokens, float scale,
                                  const co3_param_grad* dtable, void* cuda_stream) {
    if (!h || n_tokens < 0 || n_tokens > h->max_tokens || !embed_tokens_fine(h, tokens, n_tokens) || !(fabsf(scale) < INFINITY)) return CO3_EINVAL;
    if (!array_fine(dout, h->users, n_tokens, h->dim, false) || !grad_fine(dtable, h->users, h->vocab * h->dim)) return CO3_EINVAL;
    if (!device_is(h->device)) return CO3_EINVAL;
    if (n_tokens == 0 && dtable->accumulate) return CO3_OK;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    int bits = 1;                             // of the largest key, vocab
    while ((h->vocab >> bits) != 0) ++bits;
    const int width = type_width(dtable->type);
    SortArgs s;
    memset(&s, 0, sizeof(s));
    s.tokens = tokens_of(tokens); s.vocab = h->vocab; s.n_tokens = (uint32_t)n_tokens; s.pitch = h->pitch; s.users = h->users;
    s.cluster = n_tokens <= SORT_ALONE ? 1 : SORT_CLUSTER;
    s.passes = (bits + 7) / 8; s.digit_bits = (bits + s.passes - 1) / s.passes;
    for (int i = 0; i < 2; ++i) { s.key[i] = h->key[i]; s.place[i] = h->place[i]; }
    s.n_valid = h->n_valid; s.n_long = h->n_long; s.status = h->status;
    int64_t fill = 0;
    if (!dtable->accumulate) {
        s.zero = (uint8_t*)dtable->data; s.zero_stride = dtable->user_stride * width; s.zero_bytes = h->vocab * h->dim * width;
        const int64_t chunks = h->users * (s.zero_bytes / 65536 + 1);
        fill = chunks < 2 * h->sms ? chunks : 2 * h->sms;
        fill = (fill + s.cluster - 1) / s.cluster * s.cluster;
    }
    int rc = launch_early(&h->launches, sort_kernel, dim3((unsigned)(h->users * s.cluster + fill)), SORT_THREADS, 0, s.cluster, st, s);
    if (rc != CO3_OK || n_tokens == 0) return rc;
    SumArgs a;
    a.dout = dout->data; a.gu = dout->user_stride; a.gt = dout->token_stride;
    a.key = h->key[s.passes & 1]; a.place = h->place[s.passes & 1]; a.n_valid = h->n_valid;
    a.pitch = h->pitch; a.chunks = (uint32_t)((n_tokens + RUN - 1) / RUN); a.n_long = h->n_long; a.long_runs = h->long_runs; a.part = h->part;
    a.to = *dtable; a.dim = (int)h->dim; a.slabs = (int)((h->dim + SLAB - 1) / SLAB); a.items = (int64_t)h->users * a.chunks * a.slabs; a.scale = scale;
    if ((a.items + 7) / 8 > 0x7FFFFFFF) return CO3_ELIMIT;
    const bool vec = h->dim % 8 == 0 && rows_aligned(dout, h->users, n_tokens) && aligned_to(dtable->data, 16) &&
                     (h->users == 1 || dtable->user_stride * width % 16 == 0);
    if (dout->type == CO3_F32) return sums_to<OF32>(h, vec, a, st);
    if (dout->type == CO3_BF16) return sums_to<OBf16>(h, vec, a, st);
    return sums_to<OF16>(h, vec, a, st);
}

extern "C" int co3_embed_status(co3_embed* h, uint32_t* flags, uint64_t* bad_tokens, int32_t clear) {
    return h ? read_status(h->device, h->status, flags, bad_tokens, clear) : CO3_EINVAL;
}
extern "C" int64_t co3_embed_launch_count(const co3_embed* h) { return h ? h->launches : 0; }
