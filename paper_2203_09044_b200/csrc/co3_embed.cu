// Embedding lookup, and its gradient by sorted tokens (co3_embed_*).
//
// Gradient, three kernels: (1) a cluster of thread blocks per user sorts the user's tokens with their places by radix, stably, while
// the other SMs write the zeros of the table's gradient; (2) warps take 32 sorted places each, add the rows of equal tokens in their
// order and write a token's row where its run ends; a run that goes on into the next 32 places is finished by the warp in whose places it
// began; (3) runs that go on for longer are added by parts, and these are joined, in order again.  No sum depends on the order of an atomic.
#include "co3_ops.cuh"

namespace {

constexpr int SORT_THREADS = 1024, SORT_WARPS = 32, SORT_CLUSTER = 8, SORT_BITS = 9, SORT_BINS = 1 << SORT_BITS;
constexpr int SORT_SHARED = SORT_WARPS * SORT_BINS * 4;
constexpr int HELD = 8;                       // keys of a lane that are loaded at once, and kept for both walks where there are no more
constexpr int SORT_ALONE = 4096;              // tokens of a user that one thread block sorts by itself
constexpr int RUN = 32;                       // sorted places of a warp
constexpr int SLAB = 256;                     // columns of a thread block that joins parts
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

// A warp per 1024 columns of a row, all loads on their way before the first store.  Bound by memory: 65536 rows of 4096 bf16 142 us, 7.5 TB/s,
// some of the rows from L2; 512 rows of 768 2.2 us.  Element by element (not VEC) 65536 rows of 1001 bf16 take 112 us, 2.3 TB/s; of 1000 42.
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
    uint2* sorted[2];                         // [users][pitch] key and place; they end in [passes & 1]
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

// Zeros for chunk `number` of the users' parts, counted over the users; a part may begin and end at any element.  A chunk each to blocks
// that come and go: 786 MB in 108 us, 7.3 TB/s; the same chunks dealt out to blocks that stay 129 us, since not all SMs store equally fast.
constexpr int FILL_EACH = 4;
constexpr int64_t FILL_CHUNK = FILL_EACH * SORT_THREADS * 32;
__host__ __device__ inline int64_t fill_chunks(int64_t bytes) { return (bytes + 31 + FILL_CHUNK - 1) / FILL_CHUNK; }      // of a user
__device__ void fill_zeros(const SortArgs& a, int64_t number) {
    const int64_t per_user = fill_chunks(a.zero_bytes), user = number / per_user, j = number - user * per_user;
    if (user >= a.users) return;
    uint8_t* const begin = a.zero + user * a.zero_stride, *const end = begin + a.zero_bytes;
    uint8_t* const whole = (uint8_t*)((uintptr_t)begin & ~(uintptr_t)31);           // chunks count from here
    uint8_t *p = whole + j * FILL_CHUNK, *q = p + FILL_CHUNK;
    if (p >= begin && q <= end) {
#pragma unroll
        for (int i = 0; i < FILL_EACH; ++i)
            asm volatile("st.global.v8.b32 [%0], {%1,%1,%1,%1,%1,%1,%1,%1};" :: "l"(p + (i * SORT_THREADS + threadIdx.x) * 32), "r"(0) : "memory");
        return;
    }
    if (q > end) q = end;
    if (p < begin) {                          // the first chunk's bytes before the first whole 32
        uint8_t* const edge = whole + 32 < q ? whole + 32 : q;
        for (uint8_t* b = begin + 2 * threadIdx.x; b < edge; b += 2 * SORT_THREADS) *(uint16_t*)b = 0;
        p = whole + 32;
    }
    if (p >= q) return;
    const int64_t words = (q - p) / 16;
    for (int64_t w = threadIdx.x; w < words; w += SORT_THREADS) ((uint4*)p)[w] = make_uint4(0, 0, 0, 0);
    for (uint8_t* b = p + words * 16 + 2 * threadIdx.x; b < q; b += 2 * SORT_THREADS) *(uint16_t*)b = 0;
}

// The lanes whose digits (of `bits` bits; lanes that are not here have the bit above set) are this lane's.
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, int bits) {
    uint32_t same = 0xffffffffu;
    for (int b = 0; b <= bits; ++b) {
        const bool set = digit >> b & 1;
        const uint32_t with = __ballot_sync(0xffffffffu, set);
        same &= set ? with : ~with;
    }
    return same;
}

// Stable sort by radix, nine bits a pass at most: a warp ranks its keys by ballots and counts them, the counts of all warps and blocks are
// summed by digit, and each key's place is known.  Bound by the steps that wait for one another: 62 tokens 9 us, 2000 of 8 users 12,
// 65536 36, all of it behind the zeros where there are any (524 MB: 75 us).
__global__ void __launch_bounds__(SORT_THREADS, 2) sort_kernel(const __grid_constant__ SortArgs a) {
    extern __shared__ uint32_t hist[];        // [SORT_WARPS][bins]
    __shared__ uint32_t totals[SORT_BINS + 1], base[SORT_BINS], warp_sums[SORT_BINS / 32];
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t user = blockIdx.x / a.cluster, rank = blockIdx.x - user * a.cluster;
    let_next_start();
    wait_for_previous();
    if (user >= (uint32_t)a.users) {
        fill_zeros(a, (int64_t)blockIdx.x - a.users * a.cluster);
        return;
    }
    if (blockIdx.x == 0 && tid == 0) *a.n_long = 0;
    const uint32_t n = a.n_tokens;
    const uint32_t per_block = ((n + a.cluster - 1) / a.cluster + 1023) / 1024 * 1024, per_warp = per_block / 32;
    const uint64_t first = (uint64_t)rank * per_block + (uint64_t)warp * per_warp;
    const uint32_t begin = first < n ? (uint32_t)first : n, end = first + per_warp < n ? (uint32_t)(first + per_warp) : n;
    const uint32_t bins = 1u << a.digit_bits;
    const uint32_t below = (1u << lane) - 1u;
    uint32_t* const mine = hist + warp * bins;
    for (int pass = 0; pass < a.passes; ++pass) {
        const uint2* in = a.sorted[pass & 1] + (int64_t)user * a.pitch;
        uint2* out = a.sorted[~pass & 1] + (int64_t)user * a.pitch;
        const int shift = pass * a.digit_bits;
        uint32_t held[HELD], place[HELD], nth[HELD], valid = 0;
        // the next HELD * 32 keys of the warp; those of the first pass come from the tokens, and the ones that are none last
        auto load = [&](uint32_t i0, bool count) {
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                const uint32_t i = i0 + 32 * h + lane;
                place[h] = i;
                if (i >= end) held[h] = 0xFFFFFFFFu;
                else if (pass) {
                    const uint2 x = __ldcg(in + i);
                    held[h] = x.x;
                    place[h] = x.y;
                } else {
                    const int64_t token = token_at(a.tokens, user, i);
                    held[h] = token < 0 || token >= a.vocab ? (uint32_t)a.vocab : (uint32_t)token;
                    if (count && token >= a.vocab) { atomicAdd(&a.status->bad_tokens, 1ull); atomicOr(&a.status->flags, CO3_FLAG_TOKEN); }
                    valid += count && held[h] != (uint32_t)a.vocab;
                }
            }
        };
        for (uint32_t b = lane; b < bins; b += 32) mine[b] = 0;
        if (tid == 0) totals[SORT_BINS] = 0;
        __syncthreads();
        for (uint32_t i0 = begin; i0 < end; i0 += 32 * HELD) {
            load(i0, true);
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                if (i0 + 32 * h >= end) break;
                const bool here = i0 + 32 * h + lane < end;
                const uint32_t digit = here ? held[h] >> shift & (bins - 1) : bins, same = same_digit(digit, a.digit_bits);
                const uint32_t ahead = here ? mine[digit] : 0;
                nth[h] = ahead + __popc(same & below);
                __syncwarp();
                if (here && !(same & below)) mine[digit] = ahead + __popc(same);
                __syncwarp();
            }
        }
        if (pass == 0) {
#pragma unroll
            for (int o = 16; o; o >>= 1) valid += __shfl_xor_sync(0xffffffffu, valid, o);
            if (lane == 0 && valid) atomicAdd(&totals[SORT_BINS], valid);
        }
        __syncthreads();
        if (tid < bins) {                     // where each warp's part of a digit begins within the block's
            uint32_t s = 0;
#pragma unroll 8
            for (int w = 0; w < SORT_WARPS; ++w) { const uint32_t c = hist[w * bins + tid]; hist[w * bins + tid] = s; s += c; }
            totals[tid] = s;
        }
        if (a.cluster > 1) cluster_barrier();
        else __syncthreads();
        uint32_t all = 0, before = 0;
        if (tid < bins) {
            if (a.cluster == 1) all = totals[tid];
            else {
                uint32_t c[SORT_CLUSTER];
#pragma unroll
                for (int r = 0; r < SORT_CLUSTER; ++r) c[r] = peer_word(shared_at(&totals[tid]), r);
#pragma unroll
                for (int r = 0; r < SORT_CLUSTER; ++r) { if (r < (int)rank) before += c[r]; all += c[r]; }
            }
        }
        if (pass == 0 && rank == 0 && tid == SORT_THREADS - 1) {
            uint32_t s = 0;
            for (int r = 0; r < a.cluster; ++r) s += a.cluster > 1 ? peer_word(shared_at(&totals[SORT_BINS]), r) : totals[SORT_BINS];
            a.n_valid[user] = s;
        }
        uint32_t up = all;                    // places of the smaller digits, over all blocks
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, up, o); if ((int)lane >= o) up += v; }
        if (warp < SORT_BINS / 32 && lane == 31) warp_sums[warp] = up;
        __syncthreads();
        if (tid < bins) {
            for (uint32_t w = 0; w < warp; ++w) before += warp_sums[w];
            base[tid] = before + up - all;
        }
        __syncthreads();
        const bool again = per_warp > 32 * HELD;          // the ranks of the last HELD * 32 keys alone are still there
        for (uint32_t i0 = begin; i0 < end; i0 += 32 * HELD) {
            if (again) load(i0, false);
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                if (i0 + 32 * h >= end) break;
                const bool here = i0 + 32 * h + lane < end;
                const uint32_t digit = here ? held[h] >> shift & (bins - 1) : bins;
                uint32_t to = here ? base[digit] + mine[digit] : 0;
                if (again) {
                    const uint32_t same = same_digit(digit, a.digit_bits);
                    __syncwarp();
                    if (here && !(same & below)) mine[digit] += __popc(same);
                    __syncwarp();
                    to += __popc(same & below);
                } else to += nth[h];
                if (here) __stcg(out + to, make_uint2(held[h], place[h]));
            }
        }
        if (a.cluster > 1) cluster_barrier();  // also: nobody reads another block's totals any more
        else __syncthreads();
    }
}

// ---- sums ------------------------------------------------------------------------------------------------------------------
struct SumArgs {
    const void* dout;
    int64_t gu, gt;
    const uint2* sorted;                      // [users][pitch] key and place
    const uint32_t* n_valid;
    uint32_t pitch, chunks;                   // of a user
    uint32_t* n_long;
    uint32_t* long_runs;                      // [users * chunks]: user * chunks + chunk in which a longer run begins
    float* part;                              // [users * chunks][2][dim]: of a run that began before the chunk, of one that goes on after it
    co3_param_grad to;
    int64_t items;
    int dim, slabs;
    float scale;
};

// How a warp takes a row: WIDE eight neighbouring columns a lane, 16 bytes of 16-bit numbers; QUADS and PAIRS four and two, for few rows, and
// for gradients that begin anywhere; SINGLES every 32nd, two of them, for rows that begin anywhere.
enum Take { WIDE, QUADS, PAIRS, SINGLES };
template <int TAKE> constexpr int PER_LANE = TAKE == WIDE ? 8 : TAKE == QUADS ? 4 : 2;
template <int TAKE> constexpr int COLUMNS = 32 * PER_LANE<TAKE>;

__device__ __forceinline__ void add_pair(float& a, float& b, float x, float y) {      // two sums in one instruction
    asm("{\n\t.reg .b64 s, x;\n\tmov.b64 s, {%0, %1};\n\tmov.b64 x, {%2, %3};\n\tadd.rn.f32x2 s, s, x;\n\tmov.b64 {%0, %1}, s;\n\t}" : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}

template <class A, int TAKE> struct RowPart {
    typedef typename A::type type;
    static constexpr int N = PER_LANE<TAKE>, BYTES = N * sizeof(type);
    alignas(BYTES < 16 ? BYTES : 16) type x[N];
    __device__ __forceinline__ void load(const type* p, int columns) {        // columns: that are left from the lane's first
        if (TAKE == SINGLES) {
            if (columns > 0) x[0] = p[0];
            if (columns > 32) x[1] = p[32];
        } else if (columns > 0) {
            if (BYTES == 4) *(uint32_t*)x = __ldcs((const uint32_t*)p);
            else if (BYTES == 8) *(uint2*)x = __ldcs((const uint2*)p);
            else
#pragma unroll
                for (int i = 0; i < BYTES / 16; ++i) ((uint4*)x)[i] = __ldcs((const uint4*)p + i);
        }
    }
    __device__ __forceinline__ void add(float* s) const {
        float f[N];
        if constexpr (sizeof(type) == 4) {
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = A::get(x[k]);
        } else {
#pragma unroll
            for (int k = 0; k < N; k += 2) A::unpack2(*(const uint32_t*)(x + k), f[k], f[k + 1]);
        }
#pragma unroll
        for (int k = 0; k < N; k += 2) add_pair(s[k], s[k + 1], f[k], f[k + 1]);
    }
};

template <int N> struct Sums { float x[N]; };

// A run's sum to its token's row, from the lane's first column on, of which `left` are left; `part`: to its part's place instead.  (As a call, with
// its arguments moved to where calls have them, 65536 rows took 192 us with sort and zeros instead of 182.)
template <class B, int TAKE>
__device__ __forceinline__ void put_run(typename B::type* p, float* part, int left, float scale, int accumulate, Sums<PER_LANE<TAKE>> s) {
    constexpr int N = PER_LANE<TAKE>, STEP = TAKE == SINGLES ? 32 : 1;
    if (left <= 0) return;
    if (part) {
#pragma unroll
        for (int k = 0; k < N; ++k) if (STEP * k < left) part[STEP * k] = s.x[k];
        return;
    }
#pragma unroll
    for (int k = 0; k < N; ++k) s.x[k] *= scale;
    if constexpr (TAKE == WIDE) {             // the gradient's rows begin at multiples of 16 bytes
        if (accumulate) {
            float o[8];
            load8<B>(p, o);
#pragma unroll
            for (int k = 0; k < 8; ++k) s.x[k] += o[k];
        }
        store8<B>(p, s.x);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (TAKE != SINGLES || STEP * k < left) p[STEP * k] = B::put(accumulate ? B::get(p[STEP * k]) + s.x[k] : s.x[k]);
    }
}

// Reads each row of dout once, 512 bytes of it at a time, and writes a token's row once.  65536 rows of 2048 bf16 to 39217: 82 us, 5.2 TB/s; 12500
// of 768 to as many of 32 bits at an odd element: 22 us, while the zeros before it still go to memory.
template <class A, class B, int TAKE>
__global__ void __launch_bounds__(256) sum_kernel(const __grid_constant__ SumArgs a) {
    // Rows whose loads are in flight while as many are added: with 16 bytes a lane four (65536 rows of 2048 bf16 182 us with sort and zeros, eight 196), with less
    // eight (8 users' 2000 of 768 133, four 136).
    constexpr int AT_ONCE = RowPart<A, TAKE>::BYTES >= 16 ? 4 : 8;
    constexpr uint32_t NONE = 0xFFFFFFFFu;
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    let_next_start();
    wait_for_previous();
    if (item >= a.items) return;
    const uint32_t at = (uint32_t)(item / a.slabs);       // user * chunks + chunk
    const int slab = (int)(item - (int64_t)at * a.slabs);
    const uint32_t user = at / a.chunks, chunk = at - user * a.chunks, n = a.n_valid[user], i0 = chunk * RUN;
    if (i0 >= n) return;
    const uint2* sorted = a.sorted + (int64_t)user * a.pitch;
    auto at_place = [&](uint32_t i) { return i < n ? sorted[i] : make_uint2(NONE, 0); };
    const uint2 one = at_place(i0 + lane), two = at_place(i0 + RUN + lane);
    const uint32_t key = one.x, key2 = two.x, far = i0 > RUN ? sorted[i0 - RUN - 1].x : NONE, before = i0 ? sorted[i0 - 1].x : NONE, beyond = at_place(i0 + 2 * RUN).x;
    const uint32_t head = __shfl_sync(0xffffffffu, key, 0), tail = __shfl_sync(0xffffffffu, key, RUN - 1), next = __shfl_sync(0xffffffffu, key2, 0);
    int total = n - i0 < RUN ? (int)(n - i0) : RUN, skip = 0, led = 0, last_slot = -1;       // led: places of a run that is added by parts
    const bool began_before = before == head, all_one = began_before && tail == head;
    if (began_before) {
        const int same = __popc(__ballot_sync(0xffffffffu, key == head));
        if (far == head || (all_one && next == head)) led = same;
        else skip = same;                     // the warp before finishes it
    }
    if (next == tail && next != NONE && !all_one) {       // the last run goes on, and began here
        const int more = __popc(__ballot_sync(0xffffffffu, key2 == tail));
        if (more == RUN && beyond == tail) last_slot = 1;
        else total = RUN + more;
    }
    if (skip >= total) return;
    if (last_slot == 1 && slab == 0 && lane == 0) a.long_runs[atomicAdd(a.n_long, 1u)] = at;
    // where a run ends: bit i of the 64 places
    const uint32_t after = __shfl_down_sync(0xffffffffu, key, 1), after2 = __shfl_down_sync(0xffffffffu, key2, 1);
    const uint64_t ends = (uint64_t)__ballot_sync(0xffffffffu, key2 != after2) << 32 | __ballot_sync(0xffffffffu, key != (lane == 31 ? next : after)) | 1ull << (total - 1);
    const int column = slab * COLUMNS<TAKE> + (TAKE == SINGLES ? lane : lane * PER_LANE<TAKE>);
    const typename A::type* rows = (const typename A::type*)a.dout + user * a.gu + column;
    typename B::type* const to = (typename B::type*)a.to.data + user * a.to.user_stride + column;
    Sums<PER_LANE<TAKE>> sum;
#pragma unroll
    for (int k = 0; k < PER_LANE<TAKE>; ++k) sum.x[k] = 0.0f;
    RowPart<A, TAKE> now[AT_ONCE], coming[AT_ONCE];
    auto fetch = [&](RowPart<A, TAKE>(&x)[AT_ONCE], int e0) {
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) {
            const uint32_t place = __shfl_sync(0xffffffffu, e0 + e < RUN ? one.y : two.y, (e0 + e) & 31);
            if (e0 + e < total) x[e].load(rows + (int64_t)place * a.gt, a.dim - column);
        }
    };
    fetch(now, skip);
    for (int e0 = skip; e0 < total; e0 += AT_ONCE) {
        fetch(coming, e0 + AT_ONCE);
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) {
            const int i = e0 + e;
            if (i >= total) break;
            now[e].add(sum.x);
            if (!(ends >> i & 1)) continue;
            const uint32_t mine = __shfl_sync(0xffffffffu, i < RUN ? key : key2, i & 31);
            const int slot = i < led ? 0 : i + 1 == total ? last_slot : -1;
            put_run<B, TAKE>(to + (int64_t)mine * a.dim, slot < 0 ? nullptr : a.part + ((int64_t)at * 2 + slot) * a.dim + column, a.dim - column, a.scale, a.to.accumulate, sum);
#pragma unroll
            for (int k = 0; k < PER_LANE<TAKE>; ++k) sum.x[k] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) now[e] = coming[e];
    }
}

// The runs that were added by parts, each by a thread block: its warps add a stretch of the parts each, the stretches are added in order.
template <class B>
__global__ void __launch_bounds__(32 * JOIN_WARPS) join_kernel(const __grid_constant__ SumArgs a) {
    __shared__ float sh[JOIN_WARPS][SLAB];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slabs = (a.dim + SLAB - 1) / SLAB;
    let_next_start();
    wait_for_previous();
    const int64_t items = (int64_t)*a.n_long * slabs;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t at = a.long_runs[item / slabs];
        const int column = (int)(item % slabs) * SLAB;
        const uint32_t user = at / a.chunks, chunk = at - user * a.chunks, n = a.n_valid[user];
        const uint2* sorted = a.sorted + (int64_t)user * a.pitch;
        const uint32_t token = sorted[chunk * RUN + RUN - 1].x;
        uint32_t lo = (chunk + 1) * RUN, hi = n;          // the run ends before the first larger key, among lo .. hi: 32 looks at once
        while (lo < hi) {
            const uint32_t step = (hi - lo + 31) / 32, i = lo + lane * step;
            const int same = __popc(__ballot_sync(0xffffffffu, i < hi && sorted[i].x == token));
            if (!same) break;
            hi = hi - lo < same * step ? hi : lo + same * step;
            lo += (same - 1) * step + 1;
        }
        const uint32_t parts = (lo - 1) / RUN - chunk + 1, each = (parts + JOIN_WARPS - 1) / JOIN_WARPS;
        const uint32_t p0 = warp * each < parts ? warp * each : parts, p1 = p0 + each < parts ? p0 + each : parts;
        float s[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] = 0.0f;
#pragma unroll 4
        for (uint32_t p = p0; p < p1; ++p) {
            const float* part = a.part + (((int64_t)at + p) * 2 + (p ? 0 : 1)) * a.dim + column + lane;
#pragma unroll
            for (int k = 0; k < 8; ++k) if (column + lane + 32 * k < a.dim) s[k] += part[32 * k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sh[warp][lane + 32 * k] = s[k];
        __syncthreads();
        float x = 0.0f;                       // a column a thread
        for (int w = 0; w < JOIN_WARPS; ++w) x += sh[w][threadIdx.x];
        if (column + (int)threadIdx.x < a.dim) {
            typename B::type* p = (typename B::type*)a.to.data + user * a.to.user_stride + (int64_t)token * a.dim + column + threadIdx.x;
            x *= a.scale;
            *p = B::put(a.to.accumulate ? B::get(*p) + x : x);
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
    uint2* sorted[2];
    uint32_t *n_valid, *n_long, *long_runs;
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
        const size_t pairs = 8 * (size_t)h->pitch * n_users, runs = (size_t)h->chunks * n_users;
        const size_t o_status = part(sizeof(OpsStatus)), o_one = part(pairs), o_two = part(pairs);
        const size_t o_valid = part(4 * (size_t)n_users), o_count = part(4), o_long = part(4 * runs), o_part = part(runs * 2 * dim * 4);
        if (cudaMalloc(&h->slab, at) != cudaSuccess) { h->slab = nullptr; rc = CO3_ENOMEM; }
        else {
            char* base = (char*)h->slab;
            h->status = (OpsStatus*)(base + o_status);
            h->sorted[0] = (uint2*)(base + o_one); h->sorted[1] = (uint2*)(base + o_two);
            h->n_valid = (uint32_t*)(base + o_valid); h->n_long = (uint32_t*)(base + o_count); h->long_runs = (uint32_t*)(base + o_long);
            h->part = (float*)(base + o_part);
            // the sort's counts in shared memory
            if (cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SORT_SHARED) != cudaSuccess) rc = CO3_ECUDA;
            else if (cudaMemset(h->status, 0, sizeof(OpsStatus)) != cudaSuccess || cudaStreamSynchronize(nullptr) != cudaSuccess) rc = CO3_ECUDA;
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
    return k->data && aligned_to(k->data, k->type == CO3_I32 ? 4 : 8) && stride_fine(h->users, k->user_stride) && stride_fine(n, k->token_stride);
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
template <class A, class B> int sums_of(co3_embed* h, int take, SumArgs a, cudaStream_t st) {
    const int columns = take == WIDE ? COLUMNS<WIDE> : take == QUADS ? COLUMNS<QUADS> : COLUMNS<PAIRS>;
    a.slabs = (a.dim + columns - 1) / columns;
    a.items = (int64_t)h->users * a.chunks * a.slabs;
    if ((a.items + 7) / 8 > 0x7FFFFFFF) return CO3_ELIMIT;
    const dim3 grid((unsigned)((a.items + 7) / 8));
    int rc = take == WIDE ? launch_early(&h->launches, sum_kernel<A, B, WIDE>, grid, 256, 0, 1, st, a)
             : take == QUADS ? launch_early(&h->launches, sum_kernel<A, B, QUADS>, grid, 256, 0, 1, st, a)
             : take == PAIRS ? launch_early(&h->launches, sum_kernel<A, B, PAIRS>, grid, 256, 0, 1, st, a)
                             : launch_early(&h->launches, sum_kernel<A, B, SINGLES>, grid, 256, 0, 1, st, a);
    if (rc != CO3_OK || a.chunks <= 2) return rc;         // a run that is added by parts lies in three chunks at least
    const int64_t runs = (int64_t)h->users * a.chunks * ((a.dim + SLAB - 1) / SLAB), places = (int64_t)h->sms * 4;
    return launch_early(&h->launches, join_kernel<B>, dim3((unsigned)(runs < places ? runs : places)), 32 * JOIN_WARPS, 0, 1, st, a);
}
template <class A> int sums_to(co3_embed* h, int take, const SumArgs& a, cudaStream_t st) {
    if (a.to.type == CO3_F32) return sums_of<A, OF32>(h, take, a, st);
    if (a.to.type == CO3_BF16) return sums_of<A, OBf16>(h, take, a, st);
    return sums_of<A, OF16>(h, take, a, st);
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
    s.passes = (bits + SORT_BITS - 1) / SORT_BITS; s.digit_bits = (bits + s.passes - 1) / s.passes;
    s.sorted[0] = h->sorted[0]; s.sorted[1] = h->sorted[1];
    s.n_valid = h->n_valid; s.n_long = h->n_long; s.status = h->status;
    int64_t fill = 0;
    if (!dtable->accumulate) {
        s.zero = (uint8_t*)dtable->data; s.zero_stride = dtable->user_stride * width; s.zero_bytes = h->vocab * h->dim * width;
        fill = (h->users * fill_chunks(s.zero_bytes) + s.cluster - 1) / s.cluster * s.cluster;
        if (fill > 0x7FFF0000) return CO3_ELIMIT;
    }
    int rc = launch_early(&h->launches, sort_kernel, dim3((unsigned)(h->users * s.cluster + fill)), SORT_THREADS, SORT_SHARED, s.cluster, st, s);
    if (rc != CO3_OK || n_tokens == 0) return rc;
    SumArgs a;
    a.dout = dout->data; a.gu = dout->user_stride; a.gt = dout->token_stride;
    a.sorted = h->sorted[s.passes & 1]; a.n_valid = h->n_valid;
    a.pitch = h->pitch; a.chunks = (uint32_t)((n_tokens + RUN - 1) / RUN); a.n_long = h->n_long; a.long_runs = h->long_runs; a.part = h->part;
    a.to = *dtable; a.dim = (int)h->dim; a.scale = scale;
    // As many columns a lane as the arrays' beginnings allow and as leave more warps than half of what the device has places for.
    const int in = type_width(dout->type);
    auto begins = [&](int bytes) {
        bytes = bytes < 16 ? bytes : 16;
        return aligned_to(dout->data, bytes) && (n_tokens <= 1 || dout->token_stride * in % bytes == 0) && (h->users == 1 || dout->user_stride * in % bytes == 0);
    };
    auto warps = [&](int columns) { return (int64_t)h->users * a.chunks * ((h->dim + columns - 1) / columns) >= (int64_t)h->sms * 16; };
    int take = SINGLES;
    if (h->dim % 2 == 0 && begins(2 * in)) take = PAIRS;
    if (h->dim % 4 == 0 && begins(4 * in) && warps(COLUMNS<QUADS>)) take = QUADS;
    if (h->dim % 8 == 0 && begins(16) && aligned_to(dtable->data, 16) && (h->users == 1 || dtable->user_stride * width % 16 == 0) && warps(COLUMNS<WIDE>)) take = WIDE;
    if (dout->type == CO3_F32) return sums_to<OF32>(h, take, a, st);
    if (dout->type == CO3_BF16) return sums_to<OBf16>(h, take, a, st);
    return sums_to<OF16>(h, take, a, st);
}

extern "C" int co3_embed_status(co3_embed* h, uint32_t* flags, uint64_t* bad_tokens, int32_t clear) {
    return h ? read_status(h->device, h->status, flags, bad_tokens, clear) : CO3_EINVAL;
}
extern "C" int64_t co3_embed_launch_count(const co3_embed* h) { return h ? h->launches : 0; }
