// Losses of tokens over a large vocabulary, and their gradients, without the logits (co3_token_loss_*).
//
// All products run through one kernel on the tensor cores: pairs of thread blocks (two SMs) on tiles of 256 x 256, operands brought by TMA
// into a ring of stages, accumulators in tensor memory, two of them, so that the products of the next tile run while sixteen warps of
// each block work on the last one:
//   STATS   z = H W^T                     -> per row and 256 columns: largest logit, sum of exponentials, weighted target logits
//   DZ      z again, for a piece of the vocabulary -> dz, in 16 bits (and its remainder in 16 more, for 32-bit gradients of the weight)
//   DHIDDEN dz W    over the piece        -> 32-bit sums
//   DWEIGHT dz^T H  over a user's tokens  -> the user's gradient
// Before them the tokens that have a target (and, for a gradient, a dloss other than 0) are packed side by side, users at multiples of 64 rows
// with zero rows between, so that the others cost nothing and no other user's rows reach a sum.
#include <cuda.h>

#include "co3_ops.cuh"

namespace {

constexpr int TILE = 256;                     // rows and columns of a pair's tile
constexpr int KB = 64;                        // depth of a stage: 128 bytes, one swizzle span
constexpr int STAGES = 5;                     // six take as long: what the products wait for is the way from L2 to the SMs
constexpr int HALF_BYTES = 128 * KB * 2;      // one operand's part of a thread block and stage
constexpr int STAGE_BYTES = 2 * HALF_BYTES;
constexpr int FIRST_EPI = 2;                  // warps: loads, products, then those for the tiles' ends
// Each has 32 rows and 64 columns of a tile.  With half as many and 128 columns an end took 4000 (STATS) to 10000 cycles, nearly all of it
// latency of instructions that wait for one another, against the 6144 that the products of a tile take at a depth of 768.
constexpr int EPI_WARPS = 16;
constexpr int GEMM_THREADS = 32 * (FIRST_EPI + EPI_WARPS);
constexpr int OUT_BYTES = EPI_WARPS * 4096;   // a box of 32 rows of 128 bytes for each
constexpr int GEMM_SHARED = 1024 + STAGES * STAGE_BYTES + OUT_BYTES + 256;
constexpr int ALIGN_ROWS = 64;                // a user's packed rows begin at a multiple of these
constexpr int MAX_TOP = 128;
constexpr int SPAN = 64;                      // columns of a warp
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

enum Mode { STATS, DZ, DHIDDEN, DWEIGHT };

// A wait gives up after so long: no call's longest one takes a tenth of it.
constexpr unsigned long long WAIT_LIMIT_NS = 4000000000ull;

struct Packed {                               // what the packing leaves, on the device
    int32_t* offset;                          // [users + 1] first packed row of each user
    int32_t* count;                           // [users]
    float* up;                                // [users] power of two that dz is scaled by
    int32_t* row_token;                       // [rows] user * tokens + t, -1: none
    int32_t* token_row;                       // [users * tokens], -1: no target
    float* row_c;                             // [rows] factor of dz, scaled
    float* row_lse;                           // [rows] in powers of two
    int32_t* row_target;                      // [rows] (one entry a token)
};

struct GemmArgs {
    CUtensorMap a, b, a_low;                  // a_low: the remainders of dz
    CUtensorMap out, out_low;                 // what a tile's end stores: dz and its remainder, partial, or dweight
    Packed p;
    OpsStatus* status;
    int users, vocab, dim;
    int v0, columns;                          // first row of the piece, its columns
    int splits, terms;
    int64_t rows;                             // pitch of arrays [..][rows]
    float scale;                              // log2(e) / temperature
    float2* stats;                            // [tiles][rows] largest, sum
    float* dots;                              // [tiles][rows]
    const int32_t* entry; const float* entry_q; const uint8_t* entry_first;      // [tokens][top], [tokens][top], [tokens][tiles]
    int top, tiles;                           // tiles of the vocabulary
    int add;                                  // to what partial [splits][rows][dim] holds
    co3_param_grad dw;
    int dw_wide;                              // rows of dweight begin at multiples of 16 bytes and are written
};

__device__ __forceinline__ uint32_t shared_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t at_rank(uint32_t at, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(rank));
    return r;
}
__device__ __forceinline__ void bar_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, int bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
// Orders what this thread block does, no more: what the other side waits for is that tensor memory has been read, which the tcgen05 fences
// order.  (With a release for the whole cluster a warp waited here for its stores to memory, 2000 cycles a tile and more.)
__device__ __forceinline__ void bar_arrive_far(uint32_t far) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" :: "r"(far) : "memory");
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
    unsigned long long since = 0;
    for (uint32_t i = 1;; ++i) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
        if (i % 256 == 0) {
            unsigned long long now;
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
            if (!since) since = now;
            else if (now - since > WAIT_LIMIT_NS) return false;
        }
    }
}
// A box of 64 x 64 of the matrix, whose barrier is the pair's first thread block's.
__device__ __forceinline__ void tma_load(uint32_t to, const CUtensorMap* map, int x, int y, uint32_t far_bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(to), "l"(map), "r"(x), "r"(y), "r"(far_bar) : "memory");
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add) : "memory");
}
// Both blocks' barriers at this place, once the products so far are done.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" :: "r"(bar), "h"((uint16_t)3) : "memory");
}
// 32 (16) columns of the warp's 32 rows.  They are there after tmem_loaded or tmem_loaded_too, which name the same registers, so that
// nothing is done with them before.
__device__ __forceinline__ void tmem_load32(uint32_t at, float* x) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]), "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15]), "=f"(x[16]), "=f"(x[17]), "=f"(x[18]), "=f"(x[19]), "=f"(x[20]), "=f"(x[21]), "=f"(x[22]), "=f"(x[23]), "=f"(x[24]), "=f"(x[25]), "=f"(x[26]), "=f"(x[27]), "=f"(x[28]), "=f"(x[29]), "=f"(x[30]), "=f"(x[31])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_load16(uint32_t at, float* x) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]), "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_loaded32(float* x) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]), "+f"(x[8]), "+f"(x[9]), "+f"(x[10]), "+f"(x[11]), "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15]), "+f"(x[16]), "+f"(x[17]), "+f"(x[18]), "+f"(x[19]), "+f"(x[20]), "+f"(x[21]), "+f"(x[22]), "+f"(x[23]), "+f"(x[24]), "+f"(x[25]), "+f"(x[26]), "+f"(x[27]), "+f"(x[28]), "+f"(x[29]), "+f"(x[30]), "+f"(x[31]) :: "memory");
}
__device__ __forceinline__ void tmem_loaded16(float* x) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]), "+f"(x[8]), "+f"(x[9]), "+f"(x[10]), "+f"(x[11]), "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15]) :: "memory");
}
__device__ __forceinline__ void tmem_loaded32_too(float* x) {
    asm volatile("" : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]), "+f"(x[8]), "+f"(x[9]), "+f"(x[10]), "+f"(x[11]), "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15]), "+f"(x[16]), "+f"(x[17]), "+f"(x[18]), "+f"(x[19]), "+f"(x[20]), "+f"(x[21]), "+f"(x[22]), "+f"(x[23]), "+f"(x[24]), "+f"(x[25]), "+f"(x[26]), "+f"(x[27]), "+f"(x[28]), "+f"(x[29]), "+f"(x[30]), "+f"(x[31]) :: "memory");
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Shared-memory descriptor of an operand with 128-byte swizzle: rows of 128 bytes, eight of them (1024 bytes) an atom.  Depth along the
// rows (ALONG): atoms follow one another along the operand's other dimension.  Depth across them: atoms follow along the
// depth, and 64 elements further along the other dimension begin 8192 bytes on.
template <bool ALONG> __device__ __forceinline__ uint64_t operand_desc(uint32_t at) {
    const uint64_t leading = ALONG ? 1 : 8192 >> 4, stride = 1024 >> 4;
    return (uint64_t)(at >> 4 & 0x3FFF) | leading << 16 | stride << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

struct TileWork {                             // one tile of one product
    int m, n, k0, k1;                         // first row and column of the tile, first and last stage of the depth
    int user, split;
};

// Tile number i, or false where there are no more.  Rows vary fastest where a weight is read once for all of them.
template <int MODE> __device__ __forceinline__ bool tile_at(const GemmArgs& a, int rows, int64_t i, TileWork& w) {
    w.user = w.split = 0;
    w.k0 = 0;
    if (MODE == STATS || MODE == DZ) {
        const int mt = (rows + TILE - 1) / TILE;
        if (i >= (int64_t)mt * ((a.columns + TILE - 1) / TILE)) return false;
        w.n = (int)(i / mt) * TILE;
        w.m = (int)(i % mt) * TILE;
        w.k1 = (a.dim + KB - 1) / KB;
    } else if (MODE == DHIDDEN) {
        const int mt = (rows + TILE - 1) / TILE, nt = (a.dim + TILE - 1) / TILE, kb = (a.columns + KB - 1) / KB;
        if (i >= (int64_t)mt * nt * a.splits) return false;
        w.split = (int)(i / ((int64_t)mt * nt));
        i -= (int64_t)w.split * mt * nt;
        w.m = (int)(i / nt) * TILE;
        w.n = (int)(i % nt) * TILE;
        w.k0 = (int)((int64_t)kb * w.split / a.splits);
        w.k1 = (int)((int64_t)kb * (w.split + 1) / a.splits);
    } else {
        const int mt = (a.columns + TILE - 1) / TILE, nt = (a.dim + TILE - 1) / TILE;
        if (i >= (int64_t)mt * nt * a.users) return false;
        w.user = (int)(i / ((int64_t)mt * nt));
        i -= (int64_t)w.user * mt * nt;
        w.m = (int)(i / nt) * TILE;
        w.n = (int)(i % nt) * TILE;
        w.k1 = (a.p.offset[w.user + 1] - a.p.offset[w.user]) / KB * a.terms;
    }
    return true;
}

// ---- the tiles' ends: warp `part` of four has 32 rows, `quarter` says which 64 of the 256 columns; a lane has a row -----------------------
// The entries of a row that lie in its 64 columns, in order.
template <bool ONE> struct Entries {
    const int32_t* entry; const float* q;
    int left, next;
    float next_q;
    __device__ __forceinline__ void begin(const GemmArgs& a, bool here, int64_t row, int first_column) {
        next = 0x7FFFFFFF;
        next_q = 1.0f;
        left = 0;
        if (!here) return;
        if (ONE) {
            const int t = a.p.row_target[row];
            if (t >= first_column) next = t;
        } else {
            const int64_t token = a.p.row_token[row];
            if (token < 0) return;
            const int skip = a.entry_first[token * a.tiles + first_column / TILE];
            left = a.top - skip;
            entry = a.entry + token * a.top + skip;
            q = a.entry_q + token * a.top + skip;
            fetch();
            while (next < first_column) advance();        // those of the tile's columns before
        }
    }
    __device__ __forceinline__ void fetch() {
        if (left > 0) { next = *entry; next_q = *q; } else next = 0x7FFFFFFF;
    }
    __device__ __forceinline__ void advance() {
        if (ONE) { next = 0x7FFFFFFF; return; }
        --left; ++entry; ++q;
        fetch();
    }
};

// The entries among columns C .. C + 31 of the 64.  Written so that no index into the array is left, which would put it into local memory
// (the kernel of the statistics then took 1.5 times as long).
__device__ __forceinline__ void take_if(int at, int k, float x, float& z) {
    asm("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, %2;\n\tselp.f32 %0, %3, %0, p;\n\t}" : "+f"(z) : "r"(at), "r"(k), "f"(x));
}
__device__ __forceinline__ void subtract_if(int at, int k, float q, float& x) {
    asm("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, %2;\n\t@p sub.rn.f32 %0, %0, %3;\n\t}" : "+f"(x) : "r"(at), "r"(k), "f"(q));
}
template <int C, bool ONE> __device__ __forceinline__ void take_entries(const float (&x)[SPAN], int first, Entries<ONE>& e, float& dot) {
    while (e.next < first + C + 32) {
        float z = 0.0f;
#pragma unroll
        for (int k = 0; k < 32; ++k) take_if(e.next - first - C, k, x[C + k], z);
        dot = fmaf(e.next_q, z, dot);
        e.advance();
    }
}
template <int C, bool ONE> __device__ __forceinline__ void subtract_entries(float (&x)[SPAN], int first, Entries<ONE>& e) {
    while (e.next < first + C + 32) {
#pragma unroll
        for (int k = 0; k < 32; ++k) subtract_if(e.next - first - C, k, e.next_q, x[C + k]);
        e.advance();
    }
}

// `sets`: of the four warps that have the same rows, [4 quarters][32 rows] of (largest, sum, weighted logits); there are two for tiles in turn,
// and each warp waits until all have given theirs.
template <bool ONE>
__device__ __forceinline__ bool end_stats(const GemmArgs& a, const TileWork& w, int rows, float (&x)[SPAN], int64_t row, int quarter, Entries<ONE>& e, float* sets, uint32_t joined,
                                          uint32_t parity) {
    const int first = w.n + quarter * SPAN, lane = threadIdx.x & 31;      // the piece is the whole vocabulary
    float dot = 0.0f;
    take_entries<0>(x, first, e, dot);
    take_entries<32>(x, first, e, dot);
    if (first + SPAN > a.vocab)
#pragma unroll
        for (int k = 0; k < SPAN; ++k) if (first + k >= a.vocab) x[k] = -INFINITY;
    float m[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
    for (int k = 4; k < SPAN; ++k) m[k & 3] = fmaxf(m[k & 3], x[k]);
    const float top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])) * a.scale;
    const float from = top == -INFINITY ? 0.0f : -top;    // nothing but -infinity: its exponentials are 0
    const Two scale(a.scale, a.scale), shift(from, from);
    Two s[2] = {Two(0.0f, 0.0f), Two(0.0f, 0.0f)};
#pragma unroll
    for (int k = 0; k < SPAN; k += 2) {
        float y, z;
        fma(Two(x[k], x[k + 1]), scale, shift).get(y, z);
        s[k / 2 & 1] = s[k / 2 & 1] + Two(exp2_fast(y), exp2_fast(z));
    }
    float* const mine = sets + quarter * 96 + lane;
    mine[0] = top; mine[32] = (s[0] + s[1]).sum(); mine[64] = dot;
    __syncwarp();
    if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(joined) : "memory");
    if (!bar_wait(joined, parity)) return false;
    if (quarter || row >= rows) return true;
    float t[4], all = top;
#pragma unroll
    for (int i = 1; i < 4; ++i) { t[i] = sets[i * 96 + lane]; all = fmaxf(all, t[i]); }
    const float base = all == -INFINITY ? 0.0f : all;
    float sum = mine[32] * exp2_fast(top - base);
#pragma unroll
    for (int i = 1; i < 4; ++i) { sum += sets[i * 96 + 32 + lane] * exp2_fast(t[i] - base); dot += sets[i * 96 + 64 + lane]; }
    const int64_t at = (int64_t)(w.n / TILE) * a.rows + row;
    a.stats[at] = make_float2(all, sum);
    a.dots[at] = dot;
    return true;
}

// Stores of a warp go by way of shared memory: 32 rows of 128 bytes in the order of the 128-byte swizzle, from where TMA takes them.
// (Stored from registers, 16 bytes a lane and a row each, dz of 3456 x 25136 in two numbers took 305 us, against 130.)
struct OutBox {
    uint32_t at;
    // Waits until the last box has been read.
    __device__ __forceinline__ void begin() const {
        if ((threadIdx.x & 31) == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
    }
    __device__ __forceinline__ void put(int piece, uint4 u) const {           // 16 bytes of the lane's row
        const uint32_t lane = threadIdx.x & 31;
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" :: "r"(at + lane * 128 + ((piece ^ (lane & 7)) << 4)), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w) : "memory");
    }
    __device__ __forceinline__ void send2(const CUtensorMap* map, int x, int y) const {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if ((threadIdx.x & 31) == 0)
            asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];\n\tcp.async.bulk.commit_group;" :: "l"(map), "r"(x), "r"(y), "r"(at) : "memory");
    }
    __device__ __forceinline__ void send3(const CUtensorMap* map, int x, int y, int z, bool add) const {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if ((threadIdx.x & 31) == 0) {
            if (add)
                asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2, %3}], [%4];\n\tcp.async.bulk.commit_group;" :: "l"(map), "r"(x), "r"(y), "r"(z), "r"(at) : "memory");
            else
                asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];\n\tcp.async.bulk.commit_group;" :: "l"(map), "r"(x), "r"(y), "r"(z), "r"(at) : "memory");
        }
    }
    __device__ __forceinline__ void finish() const {
        if ((threadIdx.x & 31) == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
};

// dz is rounded to 16 bits, since the tensor cores take no more: a product for each further number.  dhidden and a dweight of bf16 are then 2.1e-3 to
// 2.4e-3 off where their own rounding leaves 1.7e-3.  For a dweight of 32 bits the remainder goes along in 16 bits more (LOW): 2.0e-6 off, 1.1e-3
// without it; with everything in 32 bits it would be 5e-7.
template <class T, bool ONE, bool LOW>
__device__ __forceinline__ void end_dz(const GemmArgs& a, const TileWork& w, int rows, float (&x)[SPAN], int64_t row, int row0, int quarter, Entries<ONE>& e, const OutBox& out) {
    const int column = w.n + quarter * SPAN, first = a.v0 + column;
    const bool here = row < rows;
    const float lse = here ? -a.p.row_lse[row] : 0.0f, c = here ? a.p.row_c[row] : 0.0f;
    const Two scale(a.scale, a.scale), shift(lse, lse), factor(c, c);
#pragma unroll
    for (int k = 0; k < SPAN; k += 2) {
        float y, z;
        fma(Two(x[k], x[k + 1]), scale, shift).get(y, z);
        x[k] = exp2_fast(y);
        x[k + 1] = exp2_fast(z);
    }
    subtract_entries<0>(x, first, e);
    subtract_entries<32>(x, first, e);
    if (c == 0.0f)                            // rows between users, and factors of 0: 0 whatever the logits are
#pragma unroll
        for (int k = 0; k < SPAN; ++k) x[k] = 0.0f;
    if (first + SPAN > a.vocab)
#pragma unroll
        for (int k = 0; k < SPAN; ++k) if (first + k >= a.vocab) x[k] = 0.0f;
    out.begin();
#pragma unroll
    for (int k = 0; k < SPAN; k += 8) {
#pragma unroll
        for (int j = k; j < k + 8; j += 2) (Two(x[j], x[j + 1]) * factor).get(x[j], x[j + 1]);
        const uint4 u = T::pack(x + k);
        out.put(k / 8, u);
        if (LOW) {
            float y[8];
            T::unpack(u, y);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[k + j] -= y[j];
        }
    }
    out.send2(&a.out, column, row0);
    if (LOW) {
        out.begin();
#pragma unroll
        for (int k = 0; k < SPAN; k += 8) out.put(k / 8, T::pack(x + k));
        out.send2(&a.out_low, column, row0);
    }
}

// Each sum is written or added to once: no order of additions is left open.  (Stored from registers, a row a lane, a tile's end took 20000 to
// 50000 cycles.)
__device__ __forceinline__ void end_dhidden(const GemmArgs& a, const TileWork& w, int rows, const float (&x)[SPAN], int row0, int quarter, const OutBox& out) {
    const int first = w.n + quarter * SPAN;
    if (row0 >= rows) return;                 // for the whole warp; rows behind the last one are nobody's
#pragma unroll
    for (int c = 0; c < SPAN; c += 32) {
        if (first + c >= a.dim) break;
        out.begin();
#pragma unroll
        for (int k = 0; k < 8; ++k) out.put(k, OF32::pack(x + c + 4 * k));
        out.send3(&a.out, first + c, row0, w.split, a.add);
    }
}

// dweight where its rows begin anywhere, or are added to: 32 rows of 64 columns turned round in shared memory, so that a store is one piece of
// a row, two elements of 16 bits a lane.  Four users x 1000 tokens x 50257 x 768 bf16, the whole gradient call: 784 us by TMA, 805 here, added to
// 1050 (in 32 bits 2116 .. 2282).  D: the type of dweight.
template <class D>
__device__ __forceinline__ void put_rows(const GemmArgs& a, typename D::type* base, int rows, int columns, const float (&x)[SPAN], const OutBox& out) {
    const int lane = threadIdx.x & 31;
    const uint32_t* const box = (const uint32_t*)__cvta_shared_to_generic(out.at);
    // word `lane` of row r: the 16-byte pieces of a row lie where OutBox::put has them
    auto word = [&](int r) { return box[r * 32 + (((lane >> 2) ^ (r & 7)) << 2 | (lane & 3))]; };
    const int64_t pitch = a.dim;
    if constexpr (sizeof(typename D::type) == 4) {
#pragma unroll
        for (int c = 0; c < SPAN; c += 32) {
            if (c >= columns) break;
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 8; ++k) out.put(k, D::pack(x + c + 4 * k));
            __syncwarp();
            if (c + lane >= columns) continue;
            float* p = (float*)base + c + lane;
            if (a.dw.accumulate)
#pragma unroll 8
                for (int r = 0; r < rows; ++r, p += pitch) *p += __uint_as_float(word(r));
            else
#pragma unroll 8
                for (int r = 0; r < rows; ++r, p += pitch) *p = __uint_as_float(word(r));
        }
    } else if (a.dw.accumulate) {             // added in 32 bits, rounded once: two elements a lane, two rows at a time (as quick as with sums of 16 bits)
        const int half = lane >> 4, pair = lane & 15;
#pragma unroll
        for (int c = 0; c < SPAN; c += 32) {
            if (c >= columns) break;
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 8; ++k) out.put(k, OF32::pack(x + c + 4 * k));
            __syncwarp();
            if (c + 2 * pair >= columns) continue;        // columns are even
            typename D::type* p = base + half * pitch + c + 2 * pair;
#pragma unroll 8
            for (int r = half; r < rows; r += 2, p += 2 * pitch) {
                const float2 f = *(const float2*)(box + r * 32 + (((pair >> 1) ^ (r & 7)) << 2 | (pair & 1) << 1));
                p[0] = D::put(D::get(p[0]) + f.x);
                p[1] = D::put(D::get(p[1]) + f.y);
            }
        }
    } else {
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k) out.put(k, D::pack(x + 8 * k));
        __syncwarp();
        const int pairs = columns < SPAN ? columns / 2 : SPAN / 2;            // columns are even
        typename D::type* p = base + 2 * lane;
        if (((uintptr_t)base & 2) == 0) {     // rows have an even number of elements: all begin at 4 bytes, or none does
#pragma unroll 8
            for (int r = 0; r < rows; ++r, p += pitch)
                if (lane < pairs) *(uint32_t*)p = word(r);
        } else {                              // a whole word is a pair's first element and the one before it, which the lane before has
            const bool whole = lane > 0 && lane < pairs;
#pragma unroll 8
            for (int r = 0; r < rows; ++r, p += pitch) {
                const uint32_t mine = word(r), before = __shfl_up_sync(0xffffffffu, mine, 1);
                if (whole) *(uint32_t*)(p - 1) = before >> 16 | mine << 16;
            }
            if (lane < rows) {                // the first and the last element of a row, by the lane that has it
                typename D::type* const q = base + lane * pitch;
                const int last = pairs - 1;
                q[0] = D::put(x[0]);
                ((uint16_t*)q)[2 * last + 1] = (uint16_t)(box[lane * 32 + (((last >> 2) ^ (lane & 7)) << 2 | (last & 3))] >> 16);
            }
        }
    }
}

// D: the type of dweight.
template <class D>
__device__ __forceinline__ void end_dweight(const GemmArgs& a, const TileWork& w, float (&x)[SPAN], int row0, int quarter, const OutBox& out) {
    const int first = w.n + quarter * SPAN, v = a.v0 + row0;
    if (v >= a.vocab || first >= a.dim) return;
    const float down = 1.0f / a.p.up[w.user];
    const Two by(down, down);
#pragma unroll
    for (int k = 0; k < SPAN; k += 2) (Two(x[k], x[k + 1]) * by).get(x[k], x[k + 1]);
    if (!a.dw_wide) {
        put_rows<D>(a, (typename D::type*)a.dw.data + w.user * a.dw.user_stride + (int64_t)v * a.dim + first, a.vocab - v < 32 ? a.vocab - v : 32, a.dim - first, x, out);
        return;
    }
    constexpr int BOX = 128 / sizeof(typename D::type);
#pragma unroll
    for (int c = 0; c < SPAN; c += BOX) {
        if (first + c >= a.dim) break;
        out.begin();
#pragma unroll
        for (int k = 0; k < 8; ++k) out.put(k, D::pack(x + c + k * D::EACH));
        out.send3(&a.out, first + c, v, w.user, false);
    }
}

// ---- the kernel ------------------------------------------------------------------------------------------------------------
// Stages of depth that an accumulator takes.  The tensor cores cut a sum's last bits off at each 16 of depth (0.2 .. 0.7 units in the last
// place of 32 bits, always towards zero), so where results have 32 bits, sums over more than 1024 are added up in
// registers, rounded to nearest: z over 4096 4.5e-6 of it off in one sum, 1.1e-6 in four.  Four cost 42 thousand cycles a tile, one 37, so what
// is rounded to 16 bits in the end is one sum.
template <int MODE, class D> constexpr int CHUNK = MODE == STATS ? 16 : MODE == DHIDDEN || sizeof(typename D::type) == 2 ? 1 << 20 : 16;

// What bounds it.  4096 tokens x 16384 x 4096, each of the four products 350 us, 1.57 PFLOP/s, the tensor cores at work 85 % of the time; 8192 x 131072 x 4096
// over seconds at the power limit (1.25 GHz): 27.9 .. 28.4 ms for 35 TFLOP of four products, 1.25 PFLOP/s against the 1.38 of a library's plain product.  There the
// products wait for operands on their way from L2 (64 KB a pair in 512 cycles).  At a depth of 768 a tile's end takes as long as its products.
// D: the type of dweight.  LOW: dz in two numbers.
template <int MODE, class T, class D, bool ONE, bool LOW>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(GEMM_THREADS, 1) gemm_kernel(const __grid_constant__ GemmArgs a) {
    constexpr bool A_ALONG = MODE != DWEIGHT, B_ALONG = MODE == STATS || MODE == DZ;       // whether the depth runs along the matrix' rows
    extern __shared__ uint8_t raw[];
    uint8_t* const stages = (uint8_t*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    uint64_t* const bars = (uint64_t*)(stages + STAGES * STAGE_BYTES + OUT_BYTES);
    const uint32_t full = shared_at(bars), empty = full + 8 * STAGES, done = empty + 8 * STAGES, free_ = done + 16, drained = free_ + 16, joined = drained + 8;
    volatile uint32_t* const tmem_at = (volatile uint32_t*)(bars + 2 * STAGES + 9);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) { bar_init(full + 8 * i, 1); bar_init(empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { bar_init(done + 8 * i, 1); bar_init(free_ + 8 * i, 2 * EPI_WARPS); }
        bar_init(drained, 1);
        for (int i = 0; i < 4; ++i) bar_init(joined + 8 * i, 4);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(shared_at((const void*)tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_at;
    let_next_start();
    wait_for_previous();
    asm volatile("fence.proxy.async;" ::: "memory");      // what ordinary stores of the kernels before have left is read by TMA
    const int rows = a.p.offset[a.users];
    const int64_t pair = blockIdx.x / 2, pairs = gridDim.x / 2;
    bool fine = true;
    TileWork w;
    if (warp == 0) {
        if (lane == 0) {                      // loads
            const uint32_t far_full = at_rank(full, 0);
            uint32_t s = 0, phase = 0, issued = 0;
            for (int64_t i = pair; fine && tile_at<MODE>(a, rows, i, w); i += pairs) {
                const int each = MODE == DWEIGHT ? w.k1 / a.terms : 0, r0 = MODE == DWEIGHT ? a.p.offset[w.user] : 0;
                for (int k = w.k0; k < w.k1; ++k) {
                    if (!(fine = bar_wait(empty + 8 * s, phase ^ 1))) break;
                    if (rank == 0) bar_expect(full + 8 * s, 2 * STAGE_BYTES);
                    const uint32_t to = shared_at(stages) + s * STAGE_BYTES, bar = far_full + 8 * s;
                    const CUtensorMap* ma = &a.a;
                    int depth = k * KB;
                    if (MODE == DWEIGHT) {
                        if (k >= each) { ma = &a.a_low; depth -= each * KB; }
                        depth += r0;
                    }
                    for (int j = 0; j < 2; ++j) {
                        const int m = w.m + (int)rank * 128 + j * 64, n = w.n + (int)rank * 128 + j * 64;
                        if (A_ALONG) tma_load(to + j * 8192, ma, depth, m, bar);
                        else tma_load(to + j * 8192, ma, m, depth, bar);
                        const int from = MODE == DWEIGHT ? 0 : a.v0;      // of the weight's rows
                        if (B_ALONG) tma_load(to + HALF_BYTES + j * 8192, &a.b, depth, from + n, bar);
                        else tma_load(to + HALF_BYTES + j * 8192, &a.b, n, from + depth, bar);
                    }
                    ++issued;
                    if (++s == STAGES) { s = 0; phase ^= 1; }
                }
            }
            // no product still reads a stage, and no barrier is still to be arrived at, when the block ends
            for (int j = 0; fine && j < STAGES; ++j) {
                fine = bar_wait(empty + 8 * s, phase ^ 1);
                if (++s == STAGES) { s = 0; phase ^= 1; }
            }
            if (!fine && rank == 0)           // what is on its way arrives before the block ends
                for (uint32_t j = issued > STAGES ? issued - STAGES : 0; j < issued; ++j) bar_wait(full + 8 * (j % STAGES), j / STAGES & 1);
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {         // products of both blocks
            // 32-bit sums of 16-bit products, 256 x 256
            const uint32_t kind = std::is_same<T, OBf16>::value ? 1 : 0;
            const uint32_t desc = 1u << 4 | kind << 7 | kind << 10 | (A_ALONG ? 0u : 1u << 15) | (B_ALONG ? 0u : 1u << 16) | (TILE >> 3) << 17 | (TILE >> 4) << 24;
            uint32_t s = 0, phase = 0, turn_no = 0;
            for (int64_t i = pair; fine && tile_at<MODE>(a, rows, i, w); i += pairs) {
                int k = w.k0;
                do {                          // once for a tile without depth
                    const uint32_t buffer = turn_no & 1, to = tmem + buffer * TILE;
                    if (!(fine = bar_wait(free_ + 8 * buffer, (turn_no >> 1 & 1) ^ 1))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const int k2 = w.k1 - k < CHUNK<MODE, D> ? w.k1 : k + CHUNK<MODE, D>;
                    for (bool add = false; k < k2; ++k) {
                        if (!(fine = bar_wait(full + 8 * s, phase))) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t at = shared_at(stages) + s * STAGE_BYTES;
                        const uint64_t da = operand_desc<A_ALONG>(at), db = operand_desc<B_ALONG>(at + HALF_BYTES);
#pragma unroll
                        for (int j = 0; j < KB / 16; ++j) {   // 16 deep: 32 bytes along the rows, or sixteen rows
                            mma(to, da + j * (A_ALONG ? 32 >> 4 : 2048 >> 4), db + j * (B_ALONG ? 32 >> 4 : 2048 >> 4), desc, add);
                            add = true;
                        }
                        mma_commit(empty + 8 * s);
                        if (++s == STAGES) { s = 0; phase ^= 1; }
                    }
                    if (!fine) break;
                    mma_commit(done + 8 * buffer);
                    ++turn_no;
                } while (k < w.k1);
            }
            // no product is under way when the memory is given back
            asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(drained) : "memory");
            fine &= bar_wait(drained, 0);
        }
    } else {
        const int part = warp & 3, quarter = (warp - FIRST_EPI) >> 2;         // a warp reads the fourth of the lanes that its number gives
        uint32_t turn_no = 0;
        const uint32_t far_free = at_rank(free_, 0);
        const OutBox out = {shared_at(stages + STAGES * STAGE_BYTES + (warp - FIRST_EPI) * 4096)};
        float* const sets = (float*)(stages + STAGES * STAGE_BYTES) + part * 768;
        uint32_t set = 0;
        for (int64_t i = pair; fine && tile_at<MODE>(a, rows, i, w); i += pairs) {
            const int in_tile = (int)rank * 128 + part * 32;
            const int64_t row = (int64_t)w.m + in_tile + lane;
            Entries<ONE> e;                   // looked for while the products run
            if constexpr (MODE == STATS || MODE == DZ) {
                const int first = a.v0 + w.n + quarter * SPAN;
                e.begin(a, row < rows && first < a.vocab, row, first);
            }
            float x[SPAN];
            int k = w.k0;
            do {
                const uint32_t buffer = turn_no & 1;
                if (!(fine = bar_wait(done + 8 * buffer, turn_no >> 1 & 1))) break;
                __syncwarp();
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t at = tmem + buffer * TILE + quarter * SPAN + ((uint32_t)part << 21);     // lane 32 part
                if (k == w.k0) {
                    tmem_load32(at, x);
                    tmem_load32(at + 32, x + 32);
                    tmem_loaded32(x);
                    tmem_loaded32_too(x + 32);
                } else
#pragma unroll
                    for (int c = 0; c < SPAN; c += 16) {
                        float y[16];
                        tmem_load16(at + c, y);
                        tmem_loaded16(y);
#pragma unroll
                        for (int j = 0; j < 16; ++j) x[c + j] += y[j];
                    }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) bar_arrive_far(far_free + 8 * buffer);
                ++turn_no;
                k = w.k1 - k < CHUNK<MODE, D> ? w.k1 : k + CHUNK<MODE, D>;
            } while (k < w.k1);
            if (!fine) break;
            if (w.k0 >= w.k1)                 // no depth (a user without a token that counts): the sums are 0
#pragma unroll
                for (int j = 0; j < SPAN; ++j) x[j] = 0.0f;
            if constexpr (MODE == STATS) {
                if (!(fine = end_stats<ONE>(a, w, rows, x, row, quarter, e, sets + (set & 1) * 384, joined + 8 * part, set & 1))) break;
                ++set;
            }
            if constexpr (MODE == DZ) end_dz<T, ONE, LOW>(a, w, rows, x, row, w.m + in_tile, quarter, e, out);
            if constexpr (MODE == DHIDDEN) end_dhidden(a, w, rows, x, w.m + in_tile, quarter, out);
            if constexpr (MODE == DWEIGHT) end_dweight<D>(a, w, x, w.m + in_tile, quarter, out);
            __syncwarp();
        }
        if (MODE != STATS) out.finish();
    }
    if (!fine) atomicOr(&a.status->flags, CO3_FLAG_TIMEOUT);
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
}

// ---- before and after the products -----------------------------------------------------------------------------------------
struct Targets {
    const void* data;
    int64_t user_stride, token_stride;
    int wide, top;
    const void* teacher;
    int64_t teacher_user, teacher_token;
    int teacher_type;
};
__device__ __forceinline__ int64_t index_at(const Targets& k, int64_t at) { return k.wide ? ((const int64_t*)k.data)[at] : (int64_t)((const int32_t*)k.data)[at]; }

// A warp per token: its entries in the order of their numbers, their shares q, sum q log q, and for each tile of the vocabulary how many lie before it.
struct EntryArgs {
    Targets k;
    int64_t n_all;
    uint32_t tokens;
    int vocab, tiles;
    float inv_t;
    int32_t* entry; float* q; float* constant; uint8_t* first; uint8_t* mass;
    OpsStatus* status;
};
__global__ void __launch_bounds__(256) entry_kernel(const __grid_constant__ EntryArgs a) {
    __shared__ int32_t sh_index[8][MAX_TOP], sh_sorted[8][MAX_TOP];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n = (int64_t)blockIdx.x * 8 + warp;
    let_next_start();
    wait_for_previous();
    if (n >= a.n_all) return;
    const int64_t user = n / a.tokens, t = n - user * a.tokens, top = a.k.top;
    int32_t index[4];
    float z[4], most = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = lane + 32 * i;
        index[i] = 0x7FFFFFFF;
        z[i] = -INFINITY;
        if (j < top) {
            const int64_t v = index_at(a.k, user * a.k.user_stride + t * a.k.token_stride + j);
            if (v >= a.vocab) { atomicAdd(&a.status->bad_tokens, 1ull); atomicOr(&a.status->flags, CO3_FLAG_TOKEN); }
            else if (v >= 0) {
                z[i] = load_as_f32(a.k.teacher, a.k.teacher_type, user * a.k.teacher_user + t * a.k.teacher_token + j);
                if (z[i] != -INFINITY) index[i] = (int32_t)v;        // one without mass is none
            }
            sh_index[warp][j] = index[i];
        }
        most = fmaxf(most, z[i]);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    float e[4], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {             // over the temperature only what is left of the largest: a logit itself may pass 32 bits there
        z[i] = (z[i] - most) * a.inv_t;
        e[i] = index[i] != 0x7FFFFFFF ? expf(z[i]) : 0.0f;
        sum += e[i];
    }
    sum = warp_sum_f32(sum);
    const float log_sum = logf(sum);
    float about = 0.0f;
    int kept = 0;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = lane + 32 * i;
        const bool here = j < top && index[i] != 0x7FFFFFFF;
        kept += __popc(__ballot_sync(0xffffffffu, here));
        if (j >= top) continue;
        int rank = 0;                         // those that stand twice keep their order
        for (int o = 0; o < top; ++o) {
            const int32_t x = sh_index[warp][o];
            rank += x < index[i] || (x == index[i] && o < j);
        }
        const float q = here ? e[i] / sum : 0.0f;
        if (here && q != 0.0f) about = fmaf(q, z[i] - log_sum, about);
        a.entry[n * top + rank] = index[i];
        a.q[n * top + rank] = q;
        sh_sorted[warp][rank] = index[i];
    }
    about = warp_sum_f32(about);
    if (lane == 0) {
        a.constant[n] = about;
        a.mass[n] = kept > 0;
    }
    __syncwarp();
    for (int s = lane; s < a.tiles; s += 32) {
        int lo = 0, hi = (int)top;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if ((int64_t)sh_sorted[warp][mid] < (int64_t)s * TILE) lo = mid + 1; else hi = mid;
        }
        a.first[n * a.tiles + s] = (uint8_t)lo;
    }
}

// One thread block: counts the tokens with a target, and gives each its packed row.
constexpr int SEG = 256;                      // tokens that a warp counts
constexpr int SEGS_NEAR = 2048, USERS_NEAR = 1024;
struct PackArgs {
    Targets k;
    const uint8_t* mass;                      // null: one entry a token
    uint32_t tokens, segs;
    int users, vocab;
    const float* dloss;
    float scale;                              // over the temperature
    int half;                                 // f16: dz is scaled
    int32_t *seg_count;                       // [users * segs]
    float* seg_most;
    Packed p;
    OpsStatus* status;
};
// Whether the token counts: it has a target, and a gradient is wanted of it.  (A dz of 0 alone would not do: what is not a number in its hidden
// state would reach its user's weight gradient.)
__device__ __forceinline__ bool has_target(const PackArgs& a, uint32_t user, uint32_t t, bool count) {
    const int64_t n = (int64_t)user * a.tokens + t;
    const bool wanted = !a.dloss || a.dloss[n] != 0.0f;
    if (a.mass) return wanted && a.mass[n] != 0;
    const int64_t v = index_at(a.k, user * a.k.user_stride + t * a.k.token_stride);
    if (count && v >= a.vocab) { atomicAdd(&a.status->bad_tokens, 1ull); atomicOr(&a.status->flags, CO3_FLAG_TOKEN); }
    return wanted && v >= 0 && v < a.vocab;
}
// f16: the power of two that brings the user's largest factor to 2^13 .. 2^14: dz is at most that.
__device__ __forceinline__ float scale_of(const PackArgs& a, float most, int count) {
    if (!a.half) return 1.0f;
    most = a.dloss ? most * fabsf(a.scale) : fabsf(a.scale) / (float)(count > 0 ? count : 1);
    if (!(most > 0.0f && most < INFINITY)) return 1.0f;
    int e;
    frexpf(most, &e);
    e = 14 - e;
    return ldexpf(1.0f, e > 126 ? 126 : e < -126 ? -126 : e);
}
__global__ void __launch_bounds__(1024) pack_kernel(const __grid_constant__ PackArgs a) {
    __shared__ int warp_sums[32], near_count[SEGS_NEAR], near_offset[USERS_NEAR + 1];
    __shared__ float near_most[SEGS_NEAR];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t below = (1u << lane) - 1u;
    let_next_start();
    wait_for_previous();
    const int64_t all = (int64_t)a.users * a.segs;
    // where the counts of a step are kept for the next: near if there is room
    int32_t* const seg_count = all <= SEGS_NEAR ? near_count : a.seg_count;
    float* const seg_most = all <= SEGS_NEAR ? near_most : a.seg_most;
    int32_t* const offset = a.users <= USERS_NEAR ? near_offset : a.p.offset;
    for (int64_t g = warp; g < all; g += 32) {
        const uint32_t user = (uint32_t)(g / a.segs), t0 = (uint32_t)(g - (int64_t)user * a.segs) * SEG;
        int n = 0;
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < SEG / 32; ++i) {
            const uint32_t t = t0 + i * 32 + lane;
            const bool here = t < a.tokens && has_target(a, user, t, true);
            n += __popc(__ballot_sync(0xffffffffu, here));
            if (here && a.dloss && a.half) most = fmaxf(most, fabsf(a.dloss[(int64_t)user * a.tokens + t]));
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        if (lane == 0) { seg_count[g] = n; seg_most[g] = most; }
    }
    __syncthreads();
    for (int user = warp; user < a.users; user += 32) {
        int sum = 0;
        float most = 0.0f;
        for (uint32_t s0 = 0; s0 < a.segs; s0 += 32) {
            const uint32_t s = s0 + lane;
            const int64_t g = (int64_t)user * a.segs + s;
            const int c = s < a.segs ? seg_count[g] : 0;
            if (s < a.segs) most = fmaxf(most, seg_most[g]);
            int up = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, up, o); if (lane >= o) up += v; }
            if (s < a.segs) seg_count[g] = sum + up - c;            // tokens with a target before the segment
            sum += __shfl_sync(0xffffffffu, up, 31);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        if (lane == 0) {
            a.p.count[user] = sum;
            offset[user + 1] = (sum + ALIGN_ROWS - 1) / ALIGN_ROWS * ALIGN_ROWS;
            a.p.up[user] = scale_of(a, most, sum);
        }
    }
    __syncthreads();
    int carry = 0;
    for (int u0 = 0; u0 < a.users; u0 += 1024) {          // running sum over the users
        const int user = u0 + (int)threadIdx.x;
        int up = user < a.users ? offset[user + 1] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, up, o); if (lane >= o) up += v; }
        if (lane == 31) warp_sums[warp] = up;
        __syncthreads();
        int before = 0, total = 0;
        for (int w = 0; w < 32; ++w) { before += w < warp ? warp_sums[w] : 0; total += warp_sums[w]; }
        if (user < a.users) offset[user + 1] = carry + before + up;
        carry += total;
        __syncthreads();
    }
    if (threadIdx.x == 0) offset[0] = 0;
    __syncthreads();
    for (int64_t g = warp; g < all; g += 32) {
        const uint32_t user = (uint32_t)(g / a.segs), t0 = (uint32_t)(g - (int64_t)user * a.segs) * SEG;
        int row = offset[user] + seg_count[g];
#pragma unroll
        for (int i = 0; i < SEG / 32; ++i) {
            const uint32_t t = t0 + i * 32 + lane;
            const bool here = t < a.tokens && has_target(a, user, t, false);
            const uint32_t mask = __ballot_sync(0xffffffffu, here);
            const int mine = row + __popc(mask & below);
            const int64_t n = (int64_t)user * a.tokens + t;
            if (here) a.p.row_token[mine] = (int32_t)n;
            if (t < a.tokens) a.p.token_row[n] = here ? mine : -1;
            row += __popc(mask);
        }
    }
    for (int i = threadIdx.x; offset != a.p.offset && i <= a.users; i += 1024) a.p.offset[i] = offset[i];
    for (int user = warp; user < a.users; user += 32)     // the zero rows behind a user's
        for (int r = offset[user] + a.p.count[user] + lane; r < offset[user + 1]; r += 32) a.p.row_token[r] = -1;
}

// A warp per packed row: the hidden state, and what the tiles' ends need of the token.
struct GatherArgs {
    const void* hidden;
    int64_t hu, ht;
    void* packed;
    Packed p;
    Targets k;
    const float *lse, *dloss;                 // null in the forward call; dloss null: mean
    float scale;
    uint32_t tokens;
    int users, dim;
};
template <bool VEC> __device__ __forceinline__ void gather_row(const GatherArgs& a, int64_t row, int n, uint32_t user, uint32_t t, int count, float up) {
    const int lane = threadIdx.x & 31;
    const uint16_t* from = (const uint16_t*)a.hidden + user * a.hu + t * a.ht;
    uint16_t* to = (uint16_t*)a.packed + row * a.dim;
    if (VEC) {
#pragma unroll 4
        for (int at = lane * 8; at < a.dim; at += 256) *(uint4*)(to + at) = n < 0 ? make_uint4(0, 0, 0, 0) : *(const uint4*)(from + at);
    } else {
#pragma unroll 4
        for (int at = lane; at < a.dim; at += 32) to[at] = n < 0 ? (uint16_t)0 : from[at];
    }
    if (lane) return;
    if (a.k.top == 1 && !a.k.teacher) a.p.row_target[row] = n < 0 ? -1 : (int32_t)index_at(a.k, user * a.k.user_stride + t * a.k.token_stride);
    if (!a.lse) return;
    a.p.row_lse[row] = n < 0 ? 0.0f : a.lse[n] * LOG2E;
    a.p.row_c[row] = n < 0 ? 0.0f : (a.dloss ? a.dloss[n] * a.scale : a.scale / (float)count) * up;
}
template <bool VEC> __global__ void __launch_bounds__(256) gather_kernel(const __grid_constant__ GatherArgs a) {
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    let_next_start();
    wait_for_previous();
    if (row >= a.p.offset[a.users]) return;
    const int n = a.p.row_token[row];
    const uint32_t user = n < 0 ? 0 : n / a.tokens, t = n < 0 ? 0 : n - user * a.tokens;
    gather_row<VEC>(a, row, n, user, t, n < 0 ? 0 : a.p.count[user], n < 0 ? 0.0f : a.p.up[user]);
}

// What pack_kernel and gather_kernel do, in one launch, for few tokens and users: each thread block counts all of them by itself, which is quicker than
// waiting for another, and takes a share of the rows, a warp each.  Dim 256, in two launches -> in one: 200 tokens 7.8 -> 3.1 us, 2048 8.5 -> 4.5,
// 8192 11.1 -> 9.2, 250 users of 3 32.8 -> 13.1, 200 of 40 31.2 -> 16.0.  The counts of all tokens grow with them: hence the limits.
constexpr int FEW_TOKENS = 8192, FEW_USERS = 256, FEW_WORDS = FEW_TOKENS / 32 + FEW_USERS;
template <bool VEC> __global__ void __launch_bounds__(1024) pack_few_kernel(const __grid_constant__ PackArgs a, const __grid_constant__ GatherArgs g) {
    __shared__ uint32_t mask[FEW_WORDS];                  // which tokens have a target, 32 of a user a word
    __shared__ int before[FEW_WORDS];                     // those of the user before the word's
    __shared__ float word_most[FEW_WORDS], up[FEW_USERS];
    __shared__ int count[FEW_USERS], offset[FEW_USERS + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t each = (a.tokens + 31) / 32, words = each * a.users;       // words of a user, and of all
    let_next_start();
    wait_for_previous();
    for (uint32_t w = warp; w < words; w += 32) {
        const uint32_t user = w / each, t = (w - user * each) * 32 + lane;
        const bool here = t < a.tokens && has_target(a, user, t, blockIdx.x == 0);
        const uint32_t m = __ballot_sync(0xffffffffu, here);
        float most = here && a.dloss && a.half ? fabsf(a.dloss[(int64_t)user * a.tokens + t]) : 0.0f;
#pragma unroll
        for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        if (lane == 0) { mask[w] = m; word_most[w] = most; }
    }
    __syncthreads();
    for (int user = warp; user < a.users; user += 32) {
        int sum = 0;
        float most = 0.0f;
        for (uint32_t i0 = 0; i0 < each; i0 += 32) {
            const uint32_t w = user * each + i0 + lane;
            const bool here = i0 + lane < each;
            const int c = here ? __popc(mask[w]) : 0;
            if (here) most = fmaxf(most, word_most[w]);
            int to = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, to, o); if (lane >= o) to += v; }
            if (here) before[w] = sum + to - c;
            sum += __shfl_sync(0xffffffffu, to, 31);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        if (lane == 0) { count[user] = sum; up[user] = scale_of(a, most, sum); }
    }
    __syncthreads();
    if (warp == 0) {
        int carry = 0;
        for (int u0 = 0; u0 < a.users; u0 += 32) {
            int to = u0 + lane < a.users ? (count[u0 + lane] + ALIGN_ROWS - 1) / ALIGN_ROWS * ALIGN_ROWS : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, to, o); if (lane >= o) to += v; }
            if (u0 + lane < a.users) offset[u0 + lane + 1] = carry + to;
            carry += __shfl_sync(0xffffffffu, to, 31);
        }
        if (lane == 0) offset[0] = 0;
    }
    __syncthreads();
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i <= a.users; i += 1024) {
            a.p.offset[i] = offset[i];
            if (i < a.users) { a.p.count[i] = count[i]; a.p.up[i] = up[i]; }
        }
    // tokens first, then the rows behind each user's
    const int64_t tokens = (int64_t)a.users * a.tokens, all = tokens + (int64_t)a.users * ALIGN_ROWS;
    for (int64_t i = (int64_t)blockIdx.x * 32 + warp; i < all; i += (int64_t)gridDim.x * 32) {
        int n = -1;
        uint32_t user, t = 0;
        int row;
        if (i < tokens) {
            user = (uint32_t)i / a.tokens;
            t = (uint32_t)i - user * a.tokens;
            const uint32_t w = user * each + t / 32, bit = t % 32;
            const bool here = mask[w] >> bit & 1;
            row = offset[user] + before[w] + __popc(mask[w] & ((1u << bit) - 1u));
            if (lane == 0) a.p.token_row[i] = here ? row : -1;
            if (!here) continue;
            n = (int)i;
        } else {
            user = (uint32_t)(i - tokens) / ALIGN_ROWS;
            row = offset[user] + count[user] + (int)((uint32_t)(i - tokens) % ALIGN_ROWS);
            if (row >= offset[user + 1]) continue;
        }
        if (lane == 0) a.p.row_token[row] = n;
        gather_row<VEC>(g, row, n, user, t, count[user], up[user]);
    }
}

// Statistics of the tiles to loss and lse: 32 tokens, 32 warps with a stretch of the tiles each, joined in order.
constexpr int LOSS_WARPS = 32;
struct LossArgs {
    const float2* stats;
    const float *dots, *constant;
    int64_t rows, n_all;
    int tiles;
    float inv_t;
    Packed p;
    float *loss, *lse;
};
__global__ void __launch_bounds__(32 * LOSS_WARPS) loss_kernel(const __grid_constant__ LossArgs a) {
    __shared__ float sh[LOSS_WARPS][3][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n = (int64_t)blockIdx.x * 32 + lane;
    let_next_start();
    wait_for_previous();
    const int row = n < a.n_all ? a.p.token_row[n] : -1;
    float m = -INFINITY, s = 0.0f, dot = 0.0f;
    if (row >= 0) {
        const int each = (a.tiles + LOSS_WARPS - 1) / LOSS_WARPS, end = (warp + 1) * each < a.tiles ? (warp + 1) * each : a.tiles;
        for (int i0 = warp * each; i0 < end; i0 += 8) {       // eight loads on their way
            float2 x[8];
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool here = i0 + i < end;
                x[i] = here ? a.stats[(i0 + i) * a.rows + row] : make_float2(-INFINITY, 0.0f);
                d[i] = here ? a.dots[(i0 + i) * a.rows + row] : 0.0f;
            }
            float big = m;
#pragma unroll
            for (int i = 0; i < 8; ++i) big = fmaxf(big, x[i].x);
            const float from = big == -INFINITY ? 0.0f : big;
            s *= exp2_fast(m - from);
#pragma unroll
            for (int i = 0; i < 8; ++i) { s += x[i].y * exp2_fast(x[i].x - from); dot += d[i]; }
            m = big;
        }
    }
    sh[warp][0][lane] = m; sh[warp][1][lane] = s; sh[warp][2][lane] = dot;
    __syncthreads();
    // a token a warp: its 32 stretches over the lanes
    const int64_t mine = (int64_t)blockIdx.x * 32 + warp;
    if (mine >= a.n_all) return;
    m = sh[lane][0][warp]; s = sh[lane][1][warp]; dot = sh[lane][2][warp];
    float big = m;
#pragma unroll
    for (int o = 16; o; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
    const float from = big == -INFINITY ? 0.0f : big;
    s = warp_sum_f32(s * exp2_fast(m - from));
    dot = warp_sum_f32(dot);
    if (lane) return;
    const bool none = a.p.token_row[mine] < 0;
    const float lse = none ? 0.0f : (big + log2f(s)) * LN2;
    a.lse[mine] = lse;
    a.loss[mine] = none ? 0.0f : (lse - dot * a.inv_t) + (a.constant ? a.constant[mine] : 0.0f);
}

// The splits' sums to dhidden, a warp to 256 columns of a token.
struct HiddenArgs {
    const float* partial;
    int64_t rows, items;
    int splits, dim, slabs;
    uint32_t tokens;
    Packed p;
    void* out;
    int64_t ou, ot;
};
template <class T, bool VEC> __global__ void __launch_bounds__(256) hidden_kernel(const __grid_constant__ HiddenArgs a) {
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    let_next_start();
    wait_for_previous();
    if (item >= a.items) return;
    const uint32_t n = (uint32_t)(item / a.slabs), user = n / a.tokens, t = n - user * a.tokens;
    const int column = (int)(item - (int64_t)n * a.slabs) * 256 + lane * 8, row = a.p.token_row[n];
    if (column >= a.dim) return;              // dim is a multiple of 8
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = 0.0f;
    if (row >= 0) {
        const float* from = a.partial + (int64_t)row * a.dim + column;
#pragma unroll 4
        for (int s = 0; s < a.splits; ++s) {
            float y[8];
            OF32::unpack(*(const uint4*)from, y);
            OF32::unpack(*(const uint4*)(from + 4), y + 4);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] += y[k];
            from += a.rows * a.dim;
        }
        const float down = 1.0f / a.p.up[user];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= down;
    }
    typename T::type* to = (typename T::type*)a.out + user * a.ou + t * a.ot + column;
    if (VEC) *(uint4*)to = T::pack(x);
    else
#pragma unroll
        for (int k = 0; k < 8; ++k) to[k] = T::put(x[k]);
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

}  // namespace

struct co3_token_loss {
    int64_t vocab, dim, max_tokens, rows, launches;       // rows: all packed ones there can be, to whole tiles
    int users, type, grad_type, max_top, device, pairs, tiles, max_splits;
    int64_t piece;                            // columns of dz that are held at a time
    EncodeTiled encode;
    CUtensorMap map_hidden, map_dz, map_low, map_dz_out, map_low_out, map_partial;
    void* slab;
    OpsStatus* status;
    Packed p;
    int32_t* seg_count; float* seg_most;
    void *hidden, *dz, *low;
    float2* stats; float *dots, *partial;
    int32_t* entry; float *q, *constant; uint8_t *first, *mass;
};

namespace {

CUtensorMapDataType map_type(int type) {
    return type == CO3_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : type == CO3_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
}
// A matrix of 16-bit numbers in boxes of 64 columns: 64 rows to load, 32 to store.
bool make_map(const co3_token_loss* h, CUtensorMap* map, const void* data, int64_t columns, int64_t rows, int64_t stride, int box_rows = 64) {
    const cuuint64_t dims[2] = {(cuuint64_t)columns, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, one[2] = {1, 1};
    return h->encode(map, map_type(h->type), 2, (void*)data, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// dweight in boxes of 128 bytes and 32 rows; partial likewise.
bool make_out_map(const co3_token_loss* h, CUtensorMap* map, void* data, int type, int64_t rows, int64_t pieces, int64_t piece_stride) {
    const int width = type_width(type);
    const cuuint64_t dims[3] = {(cuuint64_t)h->dim, (cuuint64_t)rows, (cuuint64_t)pieces};
    const cuuint64_t strides[2] = {(cuuint64_t)(h->dim * width), (cuuint64_t)(piece_stride * width)};
    const cuuint32_t box[3] = {(cuuint32_t)(128 / width), 32, 1}, one[3] = {1, 1, 1};
    return strides[1] < (cuuint64_t)1 << 40 &&
           h->encode(map, map_type(type), 3, data, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class K> bool big_shared(K kernel) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, GEMM_SHARED) == cudaSuccess;
}
template <class T> bool all_big() {
    return big_shared(gemm_kernel<STATS, T, T, true, false>) && big_shared(gemm_kernel<STATS, T, T, false, false>) &&
           big_shared(gemm_kernel<DZ, T, T, true, false>) && big_shared(gemm_kernel<DZ, T, T, false, false>) &&
           big_shared(gemm_kernel<DZ, T, OF32, true, false>) && big_shared(gemm_kernel<DZ, T, OF32, false, false>) &&
           big_shared(gemm_kernel<DZ, T, OF32, true, true>) && big_shared(gemm_kernel<DZ, T, OF32, false, true>) &&
           big_shared(gemm_kernel<DHIDDEN, T, T, true, false>) && big_shared(gemm_kernel<DWEIGHT, T, T, true, false>) &&
           big_shared(gemm_kernel<DWEIGHT, T, OF32, true, false>);
}

int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

int gemm(co3_token_loss* h, void (*kernel)(GemmArgs), int64_t tiles, const GemmArgs& a, cudaStream_t st) {
    const int64_t pairs = tiles < h->pairs ? tiles : h->pairs;
    return launch_early(&h->launches, kernel, dim3((unsigned)(2 * (pairs < 1 ? 1 : pairs))), GEMM_THREADS, GEMM_SHARED, 1, st, a);
}

// How many parts the depth of dhidden (in stages) is cut into.  For few tiles more of them fill the device, or its last round; each costs its
// sums' way to memory and back.
int splits_of(const co3_token_loss* h, int64_t tiles, int64_t rows, int64_t depth) {
    int best = 1;
    double least = 1e30;
    for (int s = 1; s <= h->max_splits && (s == 1 || depth / s >= 8); ++s) {
        const double stage = 0.35e-6, rate = 5e12;        // 512 cycles; bytes a second
        const double t = (double)((tiles * s + h->pairs - 1) / h->pairs) * (double)((depth + s - 1) / s) * stage + (double)s * (double)rows * (double)h->dim * 8.0 / rate;
        if (t < least) { least = t; best = s; }
    }
    return best;
}

unsigned blocks_for(int64_t n, int each) { return (unsigned)(n > 0 ? (n + each - 1) / each : 1); }

struct Call {
    Targets k;
    GemmArgs g;
    int64_t n_all, rows;                      // all rows there can be in this call
    bool one;
};

// Checks what both calls are given, and enqueues the packing.
int begin_call(co3_token_loss* h, const co3_array* hidden, const void* weight, int64_t weight_stride, const co3_tokens* targets, const co3_array* teacher,
               float temperature, int64_t n_tokens, const float* lse, const float* dloss, float scale, bool backward, Call& c, cudaStream_t st) {
    const int64_t n_all = n_tokens * h->users;
    c.n_all = n_all;
    c.one = !teacher;
    c.rows = up_to(n_tokens, ALIGN_ROWS) * h->users;
    Targets& k = c.k;
    memset(&k, 0, sizeof(k));
    k.data = targets->data; k.user_stride = targets->user_stride; k.token_stride = targets->token_stride;
    k.wide = targets->type == CO3_I64; k.top = targets->top;
    if (teacher) { k.teacher = teacher->data; k.teacher_user = teacher->user_stride; k.teacher_token = teacher->token_stride; k.teacher_type = teacher->type; }
    int rc = CO3_OK;
    if (teacher) {
        EntryArgs e;
        e.k = k; e.n_all = n_all; e.tokens = (uint32_t)n_tokens; e.vocab = (int)h->vocab; e.tiles = h->tiles; e.inv_t = 1.0f / temperature;
        e.entry = h->entry; e.q = h->q; e.constant = h->constant; e.first = h->first; e.mass = h->mass; e.status = h->status;
        rc = launch_early(&h->launches, entry_kernel, dim3(blocks_for(n_all, 8)), 256, 0, 1, st, e);
        if (rc != CO3_OK) return rc;
    }
    PackArgs p;
    p.k = k; p.mass = teacher ? h->mass : nullptr; p.tokens = (uint32_t)n_tokens; p.segs = (uint32_t)((n_tokens + SEG - 1) / SEG); p.users = h->users;
    p.vocab = (int)h->vocab; p.dloss = backward ? dloss : nullptr; p.scale = scale / temperature; p.half = backward && h->type == CO3_F16;
    p.seg_count = h->seg_count; p.seg_most = h->seg_most; p.p = h->p; p.status = h->status;
    GatherArgs g;
    g.hidden = hidden->data; g.hu = hidden->user_stride; g.ht = hidden->token_stride; g.packed = h->hidden; g.p = h->p; g.k = k;
    g.lse = backward ? lse : nullptr; g.dloss = dloss; g.scale = p.scale; g.tokens = (uint32_t)n_tokens; g.users = h->users; g.dim = (int)h->dim;
    const bool vec = rows_aligned(hidden, h->users, n_tokens);
    if (n_all > 0 && n_all <= FEW_TOKENS && h->users <= FEW_USERS) {
        const int64_t blocks = (n_all + (int64_t)h->users * ALIGN_ROWS + 31) / 32;
        const dim3 grid((unsigned)(blocks < 2 * h->pairs ? blocks : 2 * h->pairs));
        rc = vec ? launch_early(&h->launches, pack_few_kernel<true>, grid, 1024, 0, 1, st, p, g) : launch_early(&h->launches, pack_few_kernel<false>, grid, 1024, 0, 1, st, p, g);
    } else {
        rc = launch_early(&h->launches, pack_kernel, dim3(1), 1024, 0, 1, st, p);
        if (rc != CO3_OK) return rc;
        const dim3 grid(blocks_for(c.rows, 8));
        rc = vec ? launch_early(&h->launches, gather_kernel<true>, grid, 256, 0, 1, st, g) : launch_early(&h->launches, gather_kernel<false>, grid, 256, 0, 1, st, g);
    }
    if (rc != CO3_OK) return rc;
    GemmArgs& a = c.g;
    memset(&a, 0, sizeof(a));
    a.a = h->map_hidden;
    if (!make_map(h, &a.b, weight, h->dim, h->vocab, weight_stride)) return CO3_EINVAL;
    a.p = h->p; a.status = h->status; a.users = h->users; a.vocab = (int)h->vocab; a.dim = (int)h->dim; a.splits = 1; a.terms = 1; a.rows = h->rows;
    a.scale = LOG2E / temperature; a.stats = h->stats; a.dots = h->dots; a.entry = h->entry; a.entry_q = h->q; a.entry_first = h->first; a.top = k.top;
    a.tiles = h->tiles;
    return CO3_OK;
}

bool call_fine(const co3_token_loss* h, const co3_array* hidden, const void* weight, int64_t weight_stride, const co3_tokens* targets, const co3_array* teacher,
               float temperature, int64_t n_tokens) {
    if (!h || n_tokens < 0 || n_tokens > h->max_tokens) return false;
    if (!array_fine(hidden, h->users, n_tokens, h->dim, false) || hidden->type != h->type) return false;
    if (!weight || !aligned_to(weight, 16) || weight_stride < h->dim || weight_stride % 8 || weight_stride > (int64_t)1 << 38) return false;
    if (!targets || (targets->type != CO3_I32 && targets->type != CO3_I64) || targets->top < 1) return false;
    if (teacher ? targets->top > h->max_top || !array_fine(teacher, h->users, n_tokens, targets->top, false) : targets->top != 1) return false;
    if (n_tokens && (!targets->data || !aligned_to(targets->data, targets->type == CO3_I32 ? 4 : 8))) return false;
    if (!stride_fine(h->users, targets->user_stride) || !stride_fine(n_tokens, targets->token_stride)) return false;
    // its reciprocal, and that times log2(e), are normal numbers
    return temperature >= 1e-30f && temperature <= 1e30f && (teacher || temperature == 1.0f);
}

template <class T> int forward_of(co3_token_loss* h, Call& c, float temperature, float* loss, float* lse, cudaStream_t st) {
    GemmArgs& a = c.g;
    a.columns = a.vocab;
    const int64_t tiles = up_to(c.rows, TILE) / TILE * (up_to(h->vocab, TILE) / TILE);
    int rc = gemm(h, c.one ? gemm_kernel<STATS, T, T, true, false> : gemm_kernel<STATS, T, T, false, false>, tiles, a, st);
    if (rc != CO3_OK) return rc;
    LossArgs l;
    l.stats = h->stats; l.dots = h->dots; l.constant = c.one ? nullptr : h->constant; l.rows = h->rows; l.n_all = c.n_all; l.tiles = h->tiles;
    l.inv_t = 1.0f / temperature; l.p = h->p; l.loss = loss; l.lse = lse;
    return launch_early(&h->launches, loss_kernel, dim3((unsigned)((c.n_all + 31) / 32)), 32 * LOSS_WARPS, 0, 1, st, l);
}

template <class T> int backward_of(co3_token_loss* h, Call& c, const co3_array* dhidden, const co3_param_grad* dweight, int64_t n_tokens, cudaStream_t st) {
    const bool low = dweight && dweight->type == CO3_F32;
    const int64_t mt = up_to(c.rows, TILE) / TILE, nt = up_to(h->dim, TILE) / TILE;
    int rc = CO3_OK, splits = 1, wide = 0;
    CUtensorMap map_dw;
    if (dweight) {
        const int width = type_width(dweight->type);
        wide = !dweight->accumulate && aligned_to(dweight->data, 16) && h->dim * width % 16 == 0 && (h->users == 1 || dweight->user_stride * width % 16 == 0) &&
               make_out_map(h, &map_dw, dweight->data, dweight->type, h->vocab, h->users, h->users > 1 ? dweight->user_stride : h->dim * h->vocab);
    }
    if (dhidden) splits = splits_of(h, mt * nt, c.rows, up_to(h->piece < h->vocab ? h->piece : h->vocab, KB) / KB);
    for (int64_t v0 = 0; v0 < h->vocab && rc == CO3_OK; v0 += h->piece) {
        GemmArgs a = c.g;
        a.out = h->map_dz_out; a.out_low = h->map_low_out;
        a.v0 = (int)v0;
        a.columns = (int)(h->vocab - v0 < h->piece ? h->vocab - v0 : h->piece);
        const int64_t ct = up_to(a.columns, TILE) / TILE;
        // dz is summed alike with and without dweight: so dhidden has the same bits
        void (*dz)(GemmArgs) = low                       ? (c.one ? gemm_kernel<DZ, T, OF32, true, true> : gemm_kernel<DZ, T, OF32, false, true>)
                               : h->grad_type == CO3_F32 ? (c.one ? gemm_kernel<DZ, T, OF32, true, false> : gemm_kernel<DZ, T, OF32, false, false>)
                                                         : (c.one ? gemm_kernel<DZ, T, T, true, false> : gemm_kernel<DZ, T, T, false, false>);
        rc = gemm(h, dz, mt * ct, a, st);
        if (rc == CO3_OK && dhidden) {
            GemmArgs b = a;
            b.a = h->map_dz; b.out = h->map_partial; b.splits = splits; b.add = v0 > 0;
            rc = gemm(h, gemm_kernel<DHIDDEN, T, T, true, false>, mt * nt * splits, b, st);
        }
        if (rc == CO3_OK && dweight) {
            GemmArgs b = a;
            if (wide) b.out = map_dw;
            b.a = h->map_dz; b.a_low = h->map_low; b.b = h->map_hidden; b.terms = low ? 2 : 1; b.dw = *dweight;
            b.dw_wide = wide;
            rc = gemm(h, low ? gemm_kernel<DWEIGHT, T, OF32, true, false> : gemm_kernel<DWEIGHT, T, T, true, false>, ct * nt * h->users, b, st);
        }
    }
    if (rc != CO3_OK || !dhidden) return rc;
    HiddenArgs d;
    d.partial = h->partial; d.rows = h->rows; d.splits = splits; d.dim = (int)h->dim; d.slabs = (int)((h->dim + 255) / 256); d.items = c.n_all * d.slabs;
    d.tokens = (uint32_t)n_tokens; d.p = h->p; d.out = dhidden->data; d.ou = dhidden->user_stride; d.ot = dhidden->token_stride;
    const dim3 grid((unsigned)((d.items + 7) / 8));
    return rows_aligned(dhidden, h->users, n_tokens) ? launch_early(&h->launches, hidden_kernel<T, true>, grid, 256, 0, 1, st, d)
                                                     : launch_early(&h->launches, hidden_kernel<T, false>, grid, 256, 0, 1, st, d);
}

}  // namespace

extern "C" void co3_token_loss_destroy(co3_token_loss* h) {
    if (!h) return;
    if (h->slab) cudaFree(h->slab);
    delete h;
}

extern "C" int co3_token_loss_create(co3_token_loss** out, const co3_token_loss_config* cfg) {
    if (!out || !cfg) return CO3_EINVAL;
    *out = nullptr;
    if (cfg->vocab < 1 || cfg->vocab > (int64_t)1 << 30 || cfg->dim < 8 || cfg->dim % 8 || cfg->dim > 1 << 20) return CO3_EINVAL;
    if (cfg->n_users < 1 || cfg->n_users > OPS_MAX_USERS || cfg->max_tokens < 0 || cfg->max_tokens > ((int64_t)1 << 26) / cfg->n_users) return CO3_EINVAL;
    if (cfg->type != CO3_BF16 && cfg->type != CO3_F16) return CO3_EINVAL;
    if ((cfg->grad_type != CO3_F32 && cfg->grad_type != cfg->type) || cfg->max_top < 1 || cfg->max_top > MAX_TOP) return CO3_EINVAL;
    co3_token_loss* h = new (std::nothrow) co3_token_loss();
    if (!h) return CO3_ENOMEM;
    memset((void*)h, 0, sizeof(*h));
    h->vocab = cfg->vocab; h->dim = cfg->dim; h->max_tokens = cfg->max_tokens; h->users = cfg->n_users;
    h->type = cfg->type; h->grad_type = cfg->grad_type; h->max_top = cfg->max_top;
    h->tiles = (int)((h->vocab + TILE - 1) / TILE);
    h->rows = up_to(up_to(h->max_tokens, ALIGN_ROWS) * h->users, TILE);
    if (h->rows == 0) h->rows = TILE;
    // dz of a piece of the vocabulary: 256 MB, at least 2048 columns.  Pieces of one size.
    const int64_t padded = up_to(h->vocab, TILE);
    int64_t piece = ((int64_t)1 << 27) / h->rows / TILE * TILE;
    if (piece < 2048) piece = 2048;
    if (piece > padded) piece = padded;
    const int64_t pieces = (padded + piece - 1) / piece;
    h->piece = up_to((h->vocab + pieces - 1) / pieces, TILE);
    const int64_t splits = ((int64_t)1 << 25) / (h->rows * h->dim);
    h->max_splits = (int)(splits < 1 ? 1 : splits > 32 ? 32 : splits);
    int rc = CO3_OK, sms = 0;
    void* encode = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDevice(&h->device) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, h->device) != cudaSuccess || sms < 2 ||
        cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &encode, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess || !encode) rc = CO3_ECUDA;
    h->pairs = sms / 2;
    h->encode = (EncodeTiled)encode;
    if (rc == CO3_OK && !(h->type == CO3_BF16 ? all_big<OBf16>() : all_big<OF16>())) rc = CO3_ECUDA;
    if (rc == CO3_OK) {
        size_t at = 0;
        auto part = [&](size_t bytes) { const size_t o = at; at += (bytes + 1023) / 1024 * 1024; return o; };
        const size_t tokens = (size_t)(h->max_tokens * h->users), rows = (size_t)h->rows, top = h->max_top > 1 ? h->max_top : 1;
        const size_t segs = (size_t)((h->max_tokens + SEG - 1) / SEG) * h->users;
        const size_t o_status = part(sizeof(OpsStatus)), o_off = part(4 * (size_t)(h->users + 1)), o_cnt = part(4 * (size_t)h->users), o_up = part(4 * (size_t)h->users);
        const size_t o_rt = part(4 * rows), o_tr = part(4 * tokens), o_c = part(4 * rows), o_lse = part(4 * rows), o_tgt = part(4 * rows);
        const size_t o_sc = part(4 * segs), o_sm = part(4 * segs);
        const size_t o_h = part(rows * h->dim * 2), o_stats = part(8 * rows * h->tiles), o_dots = part(4 * rows * h->tiles);
        const size_t o_dz = part(rows * h->piece * 2), o_low = part(h->grad_type == CO3_F32 ? rows * h->piece * 2 : 0);
        const size_t o_part = part(4 * rows * h->dim * h->max_splits);
        const size_t o_e = part(4 * tokens * top), o_q = part(4 * tokens * top), o_k = part(4 * tokens), o_f = part(tokens * h->tiles), o_m = part(tokens);
        if (cudaMalloc(&h->slab, at) != cudaSuccess) { h->slab = nullptr; rc = CO3_ENOMEM; }
        else {
            char* base = (char*)h->slab;
            h->status = (OpsStatus*)(base + o_status);
            h->p.offset = (int32_t*)(base + o_off); h->p.count = (int32_t*)(base + o_cnt); h->p.up = (float*)(base + o_up);
            h->p.row_token = (int32_t*)(base + o_rt); h->p.token_row = (int32_t*)(base + o_tr); h->p.row_c = (float*)(base + o_c);
            h->p.row_lse = (float*)(base + o_lse); h->p.row_target = (int32_t*)(base + o_tgt);
            h->seg_count = (int32_t*)(base + o_sc); h->seg_most = (float*)(base + o_sm);
            h->hidden = base + o_h; h->stats = (float2*)(base + o_stats); h->dots = (float*)(base + o_dots);
            h->dz = base + o_dz; h->low = base + o_low; h->partial = (float*)(base + o_part);
            h->entry = (int32_t*)(base + o_e); h->q = (float*)(base + o_q); h->constant = (float*)(base + o_k); h->first = (uint8_t*)(base + o_f); h->mass = (uint8_t*)(base + o_m);
            if (cudaMemset(h->status, 0, sizeof(OpsStatus)) != cudaSuccess || cudaStreamSynchronize(nullptr) != cudaSuccess ||
                !make_map(h, &h->map_hidden, h->hidden, h->dim, h->rows, h->dim) || !make_map(h, &h->map_dz, h->dz, h->piece, h->rows, h->piece) ||
                !make_out_map(h, &h->map_partial, h->partial, CO3_F32, h->rows, h->max_splits, h->rows * h->dim) || !make_map(h, &h->map_dz_out, h->dz, h->piece, h->rows, h->piece, 32) ||
                (h->grad_type == CO3_F32 && (!make_map(h, &h->map_low, h->low, h->piece, h->rows, h->piece) || !make_map(h, &h->map_low_out, h->low, h->piece, h->rows, h->piece, 32)))) rc = CO3_ECUDA;
        }
    }
    if (rc != CO3_OK) { (void)cudaGetLastError(); co3_token_loss_destroy(h); return rc; }
    *out = h;
    return CO3_OK;
}

extern "C" int co3_token_loss_forward(co3_token_loss* h, const co3_array* hidden, const void* weight, int64_t weight_stride, const co3_tokens* targets,
                                      const co3_array* teacher, float temperature, int64_t n_tokens, float* loss, float* lse, void* cuda_stream) {
    if (!call_fine(h, hidden, weight, weight_stride, targets, teacher, temperature, n_tokens) || !device_is(h->device)) return CO3_EINVAL;
    if (n_tokens == 0) return CO3_OK;
    if (!loss || !lse || !aligned_to(loss, 4) || !aligned_to(lse, 4)) return CO3_EINVAL;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    Call c;
    const int rc = begin_call(h, hidden, weight, weight_stride, targets, teacher, temperature, n_tokens, nullptr, nullptr, 1.0f, false, c, st);
    if (rc != CO3_OK) return rc;
    return h->type == CO3_BF16 ? forward_of<OBf16>(h, c, temperature, loss, lse, st) : forward_of<OF16>(h, c, temperature, loss, lse, st);
}

extern "C" int co3_token_loss_backward(co3_token_loss* h, const co3_array* hidden, const void* weight, int64_t weight_stride, const co3_tokens* targets,
                                       const co3_array* teacher, float temperature, int64_t n_tokens, const float* lse, const float* dloss, float scale,
                                       const co3_array* dhidden, const co3_param_grad* dweight, void* cuda_stream) {
    if (!call_fine(h, hidden, weight, weight_stride, targets, teacher, temperature, n_tokens) || !device_is(h->device)) return CO3_EINVAL;
    if (dhidden && (!array_fine(dhidden, h->users, n_tokens, h->dim, true) || dhidden->type != h->type)) return CO3_EINVAL;
    if (dweight && (!grad_fine(dweight, h->users, h->vocab * h->dim) || dweight->type != h->grad_type)) return CO3_EINVAL;
    if (n_tokens && (!lse || !aligned_to(lse, 4) || !aligned_to(dloss, 4))) return CO3_EINVAL;
    if (!(fabsf(scale / temperature) < INFINITY)) return CO3_EINVAL;
    if (n_tokens == 0) dhidden = nullptr;
    if (dhidden && n_tokens * h->users * ((h->dim + 255) / 256) > (int64_t)8 * 0x7FFFFFFF) return CO3_ELIMIT;      // thread blocks of a launch
    if (!dhidden && !dweight) return CO3_OK;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    Call c;
    const int rc = begin_call(h, hidden, weight, weight_stride, targets, teacher, temperature, n_tokens, lse, dloss, scale, true, c, st);
    if (rc != CO3_OK) return rc;
    return h->type == CO3_BF16 ? backward_of<OBf16>(h, c, dhidden, dweight, n_tokens, st) : backward_of<OF16>(h, c, dhidden, dweight, n_tokens, st);
}

extern "C" int co3_token_loss_status(co3_token_loss* h, uint32_t* flags, uint64_t* bad_tokens, int32_t clear) {
    return h ? read_status(h->device, h->status, flags, bad_tokens, clear) : CO3_EINVAL;
}
extern "C" int64_t co3_token_loss_launch_count(const co3_token_loss* h) { return h ? h->launches : 0; }
