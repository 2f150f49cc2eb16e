// Shared by attn.cu and attn_backward.cu: causal attention over packed sequences
// (formulas: poseidon.h).
#pragma once
#include <algorithm>
#include <type_traits>

#include "layer_ops.cuh"
#include "tensor_core.cuh"

namespace pos {

constexpr int kAttnMaxDim = 128;
constexpr int kTile = 128;                   // rows of queries or keys of a product
constexpr int kBox = kTile * 128;            // bytes of 64 columns of a tile
constexpr int kTileBytes = 2 * kBox;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A tensor [tokens][heads][dim] of 16-bit elements.
struct AttnTensor {
    const void *p;
    int64_t token, head;  // strides in elements
};

struct AttnParams {
    AttnTensor q, k, v, o, g;   // g: o's gradient; read 16 bytes at a time (except o)
    void *out, *dq, *dk, *dv;   // outputs and their strides
    int64_t out_token, out_head;
    int64_t d_token[3], d_head[3];
    float *lse;                 // [heads_q][tokens] or NULL
    float2 *stats;              // backward: [heads_q][tokens]: lse in powers of two, D
    uint32_t *largest;          // backward in f16: bits of the largest |dO|^2 of a row, of each
                                // [sequence][key head]
    float *values;              // the largest |v|^2 of a tile, [heads_k][its first token],
    float *most;                // and of a sequence, as `largest` is
    float *part;                // backward: sums of parts of the keys' gradients
    int32_t parts, first_blocks;  // blocks of the keys' kernel that start at once (no list: all)
    const int4 *tiles;          // of the sequences (attn_tiles_kernel), or NULL: one sequence
    const int32_t *n_tiles;
    int64_t tokens;
    int32_t heads_q, heads_k, group, dim;  // dim: a multiple of 8
    int32_t dim_out;            // elements of a row that are written
    bool out_vectors, d_vectors[3];  // rows that can be written 16 bytes at a time
    float scale, scale2;        // scale2 = scale * log2(e)
    uint64_t wait_ns;           // how long a wait lasts, and a try of it
    uint32_t try_ns;
};

// A tile of queries or keys: the first token of its sequence, the sequence's
// length, which tile of it, and a number of the sequence's own.
struct AttnUnit {
    int start, len, tile, sequence;
};
template <int ROWS>
__device__ __forceinline__ bool unit_at(const AttnParams &p, int i, AttnUnit &u) {
    if (!p.tiles) {  // longest first, as the list is
        u.start = 0, u.len = (int)p.tokens, u.sequence = 0;
        u.tile = (u.len + ROWS - 1) / ROWS - 1 - i;
        return u.tile >= 0;
    }
    if (i >= *p.n_tiles) return false;
    const int4 t = p.tiles[i];
    u.start = t.x, u.len = t.y, u.tile = t.z, u.sequence = t.w;
    return true;
}

// A block's units, tiles of ROWS queries of a head, one after another: in rounds, every
// second one in the opposite order, since they are sorted by their length.
template <int ROWS>
struct BlockUnit {
    AttnUnit u;
    int head;
    __device__ __forceinline__ bool next(const AttnParams &p, int &round) {
        const int64_t total =
            (int64_t)(p.tiles ? *p.n_tiles : ((int)p.tokens + ROWS - 1) / ROWS) * p.heads_q;
        for (;; ++round) {
            const int64_t start = (int64_t)round * gridDim.x;
            if (start >= total) return false;
            const int64_t at = start + (round & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
            if (at >= total) continue;
            head = (int)(at % p.heads_q);
            unit_at<ROWS>(p, (int)(at / p.heads_q), u);
            ++round;
            return true;
        }
    }
};

// ---------------------------------------------------------------------------
// PTX
// ---------------------------------------------------------------------------
// What a block's warps share besides tiles and barriers.
struct AttnShared {
    uint32_t tmem;
    volatile int gave_up, again;        // a wait did; warps that do rows again
    uint32_t largest[2];                // of dO, units in turn
    volatile int bad[2][2][2];          // of units in turn: see the kernels
};
constexpr int kSharedBytes = 56;
static_assert(sizeof(AttnShared) <= kSharedBytes, "room for it");
__device__ __forceinline__ void init_shared(AttnShared *sh) {
    sh->gave_up = sh->again = 0;
    for (int i = 0; i < 8; ++i) sh->bad[i / 4][i / 2 % 2][i % 2] = 0;
    sh->largest[0] = sh->largest[1] = 0;
}
// Waits for a phase, two seconds at most (WaitLimit), not counting time in which the block
// does rows again.  Where one ran out, the warps that write results go on through the rest of
// the block's units without waiting, and make theirs NaN: what was in memory is not to pass for
// a result.
struct Waits {
    AttnShared *sh;
    uint64_t ns;
    uint32_t try_ns;
    __device__ __forceinline__ Waits(AttnShared *sh, const AttnParams &p)
        : sh(sh), ns(p.wait_ns), try_ns(p.try_ns) {}
};
__device__ __forceinline__ bool attn_wait_long(uint32_t bar, uint32_t parity, const Waits &w) {
    WaitLimit limit(now_ns());
    for (;;) {
        if (bar_try(bar, parity, w.try_ns)) return true;
        if (w.sh->gave_up) return false;
        if (w.sh->again) limit = WaitLimit(now_ns());
        if (w.ns == 0 || limit.reached(now_ns(), w.ns)) {
            w.sh->gave_up = 1;
            return false;
        }
    }
}
__device__ __forceinline__ bool attn_wait(uint32_t bar, uint32_t parity, const Waits &w) {
    if (bar_try(bar, parity, w.try_ns)) return true;
    return attn_wait_long(bar, parity, w);
}
// A wait of a whole warp: all lanes go on or none does.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, const Waits &w) {
    if (__all_sync(0xffffffffu, bar_try(bar, parity, w.try_ns))) return true;
    return __all_sync(0xffffffffu, attn_wait(bar, parity, w));
}
// By a warp, the rows of a mask again (row(i) does the i-th).  What its lanes stored of
// them before comes first: votes and shuffles alone order no memory.
template <typename F>
__device__ __forceinline__ void do_again(uint32_t rows, AttnShared *sh, F row) {
    if (!rows) return;
    __syncwarp();
    if (threadIdx.x % 32 == 0) atomicAdd(const_cast<int *>(&sh->again), 1);
    for (; rows; rows &= rows - 1) row(__ffs(rows) - 1);
    __syncwarp();
    if (threadIdx.x % 32 == 0) atomicAdd(const_cast<int *>(&sh->again), -1);
}
// The block's end.  Where a wait gave up, copies and products may still be on their way:
// they end by themselves within microseconds.
__device__ __forceinline__ void end_block(AttnShared *sh) {
    __syncthreads();
    if (sh->gave_up) {
        const uint64_t t0 = now_ns();
        while (now_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
}
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap *map, int x, int head,
                                         int token, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], "
        "[%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(head), "r"(token), "r"(bar)
        : "memory");
}
// Products are issued by one thread of a warp whose lanes all run the code, so that
// the operands' descriptors are computed in uniform registers: issued in a branch that
// one lane takes, a product of 128 x 128 x 16 took 90 to 130 cycles to issue, and 64 to
// compute.
__device__ __forceinline__ uint32_t one_lane() {
    uint32_t r;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(r));
    return r;
}
// Operand descriptors of a tile in shared memory: blocks of 64 columns, 128 bytes a
// row, swizzled.  Low words: rows whose elements are the products' inner index (16 of
// them 32 bytes on), and rows that are the inner index themselves (16 of them 2048
// bytes on, the next 64 columns a block on).  High words are alike.
constexpr uint32_t kDescHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t by_rows(uint32_t addr) { return (addr >> 4 & 0x3fffu) | 1u << 16; }
__device__ __forceinline__ uint32_t by_columns(uint32_t addr) {  // (in a cluster an address has
    return (addr >> 4 & 0x3fffu) | (uint32_t)(kBox >> 4) << 16;  // the block's rank above)
}
// f32 sums of 16-bit products, 128 rows, n columns.
template <typename T>
__device__ __forceinline__ uint32_t product_of(int n, bool b_by_columns) {
    constexpr uint32_t kType = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
    return 1u << 4 | kType << 7 | kType << 10 | (b_by_columns ? 1u << 16 : 0u) |
           (uint32_t)(n >> 3) << 17 | (uint32_t)(kTile >> 4) << 24;
}
// Both operands in shared memory.
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                       uint32_t add, uint32_t mine) {
    asm volatile(
        "{\n.reg .pred p, q;\n.reg .b64 a, b;\nsetp.ne.u32 p, %4, 0;\nsetp.ne.u32 q, %5, 0;\n"
        "mov.b64 a, {%1, %6};\nmov.b64 b, {%2, %6};\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(add), "r"(mine), "r"(kDescHigh)
        : "memory");
}
// The first operand in TMEM: two elements of a row in a column's word.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                       uint32_t add, uint32_t mine) {
    asm volatile(
        "{\n.reg .pred p, q;\n.reg .b64 b;\nsetp.ne.u32 p, %4, 0;\nsetp.ne.u32 q, %5, 0;\n"
        "mov.b64 b, {%2, %6};\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(add), "r"(mine), "r"(kDescHigh)
        : "memory");
}
// d = A B^T over 16 `steps` elements of the rows of two tiles.
template <typename T>
__device__ __forceinline__ void mma_rows(uint32_t d, uint32_t a, uint32_t b, int steps,
                                         uint32_t mine) {
    const uint32_t idesc = product_of<T>(kTile, false), da = by_rows(a), db = by_rows(b);
#pragma unroll
    for (int k = 0; k < kAttnMaxDim / 16; ++k) {
        const uint32_t at = (k / 4 * kBox + k % 4 * 32) >> 4;
        if (k < steps) mma_ss(d, da + at, db + at, idesc, k > 0, mine);
    }
}
// d (+)= A B, A [128][128] in TMEM, `part` columns of it one after another and then as many
// unused or with the rests of those (pack2_rest), B the rows of a tile, 16 `steps` columns of it.
template <typename T, int PART = kTile>
__device__ __forceinline__ void mma_columns(uint32_t d, uint32_t a, uint32_t b, int steps, bool add,
                                            uint32_t mine) {
    const uint32_t idesc = product_of<T>(16 * steps, true), db = by_columns(b);
#pragma unroll
    for (int k = 0; k < kTile / 16; ++k)
        mma_ts(d, a + (16 * k / PART * PART + 16 * k % PART / 2), db + k * (2048 >> 4), idesc,
               add || k > 0, mine);
}
// By one thread of a warp that remains together.
__device__ __forceinline__ void bar_arrive_one(uint32_t bar, uint32_t mine) {
    asm volatile(
        "{\n.reg .pred q;\nsetp.ne.u32 q, %1, 0;\n"
        "@q mbarrier.arrive.shared::cta.b64 _, [%0];\n}" ::"r"(bar),
        "r"(mine)
        : "memory");
}
// Arrives on a barrier once the products issued so far are done.
__device__ __forceinline__ void commit(uint32_t bar, uint32_t mine) {
    asm volatile(
        "{\n.reg .pred q;\nsetp.ne.u32 q, %1, 0;\n"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar),
        "r"(mine)
        : "memory");
}
__device__ __forceinline__ void tmem_before() {
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tmem_after() {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tmem_wait_stores() {
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// 16 or 32 columns of the warp's lanes.  A load and its wait are one instruction to the
// compiler: between the two it may not use, or copy, the registers.
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
        "%11, %12, %13, %14, %15}, [%16];\ntcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
        "%11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
        "%28, %29, %30, %31}, [%32];\ntcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(addr)
        : "memory");
}
// A thread's whole row of scores.
__device__ __forceinline__ void tmem_load128(uint32_t addr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, "
        "%12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, "
        "%24, %25, %26, %27, %28, %29, %30, %31"
        "}, [%128];\n"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, "
        "%44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, "
        "%56, %57, %58, %59, %60, %61, %62, %63"
        "}, [%129];\n"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%64, %65, %66, %67, %68, %69, %70, %71, %72, %73, %74, %75, "
        "%76, %77, %78, %79, %80, %81, %82, %83, %84, %85, %86, %87, "
        "%88, %89, %90, %91, %92, %93, %94, %95"
        "}, [%130];\n"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%96, %97, %98, %99, %100, %101, %102, %103, %104, %105, %106, %107, "
        "%108, %109, %110, %111, %112, %113, %114, %115, %116, %117, %118, %119, "
        "%120, %121, %122, %123, %124, %125, %126, %127"
        "}, [%131];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
          "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
          "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
          "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63]),
          "=r"(r[64]), "=r"(r[65]), "=r"(r[66]), "=r"(r[67]), "=r"(r[68]), "=r"(r[69]), "=r"(r[70]), "=r"(r[71]),
          "=r"(r[72]), "=r"(r[73]), "=r"(r[74]), "=r"(r[75]), "=r"(r[76]), "=r"(r[77]), "=r"(r[78]), "=r"(r[79]),
          "=r"(r[80]), "=r"(r[81]), "=r"(r[82]), "=r"(r[83]), "=r"(r[84]), "=r"(r[85]), "=r"(r[86]), "=r"(r[87]),
          "=r"(r[88]), "=r"(r[89]), "=r"(r[90]), "=r"(r[91]), "=r"(r[92]), "=r"(r[93]), "=r"(r[94]), "=r"(r[95]),
          "=r"(r[96]), "=r"(r[97]), "=r"(r[98]), "=r"(r[99]), "=r"(r[100]), "=r"(r[101]), "=r"(r[102]), "=r"(r[103]),
          "=r"(r[104]), "=r"(r[105]), "=r"(r[106]), "=r"(r[107]), "=r"(r[108]), "=r"(r[109]), "=r"(r[110]), "=r"(r[111]),
          "=r"(r[112]), "=r"(r[113]), "=r"(r[114]), "=r"(r[115]), "=r"(r[116]), "=r"(r[117]), "=r"(r[118]), "=r"(r[119]),
          "=r"(r[120]), "=r"(r[121]), "=r"(r[122]), "=r"(r[123]), "=r"(r[124]), "=r"(r[125]), "=r"(r[126]), "=r"(r[127])
        : "r"(addr), "r"(addr + 32), "r"(addr + 64), "r"(addr + 96)
        : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
        "%11, %12, %13, %14, %15, %16};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
        "r"(r[15])
        : "memory");
}
// 32 columns of the warp's 32 lanes, 8 values of each of four rows a thread: value
// 16 h + 4 b + 2 r + e is that of row 16 h + 8 r + lane / 4, column 8 b + lane % 4 * 2 + e;
// and 16 columns of pairs of 16-bit values in the same places.
__device__ __forceinline__ void tmem_load_block(uint32_t addr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
        "%11, %12, %13, %14, %15}, [%32];\n"
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%16, %17, %18, %19, %20, %21, %22, %23, %24, "
        "%25, %26, %27, %28, %29, %30, %31}, [%33];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(addr), "r"(addr + (16u << 16))
        : "memory");
}
__device__ __forceinline__ void tmem_store_block(uint32_t addr, const uint32_t *r) {
#pragma unroll
    for (int h = 0; h < 2; ++h, r += 8)
        asm volatile(
            "tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(
                addr + ((uint32_t)(16 * h) << 16)),
            "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
            : "memory");
}
// 2^x within two units of its last place; 0 below 2^-126.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3(uint32_t a, uint32_t b, uint32_t c) {  // bits of f32
    float r;
    asm("max.f32 %0, %1, %2, %3;"
        : "=f"(r)
        : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
    return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
    F2 r;
    asm("{\n.reg .b64 a, b, r;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\n"
        "add.rn.f32x2 r, a, b;\nmov.b64 {%0, %1}, r;\n}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
// Two values rounded to 16 bits, the first in the low half.
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// What pack2 cut off, in 16 bits.
template <typename T>
__device__ __forceinline__ uint32_t pack2_rest(uint32_t packed, float lo, float hi) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        return pack2<T>(lo - __uint_as_float(packed << 16), hi - __uint_as_float(packed & 0xffff0000u));
    const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&packed));
    return pack2<T>(lo - v.x, hi - v.y);
}
// Results on their way out: a thread's 16 columns from c on of a row, into a tile of
// shared memory (256 bytes a row, pieces of 16 bytes exchanged so that neither side's
// accesses meet in a bank) ...
template <typename T>
__device__ __forceinline__ void put_columns(uint32_t tile, int row, int c, const Vec8 (&x)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint4 v = from_float<T>(x[h]).a;
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                         tile + row * 256 + (((c / 8 + h) ^ (row & 7)) << 4)),
                     "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                     : "memory");
    }
}
// ... and from there whole rows at a time to memory.
template <typename T>
__device__ __forceinline__ void write_tile(uint32_t tile, int rows, T *out, int64_t token,
                                           bool vectors, int dim, int dim_out, int thread,
                                           int threads) {
    const int per = dim / 8;
    for (int i = thread; i < rows * per; i += threads) {
        const int row = i / per, c = i - row * per;
        Raw8<T> r;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r.a.x), "=r"(r.a.y), "=r"(r.a.z), "=r"(r.a.w)
                     : "r"(tile + row * 256 + ((c ^ (row & 7)) << 4)));
        if (vectors) store8<true>(out + row * token + 8 * c, r, dim_out - 8 * c);
        else store8<false>(out + row * token + 8 * c, r, dim_out - 8 * c);
    }
}
// What a tile holds that is not finite.  A product multiplies what is masked by 0 and would
// let a later token's infinities and NaNs into the rows before it in the tile on the
// diagonal (rows of other tiles see all of them), and what lies behind the sequence into
// all.  So a warp that has nothing else to do looks that tile over before its product, makes
// zeros of what is not finite, and tells the warps of sums which rows see it; those write
// NaNs there.  It adds up products with 0, four instructions for eight elements; where that
// is not 0, it looks column by column.
//   Both passes of 4096 tokens of 32 + 8 heads of 128: forward 105 -> 109 us, back 377 ->
// 389; with an infinity in one dO back the same, in all values of all inputs 0.6 ms.  (Rows whose
// products were not finite computed again by the formulas, one at a time by a warp: 229 ms
// for the infinity in one dO, and with the square of the length.)
__device__ __forceinline__ uint32_t tile_at(int row, int c) {  // 16 bytes of columns 8 c ..
    return c / 8 * kBox + row * 128 + ((c % 8 ^ (row & 7)) << 4);
}
// sum += 0 x of two elements.
template <typename T>
__device__ __forceinline__ void add_zeros(uint32_t &sum, uint32_t x) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(x), "r"(0));
    else
        asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(x), "r"(0));
}
// By a warp: rows `first` to `end` - 1 hold something that is not finite.
template <typename T>
__device__ __forceinline__ bool tile_bad(uint32_t tile, int first, int end, int boxes, int lane) {
    uint32_t sum[4] = {0, 0, 0, 0};
    for (int b = 0; b < boxes; ++b)
        for (int i0 = first * 8; i0 < end * 8; i0 += 8 * 32) {
            uint4 r[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int i = min(i0 + 32 * k + lane, end * 8 - 1);
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(r[k].x), "=r"(r[k].y), "=r"(r[k].z), "=r"(r[k].w)
                             : "r"(tile + b * kBox + 16 * i));
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                add_zeros<T>(sum[0], r[k].x), add_zeros<T>(sum[1], r[k].y);
                add_zeros<T>(sum[2], r[k].z), add_zeros<T>(sum[3], r[k].w);
            }
        }
    // (a NaN has other bits set than a zero's sign)
    return __any_sync(0xffffffffu, ((sum[0] | sum[1] | sum[2] | sum[3]) & 0x7fff7fffu) != 0);
}
// By a warp: zeros in their place, and f(column, first, last) by one lane of each column that
// had any.
template <typename T, typename F>
__device__ __forceinline__ void tile_clean(uint32_t tile, int from, int end, int boxes, int lane,
                                           F f) {
    for (int c = lane; c < 64 * boxes; c += 32) {
        int first = kTile, last = -1;
        for (int row = from; row < end; ++row) {
            const uint32_t at = tile + tile_at(row, c / 8) + 2 * (c % 8);
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
            if (f32_bits<T>(v & 0x7fffu) < 0x7f800000u) continue;
            first = min(first, row), last = row;
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"((uint16_t)0) : "memory");
        }
        if (last >= 0) f(c, first, last);
    }
}
// Rows become zeros: of another sequence or none.
__device__ __forceinline__ void zero_rows(uint32_t tile, int first, int end, int boxes, int lane) {
    for (int i = first * 8 + lane; i < end * 8; i += 32)
        for (int b = 0; b < boxes; ++b)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + b * kBox + 16 * i),
                         "r"(0)
                         : "memory");
}
// By the warp, before it tells others: its stores before the tensor cores' reads.
__device__ __forceinline__ void tile_done() {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}
__device__ __forceinline__ bool finite(float x) { return fabsf(x) < __uint_as_float(0x7f800000u); }

template <typename T>
__device__ __forceinline__ const T *row_at(const AttnTensor &t, int64_t token, int head) {
    return static_cast<const T *>(t.p) + token * t.token + head * t.head;
}
template <typename T>
__device__ __forceinline__ Vec8 load_row8(const T *at) {
    return to_float(load8<true>(at, 8));
}
template <typename T>
__device__ __forceinline__ float dot_rows(const T *a, const T *b, int dim) {
    float s = 0.f;
    for (int d = 0; d < dim; d += 8) {
        const Vec8 x = load_row8(a + d), y = load_row8(b + d);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += x.v[e] * y.v[e];
    }
    return s;
}
// A lane's part of a row: elements lane + 32 i.
struct RowPart {
    float v[kAttnMaxDim / 32];
};
template <typename T>
__device__ __forceinline__ void add_row(RowPart &sum, float w, const T *row, int dim, int lane) {
#pragma unroll
    for (int i = 0; i < kAttnMaxDim / 32; ++i)
        if (lane + 32 * i < dim) sum.v[i] += w * static_cast<float>(row[lane + 32 * i]);
}
template <typename T>
__device__ __forceinline__ void write_row(void *out, int64_t at, const RowPart &sum, float factor,
                                          int dim, int lane) {
#pragma unroll
    for (int i = 0; i < kAttnMaxDim / 32; ++i)
        if (lane + 32 * i < dim)
            static_cast<T *>(out)[at + lane + 32 * i] = T(sum.v[i] * factor);
}

// ---------------------------------------------------------------------------
// Host side (attn.cu)
// ---------------------------------------------------------------------------
pos_status check_attn(const pos_attn *a, AttnParams *p);
pos_status check_attn_tensor(const pos_attn *a, const pos_heads &t, int64_t heads, const char *what,
                             bool written);
pos_status attn_scratch(int64_t bytes, cudaStream_t s, void **out);
bool attn_direct(const pos_attn *a, const pos_heads &t, int64_t heads);
int64_t attn_copy_bytes(const pos_attn *a, int64_t heads);
pos_status attn_input(const pos_attn *a, const pos_heads &t, int64_t heads, char **copy,
                      cudaStream_t s, AttnTensor *out);
pos_status attn_map(CUtensorMap *map, const pos_attn *a, const AttnTensor &t, int64_t heads,
                    int32_t dim);
int64_t attn_most_tiles(const pos_attn *a, int rows);
int64_t attn_list_bytes(const pos_attn *a, int rows);
pos_status attn_list(const pos_attn *a, int rows, char **at, cudaStream_t s, AttnParams *p);
constexpr int kMostUnits = 1 << 30;
int attn_grid(const pos_attn *a, int rows, int64_t heads);

}  // namespace pos
