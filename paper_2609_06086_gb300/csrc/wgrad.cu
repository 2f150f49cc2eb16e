// poseidon_ckpt_wgrad: weight gradient of a linear layer from the 8-bit
// checkpoint of its input (formulas: poseidon.h).
#include <cuda.h>

#include <algorithm>
#include <mutex>

#include "layer_ops.cuh"
#include "wait_limit.h"

namespace pos {

// The gradient's transpose dW^T [cols][n] = X^T dY is what the tensor cores
// compute: M = columns of x, N = columns of dy, K = rows (tokens).  Two SMs
// share a tile of 256 x 256: each decodes the 128 columns of x of its own half
// into shared memory, loads half of dy's columns, and one thread issues the
// products for both.  Both operands keep the rows of their matrices (M and N
// contiguous), so nothing is transposed on the way in, and a warp of the
// epilogue holds 32 consecutive columns of one row of dW at a time, so its
// stores are whole 128-byte lines.
constexpr int kTileM = 256, kTileN = 256, kTileK = 64;
constexpr int kHalf = 128;              // columns of x, and of dy, of one SM
constexpr int kStages = 5;              // operands in 16 bits
constexpr int kCodeStages = 6;          // codes and scales as they come
constexpr int kABytes = kHalf * kTileK * 2, kBBytes = kHalf * kTileK * 2;
constexpr int kCodeBytes = kHalf * kTileK, kScaleBytes = kTileK * 4;
// Warpgroups: one of loads and products, two that decode every other stage
// each (the latency of a stage is then two stages long), two of sums.
constexpr int kDecodeGroups = 2, kDecodeWarps = 4, kSumWarps = 8;
constexpr int kWgradThreads = 128 * (1 + kDecodeGroups) + 32 * kSumWarps;
// Registers of a thread after the split: 32 + 2 * 56 + 2 * 168 = 480 = 5 * 96,
// what the block is launched with.
constexpr int kLoadRegs = 32, kDecodeRegs = 56, kSumRegs = 168;
constexpr int kBars = 2 * kStages + 2 * kCodeStages + 4;
constexpr int kWgradSmem = 1024 + kStages * (kABytes + kBBytes) +
                           kCodeStages * (kCodeBytes + kScaleBytes) + 8 * kBars + 16;
constexpr int kAccCols = 256;           // TMEM columns of one accumulator; two alternate
// The tensor cores cut what they add to a sum instead of rounding it, so a
// long sum drifts towards zero by about 1e-9 of its size per row (measured:
// 2.6e-6 over 4096 rows).  An accumulator therefore takes 768 rows, and the
// sums of those are added in registers, with rounding: 3.4e-7 over 4096 rows.
// 4096 x 4864 x 4096 took 103.6 us so; 106.0 with 512 rows each, 102 with 1024
// and half as much error again (now 106.6: the votes on the decoding warps' waits).
constexpr int kChunkRows = 768;

struct WgradParams {
    const uint8_t *scales;
    const float *in;
    float *out, *part;     // part: tiles [256][256] of the split tiles' partial sums
    int64_t rows, ld, spitch;
    int32_t n, cols;
    int32_t tile_n;        // columns of dy of a tile: 64, 128 or 256
    int32_t tiles_m, tiles_n;  // under tile_n = 256, tiles_n has more than 128 columns each
    int32_t tiles;         // with tiles_m narrow ones for what is left, if it is
    int32_t whole;         // tiles with all rows in one unit: the first ones
    int32_t units;         // whole + splits * (tiles - whole)
    int32_t splits;
    int64_t split_rows;    // a multiple of kTileK
};

// ---------------------------------------------------------------------------
// PTX
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void *p) {
    return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t cta) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(cta));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {  // own CTA
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// A barrier in either CTA of the pair.  The default scope (the CTA) is enough:
// what the arrival orders is this SM's own shared memory or TMEM, which this
// SM's tensor core reads or writes; a release to the whole cluster waits for
// the SM's global accesses too (1884 us instead of 1008 us for 8192 rows, n =
// 10240, cols = 8192, together with the same change of the waits).
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar)
                 : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
                 : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(1000000)  // sleeps for up to 1 ms
        : "memory");
    return ok;
}
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
// Waits for a phase, two seconds at most (WaitLimit); false: it did not come, or
// another wait of the block has already given up.
__device__ __forceinline__ bool bar_wait_long(uint32_t bar, uint32_t parity, volatile int *gave_up) {
    WaitLimit limit(now_ns());
    for (;;) {
        if (bar_try(bar, parity)) return true;
        if (*gave_up) return false;
        if (limit.reached(now_ns())) {
            *gave_up = 1;
            return false;
        }
    }
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *gave_up) {
    if (bar_try(bar, parity)) return true;
    return bar_wait_long(bar, parity, gave_up);
}
// The same by a whole warp.  Where a wait gives up its lanes may not agree (one sees
// the phase on its last try, another that the block has given up), and lanes that went
// on would wait in the warp's next vote for those that left: all go on or none does.
__device__ __forceinline__ bool bar_wait_warp(uint32_t bar, uint32_t parity,
                                              volatile int *gave_up) {
    return __all_sync(0xffffffffu, bar_wait(bar, parity, gave_up));
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int x, int y,
                                         uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], "
        "[%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
// The same with the barrier in either SM of the pair.
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap *map, int x, int y,
                                              uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
// Operand tile of 64 rows x 128 columns: two blocks of 64 columns (128 bytes,
// swizzled), kTileK rows each.  Leading offset: the next 64 columns; stride
// offset: the next 8 rows.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr) {
    return (uint64_t)(addr >> 4 & 0x3fffu) | (uint64_t)(kTileK * 128 >> 4) << 16 |
           (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                         uint32_t add) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(add)
        : "memory");
}
// Arrives on a barrier of both SMs once the products issued so far are done.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 "
        "[%0], %1;" ::"r"(bar),
        "h"((uint16_t)3)
        : "memory");
}
__device__ __forceinline__ void tmem_load8(uint32_t addr, uint32_t (&r)[8]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
// Four bytes by an asynchronous copy, or zeros.
__device__ __forceinline__ void copy_word(uint32_t dst, const void *src, bool there) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src),
                 "r"(there ? 4 : 0)
                 : "memory");
}
// Arrives once the thread's asynchronous copies so far have landed.
__device__ __forceinline__ void bar_arrive_copies(uint32_t bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
template <int R>
__device__ __forceinline__ void give_registers() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R));
}
template <int R>
__device__ __forceinline__ void take_registers() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R));
}

// ---------------------------------------------------------------------------
// Decoding codes into 16-bit values
// ---------------------------------------------------------------------------
__device__ __forceinline__ __nv_bfloat162 as_bf2(uint32_t u) {
    __nv_bfloat162 v;
    memcpy(&v, &u, 4);
    return v;
}
__device__ __forceinline__ __half2 as_h2(uint32_t u) {
    __half2 v;
    memcpy(&v, &u, 4);
    return v;
}
template <typename V>
__device__ __forceinline__ uint32_t bits_of(V v) {
    uint32_t u;
    memcpy(&u, &v, 4);
    return u;
}

// The order of the columns of x among the rows of a tile: the four of a word
// of codes give the words (0, 2) and (1, 3), which masks alone separate.
__device__ __forceinline__ int column_at(int row) {
    return (row & ~3) | (row & 1) << 1 | (row >> 1 & 1);
}

// Scales under which the short ways below are exact, or round once as
// poseidon_ckpt_unpack does, and cannot saturate.
template <typename T, int F>
__device__ __forceinline__ bool short_way(int byte) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        return byte <= (F == POS_CKPT_INT8 ? 127 + 119   // 256 * 2^e is finite
                                           : 127 + 7);   // the factor 2^(120 + e) is
    else if constexpr (F == POS_CKPT_INT8)
        return byte >= 127 - 24 && byte <= 127 + 5;    // 1024 * 2^e to 1280 * 2^e are normal
    else
        return byte >= 127 - 32 && byte <= 127 + 7;    // 2^(8 + e) is an f16, 448 * 2^7 < 65504
}
// The factor of a short way in both halves of a word; int8: what
// the code's zero stands at, 128 * 2^e in bf16 and 1024 * 2^e in f16.
template <typename T, int F>
__device__ __forceinline__ uint32_t short_factor(int byte) {
    uint32_t f;
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        f = (uint32_t)(byte + (F == POS_CKPT_INT8 ? 7 : 120)) << 7;
    } else {
        const int e = byte - 127 + (F == POS_CKPT_INT8 ? 10 : 8);
        f = e >= -14 ? (uint32_t)(e + 15) << 10 : 1u << (e + 24);
    }
    return f | f << 16;
}
// Four codes as two words.
//   int8 -> bf16: byte s m (s: one bit, m: seven) gives, under the exponent of
//     128 * 2^e, (128 + m) * 2^e and, s added to the exponent, 128 (1 + s) 2^e;
//     their difference is the value, exactly.
//   int8 -> f16: the code + 128 as the last byte of (1024 + it) 2^e, minus
//     1152 * 2^e: exact, f16 having ten bits after the first.
//   e4m3 -> bf16, f16: sign, exponent and mantissa in their places are the
//     value times 2^-120 or 2^-8, subnormals too.
template <typename T, int F>
__device__ __forceinline__ uint2 decode4(uint32_t w, uint32_t factor) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        if constexpr (F == POS_CKPT_INT8) {
            const uint32_t h = w >> 8;
            return make_uint2(bits_of(__hsub2(as_bf2((w & 0x007f007fu) | factor),
                                              as_bf2((w & 0x00800080u) + factor))),
                              bits_of(__hsub2(as_bf2((h & 0x007f007fu) | factor),
                                              as_bf2((h & 0x00800080u) + factor))));
        }
        const uint32_t even = (w << 8 & 0x80008000u) | (w << 4 & 0x07f007f0u);
        const uint32_t odd = (w & 0x80008000u) | (w >> 4 & 0x07f007f0u);
        return make_uint2(bits_of(__hmul2(as_bf2(even), as_bf2(factor))),
                          bits_of(__hmul2(as_bf2(odd), as_bf2(factor))));
    } else {
        if constexpr (F == POS_CKPT_INT8) {
            const uint32_t u = w ^ 0x80808080u, zero = factor | 0x00800080u;
            return make_uint2(bits_of(__hsub2(as_h2((u & 0x00ff00ffu) | factor), as_h2(zero))),
                              bits_of(__hsub2(as_h2((u >> 8 & 0x00ff00ffu) | factor), as_h2(zero))));
        }
        const uint32_t even = (w << 8 & 0x80008000u) | (w << 7 & 0x3f803f80u);
        const uint32_t odd = (w & 0x80008000u) | (w >> 1 & 0x3f803f80u);
        return make_uint2(bits_of(__hmul2(as_h2(even), as_h2(factor))),
                          bits_of(__hmul2(as_h2(odd), as_h2(factor))));
    }
}
// Eight codes as eight values in column_at's order.
template <typename T, int F>
__device__ __forceinline__ uint4 decode8_short(uint2 c, uint32_t factor) {
    const uint2 a = decode4<T, F>(c.x, factor), b = decode4<T, F>(c.y, factor);
    return make_uint4(a.x, a.y, b.x, b.y);
}
template <typename T, int F>
__device__ __forceinline__ uint4 decode8_long(uint2 c, int byte) {
    const Vec8 v = decode8<F>(c, scale_value(byte));
    Vec8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = v.v[(i & ~3) | (i & 1) << 1 | (i >> 1 & 1)];
    return from_float<T, true>(o).a;
}

// ---------------------------------------------------------------------------
// Kernel
// ---------------------------------------------------------------------------
struct Unit {
    int m0, n0, tn;  // first column of x, of dy; columns of dy: 64, 128 or 256
    int r0, r1;      // rows
    int part;        // partial sum that it writes, or -1
};
// Units of the pairs that run at once share columns: bands of 8 tiles of dy,
// through which the tiles of x pass.  Tiles for a last 128 columns of dy or
// fewer multiply only 128 or 64 and come last (4093 x 1283 x 5120, f16: 58.5 us
// instead of 61.6).
__device__ __forceinline__ void tile_of(const WgradParams &p, int tile, int &m0, int &n0,
                                        int &tn) {
    if (tile >= p.tiles_m * p.tiles_n) {
        m0 = (tile - p.tiles_m * p.tiles_n) * kTileM;
        n0 = p.tiles_n * kTileN;
        tn = p.n - n0 <= 64 ? 64 : 128;  // (only under tile_n = 256)
        return;
    }
    const int band = tile / (8 * p.tiles_m), n_band = min(8, p.tiles_n - 8 * band);
    tile -= band * 8 * p.tiles_m;
    m0 = tile / n_band * kTileM;
    n0 = (8 * band + tile % n_band) * p.tile_n;
    tn = p.tile_n;
}
__device__ __forceinline__ Unit unit_of(const WgradParams &p, int u) {
    Unit t;
    t.r0 = 0, t.r1 = (int)p.rows, t.part = -1;
    int tile = u;
    if (u >= p.whole) {
        t.part = u - p.whole;
        tile = p.whole + t.part / p.splits;
        t.r0 = (int)(t.part % p.splits * p.split_rows);
        t.r1 = (int)min(p.rows, t.r0 + p.split_rows);
    }
    tile_of(p, tile, t.m0, t.n0, t.tn);
    return t;
}

template <typename T, int F>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kWgradThreads, 1)
    wgrad_kernel(const __grid_constant__ CUtensorMap code_map,
                 const __grid_constant__ CUtensorMap dy_map, const WgradParams p) {
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char *aligned = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t a_at = base, b_at = a_at + kStages * kABytes, c_at = b_at + kStages * kBBytes;
    const uint32_t s_at = c_at + kCodeStages * kCodeBytes;
    const uint32_t bars = s_at + kCodeStages * kScaleBytes;
    const uint32_t full = bars, empty = full + 8 * kStages;
    const uint32_t code_full = empty + 8 * kStages, code_empty = code_full + 8 * kCodeStages;
    const uint32_t acc_full = code_empty + 8 * kCodeStages, acc_empty = acc_full + 16;
    const uint32_t slot = acc_empty + 16;
    unsigned char *tail = aligned + (slot - base);
    volatile int *gave_up = reinterpret_cast<volatile int *>(tail + 4);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, group = warp / 4;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;

    for (int i = threadIdx.x; i < kBars; i += kWgradThreads) {
        int count = 1;  // empty, acc_full: one commit
        // full: both SMs' decoding warps, and the arrival that expects both
        // halves of dy (in the first SM only)
        if (i < kStages) count = 1 + 2 * kDecodeWarps;
        const int j = i - 2 * kStages, k = j - 2 * kCodeStages;
        if (j >= 0 && j < kCodeStages) count = 1 + 32;  // codes, a warp's copies of scales
        if (j >= kCodeStages && k < 0) count = kDecodeWarps;
        if (k >= 2) count = 2 * kSumWarps;
        bar_init(bars + 8 * i, count);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (threadIdx.x == 0) *gave_up = 0;
    if (warp == 0 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&code_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&dy_map) : "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot),
                     "r"(2 * kAccCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    grid_dep_wait();
    grid_dep_trigger();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(tail);

    if (group == 0) {
        give_registers<kLoadRegs>();
        if (warp == 0 && lane == 0) {
            int s = 0;
            uint32_t ph = 1;  // an empty buffer's first wait passes
            const uint32_t leader_full = in_cta(full, 0);
            bool ok = true;
            for (int u = pair; u < p.units && ok; u += pairs) {
                const Unit t = unit_of(p, u);
                for (int r = t.r0; r < t.r1; r += kTileK) {
                    ok = bar_wait(empty + 8 * s, ph, gave_up);
                    if (!ok) break;
                    const int boxes = t.tn == kTileN ? 2 : 1;
                    if (rank == 0) bar_expect(full + 8 * s, 2 * boxes * (kTileK * 128));
                    for (int h = 0; h < boxes; ++h)
                        tma_load_pair(b_at + s * kBBytes + h * kTileK * 128, &dy_map,
                                      t.n0 + (int)rank * (t.tn / 2) + 64 * h, r,
                                      leader_full + 8 * s);
                    if (++s == kStages) s = 0, ph ^= 1;
                }
            }
        } else if (warp == 1 && rank == 0 && lane == 0) {
            constexpr uint32_t kType = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
            // f32 sums, both operands with M / N contiguous
            constexpr uint32_t kIdesc = 1u << 4 | kType << 7 | kType << 10 | 1u << 15 | 1u << 16 |
                                        (uint32_t)(kTileM >> 4) << 24;
            int s = 0, acc = 0;
            uint32_t ph = 0, aph = 1;
            bool ok = true;
            for (int u = pair; u < p.units && ok; u += pairs) {
                const Unit t = unit_of(p, u);
                const uint32_t idesc = kIdesc | (uint32_t)(t.tn >> 3) << 17;
                for (int c = t.r0; c < t.r1 && ok; c += kChunkRows) {
                    const int c1 = min(t.r1, c + kChunkRows);
                    ok = bar_wait(acc_empty + 8 * acc, aph, gave_up);
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    for (int r = c; r < c1 && ok; r += kTileK) {
                        ok = bar_wait(full + 8 * s, ph, gave_up);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint64_t a = operand_desc(a_at + s * kABytes);
                        const uint64_t b = operand_desc(b_at + s * kBBytes);
#pragma unroll
                        for (int k = 0; k < kTileK / 16; ++k)
                            mma_pair(tmem + acc * kAccCols, a + k * (2048 >> 4),
                                     b + k * (2048 >> 4), idesc, r > c || k > 0);
                        commit_pair(empty + 8 * s);
                        if (++s == kStages) s = 0, ph ^= 1;
                    }
                    if (!ok) break;
                    commit_pair(acc_full + 8 * acc);
                    acc ^= 1;
                    if (acc == 0) aph ^= 1;
                }
            }
        } else if (warp == 2) {
            // Codes, and the scales of a stage's rows, four groups (a word) each:
            // plain asynchronous copies, since their rows may start at any word.
            // Their own warp: they are wanted some stages before dy, and waiting
            // for its place as well made them late (855 us for 8192 x 10240 x
            // 8192 instead of 829).
            int cs = 0;
            uint32_t cph = 1;
            bool ok = true;
            for (int u = pair; u < p.units && ok; u += pairs) {
                const Unit t = unit_of(p, u);
                const int m0 = t.m0 + (int)rank * kHalf;
                const uint8_t *sc = p.scales + (m0 < p.cols ? m0 / kGroup : 0);
                for (int r = t.r0; r < t.r1; r += kTileK) {
                    ok = bar_wait_warp(code_empty + 8 * cs, cph, gave_up);
                    if (!ok) break;
                    if (lane == 0) {
                        bar_expect(code_full + 8 * cs, kCodeBytes);
                        tma_load(c_at + cs * kCodeBytes, &code_map, m0, r, code_full + 8 * cs);
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int at = r + lane + 32 * h;
                        // rows and columns past the end: scale 0 (codes are zeros)
                        const bool there = m0 < p.cols && at < t.r1;
                        copy_word(s_at + cs * kScaleBytes + 4 * (lane + 32 * h),
                                  sc + (there ? at * p.spitch : 0), there);
                    }
                    bar_arrive_copies(code_full + 8 * cs);
                    if (++cs == kCodeStages) cs = 0, cph ^= 1;
                }
            }
        }
        __syncwarp();
    } else if (group <= kDecodeGroups) {
        give_registers<kDecodeRegs>();
        // A thread decodes four pieces of 16 columns: eight lanes take 64
        // columns of an even row and the other 64 of the odd row after it, so
        // that both their loads and, the swizzle shifting odd rows by one
        // piece of 16 bytes, their stores cover all banks.  Pieces h = 0, 1
        // are the two blocks of 64 columns, h = 2, 3 the same 32 rows on.
        const int mine = group - 1;
        const int piece = threadIdx.x % 4, odd = threadIdx.x / 4 % 2;
        const int row = 2 * (threadIdx.x % 128 / 8) + odd;
        const uint32_t from[2] = {c_at + row * kHalf + (piece + 4 * odd) * 16,
                                  c_at + row * kHalf + (piece + 4 * (odd ^ 1)) * 16};
        const uint32_t scale_at = s_at + row * 4 + piece / 2;
        const uint32_t to_row = a_at + row * 128 + odd * (kTileK * 128);
        const uint32_t to[2] = {to_row + (((2 * piece) ^ (row & 7)) << 4),
                                to_row + (((2 * piece + 1) ^ (row & 7)) << 4)};
        const uint32_t other = odd ? 0u - kTileK * 128 : kTileK * 128;  // to the other block
        const uint32_t leader_full = in_cta(full, 0);
        int s = mine, cs = mine;
        uint32_t ph = 1, cph = 0;
        int turn = 0;  // of the groups, over all stages
        bool ok = true;
        for (int u = pair; u < p.units && ok; u += pairs) {
            const Unit t = unit_of(p, u);
            for (int r = t.r0; r < t.r1; r += kTileK) {
                const bool skip = turn != mine;
                if (++turn == kDecodeGroups) turn = 0;
                if (skip) continue;
                // Lanes may differ in whether a wait gave up, so all of them vote before
                // the loads, on their first tries alone where those pass: 154.2 us for
                // 4096 x 6144 x 4096 with dw_in, 155.5 with one vote on both waits (whose
                // loops are then in the way), 154.8 with the loads before the second
                // wait; 152.9 without any vote.
                ok = __all_sync(0xffffffffu, bar_try(code_full + 8 * cs, cph) &&
                                                 bar_try(empty + 8 * s, ph));
                if (!ok) {
                    ok = __all_sync(0xffffffffu, bar_wait(code_full + 8 * cs, cph, gave_up) &&
                                                     bar_wait(empty + 8 * s, ph, gave_up));
                    if (!ok) break;
                }
                uint4 c[4];
                uint32_t byte[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(c[h].x), "=r"(c[h].y), "=r"(c[h].z), "=r"(c[h].w)
                                 : "r"(from[h % 2] + cs * kCodeBytes + h / 2 * (32 * kHalf)));
                    asm volatile("ld.shared.u8 %0, [%1];"
                                 : "=r"(byte[h])
                                 : "r"(scale_at + 2 * (odd ^ h % 2) + cs * kScaleBytes +
                                       h / 2 * (32 * 4)));
                }
                const bool all_short = __all_sync(
                    0xffffffffu, short_way<T, F>((int)byte[0]) && short_way<T, F>((int)byte[1]) &&
                                     short_way<T, F>((int)byte[2]) && short_way<T, F>((int)byte[3]));
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const uint2 lo = make_uint2(c[h].x, c[h].y), hi = make_uint2(c[h].z, c[h].w);
                    uint4 v[2];
                    if (all_short) {
                        const uint32_t f = short_factor<T, F>((int)byte[h]);
                        v[0] = decode8_short<T, F>(lo, f);
                        v[1] = decode8_short<T, F>(hi, f);
                    } else {
                        v[0] = decode8_long<T, F>(lo, (int)byte[h]);
                        v[1] = decode8_long<T, F>(hi, (int)byte[h]);
                    }
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                                         to[q] + s * kABytes + h % 2 * other + h / 2 * (32 * 128)),
                                     "r"(v[q].x), "r"(v[q].y), "r"(v[q].z), "r"(v[q].w));
                }
                // Orders the stores before the tensor cores' reads and the loads
                // before the next copy into the codes' place: an arrival alone
                // does neither.
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    bar_arrive_cluster(leader_full + 8 * s);
                    bar_arrive(code_empty + 8 * cs);
                }
                cs += kDecodeGroups;
                if (cs >= kCodeStages) cs -= kCodeStages, cph ^= 1;
                s += kDecodeGroups;
                if (s >= kStages) s -= kStages, ph ^= 1;
            }
        }
        __syncwarp();
    } else {
        take_registers<kSumRegs>();
        // The accumulator's lanes are columns of x, its columns those of dy: a
        // warp holds 32 x 128 sums.
        const int quarter = warp % 4, side = (warp - 4 * (1 + kDecodeGroups)) / 4;
        const uint32_t leader_acc_empty = in_cta(acc_empty, 0);
        const uint32_t from = tmem + side * 128 + ((uint32_t)(32 * quarter) << 16);
        int acc = 0;
        uint32_t aph = 0;
        bool ok = true;
        for (int u = pair; u < p.units; u += pairs) {
            const Unit t = unit_of(p, u);
            const int m = (int)rank * kHalf + 32 * quarter + column_at(lane), j1 = side * 128;
            const int left = t.m0 + m < p.cols ? min(t.tn, p.n - t.n0) - j1 : 0;  // rows to write
            // dw_in is read while the first products run: all loads at once
            float sum[128];
            const float *in = p.in + (t.n0 + j1) * p.ld + t.m0 + m;
#pragma unroll
            for (int j = 0; j < 128; ++j, in += p.ld)
                sum[j] = p.in && t.part < 0 && j < left ? *in : 0.f;
            for (int c = t.r0; c < t.r1; c += kChunkRows) {
                if (ok) ok = bar_wait_warp(acc_full + 8 * acc, aph, gave_up);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int j0 = 0; j0 < 128; j0 += 8) {
                    if (j1 + j0 >= t.tn) break;  // the others of a narrow tile stay 0
                    uint32_t v[8];
                    tmem_load8(from + acc * kAccCols + j0, v);
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j0 + j] += __uint_as_float(v[j]);
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(leader_acc_empty + 8 * acc);
                acc ^= 1;
                if (acc == 0) aph ^= 1;
            }
            // a wait that gave up: no sums
            const float lost = ok ? 0.f : __uint_as_float(0x7fffffffu);
            if (t.part >= 0) {
                float *out = p.part + (int64_t)t.part * (kTileM * kTileN) + j1 * kTileM + m;
#pragma unroll
                for (int j = 0; j < 128; ++j) out[j * kTileM] = sum[j] + lost;
            } else {
                float *out = p.out + (t.n0 + j1) * p.ld + t.m0 + m;
#pragma unroll
                for (int j = 0; j < 128; ++j, out += p.ld)
                    if (j < left) *out = sum[j] + lost;
            }
        }
        __syncwarp();
    }
    // Where a wait gave up, copies and products may still be on their way:
    // they end by themselves within microseconds.
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    if (*gave_up) {
        const uint64_t t0 = now_ns();
        while (now_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                     "r"(2 * kAccCols));
    }
}

// The split tiles: dw = in + the parts of each in order.  A block takes 4 rows
// of a tile, a thread a column of them.
constexpr int kJoinRows = 4;
__global__ void __launch_bounds__(kTileM) wgrad_join_kernel(const WgradParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    const int tile = blockIdx.x / (kTileN / kJoinRows);
    const int j0 = blockIdx.x % (kTileN / kJoinRows) * kJoinRows;
    int m0, n0, tn;
    tile_of(p, p.whole + tile, m0, n0, tn);
    const float *part = p.part + (int64_t)tile * p.splits * (kTileM * kTileN) + j0 * kTileM +
                        threadIdx.x;
    float sum[kJoinRows] = {};
    if (j0 >= tn) return;
    for (int s = 0; s < p.splits; ++s) {
#pragma unroll
        for (int j = 0; j < kJoinRows; ++j)
            sum[j] += part[(int64_t)s * (kTileM * kTileN) + j * kTileM];
    }
    const int m = m0 + threadIdx.x;
    if (m >= p.cols) return;
#pragma unroll
    for (int j = 0; j < kJoinRows; ++j) {
        const int n = n0 + j0 + j;
        const int64_t at = n * p.ld + m;
        if (n < p.n) p.out[at] = p.in ? p.in[at] + sum[j] : sum[j];
    }
}

// dw = in or zeros: no rows.
__global__ void wgrad_fill_kernel(const float *in, float *out, int64_t n, int64_t cols,
                                  int64_t ld) {
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x)
        for (int64_t j = threadIdx.x; j < cols; j += blockDim.x)
            out[i * ld + j] = in ? in[i * ld + j] : 0.f;
}

// dy into rows that tensor copies can read (16-byte aligned, a multiple of 8
// elements, zeros past the last column): 8 elements a thread.
template <typename T>
__global__ void __launch_bounds__(256) wgrad_copy_kernel(const T *x, int64_t ldx, T *y,
                                                         int64_t ldy, int64_t rows, int n) {
    grid_dep_wait();
    grid_dep_trigger();
    for (int64_t j = 8 * (blockIdx.y * 256ll + threadIdx.x); j < n; j += 2048ll * gridDim.y)
        for (int64_t i = blockIdx.x; i < rows; i += gridDim.x)
            store8<true>(y + i * ldy + j, load8_shifted(x + i * ldx + j, (int)j, n - (int)j), 8);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
using EncodeTiled = decltype(&cuTensorMapEncodeTiled);
static pos_status encode_fn(EncodeTiled *out) {
    static std::mutex mu;
    static EncodeTiled fn;
    std::lock_guard<std::mutex> lock(mu);
    if (!fn) {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        POS_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000,
                                                  cudaEnableDefault, &found));
        if (found != cudaDriverEntryPointSuccess || !f)
            return fail(POS_ECUDA, "the driver has no cuTensorMapEncodeTiled");
        fn = reinterpret_cast<EncodeTiled>(f);
    }
    *out = fn;
    return POS_OK;
}

// A matrix [rows][cols] of `type`, rows `stride` bytes apart, in boxes of
// box_cols x kTileK; what lies outside reads as zeros.
static pos_status make_map(CUtensorMap *map, CUtensorMapDataType type, const void *p, int64_t rows,
                           int64_t cols, int64_t stride, int box_cols, CUtensorMapSwizzle swizzle) {
    EncodeTiled encode;
    POS_TRY(encode_fn(&encode));
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)stride};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)kTileK}, ones[2] = {1, 1};
    const CUresult r = encode(map, type, 2, const_cast<void *>(p), dims, strides, box, ones,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS)
        return fail(POS_ECUDA, "cuTensorMapEncodeTiled failed: " + std::to_string((int)r));
    return POS_OK;
}

template <typename T, int F>
static pos_status launch_wgrad(const uint8_t *ckpt, const void *dy, int64_t ld_dy,
                               WgradParams p, cudaStream_t s) {
    const CkptShape shape = ckpt_shape(p.cols);
    CUtensorMap codes, grads;
    POS_TRY(make_map(&codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, ckpt, p.rows, shape.pitch, shape.pitch,
                     kHalf, CU_TENSOR_MAP_SWIZZLE_NONE));
    POS_TRY(make_map(&grads,
                     std::is_same<T, __half>::value ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                    : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                     dy, p.rows, p.n, ld_dy * 2, 64, CU_TENSOR_MAP_SWIZZLE_128B));
    auto kern = wgrad_kernel<T, F>;
    POS_TRY(ensure_smem(reinterpret_cast<const void *>(kern), kWgradSmem));
    POS_CUDA(launch_dependent(kern, 2 * std::min(p.units, std::max(1, sm_count() / 2)),
                              kWgradThreads, kWgradSmem, s, codes, grads, p));
    const int tiles = p.tiles - p.whole;
    if (p.splits > 1)
        POS_CUDA(launch_dependent(wgrad_join_kernel, tiles * (kTileN / kJoinRows), kTileM, 0, s, p));
    return POS_OK;
}

// Tiles and cuts along the rows.  Full rounds of tiles take all rows each; the
// tiles of the last round are cut where that ends sooner, and where there are
// few tiles they are narrower.  In units of a stage (64 rows of a tile, 0.37 us,
// hardly less for a narrow tile, whose decoding is the same): a tile's sums
// leave the SM at 32 bytes a cycle, which the last one of all shows, or every
// one where there are few rows; joining takes a launch and writes and reads each
// part.  The best of all tiles and up to 24 parts, and the chosen: 8192 x 512 x 512
// 14.7 and 15.2 us, 4000 x 256 x 512 11.4 and 11.4, 4096 x 6144 x 4096 139.0 and
// 139.5, 512 x 1024 x 1024 8.2 and 8.7.
static void cut(WgradParams &p, int pairs) {
    const int64_t stages = (p.rows + kTileK - 1) / kTileK;
    double best = 1e300;
    for (int tn = kTileN; tn >= 64; tn /= 2) {
        const double stage = tn == 256 ? 1. : tn == 128 ? 0.97 : 0.95, drain = 5.5 * tn / 256;
        const int64_t n_tiles = (p.n + tn - 1) / tn, tiles = p.tiles_m * n_tiles;
        if (tn < kTileN && tiles > 4 * pairs) break;
        const int64_t whole = tiles / pairs * pairs, rest = tiles - whole;
        const double round = std::max(stages * stage, drain) + 1.;
        const double base = (double)(tiles / pairs) * round + drain;
        for (int64_t s = 1; s == 1 || (s <= stages && rest * s <= 3 * pairs && rest > 0); ++s) {
            const int64_t each = (stages + s - 1) / s;
            if ((s - 1) * each >= stages) continue;  // the last part would be empty
            const double last =
                (double)((rest * s + pairs - 1) / pairs) * (std::max(each * stage, drain) + 1.);
            const double join = 8. + 0.17 * (0.5 + 0.5 * tn / 256) * (double)(rest * s);
            const double t = base + last + (s > 1 ? join : 0.);
            if (t >= best) continue;
            best = t;
            p.tile_n = tn;
            p.tiles_n = (int32_t)(tn == kTileN ? (p.n + kTileN / 2 - 1) / kTileN : n_tiles);
            p.tiles = (int32_t)tiles;
            p.splits = (int32_t)s;
            p.split_rows = each * kTileK;
            p.whole = (int32_t)(s > 1 ? whole : tiles);
        }
    }
    p.units = p.whole + (p.tiles - p.whole) * p.splits;
}

// A block of dy's rows and columns; `codes` and `scales` at its first row.
static pos_status wgrad_block(const uint8_t *codes, const uint8_t *scales, int32_t format,
                              const void *dy, int32_t dtype, int64_t ld_dy, bool copy, int64_t rows,
                              int64_t n, int64_t cols, const float *in, float *out, int64_t ld,
                              cudaStream_t s) {
    WgradParams p = {};
    p.scales = scales;
    p.in = in, p.out = out, p.ld = ld, p.rows = rows, p.spitch = ckpt_shape(cols).spitch;
    p.n = (int32_t)n, p.cols = (int32_t)cols;
    p.tiles_m = (int32_t)((cols + kTileM - 1) / kTileM);
    if ((int64_t)p.tiles_m * ((n + kTileN - 1) / kTileN) > 0x7fffffffll / 2)
        return fail(POS_EINVAL, "wgrad: n * cols too large");
    cut(p, std::max(1, sm_count() / 2));
    // scratch: the split tiles' parts, then dy's copy
    const int64_t part_bytes =
        p.splits > 1 ? (int64_t)(p.units - p.whole) * (kTileM * kTileN) * 4 : 0;
    const int64_t ld2 = (n + 7) / 8 * 8, bytes = part_bytes + (copy ? rows * ld2 * 2 : 0);
    void *scratch = nullptr;
    if (bytes) {
        cudaMemPool_t pool;
        POS_TRY(scratch_pool(&pool));
        POS_CUDA(cudaMallocFromPoolAsync(&scratch, (size_t)bytes, pool, s));
        p.part = static_cast<float *>(scratch);
    }
    if (copy) {
        void *to = static_cast<char *>(scratch) + part_bytes;
        const dim3 grid((unsigned)std::min<int64_t>(rows, 8192),
                        (unsigned)std::min<int64_t>((ld2 / 8 + 255) / 256, 65535));
        // (either type: 16 bits are copied)
        wgrad_copy_kernel<__half><<<grid, 256, 0, s>>>(static_cast<const __half *>(dy), ld_dy,
                                                       static_cast<__half *>(to), ld2, rows,
                                                       (int)n);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) {
            cudaFreeAsync(scratch, s);
            return cuda_fail(e, "wgrad copy");
        }
        dy = to, ld_dy = ld2;
    }
    pos_status st;
    if (dtype == POS_BF16)
        st = format == POS_CKPT_INT8
                 ? launch_wgrad<__nv_bfloat16, POS_CKPT_INT8>(codes, dy, ld_dy, p, s)
                 : launch_wgrad<__nv_bfloat16, POS_CKPT_E4M3>(codes, dy, ld_dy, p, s);
    else
        st = format == POS_CKPT_INT8
                 ? launch_wgrad<__half, POS_CKPT_INT8>(codes, dy, ld_dy, p, s)
                 : launch_wgrad<__half, POS_CKPT_E4M3>(codes, dy, ld_dy, p, s);
    const cudaError_t e = scratch ? cudaFreeAsync(scratch, s) : cudaSuccess;
    if (st != POS_OK) return st;
    return e == cudaSuccess ? POS_OK : cuda_fail(e, "wgrad scratch");
}

// Where dy has to be copied, a block of it at a time, 256 MB at most: the pool that
// the copy comes from keeps what it once held.  Blocks of all rows and whole tiles of
// columns, and of fewer rows where 256 columns of all of them are more than that; the
// later ones are then added to the gradients of those before.  Every block is a launch
// of each kernel and an end with idle SMs: in blocks of 64 MB 8192 x 5121 x 512 takes
// 99 us instead of 86, 8192 x 4097 x 4096 253 instead of 241.
constexpr int64_t kCopyBytes = 256ll << 20;
// Rows of a block: the kernel counts them in 32 bits, up to kChunkRows past the last.
constexpr int64_t kBlockRows = 1ll << 30;
static pos_status wgrad(const uint8_t *ckpt, int32_t format, const void *dy, int32_t dtype,
                        int64_t ld_dy, int64_t rows, int64_t n, int64_t cols, const float *in,
                        float *out, int64_t ld, cudaStream_t s) {
    if (rows == 0) {
        wgrad_fill_kernel<<<(int)std::min<int64_t>(n, 65535), 256, 0, s>>>(in, out, n, cols, ld);
        POS_CUDA(cudaGetLastError());
        return POS_OK;
    }
    const CkptShape shape = ckpt_shape(cols);
    const bool copy = !aligned16(dy) || ld_dy % 8 || ld_dy < n;
    int64_t n_each = n, rows_each = std::min(rows, kBlockRows);
    if (copy) {
        const int64_t n8 = (n + 7) / 8 * 8;
        rows_each = std::min(
            rows_each, kCopyBytes / (2 * std::min<int64_t>(n8, kTileN)) / kTileK * kTileK);
        if (rows_each * n8 * 2 > kCopyBytes) {
            const int64_t most = kCopyBytes / (2 * rows_each) / kTileN * kTileN;
            const int64_t blocks = (n + most - 1) / most;
            n_each = ((n + blocks - 1) / blocks + kTileN - 1) / kTileN * kTileN;
        }
    }
    for (int64_t j = 0; j < n; j += n_each)
        for (int64_t r = 0; r < rows; r += rows_each)
            POS_TRY(wgrad_block(ckpt + r * shape.pitch, ckpt + rows * shape.pitch + r * shape.spitch,
                                format, static_cast<const uint16_t *>(dy) + r * ld_dy + j, dtype,
                                ld_dy, copy, std::min(rows_each, rows - r), std::min(n_each, n - j),
                                cols, r > 0 ? out + j * ld : in ? in + j * ld : nullptr,
                                out + j * ld, ld, s));
    return POS_OK;
}

}  // namespace pos

extern "C" pos_status poseidon_ckpt_wgrad(const void *d_ckpt, int32_t format, const void *d_dy,
                                          int32_t dtype, int64_t ld_dy, int64_t rows, int64_t n,
                                          int64_t cols, const float *d_dw_in, float *d_dw_out,
                                          int64_t ld_dw, void *stream) {
    using namespace pos;
    return guarded([&]() -> pos_status {
        if (!ckpt_size_ok(rows, cols) || n < 0 || rows >= (1ll << 31) - kTileK ||
            n >= (1ll << 31) - kTileN || cols >= (1ll << 31) - kTileM)
            return fail(POS_EINVAL, "wgrad: bad rows, n or cols");
        if (dtype != POS_BF16 && dtype != POS_F16)
            return fail(POS_EINVAL, "wgrad: dy must be bf16 or f16");
        if (!format_ok(format)) return fail(POS_EINVAL, "wgrad: unknown format");
        if (ld_dy < 0 || ld_dw < 0 || ld_dy >= (1ll << 38) || ld_dw >= (1ll << 31) || ld_dw < cols)
            return fail(POS_EINVAL, "wgrad: bad row stride");
        if (n == 0 || cols == 0) return POS_OK;
        if (!d_dw_out || (rows > 0 && (!d_ckpt || !d_dy)))
            return fail(POS_EINVAL, "wgrad: NULL pointer");
        if (!aligned16(d_ckpt)) return fail(POS_EINVAL, "wgrad: checkpoint not 16-byte aligned");
        if (reinterpret_cast<uintptr_t>(d_dy) % 2 || reinterpret_cast<uintptr_t>(d_dw_in) % 4 ||
            reinterpret_cast<uintptr_t>(d_dw_out) % 4)
            return fail(POS_EINVAL, "wgrad: matrix not aligned to its elements");
        return wgrad(static_cast<const uint8_t *>(d_ckpt), format, d_dy, dtype, ld_dy, rows, n, cols,
                     d_dw_in, d_dw_out, ld_dw, static_cast<cudaStream_t>(stream));
    });
}
