// poseidon_ckpt_wgrad: weight gradient of a linear layer from the 8-bit
// checkpoint of its input (formulas: poseidon.h).
#include <cuda.h>

#include <algorithm>
#include <mutex>

#include "layer_ops.cuh"

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
constexpr int kCodeStages = 6;          // codes as they come
constexpr int kABytes = kHalf * kTileK * 2, kBBytes = kHalf * kTileK * 2;
constexpr int kCodeBytes = kHalf * kTileK;
constexpr int kDecodeWarps = 8, kEpilogueWarps = 4;
constexpr int kWgradThreads = 32 * (2 + kDecodeWarps + kEpilogueWarps);
constexpr int kBars = 3 * kStages + 2 * kCodeStages + 4;
constexpr int kWgradSmem = 1024 + kStages * (kABytes + kBBytes) + kCodeStages * kCodeBytes +
                           8 * kBars + 16;
constexpr int kAccCols = 256;           // TMEM columns of one accumulator; two alternate

struct WgradParams {
    const uint8_t *scales;
    const float *in;
    float *out;
    int64_t rows, ld, spitch;
    int64_t part_stride;   // elements between the splits' partial sums (0: one split)
    int32_t n, cols;
    int32_t tiles_m, tiles_n, units;  // units = tiles * splits
    int32_t splits;
    int64_t split_rows;    // rows of a split, a multiple of chunk_rows
    int64_t chunk_rows;    // rows summed in one accumulator, a multiple of kTileK
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
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {  // any CTA of the pair
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar)
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
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok;
}
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
// Waits for a phase, two seconds at most; false: it did not come, or another
// wait of the block has already given up.
constexpr uint64_t kWaitNs = 2000000000ull;
__device__ __noinline__ bool bar_wait_long(uint32_t bar, uint32_t parity, volatile int *gave_up) {
    const uint64_t t0 = now_ns();
    for (;;) {
        for (int i = 0; i < 64; ++i)
            if (bar_try(bar, parity)) return true;
        if (*gave_up) return false;
        if (now_ns() - t0 > kWaitNs) {
            *gave_up = 1;
            return false;
        }
    }
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *gave_up) {
    if (bar_try(bar, parity)) return true;
    return bar_wait_long(bar, parity, gave_up);
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
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
          "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
          "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
          "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// ---------------------------------------------------------------------------
// Decoding 16 codes under one scale into 16-bit values
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t h2_bits(__nv_bfloat162 v) {
    uint32_t u;
    memcpy(&u, &v, 4);
    return u;
}
__device__ __forceinline__ __nv_bfloat162 bf2(uint32_t u) {
    __nv_bfloat162 v;
    memcpy(&v, &u, 4);
    return v;
}
// Four codes of a word as two words of bf16 pairs: every step is exact.
// int8: byte b of bits s m (s: 128) gives 128 + m and 128 + s as bf16, whose
// difference is the code.  e4m3: sign, exponent and mantissa moved to bf16's
// places give the value times 2^-120 (subnormals too).
template <int F>
__device__ __forceinline__ uint2 decode4_bf16(uint32_t w, __nv_bfloat162 scale) {
    uint32_t r[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (F == POS_CKPT_INT8) {
            const uint32_t b = __byte_perm(w, 0x43434343u, i ? 0x4342 : 0x4140);
            const __nv_bfloat162 q = __hsub2(bf2(b & 0xff7fff7fu), bf2(b & 0xff80ff80u));
            r[i] = h2_bits(__hmul2(q, scale));
        } else {
            const uint32_t b = __byte_perm(w, 0u, i ? 0x3424 : 0x1404);
            const uint32_t q = (b & 0x80008000u) | (b >> 4 & 0x07f007f0u);
            r[i] = h2_bits(__hmul2(__hmul2(bf2(q), bf2(0x7b807b80u)), scale));
        }
    }
    return make_uint2(r[0], r[1]);
}

// 16 codes as two 16-byte words of consecutive values.
template <typename T, int F>
__device__ __forceinline__ void decode16(uint4 c, int byte, uint4 (&v)[2]) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        // 2^e as bf16 bits, in both halves
        const uint32_t s = byte == kScaleNan ? 0x7fffu : (uint32_t)byte << 7;
        const __nv_bfloat162 s2 = bf2(s | s << 16);
        const uint2 a = decode4_bf16<F>(c.x, s2), b = decode4_bf16<F>(c.y, s2);
        const uint2 d = decode4_bf16<F>(c.z, s2), e = decode4_bf16<F>(c.w, s2);
        v[0] = make_uint4(a.x, a.y, b.x, b.y);
        v[1] = make_uint4(d.x, d.y, e.x, e.y);
    } else {
        const float s = scale_value(byte);
        v[0] = from_float<T, true>(decode8<F>(make_uint2(c.x, c.y), s)).a;
        v[1] = from_float<T, true>(decode8<F>(make_uint2(c.z, c.w), s)).a;
    }
}

// ---------------------------------------------------------------------------
// Kernel
// ---------------------------------------------------------------------------
struct Unit {
    int m0, n0;      // first column of x, of dy
    int64_t r0, r1;  // rows
    int split;
};
// Units of the pairs that run at once share columns: bands of 8 tiles of dy,
// through which the tiles of x pass.
__device__ __forceinline__ Unit unit_of(const WgradParams &p, int u) {
    Unit t;
    const int tiles = p.tiles_m * p.tiles_n;
    t.split = u / tiles;
    u -= t.split * tiles;
    const int band = u / (8 * p.tiles_m), n_band = min(8, p.tiles_n - 8 * band);
    u -= band * 8 * p.tiles_m;
    t.m0 = u / n_band * kTileM;
    t.n0 = (8 * band + u % n_band) * kTileN;
    t.r0 = t.split * p.split_rows;
    t.r1 = min(p.rows, t.r0 + p.split_rows);
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
    const uint32_t bars = c_at + kCodeStages * kCodeBytes;
    const uint32_t full = bars, empty = full + 8 * kStages;
    const uint32_t code_full = empty + 8 * kStages, code_empty = code_full + 8 * kCodeStages;
    const uint32_t acc_full = code_empty + 8 * kCodeStages, acc_empty = acc_full + 16;
    const uint32_t slot = acc_empty + 16;
    unsigned char *tail = aligned + (slot - base);
    volatile int *gave_up = reinterpret_cast<volatile int *>(tail + 4);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            // both SMs' decoding warps, and the arrival that expects both
            // halves of dy (in the first SM only)
            bar_init(full + 8 * i, 1 + 2 * kDecodeWarps);
            bar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < kCodeStages; ++i) {
            bar_init(code_full + 8 * i, 1);
            bar_init(code_empty + 8 * i, kDecodeWarps);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(acc_full + 8 * i, 1);
            bar_init(acc_empty + 8 * i, 2 * kEpilogueWarps);
        }
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
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
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(tail);

    if (warp == 0) {
        if (lane == 0) {
            int s = 0, cs = 0;
            uint32_t ph = 1, cph = 1;  // an empty buffer's first wait passes
            const uint32_t leader_full = in_cta(full, 0);
            bool ok = true;
            for (int u = pair; u < p.units && ok; u += pairs) {
                const Unit t = unit_of(p, u);
                for (int64_t r = t.r0; r < t.r1 && ok; r += kTileK) {
                    ok = bar_wait(code_empty + 8 * cs, cph, gave_up);
                    if (!ok) break;
                    bar_expect(code_full + 8 * cs, kCodeBytes);
                    tma_load(c_at + cs * kCodeBytes, &code_map, t.m0 + (int)rank * kHalf, (int)r,
                             code_full + 8 * cs);
                    if (++cs == kCodeStages) cs = 0, cph ^= 1;
                    ok = bar_wait(empty + 8 * s, ph, gave_up);
                    if (!ok) break;
                    if (rank == 0) bar_expect(full + 8 * s, 2 * kBBytes);
                    for (int h = 0; h < 2; ++h)
                        tma_load_pair(b_at + s * kBBytes + h * kTileK * 128, &dy_map,
                                      t.n0 + (int)rank * kHalf + 64 * h, (int)r,
                                      leader_full + 8 * s);
                    if (++s == kStages) s = 0, ph ^= 1;
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            constexpr uint32_t kType = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
            // f32 sums, both operands with M / N contiguous
            constexpr uint32_t kIdesc = 1u << 4 | kType << 7 | kType << 10 | 1u << 15 | 1u << 16 |
                                        (uint32_t)(kTileN >> 3) << 17 |
                                        (uint32_t)(kTileM >> 4) << 24;
            int s = 0, acc = 0;
            uint32_t ph = 0, aph = 1;
            bool ok = true;
            for (int u = pair; u < p.units && ok; u += pairs) {
                const Unit t = unit_of(p, u);
                for (int64_t c = t.r0; c < t.r1 && ok; c += p.chunk_rows) {
                    const int64_t c1 = min(t.r1, c + p.chunk_rows);
                    ok = bar_wait(acc_empty + 8 * acc, aph, gave_up);
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    for (int64_t r = c; r < c1 && ok; r += kTileK) {
                        ok = bar_wait(full + 8 * s, ph, gave_up);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint64_t a = operand_desc(a_at + s * kABytes);
                        const uint64_t b = operand_desc(b_at + s * kBBytes);
#pragma unroll
                        for (int k = 0; k < kTileK / 16; ++k)
                            mma_pair(tmem + acc * kAccCols, a + k * (2048 >> 4),
                                     b + k * (2048 >> 4), kIdesc, r > c || k > 0);
                        commit_pair(empty + 8 * s);
                        if (++s == kStages) s = 0, ph ^= 1;
                    }
                    if (!ok) break;
                    commit_pair(acc_full + 8 * acc);
                    acc ^= 1;
                    if (acc == 0) aph ^= 1;
                }
            }
        }
        __syncwarp();
    } else if (warp < 2 + kDecodeWarps) {
        // A thread decodes 16 columns of two rows of a stage.
        const int i = threadIdx.x - 64, piece = i % 8, row = i / 8;
        const int block = piece / 4, chunk = piece % 4 * 2;
        const uint32_t leader_full = in_cta(full, 0);
        int s = 0, cs = 0;
        uint32_t ph = 1, cph = 0;
        bool ok = true;
        for (int u = pair; u < p.units && ok; u += pairs) {
            const Unit t = unit_of(p, u);
            const int m0 = t.m0 + (int)rank * kHalf;
            const uint8_t *sc = p.scales + m0 / kGroup;
            uint32_t next[2];
            auto scales_at = [&](int64_t r) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t at = r + row + 32 * h;
                    // rows and columns past the end: 1 (their codes are zeros)
                    next[h] = 0x7f7f7f7fu;
                    if (m0 < p.cols && at < t.r1)
                        next[h] = __ldg(reinterpret_cast<const uint32_t *>(sc + at * p.spitch));
                }
            };
            scales_at(t.r0);
            for (int64_t r = t.r0; r < t.r1 && ok; r += kTileK) {
                const uint32_t word[2] = {next[0], next[1]};
                ok = bar_wait(code_full + 8 * cs, cph, gave_up);
                if (!ok) break;
                uint4 c[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t at = c_at + cs * kCodeBytes + (row + 32 * h) * kHalf + piece * 16;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(c[h].x), "=r"(c[h].y), "=r"(c[h].z), "=r"(c[h].w)
                                 : "r"(at)
                                 : "memory");
                }
                __syncwarp();
                if (lane == 0) bar_arrive(code_empty + 8 * cs);
                if (++cs == kCodeStages) cs = 0, cph ^= 1;
                if (r + kTileK < t.r1) scales_at(r + kTileK);
                ok = bar_wait(empty + 8 * s, ph, gave_up);
                if (!ok) break;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint4 v[2];
                    const int tr = row + 32 * h;
                    decode16<T, F>(c[h], (int)(word[h] >> (piece / 2 * 8) & 0xffu), v);
                    const uint32_t to = a_at + s * kABytes + block * (kTileK * 128) + tr * 128;
                    // the upper block's lanes store their second half first:
                    // eight lanes then cover all banks
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const int half = q ^ block;
                        const uint4 x = half ? v[1] : v[0];
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                                         to + (((chunk + half) ^ (tr & 7)) << 4)),
                                     "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w)
                                     : "memory");
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(leader_full + 8 * s);
                if (++s == kStages) s = 0, ph ^= 1;
            }
        }
    } else {
        // The accumulator's lanes are columns of x, its columns those of dy.
        const int quarter = warp % 4;
        const uint32_t leader_acc_empty = in_cta(acc_empty, 0);
        int acc = 0;
        uint32_t aph = 0;
        bool ok = true;
        for (int u = pair; u < p.units; u += pairs) {
            const Unit t = unit_of(p, u);
            const int col = t.m0 + (int)rank * kHalf + 32 * quarter + lane;
            float *out = p.out + t.split * p.part_stride + t.n0 * p.ld + col;
            const float *in = p.in ? p.in + t.n0 * p.ld + col : nullptr;
            for (int64_t c = t.r0; c < t.r1; c += p.chunk_rows) {
                if (ok) ok = bar_wait(acc_full + 8 * acc, aph, gave_up);
                ok = __all_sync(0xffffffffu, ok);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (int j0 = 0; j0 < kTileN; j0 += 32) {
                    uint32_t v[32];
                    if (ok) {
                        tmem_load32(tmem + acc * kAccCols + j0 + ((uint32_t)(32 * quarter) << 16),
                                    v);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = 0x7fffffffu;
                    }
                    if (j0 + 32 == kTileN) {
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) bar_arrive_cluster(leader_acc_empty + 8 * acc);
                    }
                    const int left = col < p.cols ? min(32, p.n - t.n0 - j0) : 0;
                    float add[32];
                    const float *from = c > t.r0 ? out : in;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        add[j] = from && j < left ? from[(j0 + j) * p.ld] : 0.f;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (j < left) out[(j0 + j) * p.ld] = __uint_as_float(v[j]) + add[j];
                }
                acc ^= 1;
                if (acc == 0) aph ^= 1;
            }
        }
    }
    // Where a wait gave up, copies and products may still be on their way:
    // they end by themselves within microseconds.
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

// dw = in or zeros: no rows.
__global__ void wgrad_fill_kernel(const float *in, float *out, int64_t n, int64_t cols,
                                  int64_t ld) {
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x)
        for (int64_t j = threadIdx.x; j < cols; j += blockDim.x)
            out[i * ld + j] = in ? in[i * ld + j] : 0.f;
}

// dy into rows that tensor copies can read (16-byte aligned).
__global__ void wgrad_copy_kernel(const uint16_t *x, int64_t ldx, uint16_t *y, int64_t ldy,
                                  int64_t rows, int64_t n) {
    for (int64_t i = blockIdx.x; i < rows; i += gridDim.x)
        for (int64_t j = threadIdx.x; j < n; j += blockDim.x) y[i * ldy + j] = x[i * ldx + j];
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
    const int pairs = std::max(1, std::min(p.units, sm_count() / 2));
    kern<<<2 * pairs, kWgradThreads, kWgradSmem, s>>>(codes, grads, p);
    POS_CUDA(cudaGetLastError());
    return POS_OK;
}

static pos_status wgrad(const uint8_t *ckpt, int32_t format, const void *dy, int32_t dtype,
                        int64_t ld_dy, int64_t rows, int64_t n, int64_t cols, const float *in,
                        float *out, int64_t ld, cudaStream_t s) {
    if (rows == 0) {
        wgrad_fill_kernel<<<(int)std::min<int64_t>(n, 65535), 256, 0, s>>>(in, out, n, cols, ld);
        POS_CUDA(cudaGetLastError());
        return POS_OK;
    }
    const CkptShape shape = ckpt_shape(cols);
    WgradParams p = {};
    p.scales = ckpt + rows * shape.pitch;
    p.in = in, p.out = out, p.ld = ld, p.rows = rows, p.spitch = shape.spitch;
    p.n = (int32_t)n, p.cols = (int32_t)cols;
    p.tiles_m = (int32_t)((cols + kTileM - 1) / kTileM);
    p.tiles_n = (int32_t)((n + kTileN - 1) / kTileN);
    if ((int64_t)p.tiles_m * p.tiles_n > 0x7fffffffll)
        return fail(POS_EINVAL, "wgrad: n * cols too large");
    p.splits = 1;
    p.units = p.tiles_m * p.tiles_n;
    p.chunk_rows = 1024;
    p.split_rows = (rows + p.chunk_rows - 1) / p.chunk_rows * p.chunk_rows;
    void *copy = nullptr;
    if (!aligned16(dy) || ld_dy % 8 || ld_dy < n) {
        cudaMemPool_t pool;
        POS_TRY(scratch_pool(&pool));
        const int64_t ld2 = (n + 7) / 8 * 8;
        POS_CUDA(cudaMallocFromPoolAsync(&copy, (size_t)(rows * ld2) * 2, pool, s));
        wgrad_copy_kernel<<<(int)std::min<int64_t>(rows, 65535), 256, 0, s>>>(
            static_cast<const uint16_t *>(dy), ld_dy, static_cast<uint16_t *>(copy), ld2, rows, n);
        dy = copy, ld_dy = ld2;
    }
    pos_status st;
    if (dtype == POS_BF16)
        st = format == POS_CKPT_INT8
                 ? launch_wgrad<__nv_bfloat16, POS_CKPT_INT8>(ckpt, dy, ld_dy, p, s)
                 : launch_wgrad<__nv_bfloat16, POS_CKPT_E4M3>(ckpt, dy, ld_dy, p, s);
    else
        st = format == POS_CKPT_INT8
                 ? launch_wgrad<__half, POS_CKPT_INT8>(ckpt, dy, ld_dy, p, s)
                 : launch_wgrad<__half, POS_CKPT_E4M3>(ckpt, dy, ld_dy, p, s);
    const cudaError_t e = copy ? cudaFreeAsync(copy, s) : cudaSuccess;
    if (st != POS_OK) return st;
    return e == cudaSuccess ? POS_OK : cuda_fail(e, "wgrad scratch");
}

}  // namespace pos

extern "C" pos_status poseidon_ckpt_wgrad(const void *d_ckpt, int32_t format, const void *d_dy,
                                          int32_t dtype, int64_t ld_dy, int64_t rows, int64_t n,
                                          int64_t cols, const float *d_dw_in, float *d_dw_out,
                                          int64_t ld_dw, void *stream) {
    using namespace pos;
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
}
