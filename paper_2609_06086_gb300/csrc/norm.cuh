// Shared by norm.cu and norm_backward.cu: RMS norm of the residual stream
// (formulas: poseidon.h).
#pragma once
#include <algorithm>

#include "dropout.cuh"

namespace pos {

constexpr int kNormMaxCols = 32768;

struct NormParams {
    const void *x, *res, *dy, *dh_in;
    const void *h_in;                  // backward: h, or NULL (the checkpoint is read)
    void *h, *y, *dh, *dx;
    const float *w;                    // NULL: ones
    float *rstd;
    uint8_t *codes_h, *scales_h;       // checkpoint of h; may be NULL
    uint8_t *codes_y, *scales_y;       // checkpoint of y; may be NULL
    float *part;                       // backward: [block][cols] partial sums, or NULL
    int64_t ldx, ldr, ldh, ldy, lddh_in, lddh, lddx;
    int64_t rows, pitch, spitch;
    int32_t cols, format;
    float eps, inv_cols, inv_cols_lo;  // 1 / cols as the sum of two
    bool w_vectors;                    // w can be read 16 bytes at a time
    bool out_aligned;                  // outputs can be written 16 bytes at a time
    int32_t depth;                     // rows on their way to shared memory
    DropParams drop;
};

// A number as the sum of two f32, of which the second is small.
struct Double32 {
    float hi, lo;
};
// Sums over a warp, in each of its lanes: as whole numbers of 2^-26 (2^-25 with signs)
// of the largest one's power of two, so that the warp's integer sums do in two steps
// what takes five exchanges of floats, and nothing is rounded after that.
__device__ __forceinline__ Double32 warp_sum_positive(float v) {
    const uint32_t big = __reduce_max_sync(0xffffffffu, __float_as_uint(v));
    if (big >= 0x7f800000u) return {__uint_as_float(big), 0.f};  // an infinity or a NaN
    const uint32_t e = max(big >> 23, 27u);
    const uint32_t total = __reduce_add_sync(
        0xffffffffu, __float2uint_rn(v * __uint_as_float((280u - e) << 23)));
    const float undo = __uint_as_float((e - 26u) << 23);
    return {(float)(total & ~255u) * undo, (float)(total & 255u) * undo};
}
__device__ __forceinline__ float warp_sum(float v) {
    const uint32_t big = __reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu);
    if (big >= 0x7f800000u) {
#pragma unroll
        for (int o = 16; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
    const uint32_t e = max(big >> 23, 27u);
    const int total = __reduce_add_sync(0xffffffffu,
                                        __float2int_rn(v * __uint_as_float((279u - e) << 23)));
    return (float)total * __uint_as_float((e - 25u) << 23);
}

// A row's threads: one warp with V vectors of 8 elements a thread (rows of 8 W of
// them share a block), or a whole block.  M: the most threads of a block, of which an SM
// holds BLOCKS at least.
template <bool WARP, int V_, int M_, int BLOCKS = 1>
struct Team {
    static constexpr bool kWarp = WARP;
    static constexpr int V = V_, M = M_, kBlocks = BLOCKS;
    static __device__ __forceinline__ int threads() { return WARP ? 32 : blockDim.x; }
    static __device__ __forceinline__ int rank() { return WARP ? threadIdx.x % 32 : threadIdx.x; }
    static __device__ __forceinline__ int teams() { return WARP ? blockDim.x / 32 : 1; }
    static __device__ __forceinline__ int index() { return WARP ? threadIdx.x / 32 : 0; }
    // The sum over the row's threads, in each of them; `turn` alternates between
    // calls, so that one barrier a call is enough.
    static __device__ __forceinline__ float sum(float v, float (*shared)[32], int turn) {
        v = warp_sum(v);
        if constexpr (WARP) return v;
        return warp_sum(of_warps(v, shared, turn));
    }
    // The same of numbers that are not negative, as exact as the threads' own sums.
    static __device__ __forceinline__ Double32 sum_positive(float v, float (*shared)[32], int turn) {
        const Double32 mine = warp_sum_positive(v);
        if constexpr (WARP) return mine;
        return warp_sum_positive(of_warps(mine.hi + mine.lo, shared, turn));
    }
    static __device__ __forceinline__ float of_warps(float v, float (*shared)[32], int turn) {
        const int lane = threadIdx.x % 32, warps = blockDim.x / 32;
        if (lane == 0) shared[turn][threadIdx.x / 32] = v;
        __syncthreads();
        return lane < warps ? shared[turn][lane] : 0.f;
    }
};

template <typename T>
__device__ __forceinline__ Raw8<T> load_vec(const T *row, int j, int cols) {
    return load8_shifted(row + 8 * j, 8 * j, cols - 8 * j);
}

// Rows on their way to shared memory, ahead of the one that is worked on.  Without them
// a row's loads, its sum over the block and its stores take turns, and registers leave
// room for few blocks an SM.  A slot of the ring is a row, a vector takes 16-byte cells of
// it: one for 16-bit elements and for codes, two for f32.  A warp copies and reads its own
// vectors, so the block need not meet.  A lane's 8 values in f32 are 32 bytes, but a copy
// or store of 16 bytes of each lane's would use half of every sector at a time: the two
// cells of a warp are the 1024 bytes as they lie in memory, which its lanes copy, and
// write from, 512 bytes at a time.
struct Ring {
    uint32_t smem;
    int step;        // bytes from cell to cell
    int lane, warp;
    __device__ __forceinline__ explicit Ring(void *at)
        : smem((uint32_t)__cvta_generic_to_shared(at)), step(16 * blockDim.x),
          lane(threadIdx.x % 32), warp(threadIdx.x / 32) {}
    __device__ __forceinline__ uint32_t own(int cell) const {
        return smem + cell * step + 16 * threadIdx.x;
    }
    // 16 bytes of two cells in memory's order; exchanged so that reading every second
    // one meets no bank twice
    __device__ __forceinline__ uint32_t word(int cell, int w) const {
        return smem + cell * step + 1024 * warp + 16 * (w ^ (w >> 3 & 1));
    }
    // The warp's vectors of a row, 8 `rank` its lane's first column.
    template <typename T>
    __device__ __forceinline__ void copy(int cell, const T *row, int rank, int cols) const {
        constexpr int kPer = 16 / sizeof(T);
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
            const int w = lane + 32 * k;
            const int c = sizeof(T) == 4 ? 8 * (rank - lane) + kPer * w : 8 * rank;
            const int n = max(0, min(kPer, cols - c));
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                             sizeof(T) == 4 ? word(cell, w) : own(cell)),
                         "l"(row + (n ? c : 0)), "r"((int)(n * sizeof(T)))
                         : "memory");
        }
    }
    template <typename T>
    __device__ __forceinline__ Raw8<T> take(int cell) const {
        Raw8<T> r;
        if constexpr (sizeof(T) == 4) r.a = read(word(cell, 2 * lane)), r.b = read(word(cell, 2 * lane + 1));
        else r.a = read(own(cell));
        return r;
    }
    // 8 codes and the word of scales that has theirs
    __device__ __forceinline__ void copy_codes(int cell, const uint8_t *codes, const uint8_t *scales,
                                               bool there) const {
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(own(cell)), "l"(codes),
                     "r"(there ? 8 : 0)
                     : "memory");
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(own(cell) + 8), "l"(scales),
                     "r"(there ? 4 : 0)
                     : "memory");
    }
    // f32: the warp's vectors through two cells to an aligned row
    __device__ __forceinline__ void store(int cell, const Raw8<float> &r, float *row, int rank,
                                          int cols) const {
        write(word(cell, 2 * lane), r.a);
        write(word(cell, 2 * lane + 1), r.b);
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int w = lane + 32 * k, c = 8 * (rank - lane) + 4 * w;
            const uint4 v = read(word(cell, w));
            if (c + 4 <= cols) {
                *reinterpret_cast<uint4 *>(row + c) = v;
            } else {
                const uint32_t e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (c + i < cols) row[c + i] = __uint_as_float(e[i]);
            }
        }
    }
    static __device__ __forceinline__ uint4 read(uint32_t at) {
        uint4 v;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "r"(at)
                     : "memory");
        return v;
    }
    static __device__ __forceinline__ void write(uint32_t at, const uint4 &v) {
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y),
                     "r"(v.z), "r"(v.w)
                     : "memory");
    }
    static __device__ __forceinline__ void row_done() {
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // All rows but the last `ahead` have arrived, for the whole warp.
    static __device__ __forceinline__ void wait(int ahead) {
        if (ahead >= 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else if (ahead == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
    }
};
constexpr int kNormDepth = 3;
// Depth of the ring whose rows take `cells` cells of `threads` threads: as deep as two
// blocks an SM allow, or one where the rows are long.
inline int ring_depth(int cells, int threads) {
    const int slot = 16 * cells * threads;
    for (int most : {110 << 10, 220 << 10})
        if (kNormDepth * slot <= most) return kNormDepth;
    return 2 * slot <= (220 << 10) ? 2 : 1;
}

// All lanes of a warp take part.
template <typename T>
__device__ __forceinline__ void store_vec(bool aligned, T *row, int j, const Raw8<T> &r, int cols) {
    const int left = cols - 8 * j, lane = threadIdx.x % 32;
    if (aligned) {
        if (left > 0) store8<true>(row + 8 * j, r, left);
    } else {
        store8_shifted(row + 8 * j, r, left, lane > 0, lane < 31);
    }
}

__device__ __forceinline__ F2 pair(const Vec8 &x, int i) { return {x.v[i], x.v[i + 1]}; }
__device__ __forceinline__ void set_pair(Vec8 &x, int i, F2 v) { x.v[i] = v.x, x.v[i + 1] = v.y; }

__device__ __forceinline__ Vec8 load_w(const NormParams &p, int j) {
    Vec8 w;
    const int left = p.cols - 8 * j;
    if (p.w && p.w_vectors && left >= 8) {
        const float4 a = *reinterpret_cast<const float4 *>(p.w + 8 * j);
        const float4 b = *reinterpret_cast<const float4 *>(p.w + 8 * j + 4);
        w.v[0] = a.x, w.v[1] = a.y, w.v[2] = a.z, w.v[3] = a.w;
        w.v[4] = b.x, w.v[5] = b.y, w.v[6] = b.z, w.v[7] = b.w;
        return w;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) w.v[i] = p.w && i < left ? p.w[8 * j + i] : 1.f;
    return w;
}

// Keeps 8 elements in 8 bits; four lanes share a group's scale.  All lanes of a
// warp take part; `live`: the vector lies within the row's codes.
template <typename T>
__device__ __forceinline__ void keep8(int format, const Raw8<T> &raw, uint8_t *codes,
                                      uint8_t *scales, int j, bool live) {
    uint32_t m = amax_bits(raw);
    m = max_bits<T>(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max_bits<T>(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const uint32_t bits = f32_bits<T>(m);
    const bool i8 = format == POS_CKPT_INT8;
    const int byte = i8 ? scale_byte<POS_CKPT_INT8>(bits) : scale_byte<POS_CKPT_E4M3>(bits);
    if (!live) return;
    const Vec8 x = to_float(raw);
    uint2 c;
    if (byte >= Fmt<POS_CKPT_E4M3>::kScaleHi)  // (the lower of the two formats' largest)
        c = i8 ? encode8<POS_CKPT_INT8>(x, byte) : encode8<POS_CKPT_E4M3>(x, byte);
    else if (i8)
        c = make_uint2(encode4_inside<POS_CKPT_INT8>(x.v[0], x.v[1], x.v[2], x.v[3], byte),
                       encode4_inside<POS_CKPT_INT8>(x.v[4], x.v[5], x.v[6], x.v[7], byte));
    else
        c = make_uint2(encode4_inside<POS_CKPT_E4M3>(x.v[0], x.v[1], x.v[2], x.v[3], byte),
                       encode4_inside<POS_CKPT_E4M3>(x.v[4], x.v[5], x.v[6], x.v[7], byte));
    *reinterpret_cast<uint2 *>(codes + 8 * j) = c;
    if (j % 4 == 0) scales[j / 4] = (uint8_t)byte;
}

// Threads of a block for a call, and which Team.  Up to 8192 columns a vector a thread:
// 64 registers, so that 32 warps an SM hide one another's sums and codes; the backward pass
// from 2056 on two, which need half as many warps to meet (16384 x 8192, stream in f32, from
// 8 bits: 280 us, with one 340; forward of the same with both checkpoints: one 283 us, with
// two 291).
struct NormShape {
    int team;     // 0..5: Team<true, 1, 256>, <false, 1, 1024>, <false, 2, 512>, <false, 4, 512>,
                  // <false, 4, 1024>, and <false, 1, 640, 2> or <false, 2, 320, 2>
    int threads, rows;  // of a block
};
inline NormShape norm_shape(int cols, bool aligned, bool wide, bool drop, bool backward) {
    // (vectors of the padded codes: 32 columns each four)
    const int nv = (cols + kGroup - 1) / kGroup * 4;
    if (nv <= 32) return {0, 256, 8};
    const int v = nv > 1024 ? 4 : backward && nv > 256 ? 2 : 1;
    const int threads = ((nv + v - 1) / v + 31) / 32 * 32;
    // Rows of 4097 to 5120 columns: two blocks an SM with a few registers less.  8192 rows of
    // 5001, off the alignment: 114 and 178 us with one forward, 195 and 342 back.  8192 of 5120,
    // whose next rows are on their way in shared memory, bf16: 54 and 59 forward, with dropout
    // 67 and 72, back with dropout 86 and 91, but without 81 and 77; and with an f32 stream, which
    // fills shared memory, 88 and 75, back 139 and 106.
    if (nv > 512 && nv <= 640 && (!aligned || (!wide && (!backward || drop))))
        return {5, threads, 1};
    return {v < 4 ? v : threads <= 512 ? 3 : 4, threads, 1};
}

pos_status check_norm(const pos_norm *n, NormParams *p);
pos_status check_matrix(const char *what, const void *d, int32_t dtype, int64_t rows, int64_t cols,
                        int64_t ld, bool written, bool *aligned);

}  // namespace pos
