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
    float eps, inv_cols;
    bool w_vectors;                    // w can be read 16 bytes at a time
    bool out_aligned;                  // outputs can be written 16 bytes at a time
    int32_t depth;                     // rows on their way to shared memory
    DropParams drop;
};

// A row's threads: one warp with V vectors of 8 elements a thread (rows of 8 W of
// them share a block), or a whole block.  M: the most threads of a block.
template <bool WARP, int V_, int M_>
struct Team {
    static constexpr bool kWarp = WARP;
    static constexpr int V = V_, M = M_;
    static __device__ __forceinline__ int threads() { return WARP ? 32 : blockDim.x; }
    static __device__ __forceinline__ int rank() { return WARP ? threadIdx.x % 32 : threadIdx.x; }
    static __device__ __forceinline__ int teams() { return WARP ? blockDim.x / 32 : 1; }
    static __device__ __forceinline__ int index() { return WARP ? threadIdx.x / 32 : 0; }
    // The sum over the row's threads, in each of them; `turn` alternates between
    // calls, so that one barrier a call is enough.
    static __device__ __forceinline__ float sum(float v, float (*shared)[32], int turn) {
#pragma unroll
        for (int o = 16; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
        if constexpr (WARP) return v;
        const int lane = threadIdx.x % 32, warps = blockDim.x / 32;
        if (lane == 0) shared[turn][threadIdx.x / 32] = v;
        __syncthreads();
        v = lane < warps ? shared[turn][lane] : 0.f;
#pragma unroll
        for (int o = 16; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
};

template <typename T>
__device__ __forceinline__ Raw8<T> load_vec(const T *row, int j, int cols) {
    return load8_shifted(row + 8 * j, 8 * j, cols - 8 * j);
}

// Rows on their way to shared memory, `depth` - 1 of them ahead: a thread copies and
// reads its own vectors, so the block need not meet.  Without them a row's loads, its
// sum over the block and its stores take turns, and registers leave room for one block of
// 512 threads an SM.  A cell is 16 bytes; a vector takes some cells, a slot of the ring
// one row.
struct Ring {
    uint32_t base;   // this thread's first cell
    int step;        // bytes from cell to cell
    __device__ __forceinline__ explicit Ring(void *smem)
        : base((uint32_t)__cvta_generic_to_shared(smem) + 16 * threadIdx.x), step(16 * blockDim.x) {}
    // 8 elements, of which `left` exist (the others read as zeros)
    template <typename T>
    __device__ __forceinline__ void copy(int cell, const T *from, int left) const {
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
            constexpr int kPer = 16 / sizeof(T);
            const int n = max(0, min(kPer, left - kPer * k));
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                             base + (cell + k) * step),
                         "l"(n ? from + kPer * k : from), "r"((int)(n * sizeof(T)))
                         : "memory");
        }
    }
    template <typename T>
    __device__ __forceinline__ Raw8<T> take(int cell) const {
        Raw8<T> r;
        r.a = word(cell);
        if constexpr (sizeof(T) == 4) r.b = word(cell + 1);
        return r;
    }
    // 8 codes and the word of scales that has theirs
    __device__ __forceinline__ void copy_codes(int cell, const uint8_t *codes, const uint8_t *scales,
                                               bool there) const {
        const uint32_t at = base + cell * step;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(at), "l"(codes),
                     "r"(there ? 8 : 0)
                     : "memory");
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(at + 8), "l"(scales),
                     "r"(there ? 4 : 0)
                     : "memory");
    }
    __device__ __forceinline__ uint4 word(int cell) const {
        uint4 v;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "r"(base + cell * step));
        return v;
    }
    static __device__ __forceinline__ void row_done() {
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // All rows but the last `ahead` have arrived.
    static __device__ __forceinline__ void wait(int ahead) {
        if (ahead >= 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else if (ahead == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
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
    *reinterpret_cast<uint2 *>(codes + 8 * j) =
        i8 ? encode8<POS_CKPT_INT8>(x, byte) : encode8<POS_CKPT_E4M3>(x, byte);
    if (j % 4 == 0) scales[j / 4] = (uint8_t)byte;
}

// Threads of a block for a call, and which Team: rows of up to 1024 columns by a warp
// each, up to 32 elements a thread else.
struct NormShape {
    int team;     // 0..4: Team<true, 1, 256>, <true, 4, 256>, <false, 2, 512>, <false, 4, 512>,
                  // <false, 4, 1024>
    int threads, rows;  // of a block
};
inline NormShape norm_shape(int cols) {
    // (vectors of the padded codes: 32 columns each four)
    const int nv = (cols + kGroup - 1) / kGroup * 4;
    if (nv <= 32) return {0, 256, 8};
    if (nv <= 128) return {1, 256, 8};
    const int v = nv <= 1024 ? 2 : 4, threads = ((nv + v - 1) / v + 31) / 32 * 32;
    return {v == 2 ? 2 : threads <= 512 ? 3 : 4, threads, 1};
}

pos_status check_norm(const pos_norm *n, NormParams *p);
pos_status check_matrix(const char *what, const void *d, int32_t dtype, int64_t rows, int64_t cols,
                        int64_t ld, bool written, bool *aligned);

}  // namespace pos
