// poseidon_norm_backward (formulas: poseidon.h).
#include "norm.cuh"

namespace pos {

// 8 values of h from its codes and a scale byte.
__device__ __forceinline__ Vec8 kept8(const NormParams &p, uint2 codes, int byte) {
    const float scale = scale_value(byte);
    return p.format == POS_CKPT_INT8 ? decode8<POS_CKPT_INT8>(codes, scale)
                                     : decode8<POS_CKPT_E4M3>(codes, scale);
}

// A team takes a row at a time, as the forward pass does.  dw is summed over a
// thread's rows in registers, over a block's teams in shared memory, and written as
// one partial sum per block, which norm_dw_kernel adds up in order: no atomics.
template <typename T, typename H, class TEAM, bool RING>
__global__ void __launch_bounds__(TEAM::M, TEAM::kBlocks) norm_backward_kernel(const NormParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    extern __shared__ uint4 cells[];
    __shared__ float shared[2][32];
    constexpr int V = TEAM::V, kX = sizeof(T) / 2, kH = sizeof(H) / 2;
    const int rank = TEAM::rank(), step = TEAM::threads();
    const uint64_t offset = drop_offset(p.drop);
    const int64_t rows_step = (int64_t)gridDim.x * TEAM::teams();
    const Ring ring(cells);
    // cells of a vector: dy, h (or its codes), dh_in or dh
    const int in_h = kX + (p.h_in ? kH : 1), per = in_h + kH;
    const auto fetch = [&](int64_t r, int slot) {
        if (r < p.rows)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int j = rank + i * step, cell = (slot * V + i) * per;
                ring.copy(cell, static_cast<const T *>(p.dy) + r * p.ldy, j, p.cols);
                if (p.h_in) {
                    ring.copy(cell + kX, static_cast<const H *>(p.h_in) + r * p.ldh, j, p.cols);
                } else {
                    const int c = 8 * j < p.cols ? 8 * j : 0;
                    ring.copy_codes(cell + kX, p.codes_h + r * p.pitch + c,
                                    p.scales_h + r * p.spitch + c / 128 * 4, 8 * j < p.cols);
                }
                if (p.dh_in)
                    ring.copy(cell + in_h, static_cast<const H *>(p.dh_in) + r * p.lddh_in, j, p.cols);
            }
        Ring::row_done();
    };
    constexpr bool kHoldW = V <= 2;  // (registers)
    Vec8 dw[V], w_held[kHoldW ? V : 1];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        dw[i] = Vec8{};
        if constexpr (kHoldW) w_held[i] = load_w(p, rank + i * step);
    }
    int turn = 0, slot = 0;
    const int64_t first = (int64_t)blockIdx.x * TEAM::teams() + TEAM::index();
    if constexpr (RING)
        for (int k = 0; k < p.depth; ++k) fetch(first + k * rows_step, k);
    float next = first < p.rows ? p.rstd[first] : 0.f;
    for (int64_t r = first; r < p.rows; r += rows_step, turn ^= 1) {
        Raw8<T> g[V];
        Raw8<H> add[V];
        Vec8 n[V];
        const float rstd = next;
        if (r + rows_step < p.rows) next = p.rstd[r + rows_step];
        if constexpr (RING) {
            Ring::wait(p.depth - 1);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int cell = (slot * V + i) * per;
                g[i] = ring.take<T>(cell);
                if (p.h_in) {
                    n[i] = to_float(ring.take<H>(cell + kX));
                } else {
                    const uint4 c = Ring::read(ring.own(cell + kX));
                    n[i] = kept8(p, make_uint2(c.x, c.y),
                                 (int)(c.z >> ((rank + i * step) / 4 % 4 * 8) & 255));
                }
                if (p.dh_in) add[i] = ring.take<H>(cell + in_h);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int j = rank + i * step;
                g[i] = load_vec(static_cast<const T *>(p.dy) + r * p.ldy, j, p.cols);
                if (p.h_in)
                    n[i] = to_float(load_vec(static_cast<const H *>(p.h_in) + r * p.ldh, j, p.cols));
                else if (8 * j < p.pitch)
                    n[i] = kept8(p, *reinterpret_cast<const uint2 *>(p.codes_h + r * p.pitch + 8 * j),
                                 p.scales_h[r * p.spitch + j / 4]);
                else
                    n[i] = Vec8{};
                if (p.dh_in)
                    add[i] = load_vec(static_cast<const H *>(p.dh_in) + r * p.lddh_in, j, p.cols);
            }
        }
        F2 dot = both(0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Vec8 v = to_float(g[i]);
            Vec8 w;
            if constexpr (kHoldW) w = w_held[i];
            else w = load_w(p, rank + i * step);
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const F2 x = mul2(pair(n[i], e), both(rstd));
                set_pair(n[i], e, x);
                set_pair(dw[i], e, fma2(pair(v, e), x, pair(dw[i], e)));
                dot = fma2(mul2(pair(v, e), pair(w, e)), x, dot);
            }
        }
        const float mean = TEAM::sum(dot.x + dot.y, shared, turn) * p.inv_cols;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!p.dh && !p.dx) break;
            const int j = rank + i * step;
            const Vec8 v = to_float(g[i]);
            Vec8 w, d;
            if constexpr (kHoldW) w = w_held[i];
            else w = load_w(p, j);
            if (p.dh_in) d = to_float(add[i]);
            else d = Vec8{};
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const F2 a = fma2(pair(n[i], e), both(-mean), mul2(pair(v, e), pair(w, e)));
                set_pair(d, e, fma2(a, both(rstd), pair(d, e)));
            }
            H *dh = static_cast<H *>(p.dh) + r * p.lddh;
            if constexpr (RING && kH == 2) {
                if (p.dh && p.out_aligned)
                    ring.store((slot * V + i) * per + in_h, from_float<H>(d), dh, j, p.cols);
                else if (p.dh) store_vec(false, dh, j, from_float<H>(d), p.cols);
            } else if (p.dh) {
                store_vec(p.out_aligned, dh, j, from_float<H>(d), p.cols);
            }
            if (!p.dx) continue;
            if (p.drop.threshold) drop8(p.drop, offset, (uint32_t)r, (uint32_t)j, d);
            T *dx = static_cast<T *>(p.dx) + r * p.lddx;
            if constexpr (RING && kX == 2) {
                if (p.out_aligned) ring.store((slot * V + i) * per, from_float<T>(d), dx, j, p.cols);
                else store_vec(false, dx, j, from_float<T>(d), p.cols);
            } else {
                store_vec(p.out_aligned, dx, j, from_float<T>(d), p.cols);
            }
        }
        if constexpr (RING) {
            __syncwarp();
            fetch(r + p.depth * rows_step, slot);
            if (++slot == p.depth) slot = 0;
        }
    }
    if (!p.part) return;
    float *part = p.part + (int64_t)blockIdx.x * p.cols;
    if constexpr (TEAM::kWarp) {
        // the block's warps, one after another
        __shared__ float sums[256 * V];
        for (int t = 0; t < TEAM::teams(); ++t) {
            if (TEAM::index() == t)
#pragma unroll
                for (int i = 0; i < V; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float &s = sums[e * 32 * V + rank + i * 32];
                        s = t ? s + dw[i].v[e] : dw[i].v[e];
                    }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < p.cols; c += blockDim.x) part[c] = sums[c % 8 * 32 * V + c / 8];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (rank + i * step);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < p.cols) part[c + e] = dw[i].v[e];
        }
    }
}

// dw = dw_in + the blocks' partial sums: a block takes 32 columns, 32 warps a strided
// share of the partial sums each.
constexpr int kNormDwWarps = 32;
__global__ void __launch_bounds__(32 * kNormDwWarps)
    norm_dw_kernel(const float *part, int n_part, int cols, const float *dw_in, float *dw) {
    grid_dep_wait();
    grid_dep_trigger();
    __shared__ float sum[kNormDwWarps][32];
    const int lane = threadIdx.x % 32, c = blockIdx.x * 32 + lane;
    float v = 0.f;
    if (c < cols)
#pragma unroll 8
        for (int b = threadIdx.x / 32; b < n_part; b += kNormDwWarps) v += part[b * (int64_t)cols + c];
    sum[threadIdx.x / 32][lane] = v;
    __syncthreads();
    if (threadIdx.x >= 32 || c >= cols) return;
    v = 0.f;
#pragma unroll
    for (int q = 0; q < kNormDwWarps; ++q) v += sum[q][lane];
    dw[c] = dw_in ? dw_in[c] + v : v;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
template <typename T, typename H, class TEAM, bool RING>
static pos_status launch_backward(NormParams &p, const NormShape &shape, const float *dw_in,
                                  float *dw, cudaStream_t s) {
    auto kern = norm_backward_kernel<T, H, TEAM, RING>;
    int smem = 0;
    if constexpr (RING) {
        constexpr int kX = sizeof(T) / 2, kH = sizeof(H) / 2;
        const int row = TEAM::V * (kX + (p.h_in ? kH : 1) + kH);
        p.depth = ring_depth(row, shape.threads);
        smem = 16 * p.depth * row * shape.threads;
        POS_TRY(ensure_smem(reinterpret_cast<const void *>(kern), smem));
    }
    int per_sm = 0;
    POS_TRY(blocks_per_sm(reinterpret_cast<const void *>(kern), shape.threads, smem, &per_sm));
    const int64_t blocks = (p.rows + shape.rows - 1) / shape.rows;
    const int grid = (int)std::min<int64_t>(blocks, (int64_t)sm_count() * std::min(per_sm, 16));
    void *scratch = nullptr;
    if (dw && grid > 0) {
        cudaMemPool_t pool;
        POS_TRY(scratch_pool(&pool, (int64_t)grid * p.cols * 4));
        POS_CUDA(cudaMallocFromPoolAsync(&scratch, (size_t)grid * p.cols * 4, pool, s));
        p.part = static_cast<float *>(scratch);
    }
    cudaError_t e =
        grid > 0 ? launch_dependent(kern, grid, shape.threads, smem, s, p) : cudaSuccess;
    if (dw && e == cudaSuccess)
        e = launch_dependent(norm_dw_kernel, (p.cols + 31) / 32, 32 * kNormDwWarps, 0, s,
                             (const float *)p.part, grid, (int)p.cols, dw_in, dw);
    const cudaError_t e2 = scratch ? cudaFreeAsync(scratch, s) : cudaSuccess;
    if (e == cudaSuccess) e = e2;
    return e == cudaSuccess ? POS_OK : cuda_fail(e, "norm backward");
}

template <typename T, typename H, class TEAM>
static pos_status launch_backward(NormParams &p, const NormShape &shape, bool aligned,
                                  const float *dw_in, float *dw, cudaStream_t s) {
    return aligned ? launch_backward<T, H, TEAM, true>(p, shape, dw_in, dw, s)
                   : launch_backward<T, H, TEAM, false>(p, shape, dw_in, dw, s);
}

template <typename T, typename H>
static pos_status backward_of(NormParams &p, bool aligned, const float *dw_in, float *dw,
                              cudaStream_t s) {
    const NormShape shape = norm_shape(p.cols, aligned, sizeof(H) == 4, p.drop.threshold > 0, true);
    switch (shape.team) {
        case 0: return launch_backward<T, H, Team<true, 1, 256>>(p, shape, aligned, dw_in, dw, s);
        case 1: return launch_backward<T, H, Team<false, 1, 1024>>(p, shape, aligned, dw_in, dw, s);
        case 2: return launch_backward<T, H, Team<false, 2, 512>>(p, shape, aligned, dw_in, dw, s);
        case 3: return launch_backward<T, H, Team<false, 4, 512>>(p, shape, aligned, dw_in, dw, s);
        case 5: return launch_backward<T, H, Team<false, 2, 320, 2>>(p, shape, aligned, dw_in, dw, s);
        default: return launch_backward<T, H, Team<false, 4, 1024>, false>(p, shape, dw_in, dw, s);
    }
}

}  // namespace pos

extern "C" pos_status poseidon_norm_backward(const pos_norm *norm, const void *d_h, int64_t ldh,
                                             const void *d_ckpt_h, const float *d_rstd,
                                             const void *d_dy, int64_t lddy, const void *d_dh_in,
                                             int64_t lddh_in, void *d_dh, int64_t lddh, void *d_dx,
                                             int64_t lddx, const float *d_dw_in, float *d_dw,
                                             void *stream) {
    using namespace pos;
    return guarded([&]() -> pos_status {
        NormParams p = {};
        bool aligned = true;
        POS_TRY(check_norm(norm, &p));
        const int64_t rows = norm->rows, cols = norm->cols;
        const int32_t over = norm->dtype_h;
        POS_TRY(check_matrix("h", d_h, over, rows, cols, ldh, false, &aligned));
        POS_TRY(check_matrix("dy", d_dy, norm->dtype, rows, cols, lddy, false, &aligned));
        POS_TRY(check_matrix("dh_in", d_dh_in, over, rows, cols, lddh_in, false, &aligned));
        p.out_aligned = true;
        POS_TRY(check_matrix("dh", d_dh, over, rows, cols, lddh, true, &p.out_aligned));
        POS_TRY(check_matrix("dx", d_dx, norm->dtype, rows, cols, lddx, true, &p.out_aligned));
        if (!aligned16(d_ckpt_h)) return fail(POS_EINVAL, "norm: checkpoint not 16-byte aligned");
        if (reinterpret_cast<uintptr_t>(d_rstd) % 4)
            return fail(POS_EINVAL, "norm: misaligned rstd");
        if (reinterpret_cast<uintptr_t>(d_dw_in) % 4 || reinterpret_cast<uintptr_t>(d_dw) % 4)
            return fail(POS_EINVAL, "norm: misaligned dw");
        if (d_dw_in && !d_dw) return fail(POS_EINVAL, "norm: dw_in without dw");
        if (rows > 0) {
            if (!d_h && !d_ckpt_h) return fail(POS_EINVAL, "norm: neither h nor its checkpoint");
            if (!d_rstd || !d_dy) return fail(POS_EINVAL, "norm: NULL rstd or dy");
        }
        p.h_in = d_h, p.ldh = ldh, p.dy = d_dy, p.ldy = lddy, p.dh_in = d_dh_in;
        p.lddh_in = lddh_in, p.dh = d_dh, p.lddh = lddh, p.dx = d_dx, p.lddx = lddx;
        p.rstd = const_cast<float *>(d_rstd);
        if (!d_h && d_ckpt_h) {
            p.codes_h = static_cast<uint8_t *>(const_cast<void *>(d_ckpt_h));
            p.scales_h = p.codes_h + rows * p.pitch;
        }
        const auto s = static_cast<cudaStream_t>(stream);
        const bool wide = over == POS_F32;
        if (norm->dtype == POS_BF16)
            return wide ? backward_of<__nv_bfloat16, float>(p, aligned, d_dw_in, d_dw, s)
                        : backward_of<__nv_bfloat16, __nv_bfloat16>(p, aligned, d_dw_in, d_dw, s);
        if (norm->dtype == POS_F16)
            return wide ? backward_of<__half, float>(p, aligned, d_dw_in, d_dw, s)
                        : backward_of<__half, __half>(p, aligned, d_dw_in, d_dw, s);
        return backward_of<float, float>(p, aligned, d_dw_in, d_dw, s);
    });
}
