// poseidon_norm_forward: the residual's addition (with dropout) and the RMS norm of
// the sum in one pass, with 8-bit checkpoints of both (formulas: poseidon.h).
#include "norm.cuh"

namespace pos {

// r = 1 / sqrt(s / cols + eps) as rsqrtf's result and a step of Newton's method from it.
__device__ __forceinline__ Double32 rstd_of(const NormParams &p, Double32 s) {
    const float m = __fmul_rn(s.hi, p.inv_cols), v = m + p.eps, c = v - m;
    const float rest = ((m - (v - c)) + (p.eps - c)) + fmaf(s.hi, p.inv_cols, -m) +
                       fmaf(s.hi, p.inv_cols_lo, s.lo * p.inv_cols);  // v's own
    const float r = rsqrtf(v), t = __fmul_rn(v, r);
    const float e = fmaf(-fmaf(rest, r, fmaf(v, r, -t)), r, fmaf(-t, r, 1.f));  // 1 - v r^2
    return {r, fabsf(e) < 0.001f ? 0.5f * r * e : 0.f};  // (r of 0 and infinity as it is)
}

// A team takes a row at a time and holds it in registers, so that every matrix goes
// through HBM once; the next rows are on their way meanwhile (RING; without it rows are
// read in place, from any alignment).  h is rounded to its type before it is squared,
// kept or normalised: what the backward pass reads is what the forward pass used.
//   The sum over a row's threads, r and h r w carry their roundings along in a second f32,
// so that y is rounded once, as if it had been computed in more bits.  Without that one in
// 130,000 bf16 values (15,000 in f16) is on the other side of a rounding border, and with
// them 8-bit codes that have a border there too.  It costs 12 of 123 us for 16384 x 4096
// bf16 with both checkpoints, where instructions bound; 16384 x 8192 with an f32 stream takes
// 283 us with the integer sums, 297 without.
template <typename T, typename H, class TEAM, bool RING>
__global__ void __launch_bounds__(TEAM::M, TEAM::kBlocks) norm_forward_kernel(const NormParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    extern __shared__ uint4 cells[];
    __shared__ float shared[2][32];
    constexpr int V = TEAM::V, kX = sizeof(T) / 2, kH = sizeof(H) / 2;
    const int rank = TEAM::rank(), step = TEAM::threads();
    const uint64_t offset = drop_offset(p.drop);
    const int64_t rows_step = (int64_t)gridDim.x * TEAM::teams();
    const Ring ring(cells);
    const auto fetch = [&](int64_t r, int slot) {
        if (r < p.rows)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int cell = (slot * V + i) * (kX + kH);
                ring.copy(cell, static_cast<const T *>(p.x) + r * p.ldx, rank + i * step, p.cols);
                if (p.res)
                    ring.copy(cell + kX, static_cast<const H *>(p.res) + r * p.ldr, rank + i * step,
                              p.cols);
            }
        Ring::row_done();
    };
    Vec8 w[V];
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = load_w(p, rank + i * step);
    bool plain = false;  // weights that are not finite: an infinity is not to become a NaN
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) plain = plain || !isfinite(w[i].v[e]);
    int turn = 0, slot = 0;
    const int64_t first = (int64_t)blockIdx.x * TEAM::teams() + TEAM::index();
    if constexpr (RING)
        for (int k = 0; k < p.depth; ++k) fetch(first + k * rows_step, k);
    for (int64_t r = first; r < p.rows; r += rows_step, turn ^= 1) {
        Raw8<T> xr[V];
        Raw8<H> hr[V];
        if constexpr (RING) {
            Ring::wait(p.depth - 1);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int cell = (slot * V + i) * (kX + kH);
                xr[i] = ring.take<T>(cell);
                if (p.res) hr[i] = ring.take<H>(cell + kX);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xr[i] = load_vec(static_cast<const T *>(p.x) + r * p.ldx, rank + i * step, p.cols);
                if (p.res)
                    hr[i] = load_vec(static_cast<const H *>(p.res) + r * p.ldr, rank + i * step, p.cols);
            }
        }
        F2 squares = both(0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int j = rank + i * step;
            Vec8 v = to_float(xr[i]);
            if (p.res) {
                add_dropped8(p.drop, offset, (uint32_t)r, (uint32_t)j, v, to_float(hr[i]));
            } else if (p.drop.threshold) {
                drop8(p.drop, offset, (uint32_t)r, (uint32_t)j, v);
            }
            hr[i] = from_float<H>(v);
            H *h = static_cast<H *>(p.h) + r * p.ldh;
            if constexpr (RING && kH == 2) {
                if (p.h && p.out_aligned)
                    ring.store((slot * V + i) * (kX + kH) + kX, hr[i], h, j, p.cols);
                else if (p.h) store_vec(false, h, j, hr[i], p.cols);
            } else if (p.h) {
                store_vec(p.out_aligned, h, j, hr[i], p.cols);
            }
            if (p.codes_h)
                keep8(p.format, hr[i], p.codes_h + r * p.pitch, p.scales_h + r * p.spitch, j,
                      8 * j < p.pitch);
            v = to_float(hr[i]);
#pragma unroll
            for (int e = 0; e < 8; e += 2) squares = fma2(pair(v, e), pair(v, e), squares);
        }
        const int done = slot;
        if constexpr (RING) {
            if constexpr (kX == 1) {  // (else y goes through x's cells first)
                __syncwarp();
                fetch(r + p.depth * rows_step, slot);
            }
            if (++slot == p.depth) slot = 0;
        }
        const Double32 rstd =
            rstd_of(p, TEAM::sum_positive(squares.x + squares.y, shared, turn));
        if (p.rstd && rank == 0) p.rstd[r] = rstd.hi + rstd.lo;
        // h of 16 bits has at most 11, so with 13 of r their product is exact
        const float r_hi = kH == 2 ? rstd.hi : __uint_as_float(__float_as_uint(rstd.hi) & ~0x7ffu);
        const float r_lo = kH == 2 ? rstd.lo : (rstd.hi - r_hi) + rstd.lo;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!p.y && !p.codes_y) break;
            const int j = rank + i * step;
            Vec8 v = to_float(hr[i]);
            // (past the last column 0, or NaN with the whole group; r is infinite where eps
            // is 0 and the squares' sum as well)
            if (plain || !isfinite(rstd.hi)) {
#pragma unroll
                for (int e = 0; e < 8; e += 2)
                    set_pair(v, e, mul2(mul2(pair(v, e), both(rstd.hi + rstd.lo)), pair(w[i], e)));
            } else {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const F2 x = pair(v, e), n = mul2(x, both(r_hi));
                    F2 rest = mul2(x, both(r_lo));
                    if constexpr (kH == 2)
                        rest = fma2(x, both(r_lo), fma2(x, both(r_hi), {-n.x, -n.y}));
                    set_pair(v, e, fma2(n, pair(w[i], e), mul2(rest, pair(w[i], e))));
                }
            }
            const Raw8<T> y = from_float<T>(v);
            T *to = static_cast<T *>(p.y) + r * p.ldy;
            if constexpr (RING && kX == 2) {
                if (p.y && p.out_aligned) ring.store((done * V + i) * (kX + kH), y, to, j, p.cols);
                else if (p.y) store_vec(false, to, j, y, p.cols);
            } else if (p.y) {
                store_vec(p.out_aligned, to, j, y, p.cols);
            }
            if (p.codes_y)
                keep8(p.format, y, p.codes_y + r * p.pitch, p.scales_y + r * p.spitch, j,
                      8 * j < p.pitch);
        }
        if constexpr (RING && kX == 2) {
            __syncwarp();
            fetch(r + p.depth * rows_step, done);
        }
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
pos_status check_norm(const pos_norm *n, NormParams *p) {
    if (!n) return fail(POS_EINVAL, "norm: NULL pointer");
    if (n->rows < 0 || n->rows >= (1ll << 31)) return fail(POS_EINVAL, "norm: bad rows");
    if (n->cols < 1 || n->cols > kNormMaxCols)
        return fail(POS_EINVAL, "norm: cols must be 1..32768");
    if (!dtype_ok(n->dtype)) return fail(POS_EINVAL, "norm: unknown dtype");
    if (n->dtype_h != n->dtype && n->dtype_h != POS_F32)
        return fail(POS_EINVAL, "norm: dtype_h must be dtype or f32");
    if (!format_ok(n->format)) return fail(POS_EINVAL, "norm: unknown format");
    if (!(n->eps >= 0.f)) return fail(POS_EINVAL, "norm: eps must be >= 0");
    if (reinterpret_cast<uintptr_t>(n->w) % 4) return fail(POS_EINVAL, "norm: misaligned w");
    POS_TRY(make_drop(n->drop, "norm", &p->drop));
    const CkptShape s = ckpt_shape(n->cols);
    p->pitch = s.pitch, p->spitch = s.spitch;
    p->rows = n->rows, p->cols = n->cols, p->format = n->format;
    p->eps = n->eps, p->inv_cols = 1.f / n->cols;
    p->inv_cols_lo = (float)(1. / n->cols - p->inv_cols);
    p->w = n->w, p->w_vectors = aligned16(n->w);
    return POS_OK;
}

// One matrix of a call, if it is there; aligned: whether all so far allow 16-byte
// accesses.
pos_status check_matrix(const char *what, const void *d, int32_t dtype, int64_t rows, int64_t cols,
                        int64_t ld, bool written, bool *aligned) {
    if (!d) return POS_OK;
    const int size = dtype_size(dtype);
    if (ld < 0 || ld >= (1ll << 31) || (written && rows > 1 && ld < cols))
        return fail(POS_EINVAL, std::string("norm: bad row stride of ") + what);
    if (reinterpret_cast<uintptr_t>(d) % size)
        return fail(POS_EINVAL, std::string("norm: misaligned ") + what);
    if (!aligned16(d) || ld * size % 16) *aligned = false;
    return POS_OK;
}

template <typename T, typename H, class TEAM, bool RING>
static pos_status launch_forward(NormParams p, const NormShape &shape, cudaStream_t s) {
    auto kern = norm_forward_kernel<T, H, TEAM, RING>;
    int smem = 0;
    if constexpr (RING) {
        const int row = TEAM::V * (int)(sizeof(T) + sizeof(H)) / 2;
        p.depth = ring_depth(row, shape.threads);
        smem = 16 * p.depth * row * shape.threads;
        POS_TRY(ensure_smem(reinterpret_cast<const void *>(kern), smem));
    }
    int per_sm = 0;
    POS_TRY(blocks_per_sm(reinterpret_cast<const void *>(kern), shape.threads, smem, &per_sm));
    const int64_t blocks = (p.rows + shape.rows - 1) / shape.rows;
    POS_CUDA(launch_dependent(kern, (int)std::min<int64_t>(blocks, (int64_t)sm_count() * per_sm),
                              shape.threads, smem, s, p));
    return POS_OK;
}

template <typename T, typename H, class TEAM>
static pos_status launch_forward(const NormParams &p, const NormShape &shape, bool aligned,
                                 cudaStream_t s) {
    return aligned ? launch_forward<T, H, TEAM, true>(p, shape, s)
                   : launch_forward<T, H, TEAM, false>(p, shape, s);
}

template <typename T, typename H>
static pos_status forward_of(const NormParams &p, bool aligned, cudaStream_t s) {
    const NormShape shape = norm_shape(p.cols, aligned, sizeof(H) == 4, p.drop.threshold > 0, false);
    switch (shape.team) {
        case 0: return launch_forward<T, H, Team<true, 1, 256>>(p, shape, aligned, s);
        case 1: return launch_forward<T, H, Team<false, 1, 1024>>(p, shape, aligned, s);
        case 3: return launch_forward<T, H, Team<false, 4, 512>>(p, shape, aligned, s);
        case 5: return launch_forward<T, H, Team<false, 1, 640, 2>>(p, shape, aligned, s);
        // (a row of 1024 threads would fill an SM's shared memory)
        default: return launch_forward<T, H, Team<false, 4, 1024>, false>(p, shape, s);
    }
}

}  // namespace pos

extern "C" pos_status poseidon_norm_forward(const pos_norm *norm, const void *d_x, int64_t ldx,
                                            const void *d_res, int64_t ldr, void *d_h, int64_t ldh,
                                            void *d_y, int64_t ldy, void *d_ckpt_h,
                                            void *d_ckpt_y, float *d_rstd, void *stream) {
    using namespace pos;
    return guarded([&]() -> pos_status {
        NormParams p = {};
        bool aligned = true;
        POS_TRY(check_norm(norm, &p));
        const int64_t rows = norm->rows, cols = norm->cols;
        POS_TRY(check_matrix("x", d_x, norm->dtype, rows, cols, ldx, false, &aligned));
        POS_TRY(check_matrix("the residual", d_res, norm->dtype_h, rows, cols, ldr, false, &aligned));
        p.out_aligned = true;
        POS_TRY(check_matrix("h", d_h, norm->dtype_h, rows, cols, ldh, true, &p.out_aligned));
        POS_TRY(check_matrix("y", d_y, norm->dtype, rows, cols, ldy, true, &p.out_aligned));
        if (!aligned16(d_ckpt_h) || !aligned16(d_ckpt_y))
            return fail(POS_EINVAL, "norm: checkpoint not 16-byte aligned");
        if (reinterpret_cast<uintptr_t>(d_rstd) % 4)
            return fail(POS_EINVAL, "norm: misaligned rstd");
        if (rows == 0) return POS_OK;
        if (!d_x) return fail(POS_EINVAL, "norm: NULL x");
        p.x = d_x, p.ldx = ldx, p.res = d_res, p.ldr = ldr, p.h = d_h, p.ldh = ldh;
        p.y = d_y, p.ldy = ldy, p.rstd = d_rstd;
        p.codes_h = static_cast<uint8_t *>(d_ckpt_h);
        p.codes_y = static_cast<uint8_t *>(d_ckpt_y);
        p.scales_h = p.codes_h ? p.codes_h + rows * p.pitch : nullptr;
        p.scales_y = p.codes_y ? p.codes_y + rows * p.pitch : nullptr;
        const auto s = static_cast<cudaStream_t>(stream);
        const bool wide = norm->dtype_h == POS_F32;
        if (norm->dtype == POS_BF16)
            return wide ? forward_of<__nv_bfloat16, float>(p, aligned, s)
                        : forward_of<__nv_bfloat16, __nv_bfloat16>(p, aligned, s);
        if (norm->dtype == POS_F16)
            return wide ? forward_of<__half, float>(p, aligned, s)
                        : forward_of<__half, __half>(p, aligned, s);
        return forward_of<float, float>(p, aligned, s);
    });
}
