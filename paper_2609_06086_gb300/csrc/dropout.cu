// poseidon_dropout: y = residual + dropout(x), the mask from a counter-based
// generator (formulas: poseidon.h).
#include <algorithm>

#include "dropout.cuh"

namespace pos {

constexpr int kDropThreads = 256;
constexpr int kDropUnroll = 1;  // vectors of 8 elements per thread (16384 x 8192 bf16, both passes:
                                // one 226 us, two 234, four 237)
constexpr int kDropBlock = kDropThreads * kDropUnroll;

struct DropoutParams {
    const void *x, *res;
    void *y;
    int64_t ldx, ldr, ldy;
    uint32_t n_vec;    // rows * ceil(cols / 8)
    int32_t cols;
    uint32_t row0;     // the first row's number
    FastDiv per_row{1};  // ceil(cols / 8)
    DropParams drop;
};

// A thread takes vectors of 8 elements, a warp 256 consecutive ones; the mask is
// computed while they are on their way.  Bound by HBM.
template <typename X, typename Y, bool ALIGNED>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const DropoutParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    const uint64_t offset = drop_offset(p.drop);
    Raw8<X> x[kDropUnroll];
    Raw8<Y> r[kDropUnroll];
    uint32_t row[kDropUnroll], j[kDropUnroll];
    int left[kDropUnroll];
#pragma unroll
    for (int i = 0; i < kDropUnroll; ++i) {
        const uint32_t v = blockIdx.x * (uint32_t)kDropBlock + i * kDropThreads + threadIdx.x;
        row[i] = p.per_row.div(v);
        j[i] = v - row[i] * p.per_row.d;
        left[i] = v < p.n_vec ? p.cols - (int)(8 * j[i]) : 0;
        const X *at = static_cast<const X *>(p.x) + row[i] * p.ldx + 8 * j[i];
        if constexpr (ALIGNED) x[i] = load8<true>(at, left[i]);
        else x[i] = load8_shifted(at, (int)(8 * j[i]), left[i]);
        if (!p.res) continue;
        const Y *add = static_cast<const Y *>(p.res) + row[i] * p.ldr + 8 * j[i];
        if constexpr (ALIGNED) r[i] = load8<true>(add, left[i]);
        else r[i] = load8_shifted(add, (int)(8 * j[i]), left[i]);
    }
#pragma unroll
    for (int i = 0; i < kDropUnroll; ++i) {
        if (ALIGNED && left[i] <= 0) continue;
        Vec8 v = to_float(x[i]);
        if (p.res) {
            // residual + x * factor with one rounding, as norm.cu has it
            const Vec8 a = to_float(r[i]);
            add_dropped8(p.drop, offset, p.row0 + row[i], j[i], v, a);
        } else if (p.drop.threshold) {
            drop8(p.drop, offset, p.row0 + row[i], j[i], v);
        }
        Y *to = static_cast<Y *>(p.y) + row[i] * p.ldy + 8 * j[i];
        if constexpr (ALIGNED) {
            store8<true>(to, from_float<Y>(v), left[i]);
        } else {
            // (a row's last vector has its end stored by its own lane: the next is of another)
            const int lane = threadIdx.x % 32;
            store8_shifted(to, from_float<Y>(v), left[i], lane > 0 && j[i] > 0 && left[i] > 0,
                           lane < 31 && j[i] + 1 < p.per_row.d && left[i] > 0);
        }
    }
}

template <typename X, typename Y>
static pos_status launch_dropout(DropoutParams p, int64_t rows, bool aligned, cudaStream_t s) {
    const int64_t per_row = (p.cols + 7ll) / 8;
    const int64_t most = std::max<int64_t>(1, (0x7fffffffll - kDropBlock) / per_row);
    auto kern = aligned ? dropout_kernel<X, Y, true> : dropout_kernel<X, Y, false>;
    for (int64_t r = 0; r < rows; r += most) {
        const int64_t n = std::min(most, rows - r);
        DropoutParams q = p;
        q.x = static_cast<const X *>(p.x) + r * p.ldx;
        q.res = p.res ? static_cast<const Y *>(p.res) + r * p.ldr : nullptr;
        q.y = static_cast<Y *>(p.y) + r * p.ldy;
        q.row0 = (uint32_t)r;
        q.n_vec = (uint32_t)(n * per_row);
        POS_CUDA(launch_dependent(kern, (int)((n * per_row + kDropBlock - 1) / kDropBlock),
                                  kDropThreads, 0, s, q));
    }
    return POS_OK;
}

template <typename X>
static pos_status dropout_to(int32_t dtype_y, const DropoutParams &p, int64_t rows, bool aligned,
                             cudaStream_t s) {
    switch (dtype_y) {
        case POS_BF16: return launch_dropout<X, __nv_bfloat16>(p, rows, aligned, s);
        case POS_F16: return launch_dropout<X, __half>(p, rows, aligned, s);
        default: return launch_dropout<X, float>(p, rows, aligned, s);
    }
}

}  // namespace pos

extern "C" pos_status poseidon_dropout(const pos_dropout *drop, int64_t rows, int64_t cols,
                                       const void *d_x, int32_t dtype, int64_t ldx,
                                       const void *d_res, int64_t ldr, void *d_y, int32_t dtype_y,
                                       int64_t ldy, void *stream) {
    using namespace pos;
    return guarded([&]() -> pos_status {
        if (!drop) return fail(POS_EINVAL, "dropout: NULL pointer");
        if (rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31) - 8)
            return fail(POS_EINVAL, "dropout: bad rows or cols");
        if (!dtype_ok(dtype) || !dtype_ok(dtype_y))
            return fail(POS_EINVAL, "dropout: unknown dtype");
        if (ldx < 0 || ldr < 0 || ldy < 0 || std::max(ldx, std::max(ldr, ldy)) >= (1ll << 31) ||
            (rows > 1 && ldy < cols))
            return fail(POS_EINVAL, "dropout: bad row stride");
        DropoutParams p = {};
        POS_TRY(make_drop(*drop, "dropout", &p.drop));
        if (rows == 0 || cols == 0) return POS_OK;
        if (!d_x || !d_y) return fail(POS_EINVAL, "dropout: NULL pointer");
        const int sx = dtype_size(dtype), sy = dtype_size(dtype_y);
        if (reinterpret_cast<uintptr_t>(d_x) % sx || reinterpret_cast<uintptr_t>(d_res) % sy ||
            reinterpret_cast<uintptr_t>(d_y) % sy)
            return fail(POS_EINVAL, "dropout: matrix not aligned to its elements");
        p.x = d_x, p.res = d_res, p.y = d_y;
        p.ldx = ldx, p.ldr = ldr, p.ldy = ldy;
        p.cols = (int32_t)cols;
        p.per_row = FastDiv((uint32_t)((cols + 7) / 8));
        const bool aligned = aligned16(d_x) && ldx * sx % 16 == 0 && aligned16(d_y) &&
                             ldy * sy % 16 == 0 && (!d_res || (aligned16(d_res) && ldr * sy % 16 == 0));
        const auto s = static_cast<cudaStream_t>(stream);
        switch (dtype) {
            case POS_BF16: return dropout_to<__nv_bfloat16>(dtype_y, p, rows, aligned, s);
            case POS_F16: return dropout_to<__half>(dtype_y, p, rows, aligned, s);
            default: return dropout_to<float>(dtype_y, p, rows, aligned, s);
        }
    });
}
