// poseidon_ckpt_bytes, poseidon_ckpt_pack, poseidon_ckpt_unpack: 8-bit
// checkpoints of activations (format: poseidon.h).
#include "layer_ops.cuh"

namespace pos {

constexpr int kPackThreads = 256;
constexpr int kPackUnroll = 4;  // vectors of 8 elements in flight per thread
constexpr int kPackBlock = kPackThreads * kPackUnroll;

struct PackParams {
    const void *x;     // pack: input; unpack: output
    uint8_t *codes, *scales;
    int64_t ld, pitch, spitch;
    uint32_t n_vec;    // rows * pitch / 8
    int32_t cols;
    FastDiv per_row;   // pitch / 8
};

// A thread takes vectors of 8 elements (a warp: 256 consecutive ones), four
// lanes share a group's largest magnitude by two shuffles.  Bound by HBM:
// every value is read once and every code written once.  Packing and unpacking
// 16384 x 8192 f32: 229 us, 5.9 TB/s.
template <typename T, int F, bool ALIGNED>
__global__ void __launch_bounds__(kPackThreads) pack_kernel(const PackParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    const T *x = static_cast<const T *>(p.x);
    Raw8<T> raw[kPackUnroll];
    uint32_t row[kPackUnroll], j[kPackUnroll];
#pragma unroll
    for (int i = 0; i < kPackUnroll; ++i) {
        const uint32_t v = blockIdx.x * (uint32_t)kPackBlock + i * kPackThreads + threadIdx.x;
        const uint32_t r = p.per_row.div(v);
        row[i] = r;
        j[i] = v - r * p.per_row.d;
        const int left = v < p.n_vec ? p.cols - (int)(8 * j[i]) : 0;
        const T *at = x + (int64_t)r * p.ld + 8 * j[i];
        if constexpr (ALIGNED) raw[i] = load8<true>(at, left);
        else raw[i] = load8_shifted(at, (int)(8 * j[i]), left);
    }
#pragma unroll
    for (int i = 0; i < kPackUnroll; ++i) {
        const uint32_t v = blockIdx.x * (uint32_t)kPackBlock + i * kPackThreads + threadIdx.x;
        uint32_t m = amax_bits(raw[i]);
        m = max_bits<T>(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max_bits<T>(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const int byte = scale_byte<F>(f32_bits<T>(m));
        if (v >= p.n_vec) continue;
        *reinterpret_cast<uint2 *>(p.codes + row[i] * p.pitch + 8 * j[i]) =
            encode8<F>(to_float(raw[i]), byte);
        if (j[i] % 4 == 0) p.scales[row[i] * p.spitch + j[i] / 4] = (uint8_t)byte;
    }
}

template <typename T, int F>
__global__ void __launch_bounds__(kPackThreads) unpack_kernel(const PackParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    T *y = static_cast<T *>(const_cast<void *>(p.x));
    uint2 code[kPackUnroll];
    int byte[kPackUnroll];
    uint32_t row[kPackUnroll], j[kPackUnroll];
#pragma unroll
    for (int i = 0; i < kPackUnroll; ++i) {
        const uint32_t v = blockIdx.x * (uint32_t)kPackBlock + i * kPackThreads + threadIdx.x;
        row[i] = p.per_row.div(v);
        j[i] = v - row[i] * p.per_row.d;
        if (v >= p.n_vec) continue;
        code[i] = *reinterpret_cast<const uint2 *>(p.codes + row[i] * p.pitch + 8 * j[i]);
        byte[i] = p.scales[row[i] * p.spitch + j[i] / 4];
    }
#pragma unroll
    for (int i = 0; i < kPackUnroll; ++i) {
        const uint32_t v = blockIdx.x * (uint32_t)kPackBlock + i * kPackThreads + threadIdx.x;
        if (v >= p.n_vec) continue;
        store8<true>(y + (int64_t)row[i] * p.ld + 8 * j[i],
                     from_float<T, true>(decode8<F>(code[i], scale_value(byte[i]))),
                     p.cols - (int)(8 * j[i]));
    }
}

// Rows that are not 16-byte aligned: a thread's 8 elements are those of an
// aligned word of y, columns 8 j - m .. 8 j - m + 7 for a row that starts m
// elements past one; their codes come from two words, under two scales.  One
// vector more per row than above.  5003 x 5001 f16: 15 us, 75% of HBM's rate
// (element by element 71 us: most of a sector is rewritten eight times).
template <typename T, int F>
__global__ void __launch_bounds__(kPackThreads) unpack_shifted_kernel(const PackParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    constexpr int kPer = 16 / sizeof(T);
    T *y = static_cast<T *>(const_cast<void *>(p.x));
    uint2 lo[kPackUnroll], hi[kPackUnroll];
    int b0[kPackUnroll], b1[kPackUnroll];
    uint32_t row[kPackUnroll], j[kPackUnroll];
#pragma unroll
    for (int i = 0; i < kPackUnroll; ++i) {
        const uint32_t v = blockIdx.x * (uint32_t)kPackBlock + i * kPackThreads + threadIdx.x;
        row[i] = p.per_row.div(v);
        j[i] = v - row[i] * p.per_row.d;
        lo[i] = hi[i] = make_uint2(0u, 0u);
        b0[i] = b1[i] = 0;
        if (v >= p.n_vec) continue;
        const uint8_t *codes = p.codes + row[i] * p.pitch, *scales = p.scales + row[i] * p.spitch;
        if (j[i] > 0) {
            lo[i] = *reinterpret_cast<const uint2 *>(codes + 8 * j[i] - 8);
            b0[i] = scales[(j[i] - 1) / 4];
        }
        if (8 * j[i] < p.pitch) {
            hi[i] = *reinterpret_cast<const uint2 *>(codes + 8 * j[i]);
            b1[i] = scales[j[i] / 4];
        }
    }
#pragma unroll
    for (int i = 0; i < kPackUnroll; ++i) {
        const uint32_t v = blockIdx.x * (uint32_t)kPackBlock + i * kPackThreads + threadIdx.x;
        if (v >= p.n_vec) continue;
        T *start = y + (int64_t)row[i] * p.ld;
        const int m = (int)(reinterpret_cast<uintptr_t>(start) / sizeof(T) % kPer);
        // bytes 8 - m .. 15 - m of the two words of codes
        const int q = (8 - m) / 4;
        const uint32_t w0 = q == 0 ? lo[i].x : q == 1 ? lo[i].y : hi[i].x;
        const uint32_t w1 = q == 0 ? lo[i].y : q == 1 ? hi[i].x : hi[i].y;
        const uint32_t w2 = q == 0 ? hi[i].x : hi[i].y;
        const uint32_t by = 8 * ((8 - m) % 4);
        Vec8 f = decode8<F>(make_uint2(__funnelshift_r(w0, w1, by), __funnelshift_r(w1, w2, by)),
                            1.f);
        const float s0 = scale_value(b0[i]), s1 = scale_value(b1[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) f.v[e] *= e < m ? s0 : s1;
        const Raw8<T> out = from_float<T, true>(f);
        const int first = (int)(8 * j[i]) - m, left = p.cols - first;  // column, columns from it
        if (first >= 0) {
            store8<true>(start + first, out, left);
        } else {  // a row's first word: from its first column on
            const uint32_t w[8] = {out.a.x, out.a.y, out.a.z, out.a.w, 0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e < m || e >= left) continue;
                if constexpr (sizeof(T) == 2)
                    reinterpret_cast<uint16_t *>(start)[first + e] =
                        (uint16_t)(w[e / 2] >> 16 * (e % 2));
                else
                    start[first + e] = f.v[e];
            }
        }
    }
}

// Both kernels over all rows, at most 2^31 vectors a launch.
template <typename T, int F>
static pos_status launch_pack(bool pack, const void *x, int64_t rows, int64_t cols, int64_t ld,
                              void *ckpt, cudaStream_t stream) {
    const CkptShape s = ckpt_shape(cols);
    const bool aligned = aligned16(x) && ld * (int64_t)sizeof(T) % 16 == 0;
    const int64_t per_row = s.pitch / 8 + (!pack && !aligned ? 1 : 0);
    const int64_t most = std::max<int64_t>(1, (0x7fffffffll - kPackBlock) / per_row);
    for (int64_t r = 0; r < rows; r += most) {
        const int64_t n = std::min(most, rows - r);
        PackParams p{static_cast<const T *>(x) + r * ld,
                     static_cast<uint8_t *>(ckpt) + r * s.pitch,
                     static_cast<uint8_t *>(ckpt) + rows * s.pitch + r * s.spitch,
                     ld, s.pitch, s.spitch, (uint32_t)(n * per_row), (int32_t)cols,
                     FastDiv((uint32_t)per_row)};
        const int grid = (int)((n * per_row + kPackBlock - 1) / kPackBlock);
        auto kern = pack ? (aligned ? pack_kernel<T, F, true> : pack_kernel<T, F, false>)
                         : (aligned ? unpack_kernel<T, F> : unpack_shifted_kernel<T, F>);
        POS_CUDA(launch_dependent(kern, grid, kPackThreads, 0, stream, p));
    }
    return POS_OK;
}

static pos_status pack_or_unpack(bool pack, const void *x, int32_t dtype, int64_t rows,
                                 int64_t cols, int64_t ld, int32_t format, void *ckpt,
                                 void *stream) {
    if (!ckpt_size_ok(rows, cols)) return fail(POS_EINVAL, "checkpoint: bad rows or cols");
    if (!dtype_ok(dtype)) return fail(POS_EINVAL, "checkpoint: unknown dtype");
    if (!format_ok(format)) return fail(POS_EINVAL, "checkpoint: unknown format");
    if (ld < 0 || ld >= (1ll << 40) || (!pack && ld < cols && rows > 1))
        return fail(POS_EINVAL, "checkpoint: bad row stride");
    if (rows == 0 || cols == 0) return POS_OK;
    if (!x || !ckpt) return fail(POS_EINVAL, "checkpoint: NULL pointer");
    if (!aligned16(ckpt)) return fail(POS_EINVAL, "checkpoint: buffer not 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(x) % dtype_size(dtype))
        return fail(POS_EINVAL, "checkpoint: matrix not aligned to its elements");
    const auto s = static_cast<cudaStream_t>(stream);
    const bool i8 = format == POS_CKPT_INT8;
    if (dtype == POS_BF16)
        return i8 ? launch_pack<__nv_bfloat16, POS_CKPT_INT8>(pack, x, rows, cols, ld, ckpt, s)
                  : launch_pack<__nv_bfloat16, POS_CKPT_E4M3>(pack, x, rows, cols, ld, ckpt, s);
    if (dtype == POS_F16)
        return i8 ? launch_pack<__half, POS_CKPT_INT8>(pack, x, rows, cols, ld, ckpt, s)
                  : launch_pack<__half, POS_CKPT_E4M3>(pack, x, rows, cols, ld, ckpt, s);
    return i8 ? launch_pack<float, POS_CKPT_INT8>(pack, x, rows, cols, ld, ckpt, s)
              : launch_pack<float, POS_CKPT_E4M3>(pack, x, rows, cols, ld, ckpt, s);
}

}  // namespace pos

extern "C" {

pos_status poseidon_ckpt_bytes(int64_t rows, int64_t cols, int64_t *bytes) {
    return pos::guarded([&] {
        if (!bytes) return pos::fail(POS_EINVAL, "checkpoint: NULL pointer");
        if (!pos::ckpt_size_ok(rows, cols))
            return pos::fail(POS_EINVAL, "checkpoint: bad rows or cols");
        const pos::CkptShape s = pos::ckpt_shape(cols);
        *bytes = rows * (s.pitch + s.spitch);
        return (pos_status)POS_OK;
    });
}

pos_status poseidon_ckpt_pack(const void *d_x, int32_t dtype, int64_t rows, int64_t cols,
                              int64_t ldx, int32_t format, void *d_ckpt, void *stream) {
    return pos::guarded([&] {
        return pos::pack_or_unpack(true, d_x, dtype, rows, cols, ldx, format, d_ckpt, stream);
    });
}

pos_status poseidon_ckpt_unpack(const void *d_ckpt, int32_t format, int64_t rows, int64_t cols,
                                void *d_y, int32_t dtype, int64_t ldy, void *stream) {
    return pos::guarded([&] {
        return pos::pack_or_unpack(false, d_y, dtype, rows, cols, ldy, format,
                                   const_cast<void *>(d_ckpt), stream);
    });
}

}  // extern "C"
