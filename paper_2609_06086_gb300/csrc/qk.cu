// poseidon_qk_forward, poseidon_qk_backward: RMS norm of every query and key
// head with the position rotation in the same pass, keeping q and k in 8 bits
// for the backward pass (formulas: poseidon.h).
#include <algorithm>

#include "layer_ops.cuh"

namespace pos {

constexpr int kQkWarps = 8;
constexpr int kQkThreads = 32 * kQkWarps;
constexpr int kQkMaxDim = 256;

struct QkTensor {
    void *p;
    int64_t token, head;  // strides in elements
};

struct QkParams {
    QkTensor a[2], b[2];       // forward: x, y; backward: dy, dx
    QkTensor x[2];             // backward without checkpoints
    const float *w[2];         // may be NULL
    float *rstd[2];            // [tokens][heads]; forward: may be NULL
    uint8_t *codes[2], *scales[2];  // checkpoint rows token * heads + head; may be NULL
    const float *cos, *sin;
    const int32_t *positions;
    float *part;               // backward: [block][2][dim] partial sums, or NULL
    int64_t tokens, tasks, n_pos;
    int32_t heads[2], dim, half, pitch, spitch;
    int32_t chunk, n_chunk;    // heads of a task, tasks of a token
    int32_t pairing, format;
    bool tables16;             // cos and sin rows can be read as 16-byte words
    float eps, inv_dim;
};

// What a thread knows of its 8 elements i = 8 l .. 8 l + 7 of every head of
// one token.  turn: element i of Rot u is u_i c_i + u_partner s_i (s with its
// sign), elements from rot on stay.
struct Turn {
    float c[8], s[8];
};

// POS_ROT_HALF: c, s per element; POS_ROT_ADJACENT: per pair, in [0, 4).
__device__ __forceinline__ void load_turn(const QkParams &p, int64_t at, int l, Turn &t) {
    const float *cs = p.cos + at * p.half, *sn = p.sin + at * p.half;
    if (p.pairing == POS_ROT_HALF) {
        const int first = 8 * l < p.half ? 8 * l : 8 * l - p.half;
        if (p.tables16 && p.half % 8 == 0) {
            if (8 * l < 2 * p.half) {
                const float4 c0 = *reinterpret_cast<const float4 *>(cs + first);
                const float4 c1 = *reinterpret_cast<const float4 *>(cs + first + 4);
                const float4 s0 = *reinterpret_cast<const float4 *>(sn + first);
                const float4 s1 = *reinterpret_cast<const float4 *>(sn + first + 4);
                const float sg = 8 * l < p.half ? -1.f : 1.f;
                const float c[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
                const float s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    t.c[e] = c[e];
                    t.s[e] = sg * s[e];
                }
            }
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = 8 * l + e;
            if (i >= 2 * p.half) continue;
            const int k = i < p.half ? i : i - p.half;
            t.c[e] = cs[k];
            t.s[e] = i < p.half ? -sn[k] : sn[k];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int k = 4 * l + e;
            if (k >= p.half) continue;
            t.c[e] = cs[k];
            t.s[e] = sn[k];
        }
    }
}

// Rot u, or with BACK its transpose, for the G lanes of a row.  Partners lie
// in the same thread (adjacent pairs), in one other lane at the same slot
// (half pairs of a half divisible by 8), or anywhere in the row, which then
// goes through shared memory (`row`, one float per element).  Lanes without
// a row take part in the exchanges.
template <int G, bool BACK>
__device__ __forceinline__ Vec8 turned(const QkParams &p, const Vec8 &u, const Turn &t, int l,
                                       float *row) {
    const int rot = 2 * p.half;
    Vec8 y = u;
    if (p.pairing == POS_ROT_ADJACENT) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = u.v[2 * e], b = u.v[2 * e + 1], s = BACK ? -t.s[e] : t.s[e];
            if (8 * l + 2 * e >= rot) continue;
            y.v[2 * e] = a * t.c[e] - b * s;
            y.v[2 * e + 1] = b * t.c[e] + a * s;
        }
        return y;
    }
    Vec8 q;
    if (p.half % 8 == 0) {
        const int d = p.half / 8;
        const int from = 8 * l < p.half ? l + d : (8 * l < rot ? l - d : l);
#pragma unroll
        for (int e = 0; e < 8; ++e) q.v[e] = __shfl_sync(0xffffffffu, u.v[e], from, G);
    } else {
        __syncwarp();
        *reinterpret_cast<float4 *>(row + 8 * l) = make_float4(u.v[0], u.v[1], u.v[2], u.v[3]);
        *reinterpret_cast<float4 *>(row + 8 * l + 4) = make_float4(u.v[4], u.v[5], u.v[6], u.v[7]);
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = 8 * l + e;
            q.v[e] = i < rot ? row[i < p.half ? i + p.half : i - p.half] : 0.f;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (8 * l + e < rot)
            y.v[e] = u.v[e] * t.c[e] + q.v[e] * (BACK ? -t.s[e] : t.s[e]);
    return y;
}

template <int G>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = 1; o < G; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

__device__ __forceinline__ Vec8 load_weights(const float *w, int l, int dim) {
    Vec8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v.v[e] = w && 8 * l + e < dim ? w[8 * l + e] : 1.f;
    return v;
}

// A token's place: its position, whether it is padding, whether the position
// lies outside the tables.
struct Place {
    int64_t at;
    bool padding, outside;
};
__device__ __forceinline__ Place place_of(const QkParams &p, int64_t token) {
    Place q;
    q.at = p.positions ? (int64_t)p.positions[token] : token;
    q.padding = q.at < 0;
    q.outside = q.at >= p.n_pos;
    return q;
}

// A task is one token and a run of its heads (queries, then keys); a warp
// takes it, G lanes a head with 8 elements a lane, 32 / G heads at once, U of
// those in flight.  The token's cosines and sines and both weights stay in
// registers over the task.  Bound by HBM: x is read once, y (and the codes)
// written once; the sum of squares, the groups' magnitudes and the partners of
// the rotation come from shuffles.
template <typename T, int G, int U, bool ALIGNED>
__global__ void __launch_bounds__(kQkThreads) qk_forward_kernel(const QkParams p) {
    constexpr int R = 32 / G;
    __shared__ float4 rows[kQkThreads * 2];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, l = lane % G, sub = lane / G;
    float *row = reinterpret_cast<float *>(rows) + warp * 256 + sub * 8 * G;
    const int64_t task = blockIdx.x * (int64_t)kQkWarps + warp;
    if (task >= p.tasks) return;
    const int64_t token = task / p.n_chunk;
    const int c0 = (int)(task - token * p.n_chunk) * p.chunk;
    const int c1 = min(c0 + p.chunk, p.heads[0] + p.heads[1]);
    const Place at = place_of(p, token);
    Vec8 w[2];
    Turn turn;
    for (int base = c0; base < c1; base += R * U) {
        Raw8<T> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = base + u * R + sub, k = c >= p.heads[0], h = k ? c - p.heads[0] : c;
            const T *x = static_cast<const T *>(p.a[k].p) + token * p.a[k].token +
                         h * p.a[k].head + 8 * l;
            raw[u] = load8<ALIGNED>(x, c < c1 ? p.dim - 8 * l : 0);
        }
        if (base == c0) {
            w[0] = load_weights(p.w[0], l, p.dim);
            w[1] = load_weights(p.w[1], l, p.dim);
#pragma unroll
            for (int e = 0; e < 8; ++e) turn.c[e] = 1.f, turn.s[e] = 0.f;
            if (!at.padding && !at.outside) load_turn(p, at.at, l, turn);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (base + u * R >= c1) break;  // no row of this step, for the whole warp
            const int c = base + u * R + sub, k = c >= p.heads[0], h = k ? c - p.heads[0] : c;
            const bool live = c < c1;
            const Vec8 x = to_float(raw[u]);
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(x.v[e], x.v[e], ss);
            float r = __frsqrt_rn(fmaf(row_sum<G>(ss), p.inv_dim, p.eps));
            const int64_t at_row = token * p.heads[k] + h;
            if (p.codes[0] || p.codes[1]) {
                uint32_t m = amax_bits(raw[u]);
                m = max_bits<T>(m, __shfl_xor_sync(0xffffffffu, m, 1));
                m = max_bits<T>(m, __shfl_xor_sync(0xffffffffu, m, 2));
                if (live && p.codes[k] && 8 * l < p.pitch) {
                    const uint32_t bits = f32_bits<T>(m);
                    const int byte = p.format == POS_CKPT_INT8 ? scale_byte<POS_CKPT_INT8>(bits)
                                                               : scale_byte<POS_CKPT_E4M3>(bits);
                    *reinterpret_cast<uint2 *>(p.codes[k] + at_row * p.pitch + 8 * l) =
                        p.format == POS_CKPT_INT8 ? encode8<POS_CKPT_INT8>(x, byte)
                                                  : encode8<POS_CKPT_E4M3>(x, byte);
                    if (l % 4 == 0) p.scales[k][at_row * p.spitch + l / 4] = (uint8_t)byte;
                }
            }
            if (live && p.rstd[k] && l == 0) p.rstd[k][at_row] = r;
            if (at.outside) r = __uint_as_float(0x7fffffffu);
            Vec8 y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y.v[e] = x.v[e] * r * (k ? w[1].v[e] : w[0].v[e]);
            y = turned<G, false>(p, y, turn, l, row);
            if (at.padding) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y.v[e] = 0.f;
            }
            T *out = static_cast<T *>(p.b[k].p) + token * p.b[k].token + h * p.b[k].head + 8 * l;
            store8<ALIGNED>(out, from_float<T>(y), live ? p.dim - 8 * l : 0);
        }
    }
}

// The same tasks, taken by a resident grid; dw is summed over a thread's rows
// in registers, over the block in shared memory, and written as one partial
// sum per block, which qk_dw_kernel adds up in order.
template <typename T, int G, int U, bool ALIGNED>
__global__ void __launch_bounds__(kQkThreads) qk_backward_kernel(const QkParams p) {
    constexpr int R = 32 / G;
    __shared__ float4 rows[kQkWarps * 2 * kQkMaxDim / 4];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, l = lane % G, sub = lane / G;
    float *row = reinterpret_cast<float *>(rows) + warp * 256 + sub * 8 * G;
    Vec8 w[2], dw[2];
    w[0] = load_weights(p.w[0], l, p.dim);
    w[1] = load_weights(p.w[1], l, p.dim);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[0].v[e] = dw[1].v[e] = 0.f;
    for (int64_t task = blockIdx.x * (int64_t)kQkWarps + warp; task < p.tasks;
         task += gridDim.x * (int64_t)kQkWarps) {
        const int64_t token = task / p.n_chunk;
        const int c0 = (int)(task - token * p.n_chunk) * p.chunk;
        const int c1 = min(c0 + p.chunk, p.heads[0] + p.heads[1]);
        const Place at = place_of(p, token);
        Turn turn;
#pragma unroll
        for (int e = 0; e < 8; ++e) turn.c[e] = 1.f, turn.s[e] = 0.f;
        if (!at.padding && !at.outside) load_turn(p, at.at, l, turn);
        for (int base = c0; base < c1; base += R * U) {
            Raw8<T> raw[U], rawx[U];
            uint2 code[U];
            int byte[U];
            float rs[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = base + u * R + sub, k = c >= p.heads[0], h = k ? c - p.heads[0] : c;
                const int n = c < c1 && !at.padding ? p.dim - 8 * l : 0;
                const int64_t at_row = token * p.heads[k] + h;
                raw[u] = load8<ALIGNED>(static_cast<const T *>(p.a[k].p) + token * p.a[k].token +
                                            h * p.a[k].head + 8 * l, n);
                rs[u] = 0.f, byte[u] = 0, code[u] = make_uint2(0u, 0u);
                if (n > 0) {
                    rs[u] = p.rstd[k][at_row];
                    if (!p.x[k].p) {
                        code[u] = *reinterpret_cast<const uint2 *>(p.codes[k] + at_row * p.pitch +
                                                                   8 * l);
                        byte[u] = p.scales[k][at_row * p.spitch + l / 4];
                    }
                }
                if (p.x[k].p)
                    rawx[u] = load8<ALIGNED>(static_cast<const T *>(p.x[k].p) +
                                                 token * p.x[k].token + h * p.x[k].head + 8 * l, n);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (base + u * R >= c1) break;  // no row of this step, for the whole warp
                const int c = base + u * R + sub, k = c >= p.heads[0], h = k ? c - p.heads[0] : c;
                const bool live = c < c1;
                const Vec8 g = turned<G, true>(p, to_float(raw[u]), turn, l, row);
                Vec8 n = p.x[k].p ? to_float(rawx[u])
                         : p.format == POS_CKPT_INT8
                             ? decode8<POS_CKPT_INT8>(code[u], scale_value(byte[u]))
                             : decode8<POS_CKPT_E4M3>(code[u], scale_value(byte[u]));
                const float r = at.outside ? __uint_as_float(0x7fffffffu) : rs[u];
                Vec8 hw;
                float dot = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    n.v[e] *= r;
                    hw.v[e] = g.v[e] * (k ? w[1].v[e] : w[0].v[e]);
                    dot = fmaf(hw.v[e], n.v[e], dot);
                    if (k) dw[1].v[e] = fmaf(g.v[e], n.v[e], dw[1].v[e]);
                    else dw[0].v[e] = fmaf(g.v[e], n.v[e], dw[0].v[e]);
                }
                dot = row_sum<G>(dot) * p.inv_dim;
                Vec8 dx;
#pragma unroll
                for (int e = 0; e < 8; ++e) dx.v[e] = r * (hw.v[e] - n.v[e] * dot);
                T *out = static_cast<T *>(p.b[k].p) + token * p.b[k].token + h * p.b[k].head + 8 * l;
                store8<ALIGNED>(out, from_float<T>(dx), live ? p.dim - 8 * l : 0);
            }
        }
    }
    if (!p.part) return;
    // [warp][2][dim], heads side by side in a warp first
    float *sum = reinterpret_cast<float *>(rows);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v = dw[k].v[e];
#pragma unroll
            for (int o = G; o < 32; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (sub == 0 && 8 * l + e < p.dim)
                sum[(warp * 2 + k) * kQkMaxDim + 8 * l + e] = v;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.dim; i += kQkThreads) {
        const int k = i >= p.dim, e = k ? i - p.dim : i;
        float v = 0.f;
        for (int q = 0; q < kQkWarps; ++q) v += sum[(q * 2 + k) * kQkMaxDim + e];
        p.part[blockIdx.x * (int64_t)(2 * p.dim) + i] = v;
    }
}

// dw = dw_in + the blocks' partial sums: a block of 32 x 32 threads takes 32
// columns, its rows a strided share of the partial sums each.
__global__ void __launch_bounds__(1024) qk_dw_kernel(const float *part, int n_part, int cols,
                                                     const float *dw_in, float *dw) {
    __shared__ float sum[32][33];
    const int i = blockIdx.x * 32 + threadIdx.x;
    float v = 0.f;
    if (i < cols)
        for (int b = threadIdx.y; b < n_part; b += 32) v += part[b * (int64_t)cols + i];
    sum[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    v = sum[threadIdx.x][threadIdx.y];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    const int j = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && j < cols) dw[j] = dw_in ? dw_in[j] + v : v;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
static pos_status check_qk(const pos_qk *q) {
    if (!q) return fail(POS_EINVAL, "q/k: NULL pointer");
    if (q->tokens < 0 || q->heads_q < 0 || q->heads_k < 0 || q->tokens >= (1ll << 40) ||
        q->heads_q >= (1 << 20) || q->heads_k >= (1 << 20))
        return fail(POS_EINVAL, "q/k: bad token or head count");
    if (q->dim < 1 || q->dim > kQkMaxDim) return fail(POS_EINVAL, "q/k: dim must be 1..256");
    if (q->rot < 0 || q->rot > q->dim || q->rot % 2)
        return fail(POS_EINVAL, "q/k: rot must be even and at most dim");
    if (q->pairing != POS_ROT_HALF && q->pairing != POS_ROT_ADJACENT)
        return fail(POS_EINVAL, "q/k: unknown pairing");
    if (!dtype_ok(q->dtype)) return fail(POS_EINVAL, "q/k: unknown dtype");
    if (!format_ok(q->format)) return fail(POS_EINVAL, "q/k: unknown format");
    if (!(q->eps >= 0.f)) return fail(POS_EINVAL, "q/k: eps must be >= 0");
    if (q->n_pos < 0) return fail(POS_EINVAL, "q/k: n_pos must be >= 0");
    if (q->rot > 0 && q->n_pos > 0 && (!q->cos || !q->sin))
        return fail(POS_EINVAL, "q/k: NULL tables");
    return POS_OK;
}

// A host array of two tensors; data may be NULL where there is nothing.
static pos_status check_heads(const pos_qk *q, const pos_heads *t, const char *what, bool written) {
    if (!t) return fail(POS_EINVAL, std::string("q/k: NULL ") + what);
    for (int k = 0; k < 2; ++k) {
        const int64_t heads = k ? q->heads_k : q->heads_q;
        if (t[k].token_stride < 0 || t[k].head_stride < 0 || t[k].token_stride >= (1ll << 40) ||
            t[k].head_stride >= (1ll << 40))
            return fail(POS_EINVAL, std::string("q/k: bad stride of ") + what);
        if (heads == 0 || q->tokens == 0) continue;
        if (!t[k].data) return fail(POS_EINVAL, std::string("q/k: NULL ") + what);
        if (reinterpret_cast<uintptr_t>(t[k].data) % dtype_size(q->dtype))
            return fail(POS_EINVAL, std::string("q/k: misaligned ") + what);
        if (written && ((heads > 1 && t[k].head_stride < q->dim) ||
                        (q->tokens > 1 && t[k].token_stride < q->dim)))
            return fail(POS_EINVAL, std::string("q/k: overlapping rows of ") + what);
    }
    return POS_OK;
}

static bool heads_aligned(const pos_qk *q, const pos_heads *t) {
    const int64_t per = 16 / dtype_size(q->dtype);
    for (int k = 0; k < 2; ++k)
        if (!aligned16(t[k].data) || t[k].token_stride % per || t[k].head_stride % per) return false;
    return q->dim % 8 == 0;
}

static QkParams make_params(const pos_qk *q) {
    QkParams p = {};
    p.w[0] = q->w_q, p.w[1] = q->w_k;
    p.cos = q->cos, p.sin = q->sin;
    p.positions = q->positions;
    p.tokens = q->tokens, p.n_pos = q->n_pos;
    p.heads[0] = q->heads_q, p.heads[1] = q->heads_k;
    p.dim = q->dim, p.half = q->rot / 2;
    const CkptShape s = ckpt_shape(q->dim);
    p.pitch = (int32_t)s.pitch, p.spitch = (int32_t)s.spitch;
    p.pairing = q->pairing, p.format = q->format;
    p.tables16 = aligned16(q->cos) && aligned16(q->sin) && p.half % 4 == 0;
    p.eps = q->eps, p.inv_dim = 1.f / q->dim;
    return p;
}

// Lanes per head: 8 elements a lane, a power of two.
static int lanes_per_head(int dim) { return dim <= 64 ? 8 : dim <= 128 ? 16 : 32; }

// Cuts a token's heads into tasks: as few as keep `warps` warps busy (each
// reads the token's cosines and sines again), at least 32 / G heads a task.
static void cut_tasks(QkParams &p, int64_t warps) {
    const int R = 32 / lanes_per_head(p.dim), heads = p.heads[0] + p.heads[1];
    const int most = (heads + R - 1) / R;
    const int64_t want = p.tokens ? (warps + p.tokens - 1) / p.tokens : 1;
    const int n = (int)std::max<int64_t>(1, std::min<int64_t>(want, most));
    p.chunk = ((most + n - 1) / n) * R;
    p.n_chunk = (heads + p.chunk - 1) / p.chunk;
    p.tasks = p.tokens * p.n_chunk;
}

template <typename T, int G, int U>
static pos_status launch_forward(const QkParams &p, bool aligned, cudaStream_t s) {
    const int64_t grid = (p.tasks + kQkWarps - 1) / kQkWarps;
    if (grid > 0x7fffffffll) return fail(POS_EINVAL, "q/k: too many tokens");
    if (aligned) qk_forward_kernel<T, G, U, true><<<(unsigned)grid, kQkThreads, 0, s>>>(p);
    else qk_forward_kernel<T, G, U, false><<<(unsigned)grid, kQkThreads, 0, s>>>(p);
    POS_CUDA(cudaGetLastError());
    return POS_OK;
}

template <typename T>
static pos_status forward_of(const QkParams &p, bool aligned, cudaStream_t s) {
    constexpr int U = sizeof(T) == 4 ? 2 : 4;
    switch (lanes_per_head(p.dim)) {
        case 8: return launch_forward<T, 8, U>(p, aligned, s);
        case 16: return launch_forward<T, 16, U>(p, aligned, s);
        default: return launch_forward<T, 32, U>(p, aligned, s);
    }
}

template <typename T, int G, int U>
static pos_status launch_backward(QkParams &p, bool aligned, const float *dw_in, float *dw,
                                  cudaStream_t s) {
    auto kern = aligned ? qk_backward_kernel<T, G, U, true> : qk_backward_kernel<T, G, U, false>;
    int per_sm = 0;
    POS_TRY(blocks_per_sm(reinterpret_cast<const void *>(kern), kQkThreads, 0, &per_sm));
    per_sm = std::max(1, std::min(per_sm, 8));
    cut_tasks(p, (int64_t)sm_count() * per_sm * kQkWarps);
    const int grid = (int)std::min<int64_t>((p.tasks + kQkWarps - 1) / kQkWarps,
                                            (int64_t)sm_count() * per_sm);
    const int cols = 2 * p.dim;
    void *scratch = nullptr;
    if (dw && grid > 0) {
        cudaMemPool_t pool;
        POS_TRY(scratch_pool(&pool));
        POS_CUDA(cudaMallocFromPoolAsync(&scratch, (size_t)grid * cols * 4, pool, s));
        p.part = static_cast<float *>(scratch);
    }
    if (grid > 0) kern<<<grid, kQkThreads, 0, s>>>(p);
    cudaError_t e = cudaGetLastError();
    if (dw && e == cudaSuccess) {
        qk_dw_kernel<<<(cols + 31) / 32, dim3(32, 32), 0, s>>>(p.part, grid, cols, dw_in, dw);
        e = cudaGetLastError();
    }
    const cudaError_t e2 = scratch ? cudaFreeAsync(scratch, s) : cudaSuccess;
    if (e == cudaSuccess) e = e2;
    return e == cudaSuccess ? POS_OK : cuda_fail(e, "q/k backward");
}

template <typename T>
static pos_status backward_of(QkParams &p, bool aligned, const float *dw_in, float *dw,
                              cudaStream_t s) {
    constexpr int U = sizeof(T) == 4 ? 1 : 2;
    switch (lanes_per_head(p.dim)) {
        case 8: return launch_backward<T, 8, U>(p, aligned, dw_in, dw, s);
        case 16: return launch_backward<T, 16, U>(p, aligned, dw_in, dw, s);
        default: return launch_backward<T, 32, U>(p, aligned, dw_in, dw, s);
    }
}

static pos_status set_ckpt(QkParams &p, const void *ckpt_q, const void *ckpt_k) {
    for (int k = 0; k < 2; ++k) {
        uint8_t *c = static_cast<uint8_t *>(const_cast<void *>(k ? ckpt_k : ckpt_q));
        if (!c) continue;
        if (!aligned16(c)) return fail(POS_EINVAL, "q/k: checkpoint not 16-byte aligned");
        p.codes[k] = c;
        p.scales[k] = c + p.tokens * p.heads[k] * p.pitch;
    }
    return POS_OK;
}

}  // namespace pos

extern "C" {

pos_status poseidon_qk_forward(const pos_qk *qk, const pos_heads *x, const pos_heads *y,
                               float *rstd_q, float *rstd_k, void *ckpt_q, void *ckpt_k,
                               void *stream) {
    using namespace pos;
    POS_TRY(check_qk(qk));
    POS_TRY(check_heads(qk, x, "x", false));
    POS_TRY(check_heads(qk, y, "y", true));
    QkParams p = make_params(qk);
    POS_TRY(set_ckpt(p, ckpt_q, ckpt_k));
    if (p.tokens == 0 || p.heads[0] + p.heads[1] == 0) return POS_OK;
    for (int k = 0; k < 2; ++k) {
        p.a[k] = {x[k].data, x[k].token_stride, x[k].head_stride};
        p.b[k] = {y[k].data, y[k].token_stride, y[k].head_stride};
    }
    p.rstd[0] = rstd_q, p.rstd[1] = rstd_k;
    cut_tasks(p, (int64_t)sm_count() * 64);
    const bool aligned = heads_aligned(qk, x) && heads_aligned(qk, y);
    const auto s = static_cast<cudaStream_t>(stream);
    switch (qk->dtype) {
        case POS_BF16: return forward_of<__nv_bfloat16>(p, aligned, s);
        case POS_F16: return forward_of<__half>(p, aligned, s);
        default: return forward_of<float>(p, aligned, s);
    }
}

pos_status poseidon_qk_backward(const pos_qk *qk, const pos_heads *x, const void *ckpt_q,
                                const void *ckpt_k, const float *rstd_q, const float *rstd_k,
                                const pos_heads *dy, const pos_heads *dx, const float *d_dw_in,
                                float *d_dw, void *stream) {
    using namespace pos;
    POS_TRY(check_qk(qk));
    if (x) POS_TRY(check_heads(qk, x, "x", false));
    POS_TRY(check_heads(qk, dy, "dy", false));
    POS_TRY(check_heads(qk, dx, "dx", true));
    QkParams p = make_params(qk);
    POS_TRY(set_ckpt(p, ckpt_q, ckpt_k));
    if (d_dw_in && !d_dw) return fail(POS_EINVAL, "q/k: dw_in without dw");
    p.rstd[0] = const_cast<float *>(rstd_q), p.rstd[1] = const_cast<float *>(rstd_k);
    for (int k = 0; k < 2; ++k) {
        p.a[k] = {dy[k].data, dy[k].token_stride, dy[k].head_stride};
        p.b[k] = {dx[k].data, dx[k].token_stride, dx[k].head_stride};
        if (x) p.x[k] = {x[k].data, x[k].token_stride, x[k].head_stride};
        if (p.tokens == 0 || p.heads[k] == 0) continue;
        if (!x && !p.codes[k]) return fail(POS_EINVAL, "q/k: neither x nor its checkpoint");
        if (!p.rstd[k]) return fail(POS_EINVAL, "q/k: NULL rstd");
    }
    const bool aligned =
        heads_aligned(qk, dy) && heads_aligned(qk, dx) && (!x || heads_aligned(qk, x));
    const auto s = static_cast<cudaStream_t>(stream);
    switch (qk->dtype) {
        case POS_BF16: return backward_of<__nv_bfloat16>(p, aligned, d_dw_in, d_dw, s);
        case POS_F16: return backward_of<__half>(p, aligned, d_dw_in, d_dw, s);
        default: return backward_of<float>(p, aligned, d_dw_in, d_dw, s);
    }
}

}  // extern "C"
