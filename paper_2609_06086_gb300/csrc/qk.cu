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
    int64_t tokens, n_pos;
    int32_t heads[2], dim, half, pitch, spitch;
    int64_t tasks[2];              // forward: all tasks,
    int32_t chunk[2], n_chunk[2];  // heads of a task, tasks of a token
    int32_t steps[2];          // backward: of a token, its heads by what a warp takes at once
    int32_t step_bytes;        // backward: shared memory of a step
    int32_t pairing, format;
    bool vectors;              // cos, sin and w can be read 16 bytes at a time
    float eps, inv_dim;
};

// A thread's 8 elements of a head, as four pairs.
struct Eight {
    F2 v[4];
};

// How a kernel reads heads: kAny one element at a time, kAligned 16 bytes at a
// time (dim is a multiple of 8: a lane has 8 elements or none), kFull likewise
// heads of exactly 8 G elements, G lanes a head, so that sizes and offsets are
// constants.
enum Loads { kAny, kAligned, kFull };
template <int G, int A>
__device__ __forceinline__ int dim_of(const QkParams &p) {
    return A == kFull ? 8 * G : p.dim;
}
template <int G, int A>
__device__ __forceinline__ int pitch_of(const QkParams &p) {
    return A == kFull ? 8 * G : p.pitch;
}
template <int G, int A>
__device__ __forceinline__ int spitch_of(const QkParams &p) {
    return A == kFull ? (G + 15) / 16 * 4 : p.spitch;
}

// Where a thread's elements lie in a head.
//   kRun: elements 8 l .. 8 l + 7.  The partners of the rotation lie in the
//     same pair (POS_ROT_ADJACENT), in one other lane (POS_ROT_HALF with
//     rot / 2 divisible by 8) or anywhere in the row.
//   kSplit (kFull, POS_ROT_HALF, rot = dim): 4 l .. 4 l + 3 and as many from
//     dim / 2 + 4 l on, so that partners lie in the same thread and a group of 32
//     columns in 8 lanes.  8192 tokens of 64 + 8 heads of 128, bf16: 73.7 us
//     forward and 79.0 us backward; exchanging kRun's partners by shuffles took
//     8 us and 19 us more.
enum Layout { kRun, kSplit };
template <int L>
__device__ __forceinline__ int first_of(int l) {  // the thread's first element
    return (L == kSplit ? 4 : 8) * l;
}
template <int G, int L>
__device__ __forceinline__ int element(int l, int e) {
    return L == kSplit && e >= 4 ? 4 * G + 4 * l + (e - 4) : first_of<L>(l) + e;
}

// The words of a thread's elements, the first of them at `at`.
template <typename T, int G, int L, int A>
__device__ __forceinline__ Raw8<T> load_row(const QkParams &p, const T *at, int l, bool live) {
    if constexpr (A == kAny) {
        return load8<false>(at, live ? p.dim - 8 * l : 0);
    } else {
        Raw8<T> r;
        zero_raw(r.a);
        if constexpr (sizeof(T) == 4) zero_raw(r.b);
        if (live && 8 * l < dim_of<G, A>(p)) {
            if constexpr (sizeof(T) == 4) {
                r.a = *reinterpret_cast<const uint4 *>(at);
                r.b = *reinterpret_cast<const uint4 *>(at + (L == kSplit ? 4 * G : 4));
            } else if constexpr (L == kRun) {
                r.a = *reinterpret_cast<const uint4 *>(at);
            } else {
                const uint2 a = *reinterpret_cast<const uint2 *>(at);
                const uint2 b = *reinterpret_cast<const uint2 *>(at + 4 * G);
                r.a = make_uint4(a.x, a.y, b.x, b.y);
            }
        }
        return r;
    }
}
template <typename T, int G, int L, int A>
__device__ __forceinline__ void store_row(const QkParams &p, T *at, int l, bool live,
                                          const Raw8<T> &r) {
    if constexpr (A == kAny) {
        store8<false>(at, r, live ? p.dim - 8 * l : 0);
    } else if (live && 8 * l < dim_of<G, A>(p)) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<uint4 *>(at) = r.a;
            *reinterpret_cast<uint4 *>(at + (L == kSplit ? 4 * G : 4)) = r.b;
        } else if constexpr (L == kRun) {
            *reinterpret_cast<uint4 *>(at) = r.a;
        } else {
            *reinterpret_cast<uint2 *>(at) = make_uint2(r.a.x, r.a.y);
            *reinterpret_cast<uint2 *>(at + 4 * G) = make_uint2(r.a.z, r.a.w);
        }
    }
}

__device__ __forceinline__ Eight pairs_of(const Vec8 &x) {
    return {{{x.v[0], x.v[1]}, {x.v[2], x.v[3]}, {x.v[4], x.v[5]}, {x.v[6], x.v[7]}}};
}
__device__ __forceinline__ Vec8 values_of(const Eight &x) {
    return {{x.v[0].x, x.v[0].y, x.v[1].x, x.v[1].y, x.v[2].x, x.v[2].y, x.v[3].x, x.v[3].y}};
}

// Every element's partner in the rotation (elements without one: anything).
// Lanes without a row take part in the exchanges.
template <int G, int L>
__device__ __forceinline__ Eight partners(const QkParams &p, const Eight &u, int l, float *row) {
    if constexpr (L == kSplit) return {{u.v[2], u.v[3], u.v[0], u.v[1]}};
    Eight q;
    if (p.pairing == POS_ROT_ADJACENT) {
#pragma unroll
        for (int i = 0; i < 4; ++i) q.v[i] = {u.v[i].y, u.v[i].x};
    } else if (p.half % 8 == 0) {
        const int d = p.half / 8;
        const int from = 8 * l < p.half ? l + d : (8 * l < 2 * p.half ? l - d : l);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            q.v[i] = {__shfl_sync(0xffffffffu, u.v[i].x, from, G),
                      __shfl_sync(0xffffffffu, u.v[i].y, from, G)};
    } else {
        // row: the warp's 256 floats
        float *own = row + 8 * (threadIdx.x % 32);
        __syncwarp();
        *reinterpret_cast<float4 *>(own) = make_float4(u.v[0].x, u.v[0].y, u.v[1].x, u.v[1].y);
        *reinterpret_cast<float4 *>(own + 4) = make_float4(u.v[2].x, u.v[2].y, u.v[3].x, u.v[3].y);
        __syncwarp();
        // partners of pairs are pairs: 4096 tokens of 72 heads of 72, bf16, take 49.4
        // us forward, element by element 59.1
        if (p.half % 2 == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = 8 * l + 2 * i;
                const float2 v = e < 2 * p.half ? *reinterpret_cast<const float2 *>(
                                                      own + 2 * i + (e < p.half ? p.half : -p.half))
                                                : make_float2(0.f, 0.f);
                q.v[i] = {v.x, v.y};
            }
            return q;
        }
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = 8 * l + e;
            o[e] = i < 2 * p.half ? own[i < p.half ? e + p.half : e - p.half] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) q.v[i] = {o[2 * i], o[2 * i + 1]};
    }
    return q;
}

// A thread's weights; ones where there are none.
template <int G, int L, int A>
__device__ __forceinline__ Eight load_weights(const QkParams &p, const float *w, int l) {
    Eight o;
    if (L == kSplit && w && p.vectors) {
        const float4 a = *reinterpret_cast<const float4 *>(w + 4 * l);
        const float4 b = *reinterpret_cast<const float4 *>(w + 4 * G + 4 * l);
        return {{{a.x, a.y}, {a.z, a.w}, {b.x, b.y}, {b.z, b.w}}};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = element<G, L>(l, 2 * i), dim = dim_of<G, A>(p);
        o.v[i] = {w && e < dim ? w[e] : 1.f, w && e + 1 < dim ? w[e + 1] : 1.f};
    }
    return o;
}

// y = x c + partner s is Rot x: the cosine of an element's pair, and its sine
// with the sign that the partner's term has; 1 and 0 from rot on.
template <int G, int L>
__device__ __forceinline__ void load_angles(const QkParams &p, int64_t at, int l, Eight &c,
                                            Eight &s) {
    const float *cs = p.cos + at * p.half, *sn = p.sin + at * p.half;
    if constexpr (L == kSplit) {
        float4 a, b;
        if (p.vectors) {
            a = *reinterpret_cast<const float4 *>(cs + 4 * l);
            b = *reinterpret_cast<const float4 *>(sn + 4 * l);
        } else {
            a = make_float4(cs[4 * l], cs[4 * l + 1], cs[4 * l + 2], cs[4 * l + 3]);
            b = make_float4(sn[4 * l], sn[4 * l + 1], sn[4 * l + 2], sn[4 * l + 3]);
        }
        c = {{{a.x, a.y}, {a.z, a.w}, {a.x, a.y}, {a.z, a.w}}};
        s = {{{-b.x, -b.y}, {-b.z, -b.w}, {b.x, b.y}, {b.z, b.w}}};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c.v[i] = both(1.f), s.v[i] = both(0.f);
            const int e = 8 * l + 2 * i;  // even, as rot is: both elements turn or none
            if (e >= 2 * p.half) continue;
            if (p.pairing == POS_ROT_ADJACENT) {
                const float a = cs[e / 2], b = sn[e / 2];
                c.v[i] = {a, a}, s.v[i] = {-b, b};
            } else {
                const int k0 = e < p.half ? e : e - p.half;
                const int k1 = e + 1 < p.half ? e + 1 : e + 1 - p.half;
                c.v[i] = {cs[k0], cs[k1]};
                s.v[i] = {e < p.half ? -sn[k0] : sn[k0], e + 1 < p.half ? -sn[k1] : sn[k1]};
            }
        }
    }
}

// x c + partner s for a lane's pair i.  Elements from rot on have no partner term: with a
// sine of 0 an infinity or NaN of theirs, or in the pair's other half, would still make
// a NaN.  turning: how many of the lane's pairs lie below rot (any number, <= 0: none).
template <int L>
__device__ __forceinline__ F2 turn(F2 x, F2 c, F2 partner, F2 s, int i, int turning) {
    const F2 y = mul2(x, c);
    return L == kSplit || i < turning ? fma2(partner, s, y) : y;
}

// The sum over a head's lanes, in each of them.
template <int G>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = 1; o < G; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float dot8(const Eight &a, const Eight &b) {
    const F2 s = fma2(a.v[3], b.v[3], fma2(a.v[2], b.v[2], fma2(a.v[1], b.v[1], mul2(a.v[0], b.v[0]))));
    return s.x + s.y;
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

// The scale bytes of the two groups whose largest magnitudes are the halves of
// m, in the halves of a word.  bf16: exponent and mantissa are the same as f32's,
// so both at once; a group with an infinity or a NaN gets the largest one.
template <typename T, int F>
__device__ __forceinline__ uint32_t scale_bytes2(uint32_t m) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        constexpr uint32_t kBoth = 0x00010001u, kLead = Fmt<F>::kLead;
        const uint32_t b = (m + (Fmt<F>::kCarry >> 16) * kBoth) >> 7 & 0x01ff01ffu;
        return __vminu2(__vmaxu2(b, (kScaleLo + kLead) * kBoth),
                        (Fmt<F>::kScaleHi + kLead) * kBoth) - kLead * kBoth;
    } else {
        const int b0 = scale_byte<F>(f32_bits<T>(m & 0xffffu));
        const int b1 = scale_byte<F>(f32_bits<T>(m >> 16));
        return (uint32_t)b0 | (uint32_t)b1 << 16;
    }
}

// Keeps a head in 8 bits; codes and scales at the thread's first columns.
template <typename T, int G, int L, int A, int F>
__device__ __forceinline__ void keep_row(const QkParams &p, const Raw8<T> &raw, const Eight &x,
                                         uint8_t *codes, uint8_t *scales, int l, bool live) {
    if constexpr (L == kRun) {
        uint32_t m = amax_bits(raw);
        m = max_bits<T>(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max_bits<T>(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const int byte = scale_byte<F>(f32_bits<T>(m));
        if (!live || 8 * l >= pitch_of<G, A>(p)) return;
        *reinterpret_cast<uint2 *>(codes) = encode8<F>(values_of(x), byte);
        if (l % 4 == 0) *scales = (uint8_t)byte;
    } else {
        // two groups: of the first and of the second half
        int b0, b1;
        uint32_t lo, hi;  // their largest magnitudes, as f32 bits or as T's
        if constexpr (sizeof(T) == 4) {
            constexpr uint32_t kAbs = 0x7fffffffu;
            lo = max(max(raw.a.x & kAbs, raw.a.y & kAbs), max(raw.a.z & kAbs, raw.a.w & kAbs));
            hi = max(max(raw.b.x & kAbs, raw.b.y & kAbs), max(raw.b.z & kAbs, raw.b.w & kAbs));
#pragma unroll
            for (int o = 1; o < 8; o *= 2) {
                lo = max(lo, __shfl_xor_sync(0xffffffffu, lo, o));
                hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
            }
            b0 = scale_byte<F>(lo), b1 = scale_byte<F>(hi);
        } else {
            // both magnitudes, 16 bits each, through one shuffle
            constexpr uint32_t kAbs = 0x7fff7fffu;
            const uint32_t a = __vmaxu2(raw.a.x & kAbs, raw.a.y & kAbs);
            const uint32_t b = __vmaxu2(raw.a.z & kAbs, raw.a.w & kAbs);
            uint32_t m = __vmaxu2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
#pragma unroll
            for (int o = 1; o < 8; o *= 2) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
            lo = m & 0xffffu, hi = m >> 16;
            const uint32_t bytes = scale_bytes2<T, F>(m);
            b0 = bytes & 0xffffu, b1 = bytes >> 16;
        }
        if (!live) return;
        uint32_t c0, c1;
        if (max(b0, b1) < Fmt<F>::kScaleHi) {
            c0 = encode4_inside<F>(x.v[0].x, x.v[0].y, x.v[1].x, x.v[1].y, b0);
            c1 = encode4_inside<F>(x.v[2].x, x.v[2].y, x.v[3].x, x.v[3].y, b1);
        } else {
            b0 = scale_byte<F>(f32_bits<T>(lo)), b1 = scale_byte<F>(f32_bits<T>(hi));
            c0 = encode4<F>(x.v[0].x, x.v[0].y, x.v[1].x, x.v[1].y, b0);
            c1 = encode4<F>(x.v[2].x, x.v[2].y, x.v[3].x, x.v[3].y, b1);
        }
        *reinterpret_cast<uint32_t *>(codes) = c0;
        *reinterpret_cast<uint32_t *>(codes + 4 * G) = c1;
        if (l % 8 == 0) {
            scales[0] = (uint8_t)b0;
            scales[G / 8] = (uint8_t)b1;
        }
    }
}

// A task is one token and a run of its query or key heads; a warp takes it, G
// lanes a head with 8 elements a lane, 32 / G heads at once, the next ones on
// their way.  With the weights in them, the token's cosines and sines make y =
// r (x c + partner s) with 16 coefficients, kept in registers over the task.
// Bound by HBM and by issuing its instructions: x is read once, y (and the codes)
// written once (8192 tokens of 64 + 8 heads of 128: bf16 73.7 us, 77% of HBM's
// rate; 4096 in f32 58.8 us, 87%).  64 registers and 32 warps an SM: with 80 and
// 24 warps it took 10 us more, at that size.  kRun's 16-bit kernels spill a little
// so: 40 to 52 bytes in f16, 4 to 28 in bf16.
template <typename T, int G, int L, int A>
__global__ void __launch_bounds__(kQkThreads, sizeof(T) == 4 ? 3 : 4)
    qk_forward_kernel(const QkParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    constexpr int R = 32 / G;
    __shared__ float4 rows[L == kSplit ? 1 : kQkThreads * 2];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, l = lane % G, sub = lane / G;
    float *row = reinterpret_cast<float *>(rows) + (L == kSplit ? 0 : warp * 256);
    int64_t task = blockIdx.x * (int64_t)kQkWarps + warp;
    const int k = task >= p.tasks[0];
    if (k) task -= p.tasks[0];
    if (task >= p.tasks[k]) return;
    const int64_t token = task / p.n_chunk[k];
    const int h0 = (int)(task - token * p.n_chunk[k]) * p.chunk[k];
    const int h1 = min(h0 + p.chunk[k], p.heads[k]);
    const Place at = place_of(p, token);
    const int64_t row0 = token * p.heads[k] + h0 + sub;
    const int pitch = pitch_of<G, A>(p), spitch = spitch_of<G, A>(p);
    // all at the thread's first element
    const T *x = static_cast<const T *>(p.a[k].p) + token * p.a[k].token +
                 (h0 + sub) * p.a[k].head + first_of<L>(l);
    T *y = static_cast<T *>(p.b[k].p) + token * p.b[k].token + (h0 + sub) * p.b[k].head +
           first_of<L>(l);
    const bool keep = p.codes[k] != nullptr;
    uint8_t *codes = p.codes[k] + row0 * pitch + first_of<L>(l);
    uint8_t *scales = p.scales[k] + row0 * spitch + first_of<L>(l) / kGroup;
    float *rstd = p.rstd[k] && l == 0 ? p.rstd[k] + row0 : nullptr;
    Raw8<T> next = load_row<T, G, L, A>(p, x, l, h0 + sub < h1);
    // y = r (x c + partner s): the weights go into c and s
    Eight c, s;
    const Eight w = load_weights<G, L, A>(p, p.w[k], l);
    if (!at.padding && !at.outside) {
        load_angles<G, L>(p, at.at, l, c, s);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) c.v[i] = both(1.f), s.v[i] = both(0.f);
    }
    const Eight w_partner = partners<G, L>(p, w, l, row);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        c.v[i] = mul2(c.v[i], w.v[i]);
        s.v[i] = mul2(s.v[i], w_partner.v[i]);
    }
    const float outside = at.outside ? __uint_as_float(0x7fffffffu) : 1.f;
    const int turning = p.half - 4 * l;
    for (int h = h0; h < h1; h += R) {
        const bool live = h + sub < h1;
        const Raw8<T> raw = next;
        x += R * p.a[k].head;
        next = load_row<T, G, L, A>(p, x, l, h + R + sub < h1);  // while this row is worked on
        const Eight v = pairs_of(to_float(raw));
        const float r = rsqrtf(fmaf(row_sum<G>(dot8(v, v)), p.inv_dim, p.eps));
        if (keep) {
            if (p.format == POS_CKPT_INT8)
                keep_row<T, G, L, A, POS_CKPT_INT8>(p, raw, v, codes, scales, l, live);
            else
                keep_row<T, G, L, A, POS_CKPT_E4M3>(p, raw, v, codes, scales, l, live);
            codes += R * pitch, scales += R * spitch;
        }
        if (rstd) {
            if (live) *rstd = r;
            rstd += R;
        }
        const Eight q = partners<G, L>(p, v, l, row);
        Eight o;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o.v[i] = mul2(turn<L>(v.v[i], c.v[i], q.v[i], s.v[i], i, turning), both(r * outside));
        Raw8<T> out = from_float<T>(values_of(o));
        if (at.padding) {
            zero_raw(out.a);
            if constexpr (sizeof(T) == 4) zero_raw(out.b);
        }
        store_row<T, G, L, A>(p, y, l, live, out);
        y += R * p.b[k].head;
    }
}

// The codes of a thread's elements and their scales times r, as n = x r.
template <int L, int F>
__device__ __forceinline__ Eight read_kept(uint2 code, int b0, int b1, float r) {
    const Vec8 v = decode8<F>(code, 1.f);
    const F2 s0 = both(scale_value(b0) * r), s1 = L == kSplit ? both(scale_value(b1) * r) : s0;
    return {{mul2({v.v[0], v.v[1]}, s0), mul2({v.v[2], v.v[3]}, s0), mul2({v.v[4], v.v[5]}, s1),
             mul2({v.v[6], v.v[7]}, s1)}};
}

// Asynchronous copies of 4, 8 or 16 bytes; zeros where `there` is false.
template <int N>
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src, bool there) {
    if constexpr (N == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
                     "r"(there ? 16 : 0)
                     : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(N),
                     "r"(there ? N : 0)
                     : "memory");
}

// What a warp holds of one step in shared memory (p.step_bytes): 256 elements of
// dy, as many codes or elements of x, and for each of its heads 16 bytes with up
// to 8 scale bytes and rstd.
template <typename T>
constexpr int kStepDy = 256 * (int)sizeof(T);
constexpr int kSteps = 4;

// A step is 32 / G query or key heads of one token, G lanes a head.  The
// steps of all tokens, the queries' and then the keys', are cut into as many
// equal runs as there are warps.
struct Run {
    int64_t at, end;
};
__device__ __forceinline__ Run run_of(const QkParams &p, int k) {
    const int64_t total = p.tokens * p.steps[k], warps = gridDim.x * (int64_t)kQkWarps;
    const int64_t w = blockIdx.x * (int64_t)kQkWarps + threadIdx.x / 32;
    const int64_t each = total / warps, more = total % warps;
    return {w * each + min(w, more), (w + 1) * each + min(w + 1, more)};
}

// A warp goes through its run, token by token.  kAligned, kFull: its rows are on
// their way to shared memory three steps ahead, which takes no registers (two rows
// prefetched in registers instead: 111 us for 8192 tokens of 64 + 8 heads of 128,
// bf16; so 78.7 us, 72% of HBM's rate, 86% from x).  Bound by issuing its instructions and
// by HBM: 16 warps an SM, since fewer than 128 registers spill.  dw is summed
// over a thread's rows in registers, over the block in shared memory, and
// written as one partial sum per block, which qk_dw_kernel adds up in order.
template <typename T, int G, int L, int A>
__global__ void __launch_bounds__(kQkThreads, 2)
    qk_backward_kernel(const QkParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    extern __shared__ float4 steps[];
    __shared__ float4 rows[kQkWarps * kQkMaxDim / 4];
    constexpr int R = 32 / G;
    const int warp = threadIdx.x / 32, l = threadIdx.x % G, sub = threadIdx.x % 32 / G;
    float *row = reinterpret_cast<float *>(rows) + warp * 256;
    const int bytes = p.step_bytes;
    const int turning = p.half - 4 * l;
    unsigned char *const mine = reinterpret_cast<unsigned char *>(steps) + warp * kSteps * bytes;
    for (int k = 0; k < 2; ++k) {
        const Eight w = load_weights<G, L, A>(p, p.w[k], l);
        const bool from_x = p.x[k].p != nullptr;
        Eight dw;
#pragma unroll
        for (int i = 0; i < 4; ++i) dw.v[i] = both(0.f);
        for (Run run = run_of(p, k); run.at < run.end;) {
            const int64_t token = run.at / p.steps[k];
            const int h0 = (int)(run.at - token * p.steps[k]) * R;
            const int h1 = (int)min((int64_t)p.heads[k], h0 + (run.end - run.at) * R);
            run.at = min(run.end, (token + 1) * p.steps[k]);
            const Place at = place_of(p, token);
            T *dx = static_cast<T *>(p.b[k].p) + token * p.b[k].token + (h0 + sub) * p.b[k].head +
                    first_of<L>(l);
            Raw8<T> zero;
            zero_raw(zero.a);
            if constexpr (sizeof(T) == 4) zero_raw(zero.b);
            // Padding: zeros, whatever its rows and the weights hold.  kAny does it at
            // every store: with this branch 4096 tokens of 72 heads of 128 at an odd
            // start take 129 us instead of 105.
            if (A != kAny && at.padding) {
                for (int h = h0; h < h1; h += R, dx += R * p.b[k].head)
                    store_row<T, G, L, A>(p, dx, l, h + sub < h1, zero);
                continue;
            }
            const int64_t row0 = token * p.heads[k] + h0 + sub;
            const T *dy = static_cast<const T *>(p.a[k].p) + token * p.a[k].token +
                          (h0 + sub) * p.a[k].head;
            const T *x = static_cast<const T *>(p.x[k].p) + token * p.x[k].token +
                         (h0 + sub) * p.x[k].head;
            const int pitch = pitch_of<G, A>(p), spitch = spitch_of<G, A>(p);
            const uint8_t *codes = p.codes[k] + row0 * pitch + 8 * l;
            const uint8_t *scales = p.scales[k] + row0 * spitch + (A == kAny ? l / 4 : 4 * l);
            const float *rstd = p.rstd[k] + row0;
            int ahead = h0 + sub, slot = 0;  // head and slot of the next copies
            dy += 8 * l, x += 8 * l;
            if constexpr (A != kAny) __syncwarp();  // the last token's rows have been read
            // (not kAny) starts the copies of one step, if there is one
            auto start = [&]() {
                const bool there = ahead < h1;
                if (ahead - sub < h1) {
                    const uint32_t to =
                        (uint32_t)__cvta_generic_to_shared(mine + slot * bytes);
                    const uint32_t el = 8 * (threadIdx.x % 32);
                    if (8 * l < dim_of<G, A>(p)) {
                        copy_async<16>(to + el * sizeof(T), dy, there);
                        if constexpr (sizeof(T) == 4) copy_async<16>(to + el * 4 + 16, dy + 4, there);
                        if (from_x) {
                            copy_async<16>(to + kStepDy<T> + el * sizeof(T), x, there);
                            if constexpr (sizeof(T) == 4)
                                copy_async<16>(to + kStepDy<T> + el * 4 + 16, x + 4, there);
                        } else {
                            copy_async<8>(to + kStepDy<T> + el, codes, there);
                        }
                    }
                    const uint32_t aux = to + bytes - 16 * R + sub * 16;
                    if (!from_x && 4 * l < spitch) copy_async<4>(aux + 4 * l, scales, there);
                    if (l == 2) copy_async<4>(aux + 8, rstd, there);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                dy += R * p.a[k].head, x += R * p.x[k].head;
                codes += R * pitch, scales += R * spitch, rstd += R;
                ahead += R;
                slot = slot + 1 == kSteps ? 0 : slot + 1;
            };
            if constexpr (A != kAny) {
#pragma unroll
                for (int i = 0; i < kSteps - 1; ++i) start();
            }
            Eight c, s;  // s with the sign of the transpose
#pragma unroll
            for (int i = 0; i < 4; ++i) c.v[i] = both(1.f), s.v[i] = both(0.f);
            if (!at.padding && !at.outside) load_angles<G, L>(p, at.at, l, c, s);
#pragma unroll
            for (int i = 0; i < 4; ++i) s.v[i] = {-s.v[i].x, -s.v[i].y};
            const float outside = at.outside ? __uint_as_float(0x7fffffffu) : 1.f;
            int at_slot = 0;
            for (int h = h0; h < h1; h += R) {
                Raw8<T> raw, raw_x;
                uint2 code = make_uint2(0u, 0u);
                int b0 = 0, b1 = 0;
                float r = 0.f;
                if constexpr (A != kAny) {
                    asm volatile("cp.async.wait_group %0;" ::"n"(kSteps - 2) : "memory");
                    __syncwarp();
                    const unsigned char *from = mine + at_slot * bytes;
                    const T *row_dy =
                        reinterpret_cast<const T *>(from) + sub * 8 * G + first_of<L>(l);
                    const unsigned char *aux = from + bytes - 16 * R + sub * 16;
                    raw = load_row<T, G, L, A>(p, row_dy, l, true);
                    r = *reinterpret_cast<const float *>(aux + 8);
                    if (from_x) {
                        raw_x = load_row<T, G, L, A>(p, row_dy + 256, l, true);
                    } else {
                        const unsigned char *row_code =
                            from + kStepDy<T> + sub * 8 * G + first_of<L>(l);
                        if (L == kSplit) {
                            code.x = *reinterpret_cast<const uint32_t *>(row_code);
                            code.y = *reinterpret_cast<const uint32_t *>(row_code + 4 * G);
                            b0 = aux[l / 8], b1 = aux[G / 8 + l / 8];
                        } else if (8 * l < dim_of<G, A>(p)) {
                            code = *reinterpret_cast<const uint2 *>(row_code);
                            b0 = aux[l / 4];
                        }
                    }
                    at_slot = at_slot + 1 == kSteps ? 0 : at_slot + 1;
                    start();
                } else {
                    const bool live = h + sub < h1 && !at.padding;
                    raw = load_row<T, G, L, A>(p, dy, l, live);
                    if (from_x) raw_x = load_row<T, G, L, A>(p, x, l, live);
                    if (live) {
                        r = *rstd;
                        if (!from_x && 8 * l < p.dim) {
                            code = *reinterpret_cast<const uint2 *>(codes);
                            b0 = *scales;
                        }
                    }
                    dy += R * p.a[k].head, x += R * p.x[k].head;
                    codes += R * pitch, scales += R * spitch, rstd += R;
                }
                r *= outside;
                const Eight v = pairs_of(to_float(raw));
                const Eight q = partners<G, L>(p, v, l, row);
                Eight n, hw;
                if (from_x) {
                    n = pairs_of(to_float(raw_x));
#pragma unroll
                    for (int i = 0; i < 4; ++i) n.v[i] = mul2(n.v[i], both(r));
                } else {
                    n = p.format == POS_CKPT_INT8 ? read_kept<L, POS_CKPT_INT8>(code, b0, b1, r)
                                                  : read_kept<L, POS_CKPT_E4M3>(code, b0, b1, r);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const F2 gi = turn<L>(v.v[i], c.v[i], q.v[i], s.v[i], i, turning);
                    dw.v[i] = fma2(gi, n.v[i], dw.v[i]);
                    hw.v[i] = mul2(gi, w.v[i]);
                }
                const F2 t = both(-r * (row_sum<G>(dot8(hw, n)) * p.inv_dim));
                Eight o;
#pragma unroll
                for (int i = 0; i < 4; ++i) o.v[i] = fma2(n.v[i], t, mul2(hw.v[i], both(r)));
                const Raw8<T> out = from_float<T>(values_of(o));
                store_row<T, G, L, A>(p, dx, l, h + sub < h1, A == kAny && at.padding ? zero : out);
                dx += R * p.b[k].head;
            }
        }
        if (!p.part) continue;
        // [warp][dim], the heads side by side in a warp first
        float *sum = reinterpret_cast<float *>(rows);
        const Vec8 f = values_of(dw);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v = f.v[e];
#pragma unroll
            for (int o = G; o < 32; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
            const int i = element<G, L>(l, e);
            if (sub == 0 && i < dim_of<G, A>(p)) sum[warp * kQkMaxDim + i] = v;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < p.dim; i += kQkThreads) {
            float v = 0.f;
            for (int q = 0; q < kQkWarps; ++q) v += sum[q * kQkMaxDim + i];
            p.part[blockIdx.x * (int64_t)(2 * p.dim) + k * p.dim + i] = v;
        }
        __syncthreads();
    }
}

// dw = dw_in + the blocks' partial sums: a block takes 8 columns, 32 threads a
// column a strided share of the partial sums each.  Small blocks find room
// beside the last ones of the kernel before.
constexpr int kDwCols = 8, kDwThreads = 32 * kDwCols;
__global__ void __launch_bounds__(kDwThreads) qk_dw_kernel(const float *part, int n_part, int cols,
                                                           const float *dw_in, float *dw) {
    grid_dep_wait();
    grid_dep_trigger();
    __shared__ float sum[kDwThreads / 32][kDwCols];
    const int c = threadIdx.x % kDwCols, i = blockIdx.x * kDwCols + c;
    float v = 0.f;
    if (i < cols)
#pragma unroll 5
        for (int b = threadIdx.x / kDwCols; b < n_part; b += 32) v += part[b * (int64_t)cols + i];
    v += __shfl_xor_sync(0xffffffffu, v, 8);
    v += __shfl_xor_sync(0xffffffffu, v, 16);
    if (threadIdx.x % 32 < kDwCols) sum[threadIdx.x / 32][c] = v;
    __syncthreads();
    if (threadIdx.x >= kDwCols || i >= cols) return;
    v = 0.f;
#pragma unroll
    for (int q = 0; q < kDwThreads / 32; ++q) v += sum[q][c];
    dw[i] = dw_in ? dw_in[i] + v : v;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
static bool aligned4(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

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
    if (!aligned4(q->w_q) || !aligned4(q->w_k) || !aligned4(q->cos) || !aligned4(q->sin) ||
        !aligned4(q->positions))
        return fail(POS_EINVAL, "q/k: misaligned weights, tables or positions");
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
        if (written &&
            rows_overlap(q->tokens, heads, q->dim, t[k].token_stride, t[k].head_stride))
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
    p.vectors = aligned16(q->cos) && aligned16(q->sin) && aligned16(q->w_q) && aligned16(q->w_k) &&
                q->dim % 4 == 0;
    p.eps = q->eps, p.inv_dim = 1.f / q->dim;
    return p;
}

// Lanes of a head: 8 elements a lane, a power of two, so that sums over a head are
// log2 of them shuffles in place; 10 of 16 hold a head of 80, the others are idle.
static int lanes_per_head(int dim) { return dim <= 64 ? 8 : dim <= 128 ? 16 : 32; }

// The kernel for a call: lanes of a head, layout, loads.
template <typename T, template <typename, int, int, int> class Kernel, int G>
static auto pick_layout(const QkParams &p, bool aligned) {
    if (!aligned) return Kernel<T, G, kRun, kAny>::fn();
    if (p.dim != 8 * G) return Kernel<T, G, kRun, kAligned>::fn();
    return p.pairing == POS_ROT_HALF && 2 * p.half == p.dim ? Kernel<T, G, kSplit, kFull>::fn()
                                                            : Kernel<T, G, kRun, kFull>::fn();
}
template <typename T, template <typename, int, int, int> class Kernel>
static auto pick(const QkParams &p, bool aligned) {
    const int g = lanes_per_head(p.dim);
    return g == 8    ? pick_layout<T, Kernel, 8>(p, aligned)
           : g == 16 ? pick_layout<T, Kernel, 16>(p, aligned)
                     : pick_layout<T, Kernel, 32>(p, aligned);
}
template <typename T, int G, int L, int A>
struct Forward {
    static auto fn() { return qk_forward_kernel<T, G, L, A>; }
};
template <typename T, int G, int L, int A>
struct Backward {
    static auto fn() { return qk_backward_kernel<T, G, L, A>; }
};

// Cuts a token's heads into tasks: as few as give `warps` of them (each reads the
// token's cosines and sines again), at least 32 / G heads a task.  One and a half
// times what the GPU holds at once: 1000 tokens of 72 heads of 128 take 10.1 us,
// with once 12.1; 4096 of them 39.0, with twice 39.5.  Three times in f32, whose
// tasks are longer, so that the last round leaves more of the GPU idle: 4096 tokens
// of 72 heads of 128 take 59.0 us, with one and a half 66.5; of 256 115.7 and 133.8;
// 5000 of 128 69.8 and 74.2.
static void cut_tasks(QkParams &p, int64_t warps) {
    const int R = 32 / lanes_per_head(p.dim);
    const int64_t least = p.tokens * ((p.heads[0] > 0) + (p.heads[1] > 0));
    const int64_t want = least ? (warps + least - 1) / least : 1;
    for (int k = 0; k < 2; ++k) {
        const int most = std::max(1, (p.heads[k] + R - 1) / R);
        const int n = (int)std::max<int64_t>(1, std::min<int64_t>(want, most));
        p.chunk[k] = ((most + n - 1) / n) * R;
        p.n_chunk[k] = std::max(1, (p.heads[k] + p.chunk[k] - 1) / p.chunk[k]);
        p.tasks[k] = p.heads[k] ? p.tokens * p.n_chunk[k] : 0;
    }
}

static void set_steps(QkParams &p) {
    const int heads = 32 / lanes_per_head(p.dim);
    for (int k = 0; k < 2; ++k) p.steps[k] = (p.heads[k] + heads - 1) / heads;
}
// Blocks: what the GPU holds at once, or fewer where there are fewer steps.
static int grid_of(const QkParams &p, int per_sm) {
    const int64_t steps = p.tokens * std::max(p.steps[0], p.steps[1]);
    return (int)std::min<int64_t>((steps + kQkWarps - 1) / kQkWarps,
                                  (int64_t)sm_count() * per_sm);
}

template <typename T>
static pos_status forward_of(QkParams &p, bool aligned, cudaStream_t s) {
    cut_tasks(p, (int64_t)sm_count() * (sizeof(T) == 4 ? 96 : 48));
    const int64_t grid = (p.tasks[0] + p.tasks[1] + kQkWarps - 1) / kQkWarps;
    if (grid > 0x7fffffffll) return fail(POS_EINVAL, "q/k: too many tokens");
    POS_CUDA(launch_dependent(pick<T, Forward>(p, aligned), (int)grid, kQkThreads, 0, s, p));
    return POS_OK;
}

template <typename T>
static pos_status backward_of(QkParams &p, bool aligned, const float *dw_in, float *dw,
                              cudaStream_t s) {
    set_steps(p);
    auto kern = pick<T, Backward>(p, aligned);
    p.step_bytes = kStepDy<T> + (p.x[0].p || p.x[1].p ? kStepDy<T> : 256) +
                   16 * (32 / lanes_per_head(p.dim));
    const int smem = aligned ? kQkWarps * kSteps * p.step_bytes : 0;
    POS_TRY(ensure_smem(reinterpret_cast<const void *>(kern), smem));
    int per_sm = 0;
    POS_TRY(blocks_per_sm(reinterpret_cast<const void *>(kern), kQkThreads, smem, &per_sm));
    const int grid = grid_of(p, std::min(per_sm, 8)), cols = 2 * p.dim;
    void *scratch = nullptr;
    if (dw && grid > 0) {
        cudaMemPool_t pool;
        POS_TRY(scratch_pool(&pool));
        POS_CUDA(cudaMallocFromPoolAsync(&scratch, (size_t)grid * cols * 4, pool, s));
        p.part = static_cast<float *>(scratch);
    }
    cudaError_t e = grid > 0 ? launch_dependent(kern, grid, kQkThreads, smem, s, p) : cudaSuccess;
    if (dw && e == cudaSuccess)
        e = launch_dependent(qk_dw_kernel, (cols + kDwCols - 1) / kDwCols, kDwThreads, 0, s,
                             (const float *)p.part,
                             grid, cols, dw_in, dw);
    const cudaError_t e2 = scratch ? cudaFreeAsync(scratch, s) : cudaSuccess;
    if (e == cudaSuccess) e = e2;
    return e == cudaSuccess ? POS_OK : cuda_fail(e, "q/k backward");
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
    return guarded([&]() -> pos_status {
        POS_TRY(check_qk(qk));
        POS_TRY(check_heads(qk, x, "x", false));
        POS_TRY(check_heads(qk, y, "y", true));
        if (!aligned4(rstd_q) || !aligned4(rstd_k)) return fail(POS_EINVAL, "q/k: misaligned rstd");
        QkParams p = make_params(qk);
        POS_TRY(set_ckpt(p, ckpt_q, ckpt_k));
        if (p.tokens == 0 || p.heads[0] + p.heads[1] == 0) return POS_OK;
        for (int k = 0; k < 2; ++k) {
            p.a[k] = {x[k].data, x[k].token_stride, x[k].head_stride};
            p.b[k] = {y[k].data, y[k].token_stride, y[k].head_stride};
        }
        p.rstd[0] = rstd_q, p.rstd[1] = rstd_k;
        const bool aligned = heads_aligned(qk, x) && heads_aligned(qk, y);
        const auto s = static_cast<cudaStream_t>(stream);
        switch (qk->dtype) {
            case POS_BF16: return forward_of<__nv_bfloat16>(p, aligned, s);
            case POS_F16: return forward_of<__half>(p, aligned, s);
            default: return forward_of<float>(p, aligned, s);
        }
    });
}

pos_status poseidon_qk_backward(const pos_qk *qk, const pos_heads *x, const void *ckpt_q,
                                const void *ckpt_k, const float *rstd_q, const float *rstd_k,
                                const pos_heads *dy, const pos_heads *dx, const float *d_dw_in,
                                float *d_dw, void *stream) {
    using namespace pos;
    return guarded([&]() -> pos_status {
        POS_TRY(check_qk(qk));
        if (x) POS_TRY(check_heads(qk, x, "x", false));
        POS_TRY(check_heads(qk, dy, "dy", false));
        POS_TRY(check_heads(qk, dx, "dx", true));
        QkParams p = make_params(qk);
        POS_TRY(set_ckpt(p, ckpt_q, ckpt_k));
        if (!aligned4(rstd_q) || !aligned4(rstd_k)) return fail(POS_EINVAL, "q/k: misaligned rstd");
        if (!aligned4(d_dw_in) || !aligned4(d_dw)) return fail(POS_EINVAL, "q/k: misaligned dw");
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
    });
}

}  // extern "C"
