// The dropout's mask (poseidon.h), shared by dropout.cu and norm.cu.
#pragma once
#include <cmath>

#include "layer_ops.cuh"

namespace pos {

constexpr int kDropRounds = 10;
struct DropParams {
    uint32_t key[2 * kDropRounds];  // of every round
    uint32_t threshold;        // of 65536; 0: everything is kept
    uint32_t below;            // threshold * 65536 - 1
    float factor;              // of what is kept
    uint64_t offset;
    const uint64_t *d_offset;  // may be NULL
};

// The counter's offset, the same for a whole call.
__device__ __forceinline__ uint64_t drop_offset(const DropParams &d) {
    return d.offset + (d.threshold && d.d_offset ? *d.d_offset : 0ull);
}

// Philox-4x32 of ten rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers:
// as easy as 1, 2, 3, 2011).  Two wide products and two three-way exclusive ors a
// round give 16 bits for each of 8 elements: five instructions an element, the
// rounds' keys being computed on the host.
__device__ __forceinline__ uint4 philox(const DropParams &d, uint64_t offset, uint32_t r,
                                        uint32_t j) {
    uint32_t c0 = j, c1 = r, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
#pragma unroll
    for (int i = 0; i < kDropRounds; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ d.key[2 * i], c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ d.key[2 * i + 1], c3 = (uint32_t)a;
    }
    return make_uint4(c0, c1, c2, c3);
}
// Whether element i of 8 is kept: its half word, moved to the top, is above `below`.
__device__ __forceinline__ bool kept(const DropParams &d, const uint32_t (&w)[4], int i) {
    return (i % 2 ? w[i / 2] : w[i / 2] << 16) > d.below;
}

// x of row r, columns 8 j .. 8 j + 7, with the dropout's factor or zeros (whatever
// a dropped element holds).
__device__ __forceinline__ void drop8(const DropParams &d, uint64_t offset, uint32_t r, uint32_t j,
                                      Vec8 &x) {
    const uint4 u = philox(d, offset, r, j);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x.v[i] = kept(d, w, i) ? x.v[i] * d.factor : 0.f;
}

// x = add + dropout(x), each with one rounding (a fused product and sum), so that
// whoever computes h in more bits and rounds it gets the same.
__device__ __forceinline__ void add_dropped8(const DropParams &d, uint64_t offset, uint32_t r,
                                             uint32_t j, Vec8 &x, const Vec8 &add) {
    if (d.threshold == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x.v[i] = __fadd_rn(add.v[i], x.v[i]);
        return;
    }
    const uint4 u = philox(d, offset, r, j);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const F2 y = fma2({x.v[i], x.v[i + 1]}, both(d.factor), {add.v[i], add.v[i + 1]});
        x.v[i] = kept(d, w, i) ? y.x : add.v[i];
        x.v[i + 1] = kept(d, w, i + 1) ? y.y : add.v[i + 1];
    }
}

inline pos_status make_drop(const pos_dropout &p, const char *what, DropParams *out) {
    if (!(p.p >= 0.f && p.p <= 1.f))
        return fail(POS_EINVAL, std::string(what) + ": p must be 0..1");
    if (reinterpret_cast<uintptr_t>(p.d_offset) % 8)
        return fail(POS_EINVAL, std::string(what) + ": misaligned d_offset");
    DropParams d = {};
    for (uint32_t i = 0; i < kDropRounds; ++i) {
        d.key[2 * i] = (uint32_t)p.seed + i * 0x9E3779B9u;
        d.key[2 * i + 1] = (uint32_t)(p.seed >> 32) + i * 0xBB67AE85u;
    }
    d.threshold = (uint32_t)std::nearbyint((double)p.p * 65536.);
    d.below = (d.threshold << 16) - 1u;  // (p = 1: 2^32 - 1)
    // (p = 1 keeps nothing, and the factor is not used)
    d.factor = d.threshold < 65536u ? (float)(65536. / (65536. - d.threshold)) : 0.f;
    d.offset = p.offset, d.d_offset = p.d_offset;
    *out = d;
    return POS_OK;
}

}  // namespace pos
