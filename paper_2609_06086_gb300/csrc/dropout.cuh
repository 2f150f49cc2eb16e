// The dropout's mask (poseidon.h), shared by dropout.cu and norm.cu.
#pragma once
#include <cmath>

#include "layer_ops.cuh"

namespace pos {

struct DropParams {
    uint32_t key0, key1;
    uint32_t threshold;        // of 65536; 0: everything is kept
    float factor;              // of what is kept
    uint64_t offset;
    const uint64_t *d_offset;  // may be NULL
};

// The counter's offset, the same for a whole call.
__device__ __forceinline__ uint64_t drop_offset(const DropParams &d) {
    return d.offset + (d.threshold && d.d_offset ? *d.d_offset : 0ull);
}

// Philox-4x32 of ten rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers:
// as easy as 1, 2, 3, 2011).  Two wide products and six bit operations a round
// give 16 bits for each of 8 elements: about ten instructions an element, less than
// HBM takes for them.
__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3,
                                        uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0, c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1, c3 = (uint32_t)a;
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// x of row r, columns 8 j .. 8 j + 7, with the dropout's factor or zeros (whatever
// a dropped element holds).
__device__ __forceinline__ void drop8(const DropParams &d, uint64_t offset, uint32_t r, uint32_t j,
                                      Vec8 &x) {
    const uint4 u = philox(j, r, (uint32_t)offset, (uint32_t)(offset >> 32), d.key0, d.key1);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
        x.v[i] = bits >= d.threshold ? x.v[i] * d.factor : 0.f;
    }
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
    const uint4 u = philox(j, r, (uint32_t)offset, (uint32_t)(offset >> 32), d.key0, d.key1);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
        x.v[i] = bits >= d.threshold ? __fmaf_rn(x.v[i], d.factor, add.v[i]) : add.v[i];
    }
}

inline pos_status make_drop(const pos_dropout &p, const char *what, DropParams *out) {
    if (!(p.p >= 0.f && p.p <= 1.f))
        return fail(POS_EINVAL, std::string(what) + ": p must be 0..1");
    if (reinterpret_cast<uintptr_t>(p.d_offset) % 8)
        return fail(POS_EINVAL, std::string(what) + ": misaligned d_offset");
    DropParams d = {};
    d.key0 = (uint32_t)p.seed, d.key1 = (uint32_t)(p.seed >> 32);
    d.threshold = (uint32_t)std::nearbyint((double)p.p * 65536.);
    // (p = 1 keeps nothing, and the factor is not used)
    d.factor = d.threshold < 65536u ? (float)(65536. / (65536. - d.threshold)) : 0.f;
    d.offset = p.offset, d.d_offset = p.d_offset;
    *out = d;
    return POS_OK;
}

}  // namespace pos
