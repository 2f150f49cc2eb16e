// poseidon_attn_backward (formulas: poseidon.h).
#include <cmath>

#include "attn.cuh"

namespace pos {

// Two kernels, so that every sum has one place and one order: the queries' gradients
// by blocks that go over the keys, the keys' and values' by blocks that go over the
// queries.  Scores and dP are computed in both, and P K for D (below): eight products instead
// of the five of a single pass, which would add up the queries' gradients across blocks.
constexpr int kSumGroups = 4;            // warpgroups of sums, a quarter of the columns each
constexpr int kCols = kTile / kSumGroups;  // columns of a tile that a thread takes
constexpr int kBackThreads = 128 * (kSumGroups + 1);  // and one of loads and products
// 4 * 104 + 64 = 480 = 5 * 96, what the block is launched with
constexpr int kBackRegs = 104, kBackIssueRegs = 64;
constexpr int kLoadWarp = 4 * kSumGroups, kIssueWarp = kLoadWarp + 1, kStatsWarp = kLoadWarp + 2;

// f16 holds probabilities of long rows and small gradients badly (below 2^-14 with
// fewer bits, below 2^-25 not at all).  There P is multiplied by 2^12 and dS by 2^k, k the
// same for a product's sums and as large as the rows' norms allow: dP and D are at most
// |dO| |v|, so |dS| <= 2 |dO| |v|, of which the largest (dO of the block's queries and v that
// they see for theirs, all of the sequence's under the key head for the keys') becomes 2^14
// to 2^15 for any values, and the smallest step of dS 2^-38 of it.
template <typename T>
struct Shift {
    static constexpr bool kOn = std::is_same<T, __half>::value;
    static constexpr float kProbs = kOn ? 12.f : 0.f;
    static constexpr float kUndoProbs = kOn ? 1.f / 4096.f : 1.f;
    float grads, undo;  // of dP - D, so that P (dP - D) has its factor; 2^-k
    // the largest |dO|^2 and |v|^2
    __device__ __forceinline__ Shift(float d_o, float v) : grads(1.f), undo(1.f) {
        if constexpr (kOn) {
            // e + 127, e the exponent of the product: e + 2 k is 26 or 27
            const uint32_t b = __float_as_uint(d_o * v) >> 23;
            const int k = b ? 77 - (int)((b + 1) / 2) : 0;
            grads = __uint_as_float((uint32_t)(127 + k - 12) << 23);
            undo = __uint_as_float((uint32_t)(127 - k) << 23);
        }
    }
    static __device__ __forceinline__ Shift of_keys(const AttnParams &p, const AttnUnit &u, int g) {
        if constexpr (!kOn) return Shift(0.f, 0.f);
        const int64_t at = (int64_t)u.sequence * p.heads_k + g;
        return Shift(__uint_as_float(p.largest[at]), p.most[at]);
    }
};

// f16: the largest |v|^2 of every tile and key head, rows that are not finite apart, and the
// zeros that the queries' kernel starts from.
template <typename T>
__global__ void __launch_bounds__(kTile) attn_values_kernel(const AttnParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    __shared__ uint32_t warps[kTile / 32];
    const int64_t units =
        (int64_t)(p.tiles ? *p.n_tiles : ((int)p.tokens + kTile - 1) / kTile) * p.heads_k;
    for (int64_t i = blockIdx.x; i < units; i += gridDim.x) {
        AttnUnit u;
        unit_at<kTile>(p, (int)(i / p.heads_k), u);
        const int g = (int)(i % p.heads_k), row = u.tile * kTile + (int)threadIdx.x;
        float sum = 0.f;
        if (row < u.len) {
            const T *v = row_at<T>(p.v, u.start + (int64_t)row, g);
#pragma unroll 4
            for (int d = 0; d < p.dim; d += 8) {
                const Vec8 x = load_row8(v + d);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += x.v[e] * x.v[e];
            }
        }
        const uint32_t most =
            __reduce_max_sync(0xffffffffu, finite(sum) ? __float_as_uint(sum) : 0u);
        if (threadIdx.x % 32 == 0) warps[threadIdx.x / 32] = most;
        __syncthreads();
        if (threadIdx.x == 0) {
            p.values[g * p.tokens + u.start + (int64_t)u.tile * kTile] =
                __uint_as_float(max(max(warps[0], warps[1]), max(warps[2], warps[3])));
            if (u.tile == 0) p.largest[(int64_t)u.sequence * p.heads_k + g] = 0;
        }
        __syncthreads();
    }
}

// Of the queries of a tile, by the 16 warps of sums: lse in powers of two (less the
// probabilities' factor) and do . o, 16 lanes a row; f16: bits of the largest |dO|^2 of the
// rows that are finite, in *largest.
template <typename T>
__device__ __forceinline__ void row_stats(const AttnParams &p, const AttnUnit &u, int head,
                                          float2 *stats, uint32_t *largest) {
    const int l = threadIdx.x % 16;
    uint32_t big = 0;
    Vec8 a[4], b[4];
    float lse[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = threadIdx.x / 16 + 32 * k, row = u.tile * kTile + r;
        const int64_t token = u.start + (int64_t)row;
        const bool there = row < u.len && 8 * l < p.dim;
        // (o may lie anywhere; past its last element dO's copy holds zeros)
        a[k] = to_float(load8_shifted(row_at<T>(p.o, token, head) + 8 * l, 8 * l,
                                      there ? p.dim_out - 8 * l : 0));
        b[k] = there ? load_row8(row_at<T>(p.g, token, head) + 8 * l) : Vec8{};
        lse[k] = row < u.len ? p.lse[head * p.tokens + token] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float d = 0.f, size = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            d += a[k].v[e] * b[k].v[e];
            if (Shift<T>::kOn) size += b[k].v[e] * b[k].v[e];
        }
#pragma unroll
        for (int o = 8; o; o /= 2) {
            d += __shfl_xor_sync(0xffffffffu, d, o);
            if (Shift<T>::kOn) size += __shfl_xor_sync(0xffffffffu, size, o);
        }
        if (Shift<T>::kOn && finite(size)) big = max(big, __float_as_uint(size));
        if (l == 0)
            stats[threadIdx.x / 16 + 32 * k] = make_float2(lse[k] * kLog2e - Shift<T>::kProbs, d);
    }
    if constexpr (Shift<T>::kOn) {
        big = __reduce_max_sync(0xffffffffu, big);
        if (threadIdx.x % 32 == 0 && big) atomicMax(largest, big);
    }
}

// The first tile's queries, whose rows are short, with its keys: their P and dS go into the
// products as two 16-bit values each, so that only the results are rounded.  (Rounded once, they
// add as much to the error as the results' own rounding does, 1.4 times that in all; in a
// few short rows it was up to 2.1.  8192 tokens of 32 + 8 heads of 128 in 80 sequences: both
// passes 436 us, with one value 417.)
__device__ __forceinline__ bool short_rows(const AttnUnit &u) { return u.tile == 0; }

__device__ __forceinline__ void sums_barrier() {  // of the warpgroups of sums
    asm volatile("barrier.sync 1, %0;" ::"n"(128 * kSumGroups) : "memory");
}

// ---------------------------------------------------------------------------
// Gradients of the queries
// ---------------------------------------------------------------------------
// A block takes 128 queries of a head and goes over the keys from the diagonal down.
// TMEM holds scores, dP = dO V^T and two sums, and is full: P takes the scores' place and
// dS = P (dP - D) that of dP, and while one of them is made, the tensor cores use up the
// other and compute what comes next in its place.
//   A block takes one such unit after another, so that the next one's first loads, scores
// and dP come while the last one ends.  Before a unit its warps
// compute D = dO . o while the first tiles are on their way (a kernel of its own took 16
// of 480 us for 4096 tokens of 32 heads of 128).
//   D has the rounding of o in it, in 16 bits, which for rows with few keys that
// count is larger than that of everything else (2 tokens of 2 heads of 64, bf16: dQ 0.7 %
// off, dK 1.2 %).  Its exact value is D + e, e = sum P (dP - D), which this kernel has
// when it is done; so it adds up P K beside dS K, and dQ = dS K - e P K.  The keys'
// gradients are then computed with D + e.
constexpr int kKeySlots = 3, kValueSlots = 2;
constexpr int kDqBars = 2 * (kKeySlots + kValueSlots) + 10;
// and the first row of each column whose key is not finite, of two units, halves
constexpr int kDqSmem = 1024 + (2 + kKeySlots + kValueSlots) * kTileBytes + 8 * kDqBars +
                        kSharedBytes + kTile * 8 + 4 * kAttnMaxDim;

template <typename T>
__global__ void __launch_bounds__(kBackThreads, 1)
    attn_dq_kernel(const __grid_constant__ CUtensorMap q_map,
                   const __grid_constant__ CUtensorMap k_map,
                   const __grid_constant__ CUtensorMap v_map,
                   const __grid_constant__ CUtensorMap g_map, const AttnParams p) {
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char *aligned = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t q_at = base, g_at = q_at + kTileBytes, k_at = g_at + kTileBytes;
    const uint32_t v_at = k_at + kKeySlots * kTileBytes;
    const uint32_t bars = v_at + kValueSlots * kTileBytes;
    const uint32_t k_full = bars, k_empty = k_full + 8 * kKeySlots;
    const uint32_t v_full = k_empty + 8 * kKeySlots, v_empty = v_full + 8 * kValueSlots;
    const uint32_t in_full = v_empty + 8 * kValueSlots, s_full = in_full + 8, dp_full = s_full + 8;
    const uint32_t p_full = dp_full + 8, ds_full = p_full + 8, dq_full = ds_full + 8;
    const uint32_t in_empty = dq_full + 8, bad_full = in_empty + 8, k_in = bad_full + 16;
    const uint32_t slot = k_in + 8;
    AttnShared *sh = reinterpret_cast<AttnShared *>(aligned + (slot - base));
    // rows' statistics, and the parts of e
    float2 *stats = reinterpret_cast<float2 *>(aligned + (slot - base) + kSharedBytes);
    uint8_t *first_bad = aligned + (slot - base) + kSharedBytes + kTile * 8;
    const Waits waits(sh, p);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, group = warp / 4;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kDqBars; ++i) {
            const uint32_t b = bars + 8 * i;
            bar_init(b, b == p_full || b == ds_full          ? 4 * kSumGroups
                        : b == bad_full || b == bad_full + 8 ? 2
                                                             : 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        init_shared(sh);
    }
    if (warp == kIssueWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot),
                     "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        tmem_before();
    }
    __syncthreads();
    tmem_after();
    grid_dep_wait();
    grid_dep_trigger();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(&sh->tmem);
    const uint32_t dp_tm = tmem + kTile, pk_tm = tmem + 2 * kTile, dq_tm = tmem + 3 * kTile;

    const int boxes = p.dim > 64 ? 2 : 1;
    BlockUnit<kTile> w;
    int round = 0;
    bool ok = true;

    if (group == kSumGroups) {
        give_registers<kBackIssueRegs>();
        if (warp == kLoadWarp) {
            int sk = 0, sv = 0;
            uint32_t phk = 1, phv = 1, ph = 1;
            while (lane == 0 && ok && w.next(p, round)) {
                const int n = w.u.tile + 1;  // tiles of keys
                const auto load = [&](uint32_t full, uint32_t empty, uint32_t at,
                                      const CUtensorMap *map, int &s, uint32_t &ph, int slots,
                                      int j) {
                    if (!attn_wait(empty + 8 * s, ph, waits)) return false;
                    bar_expect(full + 8 * s, boxes * kBox);
                    for (int b = 0; b < boxes; ++b)
                        tma_rows(at + s * kTileBytes + b * kBox, map, 64 * b, w.head / p.group,
                                 w.u.start + j * kTile, full + 8 * s);
                    if (++s == slots) s = 0, ph ^= 1;
                    return true;
                };
                // keys a step ahead of values
                for (int i = 0; i <= n && ok; ++i) {
                    if (i < n)
                        ok = load(k_full, k_empty, k_at, &k_map, sk, phk, kKeySlots, n - 1 - i);
                    if (i == 0 && ok) {
                        ok = attn_wait(in_empty, ph, waits);
                        if (!ok) break;
                        ph ^= 1;
                        bar_expect(in_full, 2 * boxes * kBox);
                        for (int b = 0; b < boxes; ++b) {
                            const int token = w.u.start + w.u.tile * kTile;
                            tma_rows(q_at + b * kBox, &q_map, 64 * b, w.head, token, in_full);
                            tma_rows(g_at + b * kBox, &g_map, 64 * b, w.head, token, in_full);
                        }
                    }
                    if (i > 0 && ok)
                        ok = load(v_full, v_empty, v_at, &v_map, sv, phv, kValueSlots, n - i);
                }
            }
        } else if (warp == kIssueWarp) {
            const uint32_t mine = one_lane();
            const int steps = (p.dim + 15) / 16;
            uint32_t ph = 0;
            int it = 0, units = 0;  // steps and units so far
            while (ok && w.next(p, round)) {
                const int n = w.u.tile + 1, base = it;
                const bool fine = short_rows(w.u);
                const auto scores = [&](int i) {
                    const int at_i = base + i, slot_i = at_i % kKeySlots;
                    if (!wait_warp(k_full + 8 * slot_i, at_i / kKeySlots & 1, waits)) return false;
                    const uint32_t at = k_at + slot_i * kTileBytes;
                    mma_rows<T>(tmem, q_at, at, steps, mine);
                    commit(s_full, mine);
                    if (i == 0) commit(k_in, mine);  // on the diagonal: the scores see it as it is
                    return true;
                };
                const auto grads = [&](int i) {  // dP
                    const int at_i = base + i, slot_i = at_i % kValueSlots;
                    if (!wait_warp(v_full + 8 * slot_i, at_i / kValueSlots & 1, waits))
                        return false;
                    mma_rows<T>(dp_tm, g_at, v_at + slot_i * kTileBytes, steps, mine);
                    commit(dp_full, mine);
                    commit(v_empty + 8 * slot_i, mine);
                    if (i == n - 1) commit(in_empty, mine);  // the last ones
                    return true;
                };
                ok = wait_warp(in_full, ph, waits);
                ph ^= 1;
                tmem_after();
                ok = ok && scores(0) && grads(0);
                for (int i = 0; i < n && ok; ++i, ++it) {
                    const uint32_t at = k_at + it % kKeySlots * kTileBytes;
                    ok = wait_warp(p_full, it & 1, waits) &&
                         (i > 0 || wait_warp(bad_full + 8 * (units & 1), units >> 1 & 1, waits));
                    if (!ok) break;
                    tmem_after();
                    // (the unit before has been read: its warps have gone on to this one)
                    mma_columns<T, kCols>(pk_tm, tmem, at, steps, i > 0, mine);
                    if (fine) mma_columns<T, kCols>(pk_tm, tmem + kCols / 2, at, steps, true, mine);
                    if (i + 1 < n) ok = scores(i + 1);
                    ok = ok && wait_warp(ds_full, it & 1, waits);
                    if (!ok) break;
                    tmem_after();
                    mma_columns<T, kCols>(dq_tm, dp_tm, at, steps, i > 0, mine);
                    if (fine) mma_columns<T, kCols>(dq_tm, dp_tm + kCols / 2, at, steps, true, mine);
                    commit(k_empty + 8 * (it % kKeySlots), mine);
                    if (i == n - 1) commit(dq_full, mine);
                    else ok = grads(i + 1);
                }
                ++units;
            }
        } else {
            // two warps look over half of the diagonal's keys each
            const int half = warp - kIssueWarp - 1;
            int it = 0, units = 0;
            while (ok && w.next(p, round)) {
                ok = wait_warp(k_in, units & 1, waits);
                if (!ok) break;
                const uint32_t at = k_at + it % kKeySlots * kTileBytes;
                const int seen = min(kTile, w.u.len - w.u.tile * kTile);
                const int from = half * (kTile / 2), end = min(seen, from + kTile / 2);
                const bool bad = tile_bad<T>(at, from, end, boxes, lane);
                if (bad) {
                    uint8_t *first = first_bad + (2 * (units & 1) + half) * kAttnMaxDim;
                    for (int c = lane; c < kAttnMaxDim; c += 32) first[c] = kTile;
                    tile_clean<T>(at, from, end, boxes, lane,
                                  [&](int c, int row, int) { first[c] = (uint8_t)row; });
                }
                zero_rows(at, max(from, seen), from + kTile / 2, boxes, lane);
                if (lane == 0) sh->bad[units & 1][0][half] = bad;
                tile_done();
                if (lane == 0) bar_arrive(bad_full + 8 * (units & 1));
                it += w.u.tile + 1, ++units;
            }
        }
        __syncwarp();
    } else {
        take_registers<kBackRegs>();
        const int side = group, mine = warp % 4 * 32 + lane;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const uint32_t s_tm = tmem + kCols * side + lanes, d_tm = dp_tm + kCols * side + lanes;
        int it = 0, units = 0;
        // The warps meet at barriers, so they end together, whether a wait of one gave up or not.
        for (; w.next(p, round); ++units) {
            const AttnUnit &u = w.u;
            const int n = u.tile + 1, head = w.head, row = u.tile * kTile + mine;
            const bool live = row < u.len, fine = short_rows(u);
            // the largest |v|^2 that the queries see (the first load while others are)
            const float *v_at =
                Shift<T>::kOn ? p.values + head / p.group * p.tokens + u.start : nullptr;
            float values = Shift<T>::kOn && lane < n ? v_at[(int64_t)lane * kTile] : 0.f;
            row_stats<T>(p, u, head, stats, sh->largest + units % 2);
            sums_barrier();
            const float2 st = stats[mine];
            const uint32_t big = sh->largest[units % 2];
            if constexpr (Shift<T>::kOn) {
                for (int i = lane + 32; i < n; i += 32)
                    values = fmaxf(values, v_at[(int64_t)i * kTile]);
                values = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(values)));
            }
            const Shift<T> shift(__uint_as_float(big), values);
            if (Shift<T>::kOn && threadIdx.x == 0) {
                const int64_t at = (int64_t)u.sequence * p.heads_k + head / p.group;
                if (big) atomicMax(p.largest + at, big);
                // (by every head of the group, the same)
                if (n * kTile >= u.len) p.most[at] = values;
                sh->largest[(units + 1) % 2] = 0;
            }
            F2 rest = both(0.f);  // e, of this part of the columns
            for (int i = 0; i < n; ++i, ++it) {
                ok = ok && wait_warp(s_full, it & 1, waits);
                if (!ok) break;
                tmem_after();
                uint32_t s[kCols], d[kCols], w[kCols / 2];
                // the last key of this part that the row sees; a row that sees one has dS = 0
                const int seen = row - (n - 1) * kTile - kCols * side;
                tmem_load32(s_tm, s);
#pragma unroll
                for (int c = 0; c < kCols; c += 2) {
                    const F2 x = fma2({__uint_as_float(s[c]), __uint_as_float(s[c + 1])},
                                      both(p.scale2), both(-st.x));
                    s[c] = __float_as_uint(exp2_fast(x.x));
                    s[c + 1] = __float_as_uint(exp2_fast(x.y));
                }
                if (i == 0) {
#pragma unroll
                    for (int c = 0; c < kCols; ++c)
                        if (c > seen) s[c] = 0;
                }
#pragma unroll
                for (int c = 0; c < kCols; c += 2)
                    w[c / 2] = pack2<T>(__uint_as_float(s[c]), __uint_as_float(s[c + 1]));
                tmem_store16(s_tm, w);
                if (fine) {
#pragma unroll
                    for (int c = 0; c < kCols; c += 2)
                        w[c / 2] = pack2_rest<T>(w[c / 2], __uint_as_float(s[c]),
                                                 __uint_as_float(s[c + 1]));
                    tmem_store16(s_tm + kCols / 2, w);
                }
                tmem_wait_stores();
                tmem_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_full);
                ok = wait_warp(dp_full, it & 1, waits);
                if (!ok) break;
                tmem_after();
                tmem_load32(d_tm, d);
#pragma unroll
                for (int c = 0; c < kCols; c += 2) {
                    const F2 e = fma2({__uint_as_float(d[c]), __uint_as_float(d[c + 1])},
                                      both(shift.grads), both(-st.y * shift.grads));
                    const F2 v = mul2({__uint_as_float(s[c]), __uint_as_float(s[c + 1])}, e);
                    d[c] = __float_as_uint(v.x), d[c + 1] = __float_as_uint(v.y);
                }
                if (i == 0) {
#pragma unroll
                    for (int c = 0; c < kCols; ++c)
                        if (c > seen || row == 0) d[c] = 0;
                }
#pragma unroll
                for (int c = 0; c < kCols; c += 2) {
                    rest = add2(rest, {__uint_as_float(d[c]), __uint_as_float(d[c + 1])});
                    w[c / 2] = pack2<T>(__uint_as_float(d[c]), __uint_as_float(d[c + 1]));
                }
                tmem_store16(d_tm, w);
                if (fine) {
#pragma unroll
                    for (int c = 0; c < kCols; c += 2)
                        w[c / 2] = pack2_rest<T>(w[c / 2], __uint_as_float(d[c]),
                                                 __uint_as_float(d[c + 1]));
                    tmem_store16(d_tm + kCols / 2, w);
                }
                tmem_wait_stores();
                tmem_before();
                __syncwarp();
                if (lane == 0) bar_arrive(ds_full);
            }
            if (ok)
                ok = wait_warp(dq_full, units & 1, waits) &&
                     wait_warp(bad_full + 8 * (units & 1), units >> 1 & 1, waits);
            tmem_after();
            // e's parts through the place of the stats, which every warp has read
            float *parts = reinterpret_cast<float *>(stats);
            float e = ok ? rest.x + rest.y : __uint_as_float(0x7fffffffu);  // (no result)
            if (side >= 2) parts[(side - 2) * kTile + mine] = e;
            sums_barrier();
            if (side < 2) parts[side * kTile + mine] += e;
            sums_barrier();
            e = (parts[mine] + parts[kTile + mine]) * shift.undo;
            if (live && side == 0)
                p.stats[head * p.tokens + u.start + row] = make_float2(st.x, st.y + e);
            const float a = ok ? p.scale * shift.undo : __uint_as_float(0x7fffffffu);
            const float b = -e * p.scale * Shift<T>::kUndoProbs;
            T *out = static_cast<T *>(p.dq) + (u.start + (int64_t)row) * p.d_token[0] +
                     head * p.d_head[0];
            // halves of the tile's keys that hold some that are not finite: rows that see them
            const int bad = sh->bad[units & 1][0][0] + 2 * sh->bad[units & 1][0][1];
            const auto mark = [&](int c, uint32_t *v) {
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    if (bad >> half & 1) {
                        const uint8_t *first =
                            first_bad + (2 * (units & 1) + half) * kAttnMaxDim + c;
#pragma unroll
                        for (int h = 0; h < 16; ++h)
                            if (mine >= first[h]) v[h] = 0x7fffffffu;
                    }
            };
            const auto write = [&](bool check) {
                for (int c = 16 * side; c < p.dim; c += 16 * kSumGroups) {
                    uint32_t v[16], k[16];
                    tmem_load16(dq_tm + lanes + c, v);
                    tmem_load16(pk_tm + lanes + c, k);
                    if (check) mark(c, v);
                    Vec8 x[2];
#pragma unroll
                    for (int h = 0; h < 16; ++h)
                        x[h / 8].v[h % 8] = __uint_as_float(v[h]) * a + __uint_as_float(k[h]) * b;
                    if (!live) continue;
#pragma unroll
                    for (int h = 0; h < 16; h += 8) {
                        if (p.d_vectors[0])
                            store8<true>(out + c + h, from_float<T>(x[h / 8]), p.dim_out - c - h);
                        else store8<false>(out + c + h, from_float<T>(x[h / 8]), p.dim_out - c - h);
                    }
                }
            };
            if (bad) write(true);  // (a copy of its own)
            else write(false);
            sums_barrier();
        }
    }
    end_block(sh);
    if (warp == kIssueWarp) {
        tmem_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
    }
}

// ---------------------------------------------------------------------------
// Gradients of the keys and values
// ---------------------------------------------------------------------------
// A block takes 128 keys of a key head and goes over the queries that see them, one
// query head of the group after another.  Everything is transposed: a thread's row is
// a key, so P and dS are the products' first operands as they stand in TMEM.  TMEM holds
// scores, dP, and both sums, and is full: P takes the scores' place and dS that of dP,
// and while one of them is made, the tensor cores use up the other and compute what
// comes next in its place.
//   Up to eight blocks share 128 keys where the most steps of one block would outlast the
// others: each takes a run of the steps and puts its sums in memory, and attn_join_kernel
// adds them up in order.  (As a cluster that adds them up through its blocks' shared
// memory, 8 microseconds more for a pair.)
constexpr int kQuerySlots = 2;
constexpr int kStatBytes = kTile * 8;
constexpr int kDkvBars = 8 * kQuerySlots + 6;
constexpr int kDkvSmem = 1024 + (2 + 2 * kQuerySlots) * kTileBytes + kQuerySlots * kStatBytes +
                         8 * kDkvBars + kSharedBytes + kAttnMaxDim;

__device__ __forceinline__ F2 load_stats(uint32_t at) {
    F2 l;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(l.x), "=f"(l.y) : "r"(at));
    return l;
}

// Where the sums of a part of a block's steps go: [tensor][16 columns][4 columns][128 keys][4].
__device__ __forceinline__ float4 *part_at(const AttnParams &p, int part, int t, int c, int key) {
    const int dim16 = (p.dim + 15) / 16 * 16;
    return reinterpret_cast<float4 *>(p.part) +
           (((int64_t)part * 2 + t) * dim16 + c) * (kTile / 4) + key;
}
// The key tile's number, steps of all heads and those of one part of them.
struct KeySteps {
    int each, first, n;  // steps of a head; the part's first, and how many it has
    __device__ __forceinline__ KeySteps(const AttnParams &p, AttnUnit &u, int part) {
        // the list is in the order of a query tile's keys; of a key tile's queries it is this
        const int tiles = (u.len + kTile - 1) / kTile;
        u.tile = tiles - 1 - u.tile;
        each = tiles - u.tile;
        first = (int)((int64_t)each * p.group * part / p.parts);
        n = (int)((int64_t)each * p.group * (part + 1) / p.parts) - first;
    }
};

template <typename T>
__global__ void __launch_bounds__(kBackThreads, 1)
    attn_dkv_kernel(const __grid_constant__ CUtensorMap q_map,
                    const __grid_constant__ CUtensorMap k_map,
                    const __grid_constant__ CUtensorMap v_map,
                    const __grid_constant__ CUtensorMap g_map, const AttnParams p) {
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char *aligned = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t k_at = base, v_at = k_at + kTileBytes, q_at = v_at + kTileBytes;
    const uint32_t g_at = q_at + kQuerySlots * kTileBytes;
    const uint32_t st_at = g_at + kQuerySlots * kTileBytes;
    const uint32_t bars = st_at + kQuerySlots * kStatBytes;
    const uint32_t q_full = bars, q_empty = q_full + 8 * kQuerySlots;
    const uint32_t g_full = q_empty + 8 * kQuerySlots, g_empty = g_full + 8 * kQuerySlots;
    const uint32_t st_full = g_empty + 8 * kQuerySlots, st_empty = st_full + 8 * kQuerySlots;
    const uint32_t in_full = st_empty + 8 * kQuerySlots, s_full = in_full + 8, dp_full = s_full + 8;
    const uint32_t p_full = dp_full + 8, ds_full = p_full + 8, out_full = ds_full + 8;
    const uint32_t q_clean = out_full + 8, g_clean = q_clean + 8 * kQuerySlots;
    const uint32_t slot = g_clean + 8 * kQuerySlots;
    AttnShared *sh = reinterpret_cast<AttnShared *>(aligned + (slot - base));
    // behind the last query of the diagonal's whose dO is not finite, of each column
    uint8_t *last_bad = aligned + (slot - base) + kSharedBytes;
    const Waits waits(sh, p);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, group = warp / 4;

    // A block that starts when others have ended, and has no tile, ends at once.
    if (blockIdx.x >= p.first_blocks) {
        grid_dep_wait();
        if (blockIdx.x / p.parts / p.heads_k >= *p.n_tiles) return;
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < kDkvBars; ++i) {
            const uint32_t b = bars + 8 * i;
            bar_init(b, b == p_full || b == ds_full || (b >= st_empty && b < in_full)
                            ? 4 * kSumGroups
                            : 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        init_shared(sh);
        for (int i = 0; i < kAttnMaxDim; ++i) last_bad[i] = 0;
    }
    if (warp == kIssueWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot),
                     "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        tmem_before();
    }
    __syncthreads();
    tmem_after();
    grid_dep_wait();
    grid_dep_trigger();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(&sh->tmem);
    const uint32_t dp_tm = tmem + kTile, dv_tm = tmem + 2 * kTile, dk_tm = tmem + 3 * kTile;

    const int unit = blockIdx.x / p.parts, part = blockIdx.x % p.parts, g = unit % p.heads_k;
    AttnUnit u;
    int each = 0, step0 = 0, n = 0;  // this block's steps: from step0 on, n of them
    if (unit_at<kTile>(p, unit / p.heads_k, u)) {
        const KeySteps steps(p, u, part);
        each = steps.each, step0 = steps.first, n = steps.n;
    }
    const int boxes = p.dim > 64 ? 2 : 1;
    bool ok = true;
    // The i-th step's tile of queries (0) or dO (1): on the diagonal it is looked over; what
    // is behind the sequence becomes zeros.
    const auto look = [&](int i, int t) {
        const int s = i % kQuerySlots, tile = (step0 + i) % each;
        if (!wait_warp((t ? g_full : q_full) + 8 * s, i / kQuerySlots & 1, waits)) return false;
        const uint32_t at = (t ? g_at : q_at) + s * kTileBytes;
        const int seen = min(kTile, u.len - (u.tile + tile) * kTile);
        if (tile == 0 && tile_bad<T>(at, 0, seen, boxes, lane)) {
            if (lane == 0 && t) sh->bad[0][0][0] = 1;
            // (P and dS of a query that is not finite are not, by its lse or D)
            tile_clean<T>(at, 0, seen, boxes, lane, [&](int c, int, int last) {
                if (t) last_bad[c] = max(last_bad[c], (uint8_t)(last + 1));
            });
        }
        zero_rows(at, seen, kTile, boxes, lane);
        tile_done();
        if (lane == 0) bar_arrive((t ? g_clean : q_clean) + 8 * s);
        return true;
    };

    if (group == kSumGroups) {
        give_registers<kBackIssueRegs>();
        if (warp == kLoadWarp) {
            if (lane == 0 && n > 0) {
                bar_expect(in_full, 2 * boxes * kBox);
                for (int b = 0; b < boxes; ++b) {
                    const int token = u.start + u.tile * kTile;
                    tma_rows(k_at + b * kBox, &k_map, 64 * b, g, token, in_full);
                    tma_rows(v_at + b * kBox, &v_map, 64 * b, g, token, in_full);
                }
                int s = 0;
                uint32_t ph = 1;
                for (int i = 0; i < n && ok; ++i) {
                    const int head = g * p.group + (step0 + i) / each;
                    const int token = u.start + (u.tile + (step0 + i) % each) * kTile;
                    for (int w = 0; w < 2 && ok; ++w) {
                        const uint32_t full = (w ? g_full : q_full) + 8 * s;
                        ok = attn_wait((w ? g_empty : q_empty) + 8 * s, ph, waits);
                        if (!ok) break;
                        bar_expect(full, boxes * kBox);
                        for (int b = 0; b < boxes; ++b)
                            tma_rows((w ? g_at : q_at) + s * kTileBytes + b * kBox,
                                     w ? &g_map : &q_map, 64 * b, head, token, full);
                    }
                    if (++s == kQuerySlots) s = 0, ph ^= 1;
                }
            }
        } else if (warp == kIssueWarp) {
            const uint32_t mine = one_lane();
            const int steps = (p.dim + 15) / 16;
            const auto arrived = [&](uint32_t clean, int i) {
                return wait_warp(clean + 8 * (i % kQuerySlots), i / kQuerySlots & 1, waits);
            };
            const auto scores = [&](int i) {
                if (!arrived(q_clean, i)) return false;
                mma_rows<T>(tmem, k_at, q_at + i % kQuerySlots * kTileBytes, steps, mine);
                commit(s_full, mine);
                return true;
            };
            const auto grads = [&](int i) {  // dP
                if (!arrived(g_clean, i)) return false;
                mma_rows<T>(dp_tm, v_at, g_at + i % kQuerySlots * kTileBytes, steps, mine);
                commit(dp_full, mine);
                return true;
            };
            if (n > 0) {
                ok = wait_warp(in_full, 0, waits);
                tmem_after();
                ok = ok && scores(0) && grads(0);
            }
            for (int i = 0; i < n && ok; ++i) {
                const int s = i % kQuerySlots;
                const bool fine = (step0 + i) % each == 0 && short_rows(u);
                ok = wait_warp(p_full, i & 1, waits);
                if (!ok) break;
                tmem_after();
                mma_columns<T, kCols>(dv_tm, tmem, g_at + s * kTileBytes, steps, i > 0, mine);
                if (fine)
                    mma_columns<T, kCols>(dv_tm, tmem + kCols / 2, g_at + s * kTileBytes, steps, true,
                                          mine);
                commit(g_empty + 8 * s, mine);
                if (i + 1 < n) ok = scores(i + 1);
                ok = ok && wait_warp(ds_full, i & 1, waits);
                if (!ok) break;
                tmem_after();
                mma_columns<T, kCols>(dk_tm, dp_tm, q_at + s * kTileBytes, steps, i > 0, mine);
                if (fine)
                    mma_columns<T, kCols>(dk_tm, dp_tm + kCols / 2, q_at + s * kTileBytes, steps, true,
                                          mine);
                commit(q_empty + 8 * s, mine);
                if (i == n - 1) commit(out_full, mine);
                if (i + 1 < n) ok = grads(i + 1);
            }
        } else if (warp == kStatsWarp) {
            // lse and D of the queries; none for rows past the sequence: their
            // probabilities are 2^(0 - inf) = 0
            const Shift<T> shift = n > 0 ? Shift<T>::of_keys(p, u, g) : Shift<T>(0.f, 0.f);
            float2 st[4];
            const auto fetch = [&](int i) {
                const int head = g * p.group + (step0 + i) / each;
                const int row = (u.tile + (step0 + i) % each) * kTile;
                const float2 *from = p.stats + head * p.tokens + u.start + row;
#pragma unroll
                for (int h = 0; h < 4; ++h)
                    st[h] = row + lane + 32 * h < u.len
                                ? from[lane + 32 * h]
                                : make_float2(__uint_as_float(0x7f800000u), 0.f);
            };
            if (n > 0) fetch(0);
            for (int i = 0; i < n && ok; ++i) {
                const int s = i % kQuerySlots;
                ok = wait_warp(st_empty + 8 * s, (i / kQuerySlots & 1) ^ 1, waits);
                if (!ok) break;
#pragma unroll
                for (int h = 0; h < 4; ++h)  // -lse in the first half, -D in the second
                    asm volatile("st.shared.f32 [%0], %1;\nst.shared.f32 [%0 + 512], %2;" ::"r"(
                                     st_at + s * kStatBytes + 4 * (lane + 32 * h)),
                                 "f"(-st[h].x), "f"(-st[h].y * shift.grads)
                                 : "memory");
                __syncwarp();
                if (lane == 0) bar_arrive(st_full + 8 * s);
                if (i + 1 < n) fetch(i + 1);
                ok = look(i, 1);
            }
        } else {
            for (int i = 0; i < n && ok; ++i) ok = look(i, 0);
        }
        __syncwarp();
    } else {
        take_registers<kBackRegs>();
        const Shift<T> shift = n > 0 ? Shift<T>::of_keys(p, u, g) : Shift<T>(0.f, 0.f);
        const int side = group, mine = warp % 4 * 32 + lane;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const uint32_t s_tm = tmem + kCols * side + lanes, d_tm = dp_tm + kCols * side + lanes;
        // A thread's 32 values are of four keys and eight queries (tmem_load_block), so that it
        // reads lse and D of eight queries and not of 32: shared memory is what bounds
        // this kernel (2786 cycles a tile of 128 x 128 with 32 of them)
        const int key = warp % 4 * 32 + lane / 4, query = kCols * side + lane % 4 * 2;
        for (int i = 0; i < n; ++i) {
            const int slot_i = i % kQuerySlots;
            const uint32_t st = st_at + slot_i * kStatBytes + 4 * query;
            ok = ok && wait_warp(st_full + 8 * slot_i, i / kQuerySlots & 1, waits) &&
                 wait_warp(s_full, i & 1, waits);
            if (!ok) break;
            tmem_after();
            uint32_t s[kCols], d[kCols], w[kCols / 2];
            tmem_load_block(s_tm, s);
            F2 l[kCols / 8];
#pragma unroll
            for (int b = 0; b < kCols / 8; ++b) l[b] = load_stats(st + 32 * b);
#pragma unroll
            for (int c = 0; c < kCols; c += 2) {
                const F2 x = fma2({__uint_as_float(s[c]), __uint_as_float(s[c + 1])},
                                  both(p.scale2), l[c / 4 % (kCols / 8)]);
                s[c] = __float_as_uint(exp2_fast(x.x));
                s[c + 1] = __float_as_uint(exp2_fast(x.y));
            }
            const bool diagonal = (step0 + i) % each == 0, fine = diagonal && short_rows(u);
            if (diagonal) {
#pragma unroll
                for (int c = 0; c < kCols; ++c)
                    if (query + c % 16 / 4 * 8 + c % 2 < key + c / 16 * 16 + c % 4 / 2 * 8) s[c] = 0;
            }
#pragma unroll
            for (int c = 0; c < kCols; c += 2)
                w[c / 2] = pack2<T>(__uint_as_float(s[c]), __uint_as_float(s[c + 1]));
            tmem_store_block(s_tm, w);
            if (fine) {
#pragma unroll
                for (int c = 0; c < kCols; c += 2)
                    w[c / 2] = pack2_rest<T>(w[c / 2], __uint_as_float(s[c]), __uint_as_float(s[c + 1]));
                tmem_store_block(s_tm + kCols / 2, w);
            }
            tmem_wait_stores();
            tmem_before();
            __syncwarp();
            if (lane == 0) bar_arrive(p_full);
#pragma unroll
            for (int b = 0; b < kCols / 8; ++b) l[b] = load_stats(st + 512 + 32 * b);
            ok = wait_warp(dp_full, i & 1, waits);
            if (!ok) break;
            tmem_after();
            tmem_load_block(d_tm, d);
#pragma unroll
            for (int c = 0; c < kCols; c += 2) {
                const F2 x = fma2({__uint_as_float(d[c]), __uint_as_float(d[c + 1])},
                                  both(shift.grads), l[c / 4 % (kCols / 8)]);
                const F2 a = mul2({__uint_as_float(s[c]), __uint_as_float(s[c + 1])}, x);
                d[c] = __float_as_uint(a.x), d[c + 1] = __float_as_uint(a.y);
            }
            if (diagonal) {  // (dS of the query that sees one key is 0, as above)
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    const int a = query + c % 16 / 4 * 8 + c % 2, b = key + c / 16 * 16 + c % 4 / 2 * 8;
                    if (a < b || a + u.tile == 0) d[c] = 0;
                }
            }
#pragma unroll
            for (int c = 0; c < kCols; c += 2)
                w[c / 2] = pack2<T>(__uint_as_float(d[c]), __uint_as_float(d[c + 1]));
            tmem_store_block(d_tm, w);
            if (fine) {
#pragma unroll
                for (int c = 0; c < kCols; c += 2)
                    w[c / 2] = pack2_rest<T>(w[c / 2], __uint_as_float(d[c]), __uint_as_float(d[c + 1]));
                tmem_store_block(d_tm + kCols / 2, w);
            }
            tmem_wait_stores();
            tmem_before();
            __syncwarp();
            if (lane == 0) {
                bar_arrive(ds_full);
                bar_arrive(st_empty + 8 * slot_i);
            }
        }
        if (n > 0) {
            if (ok)
                ok = wait_warp(out_full, 0, waits) &&
                     wait_warp(g_clean + 8 * ((n - 1) % kQuerySlots), (n - 1) / kQuerySlots & 1, waits);
            tmem_after();
        }
        const bool bad = sh->bad[0][0][0] != 0;
        // keys that see a dO that is not finite: a column of dv
        const auto mark = [&](int t, int c, uint32_t *v) {
            if (t && bad)
#pragma unroll
                for (int h = 0; h < 16; ++h)
                    if (mine < last_bad[c + h]) v[h] = 0x7fffffffu;
        };
        const float lost = __uint_as_float(0x7fffffffu);  // a wait that gave up: no sums
        if (n > 0 && p.parts > 1) {
            for (int t = 0; t < 2; ++t)
                for (int c = 16 * side; c < p.dim; c += 16 * kSumGroups) {
                    uint32_t v[16];
                    tmem_load16((t ? dv_tm : dk_tm) + lanes + c, v);
                    mark(t, c, v);
#pragma unroll
                    for (int h = 0; h < 16; ++h) v[h] = ok ? v[h] : 0x7fffffffu;
#pragma unroll
                    for (int h = 0; h < 16; h += 4)
                        *part_at(p, blockIdx.x, t, c + h, mine) =
                            make_float4(__uint_as_float(v[h]), __uint_as_float(v[h + 1]),
                                        __uint_as_float(v[h + 2]), __uint_as_float(v[h + 3]));
                }
        } else if (n > 0) {
            // every tile of queries has been used: their places hold the results
            const float factor[2] = {ok ? p.scale * shift.undo : lost,
                                     ok ? Shift<T>::kUndoProbs : lost};
            for (int t = 0; t < 2; ++t)
                for (int c = 16 * side; c < p.dim; c += 16 * kSumGroups) {
                    uint32_t v[16];
                    tmem_load16((t ? dv_tm : dk_tm) + lanes + c, v);
                    mark(t, c, v);
                    Vec8 x[2];
#pragma unroll
                    for (int h = 0; h < 16; ++h)
                        x[h / 8].v[h % 8] = __uint_as_float(v[h]) * factor[t];
                    put_columns<T>(q_at + t * kTileBytes, mine, c, x);
                }
            sums_barrier();
            const int64_t token = u.start + (int64_t)u.tile * kTile;
            const int count = min(kTile, u.len - u.tile * kTile);
            write_tile(q_at, count, static_cast<T *>(p.dk) + token * p.d_token[1] + g * p.d_head[1],
                       p.d_token[1], p.d_vectors[1], p.dim, p.dim_out, (int)threadIdx.x,
                       128 * kSumGroups);
            write_tile(q_at + kTileBytes, count,
                       static_cast<T *>(p.dv) + token * p.d_token[2] + g * p.d_head[2],
                       p.d_token[2], p.d_vectors[2], p.dim, p.dim_out, (int)threadIdx.x,
                       128 * kSumGroups);
        }
    }
    end_block(sh);
    if (warp == kIssueWarp) {
        tmem_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
    }
}

// The parts' sums, in order, as results.  A block takes every fourth 16 columns of a key
// tile's gradients, a thread a key.
template <typename T>
__global__ void __launch_bounds__(kTile) attn_join_kernel(const AttnParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    const int unit = blockIdx.x / kSumGroups, side = blockIdx.x % kSumGroups, g = unit % p.heads_k;
    AttnUnit u;
    if (!unit_at<kTile>(p, unit / p.heads_k, u)) return;
    const int given = u.tile;
    const Shift<T> shift = Shift<T>::of_keys(p, u, g);
    uint32_t used = 0;  // parts that have steps
    for (int r = 0; r < p.parts; ++r) {
        u.tile = given;
        if (KeySteps(p, u, r).n > 0) used |= 1u << r;
    }
    const int row = u.tile * kTile + threadIdx.x;
    const bool live = row < u.len;
    const int64_t token = u.start + (int64_t)row;
    for (int t = 0; t < 2; ++t) {
        const float factor = t ? Shift<T>::kUndoProbs : p.scale * shift.undo;
        T *out = static_cast<T *>(t ? p.dv : p.dk) + token * p.d_token[1 + t] + g * p.d_head[1 + t];
        for (int c = 16 * side; c < p.dim; c += 16 * kSumGroups) {
            Vec8 x[2] = {};
#pragma unroll 4
            for (int r = 0; r < p.parts; ++r) {
                if (!(used >> r & 1)) continue;
#pragma unroll
                for (int h = 0; h < 16; h += 4) {
                    const float4 v = *part_at(p, unit * p.parts + r, t, c + h, threadIdx.x);
                    float *y = &x[h / 8].v[h % 8];
                    y[0] += v.x, y[1] += v.y, y[2] += v.z, y[3] += v.w;
                }
            }
#pragma unroll
            for (int h = 0; h < 16; ++h) x[h / 8].v[h % 8] *= factor;
            if (!live) continue;
#pragma unroll
            for (int h = 0; h < 16; h += 8) {
                if (p.d_vectors[1 + t])
                    store8<true>(out + c + h, from_float<T>(x[h / 8]), p.dim_out - c - h);
                else store8<false>(out + c + h, from_float<T>(x[h / 8]), p.dim_out - c - h);
            }
        }
    }
}

// The gradients of keys and values that no query head reads: zeros.
template <typename T>
__global__ void __launch_bounds__(kTile) attn_zero_kernel(const AttnParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    const int64_t units =
        (int64_t)(p.tiles ? *p.n_tiles : ((int)p.tokens + kTile - 1) / kTile) * p.heads_k;
    for (int64_t i = blockIdx.x; i < units; i += gridDim.x) {
        AttnUnit u;
        unit_at<kTile>(p, (int)(i / p.heads_k), u);
        const int g = (int)(i % p.heads_k), rows = min(kTile, u.len - u.tile * kTile);
        const int64_t token = u.start + (int64_t)u.tile * kTile;
        for (int t = 0; t < 2; ++t)
            for (int e = threadIdx.x; e < rows * p.dim_out; e += kTile)
                static_cast<T *>(t ? p.dv : p.dk)[(token + e / p.dim_out) * p.d_token[1 + t] +
                                                  g * p.d_head[1 + t] + e % p.dim_out] = T(0.f);
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// Blocks that share 128 keys: as many as end soonest.  The steps of the longest block, or an
// even share of all (1.4 us each); a block's start and end (5 us); joining, which writes
// and reads 128 KB of sums for each block.  The lengths are on the device: sequences of
// the same length, the longest three times as long.  1024 tokens of 16 + 2 heads of 128, both
// passes: 76 us (one block each 138); 8192 of 8 + 1 471 (967); 4096 of 32 + 8 stay at
// one block each, 479 us (two 501).
static int parts_of(const pos_attn *a) {
    const double count = a->starts ? std::max(1, a->sequences) : 1, sms = sm_count();
    const double len = std::max(1., (double)a->tokens / count / kTile);
    const double group = (double)a->heads_q / a->heads_k;
    const double most =
        std::min(std::ceil((double)a->tokens / kTile), std::ceil(count > 1 ? 3 * len : len)) * group;
    const double all = count * len * (len + 1) / 2 * group * a->heads_k / sms;
    const double units = count * std::ceil(len) * a->heads_k;
    int best = 1;
    double least = 1e300;
    for (int c = 1; c <= 8; c *= 2) {
        const double t = 1.4 * std::max(std::ceil(most / c), all) +
                         5. * std::max(1., units * c / sms) + (c > 1 ? 4. + 0.055 * units * c : 0.);
        if (t < least) least = t, best = c;
    }
    // (their sums take 128 KB each)
    while (best > 1 && attn_most_tiles(a, kTile) * a->heads_k * best > 8 * (int64_t)sms) best /= 2;
    return best;
}
static int64_t part_bytes(const pos_attn *a, int parts) {
    return parts == 1 ? 0 : attn_most_tiles(a, kTile) * a->heads_k * parts *
                                ((a->dim + 15) / 16 * 16) * kTile * 8;
}

static int64_t stats_bytes(const pos_attn *a) {
    return (a->tokens * a->heads_q * 8 + 15) / 16 * 16;
}
// f16: sequences are numbered in order, or by their first tokens if fewer of these are
// possible than sequences.
static int64_t largest_bytes(const pos_attn *a) {
    const int64_t n = a->starts ? std::min<int64_t>(a->sequences, a->tokens) : 1;
    return a->dtype == POS_F16 ? (n * a->heads_k * 4 + 15) / 16 * 16 : 0;
}
static int64_t values_bytes(const pos_attn *a) {
    return a->dtype == POS_F16 ? (a->tokens * a->heads_k * 4 + 15) / 16 * 16 + largest_bytes(a) : 0;
}

template <typename T>
static pos_status launch_backward(const pos_attn *a, const AttnParams &p, cudaStream_t s) {
    CUtensorMap q, k, v, g;
    POS_TRY(attn_map(&q, a, p.q, p.heads_q, p.dim));
    POS_TRY(attn_map(&k, a, p.k, p.heads_k, p.dim));
    POS_TRY(attn_map(&v, a, p.v, p.heads_k, p.dim));
    POS_TRY(attn_map(&g, a, p.g, p.heads_q, p.dim));
    const int grid_q = attn_grid(a, kTile, a->heads_q), grid_k = attn_grid(a, kTile, a->heads_k);
    if (grid_q == 0) return POS_OK;
    if (grid_k == kMostUnits) return fail(POS_EINVAL, "attention: too many tiles of keys");
    if constexpr (Shift<T>::kOn)
        POS_CUDA(launch_dependent(attn_values_kernel<T>, std::min(grid_k, 16 * std::max(1, sm_count())),
                                  kTile, 0, s, p));
    auto dq = attn_dq_kernel<T>;
    POS_TRY(ensure_smem(reinterpret_cast<const void *>(dq), kDqSmem));
    POS_CUDA(launch_dependent(dq, std::min(grid_q, std::max(1, sm_count())), kBackThreads, kDqSmem, s,
                              q, k, v, g, p));
    auto dkv = attn_dkv_kernel<T>;
    POS_TRY(ensure_smem(reinterpret_cast<const void *>(dkv), kDkvSmem));
    POS_CUDA(launch_dependent(dkv, grid_k * p.parts, kBackThreads, kDkvSmem, s, q, k, v, g, p));
    if (p.parts > 1)
        POS_CUDA(launch_dependent(attn_join_kernel<T>, grid_k * kSumGroups, kTile, 0, s, p));
    return POS_OK;
}

static pos_status no_queries(const pos_attn *a, AttnParams p, char *at, cudaStream_t s) {
    POS_TRY(attn_list(a, kTile, &at, s, &p));
    const int grid = std::min(attn_grid(a, kTile, a->heads_k), 16 * std::max(1, sm_count()));
    if (grid == 0) return POS_OK;
    const auto kern = a->dtype == POS_BF16 ? attn_zero_kernel<__nv_bfloat16> : attn_zero_kernel<__half>;
    POS_CUDA(launch_dependent(kern, grid, kTile, 0, s, p));
    return POS_OK;
}

static pos_status backward(const pos_attn *a, const pos_heads *x, const pos_heads &d_o,
                           AttnParams p, int parts, char *at, cudaStream_t s) {
    p.largest = reinterpret_cast<uint32_t *>(at);
    at += largest_bytes(a);
    p.most = reinterpret_cast<float *>(at);
    p.values = reinterpret_cast<float *>(at + largest_bytes(a));
    at += values_bytes(a);
    p.stats = reinterpret_cast<float2 *>(at);
    at += stats_bytes(a);
    p.parts = parts, p.first_blocks = a->starts ? std::max(1, sm_count()) : 0x7fffffff;
    p.part = reinterpret_cast<float *>(at);
    at += part_bytes(a, parts);
    const pos_heads t[4] = {x[0], x[1], x[2], d_o};
    const int64_t heads[4] = {a->heads_q, a->heads_k, a->heads_k, a->heads_q};
    AttnTensor *to[4] = {&p.q, &p.k, &p.v, &p.g};
    for (int i = 0; i < 4; ++i) POS_TRY(attn_input(a, t[i], heads[i], &at, s, to[i]));
    POS_TRY(attn_list(a, kTile, &at, s, &p));
    return a->dtype == POS_BF16 ? launch_backward<__nv_bfloat16>(a, p, s)
                                : launch_backward<__half>(a, p, s);
}

}  // namespace pos

extern "C" pos_status poseidon_attn_backward(const pos_attn *attn, const pos_heads *x,
                                             const pos_heads *o, const float *d_lse,
                                             const pos_heads *d_o, const pos_heads *dx,
                                             void *stream) {
    using namespace pos;
    return guarded([&]() -> pos_status {
        AttnParams p = {};
        POS_TRY(check_attn(attn, &p));
        if (!x || !o || !d_o || !dx) return fail(POS_EINVAL, "attention: NULL pointer");
        const int64_t heads[4] = {attn->heads_q, attn->heads_k, attn->heads_k, attn->heads_q};
        const char *names[3] = {"the queries", "the keys", "the values"};
        for (int i = 0; i < 3; ++i) {
            POS_TRY(check_attn_tensor(attn, x[i], heads[i], names[i], false));
            POS_TRY(check_attn_tensor(attn, dx[i], heads[i],
                                      (std::string("the gradients of ") + names[i]).c_str(), true));
        }
        POS_TRY(check_attn_tensor(attn, *o, attn->heads_q, "o", false));
        POS_TRY(check_attn_tensor(attn, *d_o, attn->heads_q, "o's gradient", false));
        if (reinterpret_cast<uintptr_t>(d_lse) % 4)
            return fail(POS_EINVAL, "attention: misaligned lse");
        if (attn->tokens == 0 || attn->heads_k == 0) return POS_OK;
        if (!d_lse && attn->heads_q > 0) return fail(POS_EINVAL, "attention: NULL lse");
        p.o = {o->data, o->token_stride, o->head_stride};
        p.lse = const_cast<float *>(d_lse);
        void **out[3] = {&p.dq, &p.dk, &p.dv};
        for (int i = 0; i < 3; ++i) {
            *out[i] = dx[i].data, p.d_token[i] = dx[i].token_stride, p.d_head[i] = dx[i].head_stride;
            p.d_vectors[i] = aligned16(dx[i].data) && dx[i].token_stride % 8 == 0 &&
                             dx[i].head_stride % 8 == 0;
        }
        const auto s = static_cast<cudaStream_t>(stream);
        void *scratch = nullptr;
        if (attn->heads_q == 0) {
            POS_TRY(attn_scratch(attn_list_bytes(attn, kTile), s, &scratch));
            const pos_status st = no_queries(attn, p, static_cast<char *>(scratch), s);
            const cudaError_t e = scratch ? cudaFreeAsync(scratch, s) : cudaSuccess;
            if (st != POS_OK) return st;
            return e == cudaSuccess ? POS_OK : cuda_fail(e, "attention scratch");
        }
        const int parts = parts_of(attn);
        int64_t bytes = largest_bytes(attn) + values_bytes(attn) + stats_bytes(attn) + part_bytes(attn, parts) +
                        attn_list_bytes(attn, kTile);
        for (int i = 0; i < 4; ++i)
            if (!attn_direct(attn, i < 3 ? x[i] : *d_o, heads[i]))
                bytes += attn_copy_bytes(attn, heads[i]);
        POS_TRY(attn_scratch(bytes, s, &scratch));
        const pos_status st = backward(attn, x, *d_o, p, parts, static_cast<char *>(scratch), s);
        const cudaError_t e = cudaFreeAsync(scratch, s);
        if (st != POS_OK) return st;
        return e == cudaSuccess ? POS_OK : cuda_fail(e, "attention scratch");
    });
}
