// poseidon_attn_forward, and what both passes of attention share on the host
// (formulas: poseidon.h).
#include <cstdlib>

#include "attn.cuh"

namespace pos {

// ---------------------------------------------------------------------------
// The tiles of packed sequences
// ---------------------------------------------------------------------------
// Tiles of `rows` tokens of every sequence, those with the most keys first, so that
// the blocks that start last are short.  One block; sequences are counted into bins
// by the number of their tiles.  A start that is below one before it counts as
// that one, one outside 0 .. tokens as the nearest of these, so sequences never overlap.
constexpr int kListThreads = 1024, kBins = 2048;
struct AttnListParams {
    const int32_t *starts;
    int4 *tiles;
    int32_t *n_tiles;
    int64_t tokens;
    int32_t sequences, rows, shift;  // bin = tile >> shift
    int32_t bins;                    // that a tile can be in, a multiple of 32
};
__global__ void __launch_bounds__(kListThreads) attn_tiles_kernel(const AttnListParams p) {
    grid_dep_wait();
    grid_dep_trigger();
    __shared__ int bins[kBins], most[kListThreads / 32];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    for (int i = threadIdx.x; i < p.bins; i += kListThreads) bins[i] = 0;
    __syncthreads();
    // each warp a run of sequences; the largest start before the run
    const int each = (p.sequences + kListThreads / 32 - 1) / (kListThreads / 32);
    const int s0 = min(p.sequences, warp * each), s1 = min(p.sequences, s0 + each);
    const int tokens = (int)p.tokens;
    int top = 0;
    for (int s = s0 + lane; s < s1; s += 32) top = max(top, min(tokens, p.starts[s]));
    for (int o = 16; o; o /= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) most[warp] = top;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < warp; ++w) before = max(before, most[w]);
    for (int pass = 0; pass < 2; ++pass) {
        int last = before;
        for (int s = s0; s < s1; s += 32) {  // 32 starts at once, then one sequence at a time
            const int mine = min(s + lane, s1 - 1);
            int a = min(tokens, p.starts[mine]);
            for (int o = 1; o < 32; o *= 2)
                a = max(a, __shfl_up_sync(0xffffffffu, a, o));
            a = max(a, last);
            const int b = max(a, min(tokens, p.starts[mine + 1]));
            // (many may be empty)
            uint32_t there = __ballot_sync(0xffffffffu, lane < s1 - s && b > a);
            for (; there; there &= there - 1) {
                const int i = __ffs(there) - 1;
                const int at = __shfl_sync(0xffffffffu, a, i);
                const int len = __shfl_sync(0xffffffffu, b, i) - at;
                for (int t = lane; t < (len + p.rows - 1) / p.rows; t += 32) {
                    const int to = atomicAdd(&bins[t >> p.shift], 1);
                    if (pass) p.tiles[to] = make_int4(at, len, t, p.sequences > tokens ? at : s + i);
                }
            }
            last = __shfl_sync(0xffffffffu, a, 31);
        }
        __syncthreads();
        if (pass) break;
        // bins become places: the tiles of higher bins come first
        if (warp == 0) {
            int sum = 0;
            for (int b0 = p.bins - 32; b0 >= 0; b0 -= 32) {
                const int b = b0 + 31 - lane, v = bins[b];
                int up = v;
                for (int o = 1; o < 32; o *= 2) {
                    const int w = __shfl_up_sync(0xffffffffu, up, o);
                    if (lane >= o) up += w;
                }
                bins[b] = sum + up - v;
                sum += __shfl_sync(0xffffffffu, up, 31);
            }
            if (lane == 0) *p.n_tiles = sum;
        }
        __syncthreads();
    }
}

// A tensor whose rows tensor copies cannot read, in rows of a multiple of 8 elements
// one after another, zeros past the last element.
template <typename T>
__global__ void __launch_bounds__(256) attn_copy_kernel(const T *x, int64_t token, int64_t head,
                                                        int64_t tokens, int heads, int dim, T *y) {
    grid_dep_wait();
    grid_dep_trigger();
    const int per = (dim + 7) / 8;
    const int64_t n = tokens * heads * per;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += 256ll * gridDim.x) {
        const int64_t row = i / per;
        const int j = (int)(i - row * per);
        const T *from = x + row / heads * token + row % heads * head + 8 * j;
        store8<true>(y + 8 * i, load8_shifted(from, 8 * j, dim - 8 * j), 8);
    }
}

// ---------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------
// A block takes 256 queries of a head, two tiles of 128, which share the keys and
// values that pass through shared memory.  Per tile of keys: scores = Q K^T to TMEM;
// a warpgroup, a row of a tile a thread, takes its row's largest score and
// exponentials and puts them back in 16 bits in the scores' place; the sums O += P V
// stay in TMEM.  One thread issues the products of both tiles in turn, so the
// tensor cores work on one tile while the other's exponentials are computed.  Keys
// go from the diagonal down, so the first tile is the one with a mask and no row's
// largest score is ever of nothing.  A block takes one such unit after another, so that a
// unit's first loads and scores come while the one before it ends.  Two warps look over the
// values of the tiles on the diagonal, half a tile each, while the first exponentials are computed.
constexpr int kSlots = 5;                    // tiles of keys and values on their way
constexpr int kForwardRows = 2 * kTile;
constexpr int kForwardThreads = 3 * 128;     // two warpgroups of rows, one of loads and products
constexpr int kForwardBars = 2 * kSlots + 13;
// and the first row of each column whose value is not finite, of two units, tiles, halves
constexpr int kForwardSmem =
    1024 + (2 + kSlots) * kTileBytes + 8 * kForwardBars + kSharedBytes + 8 * kAttnMaxDim;
// 2 * 208 + 88 = 504 = 3 * 168, what the block is launched with
constexpr int kRowRegs = 208, kIssueRegs = 88;
// A row's reference, which its exponentials are relative to, follows its largest
// score only when that is 2^8 times more: sums of up to 2^8 times their size have
// the same precision, and O in TMEM is rescaled that much more rarely.
constexpr float kSlack = 8.f;
// Besides, in bf16 they are 2^-8 of that, 1 at most, so that sums of values near the type's
// largest do not pass f32's; in f16 2^7 of it, 2^15 at most, so that many small ones keep
// their bits: below 2^-14 f16 has fewer, below 2^-25 none, and 32768 keys of 2^-25 are 2^-10 of
// the weight, half an o's step and more.
template <typename T>
constexpr float kLift = std::is_same<T, __nv_bfloat16>::value ? -kSlack : 15.f - kSlack;

// Of references above this a step in 32 bits is 2^-3 and more, and the largest exponential, of
// the difference of an exact product and a rounded one, can be far from 1: past what 16 or 32
// bits hold, or 0.  Weights relative to one another stay right, so that a sum that is finite and
// not below one exponential tells the rows that are.
constexpr float kLarge = 1048576.f;
// One row by the formulas alone, by a warp, where that was so.  (Not inline: as a part of the
// kernel's code it costs 32768 tokens 18 us of 689, 3001 in 7 sequences 1 of 27.  All scores
// relative to the reference's, which needs none of this, were 4 % of 4096 tokens.)
template <typename T>
__device__ __noinline__ void forward_row(const AttnParams &p, const AttnUnit &u, int row, int head,
                                         int lane) {
    const int g = head / p.group;
    const T *q = row_at<T>(p.q, u.start + row, head);
    float top = -__uint_as_float(0x7f800000u), total = 0.f;
    RowPart sum = {};
    for (int j0 = 0; j0 <= row; j0 += 32) {
        const int j = j0 + lane, n = min(32, row + 1 - j0);
        float s = -__uint_as_float(0x7f800000u);
        if (j <= row) s = dot_rows(q, row_at<T>(p.k, u.start + j, g), p.dim) * p.scale2;
        float m = s;
        for (int o = 16; o; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        m = fmaxf(m, top);
        if (__any_sync(0xffffffffu, !(s == s))) m = __uint_as_float(0x7fffffffu);  // (passed over)
        const float shrink = m == top ? 1.f : exp2f(top - m);
        top = m;
        // (scores of minus infinity alone, so far: nothing yet)
        const float e = j <= row && m != -__uint_as_float(0x7f800000u) ? exp2f(s - m) : 0.f;
        total *= shrink;
#pragma unroll
        for (int i = 0; i < kAttnMaxDim / 32; ++i) sum.v[i] *= shrink;
        for (int t = 0; t < n; ++t) {
            const float w = __shfl_sync(0xffffffffu, e, t);
            total += w;
            add_row(sum, w, row_at<T>(p.v, u.start + j0 + t, g), p.dim, lane);
        }
    }
    write_row<T>(p.out, (u.start + row) * p.out_token + head * p.out_head, sum, 1.f / total,
                 p.dim_out, lane);
    if (p.lse && lane == 0)
        p.lse[head * p.tokens + u.start + row] = (top + log2f(total)) * kLn2;
}

struct ForwardUnit : BlockUnit<kForwardRows> {
    int r0, n0, n1, first;  // first token; tiles of keys that its two tiles see, the last
    __device__ __forceinline__ bool next(const AttnParams &p, int &round) {
        if (!BlockUnit::next(p, round)) return false;
        r0 = u.tile * kForwardRows;
        n0 = 2 * u.tile + 1;
        n1 = r0 + kTile < u.len ? n0 + 1 : 0;
        first = max(n0, n1) - 1;
        return true;
    }
};

template <typename T>
__global__ void __launch_bounds__(kForwardThreads, 1)
    attn_forward_kernel(const __grid_constant__ CUtensorMap q_map,
                        const __grid_constant__ CUtensorMap k_map,
                        const __grid_constant__ CUtensorMap v_map, const AttnParams p) {
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char *aligned = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t q_at = base, kv_at = q_at + 2 * kTileBytes;
    const uint32_t bars = kv_at + kSlots * kTileBytes;
    const uint32_t kv_full = bars, kv_empty = kv_full + 8 * kSlots;
    const uint32_t q_full = kv_empty + 8 * kSlots, s_full = q_full + 16, p_full = s_full + 16,
                   o_full = p_full + 16, q_empty = o_full + 16, v_in = q_empty + 16,
                   v_out = v_in + 8;
    const uint32_t slot = v_out + 16;
    AttnShared *sh = reinterpret_cast<AttnShared *>(aligned + (slot - base));
    // the first row of each column's value that is not finite, of a tile's units in turn
    uint8_t *first_bad = aligned + (slot - base) + kSharedBytes;
    const Waits waits(sh, p);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, group = warp / 4;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kForwardBars; ++i) {
            const uint32_t b = bars + 8 * i;  // p_full: a tile's four warps
            bar_init(b, b >= p_full && b < o_full ? 4 : b >= v_out ? 2 : 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        init_shared(sh);
        asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    }
    if (warp == 9) {
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

    const int boxes = p.dim > 64 ? 2 : 1;
    ForwardUnit w;
    int round = 0;
    bool ok = true;

    if (group == 2) {
        give_registers<kIssueRegs>();
        if (warp == 8) {
            int s = 0;
            uint32_t ph = 1, q_ph[2] = {1, 1};  // an empty slot's first wait passes
            while (lane == 0 && ok && w.next(p, round)) {
                const auto load = [&](bool v, int j) {
                    if (!attn_wait(kv_empty + 8 * s, ph, waits)) return false;
                    bar_expect(kv_full + 8 * s, boxes * kBox);
                    for (int b = 0; b < boxes; ++b)
                        tma_rows(kv_at + s * kTileBytes + b * kBox, v ? &v_map : &k_map, 64 * b,
                                 w.head / p.group, w.u.start + j * kTile, kv_full + 8 * s);
                    if (++s == kSlots) s = 0, ph ^= 1;
                    return true;
                };
                ok = load(false, w.first);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (!ok || (t && !w.n1)) break;
                    ok = attn_wait(q_empty + 8 * t, q_ph[t], waits);
                    if (!ok) break;
                    q_ph[t] ^= 1;
                    bar_expect(q_full + 8 * t, boxes * kBox);
                    for (int b = 0; b < boxes; ++b)
                        tma_rows(q_at + t * kTileBytes + b * kBox, &q_map, 64 * b, w.head,
                                 w.u.start + w.r0 + t * kTile, q_full + 8 * t);
                }
                for (int j = w.first; j >= 0 && ok; --j)
                    ok = load(true, j) && (j == 0 || load(false, j - 1));
            }
        } else if (warp == 9) {
            const uint32_t mine = one_lane();
            const int steps = (p.dim + 15) / 16;
            uint32_t ph[2] = {0, 0}, q_ph[2] = {0, 0};
            int base = 0;  // tiles of keys and values of the units before
            while (ok && w.next(p, round)) {
                // the i-th tile to arrive: keys 2 i, values 2 i + 1
                const auto arrived = [&](int i) {
                    return wait_warp(kv_full + 8 * ((base + i) % kSlots), (base + i) / kSlots & 1,
                                     waits);
                };
                const auto place = [&](int i) { return kv_at + (base + i) % kSlots * kTileBytes; };
                const auto scores = [&](int t, int i) {  // i: steps of keys from the first on
                    mma_rows<T>(tmem + t * kTile, q_at + t * kTileBytes, place(2 * i), steps, mine);
                    commit(s_full + 8 * t, mine);
                    if (i == w.first) commit(q_empty + 8 * t, mine);  // the last ones
                };
                ok = arrived(0);
                bar_arrive_one(v_in, mine);
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    if (ok && (t == 0 || w.n1)) {
                        ok = wait_warp(q_full + 8 * t, q_ph[t], waits);
                        q_ph[t] ^= 1;
                    }
                if (!ok) break;
                tmem_after();
                if (w.first < w.n0) scores(0, 0);
                if (w.first < w.n1) scores(1, 0);
                commit(kv_empty + 8 * (base % kSlots), mine);
                for (int j = w.first, i = 0; j >= 0 && ok; --j, ++i) {
                    ok = arrived(2 * i + 1);
                    if (!ok) break;
                    if (j > 0) ok = arrived(2 * i + 2);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const int n = t ? w.n1 : w.n0;
                        if (j < n && ok) {
                            ok = wait_warp(p_full + 8 * t, ph[t], waits);
                            if (!ok) break;
                            ph[t] ^= 1;
                            tmem_after();
                            // (the sums of the unit before have been read: its rows' warps
                            // have gone on to these probabilities)
                            mma_columns<T>(tmem + 2 * kTile + t * kTile, tmem + t * kTile,
                                           place(2 * i + 1), steps, j < n - 1, mine);
                            if (j == 0) commit(o_full + 8 * t, mine);
                        }
                        if (j > 0 && j - 1 < n && ok) scores(t, i + 1);
                    }
                    commit(kv_empty + 8 * ((base + 2 * i + 1) % kSlots), mine);
                    if (j > 0) commit(kv_empty + 8 * ((base + 2 * i + 2) % kSlots), mine);
                }
                base += 2 * (w.first + 1);
            }
        } else {
            const int half = warp - 10;
            uint32_t ph = 0;
            int base = 0, units[2] = {0, 0};
            while (ok && w.next(p, round)) {
                const auto at_tile = [&](int t) {
                    return first_bad + ((2 * (units[t] & 1) + t) * 2 + half) * kAttnMaxDim;
                };
                // t's values are the i-th tile to arrive
                const auto look = [&](int t, int i) {
                    ok = ok && wait_warp(kv_full + 8 * ((base + i) % kSlots), (base + i) / kSlots & 1,
                                         waits);
                    if (!ok) return false;
                    const uint32_t at = kv_at + (base + i) % kSlots * kTileBytes;
                    const int seen = min(kTile, w.u.len - ((t ? w.n1 : w.n0) - 1) * kTile);
                    const int from = half * (kTile / 2), end = min(seen, from + kTile / 2);
                    const bool bad = tile_bad<T>(at, from, end, boxes, lane);
                    if (bad) {
                        uint8_t *first = at_tile(t);
                        for (int c = lane; c < kAttnMaxDim; c += 32) first[c] = kTile;
                        tile_clean<T>(at, from, end, boxes, lane,
                                      [&](int c, int row, int) { first[c] = (uint8_t)row; });
                    }
                    zero_rows(at, max(from, seen), from + kTile / 2, boxes, lane);
                    tile_done();
                    return bad;
                };
                // (from its first tile on, the phases of the places are this unit's)
                ok = wait_warp(v_in, ph, waits);
                ph ^= 1;
                const bool second = w.n1 > 0 && look(1, 1);
                const bool first = look(0, w.n1 > 0 ? 3 : 1);
                if (!ok) break;
                const auto tell = [&](int t, bool bad) {
                    if (lane == 0) sh->bad[units[t] & 1][t][half] = bad;
                    __syncwarp();
                    if (lane == 0) bar_arrive(v_out + 8 * t);
                };
                if (w.n1) {  // the second tile's rows see all of the first one's
                    uint8_t *to = at_tile(1), *from = at_tile(0);
                    for (int c = lane; first && c < kAttnMaxDim; c += 32)
                        to[c] = from[c] < kTile ? 0 : second ? to[c] : kTile;
                    tell(1, first || second);
                    ++units[1];
                }
                tell(0, first);
                ++units[0];
                base += 2 * (w.first + 1);
            }
        }
        __syncwarp();
    } else {
        take_registers<kRowRegs>();
        const int t = group;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const uint32_t s_tm = tmem + t * kTile + lanes, o_tm = tmem + 2 * kTile + t * kTile + lanes;
        const int dim16 = (p.dim + 15) / 16 * 16;
        uint32_t ph = 0;
        int unit = 0;
        while (w.next(p, round)) {
            const int n = t ? w.n1 : w.n0;
            if (n == 0) continue;
            const int row = w.r0 + t * kTile + threadIdx.x % kTile;  // of the sequence
            float top = 0.f, total = 0.f;
            for (int j = n - 1; j >= 0 && ok; --j) {
                ok = wait_warp(s_full + 8 * t, ph, waits);
                if (!ok) break;
                ph ^= 1;
                tmem_after();
                uint32_t s[kTile];
                tmem_load128(s_tm, s);
                if (j == n - 1) {
                    const int seen = row - j * kTile;  // the last key that the row sees
#pragma unroll
                    for (int c = 0; c < kTile; ++c)
                        if (c > seen) s[c] = 0xff800000u;
                }
                float part[4];  // (four chains: one of 128 steps is longer than the exponentials)
#pragma unroll
                for (int c = 0; c < 4; ++c) part[c] = max3(s[c], s[c + 4], s[c + 8]);
#pragma unroll
                for (int c = 12; c + 8 <= kTile; c += 8)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        part[e] = max3(__float_as_uint(part[e]), s[c + e], s[c + e + 4]);
#pragma unroll
                for (int e = 0; e < 4; ++e) part[e] = fmaxf(part[e], __uint_as_float(s[kTile - 4 + e]));
                const float m =
                    fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])) * p.scale2;
                if (j == n - 1) {
                    // (scores of minus infinity alone, so far: nothing yet)
                    top = fmaxf(m, -__uint_as_float(0x7f7fffffu));
                } else {
                    const bool more = m > top + kSlack;
                    if (__any_sync(0xffffffffu, more)) {
                        // the scores of this step were issued after the last product into O
                        // and are there, so that one is done
                        const float shrink = more ? exp2_fast(top - m) : 1.f;
                        if (more) top = m;
                        total *= shrink;
                        for (int c = 0; c < dim16; c += 16) {
                            uint32_t o[16];
                            tmem_load16(o_tm + c, o);
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                o[e] = __float_as_uint(__uint_as_float(o[e]) * shrink);
                            tmem_store16(o_tm + c, o);
                        }
                    }
                }
                F2 sum[4] = {};
#pragma unroll
                for (int c = 0; c < kTile; c += 32) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const F2 x = fma2({__uint_as_float(s[c + 2 * e]), __uint_as_float(s[c + 2 * e + 1])},
                                          both(p.scale2), both(kLift<T> - top));
                        const F2 y = {exp2_fast(x.x), exp2_fast(x.y)};
                        sum[e % 4] = add2(sum[e % 4], y);
                        w[e] = pack2<T>(y.x, y.y);
                    }
                    tmem_store16(s_tm + c / 2, w);
                }
                const F2 a = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
                total += a.x + a.y;
                tmem_wait_stores();
                tmem_before();
                // (the values that these are multiplied by are looked over)
                if (j == n - 1) ok = wait_warp(v_out + 8 * t, unit & 1, waits);
                __syncwarp();
                if (ok && lane == 0) bar_arrive(p_full + 8 * t);
            }
            if (ok) ok = wait_warp(o_full + 8 * t, unit & 1, waits);
            tmem_after();
            const bool live = row < w.u.len;
            // halves of the tile's values that hold some that are not finite
            const int bad = sh->bad[unit & 1][t][0] + 2 * sh->bad[unit & 1][t][1];
            float factor = 1.f / total;
            if (!ok) factor = __uint_as_float(0x7fffffffu);  // a wait that gave up: no result
            T *out = static_cast<T *>(p.out) + (w.u.start + (int64_t)row) * p.out_token +
                     w.head * p.out_head;
            // rows that see values that are not finite
            const auto mark = [&](int c, uint32_t *o) {
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    if (bad >> half & 1) {
                        const uint8_t *first =
                            first_bad + ((2 * (unit & 1) + t) * 2 + half) * kAttnMaxDim + c;
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if ((int)(threadIdx.x % kTile) >= first[e]) o[e] = 0x7fffffffu;
                    }
            };
            const auto write = [&](bool check) {
                for (int c = 0; c < dim16; c += 16) {
                    uint32_t o[16];
                    tmem_load16(o_tm + c, o);
                    if (check) mark(c, o);
                    Vec8 x[2];
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e / 8].v[e % 8] = __uint_as_float(o[e]) * factor;
                    if (!live) continue;
#pragma unroll
                    for (int e = 0; e < 16; e += 8) {
                        if (p.out_vectors)
                            store8<true>(out + c + e, from_float<T>(x[e / 8]), p.dim_out - c - e);
                        else store8<false>(out + c + e, from_float<T>(x[e / 8]), p.dim_out - c - e);
                    }
                }
            };
            if (bad) write(true);  // (a copy of its own)
            else write(false);
            if (p.lse && live)
                p.lse[w.head * p.tokens + w.u.start + row] =
                    ok ? (top - kLift<T> + log2f(total)) * kLn2 : __uint_as_float(0x7fffffffu);
            if (__any_sync(0xffffffffu, fabsf(top) > kLarge)) {
                bool good = finite(total) && total > 0.5f * exp2f(kLift<T>);
                for (int c = 0; c < dim16; c += 16) {
                    uint32_t o[16];
                    tmem_load16(o_tm + c, o);
#pragma unroll
                    for (int e = 0; e < 16; ++e) good = good && finite(__uint_as_float(o[e]));
                }
                const bool large =
                    fabsf(top) > kLarge && fabsf(top) < __uint_as_float(0x7f7fffffu);
                do_again(__ballot_sync(0xffffffffu, ok && live && large && !good), sh, [&](int i) {
                    forward_row<T>(p, w.u, row - lane + i, w.head, lane);
                });
            }
            ++unit;
        }
    }
    end_block(sh);
    if (warp == 9) {
        tmem_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// How long a wait lasts: two seconds, or POSEIDON_ATTN_WAIT_NS as the process has it when
// it makes its first call.
static uint64_t wait_limit_ns() {
    static const uint64_t ns = [] {
        const char *v = std::getenv("POSEIDON_ATTN_WAIT_NS");
        char *end = nullptr;
        const uint64_t given = v ? std::strtoull(v, &end, 10) : 0;
        return v && end != v && *end == 0 ? given : kWaitNs;  // (no number: as if not set)
    }();
    return ns;
}

pos_status check_attn(const pos_attn *a, AttnParams *p) {
    if (!a) return fail(POS_EINVAL, "attention: NULL pointer");
    if (a->tokens < 0 || a->tokens >= (1ll << 31) - 2 * kForwardRows)
        return fail(POS_EINVAL, "attention: bad token count");
    if (a->heads_q < 0 || a->heads_k < 0 || a->heads_q > 65536 || a->heads_k > 65536 ||
        (a->heads_q > 0 && (a->heads_k == 0 || a->heads_q % a->heads_k)))
        return fail(POS_EINVAL, "attention: heads_q must be a multiple of heads_k");
    if (a->dim < 1 || a->dim > kAttnMaxDim)
        return fail(POS_EINVAL, "attention: dim must be 1..128");
    if (a->dtype != POS_BF16 && a->dtype != POS_F16)
        return fail(POS_EINVAL, "attention: dtype must be bf16 or f16");
    if (!(a->scale > 0.f && a->scale < 1e30f))
        return fail(POS_EINVAL, "attention: scale must be above 0 and finite");
    if (a->sequences < 0 || a->sequences > (1 << 24))
        return fail(POS_EINVAL, "attention: bad sequence count");
    if (reinterpret_cast<uintptr_t>(a->starts) % 4)
        return fail(POS_EINVAL, "attention: misaligned starts");
    p->tokens = a->tokens, p->heads_q = a->heads_q, p->heads_k = a->heads_k;
    p->group = a->heads_k ? a->heads_q / a->heads_k : 1;
    p->dim = (a->dim + 7) / 8 * 8, p->dim_out = a->dim;
    p->scale = a->scale, p->scale2 = a->scale * kLog2e;
    p->wait_ns = wait_limit_ns(), p->try_ns = (uint32_t)std::min<uint64_t>(kTryNs, p->wait_ns);
    return POS_OK;
}

pos_status check_attn_tensor(const pos_attn *a, const pos_heads &t, int64_t heads, const char *what,
                             bool written) {
    if (t.token_stride < 0 || t.head_stride < 0 || t.token_stride >= (1ll << 38) ||
        t.head_stride >= (1ll << 38))
        return fail(POS_EINVAL, std::string("attention: bad stride of ") + what);
    if (heads == 0 || a->tokens == 0) return POS_OK;
    if (!t.data) return fail(POS_EINVAL, std::string("attention: NULL ") + what);
    if (reinterpret_cast<uintptr_t>(t.data) % 2)
        return fail(POS_EINVAL, std::string("attention: misaligned ") + what);
    if (written && rows_overlap(a->tokens, heads, a->dim, t.token_stride, t.head_stride))
        return fail(POS_EINVAL, std::string("attention: overlapping rows of ") + what);
    return POS_OK;
}

pos_status attn_scratch(int64_t bytes, cudaStream_t s, void **out) {
    *out = nullptr;
    if (bytes == 0) return POS_OK;
    cudaMemPool_t pool;
    POS_TRY(scratch_pool(&pool, bytes));
    POS_CUDA(cudaMallocFromPoolAsync(out, (size_t)bytes, pool, s));
    return POS_OK;
}

// Whether tensor copies can read a tensor as it is: 16-byte steps, above 0.
bool attn_direct(const pos_attn *a, const pos_heads &t, int64_t heads) {
    return a->dim % 8 == 0 && aligned16(t.data) &&
           (a->tokens == 1 || (t.token_stride % 8 == 0 && t.token_stride > 0)) &&
           (heads == 1 || (t.head_stride % 8 == 0 && t.head_stride > 0));
}
int64_t attn_copy_bytes(const pos_attn *a, int64_t heads) {
    return a->tokens * heads * ((a->dim + 7) / 8 * 8) * 2;
}
// A tensor as the kernels read it; *copy: where its copy goes, if it needs one.
pos_status attn_input(const pos_attn *a, const pos_heads &t, int64_t heads, char **copy,
                      cudaStream_t s, AttnTensor *out) {
    if (attn_direct(a, t, heads)) {
        *out = {t.data, t.token_stride, t.head_stride};
        return POS_OK;
    }
    const int64_t dim = (a->dim + 7) / 8 * 8, n = a->tokens * heads * (dim / 8);
    const int grid = (int)std::min<int64_t>((n + 255) / 256, (int64_t)sm_count() * 16);
    // (either type: 16 bits are copied)
    POS_CUDA(launch_dependent(attn_copy_kernel<__half>, grid, 256, 0, s,
                              static_cast<const __half *>(t.data), t.token_stride, t.head_stride,
                              a->tokens, (int)heads, (int)a->dim, reinterpret_cast<__half *>(*copy)));
    *out = {*copy, heads * dim, dim};
    *copy += attn_copy_bytes(a, heads);
    return POS_OK;
}

// [tokens][heads][dim] in boxes of 128 tokens of a head and 64 elements; what lies
// outside reads as zeros.
pos_status attn_map(CUtensorMap *map, const pos_attn *a, const AttnTensor &t, int64_t heads,
                    int32_t dim) {
    EncodeTiled encode;
    POS_TRY(encode_fn(&encode));
    const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)a->tokens};
    // (a stride over a single row or head is not used)
    const cuuint64_t strides[2] = {(cuuint64_t)(heads == 1 ? dim : t.head) * 2,
                                   (cuuint64_t)(a->tokens == 1 ? dim : t.token) * 2};
    const cuuint32_t box[3] = {64, 1, kTile}, ones[3] = {1, 1, 1};
    const CUresult r = encode(
        map, a->dtype == POS_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
        3, const_cast<void *>(t.p), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS)
        return fail(POS_ECUDA, "cuTensorMapEncodeTiled failed: " + std::to_string((int)r));
    return POS_OK;
}

int64_t attn_most_tiles(const pos_attn *a, int rows) {
    // (a sequence that has a tile has a token)
    return a->starts ? a->tokens / rows + std::min<int64_t>(a->sequences, a->tokens)
                     : (a->tokens + rows - 1) / rows;
}
int64_t attn_list_bytes(const pos_attn *a, int rows) {
    return a->starts ? 16 * (attn_most_tiles(a, rows) + 1) : 0;
}
pos_status attn_list(const pos_attn *a, int rows, char **at, cudaStream_t s, AttnParams *p) {
    if (!a->starts) return POS_OK;
    AttnListParams l = {};
    l.starts = a->starts, l.tokens = a->tokens, l.sequences = a->sequences, l.rows = rows;
    l.n_tiles = reinterpret_cast<int32_t *>(*at);
    l.tiles = reinterpret_cast<int4 *>(*at + 16);
    while ((a->tokens / rows >> l.shift) >= kBins) ++l.shift;
    l.bins = (int32_t)std::min<int64_t>(kBins, ((a->tokens / rows >> l.shift) + 32) / 32 * 32);
    *at += attn_list_bytes(a, rows);
    p->tiles = l.tiles, p->n_tiles = l.n_tiles;
    POS_CUDA(launch_dependent(attn_tiles_kernel, 1, kListThreads, 0, s, l));
    return POS_OK;
}
// Units of a head of a tile each, kMostUnits at most.
int attn_grid(const pos_attn *a, int rows, int64_t heads) {
    return (int)std::min<int64_t>(attn_most_tiles(a, rows) * heads, kMostUnits);
}

template <typename T>
static pos_status launch_forward(const pos_attn *a, const AttnParams &p, int grid, cudaStream_t s) {
    CUtensorMap q, k, v;
    POS_TRY(attn_map(&q, a, p.q, p.heads_q, p.dim));
    POS_TRY(attn_map(&k, a, p.k, p.heads_k, p.dim));
    POS_TRY(attn_map(&v, a, p.v, p.heads_k, p.dim));
    auto kern = attn_forward_kernel<T>;
    POS_TRY(ensure_smem(reinterpret_cast<const void *>(kern), kForwardSmem));
    POS_CUDA(launch_dependent(kern, std::min(grid, std::max(1, sm_count())), kForwardThreads,
                              kForwardSmem, s, q, k, v, p));
    return POS_OK;
}

static pos_status forward(const pos_attn *a, const pos_heads *x, AttnParams p, char *at,
                          cudaStream_t s) {
    const int64_t heads[3] = {a->heads_q, a->heads_k, a->heads_k};
    AttnTensor *to[3] = {&p.q, &p.k, &p.v};
    for (int i = 0; i < 3; ++i) POS_TRY(attn_input(a, x[i], heads[i], &at, s, to[i]));
    POS_TRY(attn_list(a, kForwardRows, &at, s, &p));
    const int grid = attn_grid(a, kForwardRows, a->heads_q);
    if (grid == 0) return POS_OK;
    return a->dtype == POS_BF16 ? launch_forward<__nv_bfloat16>(a, p, grid, s)
                                : launch_forward<__half>(a, p, grid, s);
}

}  // namespace pos

extern "C" pos_status poseidon_attn_forward(const pos_attn *attn, const pos_heads *x,
                                            const pos_heads *o, float *d_lse, void *stream) {
    using namespace pos;
    return guarded([&]() -> pos_status {
        AttnParams p = {};
        POS_TRY(check_attn(attn, &p));
        if (!x || !o) return fail(POS_EINVAL, "attention: NULL pointer");
        const int64_t heads[3] = {attn->heads_q, attn->heads_k, attn->heads_k};
        const char *names[3] = {"the queries", "the keys", "the values"};
        for (int i = 0; i < 3; ++i)
            POS_TRY(check_attn_tensor(attn, x[i], heads[i], names[i], false));
        POS_TRY(check_attn_tensor(attn, *o, attn->heads_q, "o", true));
        if (reinterpret_cast<uintptr_t>(d_lse) % 4)
            return fail(POS_EINVAL, "attention: misaligned lse");
        if (attn->tokens == 0 || attn->heads_q == 0) return POS_OK;
        p.out = o->data, p.out_token = o->token_stride, p.out_head = o->head_stride;
        p.out_vectors = aligned16(o->data) && o->token_stride % 8 == 0 && o->head_stride % 8 == 0;
        p.lse = d_lse;
        int64_t bytes = attn_list_bytes(attn, kForwardRows);
        for (int i = 0; i < 3; ++i)
            if (!attn_direct(attn, x[i], heads[i])) bytes += attn_copy_bytes(attn, heads[i]);
        const auto s = static_cast<cudaStream_t>(stream);
        void *scratch = nullptr;
        POS_TRY(attn_scratch(bytes, s, &scratch));
        const pos_status st = forward(attn, x, p, static_cast<char *>(scratch), s);
        const cudaError_t e = scratch ? cudaFreeAsync(scratch, s) : cudaSuccess;
        if (st != POS_OK) return st;
        return e == cudaSuccess ? POS_OK : cuda_fail(e, "attention scratch");
    });
}
