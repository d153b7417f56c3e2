// Attention of a batch that shares a prefix, over a paged cache in 8 bits (dl_prefix_attention).
//
// With s the scores in units of ln 2 and u the scales of the values, a query's output is sum of 2^s u V / sum of 2^s over the codes V
// of what it sees.  A scale is taken apart, u = c d, with c within 2^-40 .. 2^40 (2^50 for float16) and d = 1 for all but rows
// of zeros and values of very unusual sizes (see dl_value_scale).  The sums are taken piece by piece with a running reference r, within 2^8 of
// the largest s + log2 c so far:
//   w = 2^(s + log2 c - r) <= 2^8,   O += w d V,   l += w / c,
// both multiplied by 2^(r before - r) when r grows.  So the weights that go to the matrix units in 16 bits are at most 2^8 (times 2^lift,
// see there) whatever the scales are, and the codes go there as they are (each is a value of both 16-bit types): the only rounding on
// the way is that of w d.  As c is bounded, l is: a key adds at most 2^(8 + lift + 40) to it, 2^30 keys no more than 2^85; and as
// 32-bit numbers are whole down to 2^-126, no key drops out of l whose 2^s is above 2^-42 of the largest.
// Pieces of the same row are joined in the same manner, in a fixed order.
//
// The key axis is cut into pieces.  A piece of the prefix serves the queries of all sequences at once: they are the rows of
// one product.  A piece of a sequence's own tokens serves the query heads that share a head of the cache.  All pieces of
// both kinds are one launch; a second one joins each row's pieces.  (Joined in the launch that makes them, by the last workgroup of a row: slower
// everywhere, 32 sequences on a prefix of 2048 17 : 104 us, one with 5000 tokens 12.0 : 13.2; pieces then have to be seen across dies.)
//
// Measured (8 heads of 128, 64 query heads, bfloat16 on fp8, unless said otherwise): 256 sequences, one query each, on a prefix of 32768 393 us,
// 277 GFLOP, 0.70 PFLOP/s where a large matrix product reaches 1.3; 48 sequences with 5 queries on 16400 (4 heads, 28 query heads, float16 on
// int8) 107 us; 4 sequences with up to 131072 tokens of their own (554 MB) 133 us, 4.2 TB/s; one with 5000 (32 query heads) 11.4 us, two
// launches and the chain of length, table, codes, join.  Heads of 256: 256 sequences on 16384 564 us, 0.50 PFLOP/s, on one wavefront a SIMD and
// with 50 registers spilled.
#include "dl_codes.h"
#include "dl_internal.h"

namespace {

constexpr uint32_t ATT_THREADS = 256;
constexpr uint32_t ATT_WAVES = ATT_THREADS / 64;
constexpr uint32_t TILE = 32;                   // keys of a wavefront's step
constexpr uint32_t STEP = TILE * ATT_WAVES;     // pieces are cut at multiples of this

struct att_args {
    dl_cache_view c;
    const char *q;
    char *out;
    float *lse;
    const int32_t *prefix_pages, *pages, *lens, *q_lens;
    // What a piece leaves behind for the join, by part: part = piece * rows + row for a piece of the prefix, and behind those
    // (prefix_splits * rows) + unit * (rows of a sequence) + row in it for one of a sequence's own tokens.
    dl_f32x2 *rl;    // r and l
    float *partial;  // head_dim sums
    uint32_t *units; // per sequence with tokens of its own: its first unit, and how many it has
    int64_t q_seq, q_token, q_head, out_seq, out_token, out_head;  // bytes
    int64_t pages_stride;
    uint32_t prefix_tokens, own_most;  // own_most: max_pages * page_tokens
    uint32_t batch, q_tokens, q_heads, group;
    uint32_t rows;                     // batch * q_tokens * q_heads
    uint32_t prefix_tiles, prefix_splits, prefix_piece;
    uint32_t own_tiles, own_target;  // own_target: see own_unit; 0: a piece a sequence
    uint32_t narrow_shared, wide_shared;  // workgroups with a piece of the prefix, of either kind
    float scale;                       // times log2 e
};

__device__ __forceinline__ uint32_t own_len(const att_args &a, uint32_t b)
{
    return a.own_most ? min((uint32_t)max(a.lens[b], 0), a.own_most) : 0u;
}
__device__ __forceinline__ uint32_t queries(const att_args &a, uint32_t b)
{
    return a.q_lens ? min((uint32_t)max(a.q_lens[b], 0), a.q_tokens) : a.q_tokens;
}

// The sequences' own tokens are cut by their lengths, which only the device knows: into pieces of as many steps (of STEP keys)
// as share the steps of all sequences out over own_target pieces.  Sequences are then of one or more pieces, own_target + batch
// in all at most, and unit n is the n-th of them.  Every wavefront works this out from the lengths for itself.
// Not so batches of more than OWN_EVEN_MAX sequences, whose lengths are not added up, and tables with room for 2^31 steps and more,
// where 32 bits may not hold the sum: a piece a sequence, whatever its length.  A long one among many short ones is then a single
// workgroup's work in each head.
constexpr uint32_t OWN_EVEN_MAX = 1024;
constexpr uint32_t OWN_LEAST_STEPS = 2;

struct own_place {
    uint32_t b, piece, pieces, keys;  // sequence, which of its pieces, how many it has, and keys of one
};
// false: there is no such unit
__device__ __forceinline__ bool own_unit(const att_args &a, uint32_t unit, own_place *at)
{
    auto steps_of = [&](uint32_t b) { return (own_len(a, b) + STEP - 1u) / STEP; };
    if (!a.own_target) {
        if (unit >= a.batch || !own_len(a, unit)) return false;
        *at = {unit, 0, 1, 1u << 31};
        return true;
    }
    const uint32_t lane = threadIdx.x % 64u;
    uint32_t all = 0, here = 0;
    for (uint32_t b0 = 0; b0 < a.batch; b0 += 64u) {
        here = b0 + lane < a.batch ? steps_of(b0 + lane) : 0u;
        all += (uint32_t)__builtin_amdgcn_readlane((int)dl_sum_up_to(here), 63);
    }
    const uint32_t size = max((all + a.own_target - 1u) / a.own_target, OWN_LEAST_STEPS);
    uint32_t before = 0;
    for (uint32_t b0 = 0; b0 < a.batch; b0 += 64u) {
        if (a.batch > 64u) here = b0 + lane < a.batch ? steps_of(b0 + lane) : 0u;
        const uint32_t pieces = (here + size - 1u) / size, up_to = before + dl_sum_up_to(pieces);
        const unsigned long long where = __ballot(up_to > unit);
        if (where) {
            const int l = __ffsll((long long)where) - 1;
            at->b = b0 + (uint32_t)l;
            at->pieces = (uint32_t)__builtin_amdgcn_readlane((int)pieces, l);
            at->piece = unit - ((uint32_t)__builtin_amdgcn_readlane((int)up_to, l) - at->pieces);
            at->keys = size * STEP;
            return true;
        }
        before = (uint32_t)__builtin_amdgcn_readlane((int)up_to, 63);
    }
    return false;
}

// The largest over the lanes that hold the same query (16 and 32 apart), in all of them: halves and quarters change places.
__device__ __forceinline__ float largest_of_quarters(float x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(dl_bits<uint32_t>(x), dl_bits<uint32_t>(x), false, false);
    const float y = fmaxf(dl_bits<float>((uint32_t)a[0]), dl_bits<float>((uint32_t)a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(dl_bits<uint32_t>(y), dl_bits<uint32_t>(y), false, false);
    return fmaxf(dl_bits<float>((uint32_t)b[0]), dl_bits<float>((uint32_t)b[1]));
}

// What is the same for a workgroup's whole piece: NT tiles of 16 rows against the keys first .. end - 1 of one head.
struct piece_args {
    const int32_t *table;
    uint64_t part;  // of row 0
    uint32_t head, first, end;
    int32_t seen_by_all;  // keys up to this one are seen by every row
};

// Where a step's keys lie, as far as a lane (i, g) = (lane % 16, lane / 16) has to know: it holds parts of the keys 8 (i / 4) + 4 t +
// i % 4 (t = 0, 1), of the values of 8 g .. 8 g + 7, and the scale of key 8 g + i % 8 (the keys' where i < 8, the values' else).
// ALIGNED (pages hold a multiple of 8 tokens): eight keys 8 x .. 8 x + 7 lie in one page, and two pages are looked up, a step
// ahead of the loads that need them.
template <bool ALIGNED>
struct place {
    uint32_t base;
    uint32_t key_page, value_page;

    static __device__ __forceinline__ uint32_t clamped(const piece_args &p, uint32_t key) { return min(key, ALIGNED ? (p.end - 1u) & ~7u : p.end - 1u); }

    __device__ __forceinline__ void look_up(const att_args &a, const piece_args &p, uint32_t at)
    {
        base = at;
        if constexpr (ALIGNED) {
            const uint32_t lane = threadIdx.x % 64u;
            key_page = (uint32_t)p.table[dl_divide(clamped(p, at + 8u * (lane % 16u / 4u)), a.c.page)];
            value_page = (uint32_t)p.table[dl_divide(clamped(p, at + 8u * (lane / 16u)), a.c.page)];
        }
    }
    // key 8 x + in, in page `page` if that is known already: the offset of its row, and whether its page is one of the pool
    __device__ __forceinline__ uint64_t offset(const att_args &a, const piece_args &p, uint32_t x, uint32_t in, uint32_t page, uint32_t page_stride,
                                               uint32_t token_stride, uint64_t from, bool *alive) const
    {
        const uint32_t key = clamped(p, base + 8u * x + (ALIGNED ? 0u : in)), n = dl_divide(key, a.c.page);
        if constexpr (!ALIGNED) page = (uint32_t)p.table[n];
        *alive = page < a.c.pages;
        page = *alive ? page : 0u;
        return from + (uint64_t)page * page_stride + (uint64_t)(key - n * a.c.page.d + (ALIGNED ? in : 0u)) * token_stride;
    }
};

// (Where head_dim ends before DP, the lanes behind it load its end once more: those dims meet zeros in the queries, and sums that
// nobody stores.)
template <int DP>
struct tile_keys {
    dl_words<16> k[2][DP / 64];  // dims 64 s + 16 g ..
    float scale;
};
template <int DP>
struct tile_values {
    dl_words<DP / 16> v[8];  // dims DP / 16 * i ..
    uint32_t dead;        // bit e: the page of key 8 g + e
};

template <int DP, bool ALIGNED>
__device__ __forceinline__ void load_keys(const att_args &a, const piece_args &p, const place<ALIGNED> &at, tile_keys<DP> &td)
{
    const uint32_t lane = threadIdx.x % 64u, i = lane % 16u, g = lane / 16u, D = a.c.head_dim;
    const uint64_t from = (uint64_t)a.c.k + (uint64_t)p.head * a.c.head_stride;
    bool alive;
    uint64_t kp = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if (t == 0 || !ALIGNED)
            kp = at.offset(a, p, i / 4u, i % 4u + 4u * t, at.key_page, a.c.page_stride, a.c.token_stride, from, &alive);
        else
            kp += 4ull * a.c.token_stride;
#pragma unroll
        for (int s = 0; s < DP / 64; ++s) td.k[t][s] = dl_load_words<16>((const char *)kp + min(16u * g + 64u * s, D - 16u));
    }
    const uint64_t scales = (uint64_t)(i < 8u ? a.c.k_scale : a.c.v_scale) + (uint64_t)p.head * a.c.scale_head_stride;
    td.scale = *(const float *)at.offset(a, p, g, i % 8u, at.value_page, a.c.scale_page_stride, a.c.scale_token_stride, scales, &alive);
}

template <int DP, bool ALIGNED>
__device__ __forceinline__ void load_values(const att_args &a, const piece_args &p, const place<ALIGNED> &at, tile_values<DP> &td)
{
    constexpr int VB = DP / 16;
    const uint32_t lane = threadIdx.x % 64u, i = lane % 16u, g = lane / 16u, D = a.c.head_dim;
    const uint64_t from = (uint64_t)a.c.v + (uint64_t)p.head * a.c.head_stride + min(VB * i, D - VB);
    bool alive;
    uint64_t vp = 0;
    td.dead = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (e == 0 || !ALIGNED) {
            vp = at.offset(a, p, g, (uint32_t)e, at.value_page, a.c.page_stride, a.c.token_stride, from, &alive);
            if (!alive) td.dead |= ALIGNED ? 0xFFu : 1u << e;
        } else {
            vp += a.c.token_stride;
        }
        td.v[e] = dl_load_words<VB>((const char *)vp);
    }
}

template <int DP, int NT>
struct sums {
    dl_f32x4 o[NT][DP / 16];  // rows of the product are dims (DP / 16 * (4 g + j) + t in lane (i, g)), its columns queries (i)
    float r[NT], low[NT];     // the reference, the same in all lanes of a query; low: less Q::lift, finite
    float l[NT];              // a lane's share
};

// (A narrow piece is bound by its loads.  Tiles of 16 rows fit a handful of queries with the least waste.  Wavefronts take different keys,
// so each loads what it needs straight into registers, no codes go through LDS, and nothing waits for another wavefront before the
// end.  Loads a step ahead: one sequence with 5000 tokens 36.8 -> 11.6 us, 4 with up to 131072 529 -> 198; pieces by length on the device
// 198 -> 132.)
//
// A step: 32 keys against NT tiles of 16 rows.  whole: all of them are seen by all.  The next step's keys are loaded as
// soon as the scores have been taken, its values after the sums, into the same registers.
template <class Q, class C, int DP, int NT, bool ALIGNED>
__device__ __forceinline__ void attend_tile(const att_args &a, const piece_args &p, const place<ALIGNED> &at, const place<ALIGNED> &then, bool whole,
                                            tile_keys<DP> &tk, tile_values<DP> &tv, const dl_u32x4 (&qf)[NT][DP / 32], const int32_t (&last)[NT], sums<DP, NT> &acc,
                                            float (&scales)[4][TILE])
{
    constexpr int VB = DP / 16, STEPS = DP / 32;
    const uint32_t lane = threadIdx.x % 64u, i = lane % 16u, g = lane / 16u, base = at.base;
    uint32_t here = 0;  // bit e: key 8 g + e is in a page of the pool, and of the piece
    bool taken_apart;   // some key's d is not 1 (what nobody sees counts as well, and does no harm)
    {
        if (!whole) {
            const uint32_t left = p.end - min(p.end, base + 8u * g);
            here = (left >= 8u ? 0xFFu : (1u << left) - 1u) & ~tv.dead;
        }
        const uint32_t key = 8u * g + i % 8u;
        const dl_value_scale<Q> u(tk.scale);
        if (i < 8u) {
            scales[0][key] = tk.scale * a.scale;
        } else {
            scales[1][key] = u.log2_c();
            scales[2][key] = u.over_c();
            scales[3][key] = u.d;
        }
        taken_apart = __any(i >= 8u && u.d != 1.0f);
    }
    // scores: the product's rows are keys (8 g + 4 t + j in lane (i, g)), its columns queries (i)
    dl_f32x4 s[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = dl_f32x4{0, 0, 0, 0};
#pragma unroll
    for (int st = 0; st < STEPS; ++st)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const dl_u32x2 x = C::template spread<Q>(tk.k[t][st / 2].w[2 * (st % 2)]), y = C::template spread<Q>(tk.k[t][st / 2].w[2 * (st % 2) + 1]);
            const dl_u32x4 kf = {x[0], x[1], y[0], y[1]};
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n][t] = Q::mfma16(kf, qf[n][st], s[n][t]);
        }
    if (then.base < p.end) load_keys<DP, ALIGNED>(a, p, then, tk);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    float ks[8], lu[8], iu[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        ks[e] = scales[0][8u * g + e];
        lu[e] = scales[1][8u * g + e];
        iu[e] = scales[2][8u * g + e];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    dl_u32x4 pf[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float x[8], top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(s[n][e / 4][e % 4], ks[e], lu[e]);
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!(here >> e & 1u) || (int32_t)(base + 8u * g + e) > last[n]) x[e] = -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, x[e]);
        // The reference follows the largest only where that is 2^8 times above it: most steps then neither ask the other
        // lanes nor touch the sums, and a weight is at most 2^(8 + lift), which both types hold.
        if (__any(top > acc.r[n] + 8.0f)) {
            const float now = fmaxf(acc.r[n], largest_of_quarters(top));
            const float ref = now == -INFINITY ? 0.0f : now;
            const float fade = __builtin_amdgcn_exp2f(acc.r[n] - ref);
            acc.r[n] = now;
            acc.low[n] = ref - Q::lift;
            acc.l[n] *= fade;
#pragma unroll
            for (int t = 0; t < DP / 16; ++t) acc.o[n][t] *= fade;
        }
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            w[e] = __builtin_amdgcn_exp2f(x[e] - acc.low[n]);
            acc.l[n] = fmaf(w[e], iu[e], acc.l[n]);
        }
        if (taken_apart) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = Q::in_range(w[e] * scales[3][8u * g + e]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        pf[n] = dl_u32x4{Q::pack(w[0], w[1]), Q::pack(w[2], w[3]), Q::pack(w[4], w[5]), Q::pack(w[6], w[7])};
    }
    if (!whole) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!(here >> e & 1u)) tv.v[e] = dl_words<VB>{};
    }
#pragma unroll
    for (int q4 = 0; q4 < VB / 4; ++q4) {
        // four keys' four dims each, turned to four dims' four keys each
        dl_u32x2 half[2][4];  // [keys 0 .. 3 and 4 .. 7][dim]: four elements
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t w0 = tv.v[4 * h].w[q4], w1 = tv.v[4 * h + 1].w[q4], w2 = tv.v[4 * h + 2].w[q4], w3 = tv.v[4 * h + 3].w[q4];
            const uint32_t a01 = __builtin_amdgcn_perm(w1, w0, 0x05010400u), a23 = __builtin_amdgcn_perm(w3, w2, 0x05010400u);
            const uint32_t b01 = __builtin_amdgcn_perm(w1, w0, 0x07030602u), b23 = __builtin_amdgcn_perm(w3, w2, 0x07030602u);
            half[h][0] = C::template spread<Q>(__builtin_amdgcn_perm(a23, a01, 0x05040100u));
            half[h][1] = C::template spread<Q>(__builtin_amdgcn_perm(a23, a01, 0x07060302u));
            half[h][2] = C::template spread<Q>(__builtin_amdgcn_perm(b23, b01, 0x05040100u));
            half[h][3] = C::template spread<Q>(__builtin_amdgcn_perm(b23, b01, 0x07060302u));
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const dl_u32x4 vf = {half[0][t][0], half[0][t][1], half[1][t][0], half[1][t][1]};
#pragma unroll
            for (int n = 0; n < NT; ++n) acc.o[n][4 * q4 + t] = Q::mfma16(vf, pf[n], acc.o[n][4 * q4 + t]);
        }
    }
    if (then.base < p.end) load_values<DP, ALIGNED>(a, p, then, tv);
}

template <int DP, int NT>
struct narrow_lds {
    float scales[ATT_WAVES][4][TILE];
    float joined[2][NT * DP / 16 * 4 + 2 * NT][64];
};

template <class Q, class C, int DP, int NT, bool ALIGNED>
__device__ __forceinline__ void attend(const att_args &a, const piece_args &p, const char *const (&qrow)[NT], const int32_t (&last)[NT],
                                       const uint32_t (&row)[NT], const bool (&store)[NT], narrow_lds<DP, NT> &lds)
{
    constexpr int VB = DP / 16, STEPS = DP / 32;
    const uint32_t lane = threadIdx.x % 64u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
    const uint32_t g = lane / 16u, D = a.c.head_dim;

    // (pages are looked up two steps ahead: loads come back in order, so one that is issued behind the last values' would
    // be known only once those have arrived)
    place<ALIGNED> at, then, after;
    at.look_up(a, p, p.first + wave * TILE);
    then.look_up(a, p, p.first + wave * TILE + STEP);
    tile_keys<DP> tk;
    tile_values<DP> tv;
    if (at.base < p.end) {
        load_keys<DP, ALIGNED>(a, p, at, tk);
        load_values<DP, ALIGNED>(a, p, at, tv);
    }

    // queries: lane (i, g) holds dims 64 s + 16 g .. of row i, eight a step
    dl_u32x4 qf[NT][STEPS];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const uint32_t d = 64u * (s / 2u) + 16u * g + 8u * (s % 2u);
            qf[n][s] = d < D ? dl_load_at<dl_u32x4>(qrow[n] + 2u * d) : dl_u32x4{0, 0, 0, 0};
        }

    sums<DP, NT> acc;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        acc.r[n] = -INFINITY;
        acc.low[n] = -Q::lift;
        acc.l[n] = 0.0f;
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) acc.o[n][t] = dl_f32x4{0, 0, 0, 0};
    }

    for (; at.base < p.end; at = then, then = after) {
        after.look_up(a, p, at.base + 2 * STEP);
        bool whole = false;
        if (ALIGNED && (int32_t)(at.base + TILE - 1u) <= p.seen_by_all) whole = !__any(at.key_page >= a.c.pages);
        attend_tile<Q, C, DP, NT, ALIGNED>(a, p, at, then, whole, tk, tv, qf, last, acc, lds.scales[wave]);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        acc.l[n] += __shfl_xor(acc.l[n], 16);
        acc.l[n] += __shfl_xor(acc.l[n], 32);
    }
    // the wavefronts' sums, two by two: 2 and 3 to 0 and 1, then 1 to 0
#pragma unroll
    for (uint32_t half = ATT_WAVES / 2; half; half /= 2) {
        if (wave >= half && wave < 2 * half) {
            float(*to)[64] = lds.joined[wave - half];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                to[2 * n][lane] = acc.r[n];
                to[2 * n + 1][lane] = acc.l[n];
#pragma unroll
                for (int t = 0; t < DP / 16; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) to[2 * NT + (n * (DP / 16) + t) * 4 + j][lane] = acc.o[n][t][j];
            }
        }
        __syncthreads();
        if (wave < half) {
            const float(*from)[64] = lds.joined[wave];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float r2 = from[2 * n][lane], now = fmaxf(acc.r[n], r2), ref = now == -INFINITY ? 0.0f : now;
                const float f = __builtin_amdgcn_exp2f(acc.r[n] - ref), f2 = __builtin_amdgcn_exp2f(r2 - ref);
                acc.r[n] = now;
                acc.l[n] = acc.l[n] * f + from[2 * n + 1][lane] * f2;
#pragma unroll
                for (int t = 0; t < DP / 16; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc.o[n][t][j] = acc.o[n][t][j] * f + from[2 * NT + (n * (DP / 16) + t) * 4 + j][lane] * f2;
            }
        }
        __syncthreads();
    }
    if (wave) return;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (!store[n]) continue;
        const uint64_t at = p.part + row[n];
        if (g == 0) a.rl[at] = dl_f32x2{acc.r[n], acc.l[n]};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t d = VB * (4u * g + j);
            if (d >= D) continue;
            float *to = a.partial + at * D + d;
#pragma unroll
            for (int t = 0; t < VB; t += 4)
                *(dl_f32x4 *)(to + t) = dl_f32x4{acc.o[n][t][j], acc.o[n][t + 1][j], acc.o[n][t + 2][j], acc.o[n][t + 3][j]};
        }
    }
}

// A workgroup's piece where few queries share it: NT * 16 rows, each wavefront every fourth tile of 32 keys.
template <class Q, class C, int DP, int NT, bool ALIGNED>
__device__ __forceinline__ void narrow_piece(const att_args &a, uint32_t block, narrow_lds<DP, NT> &lds)
{
    const uint32_t i = threadIdx.x % 16u;
    const char *qrow[NT];
    int32_t last[NT];
    uint32_t row[NT];
    bool store[NT];
    const uint32_t heads = a.c.heads, seq_rows = a.q_tokens * a.group;
    const bool prefix = block < a.narrow_shared;
    const uint32_t x = prefix ? block : block - a.narrow_shared;
    const uint32_t tiles = prefix ? a.prefix_tiles : a.own_tiles, head = x % heads, tile = x / heads % tiles, unit = x / heads / tiles;
    uint32_t b0 = 0, rows;
    int32_t own_last = 0;  // of query 0
    piece_args p;
    p.head = head;
    if (prefix) {
        p.first = unit * a.prefix_piece;
        p.end = min(p.first + a.prefix_piece, a.prefix_tokens);
        p.table = a.prefix_pages;
        p.seen_by_all = (int32_t)p.end - 1;
        p.part = (uint64_t)unit * a.rows;
        rows = a.batch * seq_rows;
    } else {
        own_place own;
        if (!own_unit(a, unit, &own)) return;
        b0 = own.b;
        const uint32_t len = own_len(a, b0);
        p.first = own.piece * own.keys;
        p.end = min(p.first + own.keys, len);
        p.table = a.pages + b0 * a.pages_stride;
        p.part = (uint64_t)a.prefix_splits * a.rows + (uint64_t)unit * (a.q_tokens * a.q_heads);
        rows = seq_rows;
        own_last = (int32_t)len - (int32_t)queries(a, b0);
        p.seen_by_all = min((int32_t)p.end - 1, own_last + (int32_t)(tile * NT * 16u / a.group));
        if (head == 0 && tile == 0 && own.piece == 0 && threadIdx.x == 0) {
            a.units[2 * b0] = unit;
            a.units[2 * b0 + 1] = own.pieces;
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        uint32_t at = (tile * NT + n) * 16u + i;
        store[n] = at < rows;
        at = min(at, rows - 1u);
        const uint32_t b = b0 + at / seq_rows, in = at % seq_rows, j = in / a.group, h = head * a.group + in - j * a.group;
        qrow[n] = a.q + b * a.q_seq + j * a.q_token + h * a.q_head;
        row[n] = ((b - b0) * a.q_tokens + j) * a.q_heads + h;
        last[n] = prefix ? (int32_t)p.end - 1 : min((int32_t)p.end - 1, own_last + (int32_t)j);
    }
    attend<Q, C, DP, NT, ALIGNED>(a, p, qrow, last, row, store, lds);
}

// The prefix against many queries.  A workgroup has 128 rows of the batch (32 a wavefront)
// and walks the keys of its piece in tiles of 64, which its wavefronts share: the codes are turned into elements of Q once, on
// their way into LDS, keys as rows and values transposed (by byte permutes while they are bytes), so that every operand of the
// 32 x 32 x 16 products is one 16-byte read.  While a tile is worked on, the next one's codes are on their way to registers and the
// pages of the one after it are looked up; a barrier a tile.
//
// What bounds it is the sum of the pipes: of the call's cycles, vector instructions (scales, exponentials, sums of weights, turning codes) are issued in
// 49 %, the matrix units work in 29 %, LDS in 44 %, and no order of the parts overlapped them better.  The largest part that could go is
// turning codes, which each of 16 tiles of rows does again: without it (and with wrong results) 291 us of 375.  256 sequences on a prefix of 32768 (see
// the top), this : 64 rows a wavefront (one a SIMD) 393 : 486 us, workgroups of 256 rows 416 : 430, two groups of wavefronts that take
// turns 393 : 409, keys in the lanes of the scores 393 : 427; scores beside the next tile's conversion and operands read a group
// ahead 393 : 380, which short prefixes lose again (32 sequences on 2048 17.8 : 18.7).
//
// Operands lie in rows of 16-byte pieces, whose places are exchanged (by an exclusive or with the row's number) so that eight
// neighbouring lanes use all banks, in reads and in writes.
constexpr uint32_t WIDE_KEYS = 64;

template <int DP>
struct alignas(16) wide_tile {  // (reads of 16 bytes that lie at fours take twice as long)
    uint32_t k[WIDE_KEYS * DP / 2];  // key, dim
    uint32_t v[WIDE_KEYS * DP / 2];  // dim, key: of each 16 keys 0 - 3, 8 - 11, 4 - 7, 12 - 15
    float ks[WIDE_KEYS], lu[WIDE_KEYS], iu[WIDE_KEYS], d[WIDE_KEYS];
    uint32_t taken_apart;  // (as in attend_tile)
};
template <int DP>
struct wide_lds {
    wide_tile<DP> tiles[2];
    uint64_t rows_at[2][WIDE_KEYS];  // offsets of the codes' rows
    uint64_t alive_at[2];            // bit k: key k is one of the piece, in a page of the pool
};

template <class Q, class C, int DP>
__device__ __forceinline__ void wide_piece(const att_args &a, uint32_t block, wide_lds<DP> &lds)
{
    constexpr uint32_t PIECES = DP / 8;                          // 16-byte pieces of a key's row
    constexpr uint32_t K_LOADS = WIDE_KEYS * PIECES / ATT_THREADS;  // of 8 codes
    constexpr uint32_t V_ITEMS = 8 * (DP / 4);                   // 8 keys (half of 16) x 4 dims
    constexpr uint32_t V_LOADS = (V_ITEMS + ATT_THREADS - 1) / ATT_THREADS;
    auto &tiles = lds.tiles;
    auto &rows_at = lds.rows_at;
    auto &alive_at = lds.alive_at;
    const uint32_t lane = threadIdx.x % 64u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
    const uint32_t i = lane % 32u, half = lane / 32u, D = a.c.head_dim;
    const uint32_t heads = a.c.heads, seq_rows = a.q_tokens * a.group, all_rows = a.batch * seq_rows;
    const uint32_t head = block % heads, piece = block / heads % a.prefix_splits, tile = block / heads / a.prefix_splits;
    const uint32_t first = piece * a.prefix_piece, end = min(first + a.prefix_piece, a.prefix_tokens);
    const char *const k_from = a.c.k + (int64_t)head * a.c.head_stride, *const v_from = a.c.v + (int64_t)head * a.c.head_stride;

    const uint32_t my = (tile * ATT_WAVES + wave) * 32u + i, at_row = min(my, all_rows - 1u);
    const uint32_t b = at_row / seq_rows, in_b = at_row - b * seq_rows, j = in_b / a.group, h = head * a.group + in_b - j * a.group;
    const char *const q = a.q + b * a.q_seq + j * a.q_token + h * a.q_head;
    dl_u32x4 qf[DP / 16];
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) qf[s] = 16u * s < D ? dl_load_at<dl_u32x4>(q + 2u * (16u * s + 8u * half)) : dl_u32x4{0, 0, 0, 0};

    // a key's page: looked up by the first two wavefronts, for the keys' and the values' scales; the first hands the rows on
    uint32_t looked_up = 0;
    auto look_up = [&](uint32_t base) {
        if (wave < 2) looked_up = (uint32_t)a.prefix_pages[dl_divide(min(base + lane, end - 1u), a.c.page)];
    };
    float scale = 0.0f;
    bool alive = false;
    auto hand_on = [&](uint32_t base, uint32_t to) {  // what was looked up for the tile at base
        if (wave < 2) {
            const uint32_t key = min(base + lane, end - 1u), in = key - dl_divide(key, a.c.page) * a.c.page.d;
            alive = base + lane < end && looked_up < a.c.pages;
            const uint64_t page = looked_up < a.c.pages ? looked_up : 0u;
            if (wave == 0) {
                rows_at[to][lane] = page * a.c.page_stride + (uint64_t)in * a.c.token_stride;
                const unsigned long long all = __ballot(alive);
                if (lane == 0) alive_at[to] = all;
            }
            scale = *(const float *)((const char *)(wave == 0 ? a.c.k_scale : a.c.v_scale) + (int64_t)head * a.c.scale_head_stride +
                                     page * a.c.scale_page_stride + (uint64_t)in * a.c.scale_token_stride);
        }
    };
    dl_words<8> kw[K_LOADS];
    uint32_t vw[V_LOADS][8];
    auto load = [&](uint32_t from) {
#pragma unroll
        for (uint32_t x = 0; x < K_LOADS; ++x) {
            const uint32_t at = threadIdx.x + x * ATT_THREADS, key = at / PIECES, d = at % PIECES * 8u;
            kw[x] = dl_load_words<8>(k_from + rows_at[from][key] + min(d, D - 8u));
        }
#pragma unroll
        for (uint32_t x = 0; x < V_LOADS; ++x) {
            const uint32_t at = threadIdx.x + x * ATT_THREADS, d = at % (DP / 4) * 4u, part = at / (DP / 4) % 8u;
            const uint32_t key = part / 2u * 16u + part % 2u * 4u;
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e)
                vw[x][e] = dl_load_at<uint32_t>(v_from + rows_at[from][key + (e & 3u) + (e >> 2) * 8u] + min(d, D - 4u));
        }
    };
    auto put = [&](uint32_t from) {  // what has been loaded, into the tile
        wide_tile<DP> &to = tiles[from];
        const uint32_t all_lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)alive_at[from]);
        const uint32_t all_hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(alive_at[from] >> 32));
        const uint64_t all = (uint64_t)all_hi << 32 | all_lo;
        if (all != ~0ull) {  // what is none counts as zero
#pragma unroll
            for (uint32_t x = 0; x < K_LOADS; ++x)
                if (!(all >> ((threadIdx.x + x * ATT_THREADS) / PIECES) & 1u)) kw[x] = dl_words<8>{};
#pragma unroll
            for (uint32_t x = 0; x < V_LOADS; ++x) {
                const uint32_t part = (threadIdx.x + x * ATT_THREADS) / (DP / 4) % 8u, key = part / 2u * 16u + part % 2u * 4u;
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e)
                    if (!(all >> (key + (e & 3u) + (e >> 2) * 8u) & 1u)) vw[x][e] = 0;
            }
        }
#pragma unroll
        for (uint32_t x = 0; x < K_LOADS; ++x) {
            const uint32_t at = threadIdx.x + x * ATT_THREADS, key = at / PIECES, c = at % PIECES;
            const dl_u32x2 p = C::template spread<Q>(kw[x].w[0]), q = C::template spread<Q>(kw[x].w[1]);
            *(dl_u32x4 *)&to.k[(key * PIECES + (c ^ (key & 7u))) * 4u] = dl_u32x4{p[0], p[1], q[0], q[1]};
        }
#pragma unroll
        for (uint32_t x = 0; x < V_LOADS; ++x) {
            const uint32_t at = threadIdx.x + x * ATT_THREADS, d = at % (DP / 4) * 4u, part = at / (DP / 4) % 8u;
            if (V_ITEMS % ATT_THREADS && at >= V_ITEMS) continue;
            dl_u32x2 four[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t w0 = vw[x][4 * h], w1 = vw[x][4 * h + 1], w2 = vw[x][4 * h + 2], w3 = vw[x][4 * h + 3];
                const uint32_t a01 = __builtin_amdgcn_perm(w1, w0, 0x05010400u), a23 = __builtin_amdgcn_perm(w3, w2, 0x05010400u);
                const uint32_t b01 = __builtin_amdgcn_perm(w1, w0, 0x07030602u), b23 = __builtin_amdgcn_perm(w3, w2, 0x07030602u);
                four[h][0] = C::template spread<Q>(__builtin_amdgcn_perm(a23, a01, 0x05040100u));
                four[h][1] = C::template spread<Q>(__builtin_amdgcn_perm(a23, a01, 0x07060302u));
                four[h][2] = C::template spread<Q>(__builtin_amdgcn_perm(b23, b01, 0x05040100u));
                four[h][3] = C::template spread<Q>(__builtin_amdgcn_perm(b23, b01, 0x07060302u));
            }
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                const uint32_t r = d + j, c = part ^ ((r & 7u) ^ (r >> 3 & 3u));
                *(dl_u32x4 *)&to.v[(r * 8u + c) * 4u] = dl_u32x4{four[0][j][0], four[0][j][1], four[1][j][0], four[1][j][1]};
            }
        }
        if (wave == 0) {
            to.ks[lane] = alive ? scale * a.scale : 0.0f;
        } else if (wave == 1) {
            const dl_value_scale<Q> u(scale);
            to.lu[lane] = alive ? u.log2_c() : -INFINITY;
            to.iu[lane] = alive ? u.over_c() : 0.0f;
            to.d[lane] = u.d;
            const bool some = __any(u.d != 1.0f);
            if (lane == 0) to.taken_apart = some;
        }
    };

    // Values times what their scales left out, in LDS, by all threads, before anybody works on the tile.  (At the weights instead, by a branch
    // between them and the products: 256 sequences on 32768 402 us, this 393, neither 387.)
    auto apart = [&](wide_tile<DP> &t) {
#pragma unroll 1
        for (uint32_t at = threadIdx.x; at < DP * 8u; at += ATT_THREADS) {
            const uint32_t r = at / 8u, part = at % 8u, key = part / 2u * 16u + part % 2u * 4u;
            uint32_t *const to = &t.v[(r * 8u + (part ^ ((r & 7u) ^ (r >> 3 & 3u)))) * 4u];
#pragma unroll
            for (uint32_t x = 0; x < 4; ++x) {
                const float *const d = &t.d[key + x / 2u * 8u + x % 2u * 2u];
                to[x] = Q::pack(Q::in_range(Q::lo(to[x]) * d[0]), Q::in_range(Q::hi(to[x]) * d[1]));
            }
        }
        __syncthreads();
    };

    dl_f32x16 o[DP / 32];
    float r = -INFINITY, low = -Q::lift, l = 0.0f;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] = 0.0f;

    look_up(first);
    hand_on(first, 0);
    __syncthreads();
    load(0);
    look_up(first + WIDE_KEYS);
    put(0);
    hand_on(first + WIDE_KEYS, 1);
    __syncthreads();
    uint32_t now = 0;
    for (uint32_t base = first; base < end; base += WIDE_KEYS, now ^= 1u) {
        const bool more = base + WIDE_KEYS < end;
        if (__builtin_amdgcn_readfirstlane((int)tiles[now].taken_apart)) apart(tiles[now]);
        if (more) {
            load(now ^ 1u);
            look_up(base + 2 * WIDE_KEYS);
        }
        const wide_tile<DP> &in = tiles[now];
#pragma unroll 1
        for (uint32_t kb = 0; kb < 2; ++kb) {
            // scores: rows of the product are keys (32 kb + 8 (e / 4) + 4 half + e % 4), its columns queries (i)
            dl_f32x16 s;
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = 0.0f;
            const uint32_t key = 32u * kb + i;
#pragma unroll
            for (uint32_t st = 0; st < DP / 16; ++st) {
                const dl_u32x4 kf = *(const dl_u32x4 *)&in.k[(key * PIECES + ((2u * st + half) ^ (key & 7u))) * 4u];
                s = Q::mfma32(kf, qf[st], s);
            }
            float ks[16], lu[16], iu[16];
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const uint32_t k4 = 32u * kb + 2u * e + 4u * half;
                const dl_f32x4 x = *(const dl_f32x4 *)&in.ks[k4], y = *(const dl_f32x4 *)&in.lu[k4], z = *(const dl_f32x4 *)&in.iu[k4];
#pragma unroll
                for (int f = 0; f < 4; ++f) ks[e + f] = x[f], lu[e + f] = y[f], iu[e + f] = z[f];
            }
            float top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[e] = fmaf(s[e], ks[e], lu[e]);
                top = fmaxf(top, s[e]);
            }
            if (__any(top > r + 8.0f)) {  // (as in attend_tile)
                const auto swapped = __builtin_amdgcn_permlane32_swap(dl_bits<uint32_t>(top), dl_bits<uint32_t>(top), false, false);
                top = fmaxf(dl_bits<float>((uint32_t)swapped[0]), dl_bits<float>((uint32_t)swapped[1]));
                const float most = fmaxf(r, top), ref = most == -INFINITY ? 0.0f : most, fade = __builtin_amdgcn_exp2f(r - ref);
                r = most;
                low = ref - Q::lift;
                l *= fade;
#pragma unroll
                for (int t = 0; t < DP / 32; ++t) o[t] *= fade;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[e] = __builtin_amdgcn_exp2f(s[e] - low);
                l = fmaf(s[e], iu[e], l);
            }
            dl_u32x4 pf[2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) pf[t][e] = Q::pack(s[8 * t + 2 * e], s[8 * t + 2 * e + 1]);
            // sums: rows of the product are dims, its columns queries
#pragma unroll
            for (uint32_t t = 0; t < 2; ++t)
#pragma unroll
                for (uint32_t dt = 0; dt < DP / 32; ++dt) {
                    const uint32_t d = 32u * dt + i, c = (4u * kb + 2u * t + half) ^ ((d & 7u) ^ (d >> 3 & 3u));
                    const dl_u32x4 vf = *(const dl_u32x4 *)&in.v[(d * 8u + c) * 4u];
                    o[dt] = Q::mfma32(vf, pf[t], o[dt]);
                }
        }
        if (more) {
            put(now ^ 1u);
            hand_on(base + 2 * WIDE_KEYS, now);
        }
        __syncthreads();
    }
    l += __shfl_xor(l, 32);
    if (my >= all_rows) return;
    const uint64_t at = (uint64_t)piece * a.rows + (b * a.q_tokens + j) * a.q_heads + h;
    if (half == 0) a.rl[at] = dl_f32x2{r, l};
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const uint32_t d = 32u * t + 2u * e + 4u * half;
            if (d < D) *(dl_f32x4 *)(a.partial + at * D + d) = dl_f32x4{o[t][e], o[t][e + 1], o[t][e + 2], o[t][e + 3]};
        }
}

// All pieces, of the prefix and of the sequences' own tokens.  WIDE: those of the prefix are wide ones (a.wide_shared workgroups).
template <class Q, class C, int DP, int NT, bool ALIGNED, bool WIDE>
__global__ void __launch_bounds__(ATT_THREADS, DP <= 128 ? 2 : 1) dl_attention_kernel(const att_args a)
{
    constexpr size_t NARROW = sizeof(narrow_lds<DP, NT>), BYTES = WIDE && sizeof(wide_lds<DP>) > NARROW ? sizeof(wide_lds<DP>) : NARROW;
    __shared__ __align__(16) char lds[BYTES];
    if constexpr (WIDE) {
        if (blockIdx.x < a.wide_shared) return wide_piece<Q, C, DP>(a, blockIdx.x, *(wide_lds<DP> *)lds);
        narrow_piece<Q, C, DP, NT, ALIGNED>(a, blockIdx.x - a.wide_shared, *(narrow_lds<DP, NT> *)lds);
    } else {
        narrow_piece<Q, C, DP, NT, ALIGNED>(a, blockIdx.x, *(narrow_lds<DP, NT> *)lds);
    }
}

// Joins the pieces of a row: a read of what they left, 3 us for a few rows, 13 us for 16384 rows of 4 pieces of 128 (35 MB).  WAVES wavefronts
// a row share them out; in a wavefront DP / 4 lanes hold a piece's sums, four
// each, so 256 / DP pieces are looked at together and four times as many are on their way.
template <class Q, int DP, int WAVES>
__global__ void __launch_bounds__(ATT_THREADS) dl_attention_join_kernel(const att_args a)
{
    constexpr uint32_t LANES = DP / 4, SIDE = 64 / LANES, AHEAD = 4;
    const uint32_t lane = threadIdx.x % 64u, wave = threadIdx.x / 64u, part = lane / LANES + (WAVES > 1 ? wave * SIDE : 0u);
    const uint32_t block = blockIdx.y * gridDim.x + blockIdx.x, row = WAVES > 1 ? block : block * ATT_WAVES + wave;
    if (row >= a.rows) return;
    const uint32_t h = row % a.q_heads, bj = row / a.q_heads, b = bj / a.q_tokens, j = bj - b * a.q_tokens, D = a.c.head_dim;
    uint32_t pieces = 0;
    uint64_t own_part = 0;  // that of the first piece of own tokens, less prefix_splits pieces
    const uint32_t unit = a.units[2 * b], units = a.units[2 * b + 1];  // (on their way with the length that says whether they are anything)
    if (j < queries(a, b)) {
        pieces = a.prefix_splits;
        if (own_len(a, b)) {
            own_part = (uint64_t)a.prefix_splits * a.rows + (row - b * a.q_tokens * a.q_heads) +
                       ((uint64_t)unit - a.prefix_splits) * (a.q_tokens * a.q_heads);
            pieces += units;
        }
    }
    const uint32_t d0 = 4u * (lane % LANES);
    float r = -INFINITY, l = 0.0f;
    dl_f32x4 o = {0, 0, 0, 0};
    for (uint32_t p0 = part; p0 < pieces; p0 += SIDE * WAVES * AHEAD) {
        dl_f32x2 rl[AHEAD];
        dl_f32x4 x[AHEAD];
#pragma unroll
        for (uint32_t k = 0; k < AHEAD; ++k) {
            const uint32_t p = p0 + k * SIDE * WAVES, q = min(p, pieces - 1u);
            const uint64_t at = q < a.prefix_splits ? (uint64_t)q * a.rows + row : own_part + (uint64_t)q * (a.q_tokens * a.q_heads);
            rl[k] = a.rl[at];
            x[k] = d0 < D ? *(const dl_f32x4 *)(a.partial + at * D + d0) : dl_f32x4{0, 0, 0, 0};
            if (p >= pieces) rl[k] = dl_f32x2{-INFINITY, 0.0f}, x[k] = dl_f32x4{0, 0, 0, 0};
        }
        float now = r;
#pragma unroll
        for (uint32_t k = 0; k < AHEAD; ++k) now = fmaxf(now, rl[k][0]);
        const float ref = now == -INFINITY ? 0.0f : now, fade = __builtin_amdgcn_exp2f(r - ref);
        r = now;
        l *= fade;
        o *= fade;
#pragma unroll
        for (uint32_t k = 0; k < AHEAD; ++k) {
            const float f = __builtin_amdgcn_exp2f(rl[k][0] - ref);
            l = fmaf(rl[k][1], f, l);
            o += x[k] * f;
        }
    }
    auto merge = [&](float r2, float l2, dl_f32x4 o2) {
        const float now = fmaxf(r, r2), ref = now == -INFINITY ? 0.0f : now;
        const float f = __builtin_amdgcn_exp2f(r - ref), f2 = __builtin_amdgcn_exp2f(r2 - ref);
        r = now;
        l = l * f + l2 * f2;
        o = o * f + o2 * f2;
    };
#pragma unroll
    for (uint32_t d = LANES; d < 64u; d *= 2) {
        dl_f32x4 o2;
#pragma unroll
        for (int t = 0; t < 4; ++t) o2[t] = __shfl_xor(o[t], (int)d);
        merge(__shfl_xor(r, (int)d), __shfl_xor(l, (int)d), o2);
    }
    if constexpr (WAVES > 1) {
        __shared__ float joined[WAVES][6][64];
        float(*mine)[64] = joined[wave];
        mine[0][lane] = r, mine[1][lane] = l;
#pragma unroll
        for (int t = 0; t < 4; ++t) mine[2 + t][lane] = o[t];
        __syncthreads();
        if (wave) return;
        for (int w = 1; w < WAVES; ++w) {
            float(*from)[64] = joined[w];
            merge(from[0][lane], from[1][lane], dl_f32x4{from[2][lane], from[3][lane], from[4][lane], from[5][lane]});
        }
    }
    if (lane >= LANES) return;
    const bool none = l == 0.0f;
    if (d0 < D) {
        char *to = a.out + b * a.out_seq + j * a.out_token + h * a.out_head + 2u * d0;
        const float f = none ? 0.0f : 1.0f / l;
        dl_store_at(to, none ? dl_u32x2{0, 0} : dl_u32x2{Q::pack(o[0] * f, o[1] * f), Q::pack(o[2] * f, o[3] * f)});
    }
    if (a.lse && lane == 0) a.lse[row] = none ? -INFINITY : ((r == -INFINITY ? 0.0f : r) - Q::lift + log2f(l)) * 0.69314718055994530942f;
}

uint32_t ceil_div(uint64_t a, uint64_t b) { return (uint32_t)((a + b - 1) / b); }

struct att_shape {
    uint32_t nt;
    bool wide;  // pieces of the prefix are wide ones
    uint32_t prefix_tiles, prefix_splits, prefix_piece, own_tiles, own_target;
    uint32_t own_units;  // at most so many pieces of own tokens, over all sequences
    uint64_t rows;
};

// In how many pieces to cut an axis of `steps`, where there are `units` such axes and room for `slots` workgroups at once: a
// round of workgroups takes as long as the steps of one and about START more, and a piece costs the join about JOIN.
uint32_t cut(uint64_t units, uint64_t steps, uint64_t slots)
{
    constexpr double START = 3.0, JOIN = 0.1;
    if (!steps) return 0;
    uint32_t best = 1;
    double least = 0.0;
    for (uint32_t n = 1; n <= 64u && n <= steps; ++n) {
        const double rounds = (double)ceil_div(units * n, slots);
        const double cost = rounds * ((double)ceil_div(steps, n) + START) + JOIN * n;
        if (n == 1 || cost < least) best = n, least = cost;
    }
    return best;
}

// How the work is cut, from sizes alone.
int att_setup(const dl_kv_cache *cache, const dl_prefix_attention_args *args, dl_cache_view *view, att_shape *sh)
{
    if (!cache || !args) return DL_ERR_INVALID;
    const int rc = dl_cache_check(cache, 0, view);
    if (rc != DL_OK) return rc;
    if (args->type != DL_TYPE_BF16 && args->type != DL_TYPE_F16) return DL_ERR_INVALID;
    if (args->batch < 0 || args->q_tokens < 0 || args->q_heads < 0 || args->q_heads % cache->heads || args->reserved != 0) return DL_ERR_INVALID;
    if (args->prefix_tokens < 0 || args->prefix_tokens > 1 << 30 || args->max_pages < 0 || args->max_pages > 1 << 30 ||
        args->max_pages * cache->page_tokens > 1 << 30)
        return DL_ERR_INVALID;
    const unsigned __int128 rows = (unsigned __int128)args->batch * (uint32_t)args->q_tokens * (uint32_t)args->q_heads;
    if (rows > DL_MAX_ROWS / 2) return DL_ERR_INVALID;
    *sh = att_shape{};
    sh->rows = (uint64_t)rows;
    if (!rows) return DL_OK;
    const uint32_t group = (uint32_t)(args->q_heads / cache->heads), seq_rows = (uint32_t)args->q_tokens * group;
    const uint64_t all_rows = (uint64_t)args->batch * seq_rows;
    sh->nt = seq_rows > 16u ? 2 : 1;
    const uint64_t prefix = cache->pages ? (uint64_t)args->prefix_tokens : 0u, own = cache->pages ? (uint64_t)args->max_pages * cache->page_tokens : 0u;
    // Wide pieces of the prefix from 2^20 scores on, and 64 rows.  Narrow : wide, rows x prefix x heads of the cache: 84 x 2048 x 4 (0.7 M)
    // 13.3 : 14.5 us, 126 x 2048 x 4 (1.0 M) 15.0 : 16.5, 168 x 2048 x 4 (1.4 M) 17.9 : 17.0, 128 x 2048 x 8 (2.1 M) 20.3 : 17.7, 84 x 10000 x 4
    // (3.4 M) 20.6 : 20.1, 2048 x 32768 x 8 885 : 393; but 42 x 20000 x 4 (3.4 M) 18.7 : 23.0.
    sh->wide = all_rows >= 64u && (uint64_t)all_rows * prefix * (uint32_t)cache->heads >= 1u << 20;
    sh->prefix_tiles = ceil_div(all_rows, sh->wide ? 32u * ATT_WAVES : 16u * sh->nt);
    sh->own_tiles = ceil_div(seq_rows, 16u * sh->nt);
    const uint32_t step = sh->wide ? WIDE_KEYS : STEP;
    // Workgroups at once, by the registers: at head_dim 65 .. 128 three a compute unit with one narrow tile (152 - 159 registers), two with two
    // (223 - 240) or with wide pieces (256, for the own ones of that launch too), one above.  Up to 64 there would be room for four with one tile (108 - 118) and
    // three with two (158 - 167), which the cut does not count on.
    const uint32_t slots = cache->head_dim > 128 ? 256u : sh->wide || sh->nt == 2u ? 512u : 768u;
    sh->prefix_splits = cut((uint64_t)cache->heads * sh->prefix_tiles, ceil_div(prefix, step), slots);
    if (sh->prefix_splits) {
        sh->prefix_piece = ceil_div(ceil_div(prefix, sh->prefix_splits), step) * step;
        sh->prefix_splits = ceil_div(prefix, sh->prefix_piece);
    }
    if (own) {
        // Own tokens: pieces for two rounds of workgroups; where the sequences alone are a round, of a quarter of a round's share,
        // which even out what the lengths do not.
        const uint32_t batch = (uint32_t)args->batch, round = slots / (uint32_t)cache->heads / sh->own_tiles;
        const bool even = batch <= OWN_EVEN_MAX && (uint64_t)batch * ceil_div(own, STEP) < 1ull << 31;
        sh->own_target = !even ? 0u : round > batch ? 2u * round - batch : round ? 4u * round : 1u;
        const uint64_t most = (uint64_t)batch * ceil_div(own, STEP * OWN_LEAST_STEPS);  // no piece is smaller, but a sequence's last
        sh->own_units = !even ? batch : (uint32_t)((uint64_t)sh->own_target + batch < most ? sh->own_target + batch : most);
    }
    return DL_OK;
}

// Parts that the pieces leave behind.
uint64_t att_parts(const att_shape &sh, uint32_t batch) { return sh.rows * sh.prefix_splits + sh.rows / (batch ? batch : 1u) * sh.own_units; }
// Where things lie in the workspace, behind the control words.
constexpr size_t align16(uint64_t n) { return (n + 15u) / 16u * 16u; }

}  // namespace

extern "C" int64_t dl_prefix_attention_workspace(const dl_kv_cache *cache, const dl_prefix_attention_args *args)
{
    dl_cache_view view;
    att_shape sh;
    const int rc = att_setup(cache, args, &view, &sh);
    if (rc != DL_OK) return rc;
    const uint64_t parts = att_parts(sh, (uint32_t)args->batch);
    return (int64_t)(DL_CONTROL_BYTES + align16(8ull * (uint32_t)args->batch) + align16(parts * sizeof(dl_f32x2)) + parts * view.head_dim * sizeof(float));
}

extern "C" int dl_prefix_attention(const dl_kv_cache *cache, const dl_prefix_attention_args *args, void *stream)
{
    DL_LOCKED;
    if (!g_dl.inited) return DL_ERR_STATE;
    if (dl_device_error_pending()) return DL_ERR_LOST;
    att_args a;
    att_shape sh;
    int rc = att_setup(cache, args, &a.c, &sh);
    if (rc != DL_OK) return rc;
    if (!sh.rows) return DL_OK;
    rc = dl_cache_check(cache, 3, &a.c);
    if (rc != DL_OK) return rc;
    if (!args->q || !args->out || (args->prefix_tokens && !args->prefix_pages) || (args->max_pages && (!args->pages || !args->lens)))
        return DL_ERR_INVALID;
    if (((uint64_t)args->q | (uint64_t)args->out) % 2u ||
        ((uint64_t)args->lse | (uint64_t)args->prefix_pages | (uint64_t)args->pages | (uint64_t)args->lens | (uint64_t)args->q_lens) % 4u)
        return DL_ERR_INVALID;
    const int64_t needed = dl_prefix_attention_workspace(cache, args);
    if (!args->workspace || (uint64_t)args->workspace % 16u || args->workspace_bytes < (uint64_t)needed) return DL_ERR_INVALID;
    a.q = (const char *)args->q;
    a.out = (char *)args->out;
    a.lse = args->lse;
    a.prefix_pages = args->prefix_pages;
    a.pages = args->pages;
    a.lens = args->lens;
    a.q_lens = args->q_lens;
    a.units = (uint32_t *)((char *)args->workspace + DL_CONTROL_BYTES);
    a.rl = (dl_f32x2 *)((char *)a.units + align16(8ull * (uint32_t)args->batch));
    a.partial = (float *)((char *)a.rl + align16(att_parts(sh, (uint32_t)args->batch) * sizeof(dl_f32x2)));
    a.q_seq = 2 * args->q_seq_stride;
    a.q_token = 2 * args->q_token_stride;
    a.q_head = 2 * args->q_head_stride;
    a.out_seq = 2 * args->out_seq_stride;
    a.out_token = 2 * args->out_token_stride;
    a.out_head = 2 * args->out_head_stride;
    a.pages_stride = args->pages_stride;
    a.prefix_tokens = cache->pages ? (uint32_t)args->prefix_tokens : 0u;
    a.own_most = cache->pages ? (uint32_t)(args->max_pages * cache->page_tokens) : 0u;
    a.batch = (uint32_t)args->batch;
    a.q_tokens = (uint32_t)args->q_tokens;
    a.q_heads = (uint32_t)args->q_heads;
    a.group = a.q_heads / a.c.heads;
    a.rows = (uint32_t)sh.rows;
    a.prefix_tiles = sh.prefix_tiles;
    a.prefix_splits = sh.prefix_splits;
    a.prefix_piece = sh.prefix_piece;
    a.own_tiles = sh.own_tiles;
    a.own_target = sh.own_target;
    a.scale = args->scale * 1.44269504088896340736f;
    const uint64_t shared = (uint64_t)a.c.heads * sh.prefix_tiles * sh.prefix_splits;
    const uint64_t grid = shared + (uint64_t)a.c.heads * sh.own_tiles * sh.own_units;
    if (grid >= (1ull << 32) / ATT_THREADS) return DL_ERR_INVALID;
    a.wide_shared = sh.wide ? (uint32_t)shared : 0u;
    a.narrow_shared = sh.wide ? 0u : (uint32_t)shared;
    hipStream_t hs = (hipStream_t)stream;
    // eight keys in a row lie in one page, see place
    const bool aligned = cache->page_tokens % 8 == 0;
    // a row's pieces: a wavefront's work while the rows alone fill the chip or the pieces are few
    const bool shared_out = sh.prefix_splits + sh.own_units / a.batch > 16u && sh.rows < 4096u;
    // (the most rows there may be are 2^24 workgroups of the join, 2^32 threads: one more than a grid is wide)
    const uint32_t blocks = ceil_div(sh.rows, ATT_WAVES), high = ceil_div(blocks, 1u << 23);
    const dim3 join(ceil_div(blocks, high), high);
    dl_with_16bit(args->type, [&](auto q) {
        auto with_dim = [&](auto dp) {
            constexpr int DP = decltype(dp)::value;
            if (grid)
                dl_with_format(cache->format, [&](auto c) {
                    dl_with_bool(aligned, [&](auto al) {
                        dl_with_bool(sh.wide, [&](auto wd) {
                            dl_with_bool(sh.nt == 2, [&](auto two) {
                                hipLaunchKernelGGL((dl_attention_kernel<decltype(q), decltype(c), DP, decltype(two)::value ? 2 : 1, decltype(al)::value,
                                                                        decltype(wd)::value>),
                                                   dim3((uint32_t)grid), dim3(ATT_THREADS), 0, hs, a);
                            });
                        });
                    });
                });
            if (shared_out)
                hipLaunchKernelGGL((dl_attention_join_kernel<decltype(q), DP, 4>), dim3((uint32_t)sh.rows), dim3(ATT_THREADS), 0, hs, a);
            else
                hipLaunchKernelGGL((dl_attention_join_kernel<decltype(q), DP, 1>), join, dim3(ATT_THREADS), 0, hs, a);
        };
        if (a.c.head_dim <= 64)
            with_dim(std::integral_constant<int, 64>{});
        else if (a.c.head_dim <= 128)
            with_dim(std::integral_constant<int, 128>{});
        else
            with_dim(std::integral_constant<int, 256>{});
    });
    DL_HIP(hipGetLastError());
    t_dl_last.mode = DL_MODE_ONESHOT;
    return DL_OK;
}
