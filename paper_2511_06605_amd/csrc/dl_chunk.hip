// Attention of chunks of new tokens over a paged cache in 8 bits (dl_chunk_attention).
//
// The sums are those of dl_attention.hip: with s the scores in units of ln 2 and u = c d a value's scale taken apart (dl_value_scale),
// w = 2^(s + log2 c - r) <= 2^(8 + lift), O += w d V, l += w / c, with a reference r that follows the largest s + log2 c.
//
// The queries that share a head of the cache are the rows of a sequence: row j * group + g is query j in the g-th of those heads.  A
// workgroup has a tile of rows and walks the keys that its last row sees in steps of 64, which its wavefronts share: codes are turned into
// elements of Q once, on their way into LDS, keys as rows and values transposed (by byte permutes while they are bytes), so that every
// operand of the 32 x 32 x 16 products is one 16-byte read.  While a step is worked on, the next one's codes are on their way to registers
// and the pages of the one after it are looked up.  Masks cost something only where a wavefront's rows end.  128 rows a tile, two workgroups
// a compute unit; 256 for many rows and up to head_dim 128 (dl_chunk_wide_kernel).  Where there are few tiles their keys are
// cut into pieces, which a second launch joins (chunk_unit).
//
// Measured (8 heads of 128, 32 query heads, bfloat16 on fp8, unless said otherwise): 2048 queries behind 30 720 tokens 1100 - 1160 us, 1065 GFLOP,
// 0.92 - 0.97 PFLOP/s where a large matrix product reaches 1.34 (128 rows a tile: 1319); a prompt of 8192 617 - 638 us, 0.86 - 0.89; three
// documents with up to 512 queries on up to 16 400 (4 heads, 28 query heads, float16 on int8) 216 - 235 us, 0.6, 18 of it the join; 16 queries
// behind 500 13.3 us, 5 sequences of up to 101 behind up to 777 (12 heads of 64) 18 us, both two launches.  A workgroup of the former is at work
// for 6 us: 1.4 until it knows its piece, 0.6 until it knows its pages, 1.1 for the codes, 1.7 for the step, 0.9 for what it leaves; one of the join 2.5.
#include "dl_codes.h"
#include "dl_internal.h"
#include "dl_packed.h"
#include "dl_pieces.h"

namespace {

constexpr uint32_t CH_THREADS = 256, CH_WAVES = CH_THREADS / 64;
constexpr uint32_t CH_KEYS = 64;

struct chunk_args {
    dl_cache_view c;
    dl_packed p;
    const char *q;
    char *out;
    float *lse;
    // What pieces leave behind for the join, by slot, head and row of the tile
    dl_f32x2 *rl;    // r and l
    float *partial;  // head_dim sums
    int64_t q_token, q_head, out_token, out_head;  // bytes
    uint32_t q_heads, group;
    dl_divider groups;  // by group
    uint32_t tile_rows;           // 32 or 64 a wavefront
    uint32_t most_cut;            // 0: nothing is cut
    bool search;                  // see chunk_unit
    float round;                  // workgroups at once, by the heads
    uint32_t *size;               // what the pieces' size has come to, for the join
    float scale;         // times log2 e
};

// The key axis of a sequence is cut into pieces where there are few tiles, by the lengths, which only the device knows: into pieces of at most
// `size` steps.  All tiles of a sequence are cut alike, at multiples of `keys`; a tile whose rows end before a piece begins has nothing of
// it.  What leaves something behind for the join are the pieces of sequences that are cut: no more than `most_cut` over all of them, and so
// no more than half as many tiles.
// Which size: a round of workgroups takes as long as the steps of one and START more, a piece costs the join JOIN steps; a lane of a
// wavefront looks at the size that cuts the longest sequence into its number + 1 pieces.  Batches of more than SEARCH_MAX sequences, and tables
// with room for more than 2^20 steps, are not looked at one by one: with T steps of all tiles, T / (most_cut / 2), so that those that are cut
// have at most twice as many pieces (dl_piece_steps).
// Every wavefront works this out from the lengths for itself.
constexpr float START = 3.0f, JOIN = 0.1f;
constexpr uint32_t SEARCH_MAX = 16;

struct chunk_place {
    uint32_t b, tile, piece, pieces, keys;
    uint32_t slot;  // of this piece; the others of the tile lie next to it
    uint32_t size;
    uint32_t first, queries, len;  // of the sequence: its first row of q
};
// The unit-th piece of all (CUT: the unit-th tile of those that are cut, its first piece); false: there is none.
template <bool CUT>
__device__ __forceinline__ bool chunk_unit(const chunk_args &a, uint32_t unit, chunk_place *at)
{
    const uint32_t lane = threadIdx.x % 64u;
    uint32_t size = DL_UNCUT, tiles = 0, steps = 0;
    const bool at_once = a.p.batch <= 64u;
    uint32_t first = 0, queries = 0, len = 0;
    auto look = [&](uint32_t b0) {
        const uint32_t b = min(b0 + lane, a.p.batch - 1u);
        first = a.p.start(b);
        queries = b0 + lane < a.p.batch ? a.p.queries(b, first) : 0u;
        len = a.p.len(b);
        tiles = (queries * a.group + a.tile_rows - 1u) / a.tile_rows;
        steps = (len + CH_KEYS - 1u) / CH_KEYS;
    };
    if (at_once) look(0);
    if (CUT) {
        size = max(*a.size, 1u);
    } else if (a.search) {
        uint32_t longest = 1;
        auto of = [&](uint32_t x, uint32_t b) { return (uint32_t)__builtin_amdgcn_readlane((int)x, (int)b); };
        for (uint32_t b = 0; b < a.p.batch; ++b) longest = of(tiles, b) ? max(longest, of(steps, b)) : longest;
        // (whole numbers up to 2^20: with half a unit in front of the quotient its rounding makes no difference)
        const float mine = ceilf(((float)longest - 0.5f) * __builtin_amdgcn_rcpf((float)(lane + 1u))), over = __builtin_amdgcn_rcpf(mine);
        float units = 0.0f, cut = 0.0f, most = 1.0f;
        for (uint32_t b = 0; b < a.p.batch; ++b) {
            const float its = (float)of(tiles, b), pieces = fmaxf(ceilf(((float)of(steps, b) - 0.5f) * over), 1.0f);
            units = fmaf(its, pieces, units);
            cut += pieces > 1.0f ? its * pieces : 0.0f;
            most = its > 0.0f ? fmaxf(most, pieces) : most;
        }
        float cost = ceilf(units / a.round) * (mine + START) + (most > 1.0f ? JOIN * most : 0.0f);
        if (cut > (float)a.most_cut) cost = INFINITY;
        const uint32_t least = ~dl_largest(~dl_bits<uint32_t>(cost));  // (costs are positive: in order as whole numbers)
        size = (uint32_t)of((uint32_t)mine, (uint32_t)__ffsll((long long)__ballot(dl_bits<uint32_t>(cost) == least)) - 1u);
    } else if (a.most_cut) {
        uint64_t all = 0;
        for (uint32_t b0 = 0; b0 < a.p.batch; b0 += 64u) {
            if (!at_once) look(b0);
            uint64_t x = (uint64_t)tiles * steps;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) x += (uint64_t)__shfl_xor((unsigned long long)x, d);
            all += x;
        }
        size = dl_piece_steps(all, a.most_cut);
    }
    uint32_t before = 0, slots = 0;
    for (uint32_t b0 = 0; b0 < a.p.batch; b0 += 64u) {
        if (!at_once) look(b0);
        const uint32_t pieces = max((steps + size - 1u) / size, 1u), cut = pieces > 1u ? tiles * pieces : 0u;
        const uint32_t counted = CUT ? (pieces > 1u ? tiles : 0u) : tiles * pieces;
        const uint32_t up_to = before + dl_sum_up_to(counted), slots_up_to = slots + dl_sum_up_to(cut);
        const unsigned long long where = __ballot(up_to > unit);
        if (where) {
            const int l = __ffsll((long long)where) - 1;
            auto of = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, l); };
            const uint32_t n = unit - (of(up_to) - of(counted)), its = of(pieces), its_steps = of(steps);
            if (n >= of(counted)) return false;  // (starts that decrease may count more tiles than 32 bits hold)
            at->b = b0 + (uint32_t)l;
            at->pieces = its;
            // even shares of the steps: no piece is longer than `size`
            at->keys = (its_steps + its - 1u) / its * CH_KEYS;
            // (the last tile first: it sees the most)
            at->tile = of(tiles) - 1u - (CUT ? n : n / its);
            at->piece = CUT ? 0u : n % its;
            at->slot = of(slots_up_to) - of(cut) + (CUT ? n * its : n);
            at->size = size;
            at->first = of(first);
            at->queries = of(queries);
            at->len = of(len);
            return true;
        }
        before = (uint32_t)__builtin_amdgcn_readlane((int)up_to, 63);
        slots = (uint32_t)__builtin_amdgcn_readlane((int)slots_up_to, 63);
    }
    return false;
}

// A tile's rows: where they are, and what they see.
struct chunk_rows {
    uint32_t first, row0, rows;  // first row of q, the tile's first row, rows of the sequence
    int32_t ahead;               // row r sees the keys up to ahead + r / group
    uint32_t end;                // keys that some row of the tile sees

    __device__ __forceinline__ chunk_rows(const chunk_args &a, const chunk_place &at)
    {
        first = at.first;
        rows = at.queries * a.group;
        row0 = at.tile * a.tile_rows;
        ahead = (int32_t)at.len - (int32_t)at.queries;
        end = seen_by(a, min(row0 + a.tile_rows, rows) - 1u);
    }
    __device__ __forceinline__ uint32_t seen_by(const chunk_args &a, uint32_t row) const { return (uint32_t)max(ahead + (int32_t)(dl_divide(row, a.groups)) + 1, 0); }
};

// Operands lie in rows with 16 bytes between them, so that eight neighbouring lanes, a row each, use all banks, and a lane's addresses
// differ by constants.
template <int DP>
struct alignas(16) chunk_tile {  // (reads of 16 bytes that lie at fours take twice as long)
    static constexpr uint32_t K_ROW = DP / 2 + 4, V_ROW = CH_KEYS / 2 + 4;
    uint32_t k[CH_KEYS * K_ROW];  // key, dim
    uint32_t v[DP * V_ROW];       // dim, key: of each 16 keys 0 - 3, 8 - 11, 4 - 7, 12 - 15
    float ks[CH_KEYS], lu[CH_KEYS], iu[CH_KEYS], d[CH_KEYS];
    uint32_t taken_apart;  // some value's d is not 1
};
template <int DP>
struct chunk_lds {
    chunk_tile<DP> tiles[2];
    uint64_t rows_at[2][CH_KEYS];  // offsets of the codes' rows
    uint64_t alive_at[2];          // bit k: key k is one of the piece, in a page of the pool
};

// Codes on their way into a tile.
template <class Q, class C, int DP>
struct chunk_feed {
    static constexpr uint32_t PIECES = DP / 8;                          // 16-byte pieces of a key's row
    static constexpr uint32_t K_LOADS = CH_KEYS * PIECES / CH_THREADS;  // of 8 codes
    static constexpr uint32_t V_ITEMS = 8 * (DP / 4);                   // 8 keys (half of 16) x 4 dims; eight neighbouring lanes fill a row
    static constexpr uint32_t V_LOADS = (V_ITEMS + CH_THREADS - 1) / CH_THREADS;
    const int32_t *table;
    const char *k_from, *v_from, *scales;
    uint32_t end, lane, wave, looked_up = 0;
    float scale = 0.0f;
    bool alive = false;
    dl_words<8> kw[K_LOADS];
    uint32_t vw[V_LOADS][8];

    __device__ __forceinline__ chunk_feed(const chunk_args &a, uint32_t b, uint32_t head, uint32_t last, uint32_t in_wave, uint32_t of_wave)
    {
        table = a.p.pages + b * a.p.pages_stride;
        k_from = a.c.k + (int64_t)head * a.c.head_stride;
        v_from = a.c.v + (int64_t)head * a.c.head_stride;
        scales = (const char *)(of_wave == 0 ? a.c.k_scale : a.c.v_scale) + (int64_t)head * a.c.scale_head_stride;
        end = last;
        lane = in_wave;
        wave = of_wave;
    }
    // A key's page: looked up by the first two wavefronts, for the keys' and the values' scales; the first hands the rows on.
    __device__ __forceinline__ void look_up(const chunk_args &a, uint32_t base)
    {
        if (wave < 2) looked_up = (uint32_t)table[dl_divide(min(base + lane, end - 1u), a.c.page)];
    }
    __device__ __forceinline__ void hand_on(const chunk_args &a, uint32_t base, uint64_t (&rows_at)[CH_KEYS], uint64_t &alive_at)  // what was looked up for the step at base
    {
        if (wave < 2) {
            const uint32_t key = min(base + lane, end - 1u), in = key - dl_divide(key, a.c.page) * a.c.page.d;
            alive = base + lane < end && looked_up < a.c.pages;
            const uint64_t page = looked_up < a.c.pages ? looked_up : 0u;
            if (wave == 0) {
                rows_at[lane] = page * a.c.page_stride + (uint64_t)in * a.c.token_stride;
                const unsigned long long all = __ballot(alive);
                if (lane == 0) alive_at = all;
            }
            scale = *(const float *)(scales + page * a.c.scale_page_stride + (uint64_t)in * a.c.scale_token_stride);
        }
    }
    // One part of LOAD_PARTS of a step's loads: where its row begins, and the load from there.
    static constexpr uint32_t LOAD_PARTS = K_LOADS + 8 * V_LOADS;
    static __device__ __forceinline__ uint64_t load_from(const uint64_t (&rows_at)[CH_KEYS], uint32_t part_of)
    {
        if (part_of < K_LOADS) return rows_at[(threadIdx.x + part_of * CH_THREADS) / PIECES];
        const uint32_t e = (part_of - K_LOADS) % 8u, part = threadIdx.x % 8u;
        return rows_at[part / 2u * 16u + part % 2u * 4u + (e & 3u) + (e >> 2) * 8u];
    }
    __device__ __forceinline__ void load_part(const chunk_args &a, uint64_t from, uint32_t part_of)
    {
        const uint32_t D = a.c.head_dim;
        if (part_of < K_LOADS) {
            kw[part_of] = dl_load_words<8>(k_from + from + min((threadIdx.x + part_of * CH_THREADS) % PIECES * 8u, D - 8u));
        } else {
            const uint32_t x = (part_of - K_LOADS) / 8u, e = (part_of - K_LOADS) % 8u;
            vw[x][e] = dl_load_at<uint32_t>(v_from + from + min((threadIdx.x + x * CH_THREADS) / 8u * 4u, D - 4u));
        }
    }
    __device__ __forceinline__ void load(const chunk_args &a, const uint64_t (&rows_at)[CH_KEYS])
    {
#pragma unroll
        for (uint32_t n = 0; n < LOAD_PARTS; ++n) load_part(a, load_from(rows_at, n), n);
    }
    // What is none counts as zero.
    __device__ __forceinline__ void clear(uint64_t alive_at)
    {
        const uint32_t all_lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)alive_at);
        const uint32_t all_hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(alive_at >> 32));
        const uint64_t all = (uint64_t)all_hi << 32 | all_lo;
        if (all == ~0ull) return;
#pragma unroll
        for (uint32_t x = 0; x < K_LOADS; ++x)
            if (!(all >> ((threadIdx.x + x * CH_THREADS) / PIECES) & 1u)) kw[x] = dl_words<8>{};
#pragma unroll
        for (uint32_t x = 0; x < V_LOADS; ++x) {
            const uint32_t part = threadIdx.x % 8u, key = part / 2u * 16u + part % 2u * 4u;
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e)
                if (!(all >> (key + (e & 3u) + (e >> 2) * 8u) & 1u)) vw[x][e] = 0;
        }
    }
    // One part of PUT_PARTS of what goes to the tile: the keys' loads, then four dims at a time of the values'.
    static constexpr uint32_t PUT_PARTS = K_LOADS + 4 * V_LOADS;
    __device__ __forceinline__ void put_part(chunk_tile<DP> &to, uint32_t part_of)
    {
        if (part_of < K_LOADS) {
            const uint32_t x = part_of, n = threadIdx.x + x * CH_THREADS, key = n / PIECES, c = n % PIECES;
            const dl_u32x2 p = C::template spread<Q>(kw[x].w[0]), r = C::template spread<Q>(kw[x].w[1]);
            *(dl_u32x4 *)&to.k[key * chunk_tile<DP>::K_ROW + c * 4u] = dl_u32x4{p[0], p[1], r[0], r[1]};
            return;
        }
        const uint32_t x = (part_of - K_LOADS) / 4u, f = (part_of - K_LOADS) % 4u;
        const uint32_t n = threadIdx.x + x * CH_THREADS, d = n / 8u * 4u, part = n % 8u;
        if (V_ITEMS % CH_THREADS && n >= V_ITEMS) return;
        dl_u32x2 two[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const uint32_t pick = f < 2 ? 0x05010400u : 0x07030602u;
            const uint32_t a01 = __builtin_amdgcn_perm(vw[x][4 * g + 1], vw[x][4 * g], pick), a23 = __builtin_amdgcn_perm(vw[x][4 * g + 3], vw[x][4 * g + 2], pick);
            two[g] = C::template spread<Q>(__builtin_amdgcn_perm(a23, a01, f % 2 ? 0x07060302u : 0x05040100u));
        }
        *(dl_u32x4 *)&to.v[(d + f) * chunk_tile<DP>::V_ROW + part * 4u] = dl_u32x4{two[0][0], two[0][1], two[1][0], two[1][1]};
    }
    __device__ __forceinline__ void put_codes(chunk_tile<DP> &to)
    {
#pragma unroll
        for (uint32_t n = 0; n < PUT_PARTS; ++n) put_part(to, n);
    }
    __device__ __forceinline__ void put_scales(const chunk_args &a, chunk_tile<DP> &to)
    {
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
    }
    // Values times what their scales left out, in LDS, by all threads, before anybody works on the step.
    static __device__ __forceinline__ void apart(chunk_tile<DP> &to)
    {
#pragma unroll 1
        for (uint32_t n = threadIdx.x; n < DP * 8u; n += CH_THREADS) {
            const uint32_t r = n / 8u, part = n % 8u, key = part / 2u * 16u + part % 2u * 4u;
            uint32_t *const v = &to.v[r * chunk_tile<DP>::V_ROW + part * 4u];
#pragma unroll
            for (uint32_t x = 0; x < 4; ++x) {
                const float *const d = &to.d[key + x / 2u * 8u + x % 2u * 2u];
                v[x] = Q::pack(Q::in_range(Q::lo(v[x]) * d[0]), Q::in_range(Q::hi(v[x]) * d[1]));
            }
        }
        __syncthreads();
    }
    // The operands of a product: keys 32 kb + i against dims 16 st + 8 half .., and dims 32 dt + i against the x-th 16 of keys 32 kb ..
    static __device__ __forceinline__ dl_u32x4 keys(const chunk_tile<DP> &in, uint32_t kb, uint32_t st, uint32_t i, uint32_t half)
    {
        return *(const dl_u32x4 *)&in.k[(32u * kb + i) * chunk_tile<DP>::K_ROW + (2u * st + half) * 4u];
    }
    static __device__ __forceinline__ dl_u32x4 values(const chunk_tile<DP> &in, uint32_t kb, uint32_t x, uint32_t dt, uint32_t i, uint32_t half)
    {
        return *(const dl_u32x4 *)&in.v[(32u * dt + i) * chunk_tile<DP>::V_ROW + (4u * kb + 2u * x + half) * 4u];
    }
};

// A row's sums, as lane (i, half) of a wavefront has them: dims 32 x + 8 (e / 4) + 4 half + e % 4.  They are what a piece leaves behind, or done.
template <class Q, int DP>
__device__ __forceinline__ void finish_row(const chunk_args &a, const chunk_place &at, const chunk_rows &t, uint32_t head, uint32_t my, uint32_t half, float r, float l,
                                           const dl_f32x16 (&o)[DP / 32])
{
    l += __shfl_xor(l, 32);
    if (my >= t.rows) return;
    const uint32_t D = a.c.head_dim;
    if (at.pieces > 1u) {
        const uint64_t to = ((uint64_t)at.slot * a.c.heads + head) * a.tile_rows + (my - t.row0);
        if (half == 0) a.rl[to] = dl_f32x2{r, l};
#pragma unroll
        for (int x = 0; x < DP / 32; ++x)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const uint32_t d = 32u * x + 2u * e + 4u * half;
                if (d < D) *(dl_f32x4 *)(a.partial + to * D + d) = dl_f32x4{o[x][e], o[x][e + 1], o[x][e + 2], o[x][e + 3]};
            }
        return;
    }
    const uint32_t j = dl_divide(my, a.groups), h = head * a.group + my - j * a.group;
    const bool none = l == 0.0f;
    const float f = none ? 0.0f : 1.0f / l;
    char *const to = a.out + (uint64_t)(t.first + j) * a.out_token + h * a.out_head;
#pragma unroll
    for (int x = 0; x < DP / 32; ++x)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const uint32_t d = 32u * x + 2u * e + 4u * half;
            if (d < D)
                dl_store_at(to + 2u * d, none ? dl_u32x2{0, 0} : dl_u32x2{Q::pack(o[x][e] * f, o[x][e + 1] * f), Q::pack(o[x][e + 2] * f, o[x][e + 3] * f)});
        }
    if (a.lse && half == 0)
        a.lse[(uint64_t)(t.first + j) * a.q_heads + h] = none ? -INFINITY : ((r == -INFINITY ? 0.0f : r) - Q::lift + log2f(l)) * DL_LN2;
}

template <class Q, class C, int DP>
__global__ void __launch_bounds__(CH_THREADS, DP <= 128 ? 2 : 1) dl_chunk_kernel(const chunk_args a)
{
    using feed_t = chunk_feed<Q, C, DP>;
    __shared__ chunk_lds<DP> lds;
    auto &tiles = lds.tiles;
    const uint32_t lane = threadIdx.x % 64u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
    const uint32_t i = lane % 32u, half = lane / 32u, D = a.c.head_dim, head = blockIdx.x, unit = blockIdx.z * gridDim.y + blockIdx.y;
    chunk_place at;
    if (!chunk_unit<false>(a, unit, &at)) return;
    if (a.most_cut && unit == 0 && head == 0 && threadIdx.x == 0) *a.size = at.size;
    const chunk_rows t(a, at);
    const uint32_t first = at.piece * at.keys, end = min(first + at.keys, t.end);
    if (at.piece && first >= end) return;
    feed_t feed(a, at.b, head, end, lane, wave);

    const uint32_t wave_row = t.row0 + wave * 32u, my = wave_row + i, row = min(my, t.rows - 1u);
    const uint32_t j = dl_divide(row, a.groups), h = head * a.group + row - j * a.group;
    const int32_t last = t.ahead + (int32_t)j;
    // keys before whole_end are seen by all rows of the wavefront, those from wave_end on by none
    const uint32_t wave_end = wave_row < t.rows ? min(t.seen_by(a, min(wave_row + 32u, t.rows) - 1u), end) : 0u;
    const uint32_t whole_end = wave_row < t.rows ? t.seen_by(a, wave_row) : 0u;
    const char *const q = a.q + (uint64_t)(t.first + j) * a.q_token + h * a.q_head;
    dl_u32x4 qf[DP / 16];
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) qf[s] = 16u * s < D ? dl_load_at<dl_u32x4>(q + 2u * (16u * s + 8u * half)) : dl_u32x4{0, 0, 0, 0};

    // (inlined whatever they cost: a call wants `feed` in memory, codes and all)
    auto hand_on = [&](uint32_t base, uint32_t to) __attribute__((always_inline)) { feed.hand_on(a, base, lds.rows_at[to], lds.alive_at[to]); };
    auto put = [&](uint32_t to) __attribute__((always_inline)) {
        feed.clear(lds.alive_at[to]);
        feed.put_codes(tiles[to]);
        feed.put_scales(a, tiles[to]);
    };

    dl_f32x16 o[DP / 32];
    float r = -INFINITY, low = -Q::lift, l = 0.0f;
#pragma unroll
    for (int x = 0; x < DP / 32; ++x)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[x][e] = 0.0f;

    if (first < end) {
        feed.look_up(a, first);
        hand_on(first, 0);
        __syncthreads();
        feed.load(a, lds.rows_at[0]);
        feed.look_up(a, first + CH_KEYS);
        put(0);
        hand_on(first + CH_KEYS, 1);
        __syncthreads();
    }
    uint32_t now = 0;
    for (uint32_t base = first; base < end; base += CH_KEYS, now ^= 1u) {
        const bool more = base + CH_KEYS < end;
        if (__builtin_amdgcn_readfirstlane((int)tiles[now].taken_apart)) feed_t::apart(tiles[now]);
        if (more) {
            feed.load(a, lds.rows_at[now ^ 1u]);
            feed.look_up(a, base + 2 * CH_KEYS);
        }
        const chunk_tile<DP> &in = tiles[now];
#pragma unroll 1
        for (uint32_t kb = 0; kb < 2; ++kb) {
            const uint32_t key0 = base + 32u * kb;
            if (key0 >= wave_end) break;
            // scores: rows of the product are keys (8 (e / 4) + 4 half + e % 4), its columns queries (i)
            dl_f32x16 s;
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = 0.0f;
#pragma unroll
            for (uint32_t st = 0; st < DP / 16; ++st) s = Q::mfma32(feed_t::keys(in, kb, st, i, half), qf[st], s);
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
            for (int e = 0; e < 16; ++e) s[e] = fmaf(s[e], ks[e], lu[e]);
            if (key0 + 32u > whole_end) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (2 * (e & ~3) + (e & 3) > last - (int32_t)(key0 + 4u * half)) s[e] = -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[e]);
            // (the reference follows the largest only where that is 2^8 times above it)
            if (__any(top > r + 8.0f)) {
                const auto swapped = __builtin_amdgcn_permlane32_swap(dl_bits<uint32_t>(top), dl_bits<uint32_t>(top), false, false);
                top = fmaxf(dl_bits<float>((uint32_t)swapped[0]), dl_bits<float>((uint32_t)swapped[1]));
                const float most = fmaxf(r, top), ref = most == -INFINITY ? 0.0f : most, fade = __builtin_amdgcn_exp2f(r - ref);
                r = most;
                low = ref - Q::lift;
                l *= fade;
#pragma unroll
                for (int x = 0; x < DP / 32; ++x) o[x] *= fade;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[e] = __builtin_amdgcn_exp2f(s[e] - low);
                l = fmaf(s[e], iu[e], l);
            }
            dl_u32x4 pf[2];
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) pf[x][e] = Q::pack(s[8 * x + 2 * e], s[8 * x + 2 * e + 1]);
            // sums: rows of the product are dims, its columns queries
#pragma unroll
            for (uint32_t x = 0; x < 2; ++x)
#pragma unroll
                for (uint32_t dt = 0; dt < DP / 32; ++dt) o[dt] = Q::mfma32(feed_t::values(in, kb, x, dt, i, half), pf[x], o[dt]);
        }
        if (more) {
            put(now ^ 1u);
            hand_on(base + 2 * CH_KEYS, now);
        }
        __syncthreads();
    }
    finish_row<Q, DP>(a, at, t, head, my, half, r, l, o);
}

// Many rows: 64 a wavefront, one wavefront a SIMD.  An operand read from LDS then serves two products, and codes are turned into elements once for
// 256 rows.  What a second wavefront would overlap is interleaved here: while the scores of 32 keys become weights, the products of the next
// 32 keys are under way, and while those weights meet the values, the next scores are scaled and the next step's codes go to LDS.  Three
// tiles in LDS: one that is worked on, the next one, and the one that is filled while somebody may still be at the first; a barrier a step.
//
// What bounds it is a lone wavefront's way through a step of 64 keys: about 630 instructions (450 vector ones, 64 products, 75 for LDS) in 5060
// cycles, 60 % of which it issues, 28 % it waits for counters or at the barrier and 12 % for its turn (counted over 2048 queries on 30 720 tokens); the matrix
// units work for 2050.  So the number of instructions counts: operands in padded rows, whose addresses differ by constants, instead of
// places exchanged by an exclusive or 1230 -> 1127 us.  The same code with 32 rows a wavefront and eight of them, two a SIMD: 1317 (twice the reads
// from LDS); operands a step further ahead and all scales a part ahead: 1160.
template <int DP>
struct wide_lds {
    chunk_tile<DP> tiles[3];
    uint64_t rows_at[2][CH_KEYS];
    uint64_t alive_at[2];
};
template <class Q, class C, int DP>
__global__ void __launch_bounds__(CH_THREADS, DP <= 64 ? 2 : 1) dl_chunk_wide_kernel(const chunk_args a)
{
    using feed_t = chunk_feed<Q, C, DP>;
    __shared__ wide_lds<DP> lds;
    const uint32_t lane = threadIdx.x % 64u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
    const uint32_t i = lane % 32u, half = lane / 32u, D = a.c.head_dim, head = blockIdx.x, unit = blockIdx.z * gridDim.y + blockIdx.y;
    chunk_place at;
    if (!chunk_unit<false>(a, unit, &at)) return;
    if (a.most_cut && unit == 0 && head == 0 && threadIdx.x == 0) *a.size = at.size;
    const chunk_rows t(a, at);
    const uint32_t first = at.piece * at.keys, end = min(first + at.keys, t.end);
    if (at.piece && first >= end) return;
    feed_t feed(a, at.b, head, end, lane, wave);
    const uint32_t wave_row = t.row0 + wave * 64u;
    // keys before whole_end are seen by all rows of the wavefront
    const uint32_t whole_end = wave_row < t.rows ? t.seen_by(a, wave_row) : 0u;
    int32_t last[2];
    dl_u32x4 qf[2][DP / 16];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const uint32_t row = min(wave_row + 32u * n + i, t.rows - 1u), j = dl_divide(row, a.groups), h = head * a.group + row - j * a.group;
        last[n] = t.ahead + (int32_t)j - 4 * (int32_t)half;
        const char *const q = a.q + (uint64_t)(t.first + j) * a.q_token + h * a.q_head;
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) qf[n][s] = 16u * s < D ? dl_load_at<dl_u32x4>(q + 2u * (16u * s + 8u * half)) : dl_u32x4{0, 0, 0, 0};
    }
    dl_f32x16 o[2][DP / 32], x[2];
    float r[2] = {-INFINITY, -INFINITY}, low[2] = {-Q::lift, -Q::lift}, l[2] = {0.0f, 0.0f}, top[2];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[n][d][e] = 0.0f;

    // scores of a block of 32 keys: rows of the product are keys (8 (e / 4) + 4 half + e % 4), its columns queries (i)
    dl_f32x16 zero;
#pragma unroll
    for (int e = 0; e < 16; ++e) zero[e] = 0.0f;
    // what is not seen, and the reference, which follows the largest only where that is 2^8 times above it
    auto settle = [&](uint32_t key0) {
        if (key0 + 32u > whole_end) {
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                top[n] = -INFINITY;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    if (2 * (e & ~3) + (e & 3) > last[n] - (int32_t)key0) x[n][e] = -INFINITY;
                    top[n] = fmaxf(top[n], x[n][e]);
                }
            }
        }
        if (__any(top[0] > r[0] + 8.0f || top[1] > r[1] + 8.0f)) {
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const auto swapped = __builtin_amdgcn_permlane32_swap(dl_bits<uint32_t>(top[n]), dl_bits<uint32_t>(top[n]), false, false);
                const float most = fmaxf(r[n], fmaxf(dl_bits<float>((uint32_t)swapped[0]), dl_bits<float>((uint32_t)swapped[1])));
                const float ref = most == -INFINITY ? 0.0f : most, fade = __builtin_amdgcn_exp2f(r[n] - ref);
                r[n] = most;
                low[n] = ref - Q::lift;
                l[n] *= fade;
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) o[n][d] *= fade;
            }
        }
    };
    // The loop's two parts, in STEPS steps of two products each.  What a step does beside its products is a share of the other work, and what it
    // reads from LDS has been asked for two steps before (operands, in a ring of four) or one (scales), across the parts' borders.  The steps'
    // order is kept (left to the compiler, all weights come first and the products behind them).
    constexpr uint32_t STEPS = DP / 16;
    dl_u32x4 pf[2][2], ring[4];
    dl_f32x16 s[2];
    dl_f32x4 iu, ks, lu;
    auto inverse = [&](const chunk_tile<DP> &of, uint32_t kb, uint32_t quad) { iu = *(const dl_f32x4 *)&of.iu[32u * kb + 8u * quad + 4u * half]; };
    auto scales = [&](const chunk_tile<DP> &of, uint32_t kb, uint32_t quad) {
        ks = *(const dl_f32x4 *)&of.ks[32u * kb + 8u * quad + 4u * half];
        lu = *(const dl_f32x4 *)&of.lu[32u * kb + 8u * quad + 4u * half];
    };
    // The scores x of block kb of `in` become weights pf, while the products of block kb_then of `then` are taken.
    auto weights_and_products = [&](const chunk_tile<DP> &in, uint32_t kb, const chunk_tile<DP> &then, uint32_t kb_then) {
        constexpr uint32_t EACH = 8 / STEPS;
#pragma unroll
        for (uint32_t st = 0; st < STEPS; ++st) {
            ring[(st + 2) % 4] = st + 2 < STEPS ? feed_t::keys(then, kb_then, st + 2, i, half)
                                                : feed_t::values(in, kb, (st + 2 - STEPS) / (DP / 32), (st + 2 - STEPS) % (DP / 32), i, half);
#pragma unroll
            for (int n = 0; n < 2; ++n) s[n] = Q::mfma32(ring[st % 4], qf[n][st], st ? s[n] : zero);
#pragma unroll
            for (uint32_t g = st * EACH; g < st * EACH + EACH; ++g) {
                const uint32_t n = g % 2, e = 4 * (g / 2);
                float w[4];
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    w[f] = __builtin_amdgcn_exp2f(x[n][e + f] - low[n]);
                    l[n] = fmaf(w[f], iu[f], l[n]);
                }
                pf[n][e / 8][e % 8 / 2] = Q::pack(w[0], w[1]);
                pf[n][e / 8][e % 8 / 2 + 1] = Q::pack(w[2], w[3]);
                if (n && e < 12) inverse(in, kb, e / 4 + 1);
            }
            if (st + 1 == STEPS) scales(then, kb_then, 0);
            // (here, and not where they are needed)
#pragma unroll
            for (int n = 0; n < 2; ++n) asm volatile("" : "+v"(l[n]));
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int p = 0; p < 2; ++p) asm volatile("" : "+v"(pf[n][p]));
    };
    // The weights of block kb of `in` meet its values, while the scores of block kb_then of `scored` are scaled and the codes that have come go
    // to tile `then` (PUT) or the next ones are asked for.
    auto sums_and_scores = [&](const chunk_tile<DP> &in, uint32_t kb, const chunk_tile<DP> &scored, uint32_t kb_then, chunk_tile<DP> &then, const uint64_t (&rows_at)[CH_KEYS],
                               auto with_put) {
        constexpr bool PUT = decltype(with_put)::value;
        constexpr uint32_t LEFT = STEPS - 1;  // (the last of the products is not done before the first step's)
        uint64_t from[2] = {};
#pragma unroll
        for (uint32_t st = 0; st < STEPS; ++st) {
            if (st + 2 < STEPS)
                ring[(st + 2) % 4] = feed_t::values(in, kb, (st + 2) / (DP / 32), (st + 2) % (DP / 32), i, half);
            else if (!PUT)
                ring[(st + 2) % 4] = feed_t::keys(then, 1, st + 2 - STEPS, i, half);
#pragma unroll
            for (int n = 0; n < 2; ++n) o[n][st % (DP / 32)] = Q::mfma32(ring[st % 4], pf[n][st / (DP / 32)], o[n][st % (DP / 32)]);
            if constexpr (PUT) {
#pragma unroll
                for (uint32_t n = st * feed_t::PUT_PARTS / STEPS; n < (st + 1) * feed_t::PUT_PARTS / STEPS; ++n) feed.put_part(then, n);
            } else {
                // (rows a step before the loads from there)
                constexpr uint32_t MOST = (feed_t::LOAD_PARTS + LEFT - 1) / LEFT;
                static_assert(MOST <= 2 || DP < 128, "two rows on their way");
                if (st)
#pragma unroll
                    for (uint32_t n = 0; n < MOST; ++n)
                        if ((st - 1) * MOST + n < feed_t::LOAD_PARTS) feed.load_part(a, n < 2 ? from[n] : feed_t::load_from(rows_at, (st - 1) * MOST + n), (st - 1) * MOST + n);
#pragma unroll
                for (uint32_t n = 0; n < 2; ++n)
                    if (st < LEFT && n < MOST && st * MOST + n < feed_t::LOAD_PARTS) from[n] = feed_t::load_from(rows_at, st * MOST + n);
            }
            if (st) {
#pragma unroll
                for (uint32_t g = (st - 1) * 8 / LEFT; g < st * 8 / LEFT; ++g) {
                    const uint32_t n = g % 2, e = 4 * (g / 2);
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        x[n][e + f] = fmaf(s[n][e + f], ks[f], lu[f]);
                        top[n] = f || e ? fmaxf(top[n], x[n][e + f]) : x[n][e + f];
                    }
                    if (n && e < 12) scales(scored, kb_then, e / 4 + 1);
                }
            }
            if (st + 1 == STEPS) {
                if (PUT)
                    inverse(in, 1, 0);
                else
                    inverse(then, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    if (first < end) {
        feed.look_up(a, first);
        feed.hand_on(a, first, lds.rows_at[0], lds.alive_at[0]);
        __syncthreads();
        feed.load(a, lds.rows_at[0]);
        feed.look_up(a, first + CH_KEYS);
        feed.clear(lds.alive_at[0]);
        feed.put_codes(lds.tiles[0]);
        feed.put_scales(a, lds.tiles[0]);
        feed.hand_on(a, first + CH_KEYS, lds.rows_at[1], lds.alive_at[1]);
        __syncthreads();
        feed.load(a, lds.rows_at[1]);
        feed.look_up(a, first + 2 * CH_KEYS);
        if (__builtin_amdgcn_readfirstlane((int)lds.tiles[0].taken_apart)) feed_t::apart(lds.tiles[0]);
        inverse(lds.tiles[0], 0, 0);
#pragma unroll
        for (uint32_t st = 0; st < 2; ++st) ring[st] = feed_t::keys(lds.tiles[0], 1, st, i, half);
#pragma unroll
        for (uint32_t st = 0; st < DP / 16; ++st)
#pragma unroll
            for (int n = 0; n < 2; ++n) s[n] = Q::mfma32(feed_t::keys(lds.tiles[0], 0, st, i, half), qf[n][st], st ? s[n] : zero);
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t key = 8u * (e / 4) + 4u * half + e % 4;
                x[n][e] = fmaf(s[n][e], lds.tiles[0].ks[key], lds.tiles[0].lu[key]);
                top[n] = e ? fmaxf(top[n], x[n][e]) : x[n][e];
            }
    }
    uint32_t now = 0, slot = 0;
    for (uint32_t base = first; base < end; base += CH_KEYS) {
        // (behind the last step whatever lies in the next tile is worked on, and not used)
        const uint32_t next = now == 2u ? 0u : now + 1u;
        chunk_tile<DP> &in = lds.tiles[now], &then = lds.tiles[next];
        settle(base);
        weights_and_products(in, 0, in, 1);
        feed.clear(lds.alive_at[slot ^ 1u]);
        // (the scores are those of this tile's second block; what goes to the next tile is its codes)
        sums_and_scores(in, 0, in, 1, then, lds.rows_at[slot], std::true_type{});
        feed.put_scales(a, then);
        feed.hand_on(a, base + 2 * CH_KEYS, lds.rows_at[slot], lds.alive_at[slot]);
        __syncthreads();
#pragma unroll
        for (uint32_t st = 0; st < 2; ++st) ring[st] = feed_t::keys(then, 0, st, i, half);
        feed.look_up(a, base + 3 * CH_KEYS);
        if (base + CH_KEYS < end && __builtin_amdgcn_readfirstlane((int)then.taken_apart)) feed_t::apart(then);
        settle(base + 32u);
        weights_and_products(in, 1, then, 0);
        sums_and_scores(in, 1, then, 0, then, lds.rows_at[slot], std::false_type{});
        now = next;
        slot ^= 1u;
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) finish_row<Q, DP>(a, at, t, head, wave_row + 32u * n + i, half, r[n], l[n], o[n]);
}

// Joins the pieces of tiles that are cut.  DP / 4 lanes hold a row's sums, four each, and a workgroup has as many rows as its lanes hold: what it
// takes is the way to its pieces (9 of them 11.6 us with four times the rows a workgroup and half the loads at once).
template <int DP>
constexpr uint32_t JOIN_ROWS = CH_THREADS / (DP / 4);
template <class Q, int DP>
__global__ void __launch_bounds__(CH_THREADS) dl_chunk_join_kernel(const chunk_args a)
{
    constexpr uint32_t LANES = DP / 4, AHEAD = 8;
    const uint32_t D = a.c.head_dim, d0 = threadIdx.x % LANES * 4u;
    const uint32_t parts = a.tile_rows / JOIN_ROWS<DP>, part = blockIdx.x % parts, head = blockIdx.x / parts % a.c.heads;
    chunk_place at;
    if (!chunk_unit<true>(a, blockIdx.x / parts / a.c.heads, &at)) return;
    const chunk_rows t(a, at);
    const uint32_t pieces = max((t.end + at.keys - 1u) / at.keys, 1u);
    const uint32_t in = part * JOIN_ROWS<DP> + threadIdx.x / LANES, row = t.row0 + in;
    if (row >= t.rows) return;
    float r = -INFINITY, l = 0.0f;
    dl_f32x4 o = {0, 0, 0, 0};
    for (uint32_t p0 = 0; p0 < pieces; p0 += AHEAD) {
        dl_f32x2 rl[AHEAD];
        dl_f32x4 x[AHEAD];
#pragma unroll
        for (uint32_t k = 0; k < AHEAD; ++k) {
            const uint64_t from = ((uint64_t)(at.slot + min(p0 + k, pieces - 1u)) * a.c.heads + head) * a.tile_rows + in;
            rl[k] = a.rl[from];
            x[k] = d0 < D ? *(const dl_f32x4 *)(a.partial + from * D + d0) : dl_f32x4{0, 0, 0, 0};
            if (p0 + k >= pieces) rl[k] = dl_f32x2{-INFINITY, 0.0f}, x[k] = dl_f32x4{0, 0, 0, 0};
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
    const bool none = l == 0.0f;
    const uint32_t j = dl_divide(row, a.groups), h = head * a.group + row - j * a.group;
    const float f = none ? 0.0f : 1.0f / l;
    if (d0 < D)
        dl_store_at(a.out + (uint64_t)(t.first + j) * a.out_token + h * a.out_head + 2u * d0,
                    none ? dl_u32x2{0, 0} : dl_u32x2{Q::pack(o[0] * f, o[1] * f), Q::pack(o[2] * f, o[3] * f)});
    if (a.lse && d0 == 0)
        a.lse[(uint64_t)(t.first + j) * a.q_heads + h] = none ? -INFINITY : ((r == -INFINITY ? 0.0f : r) - Q::lift + log2f(l)) * DL_LN2;
}

struct chunk_shape {
    uint64_t units;     // at most so many pieces a head, over all sequences
    uint32_t most_cut;  // of them of sequences that are cut
    uint32_t tile_rows, slots;
    bool search;
};

int chunk_sizes(const dl_kv_cache *cache, const dl_chunk_attention_args *args, dl_cache_view *view, chunk_shape *sh)
{
    const int rc = dl_packed_sizes(cache, args, view);
    if (rc != DL_OK) return rc;
    *sh = chunk_shape{};
    if (!args->tokens || !args->q_heads || !args->batch) return DL_OK;
    const uint64_t rows = (uint64_t)args->tokens * (uint32_t)(args->q_heads / cache->heads);
    // every sequence begins a tile of its own
    // 256 rows a tile from 1024 rows a sequence on, where the table holds 2048 tokens and more.  256 : 128, us, 8 heads of 128, 32 query heads: on 30 720
    // tokens 256 queries (1024 rows) 167 : 190, 512 305 : 351; 8 sequences on 4000 with up to 128, 192, 256, 384 queries 89 : 86, 100 : 108, 140 : 147, 173 :
    // 191.  Prompts with nothing before them, 300, 750, 1024, 1500, 2048, 4096 tokens: 26 : 23, 42 : 39, 49 : 51, 76 : 73, 90 : 94, 184 : 207; four of up to that:
    // 34 : 31, 69 : 46, 57 : 58, 92 : 87, 132 : 134; 750 queries on 1500 tokens 72 : 74.  (The table stands in for the contexts, which the host does not know: in
    // wide tables such prompts have the former.)
    const uint64_t most = (uint64_t)args->max_pages * (uint32_t)cache->page_tokens;
    sh->tile_rows = cache->head_dim <= 128 && rows >= 1024u * (uint64_t)args->batch && most >= 2048u ? 64u * CH_WAVES : 32u * CH_WAVES;
    uint64_t tiles = rows / sh->tile_rows + (uint64_t)args->batch;
    if (tiles > rows) tiles = rows;
    // Workgroups at once, by the registers and LDS: two a compute unit up to head_dim 128 (64 where there are many rows), one above.
    sh->slots = cache->head_dim > 128 || (cache->head_dim > 64 && sh->tile_rows > 32u * CH_WAVES) ? 256u : 512u;
    // Two rounds of pieces at most, and no more than a step each.
    uint64_t cut = 2u * sh->slots / (uint32_t)cache->heads;
    if (cut > tiles * ((most + CH_KEYS - 1u) / CH_KEYS)) cut = tiles * ((most + CH_KEYS - 1u) / CH_KEYS);
    if (most > CH_KEYS && cut > 1u) sh->most_cut = (uint32_t)cut;
    sh->search = sh->most_cut && args->batch <= (int32_t)SEARCH_MAX && most <= (uint64_t)CH_KEYS << 20;
    sh->units = tiles + sh->most_cut;
    return DL_OK;
}

size_t chunk_slots(const chunk_shape &sh, uint32_t heads) { return (size_t)sh.most_cut * heads * sh.tile_rows; }

}  // namespace

extern "C" int64_t dl_chunk_attention_workspace(const dl_kv_cache *cache, const dl_chunk_attention_args *args)
{
    dl_cache_view view;
    chunk_shape sh;
    const int rc = chunk_sizes(cache, args, &view, &sh);
    if (rc != DL_OK) return rc;
    return (int64_t)(DL_CONTROL_BYTES + 16u + chunk_slots(sh, view.heads) * (sizeof(dl_f32x2) + view.head_dim * sizeof(float)));
}

extern "C" int dl_chunk_attention(const dl_kv_cache *cache, const dl_chunk_attention_args *args, void *stream)
{
    DL_LOCKED;
    if (!g_dl.inited) return DL_ERR_STATE;
    if (dl_device_error_pending()) return DL_ERR_LOST;
    chunk_args a;
    chunk_shape sh;
    int rc = chunk_sizes(cache, args, &a.c, &sh);
    if (rc != DL_OK) return rc;
    if (!sh.units) return DL_OK;
    rc = dl_cache_check(cache, 3, &a.c);
    if (rc != DL_OK) return rc;
    rc = dl_packed_setup(cache, args, (size_t)dl_chunk_attention_workspace(cache, args), &a.p);
    if (rc != DL_OK) return rc;
    if (!args->q || !args->out || (uint64_t)args->out % 2u) return DL_ERR_INVALID;
    a.q = (const char *)args->q;
    a.out = (char *)args->out;
    a.lse = args->lse;
    a.size = (uint32_t *)((char *)args->workspace + DL_CONTROL_BYTES);
    a.rl = (dl_f32x2 *)(a.size + 4);
    a.partial = (float *)(a.rl + chunk_slots(sh, a.c.heads));
    a.q_token = 2 * args->q_token_stride;
    a.q_head = 2 * args->q_head_stride;
    a.out_token = 2 * args->out_token_stride;
    a.out_head = 2 * args->out_head_stride;
    a.q_heads = (uint32_t)args->q_heads;
    a.group = a.q_heads / a.c.heads;
    a.groups = dl_make_divider(a.group ? a.group : 1u);
    a.tile_rows = sh.tile_rows;
    a.most_cut = sh.most_cut;
    a.search = sh.search;
    a.round = (float)sh.slots / (float)a.c.heads;
    a.scale = args->scale * DL_LOG2E;
    // (pieces may be more than a grid is high)
    const uint32_t deep = (uint32_t)((sh.units + 65534u) / 65535u);
    const dim3 grid(a.c.heads, (uint32_t)((sh.units + deep - 1u) / deep), deep);
    hipStream_t hs = (hipStream_t)stream;
    dl_with_16bit(args->type, [&](auto q) {
        auto go = [&](auto dp) {
            constexpr int DP = decltype(dp)::value;
            dl_with_format(cache->format, [&](auto c) {
                if constexpr (DP <= 128)
                    if (sh.tile_rows > 32u * CH_WAVES) {
                        hipLaunchKernelGGL((dl_chunk_wide_kernel<decltype(q), decltype(c), DP>), grid, dim3(CH_THREADS), 0, hs, a);
                        return;
                    }
                hipLaunchKernelGGL((dl_chunk_kernel<decltype(q), decltype(c), DP>), grid, dim3(CH_THREADS), 0, hs, a);
            });
            if (sh.most_cut)
                hipLaunchKernelGGL((dl_chunk_join_kernel<decltype(q), DP>), dim3((sh.most_cut + 1u) / 2u * a.c.heads * (sh.tile_rows / JOIN_ROWS<DP>)), dim3(CH_THREADS), 0, hs, a);
        };
        if (a.c.head_dim <= 64)
            go(std::integral_constant<int, 64>{});
        else if (a.c.head_dim <= 128)
            go(std::integral_constant<int, 128>{});
        else
            go(std::integral_constant<int, 256>{});
    });
    DL_HIP(hipGetLastError());
    t_dl_last.mode = DL_MODE_ONESHOT;
    return DL_OK;
}
