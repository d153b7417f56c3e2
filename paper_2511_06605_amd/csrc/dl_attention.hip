// Attention of a batch that shares a prefix, over a paged cache in 8 bits (dl_prefix_attention).
//
// With s the scores in units of ln 2 and u the scales of the values, a query's output is sum of 2^s u V / sum of 2^s over the codes V
// of what it sees.  The sums are taken piece by piece with a running reference r = largest s + log2 u so far:
//   w = 2^(s + log2 u - r) <= 1,   O += w V,   l += w / u,
// both multiplied by 2^(r before - r) when r grows.  So the weights that go to the matrix units in 16 bits are at most 1
// (times 2^15 for float16, see lift) whatever the scales are, and the codes go there as they are (each is a value of both
// 16-bit types): the only rounding on the way is that of w.  Pieces of the same row are joined in the same manner, in a fixed order.
//
// The key axis is cut into pieces.  A piece of the prefix serves the queries of all sequences at once: they are the rows of
// one product.  A piece of a sequence's own tokens serves the query heads that share a head of the cache.  All pieces of
// both kinds are one launch; a second one joins each row's pieces.
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
    dl_f32x2 *rl;    // per piece and row: r and l
    float *partial;  // per piece and row: head_dim sums
    int64_t q_seq, q_token, q_head, out_seq, out_token, out_head;  // bytes
    int64_t pages_stride;
    uint32_t prefix_tokens, own_most;  // own_most: max_pages * page_tokens
    uint32_t batch, q_tokens, q_heads, group;
    uint32_t rows;                     // batch * q_tokens * q_heads
    uint32_t prefix_tiles, prefix_splits, prefix_piece;
    uint32_t own_tiles, own_splits;
    float scale;                       // times log2 e
};

// How a sequence's own tokens are cut: pieces of this many.
__device__ __forceinline__ uint32_t own_piece(const att_args &a, uint32_t len)
{
    const uint32_t even = (len + a.own_splits - 1u) / a.own_splits;
    return (even + STEP - 1u) / STEP * STEP;
}
__device__ __forceinline__ uint32_t own_len(const att_args &a, uint32_t b)
{
    return a.own_most ? min((uint32_t)max(a.lens[b], 0), a.own_most) : 0u;
}
__device__ __forceinline__ uint32_t queries(const att_args &a, uint32_t b)
{
    return a.q_lens ? min((uint32_t)max(a.q_lens[b], 0), a.q_tokens) : a.q_tokens;
}

// A vector of N bytes, N = 4, 8, 16, as words
template <int N>
struct words {
    uint32_t w[N / 4];
};
template <int N>
__device__ __forceinline__ words<N> load_words(const char *p)
{
    return dl_load_at<words<N>>(p);
}

// NT tiles of 16 rows against the keys first .. end - 1 of one head.
template <class Q, class C, int DP, int NT>
__device__ void attend(const att_args &a, uint32_t head, const int32_t *table, uint32_t first, uint32_t end, const char *const (&qrow)[NT],
                       const int32_t (&last)[NT], const uint32_t (&row)[NT], const bool (&store)[NT], uint32_t piece)
{
    constexpr int KB = DP / 4;    // bytes of a key's row that a lane holds: dims KB * g ..
    constexpr int VB = DP / 16;   // bytes of a value's row that a lane holds: dims VB * i ..
    constexpr int STEPS = DP / 32;
    const uint32_t lane = threadIdx.x % 64u, wave = threadIdx.x / 64u;
    const uint32_t i = lane % 16u, g = lane / 16u;
    const uint32_t D = a.c.head_dim;

    __shared__ float scales[ATT_WAVES][3][TILE];
    __shared__ float joined[2][NT * DP / 16 * 4 + 2 * NT][64];

    // queries: lane (i, g) holds dims KB * g .. of row i, eight a step
    dl_u32x4 qf[NT][STEPS];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const uint32_t d = KB * g + 8u * s;
            qf[n][s] = d < D ? dl_load_at<dl_u32x4>(qrow[n] + 2u * d) : dl_u32x4{0, 0, 0, 0};
        }

    dl_f32x4 o[NT][DP / 16];
    float r[NT], l[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        r[n] = -INFINITY;
        l[n] = 0.0f;
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) o[n][t] = dl_f32x4{0, 0, 0, 0};
    }

    for (uint32_t base = first + wave * TILE; base < end; base += STEP) {
        auto locate = [&](uint32_t key, bool *ok) {
            *ok = key < end;
            const uint32_t k = min(key, end - 1u);
            const uint32_t p = dl_divide(k, a.c.page);
            uint32_t page = (uint32_t)table[p];
            if (page >= a.c.pages) *ok = false, page = 0;
            return (int64_t)page * a.c.page_stride + (int64_t)(k - p * a.c.page.d) * a.c.token_stride + (int64_t)head * a.c.head_stride;
        };
        // keys: lane (i, g) holds its part of keys 8 (i / 4) + 4 t + i % 4, t = 0, 1
        words<16> kw[2][KB / 16];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            bool ok;
            const char *p = a.c.k + locate(base + 8u * (i / 4u) + 4u * t + i % 4u, &ok) + KB * g;
#pragma unroll
            for (int s = 0; s < KB / 16; ++s) kw[t][s] = KB * g + 16u * s < D ? load_words<16>(p + 16 * s) : words<16>{};
        }
        // values: lane (i, g) holds its part of keys 8 g + e
        words<VB> vw[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            bool ok;
            const char *p = a.c.v + locate(base + 8u * g + e, &ok) + VB * i;
            vw[e] = VB * i < D && ok ? load_words<VB>(p) : words<VB>{};
        }
        // scales: a lane a key, keys' in the lower half and values' in the upper
        bool alive;
        {
            const uint32_t key = base + lane % TILE, k = min(key, end - 1u);
            const uint32_t p = dl_divide(k, a.c.page);
            uint32_t page = (uint32_t)table[p];
            alive = key < end && page < a.c.pages;
            if (page >= a.c.pages) page = 0;
            const int64_t at = (int64_t)page * a.c.scale_page_stride + (int64_t)(k - p * a.c.page.d) * a.c.scale_token_stride +
                               (int64_t)head * a.c.scale_head_stride;
            if (lane < TILE) {
                scales[wave][0][lane] = alive ? a.c.k_scale[at] * a.scale : 0.0f;
            } else {
                const float u = fmaxf(a.c.v_scale[at], 0x1p-120f);
                const bool nan = a.c.v_scale[at] != a.c.v_scale[at];
                scales[wave][1][lane - TILE] = !alive ? -INFINITY : nan ? __builtin_nanf("") : __builtin_amdgcn_logf(u);
                scales[wave][2][lane - TILE] = !alive ? 0.0f : __builtin_amdgcn_rcpf(u);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        float ks[8], lu[8], iu[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            ks[e] = scales[wave][0][8u * g + e];
            lu[e] = scales[wave][1][8u * g + e];
            iu[e] = scales[wave][2][8u * g + e];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        // scores: the product's rows are keys (8 g + 4 t + j in lane (i, g)), its columns queries (i)
        dl_f32x4 s[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = dl_f32x4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                const dl_u32x2 x = C::template spread<Q>(kw[t][st / 2].w[2 * (st % 2)]), y = C::template spread<Q>(kw[t][st / 2].w[2 * (st % 2) + 1]);
                const dl_u32x4 kf = {x[0], x[1], y[0], y[1]};
#pragma unroll
                for (int n = 0; n < NT; ++n) s[n][t] = Q::mfma16(kf, qf[n][st], s[n][t]);
            }
        dl_u32x4 pf[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float x[8], top = -INFINITY;
            bool seen[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                seen[e] = (int32_t)(base + 8u * g + e) <= last[n] && lu[e] != -INFINITY;
                x[e] = seen[e] ? fmaf(s[n][e / 4][e % 4], ks[e], lu[e]) : -INFINITY;
                top = fmaxf(top, x[e]);
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float now = fmaxf(r[n], top);
            const float ref = now == -INFINITY ? 0.0f : now;
            const float fade = __builtin_amdgcn_exp2f(r[n] - ref);
            r[n] = now;
            const float low = ref - Q::lift;
            float w[8], sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = __builtin_amdgcn_exp2f(x[e] - low);
                sum += seen[e] ? w[e] * iu[e] : 0.0f;
            }
            l[n] = l[n] * fade + sum;
#pragma unroll
            for (int t = 0; t < DP / 16; ++t) o[n][t] *= fade;
            pf[n] = dl_u32x4{Q::pack(w[0], w[1]), Q::pack(w[2], w[3]), Q::pack(w[4], w[5]), Q::pack(w[6], w[7])};
        }
        // sums: the product's rows are dims (VB * (4 g + j) + t in lane (i, g)), its columns queries (i)
#pragma unroll
        for (int q4 = 0; q4 < VB / 4; ++q4) {
            // four keys' four dims each, turned to four dims' four keys each
            dl_u32x2 half[2][4];  // [keys 0 .. 3 and 4 .. 7][dim]: four elements
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t w0 = vw[4 * h].w[q4], w1 = vw[4 * h + 1].w[q4], w2 = vw[4 * h + 2].w[q4], w3 = vw[4 * h + 3].w[q4];
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
                for (int n = 0; n < NT; ++n) o[n][4 * q4 + t] = Q::mfma16(vf, pf[n], o[n][4 * q4 + t]);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] += __shfl_xor(l[n], 16);
        l[n] += __shfl_xor(l[n], 32);
    }
    // the wavefronts' sums, two by two: 2 and 3 to 0 and 1, then 1 to 0
#pragma unroll
    for (uint32_t half = ATT_WAVES / 2; half; half /= 2) {
        if (wave >= half && wave < 2 * half) {
            float(*to)[64] = joined[wave - half];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                to[2 * n][lane] = r[n];
                to[2 * n + 1][lane] = l[n];
#pragma unroll
                for (int t = 0; t < DP / 16; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) to[2 * NT + (n * (DP / 16) + t) * 4 + j][lane] = o[n][t][j];
            }
        }
        __syncthreads();
        if (wave < half) {
            const float(*from)[64] = joined[wave];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float r2 = from[2 * n][lane], now = fmaxf(r[n], r2), ref = now == -INFINITY ? 0.0f : now;
                const float f = __builtin_amdgcn_exp2f(r[n] - ref), f2 = __builtin_amdgcn_exp2f(r2 - ref);
                r[n] = now;
                l[n] = l[n] * f + from[2 * n + 1][lane] * f2;
#pragma unroll
                for (int t = 0; t < DP / 16; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[n][t][j] = o[n][t][j] * f + from[2 * NT + (n * (DP / 16) + t) * 4 + j][lane] * f2;
            }
        }
        __syncthreads();
    }
    if (wave) return;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (!store[n]) continue;
        const uint64_t at = (uint64_t)piece * a.rows + row[n];
        if (g == 0) a.rl[at] = dl_f32x2{r[n], l[n]};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t d = VB * (4u * g + j);
            if (d >= D) continue;
            float *to = a.partial + at * D + d;
#pragma unroll
            for (int t = 0; t < VB; t += 4) *(dl_f32x4 *)(to + t) = dl_f32x4{o[n][t][j], o[n][t + 1][j], o[n][t + 2][j], o[n][t + 3][j]};
        }
    }
}

template <class Q, class C, int DP, int NT>
__global__ void __launch_bounds__(ATT_THREADS) dl_attention_kernel(const att_args a)
{
    const uint32_t i = threadIdx.x % 16u;
    const char *qrow[NT];
    int32_t last[NT];
    uint32_t row[NT];
    bool store[NT];
    const uint32_t heads = a.c.heads, seq_rows = a.q_tokens * a.group;
    const uint32_t shared = heads * a.prefix_tiles * a.prefix_splits;
    const bool prefix = blockIdx.x < shared;
    const uint32_t x = prefix ? blockIdx.x : blockIdx.x - shared;
    const uint32_t head = x % heads, tiles = prefix ? a.prefix_tiles : a.own_tiles, tile = x / heads % tiles;
    uint32_t piece = x / heads / tiles, b0 = 0, first, end, rows;
    const int32_t *table;
    int32_t own_last = 0;  // of query 0
    if (prefix) {
        first = piece * a.prefix_piece;
        end = min(first + a.prefix_piece, a.prefix_tokens);
        table = a.prefix_pages;
        rows = a.batch * seq_rows;
    } else {
        b0 = piece % a.batch;
        piece /= a.batch;
        const uint32_t len = own_len(a, b0), step = own_piece(a, len);
        first = piece * step;
        if (first >= len) return;
        end = min(first + step, len);
        table = a.pages + b0 * a.pages_stride;
        rows = seq_rows;
        own_last = (int32_t)len - (int32_t)queries(a, b0);
        piece += a.prefix_splits;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        uint32_t at = (tile * NT + n) * 16u + i;
        store[n] = at < rows;
        at = min(at, rows - 1u);
        const uint32_t b = b0 + at / seq_rows, in = at % seq_rows, j = in / a.group, h = head * a.group + in - j * a.group;
        qrow[n] = a.q + b * a.q_seq + j * a.q_token + h * a.q_head;
        row[n] = (b * a.q_tokens + j) * a.q_heads + h;
        last[n] = prefix ? (int32_t)end - 1 : min((int32_t)end - 1, own_last + (int32_t)j);
    }
    attend<Q, C, DP, NT>(a, head, table, first, end, qrow, last, row, store, piece);
}

// Joins the pieces of a row, a wavefront a row.
template <class Q>
__global__ void __launch_bounds__(ATT_THREADS) dl_attention_join_kernel(const att_args a)
{
    const uint32_t row = (blockIdx.x * ATT_THREADS + threadIdx.x) / 64u, lane = threadIdx.x % 64u;
    if (row >= a.rows) return;
    const uint32_t h = row % a.q_heads, bj = row / a.q_heads, b = bj / a.q_tokens, j = bj - b * a.q_tokens, D = a.c.head_dim;
    uint32_t pieces = 0;
    if (j < queries(a, b)) {
        const uint32_t len = own_len(a, b), step = own_piece(a, len);
        pieces = a.prefix_splits + (len ? (len + step - 1u) / step : 0u);
    }
    float r = -INFINITY;
    for (uint32_t p = lane; p < pieces; p += 64u) r = fmaxf(r, a.rl[(uint64_t)p * a.rows + row][0]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) r = fmaxf(r, __shfl_xor(r, d));
    const float ref = r == -INFINITY ? 0.0f : r;
    float l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t d0 = 4u * lane;
    for (uint32_t p = 0; p < pieces; ++p) {
        const uint64_t at = (uint64_t)p * a.rows + row;
        const dl_f32x2 rl = a.rl[at];
        const float f = __builtin_amdgcn_exp2f(rl[0] - ref);
        l += rl[1] * f;
        if (d0 < D) {
            const dl_f32x4 x = *(const dl_f32x4 *)(a.partial + at * D + d0);
#pragma unroll
            for (int t = 0; t < 4; ++t) o[t] += x[t] * f;
        }
    }
    const bool none = l == 0.0f;
    if (d0 < D) {
        char *to = a.out + b * a.out_seq + j * a.out_token + h * a.out_head + 2u * d0;
        const float f = none ? 0.0f : 1.0f / l;
        dl_store_at(to, none ? dl_u32x2{0, 0} : dl_u32x2{Q::pack(o[0] * f, o[1] * f), Q::pack(o[2] * f, o[3] * f)});
    }
    if (a.lse && lane == 0) a.lse[row] = none ? -INFINITY : (ref - Q::lift + log2f(l)) * 0.69314718055994530942f;
}

uint32_t ceil_div(uint64_t a, uint64_t b) { return (uint32_t)((a + b - 1) / b); }

struct att_shape {
    uint32_t nt;
    uint32_t prefix_tiles, prefix_splits, prefix_piece, own_tiles, own_splits;
    uint64_t rows;
};

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
    if (rows > INT32_MAX) return DL_ERR_INVALID;
    *sh = att_shape{};
    sh->rows = (uint64_t)rows;
    if (!rows) return DL_OK;
    const uint32_t group = (uint32_t)(args->q_heads / cache->heads), seq_rows = (uint32_t)args->q_tokens * group;
    const uint64_t all_rows = (uint64_t)args->batch * seq_rows;
    sh->nt = seq_rows > 16u ? 2 : 1;
    auto cut = [&](uint64_t units, uint64_t keys) {  // pieces of an axis of `keys`, where there are `units` such axes
        if (!keys) return 0u;
        const uint64_t wanted = units >= 1024u ? 1u : (1024u + units - 1u) / units, most = (keys + STEP - 1u) / STEP;
        return (uint32_t)(wanted < most ? wanted : most);
    };
    const uint64_t prefix = cache->pages ? (uint64_t)args->prefix_tokens : 0u, own = cache->pages ? (uint64_t)args->max_pages * cache->page_tokens : 0u;
    sh->prefix_tiles = ceil_div(all_rows, 16u * sh->nt);
    sh->own_tiles = ceil_div(seq_rows, 16u * sh->nt);
    sh->prefix_splits = cut((uint64_t)cache->heads * sh->prefix_tiles, prefix);
    if (sh->prefix_splits) {
        sh->prefix_piece = ceil_div(ceil_div(prefix, sh->prefix_splits), STEP) * STEP;
        sh->prefix_splits = ceil_div(prefix, sh->prefix_piece);
    }
    sh->own_splits = cut((uint64_t)cache->heads * sh->own_tiles * (uint32_t)args->batch, own);
    return DL_OK;
}

uint64_t att_pieces(const att_shape &sh) { return (uint64_t)sh.prefix_splits + sh.own_splits; }

}  // namespace

extern "C" int64_t dl_prefix_attention_workspace(const dl_kv_cache *cache, const dl_prefix_attention_args *args)
{
    dl_cache_view view;
    att_shape sh;
    const int rc = att_setup(cache, args, &view, &sh);
    if (rc != DL_OK) return rc;
    const uint64_t at = att_pieces(sh) * sh.rows;
    return (int64_t)(DL_CONTROL_BYTES + (at * sizeof(dl_f32x2) + 15u) / 16u * 16u + at * view.head_dim * sizeof(float));
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
    a.rl = (dl_f32x2 *)((char *)args->workspace + DL_CONTROL_BYTES);
    a.partial = (float *)((char *)a.rl + (att_pieces(sh) * sh.rows * sizeof(dl_f32x2) + 15u) / 16u * 16u);
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
    a.own_splits = sh.own_splits ? sh.own_splits : 1u;
    a.scale = args->scale * 1.44269504088896340736f;
    const uint64_t shared = (uint64_t)a.c.heads * sh.prefix_tiles * sh.prefix_splits;
    const uint64_t grid = shared + (uint64_t)a.c.heads * sh.own_tiles * a.batch * sh.own_splits;
    if (grid > INT32_MAX) return DL_ERR_INVALID;
    hipStream_t hs = (hipStream_t)stream;
    dl_with_16bit(args->type, [&](auto q) {
        if (grid)
            dl_with_format(cache->format, [&](auto c) {
                auto go = [&](auto dp, auto nt) {
                    hipLaunchKernelGGL((dl_attention_kernel<decltype(q), decltype(c), decltype(dp)::value, decltype(nt)::value>), dim3((uint32_t)grid),
                                       dim3(ATT_THREADS), 0, hs, a);
                };
                auto with_rows = [&](auto dp) {
                    if (sh.nt == 1)
                        go(dp, std::integral_constant<int, 1>{});
                    else
                        go(dp, std::integral_constant<int, 2>{});
                };
                if (a.c.head_dim <= 64)
                    with_rows(std::integral_constant<int, 64>{});
                else if (a.c.head_dim <= 128)
                    with_rows(std::integral_constant<int, 128>{});
                else
                    with_rows(std::integral_constant<int, 256>{});
            });
        hipLaunchKernelGGL((dl_attention_join_kernel<decltype(q)>), dim3(ceil_div(sh.rows, ATT_WAVES)), dim3(ATT_THREADS), 0, hs, a);
    });
    DL_HIP(hipGetLastError());
    t_dl_last.mode = DL_MODE_ONESHOT;
    return DL_OK;
}
