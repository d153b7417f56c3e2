// What cached tokens have been given by queries whose sums are known (dl_kv_weigh).
//
// With the scores s and lse in units of ln 2, a token is given the sum over queries and heads of 2^(s - lse).  The lse is known, so no
// maximum is looked for and the sum is over the queries alone: a wavefront has 32 keys, as the left operand of 32 x 32 x 16 products whose
// columns are queries, and adds up in registers over heads and queries, a query a lane; the lanes' sums are added at the end.  So in the
// loop a lane needs one lse, and its keys' scales stay where they are.  All sums are taken in a fixed order.
//
// Measured: one query of 32 heads on 5000 tokens (8 heads of 128, 5.3 MB) 5.4 - 5.7 us, a launch and the way from length to table to codes; the last 32
// queries of 8 prompts of up to 16 400 (4 heads, 28 query heads, 48 MB, 11.5 GFLOP) 34 - 38 us in two launches (33 and 5), 2048 queries behind 2048
// tokens (8 heads, 32 query heads) 188 us.  What bounds the second is vector instructions, 139 a tile of 32 x 32 besides its 8 products, and waiting: for
// half of their time wavefronts wait for memory, LDS or each other, as few tiles a workgroup do not cover the way to the first.  Four of the instructions
// keep what is no number in a query out of the sums (without: 180 us; a first pass without and a second one where a sum is none: 185, and twice the code).
#include "dl_codes.h"
#include "dl_internal.h"
#include "dl_packed.h"

namespace {

struct weigh_args {
    dl_cache_view c;
    dl_packed p;
    const char *q;
    const float *lse, *before;
    float *weights;
    int64_t q_token, q_head;  // bytes
    int64_t before_stride, weights_stride;
    uint32_t width;        // entries of a row: max_pages * page_tokens (also where the pool has no pages)
    uint32_t q_heads, group;
    dl_divider groups;  // by group
    uint32_t sharing;      // few queries: wavefronts that share the heads of their keys: 1, 2, 4 or 8
    // many queries: the heads are shared out over `parts` workgroups, which leave their sums in partial [part][batch][width] (one: none)
    uint32_t parts;
    float *partial;
    float scale;  // times log2 e
};

// The last step of either kernel: x[e] of lane (i, half) is a sum over some queries for key 8 (e / 4) + 4 half + e % 4; over the 32 lanes that hold
// the same keys, halves of them swap halves of their sums, so that lane i ends with that of e = i % 16.
__device__ __forceinline__ float over_lanes(float (&x)[16], uint32_t i)
{
#pragma unroll
    for (int d = 8; d >= 1; d /= 2)
#pragma unroll
        for (int e = 0; e < d; ++e) {
            const bool up = i & (uint32_t)d;
            const float low = x[e], high = x[e + d];
            x[e] = (up ? high : low) + __shfl_xor(up ? low : high, d);
        }
    return x[0] + __shfl_xor(x[0], 16);
}

// A query's lse in units of ln 2: infinite where it is no finite number.
__device__ __forceinline__ float lse_of(float given) { return fabsf(given) < INFINITY ? given * DL_LOG2E : INFINITY; }

// A tile's scores s: rows are keys (8 (e / 4) + 4 half + e % 4, with the scales ks), columns queries.  lse: by lse_of; the scores of a query
// that gives nothing may be no numbers either, and count as 0.  Lanes that have no row have the last one's scores and lse.  masked: keys from
// `seen` + 1 on are not seen by the lane's query.
__device__ __forceinline__ void add_weights(dl_f32x16 &s, const dl_f32x4 (&ks)[4], float lse, bool row, bool masked, int32_t seen, uint32_t half, float (&sum)[16])
{
    const bool nothing = lse == INFINITY;
    if (__any(nothing)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = nothing ? 0.0f : s[e];
    }
    if (!row) lse = INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = fmaf(s[e], ks[e / 4][e % 4], -lse);
    if (masked) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (2 * (e & ~3) + (e & 3) > seen - 4 * (int32_t)half) s[e] = -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[e] += __builtin_amdgcn_exp2f(s[e]);
}

// A lane's key: where its codes and its scale are, and whether it is one.
struct weigh_key {
    const char *codes, *scale;
    bool alive;
    __device__ __forceinline__ weigh_key(const weigh_args &a, uint32_t b, uint32_t key, uint32_t len)
    {
        const uint32_t at = min(key, len - 1u), n = dl_divide(at, a.c.page), in = at - n * a.c.page.d;
        uint32_t page = (uint32_t)a.p.pages[b * a.p.pages_stride + n];
        alive = page < a.c.pages && key < len;
        page = page < a.c.pages ? page : 0u;
        codes = a.c.k + (uint64_t)page * a.c.page_stride + (uint64_t)in * a.c.token_stride;
        scale = (const char *)a.c.k_scale + (uint64_t)page * a.c.scale_page_stride + (uint64_t)in * a.c.scale_token_stride;
    }
};

// Few queries: what is read is the keys.  The wavefronts of a workgroup share out the heads of their keys, and every operand comes from memory
// straight into registers.
// WHOLE: head_dim is DP, and the places of a row's pieces are known.
constexpr uint32_t FEW_WAVES = 8;
template <class Q, class C, int DP, bool WHOLE>
__global__ void __launch_bounds__(64 * FEW_WAVES, DP <= 128 ? 4 : 2) dl_weigh_few_kernel(const weigh_args a)
{
    constexpr uint32_t PAIRS = DP / 32;  // of pieces of 16 dims, one for each half of the wavefront
    __shared__ __align__(16) float sums[FEW_WAVES][32];  // (the scales of its keys, until a wavefront has its sums)
    const uint32_t lane = threadIdx.x % 64u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
    const uint32_t i = lane % 32u, half = lane / 32u, D = WHOLE ? DP : a.c.head_dim, b = blockIdx.y;
    const uint32_t share = wave % a.sharing, block_keys = 32u * (FEW_WAVES / a.sharing);
    const uint32_t first = a.p.start(b), queries = a.p.queries(b, first), rows = queries * a.group, len = a.p.len(b);
    const int32_t ahead = (int32_t)len - (int32_t)queries;  // query j sees the keys up to ahead + j
    const uint32_t block0 = (blockIdx.z * gridDim.x + blockIdx.x) * block_keys;
    if (block0 >= a.width) return;
    const uint32_t base = block0 + wave / a.sharing * 32u;
    float sum[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[e] = 0.0f;
    uint32_t dead = ~0u;  // bit key: nothing is given to it
    if (base < len && rows) {
        const weigh_key key(a, b, base + i, len);
        dead = (uint32_t)__ballot(!key.alive);
        // rows before the first that sees any of the keys are left out, from row whole on all keys are seen
        const int64_t since = ((int64_t)base - ahead) * a.group, until = ((int64_t)base + 31 - ahead) * a.group;
        const uint32_t row0 = (uint32_t)max(since, (int64_t)0) & ~31u, whole = (uint32_t)max(until, (int64_t)0);
#pragma unroll 1
        for (uint32_t head = share; head < a.c.heads; head += a.sharing) {
            dl_u32x4 qf[2 * PAIRS];
            float given;
            int32_t last;
            auto load_queries = [&](uint32_t r0) {
                const uint32_t row = min(r0 + i, rows - 1u), j = dl_divide(row, a.groups), h = head * a.group + row - j * a.group;
                const char *const q = a.q + (uint64_t)(first + j) * a.q_token + h * a.q_head;
                given = a.lse[(uint64_t)(first + j) * a.q_heads + h];
                last = ahead + (int32_t)j - (int32_t)base;
#pragma unroll
                for (uint32_t x = 0; x < 2 * PAIRS; ++x)  // (behind head_dim the keys are zero)
                    qf[x] = dl_load_at<dl_u32x4>(q + 2u * min(16u * (2u * (x / 2) + half) + 8u * (x % 2), D - 8u));
            };
            load_queries(row0);
            dl_words<16> codes[PAIRS];
#pragma unroll
            for (uint32_t x = 0; x < PAIRS; ++x) codes[x] = dl_load_words<16>(key.codes + head * a.c.head_stride + min(16u * (2u * x + half), D - 16u));
#pragma unroll
            for (uint32_t x = 0; x < PAIRS; ++x)
                if (16u * (2u * x + half) >= D) codes[x] = dl_words<16>{};
            const float scale = *(const float *)(key.scale + head * a.c.scale_head_stride);
            // (what is none gets nothing in the end, but a number until then)
            if (half == 0) sums[wave][i] = key.alive ? scale * a.scale : 0.0f;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll 1
            for (uint32_t r0 = row0; r0 < rows; r0 += 32u) {
                const float lse = lse_of(given);
                const int32_t seen = last;
                // (elements and scales are made and read anew for each tile: kept, they would cost half the wavefronts)
#pragma unroll
                for (uint32_t x = 0; x < PAIRS; ++x)
#pragma unroll
                    for (uint32_t u = 0; u < 4; ++u) asm volatile("" : "+v"(codes[x].w[u]));
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                dl_f32x16 s;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = 0.0f;
#pragma unroll
                for (uint32_t x = 0; x < 2 * PAIRS; ++x) {
                    const dl_u32x2 lo = C::template spread<Q>(codes[x / 2].w[2 * (x % 2)]), hi = C::template spread<Q>(codes[x / 2].w[2 * (x % 2) + 1]);
                    s = Q::mfma32(dl_u32x4{lo[0], lo[1], hi[0], hi[1]}, qf[x], s);
                }
                // the next rows are on their way while this one's weights are taken
                if (r0 + 32u < rows) load_queries(r0 + 32u);
                dl_f32x4 ks[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) ks[e] = *(const dl_f32x4 *)&sums[wave][8u * e + 4u * half];
                add_weights(s, ks, lse, r0 + i < rows, r0 < whole, seen, half, sum);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    const float its = over_lanes(sum, i);
    if (i < 16u) sums[wave][8u * (i / 4u) + 4u * half + i % 4u] = its;
    __syncthreads();
    const uint32_t key = base + i;
    if (share == 0 && half == 0 && key < a.width) {
        float all = sums[wave][i];
        for (uint32_t w = 1; w < a.sharing; ++w) all += sums[wave + w][i];
        if (dead >> i & 1u) all = 0.0f;
        a.weights[b * a.weights_stride + key] = (a.before ? a.before[b * a.before_stride + key] : 0.0f) + all;
    }
}

// Many queries: a workgroup's wavefronts have keys of their own and take the same rows of the same head at a time, which go through LDS once for
// all of them: in registers a lane would load a row's pieces, and every load touch as many lines as there are rows.  Rows lie 16 bytes apart,
// so that eight neighbouring lanes, a row each, use all banks; while a tile of 32 rows is worked on, the next one is on its way.  What a product needs from LDS is asked for two products before.
constexpr uint32_t MANY_THREADS = 512, MANY_KEYS = 32 * MANY_THREADS / 64;
// Heads are shared out up to so many workgroups.  512, 1024, 2048, 4096: 8 prompts (see the top) 38.8, 37.5, 38.8, 38.9 us; 4 of up to 16 400 tokens, 8 heads
// 28.6, 27.7, 31.4, 31.4; one with 4 heads 16.7 - 16.9, one of 2048 queries the same with any.
constexpr uint32_t MANY_BLOCKS = 1024;
template <class Q, class C, int DP>
__global__ void __launch_bounds__(MANY_THREADS, DP <= 128 ? 4 : 2) dl_weigh_many_kernel(const weigh_args a)
{
    constexpr uint32_t PAIRS = DP / 32, PIECES = DP / 8, LOADS = (32 * PIECES + MANY_THREADS - 1) / MANY_THREADS;
    constexpr uint32_t ROW = PIECES * 4 + 4;
    __shared__ __align__(16) uint32_t tiles[2][32 * ROW];
    __shared__ float lses[2][32];
    __shared__ __align__(16) float scales[MANY_THREADS / 64][32];
    const uint32_t lane = threadIdx.x % 64u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
    const uint32_t i = lane % 32u, half = lane / 32u, D = a.c.head_dim, b = blockIdx.y;
    const uint32_t first = a.p.start(b), queries = a.p.queries(b, first), rows = queries * a.group, len = a.p.len(b);
    const int32_t ahead = (int32_t)len - (int32_t)queries;
    const uint32_t at = blockIdx.z * gridDim.x + blockIdx.x, part = at % a.parts, block0 = at / a.parts * MANY_KEYS, base = block0 + wave * 32u;
    if (block0 >= a.width) return;
    const uint32_t head0 = part * a.c.heads / a.parts, heads_end = (part + 1u) * a.c.heads / a.parts;
    float sum[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[e] = 0.0f;
    uint32_t dead = ~0u;
    if (block0 < len && rows) {
        const weigh_key key(a, b, base + i, len);
        dead = (uint32_t)__ballot(!key.alive);
        const int64_t of_block = ((int64_t)block0 - ahead) * a.group;
        const uint32_t row0 = (uint32_t)max(of_block, (int64_t)0) & ~31u;
        const int64_t since = ((int64_t)base - ahead) * a.group, until = ((int64_t)base + 31 - ahead) * a.group;
        const uint32_t from = base < len ? (uint32_t)max(since, (int64_t)0) : ~0u, whole = (uint32_t)max(until, (int64_t)0);
        dl_u32x4 staged[LOADS];
        float staged_lse = INFINITY;
        auto stage = [&](uint32_t head, uint32_t r0) {
#pragma unroll
            for (uint32_t x = 0; x < LOADS; ++x) {
                const uint32_t n = threadIdx.x + x * MANY_THREADS, row = min(r0 + n / PIECES, rows - 1u), j = dl_divide(row, a.groups);
                const char *const q = a.q + (uint64_t)(first + j) * a.q_token + (head * a.group + row - j * a.group) * a.q_head;
                staged[x] = dl_load_at<dl_u32x4>(q + 2u * min(n % PIECES * 8u, D - 8u));
            }
            if (threadIdx.x < 32u) {
                const uint32_t row = min(r0 + i, rows - 1u), j = dl_divide(row, a.groups);
                staged_lse = a.lse[(uint64_t)(first + j) * a.q_heads + head * a.group + row - j * a.group];
            }
        };
        auto put = [&](uint32_t to) {
#pragma unroll
            for (uint32_t x = 0; x < LOADS; ++x) {
                const uint32_t n = threadIdx.x + x * MANY_THREADS, row = n / PIECES, piece = n % PIECES;
                if (32u * PIECES % MANY_THREADS == 0 || n < 32u * PIECES) *(dl_u32x4 *)&tiles[to][row * ROW + piece * 4u] = staged[x];
            }
            if (threadIdx.x < 32u) lses[to][i] = lse_of(staged_lse);
        };
        dl_u32x4 kf[2 * PAIRS];
        stage(head0, row0);
        put(0);
        __syncthreads();
        uint32_t now = 0;
#pragma unroll 1
        for (uint32_t head = head0; head < heads_end; ++head) {
            dl_words<16> codes[PAIRS];
#pragma unroll
            for (uint32_t x = 0; x < PAIRS; ++x) codes[x] = dl_load_words<16>(key.codes + head * a.c.head_stride + min(16u * (2u * x + half), D - 16u));
            const float scale = *(const float *)(key.scale + head * a.c.scale_head_stride);
#pragma unroll
            for (uint32_t x = 0; x < 2 * PAIRS; ++x) {
                const dl_u32x2 lo = C::template spread<Q>(codes[x / 2].w[2 * (x % 2)]), hi = C::template spread<Q>(codes[x / 2].w[2 * (x % 2) + 1]);
                kf[x] = dl_u32x4{lo[0], lo[1], hi[0], hi[1]};
                if (16u * (2u * (x / 2) + half) >= D) kf[x] = dl_u32x4{0, 0, 0, 0};
            }
            if (half == 0) scales[wave][i] = key.alive ? scale * a.scale : 0.0f;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll 1
            for (uint32_t r0 = row0; r0 < rows; r0 += 32u, now ^= 1u) {
                const bool same_head = r0 + 32u < rows, more = same_head || head + 1u < heads_end;
                if (more) stage(same_head ? head : head + 1u, same_head ? r0 + 32u : row0);
                if (r0 + 32u > from) {
                    dl_f32x16 s;
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = 0.0f;
                    auto operand = [&](uint32_t x) { return *(const dl_u32x4 *)&tiles[now][i * ROW + (2u * (2u * (x / 2) + half) + x % 2u) * 4u]; };
                    dl_u32x4 ring[3];
#pragma unroll
                    for (uint32_t x = 0; x < 2; ++x) ring[x] = operand(x);
                    const float lse = lses[now][i];
                    dl_f32x4 ks[4];
#pragma unroll
                    for (uint32_t x = 0; x < 2 * PAIRS; ++x) {
                        if (x + 2 < 2 * PAIRS) ring[(x + 2) % 3] = operand(x + 2);
                        if (x + 4 >= 2 * PAIRS) ks[x + 4 - 2 * PAIRS] = *(const dl_f32x4 *)&scales[wave][8u * (x + 4 - 2 * PAIRS) + 4u * half];
                        s = Q::mfma32(kf[x], ring[x % 3], s);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    const bool masked = r0 < whole;
                    const int32_t seen = masked ? ahead + (int32_t)dl_divide(r0 + i, a.groups) - (int32_t)base : 0;
                    add_weights(s, ks, lse, r0 + i < rows, masked, seen, half, sum);
                }
                if (more) put(now ^ 1u);
                __syncthreads();
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    const float its = over_lanes(sum, i);
    const uint32_t in = 8u * (i / 4u) + 4u * half + i % 4u, key = base + in;
    if (i >= 16u || key >= a.width) return;
    const float all = dead >> in & 1u ? 0.0f : its;
    if (a.parts > 1u)
        a.partial[((uint64_t)part * a.p.batch + b) * a.width + key] = all;
    else
        a.weights[b * a.weights_stride + key] = (a.before ? a.before[b * a.before_stride + key] : 0.0f) + all;
}

// Adds the parts, in their order.
constexpr uint32_t ADD_THREADS = 256;
__global__ void __launch_bounds__(ADD_THREADS) dl_weigh_add_kernel(const weigh_args a)
{
    const uint32_t key = blockIdx.x * ADD_THREADS + threadIdx.x, b = blockIdx.y;
    if (key >= a.width) return;
    float all = 0.0f;
    if (key < a.p.len(b))
        for (uint32_t part = 0; part < a.parts; ++part) all += a.partial[((uint64_t)part * a.p.batch + b) * a.width + key];
    a.weights[b * a.weights_stride + key] = (a.before ? a.before[b * a.before_stride + key] : 0.0f) + all;
}

struct weigh_shape {
    bool many;
    uint32_t blocks, parts;
};

int weigh_sizes(const dl_kv_cache *cache, const dl_kv_weigh_args *args, dl_cache_view *view, weigh_shape *sh)
{
    const int rc = dl_packed_sizes(cache, args, view);
    if (rc != DL_OK) return rc;
    const int64_t width = args->max_pages * cache->page_tokens;
    if (width * args->batch > INT32_MAX) return DL_ERR_INVALID;
    *sh = weigh_shape{};
    if (!args->batch || !width) return DL_OK;
    // By the rows that a head of a sequence has on average: one tile of 32, or more.  few : many, us, 8 heads, 32 query heads: one sequence of 4000 tokens with
    // 2, 8, 16, 24, 32 queries (8 to 128 rows) 5.7 : 9.6, 6.8 : 9.3, 8.6 : 9.9, 10.1 : 11.0, 11.9 : 11.7; four of up to 16 400 22.2 : 22.0, 24.4 : 22.1, 28.8 : 22.5,
    // 33.8 : 24.5, 40.0 : 26.6.
    sh->many = (uint64_t)args->tokens * (uint32_t)(args->q_heads / cache->heads) > 32u * (uint64_t)args->batch;
    sh->parts = 1;
    if (sh->many) {
        sh->blocks = (uint32_t)((width + MANY_KEYS - 1) / MANY_KEYS);
        const uint64_t all = (uint64_t)sh->blocks * (uint32_t)args->batch;
        sh->parts = all >= MANY_BLOCKS ? 1u : (uint32_t)((MANY_BLOCKS + all - 1u) / all);
        if (sh->parts > (uint32_t)cache->heads) sh->parts = (uint32_t)cache->heads;
        sh->blocks *= sh->parts;
    }
    return DL_OK;
}

size_t weigh_bytes(const dl_kv_cache *cache, const dl_kv_weigh_args *args, const weigh_shape &sh)
{
    return DL_CONTROL_BYTES + (sh.parts > 1u ? (size_t)sh.parts * (uint32_t)args->batch * (uint64_t)(args->max_pages * cache->page_tokens) * sizeof(float) : 0u);
}

}  // namespace

extern "C" int64_t dl_kv_weigh_workspace(const dl_kv_cache *cache, const dl_kv_weigh_args *args)
{
    dl_cache_view view;
    weigh_shape sh;
    const int rc = weigh_sizes(cache, args, &view, &sh);
    return rc != DL_OK ? rc : (int64_t)weigh_bytes(cache, args, sh);
}

extern "C" int dl_kv_weigh(const dl_kv_cache *cache, const dl_kv_weigh_args *args, void *stream)
{
    DL_LOCKED;
    if (!g_dl.inited) return DL_ERR_STATE;
    if (dl_device_error_pending()) return DL_ERR_LOST;
    weigh_args a;
    weigh_shape sh;
    int rc = weigh_sizes(cache, args, &a.c, &sh);
    if (rc != DL_OK) return rc;
    if (!args->batch || !args->max_pages) return DL_OK;
    rc = dl_cache_check(cache, 1, &a.c);
    if (rc != DL_OK) return rc;
    rc = dl_packed_setup(cache, args, weigh_bytes(cache, args, sh), &a.p);
    if (rc != DL_OK) return rc;
    if (!args->weights || (args->tokens && args->q_heads && (!args->q || !args->lse)) || ((uint64_t)args->weights | (uint64_t)args->before) % 4u)
        return DL_ERR_INVALID;
    a.q = (const char *)args->q;
    a.lse = args->lse;
    a.before = args->before;
    a.weights = args->weights;
    a.q_token = 2 * args->q_token_stride;
    a.q_head = 2 * args->q_head_stride;
    a.before_stride = args->before_stride;
    a.weights_stride = args->weights_stride;
    a.width = (uint32_t)(args->max_pages * cache->page_tokens);
    a.q_heads = (uint32_t)args->q_heads;
    a.group = a.q_heads / a.c.heads;
    a.groups = dl_make_divider(a.group ? a.group : 1u);
    a.scale = args->scale * DL_LOG2E;
    a.parts = sh.parts;
    a.partial = (float *)((char *)args->workspace + DL_CONTROL_BYTES);
    a.sharing = 1;
    while (a.sharing < FEW_WAVES && 2u * a.sharing <= a.c.heads) a.sharing *= 2u;
    const uint32_t few_keys = 32u * (FEW_WAVES / a.sharing), blocks = sh.many ? sh.blocks : (a.width + few_keys - 1u) / few_keys;
    // (blocks may be more than a grid of so many threads is wide)
    const uint32_t high = (blocks + 65535u) / 65536u;
    const dim3 grid((blocks + high - 1u) / high, a.p.batch, high);
    dl_with_16bit(args->type, [&](auto q) {
        dl_with_format(cache->format, [&](auto c) {
            auto go = [&](auto dp) {
                constexpr int DP = decltype(dp)::value;
                if (sh.many)
                    hipLaunchKernelGGL((dl_weigh_many_kernel<decltype(q), decltype(c), DP>), grid, dim3(MANY_THREADS), 0, (hipStream_t)stream, a);
                else
                    dl_with_bool(a.c.head_dim == DP, [&](auto whole) {
                        hipLaunchKernelGGL((dl_weigh_few_kernel<decltype(q), decltype(c), DP, decltype(whole)::value>), grid, dim3(64 * FEW_WAVES), 0,
                                           (hipStream_t)stream, a);
                    });
            };
            if (a.c.head_dim <= 64)
                go(std::integral_constant<int, 64>{});
            else if (a.c.head_dim <= 128)
                go(std::integral_constant<int, 128>{});
            else
                go(std::integral_constant<int, 256>{});
        });
    });
    if (a.parts > 1u)
        hipLaunchKernelGGL(dl_weigh_add_kernel, dim3((a.width + ADD_THREADS - 1u) / ADD_THREADS, a.p.batch), dim3(ADD_THREADS), 0, (hipStream_t)stream, a);
    DL_HIP(hipGetLastError());
    t_dl_last.mode = DL_MODE_ONESHOT;
    return DL_OK;
}
