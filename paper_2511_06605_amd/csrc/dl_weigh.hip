// What cached tokens have been given by queries whose sums are known (dl_kv_weigh).
//
// With the scores s and lse in units of ln 2, a token is given the sum over queries and heads of 2^(s - lse).  The lse is known, so no
// maximum is looked for and the sum is over the queries alone: a wavefront has 32 keys in its lanes, as the right operand of 32 x 32 x 16
// products whose rows are queries, and adds up in registers over heads and queries.  The wavefronts of a workgroup share out the heads of
// their keys and add their sums in LDS at the end, in a fixed order.
#include "dl_codes.h"
#include "dl_internal.h"
#include "dl_packed.h"

namespace {

constexpr uint32_t WEIGH_WAVES = 8, WEIGH_THREADS = 64 * WEIGH_WAVES;

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
    uint32_t sharing;      // wavefronts that share the heads of their keys: 1, 2, 4 or 8
    float scale;           // times log2 e
};

template <class Q, class C, int DP>
__global__ void __launch_bounds__(WEIGH_THREADS, DP <= 128 ? 2 : 1) dl_weigh_kernel(const weigh_args a)
{
    constexpr uint32_t PAIRS = DP >= 32 ? DP / 32 : 1;  // of pieces of 16 dims, one for each half of the wavefront
    __shared__ float sums[WEIGH_WAVES][32];
    const uint32_t lane = threadIdx.x % 64u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
    const uint32_t i = lane % 32u, half = lane / 32u, D = a.c.head_dim, b = blockIdx.y;
    const uint32_t share = wave % a.sharing, block_keys = 32u * (WEIGH_WAVES / a.sharing);
    const uint32_t first = a.p.start(b), queries = a.p.queries(b, first), rows = queries * a.group, len = a.p.len(b);
    const int32_t *const table = a.p.pages + b * a.p.pages_stride;
    for (uint32_t block0 = blockIdx.x * block_keys; block0 < a.width; block0 += gridDim.x * block_keys) {
        const uint32_t base = block0 + wave / a.sharing * 32u, key = base + i;
        float sum = 0.0f;
        if (base < len && rows) {
            // the first row that sees the lane's key: that of query key - (len - queries)
            const int64_t since = ((int64_t)key - (int64_t)len + (int64_t)queries) * a.group;
            uint32_t page = ~0u, in = 0;
            if (key < len) {
                const uint32_t n = dl_divide(key, a.c.page);
                page = (uint32_t)table[n];
                in = key - n * a.c.page.d;
            }
            const bool alive = page < a.c.pages;
            const uint32_t from_row = alive ? (uint32_t)max(since, (int64_t)0) : ~0u;
            page = alive ? page : 0u;
            const char *const codes = a.c.k + (uint64_t)page * a.c.page_stride + (uint64_t)in * a.c.token_stride;
            const char *const scales = (const char *)a.c.k_scale + (uint64_t)page * a.c.scale_page_stride + (uint64_t)in * a.c.scale_token_stride;
            const int64_t wave_since = ((int64_t)base - (int64_t)len + (int64_t)queries) * a.group;
            const uint32_t row0 = (uint32_t)max(wave_since, (int64_t)0) & ~31u;
            for (uint32_t head = share; head < a.c.heads; head += a.sharing) {
                dl_words<16> k[PAIRS];
#pragma unroll
                for (uint32_t x = 0; x < PAIRS; ++x) k[x] = dl_load_words<16>(codes + head * a.c.head_stride + min(16u * (2u * x + half), D - 16u));
                float scale = *(const float *)(scales + head * a.c.scale_head_stride);
                scale = alive ? scale * a.scale : 0.0f;
                for (uint32_t r0 = row0; r0 < rows; r0 += 32u) {
                    const uint32_t row = min(r0 + i, rows - 1u), j = row / a.group, h = head * a.group + row - j * a.group;
                    const char *const q = a.q + (uint64_t)(first + j) * a.q_token + h * a.q_head;
                    const float given = a.lse[(uint64_t)(first + j) * a.q_heads + h] * DL_LOG2E;
                    // (a row that is none, or whose lse is no number: nothing is left of it)
                    const float lse = r0 + i < rows && fabsf(given) < INFINITY ? given : INFINITY;
                    dl_f32x16 s;
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = 0.0f;
#pragma unroll
                    for (uint32_t x = 0; x < PAIRS; ++x)
#pragma unroll
                        for (uint32_t u = 0; u < 2; ++u) {
                            const uint32_t d = 16u * (2u * x + half) + 8u * u;
                            const dl_u32x4 qf = d < D ? dl_load_at<dl_u32x4>(q + 2u * d) : dl_u32x4{0, 0, 0, 0};
                            const dl_u32x2 lo = C::template spread<Q>(k[x].w[2 * u]), hi = C::template spread<Q>(k[x].w[2 * u + 1]);
                            s = Q::mfma32(qf, dl_u32x4{lo[0], lo[1], hi[0], hi[1]}, s);
                        }
                    // rows of the product are queries (8 (e / 4) + 4 half + e % 4), its columns keys (i)
                    float four[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const uint32_t in_tile = 8u * (e / 4) + 4u * half + e % 4;
                        const float its = __shfl(lse, (int)in_tile);
                        const float w = __builtin_amdgcn_exp2f(fmaf(s[e], scale, -its));
                        four[e % 4] += r0 + in_tile >= from_row ? w : 0.0f;
                    }
                    sum += (four[0] + four[1]) + (four[2] + four[3]);
                }
            }
            sum += __shfl_xor(sum, 32);
        }
        if (half == 0) sums[wave][i] = sum;
        __syncthreads();
        if (share == 0 && half == 0 && key < a.width) {
            float all = sum;
            for (uint32_t w = 1; w < a.sharing; ++w) all += sums[wave + w][i];
            a.weights[b * a.weights_stride + key] = (a.before ? a.before[b * a.before_stride + key] : 0.0f) + all;
        }
        __syncthreads();
    }
}

int weigh_sizes(const dl_kv_cache *cache, const dl_kv_weigh_args *args, dl_cache_view *view)
{
    const int rc = dl_packed_sizes(cache, args, view);
    if (rc != DL_OK) return rc;
    return args->max_pages * cache->page_tokens * args->batch > INT32_MAX ? DL_ERR_INVALID : DL_OK;
}

}  // namespace

extern "C" int64_t dl_kv_weigh_workspace(const dl_kv_cache *cache, const dl_kv_weigh_args *args)
{
    dl_cache_view view;
    const int rc = weigh_sizes(cache, args, &view);
    return rc != DL_OK ? rc : (int64_t)DL_CONTROL_BYTES;
}

extern "C" int dl_kv_weigh(const dl_kv_cache *cache, const dl_kv_weigh_args *args, void *stream)
{
    DL_LOCKED;
    if (!g_dl.inited) return DL_ERR_STATE;
    if (dl_device_error_pending()) return DL_ERR_LOST;
    weigh_args a;
    int rc = weigh_sizes(cache, args, &a.c);
    if (rc != DL_OK) return rc;
    if (!args->batch || !args->max_pages) return DL_OK;
    rc = dl_cache_check(cache, 1, &a.c);
    if (rc != DL_OK) return rc;
    rc = dl_packed_setup(cache, args, DL_CONTROL_BYTES, &a.p);
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
    a.sharing = a.c.heads >= 8u ? 8u : a.c.heads >= 4u ? 4u : a.c.heads >= 2u ? 2u : 1u;
    a.scale = args->scale * DL_LOG2E;
    const uint32_t block_keys = 32u * (WEIGH_WAVES / a.sharing), blocks = (a.width + block_keys - 1u) / block_keys;
    const dim3 grid(blocks < 65536u ? blocks : 65536u, a.p.batch);
    dl_with_16bit(args->type, [&](auto q) {
        dl_with_format(cache->format, [&](auto c) {
            auto go = [&](auto dp) {
                hipLaunchKernelGGL((dl_weigh_kernel<decltype(q), decltype(c), decltype(dp)::value>), grid, dim3(WEIGH_THREADS), 0, (hipStream_t)stream, a);
            };
            if (a.c.head_dim <= 64)
                go(std::integral_constant<int, 64>{});
            else if (a.c.head_dim <= 128)
                go(std::integral_constant<int, 128>{});
            else
                go(std::integral_constant<int, 256>{});
        });
    });
    DL_HIP(hipGetLastError());
    t_dl_last.mode = DL_MODE_ONESHOT;
    return DL_OK;
}
