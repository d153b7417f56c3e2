// Eviction from a paged cache by weight (dl_kv_evict): which tokens stay, and their move to other pages.
//
// Which stay: a workgroup a sequence looks for the weight T that the last of the tokens to stay has, as a whole number in which order of
// numbers is order of weights: digit by digit from the top, each time by a count of the digits of those that share what is known of T.
// Then one walk over the tokens in their order places those above T and the first of those equal to it.  Counts are whole numbers, so the
// order of the counting does not matter.
// The move: rows of codes in 16-byte pieces, a scale by the row's first lane; memory is what bounds it.
#include "dl_codes.h"
#include "dl_internal.h"

namespace {

constexpr uint32_t PICK_THREADS = 1024, PICK_WAVES = PICK_THREADS / 64;
constexpr uint32_t DIGIT_BITS = 8, DIGITS = 1u << DIGIT_BITS;
constexpr uint32_t MOVE_THREADS = 256;

struct evict_args {
    dl_cache_view c;
    const float *weights;
    const int32_t *pages, *lens, *to_pages;
    int32_t *kept, *kept_lens;
    float *kept_weights;
    int64_t pages_stride, to_pages_stride, weights_stride, kept_weights_stride;
    uint32_t most, batch, keep, first, recent;  // most: max_pages * page_tokens
    uint32_t rows;                              // of the move: batch * keep * heads
    dl_divider heads;
    uint32_t lanes;  // a row of the move takes, a power of two
};

// Whole numbers in the order of weights: 0 for NaN, both zeros alike.
__device__ __forceinline__ uint32_t order_of(float w)
{
    const uint32_t u = dl_bits<uint32_t>(w + 0.0f);  // (-0 + 0 = 0)
    return w != w ? 0u : u >> 31 ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(PICK_THREADS) dl_evict_pick_kernel(const evict_args a)
{
    __shared__ uint32_t count[PICK_WAVES][DIGITS];
    __shared__ uint32_t above[PICK_WAVES], equal[PICK_WAVES];
    __shared__ uint32_t found[2];
    const uint32_t b = blockIdx.x, thread = threadIdx.x, lane = thread % 64u, wave = thread / 64u;
    const float *const weights = a.weights + b * a.weights_stride;
    int32_t *const kept = a.kept + (uint64_t)b * a.keep;
    float *const kept_weights = a.kept_weights ? a.kept_weights + b * a.kept_weights_stride : nullptr;
    const uint32_t n = a.most ? min((uint32_t)max(a.lens[b], 0), a.most) : 0u, m = min(n, a.keep);
    if (thread == 0) a.kept_lens[b] = (int32_t)m;
    for (uint32_t j = m + thread; j < a.keep; j += PICK_THREADS) {
        kept[j] = -1;
        if (kept_weights) kept_weights[j] = 0.0f;
    }
    if (n <= a.keep) {
        for (uint32_t j = thread; j < n; j += PICK_THREADS) {
            kept[j] = (int32_t)j;
            if (kept_weights) kept_weights[j] = weights[j];
        }
        return;
    }
    // The others: tokens first .. end - 1, of which `left` stay (fewer than there are, since n > keep).
    const uint32_t end = n - a.recent;
    uint32_t left = a.keep - a.first - a.recent, known = 0;
    if (left) {
        for (int shift = 32 - (int)DIGIT_BITS; shift >= 0; shift -= (int)DIGIT_BITS) {
            for (uint32_t x = lane; x < DIGITS; x += 64u) count[wave][x] = 0;
            __syncthreads();
            for (uint32_t i = a.first + thread; i < end; i += PICK_THREADS) {
                const uint32_t k = order_of(weights[i]);
                if (shift + (int)DIGIT_BITS == 32 || k >> (shift + (int)DIGIT_BITS) == known) atomicAdd(&count[wave][k >> shift & (DIGITS - 1u)], 1u);
            }
            __syncthreads();
            if (wave == 0) {
                // four digits a lane, the highest in lane 0; the digit at which the count from the top reaches what is left
                uint32_t own[4], sum = 0;
#pragma unroll
                for (uint32_t x = 0; x < 4u; ++x) {
                    own[x] = 0;
                    for (uint32_t v = 0; v < PICK_WAVES; ++v) own[x] += count[v][DIGITS - 1u - (4u * lane + x)];
                    sum += own[x];
                }
                uint32_t before = dl_sum_up_to(sum) - sum;
#pragma unroll
                for (uint32_t x = 0; x < 4u; ++x) {
                    if (before < left && before + own[x] >= left) found[0] = DIGITS - 1u - (4u * lane + x), found[1] = left - before;
                    before += own[x];
                }
            }
            __syncthreads();
            known = known << DIGIT_BITS | found[0];
            left = found[1];
        }
    }
    // `left`: how many of those equal to `known` stay, the lowest.  (None looked for: all are lighter than what stays.)
    const bool some = a.keep > a.first + a.recent;
    uint32_t placed = 0, ties = 0;
    for (uint32_t i0 = 0; i0 < n; i0 += PICK_THREADS) {
        const uint32_t i = i0 + thread;
        const bool there = i < n, fixed = there && (i < a.first || i >= end);
        const float w = there ? weights[i] : 0.0f;
        const uint32_t k = order_of(w);
        const bool over = fixed || (some && there && k > known), same = some && there && !fixed && k == known;
        const unsigned long long all_over = __ballot(over), all_same = __ballot(same), below = (1ull << lane) - 1u;
        if (lane == 0) above[wave] = (uint32_t)__popcll(all_over), equal[wave] = (uint32_t)__popcll(all_same);
        __syncthreads();
        uint32_t at_over = placed, at_same = ties;
        for (uint32_t v = 0; v < PICK_WAVES; ++v) {
            if (v < wave) at_over += above[v], at_same += equal[v];
            placed += above[v], ties += equal[v];
        }
        at_over += (uint32_t)__popcll(all_over & below);
        at_same += (uint32_t)__popcll(all_same & below);
        // (of those before it, the ones above and as many of the equal ones as stay)
        if (over || (same && at_same < left)) {
            const uint32_t j = at_over + min(at_same, left);
            kept[j] = (int32_t)i;
            if (kept_weights) kept_weights[j] = w;
        }
        __syncthreads();
    }
}

// blockIdx.y: 0 keys, 1 values.
template <int ROWS>
__global__ void __launch_bounds__(MOVE_THREADS) dl_evict_move_kernel(const evict_args a)
{
    const uint32_t lane = threadIdx.x & (a.lanes - 1u), per = MOVE_THREADS / a.lanes;
    const uint32_t row0 = blockIdx.x * (per * ROWS) + threadIdx.x / a.lanes;
    const bool mine = 16u * lane < a.c.head_dim;
    char *const codes = blockIdx.y ? a.c.v : a.c.k;
    char *const scales = (char *)(blockIdx.y ? a.c.v_scale : a.c.k_scale);
    uint32_t token[ROWS], head[ROWS], seq[ROWS], j[ROWS];
    int32_t source[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint32_t row = min(row0 + r * per, a.rows - 1u);
        token[r] = dl_divide(row, a.heads);
        head[r] = row - token[r] * a.heads.d;
        seq[r] = token[r] / a.keep;
        j[r] = token[r] - seq[r] * a.keep;
        source[r] = row0 + r * per < a.rows ? a.kept[token[r]] : -1;
    }
    uint32_t page[ROWS], to_page[ROWS], in[ROWS], to_in[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        page[r] = to_page[r] = ~0u;
        in[r] = to_in[r] = 0;
        if (source[r] >= 0) {
            const uint32_t p = dl_divide((uint32_t)source[r], a.c.page), t = dl_divide(j[r], a.c.page);
            page[r] = (uint32_t)a.pages[seq[r] * a.pages_stride + p];
            to_page[r] = (uint32_t)a.to_pages[seq[r] * a.to_pages_stride + t];
            in[r] = (uint32_t)source[r] - p * a.c.page.d;
            to_in[r] = j[r] - t * a.c.page.d;
        }
    }
    dl_u32x4 w[ROWS];
    float scale[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        w[r] = dl_u32x4{0, 0, 0, 0};
        scale[r] = 0.0f;
        if (page[r] < a.c.pages && to_page[r] < a.c.pages) {
            if (mine) w[r] = dl_load_at<dl_u32x4>(codes + (uint64_t)page[r] * a.c.page_stride + (uint64_t)in[r] * a.c.token_stride + head[r] * a.c.head_stride + 16u * lane);
            if (lane == 0)
                scale[r] = *(const float *)(scales + (uint64_t)page[r] * a.c.scale_page_stride + (uint64_t)in[r] * a.c.scale_token_stride + head[r] * a.c.scale_head_stride);
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        if (page[r] < a.c.pages && to_page[r] < a.c.pages) {
            if (mine) dl_store_at(codes + (uint64_t)to_page[r] * a.c.page_stride + (uint64_t)to_in[r] * a.c.token_stride + head[r] * a.c.head_stride + 16u * lane, w[r]);
            if (lane == 0)
                *(float *)(scales + (uint64_t)to_page[r] * a.c.scale_page_stride + (uint64_t)to_in[r] * a.c.scale_token_stride + head[r] * a.c.scale_head_stride) = scale[r];
        }
}

int evict_setup(const dl_kv_cache *cache, const dl_kv_evict_args *args, int sides, dl_cache_view *view)
{
    if (!cache || !args) return DL_ERR_INVALID;
    const int rc = dl_cache_check(cache, sides, view);
    if (rc != DL_OK) return rc;
    if (args->batch < 0 || args->batch > 65535 || args->keep < 0 || args->first < 0 || args->recent < 0 || (int64_t)args->first + args->recent > args->keep)
        return DL_ERR_INVALID;
    if (args->max_pages < 0 || args->max_pages > 1 << 30 || args->max_pages * cache->page_tokens > 1 << 30) return DL_ERR_INVALID;
    if ((__int128)args->batch * args->keep * cache->heads > DL_MAX_ROWS) return DL_ERR_INVALID;
    return DL_OK;
}

}  // namespace

extern "C" int64_t dl_kv_evict_workspace(const dl_kv_cache *cache, const dl_kv_evict_args *args)
{
    dl_cache_view view;
    const int rc = evict_setup(cache, args, 0, &view);
    return rc != DL_OK ? rc : (int64_t)DL_CONTROL_BYTES;
}

extern "C" int dl_kv_evict(const dl_kv_cache *cache, const dl_kv_evict_args *args, void *stream)
{
    DL_LOCKED;
    if (!g_dl.inited) return DL_ERR_STATE;
    if (dl_device_error_pending()) return DL_ERR_LOST;
    evict_args a;
    const int rc = evict_setup(cache, args, 3, &a.c);
    if (rc != DL_OK) return rc;
    if (!args->batch) return DL_OK;
    if (!args->lens || !args->kept_lens || (args->keep && (!args->kept || !args->to_pages)) || (args->max_pages && (!args->weights || !args->pages)))
        return DL_ERR_INVALID;
    if (((uint64_t)args->weights | (uint64_t)args->pages | (uint64_t)args->lens | (uint64_t)args->to_pages | (uint64_t)args->kept |
         (uint64_t)args->kept_lens | (uint64_t)args->kept_weights) % 4u)
        return DL_ERR_INVALID;
    if (!args->workspace || (uint64_t)args->workspace % 16u || args->workspace_bytes < DL_CONTROL_BYTES) return DL_ERR_INVALID;
    a.weights = args->weights;
    a.pages = args->pages;
    a.lens = args->lens;
    a.to_pages = args->to_pages;
    a.kept = args->kept;
    a.kept_lens = args->kept_lens;
    a.kept_weights = args->kept_weights;
    a.pages_stride = args->pages_stride;
    a.to_pages_stride = args->to_pages_stride;
    a.weights_stride = args->weights_stride;
    a.kept_weights_stride = args->kept_weights_stride;
    a.most = (uint32_t)(args->max_pages * cache->page_tokens);
    a.batch = (uint32_t)args->batch;
    a.keep = (uint32_t)args->keep;
    a.first = (uint32_t)args->first;
    a.recent = (uint32_t)args->recent;
    a.rows = a.batch * a.keep * a.c.heads;
    a.heads = dl_make_divider(a.c.heads);
    a.lanes = a.c.head_dim <= 16 ? 1u : a.c.head_dim <= 32 ? 2u : a.c.head_dim <= 64 ? 4u : a.c.head_dim <= 128 ? 8u : 16u;
    hipLaunchKernelGGL(dl_evict_pick_kernel, dim3(a.batch), dim3(PICK_THREADS), 0, (hipStream_t)stream, a);
    if (a.rows) {
        constexpr int ROWS = 2;
        const uint32_t per = MOVE_THREADS / a.lanes * ROWS;
        hipLaunchKernelGGL((dl_evict_move_kernel<ROWS>), dim3((a.rows + per - 1u) / per, 2), dim3(MOVE_THREADS), 0, (hipStream_t)stream, a);
    }
    DL_HIP(hipGetLastError());
    t_dl_last.mode = DL_MODE_ONESHOT;
    return DL_OK;
}
