// Eviction from a paged cache by weight (dl_kv_evict): which tokens stay, and their move to other pages.
//
// Which stay: a workgroup a sequence looks for the weight T that the last of the tokens to stay has, as a whole number in which order of
// numbers is order of weights: digit by digit from the top, each time by a count of the digits of those that share what is known of T.
// Then one walk over the tokens in their order places those above T and the first of those equal to it.  Counts are whole numbers, so the
// order of the counting does not matter.
// The move: rows of codes in 16-byte pieces, a scale by the row's first lane; memory is what bounds it.
//
// Measured: 4 sequences of up to 32 768 tokens cut to 8192 (8 heads of 128, 139 MB) 48 - 49 us, 17 to 23 of them the choice by 4 workgroups, 24 to 35 the
// move, 4.7 TB/s on average; 3 of up to 2001 cut to 500 10.6 us, two launches.  Of a choice among 25 000 (13.4 us) the first look with its count takes 5,
// each of two more digits 2.2, counting and placing 3.4.
// Above 32 768 tokens the numbers do not fit LDS, and that one workgroup reads the weights once a digit and twice more: 4 of up to 32 769 cut to 8192 61 us, of
// 131 072 124 (to 32 768, 557 MB: 217).
#include "dl_codes.h"
#include "dl_internal.h"

namespace {

constexpr uint32_t PICK_THREADS = 1024, PICK_WAVES = PICK_THREADS / 64;
constexpr uint32_t DIGIT_BITS = 8, DIGITS = 1u << DIGIT_BITS;
// Counts of a digit that lanes take in turn: weights share their upper bits, and counts at one address wait for each other.
constexpr uint32_t COPIES = 16;
constexpr uint32_t MOVE_THREADS = 256;
// From so many bytes of codes on, stores go past the caches; less stays there, for the attention that follows.  Two rows a thread.  Measured, the
// whole call, one row and plain : two and plain : two and streaming stores : two, loads as well : four and streaming, buffers in turn that no cache
// holds: 139 MB read and written 57.4 : 53.5 : 48.5 : 49.7 : 50.9 us, 132 MB in 8 sequences 51.0 : 47.3 : 42.2 : 43.6 : 44.5; 4 MB 13.3 - 14.8 all.
constexpr uint64_t MOVE_STREAM_BYTES = 32ull << 20;

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

// Whole numbers in the order of weights, both zeros alike: 1 for NaN, above it 2^23 - 1 (-infinity) to 0xFF800000.  0 is what is no token, and the
// largest number what stays in any case: so the tokens that stay are the `keep` with the largest numbers.
constexpr uint32_t FIXED = ~0u;
__device__ __forceinline__ uint32_t order_of(float w)
{
    const uint32_t u = dl_bits<uint32_t>(w + 0.0f);  // (-0 + 0 = 0)
    return w != w ? 1u : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// Numbers of so many tokens fit LDS.
constexpr uint32_t PICK_HELD = 32768;

struct pick_lds {
    __align__(16) uint32_t held[PICK_HELD];
    uint32_t count[DIGITS * COPIES];
    uint32_t totals[PICK_WAVES], above[PICK_WAVES], equal[PICK_WAVES];
    uint32_t digit, left, here;
};

// Which tokens of a sequence of n > keep stay.  A wavefront has `share` tokens in a row (a multiple of 256).  HELD: from the first look on their
// numbers come from LDS, else they are made from memory each time.
template <bool HELD>
__device__ __forceinline__ void pick(const evict_args &a, const float *weights, int32_t *kept, uint32_t n, pick_lds &lds)
{
    const uint32_t thread = threadIdx.x, lane = thread % 64u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(thread / 64u));
    const uint32_t share = (n + 4u * PICK_THREADS - 1u) / (4u * PICK_THREADS) * 256u, from = wave * share, to = from + share;
    const uint32_t end = n - a.recent;
    auto number = [&](uint32_t i, float w) { return i >= n ? 0u : i < a.first || i >= end ? FIXED : order_of(w); };
    // f(token of the first lane, four numbers a lane, one behind the other): 256 tokens at a time; tokens from n on are none
    auto from_memory = [&](auto f) {
        constexpr uint32_t AHEAD = 8;  // loads on their way at once
        for (uint32_t i0 = from; i0 < to; i0 += 256u * AHEAD) {
            dl_f32x4 w[AHEAD];
#pragma unroll
            for (uint32_t x = 0; x < AHEAD; ++x) {
                const uint32_t i = i0 + 256u * x + 4u * lane;
                if (i + 4u <= n) {
                    w[x] = dl_load_at<dl_f32x4>(weights + i);
                } else {
#pragma unroll
                    for (uint32_t c = 0; c < 4u; ++c) w[x][c] = weights[min(i + c, n - 1u)];
                }
            }
#pragma unroll
            for (uint32_t x = 0; x < AHEAD; ++x) {
                const uint32_t i = i0 + 256u * x + 4u * lane;
                if (i0 + 256u * x < to) f(i0 + 256u * x, dl_u32x4{number(i, w[x][0]), number(i + 1u, w[x][1]), number(i + 2u, w[x][2]), number(i + 3u, w[x][3])});
            }
        }
    };
    auto each = [&](auto f) {
        if constexpr (HELD) {
            constexpr uint32_t AHEAD = 2;
            for (uint32_t i0 = from; i0 < to; i0 += 256u * AHEAD) {
                dl_u32x4 k[AHEAD];
#pragma unroll
                for (uint32_t x = 0; x < AHEAD; ++x) k[x] = *(const dl_u32x4 *)&lds.held[min(i0 + 256u * x, to - 256u) + 4u * lane];
#pragma unroll
                for (uint32_t x = 0; x < AHEAD; ++x)
                    if (i0 + 256u * x < to) f(i0 + 256u * x, k[x]);
            }
        } else {
            from_memory(f);
        }
    };
    // The number of the last that stays, and how many of those equal to it do (fewer stay than there are, since n > keep).
    uint32_t left = a.keep, known = 0, mask = 0;
    for (int shift = 32 - (int)DIGIT_BITS; left && shift >= 0; shift -= (int)DIGIT_BITS) {
        for (uint32_t x = thread; x < DIGITS * COPIES; x += PICK_THREADS) lds.count[x] = 0;
        __syncthreads();
        auto count = [&](dl_u32x4 k) {
#pragma unroll
            for (uint32_t c = 0; c < 4u; ++c)
                if ((k[c] & mask) == known) atomicAdd(&lds.count[(k[c] >> shift & (DIGITS - 1u)) * COPIES + lane % COPIES], 1u);
        };
        if (HELD && !mask)
            from_memory([&](uint32_t i0, dl_u32x4 k) {
                *(dl_u32x4 *)&lds.held[i0 + 4u * lane] = k;
                count(k);
            });
        else
            each([&](uint32_t, dl_u32x4 k) { count(k); });
        __syncthreads();
        // a digit a thread, from the top; the one at which the count reaches what is left
        uint32_t own = 0;
        if (thread < DIGITS) {
#pragma unroll
            for (uint32_t c = 0; c < COPIES; ++c) own += lds.count[(DIGITS - 1u - thread) * COPIES + (c + thread) % COPIES];
        }
        const uint32_t up_to = dl_sum_up_to(own);
        if (lane == 63u) lds.totals[wave] = up_to;
        __syncthreads();
        uint32_t before = up_to - own;
        for (uint32_t v = 0; v < wave && v < DIGITS / 64u; ++v) before += lds.totals[v];
        if (before < left && before + own >= left) lds.digit = DIGITS - 1u - thread, lds.left = left - before, lds.here = own;
        __syncthreads();
        known |= lds.digit << shift;
        mask |= (DIGITS - 1u) << shift;
        left = lds.left;
        if (lds.here == left) {  // all that share what is known stay: those above the lowest that there could be, and all equal to it
            left = n;
            break;
        }
    }
    if (!left) known = FIXED;  // (none stays)
    uint32_t over_here = 0, same_here = 0;
    auto walk = [&](auto f) {
        if (HELD && !a.keep) return;  // (nothing is held)
        each(f);
    };
    walk([&](uint32_t, dl_u32x4 k) {
#pragma unroll
        for (uint32_t c = 0; c < 4u; ++c) {
            over_here += (uint32_t)__popcll(__ballot(k[c] > known));
            same_here += (uint32_t)__popcll(__ballot(k[c] == known));
        }
    });
    if (lane == 0) lds.above[wave] = over_here, lds.equal[wave] = same_here;
    __syncthreads();
    uint32_t placed = 0, ties = 0;
    for (uint32_t v = 0; v < wave; ++v) placed += lds.above[v], ties += lds.equal[v];
    walk([&](uint32_t i0, dl_u32x4 k) {
        // of the lanes before this one
        uint32_t at_over = placed, at_same = ties;
#pragma unroll
        for (uint32_t c = 0; c < 4u; ++c) {
            const unsigned long long over = __ballot(k[c] > known), same = __ballot(k[c] == known);
            at_over = __builtin_amdgcn_mbcnt_hi((uint32_t)(over >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)over, at_over));
            at_same = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, at_same));
            placed += (uint32_t)__popcll(over);
            ties += (uint32_t)__popcll(same);
        }
#pragma unroll
        for (uint32_t c = 0; c < 4u; ++c) {
            // (of those before it, the ones above and as many of the equal ones as stay)
            if (k[c] > known || (k[c] == known && at_same < left)) kept[at_over + min(at_same, left)] = (int32_t)(i0 + 4u * lane + c);
            at_over += k[c] > known;
            at_same += k[c] == known;
        }
    });
}

__global__ void __launch_bounds__(PICK_THREADS) dl_evict_pick_kernel(const evict_args a)
{
    __shared__ pick_lds lds;
    const uint32_t b = blockIdx.x, thread = threadIdx.x;
    const float *const weights = a.weights + b * a.weights_stride;
    int32_t *const kept = a.kept + (uint64_t)b * a.keep;
    const uint32_t n = a.most ? min((uint32_t)max(a.lens[b], 0), a.most) : 0u;
    if (thread == 0) a.kept_lens[b] = (int32_t)min(n, a.keep);
    if (n <= a.keep) {
        for (uint32_t j = thread; j < a.keep; j += PICK_THREADS) kept[j] = j < n ? (int32_t)j : -1;
    } else if (n <= PICK_HELD) {
        pick<true>(a, weights, kept, n, lds);
    } else {
        pick<false>(a, weights, kept, n, lds);
    }
}

// blockIdx.y: 0 keys, 1 values.  The first head's keys take a token's weight along.
template <int ROWS, bool STREAM>
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
        if (a.kept_weights && row0 + r * per < a.rows && head[r] == 0 && lane == 0 && blockIdx.y == 0)
            a.kept_weights[seq[r] * a.kept_weights_stride + j[r]] = source[r] >= 0 ? a.weights[seq[r] * a.weights_stride + source[r]] : 0.0f;
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
            if (mine) dl_put<STREAM>(codes + (uint64_t)to_page[r] * a.c.page_stride + (uint64_t)to_in[r] * a.c.token_stride + head[r] * a.c.head_stride + 16u * lane, w[r]);
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

bool overlap(const int32_t *a, int64_t a_many, const int32_t *b, int64_t b_many)
{
    return a_many && b_many && (uint64_t)a < (uint64_t)b + 4u * (uint64_t)b_many && (uint64_t)b < (uint64_t)a + 4u * (uint64_t)a_many;
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
    // (lengths and weights are read while what stays is written; lists without gaps are looked at as a whole)
    const int64_t lists = args->batch, tokens = lists * args->keep;
    if (overlap(args->lens, lists, args->kept_lens, lists) || overlap(args->lens, lists, args->kept, tokens) || overlap(args->kept_lens, lists, args->kept, tokens) ||
        (args->kept_weights && args->kept_weights == args->weights))
        return DL_ERR_INVALID;
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
        dl_with_bool(2ull * a.rows * a.c.head_dim >= MOVE_STREAM_BYTES, [&](auto streaming) {
            hipLaunchKernelGGL((dl_evict_move_kernel<ROWS, decltype(streaming)::value>), dim3((a.rows + per - 1u) / per, 2), dim3(MOVE_THREADS), 0, (hipStream_t)stream, a);
        });
    }
    DL_HIP(hipGetLastError());
    t_dl_last.mode = DL_MODE_ONESHOT;
    return DL_OK;
}
