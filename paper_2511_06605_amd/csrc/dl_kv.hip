// Quantising a cache as it is written, and reading it back (dl_kv_write, dl_kv_read).
//
// A row (the head_dim elements of one token and head) becomes codes x * ((1 / a) * LIMIT), a = max(max |x|, 2^-100), and a scale
// a * (1 / LIMIT).  The largest magnitude is needed before the first code, so a row is held in registers from its load to
// its store, as many lanes as that takes (the next power of two) side by side, and the maximum by
// swaps among them.  One pass over the data either way; memory is what bounds it.
//
// Measured, 8 heads of 128, keys and values in one launch: 20001 tokens written (float16 to int8, 124 MB moved) in 20 us, 6.2 TB/s; 16384 read
// (fp8 to bfloat16, 102 MB) in 16.0 us, 6.3 TB/s; a large copy moves 6.4 - 7.2 TB/s.  One token takes 4 us, which is an empty kernel's time.
#include "dl_codes.h"
#include "dl_internal.h"

namespace {

struct kv_args {
    dl_cache_view c;
    char *k, *v;  // rows outside the cache
    const int64_t *slots;
    int64_t k_token, k_head, v_token, v_head;  // strides in bytes
    int64_t slots_end;                         // pages * page_tokens
    uint32_t rows;                             // tokens * heads
    dl_divider heads;
    int32_t shift;  // log2 of the tokens of a page, or -1
};

// Where a row of a slot lies: false if the slot is none.
__device__ __forceinline__ bool place(const kv_args &a, int64_t slot, uint32_t head, int64_t *codes, int64_t *scale)
{
    if (slot < 0 || slot >= a.slots_end) return false;
    int64_t page, in;
    if (a.shift >= 0) {
        page = slot >> a.shift;
        in = slot & (a.c.page.d - 1u);
    } else {
        page = slot / a.c.page.d;
        in = slot - page * a.c.page.d;
    }
    *codes = (uint64_t)(uint32_t)page * a.c.page_stride + (uint64_t)(uint32_t)in * a.c.token_stride + head * a.c.head_stride;
    *scale = (uint64_t)(uint32_t)page * a.c.scale_page_stride + (uint64_t)(uint32_t)in * a.c.scale_token_stride + head * a.c.scale_head_stride;
    return true;
}

constexpr uint32_t KV_THREADS = 256;
// Elements a lane: its store is then 16 bytes, next to its neighbours' (16-bit rows; a store that lies 16 bytes from the next
// one leaves half-written lines, which cost the read of 16384 tokens of 8 x 128 more than half: 16.6 : 29.7 us).
constexpr int WRITE_ELEMENTS = 16, READ_ELEMENTS = 8;
// Requests of more than two rounds of workgroups: two rows of a lane on their way at once, and stores past the caches, which would
// not hold the result anyway.  Plain stores and one row : this, three sets of buffers in turn, write of 20001 tokens (8 x 128, float16 to
// int8) 25.6 : 21.7 us, read of 16384 (fp8 to bfloat16) 25.2 : 16.6; four rows 23.4 and 17.0.  Smaller requests stay in the caches, for
// the attention that follows.
constexpr uint64_t KV_MANY_THREADS = 1ull << 20;

// blockIdx.y: 0 keys, 1 values (a launch for one side alone has one of them).  LANES a row; MANY: two rows of a thread, both on their way before
// the first is looked at (a row's chain is its slot, then, where codes are read, the codes, then the store).
template <class T, class C, int LANES, bool MANY>
__global__ void __launch_bounds__(KV_THREADS) dl_kv_write_kernel(const kv_args a)
{
    constexpr int ROWS = MANY ? 2 : 1, N = WRITE_ELEMENTS;
    const bool values = blockIdx.y != 0 || !a.k;
    const uint32_t lane = threadIdx.x % LANES, row0 = blockIdx.x * (KV_THREADS / LANES * ROWS) + threadIdx.x / LANES;
    const bool mine = lane * (uint32_t)N < a.c.head_dim;
    float x[ROWS][N];
    int64_t slot[ROWS];
    uint32_t head[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint32_t row = min(row0 + r * (KV_THREADS / LANES), a.rows - 1u), token = dl_divide(row, a.heads);
        head[r] = row - token * a.heads.d;
        const char *const from = values ? a.v + token * a.v_token + head[r] * a.v_head : a.k + token * a.k_token + head[r] * a.k_head;
        slot[r] = a.slots[token];
#pragma unroll
        for (int i = 0; i < N; ++i) x[r][i] = 0.0f;
        if (mine) dl_load_row<T>(from + (size_t)lane * N * T::size, x[r]);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (row0 + r * (KV_THREADS / LANES) >= a.rows) return;  // all lanes of a row together
        // magnitudes as whole numbers: there infinities and NaN lie above all that is finite
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) top = max(top, dl_bits<uint32_t>(x[r][i]) & 0x7FFFFFFFu);
#pragma unroll
        for (int d = 1; d < LANES; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
        int64_t at, scale_at;
        if (!place(a, slot[r], head[r], &at, &scale_at)) continue;
        const bool finite = top < 0x7F800000u;
        const float most = fmaxf(dl_bits<float>(top), 0x1p-100f);
        const float factor = 1.0f / most * C::limit;
        dl_u32x4 w;
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            w[i] = C::code4(x[r][4 * i] * factor, x[r][4 * i + 1] * factor, x[r][4 * i + 2] * factor, x[r][4 * i + 3] * factor);
            if (!finite) w[i] = 0;
        }
        if (mine) dl_put<MANY>((values ? a.c.v : a.c.k) + at + lane * (uint32_t)N, w);
        if (lane == 0) *(float *)((char *)(values ? a.c.v_scale : a.c.k_scale) + scale_at) = finite ? most * (1.0f / C::limit) : __builtin_nanf("");
    }
}

template <class T, class C, int LANES, bool MANY>
__global__ void __launch_bounds__(KV_THREADS) dl_kv_read_kernel(const kv_args a)
{
    constexpr int ROWS = MANY ? 2 : 1, N = READ_ELEMENTS;
    const bool values = blockIdx.y != 0 || !a.k;
    const uint32_t lane = threadIdx.x % LANES, row0 = blockIdx.x * (KV_THREADS / LANES * ROWS) + threadIdx.x / LANES;
    if (lane * (uint32_t)N >= a.c.head_dim) return;
    dl_u32x2 w[ROWS];
    float scale[ROWS];
    uint32_t token[ROWS], head[ROWS];
    int64_t slot[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint32_t row = min(row0 + r * (KV_THREADS / LANES), a.rows - 1u);
        token[r] = dl_divide(row, a.heads);
        head[r] = row - token[r] * a.heads.d;
        slot[r] = a.slots[token[r]];
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        int64_t at, scale_at;
        w[r] = dl_u32x2{0, 0};
        scale[r] = 0.0f;
        if (place(a, slot[r], head[r], &at, &scale_at)) {
            w[r] = dl_load_at<dl_u32x2>((values ? a.c.v : a.c.k) + at + lane * (uint32_t)N);
            scale[r] = *(const float *)((const char *)(values ? a.c.v_scale : a.c.k_scale) + scale_at);
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (row0 + r * (KV_THREADS / LANES) >= a.rows) return;
        char *const to = values ? a.v + token[r] * a.v_token + head[r] * a.v_head : a.k + token[r] * a.k_token + head[r] * a.k_head;
        float x[N];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            float y[4];
            C::value4(w[r][i], y);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * i + j] = y[j] * scale[r];
        }
        dl_store_row<T, MANY>(to + (size_t)lane * N * T::size, x);
    }
}

int kv_setup(const dl_kv_cache *cache, const dl_kv_rows *rows, kv_args *a, bool *nothing)
{
    if (!cache || !rows) return DL_ERR_INVALID;
    const int rc = dl_cache_check(cache, (rows->k ? 1 : 0) | (rows->v ? 2 : 0), &a->c);
    if (rc != DL_OK) return rc;
    if (rows->type < DL_TYPE_F32 || rows->type > DL_TYPE_F16 || rows->reserved != 0) return DL_ERR_INVALID;
    if (rows->tokens < 0 || rows->tokens > DL_MAX_ROWS || rows->tokens * (int64_t)cache->heads > DL_MAX_ROWS) return DL_ERR_INVALID;
    *nothing = rows->tokens == 0 || (!rows->k && !rows->v);
    if (*nothing) return DL_OK;
    if (!rows->slots) return DL_ERR_INVALID;
    const int size = rows->type == DL_TYPE_F32 ? 4 : 2;
    if (((uint64_t)rows->k | (uint64_t)rows->v) % size || (uint64_t)rows->slots % 8u) return DL_ERR_INVALID;
    a->k = (char *)rows->k;
    a->v = (char *)rows->v;
    a->slots = rows->slots;
    a->k_token = rows->k_token_stride * size;
    a->k_head = rows->k_head_stride * size;
    a->v_token = rows->v_token_stride * size;
    a->v_head = rows->v_head_stride * size;
    a->slots_end = cache->pages * cache->page_tokens;
    a->rows = (uint32_t)(rows->tokens * cache->heads);
    a->heads = dl_make_divider((uint32_t)cache->heads);
    a->shift = -1;
    for (int i = 0; i < 17; ++i)
        if (cache->page_tokens == 1 << i) a->shift = i;
    return DL_OK;
}

template <bool WRITE>
int kv_run(const dl_kv_cache *cache, const dl_kv_rows *rows, void *stream)
{
    DL_LOCKED;
    if (!g_dl.inited) return DL_ERR_STATE;
    if (dl_device_error_pending()) return DL_ERR_LOST;
    kv_args a;
    bool nothing;
    const int rc = kv_setup(cache, rows, &a, &nothing);
    if (rc != DL_OK || nothing) return rc;
    dl_with_type(rows->type, [&](auto t) {
        dl_with_format(cache->format, [&](auto c) {
            dl_with_lanes<WRITE ? WRITE_ELEMENTS : READ_ELEMENTS>(a.c.head_dim, [&](auto lanes) {
                constexpr int L = decltype(lanes)::value;
                auto go = [&](auto many) {
                    constexpr bool MANY = decltype(many)::value;
                    const uint64_t threads = ((uint64_t)a.rows + MANY) / (MANY ? 2u : 1u) * L;
                    const dim3 grid((uint32_t)((threads + KV_THREADS - 1) / KV_THREADS), a.k && a.v ? 2 : 1);
                    if constexpr (WRITE)
                        hipLaunchKernelGGL((dl_kv_write_kernel<decltype(t), decltype(c), L, MANY>), grid, dim3(KV_THREADS), 0, (hipStream_t)stream, a);
                    else
                        hipLaunchKernelGGL((dl_kv_read_kernel<decltype(t), decltype(c), L, MANY>), grid, dim3(KV_THREADS), 0, (hipStream_t)stream, a);
                };
                if ((uint64_t)a.rows * L >= KV_MANY_THREADS)
                    go(std::true_type{});
                else
                    go(std::false_type{});
            });
        });
    });
    DL_HIP(hipGetLastError());
    t_dl_last.mode = DL_MODE_ONESHOT;
    return DL_OK;
}

}  // namespace

int dl_cache_check(const dl_kv_cache *c, int sides, dl_cache_view *w)
{
    if (c->format != DL_KV_FP8 && c->format != DL_KV_INT8) return DL_ERR_INVALID;
    if (c->heads < 1 || c->heads > 65535 || c->head_dim < 16 || c->head_dim > 256 || c->head_dim % 16) return DL_ERR_INVALID;
    if (c->page_tokens < 1 || c->page_tokens > 65536 || c->pages < 0 || c->pages > INT32_MAX) return DL_ERR_INVALID;
    if (c->pages && (((sides & 1) && (!c->k || !c->k_scale)) || ((sides & 2) && (!c->v || !c->v_scale)))) return DL_ERR_INVALID;
    if (((uint64_t)c->k_scale | (uint64_t)c->v_scale) % 4u) return DL_ERR_INVALID;
    w->k = (char *)c->k;
    w->v = (char *)c->v;
    w->k_scale = c->k_scale;
    w->v_scale = c->v_scale;
    if (c->page_stride < 0 || c->page_stride > UINT32_MAX || c->token_stride < 0 || c->token_stride > UINT32_MAX || c->scale_page_stride < 0 ||
        c->scale_page_stride > UINT32_MAX / 4 || c->scale_token_stride < 0 || c->scale_token_stride > UINT32_MAX / 4)
        return DL_ERR_INVALID;
    if (c->head_stride < 0 || c->head_stride > 1ll << 46 || c->scale_head_stride < 0 || c->scale_head_stride > 1ll << 44) return DL_ERR_INVALID;
    w->page_stride = (uint32_t)c->page_stride;
    w->token_stride = (uint32_t)c->token_stride;
    w->head_stride = c->head_stride;
    w->scale_page_stride = (uint32_t)(4 * c->scale_page_stride);
    w->scale_token_stride = (uint32_t)(4 * c->scale_token_stride);
    w->scale_head_stride = 4 * c->scale_head_stride;
    w->pages = (uint32_t)c->pages;
    w->heads = (uint32_t)c->heads;
    w->head_dim = (uint32_t)c->head_dim;
    w->page = dl_make_divider((uint32_t)c->page_tokens);
    return DL_OK;
}

extern "C" int dl_kv_write(const dl_kv_cache *cache, const dl_kv_rows *rows, void *stream)
{
    return kv_run<true>(cache, rows, stream);
}

extern "C" int dl_kv_read(const dl_kv_cache *cache, const dl_kv_rows *rows, void *stream)
{
    return kv_run<false>(cache, rows, stream);
}
