// Norms of queries and keys for each head, and the rotation by position, in one pass (dl_norm_rotate).
//
// A row is held in registers from its load to its store, eight elements a lane, as many lanes as it takes (the next power of two) side
// by side: the sum of squares goes round by swaps among them, and the other half of a pair is either in the lane itself (neighbours) or
// comes from the lane rotary / 16 further.  So every lane stores what it has loaded and nothing else, and an output may be its input.
// Memory is what bounds it: each row once in and once out; the table's rows come from the caches, since the heads of a token share one.
// Measured: 20 001 tokens of 32 heads of 128 in float16 (338 MB) 64.6 - 65.4 us, 5.2 TB/s; one token 3.9 us, a call.
#include "dl_codes.h"
#include "dl_internal.h"

namespace {

struct norm_side {
    const char *x;
    char *y;
    const float *weight;
    int64_t token, head, out_token, out_head;  // bytes
    uint32_t heads;
};
struct norm_args {
    norm_side q, k;
    const float *table;
    const int64_t *positions;
    int64_t table_rows, table_stride;  // floats
    uint32_t head_dim, rotary;
    // a part is a thread's heads of one token; those of q come first
    uint32_t tasks, q_parts;
    dl_divider parts;  // of a token
    float over_dim, eps;
    int32_t neighbours;
};

constexpr uint32_t NORM_THREADS = 256;
constexpr int NORM_ELEMENTS = 8;
// From so many threads on, two rows of a thread are on their way at once and stores go past the caches; from so many bytes moved on, loads
// too.  Measured with heads of 128 in 16 bits, one row and plain : two and plain loads : two and streaming loads : four and plain : four and
// streaming, 20001 tokens of 32 heads (338 MB) 81.6 : 68.5 : 65.4 : 76.4 : 71.9 us, 20001 of 40 (420 MB) 103 : 85.1 : 82.7 : 88.0 : 83.2,
// 8000 of 32 (135 MB) 29.7 : 26.1 : 28.1 : 26.5 : 31.3; plain stores cost 3.5 more.
constexpr uint64_t NORM_MANY_THREADS = 1ull << 20, NORM_STREAM_BYTES = 256ull << 20;

// Eight elements of a row.  STREAM: past the caches.
template <class T, bool STREAM>
__device__ __forceinline__ void load_eight(const char *p, float (&x)[NORM_ELEMENTS])
{
    if constexpr (STREAM && T::size == 2) {
        typedef dl_u32x4 anywhere __attribute__((aligned(1)));
        const dl_u32x4 w = __builtin_nontemporal_load((const anywhere *)p);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[2 * j] = T::lo(w[j]), x[2 * j + 1] = T::hi(w[j]);
    } else if constexpr (STREAM) {
        typedef dl_f32x4 anywhere __attribute__((aligned(1)));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const dl_f32x4 w = __builtin_nontemporal_load((const anywhere *)(p + 16 * h));
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * h + j] = w[j];
        }
    } else {
        dl_load_row<T>(p, x);
    }
}

// A thread has ROWS heads of one side of one token, which share the token's cosines and sines and the side's weights.  MODE: 0 all through the
// caches, 1 stores past them, 2 both.
template <class T, int LANES, int ROWS, int MODE>
__global__ void __launch_bounds__(NORM_THREADS) dl_norm_rotate_kernel(const norm_args a)
{
    constexpr int N = NORM_ELEMENTS;
    const uint32_t lane = threadIdx.x % LANES, task = (blockIdx.y * gridDim.x + blockIdx.x) * (NORM_THREADS / LANES) + threadIdx.x / LANES;
    const uint32_t at = lane * (uint32_t)N, half = a.rotary / 2u;
    const bool mine = at < a.head_dim, turned = at < a.rotary;
    // which pairs: of the lane's elements as first or second of theirs, or its own neighbours
    const bool second = !a.neighbours && at >= half;
    const uint32_t angle = a.neighbours ? at / 2u : second ? at - half : at;
    const uint32_t part = min(task, a.tasks - 1u), token = dl_divide(part, a.parts);
    uint32_t h0 = part - token * a.parts.d;
    const bool is_q = h0 < a.q_parts;
    const norm_side &s = is_q ? a.q : a.k;
    h0 = (is_q ? h0 : h0 - a.q_parts) * ROWS;
    const bool normed = s.weight != nullptr;
    bool live = task < a.tasks && mine;
    float x[ROWS][N], w[N], c[N], z[N];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[r][i] = 0.0f;
        if (mine) load_eight<T, MODE == 2>(s.x + token * s.token + min(h0 + r, s.heads - 1u) * s.head + (size_t)at * T::size, x[r]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = 1.0f, c[i] = 1.0f, z[i] = 0.0f;
    if (mine && normed) dl_load_row<dl_f32>((const char *)(s.weight + at), w);
    if (a.rotary) {
        const int64_t position = a.positions[token];
        const bool known = position >= 0 && position < a.table_rows;
        live &= known;
        if (turned && known) {
            const char *const p = (const char *)(a.table + position * a.table_stride + angle);
            if (a.neighbours) {
                const dl_f32x4 u = dl_load_at<dl_f32x4>(p), v = dl_load_at<dl_f32x4>(p + 4u * half);
#pragma unroll
                for (int i = 0; i < N; ++i) c[i] = u[i / 2], z[i] = v[i / 2];
            } else {
                dl_load_row<dl_f32>(p, c);
                dl_load_row<dl_f32>(p + 4u * half, z);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) sum = fmaf(x[r][i], x[r][i], sum);
#pragma unroll
        for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
        if (normed) {
            const float f = rsqrtf(fmaf(sum, a.over_dim, a.eps));
#pragma unroll
            for (int i = 0; i < N; ++i) x[r][i] = x[r][i] * f * w[i];
        }
        if (a.rotary) {
            float y[N];
            if (a.neighbours) {
#pragma unroll
                for (int i = 0; i < N; ++i) y[i] = x[r][i ^ 1] * (i % 2 ? 1.0f : -1.0f);
            } else {
                // (all lanes take part; those behind the rotated elements stay as they are, whatever they get)
                const uint32_t self = threadIdx.x % 64u, other = turned ? second ? self - half / N : self + half / N : self;
#pragma unroll
                for (int i = 0; i < N; ++i) y[i] = __shfl(x[r][i], (int)other) * (second ? 1.0f : -1.0f);
            }
            if (turned) {
#pragma unroll
                for (int i = 0; i < N; ++i) x[r][i] = fmaf(x[r][i], c[i], y[i] * z[i]);
            }
        }
        if (live && h0 + r < s.heads) dl_store_row<T, MODE != 0>(s.y + token * s.out_token + (h0 + r) * s.out_head + (size_t)at * T::size, x[r]);
    }
}

int norm_setup(const dl_norm_rotate_args *args, norm_args *a, bool *nothing)
{
    if (!args) return DL_ERR_INVALID;
    if (args->type < DL_TYPE_F32 || args->type > DL_TYPE_F16 || args->reserved != 0) return DL_ERR_INVALID;
    if (args->head_dim < 16 || args->head_dim > 256 || args->head_dim % 16 || args->rotary < 0 || args->rotary > args->head_dim || args->rotary % 16)
        return DL_ERR_INVALID;
    if (args->neighbours < 0 || args->neighbours > 1 || !(args->eps >= 0.0f)) return DL_ERR_INVALID;
    if (args->q_heads < 0 || args->k_heads < 0 || args->q_heads > 65535 || args->k_heads > 65535) return DL_ERR_INVALID;
    if (args->table_rows < 0 || args->table_rows > INT32_MAX) return DL_ERR_INVALID;
    const int64_t q_heads = args->q ? args->q_heads : 0, heads = q_heads + (args->k ? args->k_heads : 0);
    if (args->tokens < 0 || args->tokens > DL_MAX_ROWS || args->tokens * heads > DL_MAX_ROWS) return DL_ERR_INVALID;
    *nothing = args->tokens * heads == 0;
    if (*nothing) return DL_OK;
    if ((args->q && !args->q_out) || (args->k && !args->k_out)) return DL_ERR_INVALID;
    if (args->rotary && (!args->positions || (args->table_rows && !args->table))) return DL_ERR_INVALID;
    const int size = args->type == DL_TYPE_F32 ? 4 : 2;
    if (((uint64_t)args->q | (uint64_t)args->k | (uint64_t)args->q_out | (uint64_t)args->k_out) % size ||
        ((uint64_t)args->q_weight | (uint64_t)args->k_weight | (uint64_t)args->table) % 4u || (uint64_t)args->positions % 8u)
        return DL_ERR_INVALID;
    a->q = {(const char *)args->q, (char *)args->q_out, args->q_weight, args->q_token_stride * size, args->q_head_stride * size,
            args->q_out_token_stride * size, args->q_out_head_stride * size, (uint32_t)q_heads};
    a->k = {(const char *)args->k, (char *)args->k_out, args->k_weight, args->k_token_stride * size, args->k_head_stride * size,
            args->k_out_token_stride * size, args->k_out_head_stride * size, (uint32_t)(heads - q_heads)};
    a->table = args->table;
    a->positions = args->positions;
    a->table_rows = args->table_rows;
    a->table_stride = args->table_stride;
    a->head_dim = (uint32_t)args->head_dim;
    a->rotary = (uint32_t)args->rotary;
    a->over_dim = 1.0f / (float)args->head_dim;
    a->eps = args->eps;
    a->neighbours = args->neighbours;
    return DL_OK;
}

}  // namespace

extern "C" int dl_norm_rotate(const dl_norm_rotate_args *args, void *stream)
{
    DL_LOCKED;
    if (!g_dl.inited) return DL_ERR_STATE;
    if (dl_device_error_pending()) return DL_ERR_LOST;
    norm_args a;
    bool nothing;
    const int rc = norm_setup(args, &a, &nothing);
    if (rc != DL_OK || nothing) return rc;
    dl_with_type(args->type, [&](auto t) {
        dl_with_lanes<NORM_ELEMENTS>(a.head_dim, [&](auto lanes) {
            constexpr int L = decltype(lanes)::value;
            auto go = [&](auto rows, auto mode) {
                constexpr int ROWS = decltype(rows)::value;
                a.q_parts = (a.q.heads + ROWS - 1u) / ROWS;
                const uint32_t parts = a.q_parts + (a.k.heads + ROWS - 1u) / ROWS;
                a.parts = dl_make_divider(parts);
                a.tasks = (uint32_t)args->tokens * parts;
                // (rows of 256 elements may be one workgroup more than a grid is wide, 2^32 threads)
                const uint32_t blocks = (a.tasks + NORM_THREADS / L - 1u) / (NORM_THREADS / L), high = (blocks + (1u << 23) - 1u) >> 23;
                hipLaunchKernelGGL((dl_norm_rotate_kernel<decltype(t), L, ROWS, decltype(mode)::value>), dim3((blocks + high - 1u) / high, high),
                                   dim3(NORM_THREADS), 0, (hipStream_t)stream, a);
            };
            const uint64_t rows = (uint64_t)args->tokens * (a.q.heads + a.k.heads);
            // (a single head of a side, and the last of an odd number, cost a thread as much as two)
            const bool paired = (a.q.heads + 1u) / 2u + (a.k.heads + 1u) / 2u <= (a.q.heads + a.k.heads) * 5u / 8u;
            if (rows * L < NORM_MANY_THREADS)
                go(std::integral_constant<int, 1>{}, std::integral_constant<int, 0>{});
            else if (!paired)
                go(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
            else if (2u * rows * a.head_dim * decltype(t)::size < NORM_STREAM_BYTES)
                go(std::integral_constant<int, 2>{}, std::integral_constant<int, 1>{});
            else
                go(std::integral_constant<int, 2>{}, std::integral_constant<int, 2>{});
        });
    });
    DL_HIP(hipGetLastError());
    t_dl_last.mode = DL_MODE_ONESHOT;
    return DL_OK;
}
