// Verification of drafted tokens from given random numbers (dl_verify_draft).
//
// A draft x is accepted if u q(x) < p(x), which happens with probability min(1, p / q); behind the accepted ones the next token is
// drawn from what p has more than q (after a refusal) or from p.  The draw is a race: with e_v exponential of rate 1,
// the v with the largest w_v / e_v has probability w_v / sum of w.  So the draw is a maximum, and one of (quotient, lowest
// index) pairs at that: whole numbers of 64 bits, whose maximum does not depend on the order in which it is taken.
//
// Which row of p (and q) is drawn from follows from at most 63 pairs of probabilities; every wavefront finds it out for
// itself, a lane a draft.  Then one pass over that row, split over as many workgroups as fill the chip; the last one of a
// sequence to finish writes the result.  What is read is one row of p, race and, after a refusal, q: the rows of the
// other drafts are not touched beyond their own token.
#include "dl_codes.h"
#include "dl_internal.h"

namespace {

constexpr uint32_t VERIFY_THREADS = 256;

struct verify_args {
    const char *target, *draft;
    const int32_t *draft_tokens, *draft_lens;
    const float *uniform, *race;
    int32_t *tokens, *accepted;
    unsigned long long *best;  // per sequence: the largest pair so far; zero between calls
    uint32_t *arrived;         // per sequence: workgroups that have finished; zero between calls
    int64_t target_seq, target_row, draft_seq, draft_row;  // bytes
    int64_t race_seq;                                      // floats
    uint32_t drafts, vocab;
    uint32_t piece;  // entries of the row for a workgroup
};

template <class T>
__device__ __forceinline__ float probability(const char *row, uint32_t v)
{
    if constexpr (T::size == 4)
        return dl_load_at<float>(row + 4 * (size_t)v);
    else
        return T::one(dl_load_at<uint16_t>(row + 2 * (size_t)v));
}

template <class V>
__device__ __forceinline__ V load_once(const void *p)
{
    typedef V anywhere __attribute__((aligned(1)));
    return __builtin_nontemporal_load((const anywhere *)p);
}

// Four neighbours, which nobody else will read: past the caches.
template <class T>
__device__ __forceinline__ void probability4(const char *row, uint32_t v, float (&x)[4])
{
    if constexpr (T::size == 4) {
        const dl_f32x4 w = load_once<dl_f32x4>(row + 4 * (size_t)v);
        x[0] = w[0], x[1] = w[1], x[2] = w[2], x[3] = w[3];
    } else {
        const dl_u32x2 w = load_once<dl_u32x2>(row + 2 * (size_t)v);
        x[0] = T::lo(w[0]), x[1] = T::hi(w[0]), x[2] = T::lo(w[1]), x[3] = T::hi(w[1]);
    }
}

// The pair that stands for entry v of weight w: larger quotients first, then lower indexes; 0 for none.
__device__ __forceinline__ unsigned long long pair_of(float w, float e, uint32_t v)
{
    const float score = w / e;
    return w > 0.0f && score >= 0.0f ? (unsigned long long)dl_bits<uint32_t>(score) << 32 | (0xFFFFFFFFu - v) : 0ull;
}

__device__ __forceinline__ unsigned long long larger(unsigned long long a, unsigned long long b) { return a > b ? a : b; }

// The largest pair of entries first .. end - 1, in every thread of the workgroup.  q: subtracted where it is not null;
// without: this entry weighs nothing (0xFFFFFFFF: all count).
template <class T>
__device__ unsigned long long best_of(const char *p, const char *q, const float *race, uint32_t without, uint32_t first, uint32_t end)
{
    __shared__ unsigned long long part[VERIFY_THREADS / 64];
    unsigned long long best = 0;
    uint32_t v = first + threadIdx.x * 4u;
    auto look = [&](auto at_once) {  // as many fours of this thread at once, all of their loads in front of the first quotient
        constexpr uint32_t N = decltype(at_once)::value;
        for (; v + (N - 1u) * VERIFY_THREADS * 4u + 4u <= end; v += N * VERIFY_THREADS * 4u) {
            float w[N][4], x[N][4];
            dl_f32x4 e[N];
#pragma unroll
            for (uint32_t n = 0; n < N; ++n) {
                const uint32_t at = v + n * VERIFY_THREADS * 4u;
                probability4<T>(p, at, w[n]);
                e[n] = load_once<dl_f32x4>(race + at);
                if (q) probability4<T>(q, at, x[n]);
            }
#pragma unroll
            for (uint32_t n = 0; n < N; ++n)
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    const uint32_t at = v + n * VERIFY_THREADS * 4u + i;
                    if (q) w[n][i] -= x[n][i];
                    best = larger(best, pair_of(at == without ? 0.0f : w[n][i], e[n][i], at));
                }
        }
    };
    look(std::integral_constant<uint32_t, 4>{});
    look(std::integral_constant<uint32_t, 2>{});
    look(std::integral_constant<uint32_t, 1>{});
    for (; v < end; ++v) {  // one thread's: the end of the row inside its four
        float w = probability<T>(p, v);
        if (q) w -= probability<T>(q, v);
        best = larger(best, pair_of(v == without ? 0.0f : w, race[v], v));
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) best = larger(best, (unsigned long long)__shfl_xor((long long)best, d));
    __syncthreads();  // the words may still be read from an earlier call
    if (threadIdx.x % 64u == 0) part[threadIdx.x / 64u] = best;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < VERIFY_THREADS / 64; ++i) best = larger(best, part[i]);
    return best;
}

template <class T>
__global__ void __launch_bounds__(VERIFY_THREADS) dl_verify_kernel(const verify_args a)
{
    const uint32_t b = blockIdx.y, lane = threadIdx.x % 64u;
    uint32_t n = a.drafts;
    if (a.draft_lens) n = (uint32_t)min(max(a.draft_lens[b], 0), (int32_t)a.drafts);
    const char *const target = a.target + b * a.target_seq;
    const char *const draft = a.draft ? a.draft + b * a.draft_seq : nullptr;

    int32_t x = -1;
    bool refused = false;
    if (lane < n) {
        x = a.draft_tokens[(size_t)b * a.drafts + lane];
        refused = true;
        if (x >= 0 && (uint32_t)x < a.vocab) {
            const float u = a.uniform[(size_t)b * a.drafts + lane];
            const float p = probability<T>(target + lane * a.target_row, (uint32_t)x);
            const float q = draft ? probability<T>(draft + lane * a.draft_row, (uint32_t)x) : 1.0f;
            refused = !(u * q < p);
        }
    }
    const unsigned long long where = __ballot(refused);
    const uint32_t taken = where ? (uint32_t)__ffsll((long long)where) - 1u : n;
    const bool rest = taken < n;

    const char *const p = target + taken * a.target_row;
    const char *const q = rest && draft ? draft + taken * a.draft_row : nullptr;
    // (a draft outside the vocabulary is -1 or at least vocab as an unsigned number: no entry)
    const uint32_t without = rest && !draft ? (uint32_t)__shfl(x, (int)taken) : 0xFFFFFFFFu;
    const float *const race = a.race + b * a.race_seq;
    const uint32_t first = blockIdx.x * a.piece, end = min(first + a.piece, a.vocab);
    unsigned long long best = best_of<T>(p, q, race, without, first, end);

    if (gridDim.x > 1) {
        __shared__ unsigned long long joined;
        __shared__ bool last;
        if (threadIdx.x == 0) {
            // Both words change by atomic operations alone, which all take place where all XCDs see them, and the second is issued once
            // the first has returned: no cache has to be written back or emptied for that, which an ordering operation would do.
            unsigned long long before = __hip_atomic_fetch_max(a.best + b, best, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" : "+v"(before)::"memory");
            last = __hip_atomic_fetch_add(a.arrived + b, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1u;
            if (last) {
                joined = __hip_atomic_exchange(a.best + b, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __hip_atomic_store(a.arrived + b, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
        __syncthreads();
        if (!last) return;
        best = joined;
    }
    // nothing left of p beyond q (both equal, say, and p zero at the draft): from p itself
    if (!best && rest) best = best_of<T>(p, nullptr, race, 0xFFFFFFFFu, 0, a.vocab);
    if (threadIdx.x <= a.drafts) {  // at most 64 entries: the first wavefront, whose lanes hold the drafts
        const int32_t next = best ? (int32_t)(0xFFFFFFFFu - (uint32_t)best) : -1;
        a.tokens[(size_t)b * (a.drafts + 1u) + threadIdx.x] = threadIdx.x < taken ? x : threadIdx.x == taken ? next : -1;
        if (threadIdx.x == 0) a.accepted[b] = (int32_t)taken;
    }
}

// Entries of a workgroup's piece of a row: so many that the batch makes two workgroups for each of the chip's 256 compute units, a
// multiple of what the threads look at at once.  More workgroups only find out more often where to look: 128 sequences of 4
// drafts over 128000 entries 30.7 us with 512, 32.2 with 1024, and (with loads that stay in the caches) 35.0, 36.0, 36.8, 42.0 and 66.9
// with 512, 1024, 2048, 4096 and 8192.  At 30 us that case reads 5.7 TB/s; 26 us is what its 170 MB take at the rate of a large copy.
uint32_t verify_piece(int32_t batch, int32_t vocab)
{
    const uint32_t split = (512u + (uint32_t)batch - 1u) / (uint32_t)batch, step = 4u * VERIFY_THREADS;
    return (((uint32_t)vocab + split - 1u) / split + step - 1u) / step * step;
}

constexpr int32_t VERIFY_MAX_BATCH = 1 << 20;
// sequences that are split (at most 511 of them) have a pair and a counter each in the control words
static_assert(512 * (sizeof(unsigned long long) + sizeof(uint32_t)) <= DL_CONTROL_BYTES, "control words of the sequences that are split");

int verify_check(const dl_verify_draft_args *a)
{
    if (!a) return DL_ERR_INVALID;
    if (a->type < DL_TYPE_F32 || a->type > DL_TYPE_F16) return DL_ERR_INVALID;
    if (a->batch < 0 || a->batch > VERIFY_MAX_BATCH || a->drafts < 0 || a->drafts > DL_MAX_DRAFTS || a->vocab < 1 || a->vocab > 1 << 30)
        return DL_ERR_INVALID;
    return DL_OK;
}

}  // namespace

extern "C" int64_t dl_verify_draft_workspace(const dl_verify_draft_args *args)
{
    const int rc = verify_check(args);
    return rc != DL_OK ? rc : (int64_t)DL_CONTROL_BYTES;
}

extern "C" int dl_verify_draft(const dl_verify_draft_args *args, void *stream)
{
    DL_LOCKED;
    if (!g_dl.inited) return DL_ERR_STATE;
    if (dl_device_error_pending()) return DL_ERR_LOST;
    const int rc = verify_check(args);
    if (rc != DL_OK) return rc;
    if (args->batch == 0) return DL_OK;
    if (!args->target || !args->race || !args->tokens || !args->accepted) return DL_ERR_INVALID;
    if (args->drafts && (!args->draft_tokens || !args->uniform)) return DL_ERR_INVALID;
    const uint64_t size = args->type == DL_TYPE_F32 ? 4 : 2;
    if (((uint64_t)args->target | (uint64_t)args->draft) % size) return DL_ERR_INVALID;
    if (((uint64_t)args->race | (uint64_t)args->uniform | (uint64_t)args->draft_tokens | (uint64_t)args->draft_lens | (uint64_t)args->tokens |
         (uint64_t)args->accepted) %
        4u)
        return DL_ERR_INVALID;
    const uint32_t piece = verify_piece(args->batch, args->vocab);
    if (piece < (uint32_t)args->vocab && (!args->workspace || args->workspace_bytes < DL_CONTROL_BYTES || (uint64_t)args->workspace % 16u)) return DL_ERR_INVALID;
    verify_args a;
    a.target = (const char *)args->target;
    a.draft = (const char *)args->draft;
    a.draft_tokens = args->draft_tokens;
    a.draft_lens = args->draft_lens;
    a.uniform = args->uniform;
    a.race = args->race;
    a.tokens = args->tokens;
    a.accepted = args->accepted;
    a.best = (unsigned long long *)args->workspace;
    a.arrived = (uint32_t *)(a.best + 512);
    a.target_seq = args->target_seq_stride * (int64_t)size;
    a.target_row = args->target_row_stride * (int64_t)size;
    a.draft_seq = args->draft_seq_stride * (int64_t)size;
    a.draft_row = args->draft_row_stride * (int64_t)size;
    a.race_seq = args->race_stride;
    a.drafts = (uint32_t)args->drafts;
    a.vocab = (uint32_t)args->vocab;
    a.piece = piece;
    const dim3 grid(((uint32_t)args->vocab + a.piece - 1u) / a.piece, 1);
    dl_with_type(args->type, [&](auto t) {
        // (a grid is at most 65 535 high)
        for (int32_t b0 = 0; b0 < args->batch; b0 += 65535) {
            const uint32_t n = (uint32_t)(args->batch - b0 < 65535 ? args->batch - b0 : 65535);
            verify_args c = a;
            c.target += b0 * a.target_seq;
            if (c.draft) c.draft += b0 * a.draft_seq;
            if (c.draft_tokens) c.draft_tokens += (int64_t)b0 * args->drafts;
            if (c.draft_lens) c.draft_lens += b0;
            if (c.uniform) c.uniform += (int64_t)b0 * args->drafts;
            c.race += b0 * a.race_seq;
            c.tokens += (int64_t)b0 * (args->drafts + 1);
            c.accepted += b0;
            hipLaunchKernelGGL((dl_verify_kernel<decltype(t)>), dim3(grid.x, n), dim3(VERIFY_THREADS), 0, (hipStream_t)stream, c);
        }
    });
    DL_HIP(hipGetLastError());
    t_dl_last.mode = DL_MODE_ONESHOT;
    return DL_OK;
}
