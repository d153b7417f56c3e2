// Whether pieces of the size that dl_piece_steps gives stay within what a workspace has room for: batches given as (tiles, steps, how many
// such sequences).
#include <cstdint>
#include <cstdio>
#include <vector>

#include "../../paper_2511_06605_amd/csrc/dl_pieces.h"

struct run {
    uint64_t tiles, steps, times;
};

static int bad;
static void check(uint32_t most_cut, const std::vector<run> &batch)
{
    unsigned __int128 all = 0;
    for (const run &r : batch) all += (unsigned __int128)r.tiles * r.steps * r.times;
    if (all >> 64) return;  // (more sequences, tiles and steps than a call has)
    const uint32_t size = dl_piece_steps((uint64_t)all, most_cut);
    unsigned __int128 cut = 0;
    for (const run &r : batch) {
        const uint64_t pieces = (r.steps + size - 1) / size;
        if (pieces > 1) cut += (unsigned __int128)r.tiles * pieces * r.times;
    }
    if (!size || size > DL_UNCUT || cut > most_cut) {
        std::printf("most_cut %u, size %u: %llu pieces\n", most_cut, size, (unsigned long long)cut);
        bad = 1;
    }
}

int main()
{
    const uint64_t long_ = 1ull << 24;
    // sixteen sequences of 8192 tiles and one of a single tile, all of 2^30 tokens: 2^32 + 2^15 steps a half of the pieces
    check(1024, {{8192, long_, 16}, {1, long_, 1}});
    check(2, {{1, long_, 257}});
    check(2, {{1, long_, 256}});
    check(2, {{1, long_, 255}, {1, 1, 60000}});
    // starts that decrease: every other sequence has all rows
    check(1024, {{1 << 19, long_, 32767}});
    check(3, {{1 << 19, long_, 32767}, {1, 0, 1}});
    check(1024, {{0, long_, 65535}});
    check(1024, {});
    uint64_t x = 88172645463325252ull;
    auto next = [&](uint64_t n) {
        x ^= x << 13, x ^= x >> 7, x ^= x << 17;
        return x % n;
    };
    for (int n = 0; n < 200000; ++n) {
        std::vector<run> batch(next(5) + 1);
        for (run &r : batch) r = {next(1ull << next(20)), next((1ull << next(25)) + 1), next(1ull << next(14)) + 1};
        check((uint32_t)next(1023) + 2u, batch);
    }
    // what it was before wherever that was right
    for (uint64_t all : {0ull, 1ull, 511ull, 512ull, 513ull, 1ull << 26, (1ull << 35) - 1, 1ull << 35}) {
        const uint64_t was = (all + 511) / 512;
        if (was <= DL_UNCUT && dl_piece_steps(all, 1024) != (was ? was : 1)) bad = 1;
    }
    std::puts(bad ? "wrong" : "ok");
    return bad;
}
