// Internal declarations of what a server runs around the 8-bit paged cache (include/lookat_serve.h).
#pragma once

#include "common.cuh"
#include "lookat_serve.h"
#include "q8.cuh"

namespace lookat {

constexpr int kStatusBadStart = 16;         // a packed row's start or end out of range or order: taken as empty

// fp16 vectors of packed tokens (strides in elements; those of a single token or head are 0)
struct Rows {
    __half *p;
    long long ts, hs;
};

struct RopeArgs {
    Rows in[2], out[2];             // queries, keys; no heads: not given
    int heads[2];
    const int32_t *positions;
    const unsigned long long *turns;
    long long n;
    int d, r, interleaved;
    float amplitude;
};
lookat_status launch_rope(Ctx *ctx, const RopeArgs &a);

// Row b's tokens, or none where they are out of range or order.
struct Packed {
    const int32_t *starts;          // [B + 1]
    int B, n;                       // rows, tokens
    int *status;
};
__device__ __forceinline__ int packed_row(const Packed &p, int b, int &first)
{
    const int lo = p.starts[b], hi = p.starts[b + 1];
    const bool good = lo >= 0 && hi >= lo && hi <= p.n;
    first = good ? lo : 0;
    return good ? hi - lo : 0;
}

// the findings among all rows' starts, by a group of `threads`
__device__ __forceinline__ void packed_check(const Packed &p, int thread, int threads)
{
    for (int b = thread; b < p.B; b += threads) {
        const int lo = p.starts[b], hi = p.starts[b + 1];
        if (lo < 0 || hi < lo || hi > p.n) q8_report(p.status, kStatusBadStart);
    }
}

// Tile `item` of all rows' tiles of `per` lines each, a row of n tokens having n * g lines: by falling place within their rows, so
// that the tiles with the most tokens to attend start first.  Called by a whole warp; false behind the last tile.
//   With A(x) the number of tiles at place x or later (the sum over rows of tiles - x, where positive), the tile's place is the x
// with A(x + 1) <= item < A(x), found by bisection, and it is row number item - A(x + 1) of those with more than x tiles.
__device__ inline bool packed_tile(const Packed &p, int g, int per, int item, int lane, int &b, int &place, int &first, int &n)
{
    auto tiles_of = [&](int row, int &at, int &len) {
        len = row < p.B ? packed_row(p, row, at) : 0;
        return (int)(((long long)len * g + per - 1) / per);
    };
    int at, len;
    const int mine = tiles_of(lane, at, len);                   // (all there is for up to 32 rows)
    int most = mine;
    for (int row = lane + 32; row < p.B; row += 32) {
        int t, l;
        most = max(most, tiles_of(row, t, l));
    }
    most = __reduce_max_sync(0xffffffffu, most);
    auto later = [&](int x) {                                   // A(x)
        int sum = max(mine - x, 0);
        for (int row = lane + 32; row < p.B; row += 32) {
            int t, l;
            sum += max(tiles_of(row, t, l) - x, 0);
        }
        return __reduce_add_sync(0xffffffffu, sum);
    };
    int lo = 0, hi = most;                                      // A(lo) > item >= A(hi), if any
    if (later(0) <= item) return false;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        (later(mid) > item ? lo : hi) = mid;
    }
    place = lo;
    int rank = item - later(lo + 1);
    for (int row0 = 0; row0 < p.B; row0 += 32) {
        int t = at, l = len, tiles = mine;
        if (row0) tiles = tiles_of(row0 + lane, t, l);
        const unsigned who = __ballot_sync(0xffffffffu, tiles > lo);
        const int count = __popc(who);
        if (rank < count) {
            const int src = __ffs(__ballot_sync(0xffffffffu, tiles > lo && __popc(who & ((1u << lane) - 1)) == rank)) - 1;
            b = row0 + src;
            first = __shfl_sync(0xffffffffu, t, src);
            n = __shfl_sync(0xffffffffu, l, src);
            return true;
        }
        rank -= count;
    }
    return false;
}

struct PackedAttendArgs {
    Packed rows;
    Rows q, k, v, out;
    int H_q, H_kv, g, d_k, d_v;
    float scale_log2;               // softmax scale * log2(e)
};
lookat_status launch_attend_packed(Ctx *ctx, const PackedAttendArgs &a);
// on tcgen05 (attend_packed_umma.cu)
bool attend_packed_umma_covers(const Ctx *ctx, const PackedAttendArgs &a);
lookat_status launch_attend_packed_umma(Ctx *ctx, const PackedAttendArgs &a);
// How far the running exponent of a query lies below its largest score (base 2), so that the fp16 weights use fp16's range.
constexpr float kPackedLift = 7.f;

struct BeamArgs {
    float *scores;
    int32_t *lengths, *finished, *tokens;
    const float *logits;
    long long stride;
    int groups, beams, max_len, vocab, eos;
    double penalty;
    int32_t *next_ids, *parents;
};
lookat_status launch_beam_select(Ctx *ctx, const BeamArgs &a);

}  // namespace lookat
