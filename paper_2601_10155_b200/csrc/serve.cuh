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

// Tile `item` of all rows' tiles of `per` lines each, a row of n tokens having n * g lines.  Called by a whole warp; kTile, or kNoTile
// (this number has none, later ones may), or kNoMore.  There are at most n_tokens * g / per + B numbers.
//   Up to kSortedRows rows: by falling place within their rows, so that the tiles with the most tokens to attend start first.  With
// A(x) the number of tiles at place x or later (the sum over rows of tiles - x, where positive; below 2^31, as lines are), the tile's
// place is the x with A(x + 1) <= item < A(x), found by bisection, and it is row number item - A(x + 1) of those with more than x.
//   More rows: in their order, a row's tiles from number starts * g / per + row on, which a bisection over the rows finds.  (Looking
// through all rows takes longer than what the order gains: 256 rows of up to 500 tokens, 32 and 8 heads of 128, 622 us by place, 531
// in their order; 64 rows of up to 1500 698 and 690; 33 rows of up to 2000, 12 heads of 64, 180 and 204.)
enum { kNoMore = -1, kNoTile = 0, kTile = 1 };
constexpr int kSortedRows = 64;
__device__ inline int packed_tile(const Packed &p, int g, int per, int item, int lane, int &place, int &first, int &n)
{
    auto tiles_of = [&](int row, int &at, int &len) {
        len = row < p.B ? packed_row(p, row, at) : 0;
        return (int)(((long long)len * g + per - 1) / per);
    };
    if (p.B > kSortedRows) {
        if (item >= (long long)p.n * g / per + p.B) return kNoMore;
        auto number0 = [&](int row) { return (long long)min(max(p.starts[row], 0), p.n) * g / per + row; };
        int lo = 0, hi = p.B;                                   // the last row whose first number is not behind this one
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            (number0(mid) <= item ? lo : hi) = mid;
        }
        place = (int)(item - number0(lo));
        return place >= 0 && place < tiles_of(lo, first, n) ? kTile : kNoTile;
    }
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
    if (later(0) <= item) return kNoMore;
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
            first = __shfl_sync(0xffffffffu, t, src);
            n = __shfl_sync(0xffffffffu, l, src);
            return kTile;
        }
        rank -= count;
    }
    return kNoMore;
}

// numbers that packed_tile is to be asked for, whatever the rows' lengths (by place, there are no tiles of empty rows between)
inline long long packed_tiles(const Packed &p, int g, int per)
{
    return (long long)p.n * g / per + (p.B > kSortedRows || p.B < p.n ? p.B : p.n);
}

struct PackedAttendArgs {
    Packed rows;
    Rows q, k, v, out;
    int H_q, H_kv, g, d_k, d_v;
    float scale_log2;               // softmax scale * log2(e)
};
lookat_status launch_attend_packed(Ctx *ctx, const PackedAttendArgs &a);
lookat_status launch_attend_packed_any(Ctx *ctx, const PackedAttendArgs &a);       // any dims, on mma.sync
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
