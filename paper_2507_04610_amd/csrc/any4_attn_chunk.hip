// any4_attn_chunk / any4_attn_prompt_window: the newest tokens of each request attend, causally, to its tokens in the paged cache (16 bits, or codes
// of 8 or 4), or packed prompts to packed keys; with a window each query sees the last keys up to its own and the first of the request.
//
//     s_ij = scale q_i . k_j,   o_i = sum_j exp(s_ij - m_i) v_j / sum_j exp(s_ij - m_i)     over j <= p_i, j > p_i - window or j < sinks
// in one pass over the keys with a running maximum, as any4_attn_prompt does it.
//
// A row is a query of one of the heads that share a KV head, a query's heads side by side, so that a few new tokens fill a block with their heads and
// read k and v once.  A block takes 128 rows, a wavefront 32 of them, and walks over the keys 64 at a time: S^T = K Q^T with
// v_mfma_f32_32x32x16, the scores of a row in two lanes, the weights at once the B operand of O^T = V^T P^T.  Tiles outside of what the block's rows see (behind
// the last query, between the first tokens and the window) are left out.  Of up to 32 rows each wavefront takes all and every fourth 32 keys, in LDS of its
// own, and the four meet at the end: nobody waits in front of a tile (up to 8 drafted tokens for each of 16 requests over a cache of 4 bits: 174 -> 106 us).
//
// 16 bits: k and v are copied to LDS without passing registers, the next 64 keys while these are worked on.  Codes c become fp16 on their way
// to LDS, exactly (k: c + kBias, v: c - kCentre), and scales and offsets are applied to sums, so that codes cost no rounding of their own:
//     q . k_j = ks_j (q . c'_j) + (ko_j - kBias ks_j) sum(q)
//     o = sum_j (p_j vs_j) (c_j - kCentre) + sum_j p_j (vo_j + kCentre vs_j)
// bf16 queries become fp16 for that: a row is scaled by a power of two, which is exact down to 2^-15 of its largest value and off by 2^-26 of that
// below, less than the fp32 sums are.  The product p_j vs_j is rounded to fp16; the exponent of the largest product that a row has had is taken off it together
// with the running maximum (that of the largest vs_j alone would leave nothing of the others beside a large value of no weight).
//
// Who does what.  Lengths are the device's, so each block finds its rows itself, of more than 64 requests in what a first launch of one block writes down
// (a token each of 2048 requests over 300 tokens in 8 bits: 449 us, 670 if each block looks).  Where whole tiles of rows do not fill the chip, their keys are cut
// into pieces, no more than it takes; pieces leave sums, maximum and sum of weights in the workspace, and a last launch joins them (3 to 5 us: short
// calls are not cut).
//
// Rounding: scores, maxima, sums and accumulators are fp32; the weights (times vs_j) are rounded to 16 bits for the matrix cores, once.
//
// Measured, 8 KV heads, us (what bounds it):
//     16 bits, 2048 tokens behind 30720, 32 query heads of 128     1005 - 1055  (1.01 - 1.06 PFLOP/s: matrix cores busy 49 %, vector units 49 %;
//                                                                               wavefronts wait 27 % of their time for LDS and each other)
//     the same, window of 4096 and first 4                           154 - 159  (0.89 PFLOP/s)
//     the same over 8 and 4 bits, bf16                     1405 - 1480, 1385 - 1445  (0.72 - 0.77 PFLOP/s); 8 bits with the window 205 (0.67)
//     8 bits, 24 requests of 1 .. 511 tokens, fp16                   410 - 435  (0.57 PFLOP/s: vector units busy 50 %, LDS 37 %, matrix cores 24 %; 6.5 of 8
//                                                                               wavefronts there on average, which wait 31 % of their time)
//     4 bits, 16 requests, up to 8 drafted tokens                     63 -  68  (2.2 TB/s: vector units 51 %; 5 of it the join; 5.6 of 8 wavefronts)
//     16 bits, 19 tokens behind 333                                   9.5       (loads that wait for each other: starts, lengths, page, k and v)
//     packed rows, a prompt of 12011, window 2048                   412 - 425   (0.88 - 0.90 PFLOP/s)
//     packed rows, fp16, 8450 tokens, 16 heads of 64 on 2, window 777  54       (0.50 PFLOP/s: 1060 blocks of 13 tiles of keys, whose beginnings and
//                                                                               ends and the second round of them cost as much as the tiles)
// Without gain: longest pieces first, more and smaller pieces than fill the chip, a fixed priority for one of a SIMD's wavefronts, an order of loads and products
// prescribed to the compiler, a closer search for the length of pieces.
#include "any4_attn.h"
#include "any4_attn_tile.h"
#include "any4_internal.h"
#include "any4_launches.h"
#include "any4_lds_copy.h"

namespace any4 {

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kRowTile = 32 * kWaves;
// Costs are counted in tiles of keys for 32 rows.  Figures: us with 32 query heads on 8 KV heads of 128, 16 bits unless said otherwise.
constexpr int kNarrow = 4;                                      // so many take as long as one for 128
constexpr int kFewRows = 64;                                    // requests of up to so many rows have tiles of 32, as small calls (65 requests of 64 rows
                                                                // over 1000 tokens in 8 bits: 78 us, in tiles of 128 94)
// Least of a piece.  19 of 1000 tokens: 12.6, with 8 14.4, with 16 17.9; one of 8000 16.1, 15.6, 19.1.
constexpr int kLeastPiece = 4;
// Tiles of 32 rows, of 128 rows, of so much are not cut: writing pieces and joining them costs as much.  19 of 700 tokens (11 tiles): whole 13.2, cut 12.5; of 1000
// whole 15.8, cut 12.6; of 1500 whole 20.6, cut 13.0.  Where no request can have more, the join is not launched either (1024 of 1024 tokens 30.3, with a join of nothing 33;
// 64 requests of a token of 1000 in 8 bits 28.4 and 33.3).
constexpr int kWholeFew = 12, kWhole = 40;
// Calls of so much for 128 rows at a time take 32 at a time: more blocks, each done sooner.  19 of 32000 tokens: 38.9, with 4096 50.2; 512 of 512 13.0, 18.1; 4 requests
// of 100 of 1000 tokens in 8 bits 30.9, 35.2; but 512 of 8000 86, with 65536 111, and 2048 of 2048 61.6, 81.3.
constexpr int kSmall = 16384;
constexpr int kNoWindow = 0x7FFFF800;                           // more than any request's tokens
// Codes: what is taken off the exponents of the products p_j vs_j goes with the maximum as far as 2^+-kFold: beyond, weights of tokens whose scales differ by 2^126 and
// more would be lost to the sum of weights.  The rest is taken off the products themselves.
constexpr int kFold = 40;
// The largest product stands 2^kUp above 1 (2^kSlack more at most, below 2^15 in all): fp16 has steps of 2^-24 down there, and tokens of small weight are many.
constexpr int kUp = 6;
// Scales of a tile that lie within 2^kSpread are taken as the largest of them (the largest product then lies as much lower at most), others with their scores.
constexpr int kSpread = 8;
typedef __attribute__((address_space(3))) float* lds_f;
typedef __attribute__((address_space(3))) f32x4* lds_f4;
typedef __attribute__((address_space(3))) uint32_t* lds_u1;
constexpr int kRows = 0;                                        // SOURCE: packed rows (whose keys are never cut); otherwise the cache's bits

struct Args {
    Rows q, k, v;                      // k, v: packed keys
    KvPages c;
    const int32_t* table;
    int64_t table_stride;
    int table_width;
    const int32_t* q_starts;
    const int32_t* k_starts;           // packed keys
    const int32_t* lengths;            // cache
    int q_tokens, k_tokens, requests, heads, kv_heads, shared, window, sinks;
    int target, slots;                 // blocks that fill the chip (0: nothing is cut); pieces that the workspace has room for
    int small;                         // whether the call may be one that takes 32 rows at a time
    const int* plan;                   // more than 64 requests: where each one's blocks end (see Plan); NULL: blocks look for themselves
    int* joins;                        // what the join has to do (see Join); NULL: nothing is cut
    int cut_tiles;                     // room in it
    unsigned first_block;              // of this launch
    float scale_log2;
    uint16_t* out;
    float* partial;
    // row / shared by a product: with 2^(s - 1) < shared <= 2^s and mul = 2^(31 + s) / shared rounded up, below 2^32, exact for rows below 2^31
    uint32_t shared_mul;
    int shared_shift;                  // 31 + s
    __device__ __forceinline__ int query_of(int row) const { return (int)(((uint64_t)(uint32_t)row * shared_mul) >> shared_shift); }
};

// A request's rows and keys.
struct Request {
    int q_at, lq, k_at, lk;
    bool back;                         // its rows would end in front of where they begin
};
template <int SOURCE> __device__ __forceinline__ Request request_of(const Args& a, int r) {
    Request q;
    q.q_at = min(max(a.q_starts[r], 0), a.q_tokens);
    const int lq = min(max(a.q_starts[r + 1], 0), a.q_tokens) - q.q_at;
    q.lq = max(lq, 0);
    q.back = lq < 0;
    if constexpr (SOURCE == kRows) {
        q.k_at = min(max(a.k_starts[r], 0), a.k_tokens);
        q.lk = max(min(max(a.k_starts[r + 1], 0), a.k_tokens) - q.k_at, 0);
    } else {
        q.k_at = 0;
        q.lk = (int)min((int64_t)max(a.lengths[r], 0), (int64_t)a.table_width << a.c.page_shift);
    }
    return q;
}

// The tiles of keys that a tile of rows sees: the first `front`, then from the one in which the window begins, `gap` tiles further on.
struct Span {
    int first, last;                   // first and last query
    int front, gap, tiles, end;        // end: of the keys that the last query sees
    __device__ __forceinline__ int real(int t) const { return t < front ? t : t + gap; }
};
__device__ __forceinline__ Span span_of(const Args& a, const Request& r, int tile, int height) {
    Span s;
    const int rows = r.lq * a.shared, ahead = r.lk - r.lq;
    s.first = a.query_of(tile * height);
    s.last = a.query_of(min(tile * height + height, rows) - 1);
    const int end = s.end = max(ahead + s.last + 1, 0), start = max(max(ahead + s.first, 0) + 1 - a.window, 0);
    const int begin = start / kKeys;
    s.front = min((int)(((unsigned)min(a.sinks, end) + kKeys - 1) / kKeys), begin);
    s.gap = begin - s.front;
    s.tiles = (int)(((unsigned)end + kKeys - 1) / kKeys) - s.gap;
    return s;
}

// Which rows and keys a block has.  Blocks of a request: tile of rows by tile of rows, each tile's pieces side by side.
struct Work {
    int request, tile, piece, pieces, slot, height;
    int join;                          // which of the tiles of rows that are cut (without KV heads)
    Request r;
};
struct Shares {                        // of 64 requests, a lane each
    Request r;
    int tiles, pieces;
};
// rows of a request's tiles, in a call whose requests of many rows have tiles of `most`
__device__ __forceinline__ int height_of(const Args& a, const Request& r, int most) { return r.lq * a.shared <= kFewRows ? 32 : most; }
__device__ __forceinline__ int tiles_of(const Args& a, const Request& r, int most) {
    const int height = height_of(a, r, most);
    return (int)(((unsigned)(r.lq * a.shared) + (unsigned)height - 1) >> (height == 32 ? 5 : 7));
}
// what its last (and longest) tile of rows costs, and what may be cut
__device__ __forceinline__ int costs_of(const Args& a, const Request& r, int tiles, int most) {
    const int height = height_of(a, r, most), of_keys = span_of(a, r, tiles - 1, height).tiles;
    return height == 32 ? of_keys : kNarrow * of_keys;
}
__device__ __forceinline__ int whole_of(const Args& a, const Request& r, int most) { return height_of(a, r, most) == 32 ? kWholeFew : kWhole; }
// How a call is cut: rows of a tile, and the most that a piece costs (0: nothing is cut).  Sums in fp32, in one order everywhere.
struct Cut {
    int height, least;
};
// over all lanes, in each of them
__device__ __forceinline__ float lanes_total(float v) {
    auto add = [&](auto ctrl, auto rows) { v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), decltype(ctrl)::value, decltype(rows)::value, 0xF, true)); };
    add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xF>{});       // row_shr:1
    add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xF>{});
    add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xF>{});
    add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xF>{});
    add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});       // row_bcast:15
    add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});       // row_bcast:31
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}
// sum(f): f of all requests, added up
template <class Sum> __device__ __forceinline__ Cut cut_of(const Args& a, Sum sum) {
    Cut cut{a.small ? 32 : kRowTile, 0};
    if (a.target == 0) return cut;                              // (then the host knows)
    const float heads = (float)a.kv_heads, target = (float)a.target;
    auto costs = [&](int height) {
        return sum([&](const Request& r) -> float {
            const int n = tiles_of(a, r, height);
            // (where starts go back, requests may have more tiles together than there are blocks, and nothing is cut)
            return r.back ? 1e30f : n > 0 ? (float)n * (float)costs_of(a, r, n, height) : 0.0f;
        }) * heads;
    };
    float all = costs(kRowTile);
    cut.height = kRowTile;
    if (a.small && all <= (float)kSmall) {
        cut.height = 32;
        all = costs(32);
    }
    // Pieces of all: at most cost / least and one for each tile, together no more than fill the chip, as far as that leaves pieces to cut.  That counts a
    // piece's rounding up as a whole one: shorter ones are tried, and taken if they are no more than fill the chip.
    const float tiles = sum([&](const Request& r) { return (float)tiles_of(a, r, cut.height); }) * heads, limit = 1073741824.0f;
    const int most = max((int)fminf(ceilf(all / fmaxf(target - tiles, 0.5f * target)), limit), kLeastPiece);
    const int low = max((int)fminf(ceilf(all / target), limit), kLeastPiece);
    cut.least = most;
    for (int third = 0; third < 3; ++third) {
        const int shorter = low + (most - low) * third / 3;
        if (shorter >= most) break;
        const float pieces = sum([&](const Request& r) -> float {
            const int n = tiles_of(a, r, cut.height), cost = n > 0 ? costs_of(a, r, n, cut.height) : 0;
            return cost > whole_of(a, r, cut.height) ? (float)n * (float)((cost + shorter - 1) / shorter) : (float)n;
        });
        if (pieces * heads <= target) {
            cut.least = shorter;
            break;
        }
    }
    cut.height = __builtin_amdgcn_readfirstlane(cut.height);
    cut.least = __builtin_amdgcn_readfirstlane(cut.least);
    return cut;
}
__device__ __forceinline__ Shares shares_of(const Args& a, const Request& r, const Cut& cut) {
    Shares s{r, tiles_of(a, r, cut.height), 1};
    if (s.tiles > 0 && cut.least > 0) {
        const int cost = costs_of(a, r, s.tiles, cut.height);
        if (cost > whole_of(a, r, cut.height)) s.pieces = (cost + cut.least - 1) / cut.least;
    }
    return s;
}
// Tiles of rows that are cut, for the launch that joins them, which then has nothing to look for (where nothing turns out to be cut that is 3 us less than if its
// blocks looked: 4 requests of 100 of 1000 tokens 34.5 -> 31.7 us).  First how many there are, then of each:
struct alignas(16) Join {
    int q_at, rows, row, height;       // the request's first query and rows, the tile's first row, its rows at most
    int pieces, slot, unused[2];       // pieces with keys, the first one's place
    __host__ __device__ static int64_t bytes(int64_t tiles) { return ((tiles + 1) * (int64_t)sizeof(Join) + 255) / 256 * 256; }
};
// More than 64 requests: a launch in front of the others has one block find out what each would find for itself.
struct Plan {
    // [4][requests] behind the height of tiles of rows: where a request's blocks end, where its tiles that are cut begin, its first piece's place (all
    // without KV heads), its pieces
    static constexpr int kHeader = 4;
    __host__ __device__ static int64_t bytes(int64_t requests) { return (4 * (kHeader + 4 * requests) + 255) / 256 * 256; }
};
constexpr int kPlanThreads = 1024;
template <int SOURCE>
__global__ __launch_bounds__(kPlanThreads) void attn_chunk_plan_kernel(Args a, int* plan) {
    constexpr int WAVES = kPlanThreads / 64;
    __shared__ float partial[WAVES];
    __shared__ int sums[3][WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Cut how = cut_of(a, [&](auto f) {
        float mine = 0.0f, all = 0.0f;
        for (int r = threadIdx.x; r < a.requests; r += kPlanThreads) mine += f(request_of<SOURCE>(a, r));
        mine = lanes_total(mine);
        __syncthreads();
        if (lane == 0) partial[wave] = mine;
        __syncthreads();
        for (int i = 0; i < WAVES; ++i) all += partial[i];
        return all;
    });
    if (threadIdx.x == 0) plan[0] = how.height;
    int* const at = plan + Plan::kHeader;
    int before[3] = {0, 0, 0};
    for (int r0 = 0; r0 < a.requests; r0 += kPlanThreads) {
        const int r = r0 + (int)threadIdx.x;
        Shares s = shares_of(a, r < a.requests ? request_of<SOURCE>(a, r) : Request{}, how);
        // each thread gets the sum of the threads up to its own
        auto scan = [&](int which, int v) -> int {
            const int up_to = lanes_scan(v);
            if (lane == 63) sums[which][wave] = up_to;
            __syncthreads();
            int here = before[which];
            for (int w = 0; w < WAVES; ++w) {
                if (w < wave) here += sums[which][w];
                before[which] += sums[which][w];
            }
            __syncthreads();
            return here + up_to;
        };
        const int cut = s.pieces > 1 ? s.tiles * s.pieces : 0, cut_end = scan(0, cut);
        // (as many as were planned for; were there more, they would be left whole)
        if (cut > 0 && (int64_t)cut_end * a.kv_heads > a.slots) s.pieces = 1;
        const int joins = s.pieces > 1 ? s.tiles : 0, end = scan(1, s.tiles * s.pieces), join_end = scan(2, joins);
        if (r < a.requests) {
            at[r] = end;
            at[a.requests + r] = join_end - joins;
            at[2 * a.requests + r] = cut_end - cut;
            at[3 * a.requests + r] = s.pieces;
        }
    }
    if (a.joins && threadIdx.x == 0) a.joins[0] = before[2] * a.kv_heads;
}
template <int SOURCE> __device__ __forceinline__ Work planned(const Args& a, unsigned place, unsigned kv_head, int lane) {
    Work w{-1, 0, 0, 1, 0, a.plan[0], 0, {}};
    const int* const ends = a.plan + Plan::kHeader;
    // the first request that ends behind `place`, among 64 at a time
    int from = 0, n = a.requests;
    for (;;) {
        const int step = (n + 63) / 64, mine = min((lane + 1) * step, n) - 1;
        const unsigned long long past = __builtin_amdgcn_ballot_w64((unsigned)ends[from + mine] > place);
        if (!past) return w;
        const int f = __builtin_ctzll(past);
        from += f * step;
        n = min(step, n - f * step);
        if (step == 1) break;
    }
    w.request = __builtin_amdgcn_readfirstlane(from);
    w.r = request_of<SOURCE>(a, w.request);
    w.height = height_of(a, w.r, w.height);
    w.pieces = ends[3 * a.requests + w.request];
    const int begin = w.request > 0 ? ends[w.request - 1] : 0, all = ends[w.request] - begin, own = (int)place - begin, tile = own / w.pieces;
    w.piece = own - tile * w.pieces;
    w.tile = all / w.pieces - 1 - tile;                         // the most keys first
    w.join = ends[a.requests + w.request] + tile;
    w.slot = (ends[2 * a.requests + w.request] + tile * w.pieces + w.piece) * a.kv_heads + (int)kv_head;
    if ((unsigned)own >= (unsigned)all) w.request = -1;         // (starts that do not ascend can add up to more than 32 bits hold)
    return w;
}

// place: of the block, without KV heads
template <int SOURCE> __device__ __forceinline__ Work work_of(const Args& a, unsigned place, unsigned kv_head, int lane) {
    constexpr bool CUTS = SOURCE != kRows;
    if constexpr (CUTS) {
        if (a.plan) return planned<SOURCE>(a, place, kv_head, lane);
    }
    // (where something is cut there are no more than 64 requests)
    const Request first = lane < a.requests ? request_of<SOURCE>(a, lane) : Request{};
    Cut how{a.small ? 32 : kRowTile, 0};
    if constexpr (CUTS) how = cut_of(a, [&](auto f) { return lanes_total(f(first)); });
    Work w{-1, 0, 0, 1, 0, how.height, 0, {}};
    for (int r0 = 0, before = 0, cut_before = 0; r0 < a.requests && w.request < 0; r0 += 64) {
        Request r = first;
        if (r0 > 0) r = r0 + lane < a.requests ? request_of<SOURCE>(a, r0 + lane) : Request{};
        Shares s = shares_of(a, r, how);
        int cut_sum = 0;
        if constexpr (CUTS) {
            const int cut = s.pieces > 1 ? s.tiles * s.pieces : 0;
            cut_sum = lanes_scan(cut);
            // (as many as were planned for; were there more, they would be left whole)
            if (cut > 0 && (int64_t)(cut_before + cut_sum) * a.kv_heads > a.slots) s.pieces = 1;
        }
        const int own = s.tiles * s.pieces, sum = lanes_scan(own), joins = s.pieces > 1 ? s.tiles : 0;
        int joins_sum = 0;
        if (CUTS && a.joins) {
            joins_sum = lanes_scan(joins);
            if ((place | kv_head) == 0u && threadIdx.x == 63) a.joins[0] = joins_sum * a.kv_heads;
        }
        const unsigned long long past = __builtin_amdgcn_ballot_w64((unsigned)(before + sum) > place);
        if (past) {
            const int f = __builtin_ctzll(past);
            w.request = r0 + f;
            w.r.q_at = __builtin_amdgcn_readlane(s.r.q_at, f);
            w.r.lq = __builtin_amdgcn_readlane(s.r.lq, f);
            w.r.k_at = __builtin_amdgcn_readlane(s.r.k_at, f);
            w.r.lk = __builtin_amdgcn_readlane(s.r.lk, f);
            w.height = height_of(a, w.r, how.height);
            w.pieces = __builtin_amdgcn_readlane(s.pieces, f);
            const int tiles = __builtin_amdgcn_readlane(s.tiles, f);
            const int all = __builtin_amdgcn_readlane(own, f), at = (int)place - (before + __builtin_amdgcn_readlane(sum, f) - all);
            if ((unsigned)at >= (unsigned)all) {                // (starts that do not ascend can add up to more than 32 bits hold)
                w.request = -1;
                break;
            }
            const int tile = at / w.pieces;
            w.piece = at - tile * w.pieces;
            w.tile = tiles - 1 - tile;                          // the most keys first
            w.join = __builtin_amdgcn_readlane(joins_sum - joins, f) + tile;
            w.slot = (cut_before + __builtin_amdgcn_readlane(cut_sum, f) - tiles * w.pieces + tile * w.pieces + w.piece) * a.kv_heads + (int)kv_head;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
        cut_before += __builtin_amdgcn_readlane(cut_sum, 63);
    }
    return w;
}

// How v's pieces of 16 bytes lie in a tile's row: four neighbouring rows' in different banks for the transposing reads, and in the last two bits in
// different ones for the writes of widened codes, whose lanes have pieces four (two) apart.
template <int D> __device__ __forceinline__ constexpr int swizzle_v(int row) { return D == 128 ? 5 * (row & 3) : ((row >> 1) & 1) << 2 | ((row >> 1) & 3); }

// LDS aside from the tiles.  Scales of TOKENS tokens: k's scale and offset, v's likewise, the exponent of v's; then the largest of those, whether they lie
// far apart, whose v's are not finite.
template <int TOKENS> constexpr int kScaleBytes = 20 * TOKENS + 16;
template <bool CODES> constexpr int kAsideAll = CODES ? kWaves * kScaleBytes<32> : kWaves * 32 * 8;

// floats of a piece: sums [wavefront][4 values of a row][lane][4], then [row] maximum and sum of weights
template <int D> constexpr int kPieceFloats = kRowTile * (D + 2);

// a - b where a may come out of a product: that is rounded first (from 2^31 on its rounding alone would be hundreds)
__device__ __forceinline__ float difference(float a, float b) {
#pragma clang fp contract(off)
    return a - b;
}
// Of the exponent taken off products: with the maximum m, and off the products themselves.  (All of it there where m is far, or without a score yet -inf: a sum with m would round it away.)
__device__ __forceinline__ float with_maximum(float m, float e) { return fabsf(m) > kFar ? 0.0f : fminf(fmaxf(e, (float)-kFold), (float)kFold); }
__device__ __forceinline__ int folded(float m, float e) { return (int)(e - with_maximum(m, e)); }

// the largest of LANES lanes (32, the first, or 64), in all.  (No lane reads LDS for that, as shuffles do: others wait for the wavefront that is at a tile's scales.)
template <int LANES> __device__ __forceinline__ float lanes_largest(float v) {
    v = lanes_reduce<16>(v, [](float a, float b) { return fmaxf(a, b); });
    auto before = [&](auto ctrl, auto rows) {
        v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(v), __float_as_uint(v), decltype(ctrl)::value, decltype(rows)::value, 0xF, false)));
    };
    before(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});    // row_bcast:15
    if constexpr (LANES == 64) before(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});    // row_bcast:31
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), LANES - 1));
}

// What is kept of a token's v for that: the exponent of its scale (of its middle times 2^-64 if that is more: a constant vector has scale 1 however large it is,
// and its product with the weight is to stay in fp32's range), 2^kUp lower.
__device__ __forceinline__ float exponent_of(float vs, float mid) {
    return fmaxf(ceilf(__builtin_amdgcn_logf(fmaxf(fabsf(vs), fabsf(mid) * 0x1p-64f))), -126.0f) - (float)kUp;
}

template <int BITS> struct Codes {
    static constexpr float kBias = BITS == 8 ? 1024.0f : 64.0f, kCentre = (float)(1 << (BITS - 1));
};
// Scores over codes of bf16 pass fp32 between q in fp16's range and the end, whatever the sizes of q and k: k's scales and offsets lie in LDS 2^kDown lower (exactly,
// as every bf16 value does that far down), q's largest value lies at 2^kTop, so that its product with codes, their bias and the largest scale stays below 2^127; or, where
// with the softmax scale it comes to 2^kLarge and more, so that what undoes all that has to stay there as well, at 2^kTopLarge.
constexpr int kDown = 14, kTop = 1, kLarge = 32, kTopLarge = 15;
template <bool F16> constexpr float kLowered = F16 ? 1.0f : 1.0f / (float)(1 << kDown);
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t add_f16(uint32_t x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, x) + f16x2{(_Float16)y, (_Float16)y});
}
// codes of a word as fp16, k: c + kBias, v: c - kCentre; with 4 bits in the order 0 4 1 5 2 6 3 7 (q's values are put in it beforehand, the
// result's out of it afterwards)
template <int BITS, bool V> __device__ __forceinline__ void widen(uint32_t w, uint32_t* to) {
    if constexpr (BITS == 8) {
        to[0] = __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u);
        to[1] = __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u);
        if constexpr (V) {
            to[0] = add_f16(to[0], -1152.0f);
            to[1] = add_f16(to[1], -1152.0f);
        }
    } else {
        // 1024 + c where a code lies in the last bits of a half, 64 + c four bits further up
        const uint32_t u = w >> 8;
        uint32_t x[4] = {(w & 0x000F000Fu) | 0x64006400u, (w & 0x00F000F0u) | 0x54005400u, (u & 0x000F000Fu) | 0x64006400u, (u & 0x00F000F0u) | 0x54005400u};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (V) x[i] = add_f16(x[i], i & 1 ? -72.0f : -1032.0f);
            else if (!(i & 1)) x[i] = add_f16(x[i], -960.0f);
            to[i] = x[i];
        }
    }
}

// four sums of a row in each half of the wavefront, out of the order of 4 bits
__device__ __forceinline__ f32x4 in_order(const f32x4& v) {
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v[0]), __float_as_uint(v[1]), false, false));
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v[2]), __float_as_uint(v[3]), false, false));
    return f32x4{__uint_as_float(a[0]), __uint_as_float(b[0]), __uint_as_float(a[1]), __uint_as_float(b[1])};
}

// bytes that a thread loads at a time, as words
template <int N> __device__ __forceinline__ void load_bytes(const uint8_t* p, uint32_t (&w)[N]) {
    if constexpr (N == 4) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = x[i];
    } else {
        static_assert(N == 2, "a thread's part of a tile");
        const u32x2 x = *reinterpret_cast<const u32x2*>(p);
        w[0] = x[0];
        w[1] = x[1];
    }
}

// two weights for the matrix cores, the first in the low half
template <bool F16> __device__ __forceinline__ uint32_t pack(float a, float b) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    if constexpr (F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), f16x2));
    else return f32x2_to_h16x2<false>(a, b);
}

// (what is seldom so is kept out of the way: copies of sums that the compiler puts around a branch go into it)
__device__ __forceinline__ bool seldom(bool x) { return __builtin_expect(x, 0); }

// the other half of the wavefront's
__device__ __forceinline__ float other_half(float v) {
    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return __uint_as_float((threadIdx.x & 32) ? x[0] : x[1]);
}

template <int SOURCE, int D, bool F16>
__global__ __launch_bounds__(kThreads, 2) void attn_chunk_kernel(Args a) {
    using T = Tile<D, kWaves>;
    constexpr bool CODES = SOURCE == 8 || SOURCE == 4, PAGED = SOURCE != kRows, CUTS = PAGED, MMA16 = F16 || CODES;
    constexpr int QM = D / 16, OM = D / 32;
    // LDS: two tiles of k, two of v; per tile either rows of v that are not finite (16 bits a wavefront), or the tokens' scales, the largest, and whose are not finite
    constexpr uint32_t kAside = 4 * T::kBytes, kAsideBytes = CODES ? kScaleBytes<kKeys> : 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, g = lane >> 5;

    // KV heads fastest: blocks that read the same keys tend to share an XCD and its L2
    const unsigned block = a.first_block + blockIdx.x, place = block / (unsigned)a.kv_heads, kv_head = block - place * (unsigned)a.kv_heads;
    const Work w = work_of<SOURCE>(a, place, kv_head, lane);
    if (w.request < 0) return;
    const int lq = w.r.lq, lk = w.r.lk, rows = lq * a.shared, ahead = lk - lq;
    const Span span = span_of(a, w.r, w.tile, w.height);
    const int each = CUTS ? (span.tiles + w.pieces - 1) / w.pieces : span.tiles;
    const int t_first = CUTS ? w.piece * each : 0, t_end = min(span.tiles, t_first + each);
    const bool in_pieces = CUTS && w.pieces > 1;
    if (in_pieces) {
        const int at = w.join * a.kv_heads + (int)kv_head;
        if (w.piece == 0 && threadIdx.x == 0 && at < a.cut_tiles)
            reinterpret_cast<Join*>(a.joins)[1 + at] = Join{w.r.q_at, rows, w.tile * w.height, w.height, each > 0 ? (span.tiles + each - 1) / each : 0, w.slot, {0, 0}};
        if (t_first >= t_end) return;                           // (the join knows)
    }

    // Up to 32 rows: each wavefront takes all of them and every fourth 32 keys, otherwise 32 rows and all keys.
    const bool narrow = w.height == 32 || rows - w.tile * kRowTile <= 32;
    const int row0 = w.tile * w.height + (narrow ? 0 : 32 * wave), row = min(row0 + n, rows - 1);
    const bool active = row0 < rows;
    const int query = a.query_of(row);
    // this row sees keys up to `lim` that lie in its window or are among the first `sinks`
    const int lim = ahead + query;
    // all rows see keys up to `all_lim` that lie at `all_lo` or behind it or are among the first
    const int all_lim = ahead + span.first, all_lo = max(ahead + span.last, 0) + 1 - a.window;

    // Q^T, fp16 for codes: a row of bf16 is scaled by a power of two into fp16's range
    u32x4 q[QM];
    float scale = a.scale_log2, sum_q = 0.0f;
    {
        const int head = (int)kv_head * a.shared + (row - query * a.shared);
        const uint16_t* qp = a.q.p + (int64_t)(w.r.q_at + query) * a.q.token + (int64_t)head * a.q.head;
        // places 16 i + 8 g .. of product i, or, with codes in narrow tiles, those that a lane's 16 bytes of k hold one after the other
        constexpr int kEach = SOURCE == 4 ? 4 : 2;
#pragma unroll
        for (int i = 0; i < QM; ++i) {
            const int at = CODES && narrow ? 16 * kEach * (i / kEach) + 8 * kEach * g + 8 * (i % kEach) : 16 * i + 8 * g;
            q[i] = *reinterpret_cast<const u32x4*>(qp + at);
        }
        if constexpr (CODES) {
            if constexpr (!F16) {
                float top = 0.0f;
#pragma unroll
                for (int i = 0; i < QM; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) top = fmaxf(top, fmaxf(fabsf(bf16lo_to_f32(q[i][j])), fabsf(bf16hi_to_f32(q[i][j]))));
                top = fmaxf(top, other_half(top));
                const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, -126), 127), of_scale = (int)(__float_as_uint(scale) >> 23) - 127;
                const int less = e - (e + of_scale < kLarge ? kTop : kTopLarge);
                const float by = __builtin_ldexpf(1.0f, -less);
                scale = __builtin_ldexpf(scale, less + kDown);
#pragma unroll
                for (int i = 0; i < QM; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) q[i][j] = pack<true>(bf16lo_to_f32(q[i][j]) * by, bf16hi_to_f32(q[i][j]) * by);
            }
#pragma unroll
            for (int i = 0; i < QM; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum_q += h16lo_to_f32<true>(q[i][j]) + h16hi_to_f32<true>(q[i][j]);
            sum_q += other_half(sum_q);
            if constexpr (SOURCE == 4) {
#pragma unroll
                for (int i = 0; i < QM; ++i) {
                    const u32x4 r = q[i];
                    q[i] = u32x4{__builtin_amdgcn_perm(r[2], r[0], 0x05040100u), __builtin_amdgcn_perm(r[2], r[0], 0x07060302u),
                                 __builtin_amdgcn_perm(r[3], r[1], 0x05040100u), __builtin_amdgcn_perm(r[3], r[1], 0x07060302u)};
                }
            }
        }
    }

    // Pages of a tile: lane 0 .. 3's of 16 tokens each (the last token's again behind it).
    const int page_mask = PAGED ? (1 << a.c.page_shift) - 1 : 0;
    const int32_t* table = PAGED ? a.table + (int64_t)w.request * a.table_stride : nullptr;
    auto pages_of = [&](int t) -> int {
        if constexpr (PAGED) return table[min(span.real(t) * kKeys + 16 * (lane & 3), lk - 1) >> a.c.page_shift];
        else return 0;
    };
    // a page that does not exist has no tokens: the first one is read in its place and masked
    auto there = [&](int page) -> bool { return !PAGED || (page >= 0 && page < a.c.pages); };
    auto valid_of = [&](int page) -> unsigned { return (unsigned)__builtin_amdgcn_ballot_w64(there(page)) & 15u; };

    // 16 bits.  Copies: lane -> row and piece of each instruction; LDS has piece c of row r at c ^ swizzle(r).
    const int copy_row = T::kCopies * T::kRows * wave + lane / T::kPieces, copy_piece = lane % T::kPieces;
    const uint32_t k_step = SOURCE == kRows ? (uint32_t)a.k.token * 2u : (uint32_t)T::kRow, v_step = SOURCE == kRows ? (uint32_t)a.v.token * 2u : (uint32_t)T::kRow;
    auto copy_tile = [&](int t, int page, uint32_t parity) {
        const int k0 = span.real(t) * kKeys;
        const char *kb, *vb;
        int first;                                              // the token that row 0's address would be of
        if constexpr (SOURCE == kRows) {
            first = k0;
            kb = reinterpret_cast<const char*>(a.k.p + (int64_t)w.r.k_at * a.k.token + (int64_t)kv_head * a.k.head) + (int64_t)k0 * k_step;
            vb = reinterpret_cast<const char*>(a.v.p + (int64_t)w.r.k_at * a.v.token + (int64_t)kv_head * a.v.head) + (int64_t)k0 * v_step;
        } else {
            // (a wavefront's 16 rows are one page's)
            static_assert(T::kCopies * T::kRows == 16, "a wavefront copies 16 rows");
            const int p = __builtin_amdgcn_readlane(there(page) ? page : 0, wave);
            const int tok = min(k0 + 16 * wave, lk - 1);
            const int64_t at = (a.c.first_token(p, (int)kv_head) + (tok & page_mask)) * T::kRow;
            kb = reinterpret_cast<const char*>(a.c.k) + at;
            vb = reinterpret_cast<const char*>(a.c.v) + at;
            first = tok;
        }
#pragma unroll
        for (int j = 0; j < T::kCopies; ++j) {
            const int r = copy_row + j * T::kRows, base = SOURCE == kRows ? 0 : 16 * wave;
            // (rows past the last are copies of it; they are masked)
            const uint32_t from = (uint32_t)min(r - base, lk - 1 - first);
            const uint32_t to = parity * T::kBytes + (uint32_t)(T::kCopies * wave + j) * 1024u;
            copy_to_lds(to, kb, from * k_step + 16u * (uint32_t)(copy_piece ^ T::swizzle_k(r)));
            copy_to_lds(to + 2 * T::kBytes, vb, from * v_step + 16u * (uint32_t)(copy_piece ^ swizzle_v<D>(r)));
        }
    };
    // which of this wavefront's 16 rows of a tile of v are not finite
    auto look_at_v = [&](uint32_t parity) {
        constexpr uint32_t kExp = F16 ? 0x7C007C00u : 0x7F807F80u, kOne = F16 ? 0x04000400u : 0x00800080u;
        uint32_t bad = 0u;
#pragma unroll
        for (int j = 0; j < T::kCopies; ++j) {
            const u32x4 v = *(lds_u4)((2 + parity) * T::kBytes + (uint32_t)(T::kCopies * wave + j) * 1024u + 16u * (uint32_t)lane);
            uint32_t bits = 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) bits |= (v[i] & kExp) + kOne;               // (an exponent of all ones carries into the half's top bit)
            const unsigned long long lanes = __builtin_amdgcn_ballot_w64((bits & 0x80008000u) != 0u);
            if (lanes) {
#pragma unroll
                for (int r = 0; r < T::kRows; ++r)
                    bad |= ((lanes >> (r * T::kPieces)) & ((1ull << T::kPieces) - 1) ? 1u : 0u) << (j * T::kRows + r);
            }
        }
        if (lane == 0) *(lds_u1)(kAside + parity * kAsideBytes + 4u * (uint32_t)wave) = bad;
    };
    // Such rows are taken out of the tile, when all wavefronts have had what they need of them.
    auto take_out = [&](uint32_t parity, unsigned long long bad) {
        lds_barrier();
#pragma unroll
        for (int j = 0; j < T::kCopies; ++j)
            if ((bad >> (copy_row + j * T::kRows)) & 1ull)
                *(lds_u4)((2 + parity) * T::kBytes + (uint32_t)(T::kCopies * wave + j) * 1024u + 16u * (uint32_t)lane) = u32x4{0u, 0u, 0u, 0u};
        lds_barrier();
    };
    // tokens of a tile whose v is not finite (codes: whose scale or offset is not), where the tile was looked at
    auto bad_of_tile = [&](uint32_t parity) -> unsigned long long {
        unsigned long long bad = 0ull;
        if constexpr (CODES) {
            const u32x2 two = *(lds_u2)(kAside + parity * kAsideBytes + 20 * kKeys + 8);
            bad = (unsigned long long)two[1] << 32 | two[0];
        } else {
#pragma unroll
            for (int i = 0; i < kWaves; ++i) bad |= (unsigned long long)*(lds_u1)(kAside + parity * kAsideBytes + 4u * (uint32_t)i) << (16 * i);
        }
        return (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)bad) | (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(bad >> 32)) << 32;
    };

    // Codes: a thread's part of a tile, loaded two tiles ahead and widened into LDS one tile ahead.
    constexpr int kPart = CODES ? kKeys * D * SOURCE / 8 / kThreads : 16, kLoad = kPart < 16 ? kPart : 16, kPasses = kPart / kLoad;
    constexpr int kLanesRow = CODES ? D * SOURCE / 8 / kLoad : 1, kPassRows = kThreads / kLanesRow, kCodes = CODES ? kLoad * 8 / SOURCE : 8;
    struct Raw {
        uint32_t k[kPasses][kLoad / 4], v[kPasses][kLoad / 4];
        u32x2 scales;
    };
    Raw raw;
    auto load_raw = [&](int t, int page) {
        if constexpr (CODES) {
            const int k0 = span.real(t) * kKeys, pages = there(page) ? page : 0;
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                const int r = i * kPassRows + (int)threadIdx.x / kLanesRow, first = i * kPassRows + 64 / kLanesRow * wave;
                const int64_t at = a.c.first_token(__builtin_amdgcn_readlane(pages, first / 16), (int)kv_head) * (D * SOURCE / 8);
                const uint32_t off = (uint32_t)(min(k0 + r, lk - 1) & page_mask) * (D * SOURCE / 8) + (uint32_t)(threadIdx.x % kLanesRow) * kLoad;
                load_bytes(a.c.k + at + off, raw.k[i]);
                load_bytes(a.c.v + at + off, raw.v[i]);
            }
            if (wave == (t & (kWaves - 1))) {
                const int64_t at = a.c.first_token(__shfl(pages, lane >> 4), (int)kv_head) + (min(k0 + lane, lk - 1) & page_mask);
                raw.scales = *reinterpret_cast<const u32x2*>(a.c.scales + 4 * at);
            }
        }
    };
    // (the first row's first piece; the others' follow from it by an exclusive or and a constant)
    const int stage_row = (int)threadIdx.x / kLanesRow, stage_piece = (int)(threadIdx.x % kLanesRow) * (kCodes / 8);
    const uint32_t to_k = (uint32_t)(stage_row * T::kRow) + 16u * (uint32_t)(stage_piece ^ T::swizzle_k(stage_row));
    const uint32_t to_v = 2 * T::kBytes + (uint32_t)(stage_row * T::kRow) + 16u * (uint32_t)(stage_piece ^ swizzle_v<D>(stage_row));
    auto stage = [&](int t, uint32_t parity) {
        if constexpr (CODES) {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                uint32_t wide[kCodes / 2];
#pragma unroll
                for (int of_v = 0; of_v < 2; ++of_v) {
#pragma unroll
                    for (int x = 0; x < kLoad / 4; ++x) {
                        if (of_v) widen<CODES ? SOURCE : 8, true>(raw.v[i][x], wide + x * 16 / (CODES ? SOURCE : 8));
                        else widen<CODES ? SOURCE : 8, false>(raw.k[i][x], wide + x * 16 / (CODES ? SOURCE : 8));
                    }
#pragma unroll
                    for (int x = 0; x < kCodes / 8; ++x) {
                        const uint32_t other = 16u * (uint32_t)(x ^ (of_v ? swizzle_v<D>(i * kPassRows) : T::swizzle_k(i * kPassRows)));
                        *(lds_u4)((((of_v ? to_v : to_k) + parity * T::kBytes) ^ other) + (uint32_t)(i * kPassRows * T::kRow)) = u32x4{wide[4 * x], wide[4 * x + 1], wide[4 * x + 2], wide[4 * x + 3]};
                    }
                }
            }
            if (wave == (t & (kWaves - 1))) {
                using C = Codes<CODES ? SOURCE : 8>;
                const float ks = kLowered<F16> * bf16lo_to_f32(raw.scales[0]), ko = kLowered<F16> * bf16hi_to_f32(raw.scales[0]), vs = bf16lo_to_f32(raw.scales[1]), vo = bf16hi_to_f32(raw.scales[1]);
                const float mid = fmaf(C::kCentre, vs, vo);
                const bool fine = fabsf(mid) < __builtin_inff();   // (a v without numbers counts for nothing here; see below)
                const uint32_t aside = kAside + parity * kAsideBytes, to = aside + 4u * (uint32_t)lane;
                *(lds_f)(to) = ks;
                *(lds_f)(to + 256) = fmaf(-C::kBias, ks, ko);
                const float vs_used = fine ? vs : 0.0f, mid_used = fine ? mid : 0.0f, high = exponent_of(vs_used, mid_used);
                *(lds_f)(to + 512) = vs_used;
                *(lds_f)(to + 768) = mid_used;
                *(lds_f)(to + 1024) = high;
                const float big = lanes_largest<64>(high);
                const bool apart = __builtin_amdgcn_ballot_w64(vs_used != 0.0f && big - high > (float)kSpread) != 0ull;
                const unsigned long long bad = __builtin_amdgcn_ballot_w64(!fine);
                if (lane == 0) {
                    *(lds_u2)(aside + 20 * kKeys) = u32x2{__float_as_uint(big), apart ? 1u : 0u};
                    *(lds_u2)(aside + 20 * kKeys + 8) = u32x2{(uint32_t)bad, (uint32_t)(bad >> 32)};
                }
            }
        }
    };

    // operand addresses within a tile: the swizzles are exclusive ors, so that pieces further along the head are the first one's with two or four
    // times 16 bytes put in the same way
    const int i16 = lane & 15, v_row = 4 * g + (i16 >> 2);
    const uint32_t k_lane = (uint32_t)(n * T::kRow + ((g ^ T::swizzle_k(n)) << 4));
    const uint32_t v_lane = (uint32_t)(v_row * T::kRow + 8 * (i16 & 1) + (((2 * ((lane >> 4) & 1) + ((i16 >> 1) & 1)) ^ swizzle_v<D>(v_row)) << 4));
    auto v_operand = [&](uint32_t first, int c, int m) -> u32x4 {
        const uint32_t at = (first ^ (uint32_t)(m << 6)) + (uint32_t)(c * 16 * T::kRow);
        const u32x2 lo = lds_read_transposed(at), hi = lds_read_transposed(at + 8 * T::kRow);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    };

    float m_ref = -__builtin_inff(), l = 0.0f, v_sum = 0.0f;
    float exponent = 0.0f;                                      // codes: of the largest product of a weight exp2(s - m_ref) and vs, a whole number
    float m_used = 0.0f;                                        // what is taken off the scores: maximum and exponent
    int far = 0, folds = 0;                                     // whether that is so for some row
    f32x16 o[OM];
#pragma unroll
    for (int m = 0; m < OM; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[m][r] = 0.0f;

    // k's operands out of a tile in LDS
    auto k_of = [&](uint32_t buf) {
        uint32_t at = k_lane + buf;
        asm volatile("" : "+v"(at));
        return [at](int u, int i) -> u32x4 { return *(lds_u4)((at ^ (uint32_t)(i << 5)) + (uint32_t)(u * 32 * T::kRow)); };
    };
    // 32 U keys from k0 on, whose v and scales lie in LDS; `whole`: all rows see all of them; valid: a bit for each 16 whose page exists.  The
    // steps: after_scores, before_product (v has to be there then), bad_of the keys whose v is not finite, take_out of them.
    auto attend = [&](auto blocks, int k0, auto k_operand, uint32_t v_buf, uint32_t scales, unsigned valid, bool whole, auto after_scores, auto before_product,
                      auto bad_of, auto take_out) {
        constexpr int U = decltype(blocks)::value;
        // four tokens' of an array of scales: keys 32 u + 8 c + 4 g ..
        auto four_of = [&](int array, int u, int c) -> f32x4 { return *(lds_f4)(scales + (uint32_t)(128 * U * array + 4 * (32 * u + 8 * c)) + 16u * (uint32_t)g); };
        // The two wavefronts of a SIMD take turns at its matrix cores and its vector units: one that turns scores into weights goes first, so that its
        // products come while the other is at its scores or weights.  (2048 tokens behind 30 k in 16 bits 1063 -> 1004 us, with the priority until behind
        // the product 1030; a mixed batch in 8 bits 451 and 434 the other way round.  Heads of 64 have a third wavefront and lose 4 % by it.)
        constexpr bool kFirst = D == 128;
        f32x16 s[U];
        uint32_t v_at = v_lane + v_buf;
        asm volatile("" : "+v"(v_at));                           // (or every operand's address is kept in a register)
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[u][r] = 0.0f;
#pragma unroll
            for (int i = 0; i < QM; ++i) {
                s[u] = mma32<MMA16>(k_operand(u, i), q[i], s[u]);
            }
        }
        if constexpr (kFirst) __builtin_amdgcn_s_setprio(1);
        if constexpr (CODES) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const f32x4 ks = four_of(0, u, c), ko = four_of(1, u, c);
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[u][4 * c + r] = fmaf(ks[r], s[u][4 * c + r], ko[r] * sum_q);
                }
        }
        after_scores();
        u32x2 of_all = {0u, 0u};                                 // codes: the largest exponent of the scales, whether they lie far apart
        if constexpr (CODES) of_all = *(lds_u2)(scales + 640 * U);
        // (places relative to the tile's first key of this half, which may be those of no page)
        const int base = k0 + 4 * g, lim_at = lim - base, lo_at = (max(lim, 0) + 1 - base) - a.window, sinks_at = a.sinks - base;
        auto key_of = [](int u, int r) -> int { return 32 * u + 8 * (r >> 2) + (r & 3); };
        auto last_of = [&](int u, int r) -> int { return !PAGED || ((valid >> (2 * u + (r >> 3))) & 1u) ? lim_at : -0x7FFFFFFF; };
        auto in_part = [&](int u, int r) -> bool { return (bool)((int)(key_of(u, r) >= lo_at) | (int)(key_of(u, r) < sinks_at)); };
        if (seldom(!whole)) {
            // (behind the last one or on a page that does not exist; in front of the window)
            if (k0 + 32 * U - 1 > all_lim || valid != (1u << 2 * U) - 1u) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[u][r] = key_of(u, r) <= last_of(u, r) ? s[u][r] : -__builtin_inff();
            }
            if (k0 < all_lo && k0 + 32 * U > a.sinks) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[u][r] = in_part(u, r) ? s[u][r] : -__builtin_inff();
            }
        }

        // The maximum in use is raised only when a score exceeds it by 2^kSlack, which spares nearly all rescaling of o.
        float top = s[0][0];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[u][r]);
        top = fmaxf(top, other_half(top)) * scale;
        bool moved = top > m_ref + kSlack;
        const float higher = fmaxf(m_ref, top);
        float product = 0.0f;                                    // codes: exponent of the largest product of this step, less `higher`
        if constexpr (CODES) {
            // (a large scale alone is none: its token may have a weight of nothing, and the others' products are not to vanish beside a product that is none)
            product = difference(top, higher) + __uint_as_float(of_all[0]);
            if (seldom((int)!whole | __builtin_amdgcn_readfirstlane((int)of_all[1]))) {
                product = -__builtin_inff();
                float by = scale;
                asm volatile("" : "+v"(by));                     // (or these products and those of far scores are made in front of both branches)
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const f32x4 high = four_of(4, u, c);
#pragma unroll
                        for (int r = 0; r < 4; ++r) product = fmaxf(product, difference(s[u][4 * c + r] * by, higher) + high[r]);
                    }
                product = fmaxf(product, other_half(product));
            }
            moved |= product + (higher - m_ref) > exponent + kSlack;
        }
        // A weight's exponent is scale s - m_sub: a product that is not rounded, less a maximum that is.  Beyond 2^31 that rounding alone would leave
        // the exponents' range: where some row's maximum lies beyond kFar, the scores are replaced by their distance from it, both rounded alike.
        // (All that follows from the maximum and the exponent is set here: set after the branch, the compiler has the sums copied around it.)
        if (seldom(__builtin_amdgcn_ballot_w64(moved) != 0ull)) {
            const float m_new = moved ? higher : m_ref;
            if constexpr (CODES) {
                // (sums are relative to m_used, o to that and what is taken off the products; without a score yet they are zeros)
                const float before = m_ref == -__builtin_inff() ? m_ref : m_used;
                const int was = folded(m_ref, exponent);
                exponent = moved ? fmaxf(fmaxf(floorf(exponent + (m_ref - m_new)), ceilf(product)), -300.0f) : exponent;   // (down, or it would rise with every move)
                m_used = (m_new == -__builtin_inff() ? 0.0f : m_new) + with_maximum(m_new, exponent);
                const float less = before - m_used, alpha = exp2_fast(less);
                l *= alpha;
                v_sum *= alpha;
                const int is = folded(m_new, exponent);
                const float f = exp2_fast(less + (float)(was - is));
#pragma unroll
                for (int m = 0; m < OM; ++m) o[m] *= f;
                folds = __builtin_amdgcn_ballot_w64(is != 0) != 0ull ? 1 : 0;
            } else {
                const float alpha = exp2_fast(m_new > m_ref ? m_ref - m_new : 0.0f);
                l *= alpha;
#pragma unroll
                for (int m = 0; m < OM; ++m) o[m] *= alpha;
                m_used = m_new == -__builtin_inff() ? 0.0f : m_new;
            }
            m_ref = m_new;
            far = __builtin_amdgcn_ballot_w64(fabsf(m_used) > kFar) != 0ull ? 1 : 0;
        }
        float m_sub = m_used;
        if (seldom(far != 0)) {
            const float back = 1.0f / scale;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
#pragma clang fp contract(off)
                    const float scaled = s[u][r] * scale;
                    s[u][r] = (scaled - m_sub) * back;
                }
            m_sub = 0.0f;
        }

        u32x4 p[2 * U];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                f32x4 e;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    e[r] = exp2_fast(fmaf(s[u][4 * c + r], scale, -m_sub));
                    l += e[r];
                }
                if constexpr (CODES) {
                    const f32x4 vs = four_of(2, u, c), vo = four_of(3, u, c);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        v_sum = fmaf(e[r], vo[r], v_sum);
                        s[u][4 * c + r] = e[r] * vs[r];
                    }
                } else {
                    p[2 * u + (c >> 1)][2 * (c & 1)] = pack<MMA16>(e[0], e[1]);
                    p[2 * u + (c >> 1)][2 * (c & 1) + 1] = pack<MMA16>(e[2], e[3]);
                }
            }
        if constexpr (CODES) {
            // (off the products: a scale alone may lie further from the largest product than fp32 reaches)
            if (seldom(folds != 0)) {
                const int less = -folded(m_ref, exponent);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[u][r] = __builtin_ldexpf(s[u][r], less);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int x = 0; x < 8; ++x) p[2 * u + (x >> 2)][x & 3] = pack<MMA16>(s[u][2 * x], s[u][2 * x + 1]);
        }

        // 0 times what is not finite would be NaN: tokens with such a v (in tiles that not all rows see, with codes in all) are added one by one to
        // the rows that see them, and are zeros in the product.
        before_product();
        if (CODES || !whole) {
            const unsigned long long bad = bad_of();
            if (seldom(bad != 0ull)) {
#pragma unroll 1
                for (unsigned long long left = bad; left; left &= left - 1) {
                    const int key = __builtin_ctzll(left), at = k0 + key;
                    const bool seen = at <= lim && (at >= max(lim, 0) + 1 - a.window || at < a.sinks) && (!PAGED || ((valid >> (key >> 4)) & 1u));
                    if constexpr (CODES) {
                        if (seen) v_sum = __builtin_nanf("");
                    } else {
                        const int c = key >> 4, half = (key >> 2) & 1, slot = (key & 3) | ((key >> 1) & 4);
                        uint32_t pair = 0u;
#pragma unroll
                        for (int x = 0; x < 8 * U; ++x) pair = x == 4 * c + (slot >> 1) ? p[x >> 2][x & 3] : pair;
                        const float mine = slot & 1 ? h16hi_to_f32<MMA16>(pair) : h16lo_to_f32<MMA16>(pair), other = other_half(mine);
                        const float weight = g == half ? mine : other;
#pragma unroll
                        for (int m = 0; m < OM; ++m)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const uint32_t piece = (uint32_t)((4 * m + r) ^ swizzle_v<D>(key));
                                const u32x2 v = *(lds_u2)(v_buf + (uint32_t)(key * T::kRow) + 16u * piece + 8u * (uint32_t)g);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const float x = e & 1 ? h16hi_to_f32<F16>(v[e >> 1]) : h16lo_to_f32<F16>(v[e >> 1]);
                                    o[m][4 * r + e] = seen ? fmaf(weight, x, o[m][4 * r + e]) : o[m][4 * r + e];
                                }
                            }
                    }
                }
                if constexpr (!CODES) take_out(bad);
            }
        }
        if constexpr (kFirst && !CODES) __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int c = 0; c < 2 * U; ++c)
#pragma unroll
            for (int m = 0; m < OM; ++m) o[m] = mma32<MMA16>(v_operand(v_at, c, m), p[c], o[m]);
        if constexpr (kFirst && CODES) __builtin_amdgcn_s_setprio(0);
    };

    auto wide_rows = [&] {
        // `page` is that of the tile whose loads go out next: the next tile's, with codes the one behind it.
        int page = 0;
        unsigned valid = 15u, valid_next = 15u;                     // of tiles t and t + 1
        if (t_first < t_end) {
            page = pages_of(t_first);
            valid = valid_of(page);
            if constexpr (CODES) {
                load_raw(t_first, page);
                stage(t_first, t_first & 1);
                if (t_first + 1 < t_end) {
                    page = pages_of(t_first + 1);
                    valid_next = valid_of(page);
                    load_raw(t_first + 1, page);
                    if (t_first + 2 < t_end) page = pages_of(t_first + 2);
                }
            } else {
                copy_tile(t_first, page, t_first & 1);
                if (t_first + 1 < t_end) page = pages_of(t_first + 1);
            }
        }
        // up to where tile t is there and the loads for those behind it are on their way; whether all rows see all of it
        auto begin = [&](int t, uint32_t parity, unsigned& valid_after) -> bool {
            const int k0 = span.real(t) * kKeys;
            const bool whole = k0 + kKeys - 1 <= all_lim && (k0 >= all_lo || k0 + kKeys <= a.sinks) && valid == 15u;
            if constexpr (!CODES) {
                loads_left<0>();
                if (!whole) look_at_v(parity);
            }
            lds_barrier();                                          // (and nobody reads the one in front of it any more)
            if constexpr (CODES) {
                if (t + 1 < t_end) stage(t + 1, parity ^ 1u);
                if (t + 2 < t_end) {
                    valid_after = valid_of(page);
                    load_raw(t + 2, page);
                    if (t + 3 < t_end) page = pages_of(t + 3);
                }
            } else if (t + 1 < t_end) {
                valid_next = valid_of(page);
                copy_tile(t + 1, page, parity ^ 1u);
                if (t + 2 < t_end) page = pages_of(t + 2);
            }
            return whole;
        };
        // (a loop of their own for wavefronts without rows: a branch around the sums would have them copied in every round)
        if (active) {
#pragma unroll 1
            for (int t = t_first; t < t_end; ++t) {
                const uint32_t parity = (uint32_t)(t & 1);
                unsigned valid_after = 15u;
                const bool whole = begin(t, parity, valid_after);
                attend(std::integral_constant<int, 2>{}, span.real(t) * kKeys, k_of(parity * T::kBytes), (2 + parity) * T::kBytes, kAside + parity * kAsideBytes, valid,
                       whole, [] {}, [] {}, [&] { return bad_of_tile(parity); }, [&](unsigned long long bad) { take_out(parity, bad); });
                valid = valid_next;
                valid_next = valid_after;
            }
        } else {
#pragma unroll 1
            for (int t = t_first; t < t_end; ++t) {
                const uint32_t parity = (uint32_t)(t & 1);
                unsigned valid_after = 15u;
                const bool whole = begin(t, parity, valid_after);
                if (!CODES && !whole) {
                    if (const unsigned long long bad = bad_of_tile(parity)) take_out(parity, bad);
                }
                valid = valid_next;
                valid_next = valid_after;
            }
        }
    };

    // Up to 32 rows.  A wavefront's own part of LDS: 32 keys of k, 32 of v; k's next 32 are on their way while v's are used, and the other way round.
    auto narrow_rows = [&] {
        constexpr uint32_t kHalf = 32 * T::kRow, kCopies = kHalf / 1024;
        const uint32_t k_buf = (uint32_t)wave * 2 * kHalf, v_buf = k_buf + kHalf, scales = kAside + (uint32_t)wave * kScaleBytes<32>;
        const int h_end = 2 * t_end - (t_end > t_first && span.real(t_end - 1) * kKeys + 32 >= span.end ? 1 : 0);
        auto key_of = [&](int h) -> int { return span.real(h >> 1) * kKeys + 32 * (h & 1); };
        // the pages of its two 16 tokens
        struct Two {
            int page[2];
        };
        auto pages_of_half = [&](int h) -> Two {
            Two two{{0, 0}};
            if constexpr (PAGED) {
                // codes: loads of the lanes' (a scalar load would be waited for at the next wait for LDS); 16 bits: scalar ones (the others' wait would
                // be one for the copies that the compiler does not see)
                const auto entries = (const __attribute__((address_space(4))) int32_t*)reinterpret_cast<uintptr_t>(table);
                const int k0 = key_of(h);
                int zero = 0;
                if constexpr (CODES) asm volatile("" : "+v"(zero));
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int at = min(k0 + 16 * i, lk - 1) >> a.c.page_shift;
                    two.page[i] = CODES ? table[at + zero] : entries[at];
                }
            }
            return two;
        };
        auto page_of = [&](const Two& two, int i) -> int { return CODES ? __builtin_amdgcn_readfirstlane(two.page[i]) : two.page[i]; };
        auto valid_of_half = [&](const Two& two) -> unsigned { return (there(page_of(two, 0)) ? 1u : 0u) | (there(page_of(two, 1)) ? 2u : 0u); };
        auto first_of = [&](const Two& two, int i) -> int64_t {
            const int page = page_of(two, i);
            return PAGED ? a.c.first_token(there(page) ? page : 0, (int)kv_head) : 0;
        };

        // 16 bits: 64 lanes copy kRows rows at a time
        auto copy_half = [&](int h, const Two& two, bool of_v) {
            const int k0 = key_of(h);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // (what is read from there has been read)
#pragma unroll
            for (int j = 0; j < (int)kCopies; ++j) {
                const int first = j * T::kRows, r = first + lane / T::kPieces, i = first / 16;
                const int tok = min(k0 + r, lk - 1);
                const uint32_t piece = 16u * (uint32_t)(copy_piece ^ (of_v ? swizzle_v<D>(r) : T::swizzle_k(r)));
                const uint32_t to = (of_v ? v_buf : k_buf) + 1024u * (uint32_t)j;
                if constexpr (SOURCE == kRows) {
                    const Rows& rows_of = of_v ? a.v : a.k;
                    const uint32_t step = of_v ? v_step : k_step;
                    const char* base = reinterpret_cast<const char*>(rows_of.p + (int64_t)w.r.k_at * rows_of.token + (int64_t)kv_head * rows_of.head) + (int64_t)k0 * step;
                    copy_to_lds(to, base, (uint32_t)(tok - k0) * step + piece);
                } else {
                    const char* base = reinterpret_cast<const char*>(of_v ? a.c.v : a.c.k) + first_of(two, i) * T::kRow;
                    copy_to_lds(to, base, (uint32_t)(tok & page_mask) * (uint32_t)T::kRow + piece);
                }
            }
        };
        auto bad_of_half = [&]() -> unsigned long long {
            constexpr uint32_t kExp = F16 ? 0x7C007C00u : 0x7F807F80u, kOne = F16 ? 0x04000400u : 0x00800080u;
            unsigned long long bad = 0ull;
#pragma unroll 1
            for (int j = 0; j < (int)kCopies; ++j) {
                const u32x4 v = *(lds_u4)(v_buf + 1024u * (uint32_t)j + 16u * (uint32_t)lane);
                uint32_t bits = 0u;
#pragma unroll
                for (int i = 0; i < 4; ++i) bits |= (v[i] & kExp) + kOne;
                const unsigned long long lanes = __builtin_amdgcn_ballot_w64((bits & 0x80008000u) != 0u);
                if (lanes) {
#pragma unroll
                    for (int r = 0; r < T::kRows; ++r) bad |= ((lanes >> (r * T::kPieces)) & ((1ull << T::kPieces) - 1) ? 1ull : 0ull) << (j * T::kRows + r);
                }
            }
            return bad;
        };
        auto take_out_of_half = [&](unsigned long long bad) {
#pragma unroll 1
            for (int j = 0; j < (int)kCopies; ++j)
                if ((bad >> (j * T::kRows + lane / T::kPieces)) & 1ull) *(lds_u4)(v_buf + 1024u * (uint32_t)j + 16u * (uint32_t)lane) = u32x4{0u, 0u, 0u, 0u};
        };

        // codes: 16 bytes a lane at a time; k's as operands, without LDS (a lane has its token's every second 16 bytes), v's into LDS
        constexpr int kRowBytes = CODES ? D * SOURCE / 8 : 64, kRowLanes = kRowBytes / 16, kLoads = 32 / (64 / kRowLanes), kRowsAtOnce = 64 / kRowLanes;
        constexpr int kPer = CODES ? 16 * 8 / SOURCE : 8;          // codes of a load
        uint32_t raw_k[kLoads][4], raw_v[kLoads][4];
        u32x2 raw_scales = {0u, 0u};
        auto load_k = [&](int h, const Two& two) {
            const int64_t first = n < 16 ? first_of(two, 0) : first_of(two, 1);
            const uint8_t* p = a.c.k + (first + (min(key_of(h) + n, lk - 1) & page_mask)) * kRowBytes + 16 * g;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) load_bytes(p + 32 * i, raw_k[i]);
        };
        auto k_raw = [&](int, int i) -> u32x4 {
            constexpr int BITS = CODES ? SOURCE : 8, kWords = 8 * BITS / 32;
            uint32_t wide[4];
#pragma unroll
            for (int x = 0; x < kWords; ++x) widen<BITS, false>(raw_k[i * kWords / 4][i * kWords % 4 + x], wide + x * 16 / BITS);
            return u32x4{wide[0], wide[1], wide[2], wide[3]};
        };
        auto load_v = [&](int h, const Two& two) {
            const int k0 = key_of(h);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int r = i * kRowsAtOnce + lane / kRowLanes;
                const int64_t first = (kRowsAtOnce <= 16 ? (i * kRowsAtOnce < 16) : r < 16) ? first_of(two, 0) : first_of(two, 1);
                load_bytes(a.c.v + (first + (min(k0 + r, lk - 1) & page_mask)) * kRowBytes + 16 * (lane % kRowLanes), raw_v[i]);
            }
            if (lane < 32) raw_scales = *reinterpret_cast<const u32x2*>(a.c.scales + 4 * ((lane < 16 ? first_of(two, 0) : first_of(two, 1)) + (min(k0 + lane, lk - 1) & page_mask)));
        };
        auto stage_v = [&] {
            constexpr int BITS = CODES ? SOURCE : 8;
            // (the first row's first piece; a register of its own in each round, as the others' would be if they were kept)
            const int r0 = lane / kRowLanes, piece0 = (lane % kRowLanes) * (kPer / 8);
            uint32_t to = v_buf + (uint32_t)(r0 * T::kRow) + 16u * (uint32_t)(piece0 ^ swizzle_v<D>(r0));
            asm volatile("" : "+v"(to));
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                uint32_t wide[kPer / 2];
#pragma unroll
                for (int x = 0; x < 4; ++x) widen<BITS, true>(raw_v[i][x], wide + x * 16 / BITS);
#pragma unroll
                for (int x = 0; x < kPer / 8; ++x) {
                    const uint32_t other = 16u * (uint32_t)(x ^ swizzle_v<D>(i * kRowsAtOnce));
                    *(lds_u4)((to ^ other) + (uint32_t)(i * kRowsAtOnce * T::kRow)) = u32x4{wide[4 * x], wide[4 * x + 1], wide[4 * x + 2], wide[4 * x + 3]};
                }
            }
            using C = Codes<BITS>;
            const float ks = kLowered<F16> * bf16lo_to_f32(raw_scales[0]), ko = kLowered<F16> * bf16hi_to_f32(raw_scales[0]), vs = bf16lo_to_f32(raw_scales[1]), vo = bf16hi_to_f32(raw_scales[1]);
            const float mid = fmaf(C::kCentre, vs, vo);
            const bool fine = fabsf(mid) < __builtin_inff();
            const float vs_used = fine ? vs : 0.0f, mid_used = fine ? mid : 0.0f, high = exponent_of(vs_used, mid_used);
            if (lane < 32) {
                const uint32_t at = scales + 4u * (uint32_t)lane;
                *(lds_f)(at) = ks;
                *(lds_f)(at + 128) = fmaf(-C::kBias, ks, ko);
                *(lds_f)(at + 256) = vs_used;
                *(lds_f)(at + 384) = mid_used;
                *(lds_f)(at + 512) = high;
            }
            // (lanes from 32 on have no tokens: scales of 0)
            const float big = lanes_largest<32>(high);
            const bool apart = __builtin_amdgcn_ballot_w64(vs_used != 0.0f && big - high > (float)kSpread) != 0ull;
            const unsigned long long bad = __builtin_amdgcn_ballot_w64(!fine && lane < 32);
            if (lane == 0) {
                *(lds_u2)(scales + 640) = u32x2{__float_as_uint(big), apart ? 1u : 0u};
                *(lds_u2)(scales + 648) = u32x2{(uint32_t)bad, 0u};
            }
        };

        int h = 2 * t_first + wave;
        // pages of the half whose loads go out next (codes: k's), and of the one behind it (codes: v's)
        Two two{{0, 0}}, two_next{{0, 0}}, two_after{{0, 0}};
        unsigned valid = 3u, valid_next = 3u;
        if (h < h_end) {
            two = pages_of_half(h);
            valid = valid_of_half(two);
            if constexpr (CODES) {
                load_v(h, two);
                load_k(h, two);
                if (h + kWaves < h_end) two = pages_of_half(h + kWaves);
                if (h + 2 * kWaves < h_end) two_next = pages_of_half(h + 2 * kWaves);
                stage_v();
                if (h + kWaves < h_end) {
                    valid_next = valid_of_half(two);
                    load_v(h + kWaves, two);
                }
            } else {
                copy_half(h, two, false);
                copy_half(h, two, true);
                if (h + kWaves < h_end) two = pages_of_half(h + kWaves);
            }
        }
#pragma unroll 1
        for (; h < h_end; h += kWaves) {
            const int next = h + kWaves, after = h + 2 * kWaves, k0 = key_of(h);
            const bool whole = k0 + 31 <= all_lim && (k0 >= all_lo || k0 + 32 <= a.sinks) && valid == 3u;
            unsigned valid_after = 3u;
            if constexpr (CODES) {
                if (after + kWaves < h_end) two_after = pages_of_half(after + kWaves);
                attend(std::integral_constant<int, 1>{}, k0, k_raw, v_buf, scales, valid, whole,
                       [&] {
                           if (next < h_end) load_k(next, two);
                       },
                       [] {},
                       [&]() -> unsigned long long { return (unsigned)__builtin_amdgcn_readfirstlane((int)*(lds_u1)(scales + 648)); }, [](unsigned long long) {});
                if (next < h_end) stage_v();
                if (after < h_end) {
                    valid_after = valid_of_half(two_next);
                    load_v(after, two_next);
                }
                two = two_next;
                two_next = two_after;
            } else {
                if (next < h_end) valid_next = valid_of_half(two);
                loads_left<(int)kCopies>();                         // k is there; v's copies may be on their way
                attend(std::integral_constant<int, 1>{}, k0, k_of(k_buf), v_buf, scales, valid, whole,
                       [&] {
                           if (next < h_end) copy_half(next, two, false);
                           if (after < h_end) two_next = pages_of_half(after);
                       },
                       [&] {
                           if (next < h_end) loads_left<(int)kCopies>();
                           else loads_left<0>();
                       },
                       bad_of_half, take_out_of_half);
                if (next < h_end) copy_half(next, two, true);
                two = two_next;
            }
            valid = valid_next;
            valid_next = valid_after;
        }
    };

    if (narrow) narrow_rows();
    else wide_rows();
    if (!active) return;                                        // (of a narrow tile all are)

    // (the lane's number anew: what follows from it is not to take registers from the loop above)
    int thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    const int n_e = thread & 31, g_e = (thread >> 5) & 1;

    l += other_half(l);
    if constexpr (CODES) {
        v_sum += other_half(v_sum);
        if (seldom(folds != 0)) {
            const int unfold = folded(m_ref, exponent);
#pragma unroll
            for (int m = 0; m < OM; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[m][r] = __builtin_ldexpf(o[m][r], unfold);
        }
#pragma unroll
        for (int m = 0; m < OM; ++m) o[m] += v_sum;
        if constexpr (SOURCE == 4) {
#pragma unroll
            for (int m = 0; m < OM; ++m)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const f32x4 v = in_order(f32x4{o[m][r], o[m][r + 1], o[m][r + 2], o[m][r + 3]});
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[m][r + e] = v[e];
                }
        }
    }
    auto store_row = [&](int row, int four, f32x4 v) {           // four of 4 * OM, for this lane's half
        const int query_e = a.query_of(row), head = (int)kv_head * a.shared + (row - query_e * a.shared);
        uint16_t* out = a.out + ((int64_t)(w.r.q_at + query_e) * a.heads + head) * D + 4 * g_e + 8 * four;
        *reinterpret_cast<u32x2*>(out) = u32x2{pack<F16>(v[0], v[1]), pack<F16>(v[2], v[3])};
    };
    const float m_own = m_ref == -__builtin_inff() ? m_ref : m_used;
    if (narrow) {
        // the wavefronts' sums meet in LDS, [wavefront][4 OM][lane], and each adds up a quarter of the places
        lds_barrier();
        const uint32_t at = 16u * (uint32_t)(thread & 63);
#pragma unroll
        for (int m = 0; m < OM; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *(lds_f4)((uint32_t)(wave * 4 * OM + 4 * m + r) * 1024u + at) = f32x4{o[m][4 * r], o[m][4 * r + 1], o[m][4 * r + 2], o[m][4 * r + 3]};
        if (g_e == 0) *(lds_u2)(kAside + (uint32_t)(8 * (32 * wave + n_e))) = u32x2{__float_as_uint(m_own), __float_as_uint(l)};
        lds_barrier();
        float m[kWaves], top = -__builtin_inff(), sum = 0.0f;
        u32x2 ml[kWaves];
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            ml[i] = *(lds_u2)(kAside + (uint32_t)(8 * (32 * i + n_e)));
            top = fmaxf(top, __uint_as_float(ml[i][0]));
        }
        const float use = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            m[i] = exp2_fast(__uint_as_float(ml[i][0]) - use);
            sum = fmaf(m[i], __uint_as_float(ml[i][1]), sum);
        }
        const float inv = in_pieces ? 1.0f : sum == 0.0f ? 0.0f : 1.0f / sum;
        float* to = a.partial + (int64_t)w.slot * kPieceFloats<D>;
#pragma unroll
        for (int x = 0; x < OM; ++x) {
            const int four = wave * OM + x;
            f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                const f32x4 y = *(lds_f4)((uint32_t)(i * 4 * OM + four) * 1024u + at);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = fmaf(m[i], y[e], v[e]);
            }
            if (in_pieces) reinterpret_cast<f32x4*>(to)[four * 64 + (thread & 63)] = v;
            else if (row0 + n_e < rows) store_row(row0 + n_e, four, f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv});
        }
        if (in_pieces && wave == 0 && g_e == 0) reinterpret_cast<f32x2*>(to + kRowTile * D)[n_e] = f32x2{top, sum};
        return;
    }
    if (in_pieces) {
        float* to = a.partial + (int64_t)w.slot * kPieceFloats<D>;
        f32x4* sums = reinterpret_cast<f32x4*>(to) + wave * (4 * OM) * 64 + (thread & 63);
#pragma unroll
        for (int m = 0; m < OM; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) sums[(4 * m + r) * 64] = f32x4{o[m][4 * r], o[m][4 * r + 1], o[m][4 * r + 2], o[m][4 * r + 3]};
        if (g_e == 0) reinterpret_cast<f32x2*>(to + kRowTile * D)[32 * wave + n_e] = f32x2{m_own, l};
        return;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;              // (no key seen: o is 0 as well)
    if (row0 + n_e < rows) {
#pragma unroll
        for (int m = 0; m < OM; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) store_row(row0 + n_e, 4 * m + r, f32x4{o[m][4 * r] * inv, o[m][4 * r + 1] * inv, o[m][4 * r + 2] * inv, o[m][4 * r + 3] * inv});
    }
}

// Joins the pieces of tiles of rows that were cut: a wavefront has 32 rows at a time and four values of each, in the pieces' own order of lanes.
constexpr int kAtOnce = 8, kFewPieces = 4;                      // pieces whose loads are out at a time
template <int D, bool F16>
__global__ __launch_bounds__(256) void attn_chunk_join_kernel(Args a) {
    const int lane = threadIdx.x & 63, n = lane & 31, g = lane >> 5;
    if ((int)blockIdx.x >= a.joins[0]) return;
    const unsigned kv_head = blockIdx.x % (unsigned)a.kv_heads;
    const Join w = reinterpret_cast<const Join*>(a.joins)[1 + blockIdx.x];
    const int rows = w.rows, pieces = w.pieces;
    const int64_t step = (int64_t)a.kv_heads * kPieceFloats<D>;
    const float* first = a.partial + (int64_t)w.slot * kPieceFloats<D>;
    const int four = 4 * (int)blockIdx.y + (int)(threadIdx.x >> 6);
    for (int part = 0; 32 * part < w.height && w.row + 32 * part < rows; ++part) {
        const int row = w.row + 32 * part + n;
        const float* ml = first + kRowTile * D + 2 * (32 * part + n);
        const int query = a.query_of(min(row, rows - 1)), head = (int)kv_head * a.shared + (min(row, rows - 1) - query * a.shared);
        const float* sums = first + 4 * ((part * (D / 8) + four) * 64 + lane);
        float top = -__builtin_inff(), sum = 0.0f;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        auto add = [&](auto at_once, int p0) {
            constexpr int N = decltype(at_once)::value;
            f32x2 x[N];
            f32x4 y[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int64_t at = min(p0 + i, pieces - 1) * step;
                x[i] = *reinterpret_cast<const f32x2*>(ml + at);
                y[i] = *reinterpret_cast<const f32x4*>(sums + at);
            }
            float higher = top;
#pragma unroll
            for (int i = 0; i < N; ++i) higher = fmaxf(higher, x[i][0]);
            const float use = higher == -__builtin_inff() ? 0.0f : higher, f = exp2_fast(top - use);
            sum *= f;
            v *= f;
            top = higher;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                // (a factor of 0 is no reason to leave a piece out: what is not finite in it has to reach the result, and a row whose scores in a piece are all NaN
                // has a maximum of -inf there)
                if (p0 + i < pieces) {
                    const float e = exp2_fast(x[i][0] - use);
                    sum = fmaf(e, x[i][1], sum);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = fmaf(e, y[i][j], v[j]);
                }
            }
        };
        if (pieces <= kFewPieces) {
            if (pieces > 0) add(std::integral_constant<int, kFewPieces>{}, 0);
        } else {
            for (int p0 = 0; p0 < pieces; p0 += kAtOnce) add(std::integral_constant<int, kAtOnce>{}, p0);
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (row < rows) {
            uint16_t* out = a.out + ((int64_t)(w.q_at + query) * a.heads + head) * D + 8 * four + 4 * g;
            *reinterpret_cast<u32x2*>(out) = u32x2{pack<F16>(v[0] * inv, v[1] * inv), pack<F16>(v[2] * inv, v[3] * inv)};
        }
    }
}

template <int SOURCE, int D, bool F16> hipError_t launch(Args a, const ChunkPlan& pl, hipStream_t stream) {
    constexpr auto kernel = attn_chunk_kernel<SOURCE, D, F16>;
    constexpr int bytes = 4 * Tile<D, kWaves>::kBytes + kAsideAll<SOURCE == 8 || SOURCE == 4>;
    static_assert(kRowTile == 128 && kFewRows <= 64, "tiles of rows are counted by shifts, and two for few rows");
    static_assert(kAsideAll<true> >= 2 * kScaleBytes<kKeys>, "two tiles' scales");
    if (hipError_t e = ensure_lds<kernel>(bytes); e != hipSuccess) return e;
    a.target = pl.target;
    a.slots = pl.slots;
    a.small = pl.small;
    if constexpr (SOURCE != kRows) {
        int* const plan = reinterpret_cast<int*>(a.partial);
        a.partial += pl.plan_bytes / sizeof(float);
        if (pl.target > 0) {
            a.joins = reinterpret_cast<int*>(a.partial);
            a.cut_tiles = pl.cut_tiles;
            a.partial += Join::bytes(pl.cut_tiles) / sizeof(float);
        }
        if (pl.plan_bytes > 0) {
            hipLaunchKernelGGL((attn_chunk_plan_kernel<SOURCE>), dim3(1), dim3(kPlanThreads), 0, stream, a, plan);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
            a.plan = plan;
        }
    }
    const hipError_t e = launch_blocks(pl.blocks, kThreads, hipSuccess, [&](int64_t first, int64_t count) {
        a.first_block = (unsigned)first;
        hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3(kThreads), bytes, stream, a);
        return hipGetLastError();
    });
    if (SOURCE == kRows || e != hipSuccess || pl.target == 0) return e;
    hipLaunchKernelGGL((attn_chunk_join_kernel<D, F16>), dim3((unsigned)pl.cut_tiles, D / 32), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

ChunkPlan plan_attn_chunk(int64_t requests, int64_t q_tokens, int heads, int kv_heads, int head_dim, int64_t max_tokens, bool cut, int cus) {
    ChunkPlan p{};
    const int64_t shared = heads / kv_heads, some = requests < q_tokens ? requests : q_tokens;
    // (a request's last tile may be short; one of few rows has two)
    auto tiles_of = [&](int height) { return (q_tokens * shared / height + 2 * some) * kv_heads; };
    int64_t tiles = tiles_of(kRowTile);
    const int64_t units = (max_tokens + kKeys - 1) / kKeys;
    const bool cuts = cut && units > kWholeFew;
    // small for sure, or (a call of so few rows) if its requests are short
    p.small = (cuts ? q_tokens * shared / kRowTile * kv_heads : tiles * units) <= kSmall / kNarrow;
    if (p.small) tiles = tiles_of(32);
    p.blocks = tiles;
    if (cut && requests > 64) p.plan_bytes = p.workspace = (size_t)Plan::bytes(requests);
    if (!cuts) return p;
    p.target = 2 * cus;
    // (pieces of tiles that are cut: cut_of() has it that there are no more than that, but for the rounding of its sums)
    const int64_t most = (int64_t)p.target + kv_heads, own = tiles * ((kNarrow * units + kLeastPiece - 1) / kLeastPiece);
    p.slots = (int)(own < most ? own : most);
    // (each in two pieces and more)
    const int64_t cut_tiles = p.slots / 2 + kv_heads;
    p.cut_tiles = (int)(tiles < cut_tiles ? tiles : cut_tiles);
    p.blocks = tiles + p.slots;
    p.workspace += (size_t)Join::bytes(p.cut_tiles) + (size_t)p.slots * kRowTile * (head_dim + 2) * sizeof(float);
    return p;
}

hipError_t launch_attn_chunk(const ChunkArgs& c, const any4_kv_cache* cache, const ChunkPlan& pl, void* workspace, hipStream_t stream) {
    Args a{c.q, c.k, c.v, {}, c.table, c.table_stride, (int)c.table_width, c.q_starts, c.k_starts, c.lengths, (int)c.q_tokens, (int)c.k_tokens, c.requests,
           c.heads, c.kv_heads, c.heads / c.kv_heads, c.window > 0 ? c.window : kNoWindow, c.sinks, 0, 0, 0, nullptr, nullptr, 0, 0u, c.softmax_scale * kLog2e, c.out,
           static_cast<float*>(workspace), 0u, 31};
    while ((int64_t)1 << (a.shared_shift - 31) < a.shared) ++a.shared_shift;
    a.shared_mul = (uint32_t)((((uint64_t)1 << a.shared_shift) + (uint64_t)a.shared - 1) / (uint64_t)a.shared);
    if (cache) a.c = kv_pages(*cache);
    auto types = [&](auto source, auto dim) {
        return c.f16 ? launch<decltype(source)::value, decltype(dim)::value, true>(a, pl, stream)
                     : launch<decltype(source)::value, decltype(dim)::value, false>(a, pl, stream);
    };
    auto dims = [&](auto source) {
        return c.head_dim == 128 ? types(source, std::integral_constant<int, 128>{}) : types(source, std::integral_constant<int, 64>{});
    };
    if (!cache) return dims(std::integral_constant<int, kRows>{});
    return cache->bits == 16 ? dims(std::integral_constant<int, 16>{}) : cache->bits == 8 ? dims(std::integral_constant<int, 8>{})
                                                                        : dims(std::integral_constant<int, 4>{});
}

}  // namespace any4
