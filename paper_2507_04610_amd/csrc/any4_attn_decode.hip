// any4_attn_decode: one new token for each request attends to its tokens in the paged cache.
//
// For a KV head and the up to 16 query heads that share it, tokens j:
//     s_j = scale q . k_j,   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),   m = max_j s_j
// in one pass over the cache with a running maximum.  The cache is read once (with more than 16 query heads on a KV head once for every 16
// of them), and that bounds the operator: a few floating-point operations for each byte at up to 16 heads.  Everything else is arranged so
// that no byte takes a detour.
//
// A wavefront takes 32 tokens a step, for all heads of the KV head.  S^T = K Q^T with v_mfma_f32_16x16x32, k's rows as the A
// operand straight from memory (lane: token l % 16, 8 values along the head); the scores of a head then lie in the 4 lanes l % 16 =
// head, 8 tokens in each, and that is already the B operand of O^T = V^T P^T over 32 tokens, the tokens of lane l / 16 = g being
// 4 g .. 4 g + 3 of either 16.  V^T's lanes hold 8 tokens of one place along the head, which 8 loads of D / 16 places each give after
// half a v_perm a value: no LDS, no exchange between lanes but a head's maximum.
//
// Codes c of 8 or 4 bits go to the matrix cores as 16-bit floats that hold them exactly (c + kBias: 1024 + c in fp16 and 128 + c in
// bf16 take two bits set in place; c itself for 8 bits in bf16), scale and offset are applied to sums:
//     q . k_j = ks_j (q . c'_j - kBias sum(q)) + ko_j sum(q)
//     o = sum_j (p_j vs_j) (c_j - kCentre) + sum_j p_j (vo_j + kCentre vs_j)
// where the first sum has p_j vs_j rounded to 16 bits, and every step takes (kBias + kCentre) sum(..) of the same rounded weights off it in
// front of adding sum(.. c'_j), both on the matrix cores: the rounding of the weights meets values around 0 as it does without codes, and the running sums
// hold no bias, whose roundings would grow with the tokens (taken off once at the end: 1e-2 of the result at 131072 tokens a block, fp16, 4 bits).
//
// Rounding: scores, maxima, sums and accumulators are fp32; p (times vs) is rounded to 16 bits for the matrix cores, once; in fp16 with the exponent of a head's largest
// such product taken off (that of its largest vs alone would leave nothing of the others beside a large value of no weight).
//
// Who does what.  Lengths are the device's, so each block finds its share itself: a request has units of 32 tokens a wavefront (128 or
// 256 tokens a block), all units of all requests and KV heads stand in one line, and the blocks that fit the chip take equal parts
// of it.  However ragged the lengths, all blocks end together; a block cuts at most two groups (request, KV head), whose
// pieces' sums and maxima go to the workspace, and the last of a group's pieces to come joins them in the same launch.  (A fixed
// piece length had a block for each piece: 5 us of beginning and end for every one, 64 requests of 2048 .. 8192 tokens took 305 us with
// 2048 tokens a piece and 441 with 512.)  Groups with fewer than kWholeUnits units on average are not cut for the sake of more blocks:
// the join costs as much as four steps.
//
// Measured, 8 KV heads of 128, us (bytes of the cache / time):
//     16 bits, 64 requests of 2048 .. 8192 tokens, 32 query heads          208   (6.5 TB/s; the fastest read-only stream measured here reaches 6.8)
//     8 bits, 32 requests of 1 .. 4096 tokens, 32 query heads               34   (4.1 TB/s)
//     4 bits, one request of 131071 tokens, 64 query heads                  39   (3.7 TB/s; 3 us until the first bytes are asked for, 6 for the
//                                                                                join of 32 pieces; vector units busy half of the time)
//     16 bits, one request of 333 tokens, 32 query heads                     8.3 (loads that wait for each other: length, page, k and v)
//     16 bits, 48 requests of 1 .. 32768 tokens, window 4096, 32 query heads 124 (6.0 TB/s; over 8 bits 76, 5.1 TB/s, over 4 bits 52, 3.9 TB/s)
//     4 bits, fp16, one request, window, heads of 64                         10.9
#include "any4_attn.h"
#include "any4_internal.h"
#include "any4_splitk.h"

namespace any4 {

namespace {

constexpr int kStep = 32;                                       // tokens of a wavefront's step
constexpr int kFewGroups = 64;                                  // below: blocks of 8 wavefronts, one for a compute unit; from there on two or three of 4
constexpr int kMaxRequests = 2048;                              // of a launch: their units' beginnings lie in LDS
constexpr int kWholeUnits = 4;                                  // with fewer units a group (on average) no group is cut for the sake of more blocks
constexpr int kJoin = 16;                                       // pieces whose loads are out at a time
// fp16 weights p * vs: the largest lies 2^kUp above 1 (fp16 has steps of 2^-24 down there, and tokens of small weight are many).  Scales of a step within 2^kSpread are
// taken as the largest of them (the largest product then lies as much lower at most), others with their scores.
constexpr float kUp = 6.0f, kSpread = 256.0f;

// where the join's parts begin in LDS, behind a factor for each head and piece: they are pairs of floats
__host__ __device__ constexpr int parts_at(int heads, int pieces) { return (heads * pieces + 1) & ~1; }

struct DecodeArgs {
    Rows q;
    KvPages c;
    const int32_t* table;
    int64_t table_stride;
    int table_width;
    const int32_t* lengths;
    int requests, heads, shared, head_tiles;
    int window, sinks;                 // tokens seen at the end and at the beginning (WINDOW variants)
    float scale_log2;                  // softmax scale * log2(e)
    uint16_t* out;
    float* partial;                    // [block][2][query head][D + 2]: sums, then maximum and sum of weights of every head
    uint8_t* words;                    // an arrival word for each (request, KV head, head tile)
};

// One arrival at a word; true if it is the last of `pieces` (at most 2^16 - 1).  As arrive_one(), with 16 bits to count in.
__device__ __forceinline__ bool arrive_piece(unsigned long long* word, int pieces) {
    constexpr unsigned long long kTag = 0xA4C0DEDECull << 16;
    auto own = [&](unsigned long long v) -> bool { return (v >> 16) == (kTag >> 16) && (int)(v & 0xFFFFull) < pieces; };
    unsigned long long old = __hip_atomic_fetch_add(word, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), count;
    if (own(old)) {
        count = (old & 0xFFFFull) + 1ull;
    } else {
        old += 1ull;                                            // the add went into a foreign word and is dropped with it
        for (;;) {
            count = own(old) ? (old & 0xFFFFull) + 1ull : 1ull;
            if (__hip_atomic_compare_exchange_strong(word, &old, kTag | count, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) break;
        }
    }
    const bool last = (int)count == pieces;
    if (last) __hip_atomic_store(word, kTag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return last;
}

// two floats between blocks, as splitk_store() and splitk_load()
__device__ __forceinline__ void store_pair(float* p, f32x2 v) {
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), __builtin_bit_cast(unsigned long long, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 load_pair(const float* p) {
    return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// What a kernel only reads, at an address that all lanes share: scalar loads, which do not queue behind the vector loads.
typedef const __attribute__((address_space(4))) int32_t* scalar_i32;
__device__ __forceinline__ scalar_i32 scalar(const int32_t* p) { return (scalar_i32)reinterpret_cast<uintptr_t>(p); }

// The cache is read once: loads that leave nothing behind in L2.
template <class V> __device__ __forceinline__ V load_once(const void* p) { return __builtin_nontemporal_load(static_cast<const V*>(p)); }

template <int N> __device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
    if constexpr (N >= 4) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const u32x4 x = load_once<u32x4>(p + 16 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[4 * i + j] = x[j];
        }
    } else if constexpr (N == 2) {
        const u32x2 x = load_once<u32x2>(p);
        w[0] = x[0];
        w[1] = x[1];
    } else {
        w[0] = load_once<uint32_t>(p);
    }
}

__device__ __forceinline__ float ubyte(uint32_t w, int j) { return (float)((w >> (8 * j)) & 0xFFu); }
// high halves of two fp32 values: their bf16 where nothing is lost
__device__ __forceinline__ uint32_t high_halves(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

template <int BITS, bool F16> struct Codes {
    static constexpr int kBias = BITS == 16 ? 0 : F16 ? 1024 : BITS == 4 ? 128 : 0;
    static constexpr int kCentre = BITS == 16 ? 0 : 1 << (BITS - 1);
    static constexpr uint32_t kMagic = F16 ? 0x64006400u : 0x43004300u;
    // -(kBias + kCentre) twice in 16 bits, exact: fp16 -1032 and -1152, bf16 -136 and -128
    static constexpr uint32_t kOff = F16 ? (BITS == 4 ? 0xE408E408u : 0xE480E480u) : BITS == 4 ? 0xC308C308u : 0xC300C300u;
};

// A operand of S^T from a token's words: matrix instruction i
template <int BITS, bool F16, int N> __device__ __forceinline__ u32x4 k_operand(const uint32_t (&w)[N], int i) {
    using C = Codes<BITS, F16>;
    if constexpr (BITS == 16) return u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
    if constexpr (BITS == 8 && F16) {
        return u32x4{__builtin_amdgcn_perm(0x64646464u, w[2 * i], 0x04010400u), __builtin_amdgcn_perm(0x64646464u, w[2 * i], 0x04030402u),
                     __builtin_amdgcn_perm(0x64646464u, w[2 * i + 1], 0x04010400u), __builtin_amdgcn_perm(0x64646464u, w[2 * i + 1], 0x04030402u)};
    }
    if constexpr (BITS == 8 && !F16) {
        const uint32_t a = w[2 * i], b = w[2 * i + 1];
        return u32x4{high_halves(ubyte(a, 0), ubyte(a, 1)), high_halves(ubyte(a, 2), ubyte(a, 3)), high_halves(ubyte(b, 0), ubyte(b, 1)),
                     high_halves(ubyte(b, 2), ubyte(b, 3))};
    }
    if constexpr (BITS == 4) {
        const uint32_t a = w[i];                               // pairs (code x, code x + 4)
        return u32x4{(a & 0x000F000Fu) | C::kMagic, ((a >> 4) & 0x000F000Fu) | C::kMagic, ((a >> 8) & 0x000F000Fu) | C::kMagic,
                     ((a >> 12) & 0x000F000Fu) | C::kMagic};
    }
}

// two tokens' values of place m, the first in the low half
template <int BITS, bool F16, int N> __device__ __forceinline__ uint32_t v_pair(const uint32_t (&a)[N], const uint32_t (&b)[N], int m) {
    using C = Codes<BITS, F16>;
    if constexpr (BITS == 16) return __builtin_amdgcn_perm(b[m >> 1], a[m >> 1], m & 1 ? 0x07060302u : 0x05040100u);
    if constexpr (BITS == 8 && F16) {
        const uint32_t sel = 0x0C000C00u | (uint32_t)(4 + (m & 3)) << 16 | (uint32_t)(m & 3);
        return __builtin_amdgcn_perm(b[m >> 2], a[m >> 2], sel) | C::kMagic;
    }
    if constexpr (BITS == 8 && !F16) return high_halves(ubyte(a[m >> 2], m & 3), ubyte(b[m >> 2], m & 3));
    if constexpr (BITS == 4) {
        const uint32_t w = __builtin_amdgcn_perm(b[0], a[0], m < 4 ? 0x05040100u : 0x07060302u);
        return ((w >> (4 * (m & 3))) & 0x000F000Fu) | C::kMagic;
    }
}

// units of UNIT tokens of a request; one without tokens has one, in which its zeros are written
template <int UNIT> __device__ __forceinline__ int units_of(int length, int64_t capacity) {
    return (int)max((min((int64_t)length, capacity) + UNIT - 1) / UNIT, (int64_t)1);
}

// With a window a request's work is the steps that hold a token it sees: those of the first tokens (`sinks`), then from the step in which
// the window begins.  Tokens are counted without the whole steps in between, `hidden` of them behind the first `front`.
struct Seen {
    int start, front, hidden;
    __device__ __forceinline__ Seen(int len, int window, int sinks) {
        start = max(len - window, 0);
        const int base = start & ~(kStep - 1);
        front = min((sinks + kStep - 1) & ~(kStep - 1), base);
        hidden = base - front;
    }
};

// over the four lanes that hold a head's tokens
template <class F> __device__ __forceinline__ float head_reduce(float v, F f) {
    u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    v = f(__uint_as_float(x[0]), __uint_as_float(x[1]));
    x = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return f(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
// over all lanes of a wavefront
template <class F> __device__ __forceinline__ float wave_reduce(float v, F f) { return head_reduce(lanes_reduce<16>(v, f), f); }

// WAVES 8: one block for a compute unit, for few groups, whose pieces are then few to join (one request of 32768 tokens, 8 groups, 16 / 8 / 4 bits:
// 28 / 22 / 17 us, with 4 wavefronts 34 / 25 / 29); WAVES 4: two or three, whose beginnings and ends overlap (32 requests of 1 .. 4096, 256
// groups: 52 / 33 / 27 against 52 / 41 / 35).  AHEAD: a step's loads are out before the step in front of it is worked on, which takes a
// second step's registers; otherwise the other wavefronts of the SIMD cover for it (4 wavefronts, 32 and 16 requests of 1 .. 4096: 8 bits 33.4
// and 21.3 us, with it 35.2 and 23.8; 4 bits 27.5 and 19.5, with it 35.5 and 24.8).
template <int BITS, int D, bool F16, int WAVES, bool AHEAD, bool WINDOW>
__global__ __launch_bounds__(64 * WAVES, AHEAD ? 2 : 3) void attn_decode_kernel(DecodeArgs a) {
    using C = Codes<BITS, F16>;
    constexpr int THREADS = 64 * WAVES, UNIT = kStep * WAVES;
    constexpr int KM = D / 32, VM = D / 16;                     // matrix instructions of S^T (16 tokens) and of O^T (32 tokens)
    constexpr int ROW = D * BITS / 8;                           // bytes of a token
    constexpr int KW = D * BITS / 128;                          // words of a lane: k of one token
    constexpr int VB = VM * BITS / 8, VW = VB < 4 ? 1 : VB / 4; // bytes and words of a lane: v of one token
    constexpr bool QUANT = BITS != 16;
    constexpr int PAD = D + 4;                                  // a head's sums in LDS: 16 heads' pieces in different banks
    extern __shared__ __attribute__((aligned(16))) float lds[];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int most = min(16, a.shared), room = most * (D + 2);  // query heads of a full head tile; floats of a piece's result
    const int64_t capacity = (int64_t)a.table_width << a.c.page_shift;

    auto request_units = [&](int length) -> int {
        if constexpr (WINDOW) {
            const int len = (int)min((int64_t)max(length, 0), capacity);
            return units_of<UNIT>(len - Seen(len, a.window, a.sinks).hidden, capacity);
        } else {
            return units_of<UNIT>(length, capacity);
        }
    };

    // Where the requests' units begin: with up to 64 requests in the lanes, with more in LDS behind the wavefronts' sums or the
    // pieces' factors and parts.
    const bool many = a.requests > 64;
    int* begins = reinterpret_cast<int*>(lds + max(WAVES * most * (PAD + 2), parts_at(most, (int)gridDim.x) + 2 * THREADS));
    int lane_begin, lane_end, units_of_all;
    if (!many) {
        const int r = min(lane, a.requests - 1);
        const int units = lane < a.requests ? request_units(a.lengths[r]) : 0;
        lane_end = lanes_scan(units);
        lane_begin = lane_end - units;
        units_of_all = __builtin_amdgcn_readlane(lane_end, 63);
    } else {
        int* sums = begins + a.requests + 1;
        int before = 0;
        for (int r0 = 0; r0 < a.requests; r0 += THREADS) {
            const int r = r0 + (int)threadIdx.x;
            const int sum = lanes_scan(r < a.requests ? request_units(a.lengths[r]) : 0);
            if (lane == 63) sums[wave] = sum;
            __syncthreads();
            int here = before;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                if (w < wave) here += sums[w];
                before += sums[w];
            }
            if (r < a.requests) begins[r + 1] = here + sum;
            if (r == 0) begins[0] = 0;
            __syncthreads();
        }
        lane_begin = lane_end = 0;
        units_of_all = __builtin_amdgcn_readfirstlane(before);
    }
    // That many units there are for each of `groups` (KV head, head tile), a request's groups one behind the other, and `blocks` blocks
    // share them evenly, the first `longer` of them with one more than `each`.  (The host sees to it that they are fewer than 2^31.)
    const unsigned groups = (unsigned)(a.c.kv_heads * a.head_tiles), all = (unsigned)units_of_all * groups;
    const unsigned blocks = min(gridDim.x, all < kWholeUnits * (unsigned)a.requests * groups ? (unsigned)a.requests * groups : all);
    if (blockIdx.x >= blocks) return;
    const unsigned each = all / blocks, longer = all - each * blocks;
    unsigned at = blockIdx.x * each + min(blockIdx.x, longer);
    const unsigned end = at + each + (blockIdx.x < longer ? 1u : 0u);
    auto block_of = [&](unsigned unit) -> int {
        return (int)(unit < longer * (each + 1) ? unit / (each + 1) : longer + (unit - longer * (each + 1)) / each);
    };
    int request;
    {
        const int y = (int)(at / groups);                       // the last request that begins at or before y
        if (!many) {
            request = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(lane < a.requests && lane_begin <= y));
        } else {
            int lo = 0;
            for (int hi = a.requests - 1; lo < hi;) {
                const int mid = (lo + hi + 1) >> 1;
                if (__builtin_amdgcn_readfirstlane(begins[mid]) <= y) lo = mid;
                else hi = mid - 1;
            }
            request = lo;
        }
    }
    for (; at < end; ++request) {
        const int len = (int)min((int64_t)max(scalar(a.lengths)[request], 0), capacity);
        const Seen seen(len, WINDOW ? a.window : len, WINDOW ? a.sinks : 0);
        // a counted token's place in the request
        auto real = [&](int t) -> int { return !WINDOW || t < seen.front ? t : t + seen.hidden; };
        const scalar_i32 table = scalar(a.table + (int64_t)request * a.table_stride);
        const unsigned begin = many ? __builtin_amdgcn_readfirstlane(begins[request]) : __builtin_amdgcn_readlane(lane_begin, request & 63);
        const unsigned units = (many ? __builtin_amdgcn_readfirstlane(begins[request + 1]) : __builtin_amdgcn_readlane(lane_end, request & 63)) - begin;
        const unsigned request_at = begin * groups;
        for (int group = (int)((at - request_at) / units); group < (int)groups && at < end; ++group) {
            const unsigned group_at = request_at + (unsigned)group * units;
            const int from = (int)(at - group_at), to = (int)min(units, end - group_at);
            at = group_at + (unsigned)to;
            const int kv_head = a.head_tiles == 1 ? group : group / a.head_tiles;
            const int head_tile = group - kv_head * a.head_tiles;
            const int first_head = kv_head * a.shared + head_tile * 16, here = min(16, a.shared - head_tile * 16);
            const int t0 = from * UNIT, t1 = min(WINDOW ? len - seen.hidden : len, to * UNIT);

            float m_ref = -__builtin_inff(), l = 0.0f, vo_sum = 0.0f;
            f32x4 o[VM];
#pragma unroll
            for (int m = 0; m < VM; ++m) o[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            // fp16 weights p * vs: held as p * (vs * 2^-exponent), the exponent being that of the largest so far, less kUp
            float exponent = 0.0f;

            // One step's tokens: which of the two 16s' exist, and what the lanes load of them.
            struct Step {
                int there[2];
                uint32_t kw[2][KW], vw[8][VW];
                u32x4 so[2][2];
            };
            const int page_mask = (1 << a.c.page_shift) - 1;
            // the pages of a step at t (its own, again, past the end)
            auto pages_of = [&](int t, int (&page)[2]) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int th = t + 16 * h < t1 ? t + 16 * h : t < t1 ? t : t0;
                    page[h] = table[real(th) >> a.c.page_shift];
                }
            };
            auto load = [&](int t, const int (&page)[2], Step& st) {
                int64_t tok[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int th = real(t + 16 * h < t1 ? t + 16 * h : t);
                    const bool ok = page[h] >= 0 && page[h] < a.c.pages;           // a page that does not exist has no tokens
                    st.there[h] = ok ? min(max(len - (WINDOW ? real(t) + 16 * h : t + 16 * h), 0), 16) : 0;
                    tok[h] = a.c.first_token(ok ? page[h] : 0, kv_head) + (th & page_mask);
                    const uint8_t* kp = a.c.k + tok[h] * ROW;
                    if constexpr (BITS == 16) {
#pragma unroll
                        for (int i = 0; i < KM; ++i) {
                            const u32x4 x = load_once<u32x4>(kp + (uint32_t)(col * ROW + 64 * i + 16 * g));
#pragma unroll
                            for (int j = 0; j < 4; ++j) st.kw[h][4 * i + j] = x[j];
                        }
                    } else {
                        load_words(kp + (uint32_t)(col * ROW + (ROW / 4) * g), st.kw[h]);
                        const uint8_t* sp = reinterpret_cast<const uint8_t*>(a.c.scales + tok[h] * 4) + (uint32_t)(32 * g);
                        st.so[h][0] = load_once<u32x4>(sp);
                        st.so[h][1] = load_once<u32x4>(sp + 16);
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint8_t* vp = a.c.v + tok[j >> 2] * ROW + (uint32_t)((4 * g + (j & 3)) * ROW + VB * col);
                    if constexpr (VB == 2) st.vw[j][0] = load_once<uint16_t>(vp);
                    else load_words(vp, st.vw[j]);
                }
            };

            // A step's loads are out before the step in front of it is worked on, its pages' numbers one step earlier.
            Step st;
            int page[2];
            const int first = t0 + kStep * wave;
            pages_of(first, page);
            u32x4 q[KM];
            {
                int q_lane = lane;
                asm volatile("" : "+v"(q_lane));
                const int col = q_lane & 15, g = q_lane >> 4;
                const uint16_t* qp = a.q.p + (int64_t)request * a.q.token + (int64_t)(first_head + min(col, here - 1)) * a.q.head;
#pragma unroll
                for (int i = 0; i < KM; ++i) q[i] = *reinterpret_cast<const u32x4*>(qp + (QUANT ? (D / 4) * g + 8 * i : 32 * i + 8 * g));
            }
            if (AHEAD && first < t1) load(first, page, st);
            if (AHEAD) pages_of(first + UNIT, page);
            __builtin_amdgcn_sched_barrier(0);
            // Q^T, columns past `here` are zeros
            float sum_q = 0.0f;
#pragma unroll
            for (int i = 0; i < KM; ++i) {
                if (col >= here) q[i] = u32x4{0u, 0u, 0u, 0u};
                if constexpr (QUANT) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum_q += h16lo_to_f32<F16>(q[i][j]) + h16hi_to_f32<F16>(q[i][j]);
                }
                if constexpr (BITS == 4) {                              // pairs (x, x + 4), as the codes come
                    const u32x4 r = q[i];
                    q[i] = u32x4{__builtin_amdgcn_perm(r[2], r[0], 0x05040100u), __builtin_amdgcn_perm(r[2], r[0], 0x07060302u),
                                 __builtin_amdgcn_perm(r[3], r[1], 0x05040100u), __builtin_amdgcn_perm(r[3], r[1], 0x07060302u)};
                }
            }
            if constexpr (QUANT) sum_q = head_reduce(sum_q, [](float x, float y) { return x + y; }) * a.scale_log2;
            for (int t = first; t < t1; t += UNIT) {
                Step next;
                if (!AHEAD) load(t, page, st);
                if (AHEAD && t + UNIT < t1) load(t + UNIT, page, next);
                pages_of(t + (AHEAD ? 2 : 1) * UNIT, page);
                __builtin_amdgcn_sched_barrier(0);                      // (left alone, the loads sink to where their values are used)
                auto& kw = st.kw;
                auto& vw = st.vw;
                auto& so = st.so;
                const int there[2] = {st.there[0], st.there[1]};

                f32x4 s[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    s[h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int i = 0; i < KM; ++i) s[h] = mma16<F16>(k_operand<BITS, F16>(kw[h], i), q[i], s[h]);
                }
                float x[8], vs[8], vo[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int h = j >> 2, r = j & 3;
                    if constexpr (QUANT) {
                        const uint32_t kk = so[h][r >> 1][2 * (r & 1)], vv = so[h][r >> 1][2 * (r & 1) + 1];
                        const float u = fmaf(s[h][r], a.scale_log2, -(float)C::kBias * sum_q);
                        x[j] = fmaf(bf16lo_to_f32(kk), u, bf16hi_to_f32(kk) * sum_q);
                        vs[j] = bf16lo_to_f32(vv);
                        vo[j] = fmaf((float)C::kCentre, vs[j], bf16hi_to_f32(vv));
                    } else {
                        x[j] = s[h][r] * a.scale_log2;
                    }
                }
                const int at = real(t);
                if (there[0] + there[1] < 32 || (WINDOW && at < seen.start && at + kStep > a.sinks)) {
                    // what lies behind the last token, outside of the window or in a page that does not exist may be anything: none of it
                    // comes near a sum
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int in_half = 4 * g + (j & 3), place = at + 16 * (j >> 2) + in_half;
                        const bool ok = in_half < there[j >> 2] && (!WINDOW || place >= seen.start || place < a.sinks);
                        x[j] = ok ? x[j] : -__builtin_inff();
                        if constexpr (QUANT) {
                            vs[j] = ok ? vs[j] : 0.0f;
                            vo[j] = ok ? vo[j] : 0.0f;
                        } else {
#pragma unroll
                            for (int w = 0; w < VW; ++w) vw[j][w] = ok ? vw[j][w] : 0u;
                        }
                    }
                }

                float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
                top = head_reduce(top, [](float u, float v) { return fmaxf(u, v); });
                bool moved = top > m_ref;
                float product = 0.0f;                                   // the exponent of this step's largest product, less the maximum behind it
                if constexpr (QUANT && F16) {
                    const float higher = fmaxf(m_ref, top);
                    float big = 0.0f, least = __builtin_inff();
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        big = fmaxf(big, fabsf(vs[j]));
                        least = fminf(least, fabsf(vs[j]));
                    }
                    big = head_reduce(big, [](float u, float v) { return fmaxf(u, v); });
                    product = (top - higher) + __builtin_amdgcn_logf(big);
                    if (__builtin_expect(__builtin_amdgcn_ballot_w64(least * kSpread < big) != 0ull, 0)) {
                        product = -__builtin_inff();
#pragma unroll
                        for (int j = 0; j < 8; ++j) product = fmaxf(product, (x[j] - higher) + __builtin_amdgcn_logf(fabsf(vs[j])));
                        product = head_reduce(product, [](float u, float v) { return fmaxf(u, v); });
                    }
                    product = fminf(fmaxf(ceilf(product) - kUp, -126.0f), 126.0f);
                    moved |= product + (higher - m_ref) > exponent;
                }
                if (__builtin_amdgcn_ballot_w64(moved)) {
                    const float m_new = fmaxf(m_ref, top), less = m_new > m_ref ? m_ref - m_new : 0.0f;
                    const float alpha = exp2_fast(less);
                    m_ref = m_new;
                    l *= alpha;
                    vo_sum *= alpha;
                    float f = alpha;
                    if constexpr (QUANT && F16) {
                        const float before = exponent;
                        // (a whole number, so that a weight of 1 costs vs nothing; down, or it would rise with every move)
                        exponent = fmaxf(floorf(exponent + less), product);
                        f = exp2_fast(less + (before - exponent));
                    }
#pragma unroll
                    for (int m = 0; m < VM; ++m) o[m] *= f;
                }
                const float m_use = m_ref == -__builtin_inff() ? 0.0f : m_ref;
                const float unit = __builtin_ldexpf(1.0f, -(int)exponent);
                u32x4 p;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[j] = exp2_fast(x[j] - m_use);
                    l += x[j];
                    if constexpr (QUANT) {
                        vo_sum = fmaf(x[j], vo[j], vo_sum);
                        x[j] *= vs[j];
                        if constexpr (F16) x[j] *= unit;
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) p[j] = f32x2_to_h16x2<F16>(x[2 * j], x[2 * j + 1]);
                if constexpr (QUANT) {
#pragma unroll
                    for (int m = 0; m < VM; ++m) o[m] = mma16<F16>(u32x4{C::kOff, C::kOff, C::kOff, C::kOff}, p, o[m]);
                }
#pragma unroll
                for (int m = 0; m < VM; ++m) {
                    u32x4 v;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = v_pair<BITS, F16>(vw[2 * j], vw[2 * j + 1], m);
                    o[m] = mma16<F16>(v, p, o[m]);
                }
                if (AHEAD) st = next;
            }

            // (the lane's number anew: what follows from it below is not to take registers from the loop above)
            int thread = threadIdx.x;
            asm volatile("" : "+v"(thread));
            const int col_e = thread & 15, g_e = (thread >> 4) & 3;
            // The wavefronts' results meet in LDS: [wave][head][PAD], then [wave][head] maximum and sum of weights.
            auto add = [](float u, float v) { return u + v; };
            l = head_reduce(l, add);
            if constexpr (QUANT) vo_sum = head_reduce(vo_sum, add);
            float* ml = lds + WAVES * here * PAD;
            __syncthreads();                                            // (nobody reads what another piece left there)
            if (col_e < here) {
                const float back = QUANT && F16 ? __builtin_ldexpf(1.0f, (int)exponent) : 1.0f;
                float* to_lds = lds + (wave * here + col_e) * PAD;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int m = 0; m < VM; m += 4) {
                        f32x4 v = {o[m][r], o[m + 1][r], o[m + 2][r], o[m + 3][r]};
                        if constexpr (QUANT) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) v[j] = fmaf(back, v[j], vo_sum);
                        }
                        *reinterpret_cast<f32x4*>(to_lds + VM * (4 * g_e + r) + m) = v;
                    }
                if (g_e == 0) {
                    ml[2 * (wave * here + col_e)] = m_ref;
                    ml[2 * (wave * here + col_e) + 1] = l;
                }
            }
            __syncthreads();
            uint16_t* out = a.out + ((int64_t)request * a.heads + first_head) * D;
            const bool split = from > 0 || to < units;
            // A block has at most two groups that it shares with others: one that begins in front of it, one that goes on behind it.
            float* mine = a.partial + ((int64_t)blockIdx.x * 2 + (from > 0 ? 0 : 1)) * room;
            for (int i = thread; i < here * D / 2; i += THREADS) {      // two places of a head each
                const int n = i / (D / 2), d = 2 * i - n * D;
                float top = -__builtin_inff();
#pragma unroll
                for (int w = 0; w < WAVES; ++w) top = fmaxf(top, ml[2 * (w * here + n)]);
                const float use = top == -__builtin_inff() ? 0.0f : top;
                float sum = 0.0f;
                f32x2 v = {0.0f, 0.0f};
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float f = exp2_fast(ml[2 * (w * here + n)] - use);
                    sum = fmaf(f, ml[2 * (w * here + n) + 1], sum);
                    const f32x2 x = *reinterpret_cast<const f32x2*>(lds + (w * here + n) * PAD + d);
                    v = f32x2{fmaf(f, x[0], v[0]), fmaf(f, x[1], v[1])};
                }
                if (!split) {
                    reinterpret_cast<uint32_t*>(out)[i] = sum == 0.0f ? 0u : f32x2_to_h16x2<F16>(v[0] / sum, v[1] / sum);
                } else {
                    store_pair(mine + 2 * i, v);
                    if (d == 0) store_pair(mine + here * D + 2 * n, f32x2{top, sum});
                }
            }
            if (!split) continue;

            // The last piece of a group to come adds all of them: first the pieces' factors, a wavefront for a head and a lane for a piece,
            // then the sums in the pieces' order, with the pieces dealt out to as many threads as there are for each two places.  (One compute
            // unit reads what the others wrote: all its loads are out at once, or this takes longer than the rest of a short call.)
            const int first_block = block_of(group_at), pieces = block_of(group_at + units - 1) - first_block + 1;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            int* last = reinterpret_cast<int*>(lds);
            if (thread == 0)
                *last = arrive_piece(reinterpret_cast<unsigned long long*>(a.words + ((int64_t)request * groups + group) * kWordBytes), pieces);
            __syncthreads();
            const bool joins = *last != 0;
            __syncthreads();
            if (!joins) continue;
            // (the first piece lies in its block's second place, the others in their blocks' first)
            const float* base = a.partial + (int64_t)first_block * 2 * room;
            auto piece_at = [&](int w) -> const float* { return base + (w == 0 ? room : w * 2 * room); };
            const int items = here * D / 2, slices = max(THREADS / items, 1), span = (pieces + slices - 1) / slices;
            const int slice = thread / items, w_first = slice * span, w_end = slice < slices ? min(pieces, w_first + span) : 0;
            float* factor = lds;                                        // [head][pieces]
            float* parts = lds + parts_at(here, pieces);                // [slice][items][2], behind the factors
            f32x2 x[kJoin];
            auto load_parts = [&](int w0, int i) {
#pragma unroll
                for (int w = 0; w < kJoin; ++w)
                    x[w] = w0 + w < w_end && i < items ? load_pair(piece_at(w0 + w) + 2 * i) : f32x2{0.0f, 0.0f};
            };
            auto load_ml = [&](int w, int n) -> f32x2 {
                return w < pieces && n < here ? load_pair(piece_at(w) + here * D + 2 * n) : f32x2{-__builtin_inff(), 0.0f};
            };
            const int lane_e = thread & 63;
            f32x2 ml_of = load_ml(lane_e, wave);
            load_parts(w_first, thread - slice * items);                // (on their way while the factors are made)
            for (int n = wave; n < here; n += WAVES) {
                if (n != wave) ml_of = load_ml(lane_e, n);
                float top = -__builtin_inff(), sum = 0.0f;
                for (int w = lane_e; w < pieces; w += 64) {
                    if (w >= 64) ml_of = load_ml(w, n);
                    factor[n * pieces + w] = ml_of[0];
                    const float higher = fmaxf(top, ml_of[0]), use = higher == -__builtin_inff() ? 0.0f : higher;
                    sum = fmaf(exp2_fast(top - use), sum, exp2_fast(ml_of[0] - use) * ml_of[1]);
                    top = higher;
                }
                const float own_top = top;
                top = wave_reduce(top, [](float u, float v) { return fmaxf(u, v); });
                const float use = top == -__builtin_inff() ? 0.0f : top;
                sum = wave_reduce(sum * exp2_fast(own_top - use), add);
                const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                for (int w = lane_e; w < pieces; w += 64) factor[n * pieces + w] = exp2_fast(factor[n * pieces + w] - use) * inv;
            }
            __syncthreads();
            for (int i0 = 0; i0 < items; i0 += THREADS) {
                const int i = i0 + thread - slice * items, n = min(i / (D / 2), here - 1);
                if (i0 > 0) load_parts(w_first, i);
                f32x2 v = {0.0f, 0.0f};
                for (int w0 = w_first; w0 < w_end; w0 += kJoin) {
                    if (w0 > w_first) load_parts(w0, i);
#pragma unroll
                    for (int w = 0; w < kJoin; ++w)
                        if (w0 + w < w_end) {
                            const float f = factor[n * pieces + w0 + w];
                            v = f32x2{fmaf(f, x[w][0], v[0]), fmaf(f, x[w][1], v[1])};
                        }
                }
                if (slices > 1) {
                    if (slice < slices) reinterpret_cast<f32x2*>(parts)[thread] = v;
                    __syncthreads();
                    if (slice == 0)
                        for (int s = 1; s < slices; ++s) {
                            const f32x2 other = reinterpret_cast<const f32x2*>(parts)[s * items + i];
                            v = f32x2{v[0] + other[0], v[1] + other[1]};
                        }
                }
                if (i < items && slice == 0) reinterpret_cast<uint32_t*>(out)[i] = f32x2_to_h16x2<F16>(v[0], v[1]);
            }
        }
    }
}

template <int BITS, int D, bool F16, int WAVES, bool WINDOW> hipError_t launch(const DecodeArgs& a, const DecodePlan& pl, hipStream_t stream) {
    constexpr auto kernel = attn_decode_kernel<BITS, D, F16, WAVES, BITS == 16 || WAVES == 8, WINDOW>;
    auto bytes = [](int heads, int requests, int blocks) {
        const int own = WAVES * heads * (D + 6), join = parts_at(heads, blocks) + 128 * WAVES;
        return (int)sizeof(float) * ((own > join ? own : join) + requests + 1 + WAVES);
    };
    if (hipError_t e = ensure_lds<kernel>(bytes(16, kMaxRequests, 1024)); e != hipSuccess) return e;
    const int most = pl.shared < 16 ? pl.shared : 16;
    // Blocks of 4 wavefronts: two for a compute unit, with 4 bits three.  What decides is how many units a block gets beside its beginning and
    // end; by bits, us with two / three blocks for 16 requests of 1 .. 4096 tokens, 32 of them, 64 of 100 .. 2048, 64 of 2048 .. 8192:
    //     16 bits 30.7 / 35.5   52.2 / 61.9   57.2 / 66.9   208 / 210
    //      8      21.3 / 22.6   33.4 / 35.7   39.7 / 37.6   121 / 125
    //      4      18.8 / 19.5   29.4 / 27.3   33.5 / 27.6    87 /  81
    const int fill = pl.cus * (WAVES == 8 ? 1 : BITS == 4 ? 3 : 2), blocks = pl.blocks < fill ? pl.blocks : fill;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * WAVES), bytes(most, a.requests, blocks), stream, a);
    return hipGetLastError();
}

}  // namespace

DecodePlan plan_attn_decode(int64_t requests, int heads, int kv_heads, int head_dim, int64_t max_tokens, int cus) {
    DecodePlan p{};
    p.cus = cus;
    p.shared = heads / kv_heads;
    p.head_tiles = (p.shared + 15) / 16;
    // (units are counted in 32 bits)
    const int64_t longest = (max_tokens + kStep * 4 - 1) / (kStep * 4) * kv_heads * p.head_tiles;
    p.at_once = (int)(0x7FFFFFFF / longest < kMaxRequests ? 0x7FFFFFFF / longest : kMaxRequests);
    if (p.at_once < 1) p.at_once = 1;
    const int64_t groups = (requests < p.at_once ? requests : p.at_once) * kv_heads * p.head_tiles;
    p.waves = groups < kFewGroups ? 8 : 4;
    const int64_t unit = kStep * p.waves, most_blocks = (int64_t)cus * (p.waves == 8 ? 1 : 3);
    // no more blocks than there are groups, or units if all requests are as long as they may be
    const int64_t units = (max_tokens + unit - 1) / unit, useful = units < kWholeUnits ? groups : groups * units;
    p.blocks = (int)(useful < most_blocks ? useful : most_blocks);
    if (max_tokens > unit) {
        const int most = p.shared < 16 ? p.shared : 16;
        p.words_bytes = (size_t)groups * kWordBytes;
        p.workspace = p.words_bytes + (size_t)p.blocks * 2 * most * (head_dim + 2) * sizeof(float);
    }
    return p;
}

hipError_t launch_attn_decode(const Rows& q, const any4_kv_cache& c, const int32_t* table, int64_t table_stride, int64_t table_width,
                              const int32_t* lengths, int64_t requests, int heads, int window, int sinks, float softmax_scale, uint16_t* out,
                              const DecodePlan& pl, void* workspace, hipStream_t stream) {
    DecodeArgs a{q, kv_pages(c), table, table_stride, (int)table_width, lengths, 0, heads, pl.shared, pl.head_tiles, window, sinks, softmax_scale * kLog2e, out,
                 nullptr, static_cast<uint8_t*>(workspace)};
    a.partial = reinterpret_cast<float*>(a.words + pl.words_bytes);
    auto windows = [&](auto bits, auto f16, auto dim, auto waves) {
        constexpr int BITS = decltype(bits)::value, D = decltype(dim)::value, WAVES = decltype(waves)::value;
        return window > 0 ? launch<BITS, D, decltype(f16)::value, WAVES, true>(a, pl, stream) : launch<BITS, D, decltype(f16)::value, WAVES, false>(a, pl, stream);
    };
    auto waves = [&](auto bits, auto f16, auto dim) {
        return pl.waves == 8 ? windows(bits, f16, dim, std::integral_constant<int, 8>{}) : windows(bits, f16, dim, std::integral_constant<int, 4>{});
    };
    auto dims = [&](auto bits, auto f16) {
        return c.head_dim == 128 ? waves(bits, f16, std::integral_constant<int, 128>{}) : waves(bits, f16, std::integral_constant<int, 64>{});
    };
    auto types = [&](auto bits) { return c.f16 ? dims(bits, std::true_type{}) : dims(bits, std::false_type{}); };
    hipError_t e = hipSuccess;
    for (int64_t r = 0; r < requests && e == hipSuccess; r += pl.at_once) {           // (one launch, but for thousands)
        a.requests = (int)(requests - r < pl.at_once ? requests - r : pl.at_once);
        a.q.p = q.p + r * q.token;
        a.table = table + r * table_stride;
        a.lengths = lengths + r;
        a.out = out + r * heads * c.head_dim;
        e = c.bits == 16 ? types(std::integral_constant<int, 16>{}) : c.bits == 8 ? types(std::integral_constant<int, 8>{}) : types(std::integral_constant<int, 4>{});
    }
    return e;
}

}  // namespace any4
