// Attention of a step's tokens over the paged cache of their requests.
//
//   s_j = scale (q . k_j),  out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)
//
// over the keys j that the token sees, in one pass with the running maximum m and
// the running sum of each row.  A row is a (token, query head) pair; the rows of one
// key head belong together, since they read the same keys.
//
// Both products are matrix instructions with the keys along the first axis of the
// first and the rows along its second, S^T = K Q^T, then O^T = V^T P^T: a lane holds
// the scores of one row, so maximum, exponential and rescaling are per lane, and
// the weights it computes are already the operand of the second product (its sum
// over the keys takes them in any order, as long as V^T comes in the same one).
// V^T is read from LDS by the transposing reads (ds_read_tr).
//
// Work is dealt in blocks of 64 keys.  A unit is one key head of one request and a
// tile of its rows; the blocks of all units, one behind the other and weighed by what
// they cost, are cut into equal ranges, one per workgroup, whatever the lengths are.
// A unit that is cut leaves a part (maximum, sum, O) per workgroup in the workspace,
// and the last workgroup to finish one joins them in order.  attend_plan_kernel finds
// where each range starts.  Short tiles of a long launch are taken from a queue at the
// ends of the ranges, each as a whole.
//
// Two kinds of unit, each with an inner loop of its own:
//   tile unit   128 rows; the workgroup's four waves take 32 rows each and share K
//               and V in LDS (chunks of a prompt: the matrix units are the bound)
//   row unit    16 or 32 rows; the waves take keys of their own (decode and drafted
//               tokens, where the cache is read once and memory is the bound)
// A launch whose requests all have few rows is of row units alone; in any other, the
// requests that do have few go as row units among the tiles.
#include "common.hpp"
#include "kernels.hpp"
#include "launch.hpp"
#include "paged.hpp"

namespace xmix {

template <>
struct ArgPointers<AttendIn> {
    static std::vector<uint16_t> offsets() {
        return {offsetof(AttendIn, q), offsetof(AttendIn, cu), offsetof(AttendIn, kv_len),
                offsetof(AttendIn, out), offsetof(AttendIn, lse), offsetof(AttendIn, err_word),
                offsetof(AttendIn, T_valid)};
    }
};

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));

constexpr int kAttendThreads = 256, kAttendWaves = 4;
constexpr int kBlockKeys = 64;     // keys of a block
constexpr int kGroupKeys = 16;     // keys that surely lie in one page
constexpr int kTileRows = 128;     // rows of a tile unit
constexpr int kFewRows = 16;       // rows of a request that are a row unit among tiles
constexpr int kMaxRequests = 4096, kMaxRanges = 512;
constexpr int kPlanThreads = 1024;
constexpr int kPlanRanges = 8;     // of one workgroup, and the start of the next one's
constexpr int kTilesEach = 4;      // tiles of a request that one thread walks over
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
// A running maximum is raised only by a score this far above it (powers of two): the
// weights stay below 2^8, which neither fp32 sums nor bf16 weights mind, and the
// rescaling of O, rare after the first blocks, is skipped by a wave vote.
constexpr float kRaise = 8.0f;

// A workgroup's range, for the workgroup of that index in the launch: places counted
// in blocks over all units.
struct WorkRange {
    int64_t at;                      // place of the unit it begins in
    int64_t end;                     // where it ends
    int64_t share;                   // places of a range before its ends were moved
    int32_t req, head, tile, block;  // the unit, and its block that is the first
    int32_t lo, n, len;              // the request's span and keys
    int32_t nth;                     // its place among the ranges
    int32_t queued;                  // units of the launch in the queue
};
// What is dealt: a unit's place is `extra` for what it costs beside its blocks (its
// queries, the first copies, its rows), then `step` for each block (`few_step` where
// a request of a launch of tiles has few rows).
struct Deal {
    int32_t rows;                   // of a unit
    int32_t extra, step, few_step;
    int32_t least;                  // places of a range, at least a step: no range between
                                    // the first and the last of a unit is without a block
    int32_t whole;                  // tiles of so many blocks are not cut
    int32_t small;                  // leading tiles of so many blocks are not dealt but
    int32_t queue_from;             // queued, in launches of so many places a workgroup
};
// A block of a tile takes half as long again as one of a row unit (1.4 us and 0.9 us
// at head_dim 64, two workgroups on a CU), a unit's own cost is 6 to 8 us.  The numbers
// were found at head_dim 64 and 128 in bf16; us with others, at every width and type:
//   extra of a row unit (256 requests of up to 8192 keys)      2     4     8
//     head_dim 64, bf16 and e4m3                         344 186  335 182  338 175
//     128, bf16 and e4m3 (24 requests of up to 65536)    640 321  642 320  667 320
//     256, bf16 and e4m3                                 629 385  628 366  642 368
//     128, bf16, one request of 1024 keys                  18.0     15.5    15.6
//   extra of a tile                                            6     9    14
//     sixteen prompts, 128, bf16 and e4m3                139 136  138 136  138 137
//     the same at 256                                    109 108  109 108  108 108
//     95 single tokens and a chunk, 64, bf16 and e4m3    128 132  127 133  127 134
//     the same at 256, bf16                                 258     246     256
//   few_step (the single tokens and the chunk)                 1     2     4
//     64, bf16 and e4m3                                  129 120  127 133  156 127
//     256, bf16                                             333     246     295
// One set serves them within 5 %, but for single tokens among tiles in e4m3.
// Of a long launch of tiles the short units that lead each request (the first tokens of
// a prompt) are left for whoever ends its range first: sixteen prompts 153 -> 142 us,
// one of 2000 tokens 138 -> 119.  A short launch would pay for the queue's round trips
// (one prompt of 40 tokens 15.5 -> 20.4), and row units in it leave the matrix units
// idle at the end (95 single tokens and a chunk 128 -> 138).
constexpr Deal kDealRows = {0, 4, 1, 1, 4, 0, 0, 0}, kDealTiles = {kTileRows, 9, 3, 2, 3, 18, 4, 32};
__host__ __device__ constexpr Deal deal_of(int32_t rows) {
    Deal d = rows == kTileRows ? kDealTiles : kDealRows;
    d.rows = rows;
    return d;
}
// The workspace: a range per workgroup, a count of finished parts per range that
// begins a cut unit, the queue, and two parts per range.  The queue: how many of its
// units are taken; from kQueueHead on how many units there are up to each request
// (R_max + 1 numbers); then each request's leading tiles that are in it (R_max).
struct AttendWs {
    WorkRange* range;
    int32_t* done;
    int32_t* queue;
    float* parts;
};
constexpr int kQueueHead = 4;
template <>
struct ArgPointers<AttendWs> {
    static std::vector<uint16_t> offsets() {
        return {offsetof(AttendWs, range), offsetof(AttendWs, done), offsetof(AttendWs, queue),
                offsetof(AttendWs, parts)};
    }
};

// ------------------------------------------------------------------- geometry

// a / b of numbers that are not negative: 64 bits are divided in some 150 instructions,
// and few batches need them.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// A value that nothing writes during the launch, at a uniform place: a scalar load,
// which waits for no vector load before it (a page id behind the copies of the
// block before would wait for all of them).
template <typename T>
__device__ __forceinline__ T scalar_load(const T* p) {
    return *(const __attribute__((address_space(4))) T*)reinterpret_cast<uintptr_t>(p);
}

// A request's span and keys; n = 0 where it has no rows to write.  Of a span that runs
// past the valid tokens the ones before stay, at their positions (len is then the key
// count up to the last of them, and negative where none of them has a key).
struct Span {
    int32_t lo, n, len;
};
__device__ __forceinline__ Span span_of(const AttendIn& in, const KvCacheIn& c, int32_t lo, int32_t hi,
                                        int32_t len, bool* bad = nullptr) {
    Span s{lo, 0, len};
    if (lo < 0 || hi < lo || hi > in.T_max) {
        if (bad) *bad = true;
        return s;
    }
    if (hi == lo) return s;
    if (hi - lo > in.max_q || len < 0 || len > c.max_pages << c.page_log2) {
        if (bad) *bad = true;
        return s;
    }
    const int32_t end = in.T_valid ? min(hi, scalar_load(in.T_valid)) : hi;
    if (end <= lo) return s;
    s.n = end - lo;
    s.len = len - (hi - end);
    return s;
}
__device__ __forceinline__ Span span_of(const AttendIn& in, const KvCacheIn& c, int32_t r, bool* bad = nullptr) {
    return span_of(in, c, in.cu[r], in.cu[r + 1], in.kv_len[r], bad);
}
// The same of a uniform request.
__device__ __forceinline__ Span scalar_span(const AttendIn& in, const KvCacheIn& c, int32_t r) {
    return span_of(in, c, scalar_load(in.cu + r), scalar_load(in.cu + r + 1), scalar_load(in.kv_len + r));
}
// A uniform value in a scalar register, where the compiler has put it in a vector one
// (a resource made of it would be rebuilt lane by lane).
__device__ __forceinline__ int32_t scalar(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }
// A request whose rows are a row unit's in a launch of tiles.
__device__ __forceinline__ bool few_rows(int32_t n, const HeadGroup& group) { return n * group.n <= kFewRows; }
__device__ __forceinline__ int32_t tiles_of(int32_t n, const HeadGroup& group, int32_t rows) {
    return static_cast<int32_t>((static_cast<uint32_t>(n) * group.n + rows - 1) / rows);
}
// The keys that some row of tile t sees, in blocks: [first, first + count), one block
// at least (a tile without a key still has rows to write).
struct Blocks {
    int32_t first, count;
};
__device__ __forceinline__ Blocks blocks_of(const Span& s, int32_t t, const HeadGroup& group, int32_t rows,
                                            int32_t window) {
    const int32_t tok0 = group.div(t * rows), tok1 = min(group.div((t + 1) * rows - 1), s.n - 1);
    const int32_t hi = s.len - s.n + tok1 + 1, p0 = s.len - s.n + tok0;
    const int32_t lo = window > 0 && p0 >= window ? p0 - window + 1 : 0;
    const int32_t first = hi > 0 ? lo / kBlockKeys : 0;
    const int32_t end = hi > 0 ? (hi - 1) / kBlockKeys + 1 : 1;  // (hi may be next to 2^31)
    return {first, end - first};
}

// ----------------------------------------------------------------------- plan

__device__ __forceinline__ int64_t wave_sum64(int64_t v) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Blocks of each request, their prefix, then the start of every range by a search in
// the prefix and among the request's tiles.  Where no request can have more than
// kTilesEach tiles, one workgroup with a thread a request and a thread a range; where
// one may (MANY), a wave for each that does and a wave a range, with as many
// workgroups as there are ranges for (all find the same prefix): walking over 64 tiles
// a thread took 25 us on the one CU.  Chains of round trips and of 64-bit divisions
// are what it costs (spans in LDS and short divisions saved 3 us of 11 in a batch of 96
// requests, before the queue).  In a trace it takes 5 us for one request, 8 for 256 of
// one token, and 12 to 13 in the form for many tiles, for 96 requests, 16 or one.
//
// A range that would begin inside a short tile unit (up to `whole` blocks) begins at
// the nearer end of it instead: its parts would take their way through memory, 64 KB
// each, and sixteen prompts of 128 to 1024 tokens took 245 us with every end cut and
// 211 so.
template <bool MANY, bool TILES>
__global__ void __launch_bounds__(kPlanThreads)
attend_plan_kernel(AttendIn in, KvCacheIn cache, AttendWs ws, Deal deal, int32_t n_wg) {
    __shared__ Span spans[kMaxRequests];
    __shared__ int64_t upto[kMaxRequests + 1], begins[kMaxRanges + 1];
    __shared__ int64_t wave_total[kPlanThreads / kWave];
    __shared__ uint64_t tile_ranges[kMaxRanges / kWave];
    constexpr int kQueued = TILES ? kMaxRequests : 0;
    __shared__ int32_t queued[kQueued + 1];       // units in the queue up to a request
    __shared__ int32_t wave_queued[kPlanThreads / kWave];
    __shared__ uint8_t lead[kQueued + 1];         // a request's tiles in the queue, of each head,
    __shared__ int32_t lead_places[kQueued + 1];  // and their places
    __shared__ uint16_t many[MANY ? kMaxRequests : 1];  // requests of many tiles
    __shared__ int n_many;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t R = cache.R_max;
    const HeadGroup group = in.group;
    const int32_t rows = deal.rows, extra = deal.extra;
    auto step_of = [&](int32_t n) { return few_rows(n, group) ? deal.few_step : deal.step; };
    auto count_of = [&](const Span& s, int32_t t) { return blocks_of(s, t, group, rows, in.window).count; };
    auto small_of = [&](int32_t n) { return few_rows(n, group) ? 0 : deal.small; };
    if (MANY && tid == 0) n_many = 0;
    __syncthreads();
    bool bad = false;
    for (int32_t r = tid; r < R; r += kPlanThreads) {
        const Span s = span_of(in, cache, r, &bad);
        spans[r] = s;
        const int32_t tiles = tiles_of(s.n, group, rows), step = step_of(s.n);
        if (MANY && tiles > kTilesEach) {
            many[atomicAdd(&n_many, 1)] = static_cast<uint16_t>(r);
            continue;
        }
        const int32_t small = small_of(s.n);
        int64_t sum = 0, led = 0;
        int32_t n = 0;
        for (int32_t t = 0; t < tiles; ++t) {
            const int32_t count = count_of(s, t), places = count * step + extra;
            if (TILES && n == t && count <= small) {
                ++n;
                led += places;
            }
            sum += places;
        }
        upto[r + 1] = sum * cache.n_kv;
        if constexpr (TILES) {
            lead[r] = static_cast<uint8_t>(n);
            lead_places[r] = static_cast<int32_t>(led);
        }
    }
    if constexpr (MANY) {
        __syncthreads();
        for (int32_t i = wave; i < n_many; i += kPlanThreads / kWave) {
            const int32_t r = many[i];
            const Span s = spans[r];
            const int32_t tiles = tiles_of(s.n, group, rows), step = step_of(s.n);
            const uint64_t large = wave_ballot(lane >= tiles || count_of(s, lane) > small_of(s.n));
            const int32_t n = large ? __builtin_ctzll(large) : kWave;
            int64_t sum = 0, led = 0;
            for (int32_t t = lane; t < tiles; t += kWave) {
                const int32_t places = count_of(s, t) * step + extra;
                sum += places;
                if (t < n) led += places;
            }
            sum = wave_sum64(sum);
            led = wave_sum64(led);
            if (lane == 0) {
                upto[r + 1] = sum * cache.n_kv;
                lead[r] = static_cast<uint8_t>(n);
                lead_places[r] = static_cast<int32_t>(led);
            }
        }
    }
    if (bad && blockIdx.x == 0) atomicOr(in.err_word, kErrKvSpan);
    if (tid == 0) upto[0] = queued[0] = 0;
    __syncthreads();
    // prefix over the requests, four to a thread
    constexpr int kEach = kMaxRequests / kPlanThreads;
    if constexpr (TILES) {  // whether the launch is long enough for a queue
        int64_t mine = 0;
        for (int i = 0; i < kEach; ++i)
            if (tid * kEach + i < R) mine += upto[tid * kEach + i + 1];
        mine = wave_sum64(mine);
        if (lane == 0) wave_total[wave] = mine;
        __syncthreads();
        int64_t all = 0;
        for (int w = 0; w < kPlanThreads / kWave && w * kWave * kEach < R; ++w) all += wave_total[w];
        const bool queue = all >= static_cast<int64_t>(deal.queue_from) * n_wg;
        for (int i = 0; i < kEach; ++i) {
            const int32_t r = tid * kEach + i;
            if (r >= R) break;
            if (queue) upto[r + 1] -= static_cast<int64_t>(lead_places[r]) * cache.n_kv;
            else lead[r] = 0;
        }
        __syncthreads();
    }
    int64_t v[kEach], sum = 0;
    int32_t q[kEach], q_sum = 0;
    for (int i = 0; i < kEach; ++i) {
        const int32_t r = tid * kEach + i;
        sum += r < R ? upto[r + 1] : 0;
        v[i] = sum;
        if constexpr (TILES) q_sum += r < R ? lead[r] * cache.n_kv : 0;
        q[i] = q_sum;
    }
    int64_t incl = sum;
    int32_t q_incl = q_sum;
    for (int o = 1; o < kWave; o <<= 1) {
        const int64_t up = __shfl_up(incl, o);
        const int32_t q_up = TILES ? __shfl_up(q_incl, o) : 0;
        if (lane >= o) {
            incl += up;
            q_incl += q_up;
        }
    }
    if (lane == kWave - 1) {
        wave_total[wave] = incl;
        wave_queued[wave] = q_incl;
    }
    __syncthreads();
    int64_t before = incl - sum;
    int32_t q_before = q_incl - q_sum;
    for (int w = 0; w < wave && w * kWave * kEach < R; ++w) {
        before += wave_total[w];
        q_before += wave_queued[w];
    }
    for (int i = 0; i < kEach; ++i)
        if (tid * kEach + i < R) {
            upto[tid * kEach + i + 1] = before + v[i];
            if constexpr (TILES) queued[tid * kEach + i + 1] = q_before + q[i];
        }
    __syncthreads();
    if (TILES && blockIdx.x == 0) {
        if (tid == 0) ws.queue[0] = 0;
        for (int32_t r = tid; r <= R; r += kPlanThreads) ws.queue[kQueueHead + r] = queued[r];
        for (int32_t r = tid; r < R; r += kPlanThreads) ws.queue[kQueueHead + R + 1 + r] = lead[r];
    }
    const int64_t places = upto[R];
    const int64_t share = max(static_cast<int64_t>(deal.least), quotient(places + n_wg - 1, n_wg));
    // The last request that starts at or before a place.
    auto request_at = [&](int64_t at) {
        int32_t lo = 0, hi = R - 1;
        while (lo < hi) {
            const int32_t mid = (lo + hi + 1) >> 1;
            if (upto[mid] <= at) lo = mid;
            else hi = mid - 1;
        }
        return lo;
    };
    // The unit and its block at position `at` (uniform where MANY), and the unit's blocks.
    auto locate = [&](int64_t at, int32_t* count) {
        const int32_t lo = request_at(at);
        const Span s = spans[lo];
        const int64_t a_head = quotient(upto[lo + 1] - upto[lo], cache.n_kv), rest = at - upto[lo];
        const int32_t head = static_cast<int32_t>(quotient(rest, a_head));
        WorkRange st{at, 0, share, lo, head, TILES ? lead[lo] : 0, 0, s.lo, s.n, s.len, 0, 0};
        int64_t left = rest - head * a_head;
        const int32_t tiles = tiles_of(s.n, group, rows), step = step_of(s.n);
        *count = 1;
        if constexpr (MANY) {  // 64 tiles at a time
            for (; st.tile < tiles; st.tile += kWave) {
                const int32_t t = st.tile + lane;
                const int32_t mine = t < tiles ? count_of(s, t) : 0;
                int64_t incl = t < tiles ? mine * step + extra : 0;
                for (int o = 1; o < kWave; o <<= 1) {
                    const int64_t up = __shfl_up(incl, o);
                    if (lane >= o) incl += up;
                }
                const uint64_t beyond = wave_ballot(incl > left);
                if (beyond) {
                    const int first = __builtin_ctzll(beyond);
                    if (first > 0) left -= __shfl(incl, first - 1);
                    *count = __shfl(mine, first);
                    st.tile += first;
                    break;
                }
                left -= __shfl(incl, kWave - 1);
            }
        } else {
            for (; st.tile < tiles; ++st.tile) {
                *count = count_of(s, st.tile);
                if (left < *count * step + extra) break;
                left -= *count * step + extra;
            }
        }
        st.at -= left;  // the unit's own
        st.block = (max(0, static_cast<int32_t>(left) - extra) + step - 1) / step;
        return st;
    };
    auto begin_of = [&](int32_t w) {
        WorkRange st{places, 0, share, 0, 0, 0, 0, 0, 0, 0, 0, 0};
        int32_t count;
        if (w * share < places) {
            st = locate(w * share, &count);
            const int32_t step = step_of(st.n);
            const bool uncut = count <= deal.whole && !few_rows(st.n, group);
            if (st.block == count || (uncut && st.block != 0)) {
                const bool next = 2 * st.block > count;
                st.block = 0;
                if (next) st.at += count * step + extra;
                if (next && st.at < places) st = locate(st.at, &count);
            }
        }
        return st;
    };
    // The workgroups are dealt over the XCDs in turn, workgroup b to XCD b % 8.
    // Neighbouring ranges, which read the same keys, go to one XCD and its L2, and few
    // ranges still to all of them; but tiles, which keep the matrix units busy, and
    // rows, which wait for memory, are spread over the XCDs each on their own, the
    // tiles first, such that a CU, whose second workgroup is 32 behind its first, has
    // both: 95 single tokens and a chunk of 1001 took 134 us so, 140 with the ranges
    // in their order and 161 with the rows first.
    const int32_t used = static_cast<int32_t>(min(static_cast<int64_t>(n_wg), quotient(places + share - 1, share)));
    const int32_t each = (used + 7) / 8;
    if constexpr (TILES) {
        if (tid < kMaxRanges) {
            bool tile = false;
            if (tid < used) {
                const int32_t r = request_at(tid * share);
                tile = !few_rows(spans[r].n, group);
            }
            const uint64_t mask = wave_ballot(tile);
            if (lane == 0) tile_ranges[wave] = mask;
        }
        __syncthreads();
    }
    auto workgroup_of = [&](int32_t w) {
        if (w >= 8 * each) return w;
        if (!TILES) return w / each + 8 * (w % each);
        int32_t before = 0, all = 0;  // ranges of tiles
        for (int32_t i = 0; i < kMaxRanges / kWave; ++i) {
            const uint64_t mask = tile_ranges[i];
            all += __popcll(mask);
            const int32_t n = min(max(w - i * kWave, 0), kWave);
            before += __popcll(n == kWave ? mask : mask & ((1ull << n) - 1));
        }
        const bool tile = (tile_ranges[w / kWave] >> (w % kWave)) & 1u;
        for (int32_t x = 0;; ++x) {  // XCD x: `each` ranges, of them an eighth of the tiles
            const int32_t t0 = x * all / 8, t1 = (x + 1) * all / 8;
            const int32_t at = tile ? before - t0 : w - before - (x * each - t0);
            const int32_t n = tile ? t1 - t0 : each - (t1 - t0);
            if (at < n || x == 7) return x + 8 * (tile ? at : t1 - t0 + at);
        }
    };
    // this workgroup's ranges, and where the one behind them begins
    const int32_t per = n_wg / gridDim.x, w0 = blockIdx.x * per;
    auto note_begin = [&](int32_t i, const WorkRange& st) {
        const int32_t step = step_of(st.n);
        begins[i] = st.at + (st.block ? extra + st.block * step : 0);
    };
    auto put_range = [&](int32_t i, WorkRange st) {
        const int32_t w = w0 + i;
        ws.done[w] = 0;
        st.end = begins[i + 1];
        if (begins[i] == st.end) st.end = st.at;  // nothing to do
        st.nth = w;
        st.queued = TILES ? queued[R] : 0;
        ws.range[workgroup_of(w)] = st;
    };
    if constexpr (MANY) {  // a wave a range
        WorkRange st;
        if (wave <= per) {
            st = begin_of(w0 + wave);
            if (lane == 0) note_begin(wave, st);
        }
        __syncthreads();
        if (wave < per && lane == 0) put_range(wave, st);
    } else {  // a thread a range
        WorkRange st;
        if (tid <= per) {
            st = begin_of(w0 + tid);
            note_begin(tid, st);
        }
        __syncthreads();
        if (tid < per) put_range(tid, st);
    }
}

// ------------------------------------------------------------- cached values

// Rows of one head of the cache in LDS: how the 16-byte pieces of a row are permuted
// (the copies into LDS place each piece linearly, so it is the source address that
// is permuted), such that the lanes of one read cover all banks.
//   K (both kinds): 16 lanes read one piece each of 16 rows
//   V: the transposing reads take 4 rows of 32 bytes (bf16) or 8 of 16 bytes (e4m3)
//   per 16 lanes; which rows and columns 32 lanes take differs between the kinds
template <int RB>
__device__ __forceinline__ int swz_k(int row) {
    constexpr int per = RB >= 256 ? 1 : 256 / RB, mask = RB >= 256 ? 15 : RB / 16 - 1;
    return (row / per) & mask;
}
template <int RB, bool E4M3>
__device__ __forceinline__ int swz_v_tile(int row) {
    if constexpr (!E4M3) return RB >= 256 ? (row & 3) << 2 : ((row >> 1) & 1) << 2;
    else if constexpr (RB >= 256) return (row & 3) << 1 | ((row >> 3) & 1) << 3;
    else if constexpr (RB == 128) return ((row >> 1) & 1) << 1 | ((row >> 3) & 1) << 2;
    else return ((row >> 3) & 1) << 1;
}
template <int RB, bool E4M3>
__device__ __forceinline__ int swz_v_row(int row) {
    if constexpr (!E4M3) return RB >= 256 ? (row & 7) << 1 : ((row >> 1) & 3) << 1;
    else if constexpr (RB >= 256) return (row & 7) | ((row >> 4) & 1) << 3;
    else if constexpr (RB == 128) return ((row >> 1) & 3) | ((row >> 4) & 1) << 2;
    else return ((row >> 2) & 1) | ((row >> 4) & 1) << 1;
}

// A buffer resource over the rows of one head that hold the keys from `key` on, of
// at most 16 (one page): past the request's last key, and in a page that is not
// there, it reads zeros and touches no memory.
template <int RB>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t group_rows(const void* base, const KvCacheIn& c,
                                                             int32_t page, int32_t head,
                                                             int32_t key, int32_t len) {
    const bool ok = page_ok(c, page);
    const int64_t row = page_row(c, ok ? page : 0, head, key & ((1 << c.page_log2) - 1));
    const int32_t live = scalar(ok ? max(0, min(kGroupKeys, len - key)) : 0);
    return __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>(static_cast<const char*>(base)) + row * RB, 0, live * RB, kBufferDword3);
}
// The page ids of the groups of 16 keys from key0 on, one per lane from lane 0 (past
// the request's last key, that one's).  They are loaded a step before they are needed,
// by a vector load, which completes in order with the copies around it; a scalar load
// would make every wait for LDS one for everything.
// A key0 past the last one may be past 2^31 too.
__device__ __forceinline__ int32_t page_ids(const KvCacheIn& c, int32_t req, uint32_t key0, int32_t len,
                                            int groups) {
    const uint32_t key = key0 + (lane_id() & (groups - 1)) * kGroupKeys;
    const uint32_t nth = min(key, static_cast<uint32_t>(max(0, len - 1))) >> c.page_log2;
    return (c.pages + static_cast<int64_t>(req) * c.max_pages)[nth];
}
// The groups whose page is not there, as bits.
__device__ __forceinline__ uint32_t groups_gone(const KvCacheIn& c, int32_t ids, int groups) {
    return static_cast<uint32_t>(wave_ballot(!page_ok(c, ids))) & ((1u << groups) - 1);
}

// Whether a missing group (`gone`, of the block from key0 on) has a key that rows at the
// positions p_first to p_last see.  A block begins at a multiple of its keys: the pages
// wholly behind a window may have been given away.
__device__ __forceinline__ bool gone_seen(uint32_t gone, int32_t key0, int32_t p_first, int32_t p_last,
                                          int32_t window) {
    if (p_last < key0) return false;
    const int32_t from = window > 0 && p_first >= window ? p_first - window + 1 : 0;
    const int32_t a = max(from - key0, 0) / kGroupKeys, b = min(p_last - key0, kBlockKeys - 1) / kGroupKeys;
    return a <= b && (gone & ((2u << b) - (1u << a))) != 0;
}

// An offset that the compiler computes from here on anew: a tile's reads differ by an
// exclusive or with a constant (the permutation of the pieces), one instruction each,
// and kept apart would hold a register each through the whole loop.
__device__ __forceinline__ int fresh(int off) {
    asm volatile("" : "+v"(off));
    return off;
}
__device__ __forceinline__ const uint4* at_bytes(const uint4* p, int off) {
    return reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) + off);
}

// Operands read from LDS are taken kAhead reads before their use, in an order that
// this fixes: left to itself the compiler reads each one right before its matrix
// instruction and waits for it.
constexpr int kAhead = 4;
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0); }

typedef __attribute__((address_space(3))) void* lds_ptr;
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4;
typedef __attribute__((address_space(3))) i32x2_t* lds_i32x2;

// Sixteen bytes per lane from `off` bytes into the resource to dst (uniform) + lane.
constexpr int kOnce = 2;  // the nt bit of a buffer access: bytes that nobody reads again
template <int AUX = 0>
__device__ __forceinline__ void copy16(__amdgpu_buffer_rsrc_t r, uint4* dst, int32_t off) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr)dst, 16, off, 0, 0, AUX);
}
// Waits until at most n of this wave's vector loads and copies are outstanding.
template <int n>
__device__ __forceinline__ void wait_all_but() {
    __builtin_amdgcn_s_waitcnt((n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14));
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ bf16x8_t as_bf16x8(const uint4& v) {
    return __builtin_bit_cast(bf16x8_t, v);
}
// Eight e4m3 values, exactly.
__device__ __forceinline__ bf16x8_t e4m3_to_bf16(int lo, int hi) {
    uint4 w;
    w.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
    w.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
    w.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
    w.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
    return as_bf16x8(w);
}
// What a product q . k is multiplied by, for powers of two.  Where it leaves fp32's range
// it is the least or the largest number there: zero would make NaN of a masked score
// (-inf), an infinity of a product of zero.
__device__ __forceinline__ float score_scale(float scale, float k_scale) {
    const float c = scale * k_scale * kLog2e;
    return c == 0.0f ? 0x1p-149f : c == INFINITY ? 0x1.fffffep127f : c;
}
// Weights to bf16, nearest even, at most 2^-8 of each: the matrix instructions take both
// operands in one type, and a second one for what is cut off would be half as many again.
// The sum over many keys averages it out: the result's relative error (its norm) is 0.0020
// to 0.0023, of which its own rounding alone makes 0.0017.  The sum of the weights keeps
// them in fp32.
__device__ __forceinline__ uint32_t weights2(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{a, b}, bf16x2_t));
}

// Both halves' (lanes l and l ^ 32), and all four quarters', largest and sum.
__device__ __forceinline__ float half_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float quarter_max(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quarter_sum(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Values that are not finite.  A masked key's weight is zero, and zero times an
// infinity or NaN is not nothing.  Where O comes out not finite, the unit is done
// again ("careful"): each V tile is made finite in LDS first, its columns' keys of
// +inf (or NaN) and -inf (or NaN) go into 64-bit masks, and each row that sees one of
// them notes the column; the notes become infinities when the rows are stored.
struct OddKeys {
    uint64_t up, down;
};
// Takes the odd values out of one piece (bf16, or e4m3, which has NaN alone) of the
// tile at `piece`; `cols` are the masks of its columns, `key` the tile's key.
template <bool E4M3>
__device__ __forceinline__ void take_odd(uint4* piece, OddKeys* cols, int key) {
    constexpr int n = E4M3 ? 16 : 8;
    uint32_t* w = reinterpret_cast<uint32_t*>(piece);
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        const int sh = E4M3 ? 8 * (i & 3) : 16 * (i & 1), at = E4M3 ? i >> 2 : i >> 1;
        const uint32_t x = (w[at] >> sh) & (E4M3 ? 0xFFu : 0xFFFFu);
        const bool odd = E4M3 ? (x & 0x7Fu) == 0x7Fu : (x & 0x7F80u) == 0x7F80u;
        if (!odd) continue;
        const bool nan = E4M3 || (x & 0x7Fu);
        w[at] &= ~((E4M3 ? 0xFFu : 0xFFFFu) << sh);
        if (nan || !(x & 0x8000u)) atomicOr(reinterpret_cast<unsigned long long*>(&cols[i].up), 1ull << key);
        if (nan || (x & 0x8000u)) atomicOr(reinterpret_cast<unsigned long long*>(&cols[i].down), 1ull << key);
    }
}
// The notes of a unit's rows: a bit per column, of the two kinds.
template <int M, int HD>
struct OddNotes {
    uint32_t bits[2][M][HD / 32];
    __device__ __forceinline__ void clear(int tid) {
        uint32_t* w = &bits[0][0][0];
        for (int i = tid; i < 2 * M * HD / 32; i += kAttendThreads) w[i] = 0;
    }
    // Row `row` sees the keys `see` of the tile whose columns' masks are `cols`.
    __device__ __forceinline__ void note(int kind, int row, uint64_t see, const OddKeys* cols) {
#pragma unroll 1
        for (int c = 0; c < HD; ++c)
            if ((kind ? cols[c].down : cols[c].up) & see) atomicOr(&bits[kind][row][c / 32], 1u << (c % 32));
    }
    __device__ __forceinline__ float apply(float o, int row, int c) const {
        if ((bits[0][row][c / 32] >> (c % 32)) & 1u) o += INFINITY;
        if ((bits[1][row][c / 32] >> (c % 32)) & 1u) o -= INFINITY;
        return o;
    }
};
// The keys of a block of n (at most 64) from key0 on that a row sees.
__device__ __forceinline__ uint64_t seen_keys(int32_t key0, int32_t pos, int32_t window, uint32_t gone) {
    uint64_t see = pos < key0 ? 0 : pos - key0 >= 63 ? ~0ull : (2ull << (pos - key0)) - 1;
    if (window > 0 && pos - window >= key0) {
        const int32_t hidden = pos - window - key0;  // the last hidden one
        see = hidden >= 63 ? 0 : see & ~((2ull << hidden) - 1);
    }
    for (int g = 0; g < kBlockKeys / kGroupKeys; ++g)
        if ((gone >> g) & 1u) see &= ~(0xFFFFull << (kGroupKeys * g));
    return see;
}

// ------------------------------------------------------------- joining parts

constexpr int kThrough = 16;  // the sc1 bit of a buffer access: past the XCD's L2
__device__ __forceinline__ void store_through(__amdgpu_buffer_rsrc_t r, int off, float v) {
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r, off, 0, kThrough);
}
__device__ __forceinline__ void store_through(__amdgpu_buffer_rsrc_t r, int off, const f32x4_t& v) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), r, off, 0, kThrough);
}
__device__ __forceinline__ float load_through(__amdgpu_buffer_rsrc_t r, int off) {
    return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, off, 0, kThrough));
}
__device__ __forceinline__ f32x4_t load4_through(__amdgpu_buffer_rsrc_t r, int off) {
    return __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, kThrough));
}

// A part: the rows' maxima (powers of two, -inf: no key) and sums, then O [row][HD],
// with room for SLOT rows.
// Parts pass between XCDs, whose L2 caches do not see each other's writes: they are
// stored through to memory and loaded from there (sc1), which needs no fence.  An
// agent fence writes the whole L2 back, a good half microsecond each, one after the
// other: one request of 1024 keys took 37.8 us with them and 16.7 without.
template <int M, int HD, int SLOT>
struct Part {
    static constexpr int kFloats = SLOT * (HD + 2);
    __amdgpu_buffer_rsrc_t r;
    __device__ __forceinline__ Part(const AttendWs& ws, int32_t wg, bool opens) {
        float* p = ws.parts + (2 * static_cast<int64_t>(wg) + (opens ? 1 : 0)) * kFloats;
        r = __builtin_amdgcn_make_buffer_rsrc(p, 0, kFloats * 4, kBufferDword3);
    }
    __device__ __forceinline__ void put(int at, float v) const { store_through(r, at * 4, v); }
    __device__ __forceinline__ void put4(int at, const f32x4_t& v) const { store_through(r, at * 4, v); }
    __device__ __forceinline__ float get(int at) const { return load_through(r, at * 4); }
    __device__ __forceinline__ f32x4_t get4(int at) const { return load4_through(r, at * 4); }
};

// The rows of a unit in the caller's tensors.
struct RowsOut {
    int32_t lo, n_rows, row0, head;  // first token of the span; its rows; the tile's first
    HeadGroup group;
};
__device__ __forceinline__ uint16_t* out_row(const AttendIn& in, const RowsOut& u, int32_t row,
                                             int hd) {
    const int32_t at = u.row0 + row, tok = u.group.div(at), g = at - tok * u.group.n;
    return in.out + (u.lo + tok) * in.out_stride + static_cast<int64_t>(u.head * u.group.n + g) * hd;
}
__device__ __forceinline__ void store_lse(const AttendIn& in, const RowsOut& u, int32_t row, float m,
                                          float l) {
    if (!in.lse) return;
    const int32_t at = u.row0 + row, tok = u.group.div(at), g = at - tok * u.group.n;
    in.lse[static_cast<int64_t>(u.head * u.group.n + g) * in.T_max + u.lo + tok] =
        l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}
__device__ __forceinline__ float weight_of(float m, float top) {
    return m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top);
}

// Joins the parts of a unit, kLoads of them in flight at a time.
template <int M, int HD, int SLOT, int kLoads>
__device__ __forceinline__ void join_rows(const AttendIn& in, const AttendWs& ws, const RowsOut& u,
                                          int32_t first, int32_t last, float v_scale) {
    constexpr int kVec = HD / 4;
    const int32_t rows = min(M, u.n_rows - u.row0);
    for (int32_t e = threadIdx.x; e < rows * kVec; e += kAttendThreads) {
        const int32_t row = e / kVec, c = e % kVec;
        float top = -INFINITY, l = 0.0f;
        f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int32_t w0 = first; w0 <= last; w0 += kLoads) {
            float m[kLoads], s[kLoads];
            f32x4_t x[kLoads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int32_t w = min(w0 + i, last);
                const Part<M, HD, SLOT> p(ws, w, w == first);
                m[i] = p.get(row);
                s[i] = p.get(M + row);
                x[i] = p.get4(2 * M + row * HD + 4 * c);
            }
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if (w0 + i > last) {  // (the last one again)
                    m[i] = -INFINITY;
                    s[i] = 0.0f;
                    x[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
                }
                const float top2 = fmaxf(top, m[i]);
                const float a = weight_of(top, top2), b = weight_of(m[i], top2);
                l = l * a + s[i] * b;
                o = o * a + x[i] * b;
                top = top2;
            }
        }
        const float inv = l == 0.0f ? 0.0f : v_scale / l;
        *reinterpret_cast<uint2*>(out_row(in, u, row, HD) + 4 * c) =
            make_uint2(weights2(o[0] * inv, o[1] * inv), weights2(o[2] * inv, o[3] * inv));
        if (c == 0) store_lse(in, u, row, top, l);
    }
}
// After this workgroup's part has reached memory (a wait by every wave, and a
// barrier): the last of the unit's workgroups joins the parts, in their order, and
// writes the rows.
template <int M, int HD, int SLOT>
__device__ void join_parts(const AttendIn& in, const AttendWs& ws, const RowsOut& u, int32_t first,
                           int32_t last, float v_scale, int* flag) {
    // (in the workspace also if a caller changes the lengths under the call)
    last = min(last, static_cast<int32_t>(gridDim.x) - 1);
    first = min(first, last);
    if (threadIdx.x == 0)
        *flag = __hip_atomic_fetch_add(ws.done + first, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                last - first;
    __syncthreads();
    if (!scalar(*flag)) return;
    if (last - first < 4 || M >= kTileRows) join_rows<M, HD, SLOT, 4>(in, ws, u, first, last, v_scale);
    else join_rows<M, HD, SLOT, 16>(in, ws, u, first, last, v_scale);
}

// This workgroup's range.
__device__ __forceinline__ WorkRange range_of(const AttendWs& ws) {
    const WorkRange* r = ws.range + blockIdx.x;
    return {scalar_load(&r->at), scalar_load(&r->end), scalar_load(&r->share), scalar_load(&r->req),
            scalar_load(&r->head), scalar_load(&r->tile), scalar_load(&r->block), scalar_load(&r->lo),
            scalar_load(&r->n), scalar_load(&r->len), scalar_load(&r->nth), scalar_load(&r->queued)};
}

// ------------------------------------------------------------------ tile units

// LDS of a workgroup, for units of either kind.
struct UnitLds {
    uint4 *a, *b;       // two steps of K and V (tiles) or of the waves' V (rows)
    OddKeys* odd_keys;  // a tile's columns, or the waves' own
    uint32_t* notes;
    float *wm, *wl;     // the waves' maxima and sums
    int *flag, *odd_unit;  // odd_unit: the last unit with values that are not finite
};

// `count` blocks from the range's on of a unit of 128 rows, whose first and last block
// are at the places `begin` and `last`.  A wave's 32 rows are one side of a 32 x 32
// product; K and V of a block come by copies into LDS, the block behind it while this
// one is multiplied, and every operand read from there serves 32 rows.
//
// The matrix units bound it: 4096 tokens over 32768 keys, 32 heads of 128, run at 930 to
// 960 TFLOP/s (2.15 to 2.22 ms, 52 % of the cycles in matrix instructions, at a clock of
// about 1.8 GHz; the library's plain product reaches 1249).  In e4m3, with a conversion
// of every operand and half the bytes, the same takes 2.1 to 2.2 ms; at head_dim 256, one
// workgroup on a CU and some registers spilled, 2.5.  With few blocks a unit its start
// bounds it, the chain from page id to copy to first product: sixteen prompts of up to
// 1024 tokens take 138 to 145 us, 480 to 500 TFLOP/s; with time stamps in the kernel,
// which make it 25 % slower, units of one block take 14 us there and of eight 25 to 28.
// The next unit's first copies issued before this one's rows are stored did not help
// (147 us before the queue, 147 to 159 so), the CU's second workgroup being at work
// meanwhile.
template <int HD, bool E4M3>
__device__ __forceinline__ void tile_unit(const AttendIn& in, const KvCacheIn& cache, const AttendWs& ws,
                                          const WorkRange& st, const Span& s, const Blocks& bl,
                                          int64_t begin, int64_t last, int32_t count, int unit, const UnitLds& lds) {
    constexpr int RB = HD * (E4M3 ? 1 : 2);      // bytes of a cached row
    constexpr int kTile = kBlockKeys * RB / 16;  // pieces of a block
    constexpr int kCopies = kGroupKeys * RB / 1024;
    constexpr int kSteps = HD / 16, kCols = HD / 32;
    uint4 *const kA = lds.a, *const vA = lds.a + kTile, *const kB = lds.b, *const vB = lds.b + kTile;
    auto& notes = *reinterpret_cast<OddNotes<kTileRows, HD>*>(lds.notes);
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, n32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const HeadGroup group = in.group;

    // this lane's sources within a group of 16 rows, and its reads of a block
    int32_t src_k[kCopies], src_v[kCopies];
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
        const int at16 = i * 64 + lane, row = at16 / (RB / 16), slot = at16 % (RB / 16);
        src_k[i] = row * RB + ((slot ^ swz_k<RB>(row)) * 16);
        src_v[i] = row * RB + ((slot ^ swz_v_tile<RB, E4M3>(row)) * 16);
    }
    // K: piece 2 i + half of row n32.  V: column block h of four (bf16) or eight keys.
    const int i16 = lane & 15, side = (lane >> 4) & 1;
    const int k_off = n32 * RB + ((half ^ swz_k<RB>(n32)) * 16);
    const int v_row = E4M3 ? 8 * (i16 >> 3) + 4 * half + ((i16 >> 1) & 3) : 4 * half + (i16 >> 2);
    const int v_piece = E4M3 ? side : 2 * side + ((i16 & 3) >> 1);
    const int v_off = v_row * RB + ((v_piece ^ swz_v_tile<RB, E4M3>(v_row)) * 16) + 8 * (i16 & 1);
    const RowsOut u{s.lo, s.n * group.n, st.tile * kTileRows, st.head, group};
    const float c2 = score_scale(in.scale, E4M3 ? scalar_load(cache.k_scale + st.head) : 1.0f);
    const float v_scale = E4M3 ? scalar_load(cache.v_scale + st.head) : 1.0f;
    // this lane's row, and the tokens of the wave's rows
    const int32_t row = u.row0 + wave * 32 + n32;
    const bool row_ok = row < u.n_rows;
    const int32_t tok = group.div(min(row, u.n_rows - 1));
    const int32_t base = s.len - s.n;
    const int32_t pos = base + tok;  // (rows past the last repeat it and are not stored)
    const int32_t wrow0 = u.row0 + wave * 32;
    const bool wave_on = wrow0 < u.n_rows;
    const int32_t p_first = base + group.div(min(wrow0, u.n_rows - 1));
    const int32_t p_last = base + group.div(min(wrow0 + 31, u.n_rows - 1));
    bf16x8_t Q[kSteps];
    {
        const uint16_t* qr = in.q + (u.lo + tok) * in.q_stride +
                             static_cast<int64_t>(u.head * group.n + min(row, u.n_rows - 1) - tok * group.n) * HD;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int c = E4M3 ? 4 * (i >> 1) + 2 * half + (i & 1) : 2 * i + half;
            Q[i] = as_bf16x8(reinterpret_cast<const uint4*>(qr)[c]);
        }
    }

    constexpr int kGroups = kBlockKeys / kGroupKeys;
    int32_t ids;        // of the block to be copied next
    uint32_t gone = 0;  // of the block whose turn it is
    auto load_ids = [&](int32_t block) __attribute__((always_inline)) {
        ids = page_ids(cache, st.req, static_cast<uint32_t>(block) * kBlockKeys, s.len, kGroups);
    };
    // Copies a block and asks for the ids of the one after it.
    auto stage = [&](int32_t block, uint4* kd, uint4* vd) __attribute__((always_inline)) {
        const int32_t key = block * kBlockKeys + wave * kGroupKeys;
        const int32_t page = __builtin_amdgcn_readlane(ids, wave);
        const uint32_t next_gone = groups_gone(cache, ids, kGroups);
        const __amdgpu_buffer_rsrc_t kr = group_rows<RB>(cache.k, cache, page, st.head, key, s.len);
        const __amdgpu_buffer_rsrc_t vr = group_rows<RB>(cache.v, cache, page, st.head, key, s.len);
#pragma unroll
        for (int i = 0; i < kCopies; ++i)
            copy16(kr, kd + wave * (kTile / 4) + i * 64, src_k[i]);
#pragma unroll
        for (int i = 0; i < kCopies; ++i)
            copy16(vr, vd + wave * (kTile / 4) + i * 64, src_v[i]);
        load_ids(block + 1);
        return next_gone;
    };

    float m, l;
    f32x16_t O[kCols];
    bool careful = false;
    // One block: scores, weights, O.
    auto block_step = [&](int32_t block, const uint4* kt, uint4* vt) __attribute__((always_inline)) {
        const int32_t key0 = block * kBlockKeys;
        if (careful) {
            for (int c = tid; c < HD; c += kAttendThreads) lds.odd_keys[c] = OddKeys{0, 0};
            __syncthreads();
            for (int e = tid; e < kTile; e += kAttendThreads) {
                const int kr = e / (RB / 16), slot = (e % (RB / 16)) ^ swz_v_tile<RB, E4M3>(kr);
                take_odd<E4M3>(vt + e, lds.odd_keys + slot * (E4M3 ? 16 : 8), kr);
            }
            __syncthreads();
            const int r = tid % kTileRows;
            notes.note(tid / kTileRows, r,
                       seen_keys(key0, base + group.div(min(u.row0 + r, u.n_rows - 1)), in.window, gone),
                       lds.odd_keys);
        }
        if (!wave_on || key0 > p_last) return;
        f32x16_t S[2] = {f32x16_t{}, f32x16_t{}};
        {
            constexpr int kReads = E4M3 ? kSteps : 2 * kSteps;  // a step of both halves of the keys
            const int ko = fresh(k_off);
            auto read_k = [&](int i) { return *at_bytes(kt + 32 * (i & 1) * (RB / 16), ko ^ (32 * (i >> 1))); };
            uint4 w[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) w[i] = read_k(i);
            keep_order();
#pragma unroll
            for (int i = 0; i < kReads; ++i) {
                const int b = i & 1, step = i >> 1;
                const uint4 x = w[i % kAhead];
                if constexpr (E4M3) {
                    S[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(e4m3_to_bf16(x.x, x.y), Q[2 * step], S[b], 0, 0, 0);
                    S[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(e4m3_to_bf16(x.z, x.w), Q[2 * step + 1], S[b], 0, 0, 0);
                } else {
                    S[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(x), Q[step], S[b], 0, 0, 0);
                }
                if (i + kAhead < kReads) w[i % kAhead] = read_k(i + kAhead);
                keep_order();
            }
        }
        if (gone || key0 + kBlockKeys - 1 > p_first ||
            (in.window > 0 && key0 <= p_last - in.window)) {
            if (gone && lane == 0 && gone_seen(gone, key0, p_first, p_last, in.window))
                atomicOr(in.err_word, kErrKvPage);
            const int32_t from = in.window > 0 ? pos - in.window : -1;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int k = 32 * b + 8 * (i / 4) + 4 * half + i % 4;
                    const bool see = key0 + k <= pos && key0 + k > from && !((gone >> (k / kGroupKeys)) & 1u);
                    if (!see) S[b][i] = -INFINITY;
                }
        }
        float top = S[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) top = fmaxf(top, S[i / 16][i % 16]);
        top = half_max(top) * c2;
        const bool raise = top > m + kRaise;
        if (__any(raise)) {
            const float m2 = raise ? top : m;
            const float fade = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - m2);
            m = m2;
            l *= fade;
#pragma unroll
            for (int h = 0; h < kCols; ++h)
#pragma unroll
                for (int i = 0; i < 16; ++i) O[h][i] *= fade;
        }
        const float off = m == -INFINITY ? 0.0f : m;
        // V^T operand j: column block j % kCols, 16 keys at j / kCols
        const int vo = fresh(v_off);
        auto read_v = [&](int j) {
            const int t = j / kCols, h = j % kCols;
            uint4 w = make_uint4(0u, 0u, 0u, 0u);
            if constexpr (E4M3) {
                const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                    (lds_i32x2)at_bytes(vt, (vo ^ (32 * h)) + 16 * t * RB)));
                w.x = x.x;
                w.y = x.y;
            } else {
                const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_s16x4)at_bytes(vt, (vo ^ (64 * h)) + 16 * t * RB)));
                const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_s16x4)at_bytes(vt, (vo ^ (64 * h)) + (16 * t + 8) * RB)));
                w = make_uint4(x.x, x.y, y.x, y.y);
            }
            return w;
        };
        uint4 vw[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) vw[j] = read_v(j);
        keep_order();
        uint32_t P[2][8];
        float sum = 0.0f;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(S[b][i], c2, -off));
                const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(S[b][i + 1], c2, -off));
                sum += x;
                sum += y;
                P[b][i / 2] = weights2(x, y);
            }
        l += sum;
#pragma unroll
        for (int j = 0; j < 4 * kCols; ++j) {
            const int t = j / kCols, h = j % kCols, b = t / 2, i0 = 4 * (t % 2);
            const bf16x8_t p = as_bf16x8(make_uint4(P[b][i0], P[b][i0 + 1], P[b][i0 + 2], P[b][i0 + 3]));
            bf16x8_t v;
            if constexpr (E4M3) v = e4m3_to_bf16(vw[j % kAhead].x, vw[j % kAhead].y);
            else v = as_bf16x8(vw[j % kAhead]);
            O[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p, O[h], 0, 0, 0);
            if (j + kAhead < 4 * kCols) vw[j % kAhead] = read_v(j + kAhead);
            keep_order();
        }
    };
    for (;;) {
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int h = 0; h < kCols; ++h) O[h] = f32x16_t{};
        const int32_t b0 = bl.first + st.block;
        if (careful) {
            notes.clear(tid);
            __syncthreads();
        }
        load_ids(b0);
        gone = stage(b0, kA, vA);
        for (int32_t i = 0; i < count; i += 2) {
            uint32_t after = 0;
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
            if (i + 1 < count) after = stage(b0 + i + 1, kB, vB);
            block_step(b0 + i, kA, vA);
            gone = after;
            if (i + 1 >= count) break;
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
            if (i + 2 < count) after = stage(b0 + i + 2, kA, vA);
            block_step(b0 + i + 1, kB, vB);
            gone = after;
        }
        // any value of O that is not finite makes this NaN
        float odd = 0.0f;
#pragma unroll
        for (int h = 0; h < kCols; ++h)
#pragma unroll
            for (int i = 0; i < 16; ++i) odd = __builtin_fmaf(O[h][i], 0.0f, odd);
        if (__any(odd != odd) && lane == 0) *lds.odd_unit = unit;
        l = half_sum(l);
        if (careful) {
            __syncthreads();
#pragma unroll
            for (int h = 0; h < kCols; ++h)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    O[h][i] = notes.apply(O[h][i], wave * 32 + n32, 32 * h + 8 * (i / 4) + 4 * half + i % 4);
        }
        if (count == bl.count) {
            if (row_ok) {
                const float inv = l == 0.0f ? 0.0f : v_scale / l;
                uint16_t* out = out_row(in, u, wave * 32 + n32, HD);
#pragma unroll
                for (int h = 0; h < kCols; ++h)
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        *reinterpret_cast<uint2*>(out + 32 * h + 2 * i + 4 * half) =
                            make_uint2(weights2(O[h][i] * inv, O[h][i + 1] * inv),
                                       weights2(O[h][i + 2] * inv, O[h][i + 3] * inv));
                if (half == 0) store_lse(in, u, wave * 32 + n32, m, l);
            }
        } else {
            const Part<kTileRows, HD, kTileRows> part(ws, st.nth, st.block == 0);
            const int r = wave * 32 + n32;
            if (half == 0) {
                part.put(r, m);
                part.put(kTileRows + r, l);
            }
#pragma unroll
            for (int h = 0; h < kCols; ++h)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    part.put4(2 * kTileRows + r * HD + 32 * h + 2 * i + 4 * half,
                              f32x4_t{O[h][i], O[h][i + 1], O[h][i + 2], O[h][i + 3]});
            __builtin_amdgcn_s_waitcnt(0);
        }
        __syncthreads();  // the buffers are free, a part has reached memory, odd_unit is known
        if (careful || scalar(*lds.odd_unit) != unit) break;
        careful = true;
    }
    if (count != bl.count) {
        join_parts<kTileRows, HD, kTileRows>(in, ws, u, static_cast<int32_t>(quotient(begin, st.share)),
                                  static_cast<int32_t>(quotient(last, st.share)), v_scale, lds.flag);
    }
}

// ------------------------------------------------------------------- row units

// Pieces of V that a wave copies for a step of row units, and the step's keys.
template <int HD, bool E4M3>
struct RowStep {
    static constexpr int kKeys = !E4M3 && HD >= 128 ? 32 : 64;
    static constexpr int kTile = kKeys * HD * (E4M3 ? 1 : 2) / 16;
};

// The same of a unit of 16 NB rows; SLOT: rows that a part has room for.  Each wave
// takes every fourth step of 32 or 64 keys by itself: K from memory into the registers
// that the product takes it from, V through LDS of the wave's own, both a step ahead.
//
// Memory bounds it: 256 requests of up to 8192 keys, heads of 128, read 4.1 GB (what
// they hold, by the counters too) in 643 us, 6.4 TB/s of the 7.0 that a plain read
// reaches; in e4m3 2.0 GB take 320 us, 6.3 TB/s; at head_dim 256 4.1 GB take 630 us, and
// 2.0 GB of e4m3 366; at 64 2.0 GB take 335 and 1.0 GB of e4m3 182.  With 32 rows a unit
// (five tokens a request, a window of 4096) 0.84 GB take 174 to 180 us, where a unit's
// start, its parts and their join are 16 to 20 of about 130.
template <int HD, bool E4M3, int NB, int SLOT>
__device__ __forceinline__ void row_unit(const AttendIn& in, const KvCacheIn& cache, const AttendWs& ws,
                                         const WorkRange& st, const Span& s, const Blocks& bl,
                                         int64_t begin, int64_t last, int32_t count, int unit, const UnitLds& lds) {
    constexpr int RB = HD * (E4M3 ? 1 : 2);
    constexpr int KS = RowStep<HD, E4M3>::kKeys;
    constexpr int kGroups = KS / kGroupKeys;
    constexpr int kLoads = RB / 64;               // 16-byte loads of a lane per 16 keys
    constexpr int kCopies = kGroupKeys * RB / 1024;
    constexpr int kSteps = HD / 32, kCols = HD / 16, M = 16 * NB;
    constexpr int kTile = KS * RB / 16;           // pieces of a step's V
    static_assert(kAttendWaves * kTile >= kAttendWaves * 16 * HD / 4, "room to join the waves");
    uint4 *const vA = lds.a, *const vB = lds.b;
    auto* const wm = reinterpret_cast<float (*)[M]>(lds.wm);
    auto* const wl = reinterpret_cast<float (*)[M]>(lds.wl);
    auto* const odd_keys = reinterpret_cast<OddKeys (*)[HD]>(lds.odd_keys);
    auto& notes = *reinterpret_cast<OddNotes<M, HD>*>(lds.notes);
    const int tid = threadIdx.x, lane = tid & 63, g4 = lane >> 4, n16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const HeadGroup group = in.group;

    // This lane's K, its part of V's copies and its reads of V.  A copy of 1 KB takes
    // 1024 / RB rows, so the permutation, by the row's low bits, changes from copy
    // to copy; where the kinds repeat, the offsets are the same but for a constant.
    const int k_src = n16 * RB + g4 * 16;
    constexpr int kRows = 1024 / RB, kKinds = KS * RB / 1024;
    int32_t src_v[kKinds];
#pragma unroll
    for (int i = 0; i < kKinds; ++i) {
        const int row = i * kRows + lane / (RB / 16), slot = lane % (RB / 16);
        src_v[i] = (lane / (RB / 16)) * RB + ((slot ^ swz_v_row<RB, E4M3>(row)) * 16);
    }
    const int v_row = E4M3 ? 16 * (n16 >> 3) + 4 * g4 + ((n16 >> 1) & 3) : 4 * g4 + (n16 >> 2);
    const int v_piece = E4M3 ? 0 : (n16 & 3) >> 1;
    const int v_off = wave * kTile * 16 + v_row * RB + ((v_piece ^ swz_v_row<RB, E4M3>(v_row)) * 16) +
                      8 * (n16 & 1);
    const RowsOut u{s.lo, s.n * group.n, 0, st.head, group};
    const float c2 = score_scale(in.scale, E4M3 ? scalar_load(cache.k_scale + st.head) : 1.0f);
    const int32_t base = s.len - s.n;
    const int32_t p_first = base, p_last = s.len - 1;
    int32_t pos[NB];
    bf16x8_t Q[NB][kSteps];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int32_t row = 16 * b + n16, held = min(row, u.n_rows - 1), tok = group.div(held);
        pos[b] = base + tok;  // (rows past the last repeat it and are not stored)
        const uint16_t* qr = in.q + (u.lo + tok) * in.q_stride +
                             static_cast<int64_t>(u.head * group.n + held - tok * group.n) * HD;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int c = E4M3 ? 8 * (i >> 1) + 2 * g4 + (i & 1) : 4 * i + g4;
            Q[b][i] = as_bf16x8(reinterpret_cast<const uint4*>(qr)[c]);
        }
    }
    // this wave's steps: of the segment's, every fourth
    const int32_t key_from = (bl.first + st.block) * kBlockKeys;
    const int32_t steps = count * (kBlockKeys / KS);

    uint4 KA[kGroups][kLoads], KB[kGroups][kLoads];
    uint32_t goneA, goneB;
    // Every step of the pipeline issues its loads, past the last one of nothing
    // (resources without rows): with a branch around them the wait for one step's
    // K would be for everything outstanding.
    int32_t ids;  // page ids of the step whose loads come next
    auto load_ids = [&](int32_t step) __attribute__((always_inline)) {
        ids = page_ids(cache, st.req, static_cast<uint32_t>(key_from) + static_cast<uint32_t>(step) * KS, s.len,
                       kGroups);
    };
    auto stage = [&](int32_t step, uint4 (&K)[kGroups][kLoads], uint4* vd, uint32_t& gone)
        __attribute__((always_inline)) {
        const bool on = step < steps;
        const int32_t key0 = on ? key_from + step * KS : 0, len = on ? s.len : 0;
        __amdgpu_buffer_rsrc_t vr[kGroups];
        int32_t page[kGroups];
        gone = groups_gone(cache, ids, kGroups);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) page[g] = __builtin_amdgcn_readlane(ids, g);
        load_ids(step + kAttendWaves);
        const int ko = fresh(k_src);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int32_t key = key0 + g * kGroupKeys;
            const __amdgpu_buffer_rsrc_t kr = group_rows<RB>(cache.k, cache, page[g], st.head, key, len);
            vr[g] = group_rows<RB>(cache.v, cache, page[g], st.head, key, len);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const u32x4_t w = __builtin_bit_cast(
                    u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(kr, ko + 64 * i, 0, kOnce));
                K[g][i] = make_uint4(w.x, w.y, w.z, w.w);
            }
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int i = 0; i < kCopies; ++i)
                copy16<kOnce>(vr[g], vd + wave * kTile + g * (kGroupKeys * RB / 16) + i * 64,
                              src_v[g * kCopies + i] + 1024 * i);
    };

    float m[NB], l[NB];
    f32x4_t O[NB][kCols];
    bool careful = false;
    auto key_step = [&](int32_t step, const uint4 (&K)[kGroups][kLoads], uint4* vt, uint32_t gone)
        __attribute__((always_inline)) {
        const int32_t key0 = key_from + step * KS;
        if (careful) {  // the tile and the masks are this wave's own
            for (int c = lane; c < HD; c += kWave) odd_keys[wave][c] = OddKeys{0, 0};
            __builtin_amdgcn_s_waitcnt(0);
            for (int e = lane; e < kTile; e += kWave) {
                const int kr = e / (RB / 16), slot = (e % (RB / 16)) ^ swz_v_row<RB, E4M3>(kr);
                take_odd<E4M3>(vt + wave * kTile + e, odd_keys[wave] + slot * (E4M3 ? 16 : 8), kr);
            }
            __builtin_amdgcn_s_waitcnt(0);
            if (lane < 2 * M)
                notes.note(lane / M, lane % M,
                           seen_keys(key0, base + group.div(min(lane % M, u.n_rows - 1)), in.window, gone),
                           odd_keys[wave]);
        }
        f32x4_t S[NB][kGroups];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
#pragma unroll
            for (int b = 0; b < NB; ++b) S[b][g] = f32x4_t{};
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                bf16x8_t k;
                if constexpr (E4M3) {
                    const uint4 w = K[g][i >> 1];
                    k = i & 1 ? e4m3_to_bf16(w.z, w.w) : e4m3_to_bf16(w.x, w.y);
                } else {
                    k = as_bf16x8(K[g][i]);
                }
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    S[b][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, Q[b][i], S[b][g], 0, 0, 0);
            }
        }
        if (gone || key0 + KS - 1 > p_first || (in.window > 0 && key0 <= p_last - in.window)) {
            if (gone && lane == 0 && gone_seen(gone, key0, p_first, p_last, in.window))
                atomicOr(in.err_word, kErrKvPage);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int32_t from = in.window > 0 ? pos[b] - in.window : -1;
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int32_t k = key0 + 16 * g + 4 * g4 + i;
                        if (!(k <= pos[b] && k > from && !((gone >> g) & 1u))) S[b][g][i] = -INFINITY;
                    }
            }
        }
        float top[NB];
        bool raise = false;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            top[b] = S[b][0][0];
#pragma unroll
            for (int i = 1; i < 4 * kGroups; ++i) top[b] = fmaxf(top[b], S[b][i / 4][i % 4]);
            top[b] = quarter_max(top[b]) * c2;
            raise |= top[b] > m[b] + kRaise;
        }
        if (__any(raise)) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const float m2 = top[b] > m[b] + kRaise ? top[b] : m[b];
                const float fade = m[b] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[b] - m2);
                m[b] = m2;
                l[b] *= fade;
#pragma unroll
                for (int h = 0; h < kCols; ++h) O[b][h] *= fade;
            }
        }
        // V^T operand j: column block j % kCols, 32 keys at j / kCols
        constexpr int kReads = kCols * kGroups / 2;
        wait_all_but<1 + kGroups * (kLoads + kCopies)>();  // the next step's loads: V is there
        const int vo = fresh(v_off);
        auto read_v = [&](int j) {
            const int t = j / kCols, h = j % kCols;
            uint4 w = make_uint4(0u, 0u, 0u, 0u);
            if constexpr (E4M3) {
                const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                    (lds_i32x2)at_bytes(vt, (vo ^ (16 * h)) + 32 * t * RB)));
                w.x = x.x;
                w.y = x.y;
            } else {
                const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_s16x4)at_bytes(vt, (vo ^ (32 * h)) + 32 * t * RB)));
                const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_s16x4)at_bytes(vt, (vo ^ (32 * h)) + (32 * t + 16) * RB)));
                w = make_uint4(x.x, x.y, y.x, y.y);
            }
            return w;
        };
        uint4 vw[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) vw[j] = read_v(j);
        keep_order();
        uint32_t P[NB][kGroups][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const float off = m[b] == -INFINITY ? 0.0f : m[b];
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(S[b][g][2 * i], c2, -off));
                    const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(S[b][g][2 * i + 1], c2, -off));
                    l[b] += x + y;
                    P[b][g][i] = weights2(x, y);
                }
        }
#pragma unroll
        for (int j = 0; j < kReads; ++j) {
            const int t = j / kCols, h = j % kCols;
            bf16x8_t v;
            if constexpr (E4M3) v = e4m3_to_bf16(vw[j % kAhead].x, vw[j % kAhead].y);
            else v = as_bf16x8(vw[j % kAhead]);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const bf16x8_t p = as_bf16x8(make_uint4(P[b][2 * t][0], P[b][2 * t][1], P[b][2 * t + 1][0],
                                                        P[b][2 * t + 1][1]));
                O[b][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p, O[b][h], 0, 0, 0);
            }
            if (j + kAhead < kReads) vw[j % kAhead] = read_v(j + kAhead);
            keep_order();
        }
    };
    for (;;) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            m[b] = -INFINITY;
            l[b] = 0.0f;
#pragma unroll
            for (int h = 0; h < kCols; ++h) O[b][h] = f32x4_t{};
        }
        if (careful) {
            notes.clear(tid);
            __syncthreads();
        }
        load_ids(wave);
        stage(wave, KA, vA, goneA);
        for (int32_t i = wave; i < steps; i += 2 * kAttendWaves) {
            stage(i + kAttendWaves, KB, vB, goneB);
            key_step(i, KA, vA, goneA);
            stage(i + 2 * kAttendWaves, KA, vA, goneA);
            if (i + kAttendWaves < steps) key_step(i + kAttendWaves, KB, vB, goneB);
        }
        float odd = 0.0f;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int h = 0; h < kCols; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) odd = __builtin_fmaf(O[b][h][i], 0.0f, odd);
        if (__any(odd != odd) && lane == 0) *lds.odd_unit = unit;
        __builtin_amdgcn_s_waitcnt(0);  // also the copies of steps past the last
        __syncthreads();
        if (careful || scalar(*lds.odd_unit) != unit) break;
        careful = true;
    }

    // the waves' rows joined in LDS (where V was), 16 at a time
    const bool whole = count == bl.count;
    const float v_scale = E4M3 ? scalar_load(cache.v_scale + st.head) : 1.0f;
    const Part<M, HD, SLOT> part(ws, st.nth, st.block == 0);
    f32x4_t* const pool = reinterpret_cast<f32x4_t*>(vA);
    constexpr int kVec = HD / 4;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const float lsum = quarter_sum(l[b]);
        if (g4 == 0) {
            wm[wave][16 * b + n16] = m[b];
            wl[wave][16 * b + n16] = lsum;
        }
        __syncthreads();  // V (or the rows before) is no longer read
#pragma unroll
        for (int h = 0; h < kCols; ++h)
            pool[(wave * 16 + n16) * kVec + ((4 * h + g4) ^ n16)] = O[b][h];
        __syncthreads();
        for (int e = tid; e < 16 * kVec; e += kAttendThreads) {
            const int r = e / kVec, c = e % kVec, row = 16 * b + r;
            float top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) top = fmaxf(top, wm[w][row]);
            f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) {
                const float f = weight_of(wm[w][row], top);
                sum += wl[w][row] * f;
                o += pool[(w * 16 + r) * kVec + (c ^ r)] * f;
            }
            if (careful)
                for (int i = 0; i < 4; ++i) o[i] = notes.apply(o[i], row, 4 * c + i);
            if (!whole) {
                if (c == 0) {
                    part.put(row, top);
                    part.put(M + row, sum);
                }
                part.put4(2 * M + row * HD + 4 * c, o);
            } else if (row < u.n_rows) {
                const float inv = sum == 0.0f ? 0.0f : v_scale / sum;
                *reinterpret_cast<uint2*>(out_row(in, u, row, HD) + 4 * c) =
                    make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
                if (c == 0) store_lse(in, u, row, top, sum);
            }
        }
    }
    if (!whole) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        join_parts<M, HD, SLOT>(in, ws, u, static_cast<int32_t>(quotient(begin, st.share)),
                          static_cast<int32_t>(quotient(last, st.share)), v_scale, lds.flag);
    }
    __syncthreads();  // before V is copied in again
}

// ----------------------------------------------------------------- the kernel

// NB 0: units of 128 rows, and those of a request with few rows as row units of 16;
// otherwise row units of 16 NB rows.
template <int HD, bool E4M3, int NB>
__global__ void __launch_bounds__(kAttendThreads, HD > 128 ? 1 : 2)
attend_kernel(AttendIn in, KvCacheIn cache, AttendWs ws) {
    constexpr int RB = HD * (E4M3 ? 1 : 2);
    constexpr int kRows = NB ? 16 * NB : kTileRows;
    constexpr Deal kDeal = deal_of(kRows);
    constexpr int kRowBuf = kAttendWaves * RowStep<HD, E4M3>::kTile, kTileBuf = 2 * kBlockKeys * RB / 16;
    constexpr int kBuf = NB || kRowBuf > kTileBuf ? kRowBuf : kTileBuf;
    __shared__ uint4 a[kBuf], b[kBuf];
    __shared__ OddKeys odd_keys[kAttendWaves * HD];
    __shared__ uint32_t notes[2 * kRows * HD / 32];
    __shared__ float wm[kAttendWaves * (NB ? kRows : kFewRows)], wl[kAttendWaves * (NB ? kRows : kFewRows)];
    __shared__ int flag, odd_unit, taken;
    const UnitLds lds{a, b, odd_keys, notes, wm, wl, &flag, &odd_unit};
    WorkRange st = range_of(ws);
    if (st.at >= st.end && !(NB == 0 && st.queued)) return;
    if (threadIdx.x == 0) odd_unit = -1;
    __syncthreads();
    // The range first, then units of the queue: whole and short ones, which even out
    // when the workgroups end; who takes one makes no difference to its result.
    Span s{st.lo, st.n, st.len};
    for (int unit = 0;; ++unit) {
        const bool dealt = st.at < st.end;
        if (!dealt) {
            if constexpr (NB) break;
            if (!st.queued) break;
            if (threadIdx.x == 0)
                taken = __hip_atomic_fetch_add(ws.queue, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();  // (a unit has barriers, so the one before has been read)
            const int32_t nth = scalar(taken);
            if (nth >= st.queued) break;
            const int32_t* upto = ws.queue + kQueueHead;
            int32_t lo = 0, hi = cache.R_max - 1;  // the last request that starts at or before nth
            while (lo < hi) {
                const int32_t mid = (lo + hi + 1) >> 1;
                if (scalar_load(upto + mid) <= nth) lo = mid;
                else hi = mid - 1;
            }
            const int32_t rest = nth - scalar_load(upto + lo);
            const int32_t lead = scalar_load(upto + cache.R_max + 1 + lo);
            s = scalar_span(in, cache, lo);
            st.req = lo;
            st.head = scalar(static_cast<int32_t>(static_cast<uint32_t>(rest) / static_cast<uint32_t>(max(lead, 1))));
            st.tile = rest - st.head * lead;
            st.block = 0;
        }
        if (st.tile >= tiles_of(s.n, in.group, kRows)) break;  // (lengths changed under the call)
        const Blocks bl = blocks_of(s, st.tile, in.group, kRows, in.window);
        const int64_t begin = st.at + kDeal.extra;
        const int32_t step = few_rows(s.n, in.group) ? kDeal.few_step : kDeal.step, all = bl.count * step;
        const int32_t count =
            dealt ? static_cast<int32_t>(min(st.end - begin, static_cast<int64_t>(all))) / step - st.block : bl.count;
        if constexpr (NB) {
            row_unit<HD, E4M3, NB, kRows>(in, cache, ws, st, s, bl, begin, begin + all - step, count, unit, lds);
        } else {
            if (few_rows(s.n, in.group))
                row_unit<HD, E4M3, 1, kTileRows>(in, cache, ws, st, s, bl, begin, begin + all - step, count, unit, lds);
            else
                tile_unit<HD, E4M3>(in, cache, ws, st, s, bl, begin, begin + all - step, count, unit, lds);
        }
        if (!dealt) continue;
        if (st.block + count < bl.count) {
            st.at = st.end;
            continue;
        }
        st.at += kDeal.extra + all;
        st.block = 0;
        if (!NB && ++st.tile < tiles_of(s.n, in.group, kRows)) continue;
        st.tile = NB ? 0 : scalar_load(ws.queue + kQueueHead + cache.R_max + 1 + st.req);
        if (++st.head < cache.n_kv || st.at >= st.end) continue;
        st.head = 0;
        do {
            ++st.req;
            s = scalar_span(in, cache, st.req);
            if (!NB) st.tile = scalar_load(ws.queue + kQueueHead + cache.R_max + 1 + st.req);
        } while (st.req < cache.R_max - 1 && (s.n == 0 || (!NB && st.tile >= tiles_of(s.n, in.group, kRows))));
    }
}

// --------------------------------------------------------------------- launch

namespace {

// Rows of a unit: all rows that a request can have where those are few.  64 requests
// with 5 drafted tokens each, 4 heads to a key head: 102 us as units of 32 rows, 117
// as tiles at head_dim 64, 185 and 230 at 128; at 256 their registers spill, and tiles
// take as long in bf16 (396 us) and less in e4m3 (279 us for 325).
int32_t unit_rows(int32_t n_q, int32_t max_q, const KvCacheIn& c) {
    const int64_t rows = static_cast<int64_t>(max_q) * (n_q / c.n_kv);
    return rows <= 16 ? 16 : rows <= 32 && c.head_dim < 256 ? 32 : kTileRows;
}
// Workgroups of a launch: as many as the chip holds at a time, two on a CU where their
// registers and LDS allow it.  At head_dim 256 they do not, and twice as many, one round
// behind the other, take 650 us for 628 (256 single tokens), 124 for 109 (prompts), 318
// for 246 (single tokens and a chunk).
int32_t workgroups(int32_t rows, const KvCacheIn& c) {
    return c.head_dim > 128 ? 256 : 512;
}

struct WsLayout {
    size_t done, queue, parts, bytes;
};
WsLayout ws_layout(int32_t rows, const KvCacheIn& c) {
    const size_t n = static_cast<size_t>(workgroups(rows, c));
    WsLayout w;
    w.done = n * sizeof(WorkRange);
    w.queue = w.done + n * sizeof(int32_t);
    w.parts = w.queue;
    if (rows == kTileRows) w.parts += (kQueueHead + 2 * static_cast<size_t>(c.R_max) + 1 + 3) / 4 * 16;
    w.bytes = w.parts + 2 * n * rows * static_cast<size_t>(c.head_dim + 2) * sizeof(float);
    return w;
}

using AttendKernel = void (*)(AttendIn, KvCacheIn, AttendWs);
// Indexed by head_dim (64, 128, 256), type and rows of a unit (16, 32, 128).
constexpr AttendKernel kKernels[3][2][3] = {
    {{attend_kernel<64, false, 1>, attend_kernel<64, false, 2>, attend_kernel<64, false, 0>},
     {attend_kernel<64, true, 1>, attend_kernel<64, true, 2>, attend_kernel<64, true, 0>}},
    {{attend_kernel<128, false, 1>, attend_kernel<128, false, 2>, attend_kernel<128, false, 0>},
     {attend_kernel<128, true, 1>, attend_kernel<128, true, 2>, attend_kernel<128, true, 0>}},
    {{attend_kernel<256, false, 1>, nullptr, attend_kernel<256, false, 0>},
     {attend_kernel<256, true, 1>, nullptr, attend_kernel<256, true, 0>}}};
AttendKernel kernel_for(int32_t hd, bool e4m3, int32_t rows) {
    return kKernels[hd == 64 ? 0 : hd == 128 ? 1 : 2][e4m3][rows == 16 ? 0 : rows == 32 ? 1 : 2];
}

}  // namespace

size_t attend_workspace(int32_t n_q, int32_t max_q, const KvCacheIn& cache) {
    return ws_layout(unit_rows(n_q, max_q, cache), cache).bytes;
}

hipError_t launch_attend(const AttendIn& in, const KvCacheIn& cache, bool e4m3, void* ws,
                         hipStream_t stream) {
    const int32_t rows = unit_rows(in.n_q, in.max_q, cache), n_wg = workgroups(rows, cache);
    const WsLayout w = ws_layout(rows, cache);
    char* p = static_cast<char*>(ws);
    const AttendWs aw{reinterpret_cast<WorkRange*>(p), reinterpret_cast<int32_t*>(p + w.done),
                      reinterpret_cast<int32_t*>(p + w.queue), reinterpret_cast<float*>(p + w.parts)};
    const int64_t most = (static_cast<int64_t>(in.max_q) * (in.n_q / cache.n_kv) + rows - 1) / rows;
    const auto plan = rows != kTileRows     ? attend_plan_kernel<false, false>
                      : most <= kTilesEach ? attend_plan_kernel<false, true>
                                           : attend_plan_kernel<true, true>;
    hipLaunchKernelGGL(plan, dim3(most <= kTilesEach ? 1 : n_wg / kPlanRanges), dim3(kPlanThreads), 0, stream, in,
                       cache, aw, deal_of(rows), n_wg);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel_for(cache.head_dim, e4m3, rows), dim3(n_wg), dim3(kAttendThreads), 0, stream,
                       in, cache, aw);
    return hipGetLastError();
}

void add_attend_kernels(std::vector<KernelInfo>& t) {
    t.push_back(kernel_info(attend_plan_kernel<false, false>));
    t.push_back(kernel_info(attend_plan_kernel<false, true>));
    t.push_back(kernel_info(attend_plan_kernel<true, true>));
    for (const auto& width : kKernels)
        for (const auto& type : width)
            for (const AttendKernel k : type)
                if (k) t.push_back(kernel_info(k));
}

}  // namespace xmix
