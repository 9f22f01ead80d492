// Per-head passes of an attention layer's rows: norm and position rotation of
// queries and keys, and the append of keys and values to the paged cache.
//
// Both read every value once and write it once, so memory bounds them (and at
// decode sizes the latency of one chain: position, rows, result).
#include "common.hpp"
#include "kernels.hpp"
#include "launch.hpp"
#include "paged.hpp"
#include "rope.hpp"

namespace xmix {

template <>
struct ArgPointers<RopeIn> {
    static std::vector<uint16_t> offsets() { return {offsetof(RopeIn, inv_freq)}; }
};
template <>
struct ArgPointers<HeadRows> {
    static std::vector<uint16_t> offsets() {
        return {offsetof(HeadRows, x), offsetof(HeadRows, weight), offsetof(HeadRows, out)};
    }
};
constexpr int kHeadThreadsLog2 = 8, kHeadThreads = 1 << kHeadThreadsLog2;

// The workgroup's place, in rows of the grid: the threads of one dimension of a grid
// number less than 2^32.
constexpr int32_t kGridRow = 1 << 20;
__device__ __forceinline__ int32_t grid_place() {
    return static_cast<int32_t>(blockIdx.y * kGridRow + blockIdx.x);
}
// A token has the threads that its heads need, a power of two and a workgroup's at most:
// 9982 tokens of one key and one value head took 10.5 us with a workgroup each, 4.4 so.
struct TokenThreads {
    int32_t lanes_log2, threads_log2;  // of a head, of a token
    dim3 grid;
};
inline TokenThreads token_threads(int32_t head_dim, int32_t heads, int32_t T_max) {
    TokenThreads n{0, 0, dim3()};
    while ((1 << n.lanes_log2) < head_lanes(head_dim)) ++n.lanes_log2;
    n.threads_log2 = n.lanes_log2;
    while (n.threads_log2 < kHeadThreadsLog2 && (1 << (n.threads_log2 - n.lanes_log2)) < heads) ++n.threads_log2;
    const int32_t groups = ((T_max - 1) >> (kHeadThreadsLog2 - n.threads_log2)) + 1;
    n.grid = groups <= kGridRow ? dim3(groups) : dim3(kGridRow, (groups - 1) / kGridRow + 1);
    return n;
}

// Sum over the n lanes (a power of two up to 16) that share a head.
__device__ __forceinline__ float head_sum(float v, int n) {
    if (n > 1) v += dpp_f<kDppXor1>(v);
    if (n > 2) v += dpp_f<kDppXor2>(v);
    if (n > 4) v += dpp_f<kDppHalfMirror>(v);
    if (n > 8) v += dpp_f<kDppMirror>(v);
    return v;
}

// The token's lanes form groups of one head each, which take its query heads and then
// its key heads in turn, the next head's rows on their way while one is worked on; a
// lane's angles are computed once for all of them.
//   y = x (mean(x^2) + eps)^(-1/2) w,   out = round(rotate(y))
// 8192 tokens of 64 + 8 heads of 128: 58 us for 302 MB, 5.2 TB/s, past a large copy's
// 4.7, and 49.8 us where rows are still in the last cache (61.6 with a head loaded after
// the one before it was stored); 256 tokens of 32 + 8: 4.7 us, launch and one round trip.
template <bool BF16>
__global__ void __launch_bounds__(kHeadThreads)
norm_rope_kernel(HeadRows q, HeadRows k, int32_t head_dim, int32_t lanes_log2, int32_t threads_log2,
                 int32_t T_max, const int32_t* __restrict__ pos_of_token,
                 const int32_t* __restrict__ T_valid, float eps, RopeIn rope) {
    const int tid = threadIdx.x & ((1 << threads_log2) - 1);  // of the token's
    const int64_t at = (static_cast<int64_t>(grid_place()) * kHeadThreads + threadIdx.x) >> threads_log2;
    if (at >= T_max) return;
    const int32_t t = static_cast<int32_t>(at);
    const int lanes = 1 << lanes_log2, u = tid & (lanes - 1), heads = (1 << threads_log2) >> lanes_log2;
    const bool mine = 2 * kChunk * u < head_dim;
    const HeadPart part = head_part(u, rope);
    constexpr int kBytes = BF16 ? 2 : 4;
    auto load = [&](int h, Raw<BF16>* a, Raw<BF16>* b) {
        const HeadRows& r = h < q.n ? q : k;
        const char* x = static_cast<const char*>(r.x) +
                        (t * r.stride + (h < q.n ? h : h - q.n) * static_cast<int64_t>(head_dim)) * kBytes;
        *a = load_chunk<BF16>(x, part.a);
        *b = load_chunk<BF16>(x, part.b);
    };
    int h = tid >> lanes_log2;
    Raw<BF16> ra = {}, rb = {};
    if (mine && h < q.n + k.n) load(h, &ra, &rb);  // on their way while the position is looked up
    const int32_t pos = pos_of_token[t];
    if (pos < 0 || (T_valid && t >= *T_valid)) return;
    Angles g;
    if (part.turned) angles(g, rope, u, pos);
    while (h < q.n + k.n) {
        const HeadRows& r = h < q.n ? q : k;
        const int64_t row = (h < q.n ? h : h - q.n) * static_cast<int64_t>(head_dim);
        float a[kChunk], b[kChunk];
        widen<BF16>(ra, a);
        widen<BF16>(rb, b);
        h += heads;
        if (mine && h < q.n + k.n) load(h, &ra, &rb);
        if (r.weight) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < kChunk; ++i) sum += a[i] * a[i] + b[i] * b[i];
            sum = head_sum(sum, lanes);
            const float inv = 1.0f / sqrtf(sum / static_cast<float>(head_dim) + eps);
            if (mine) {
                float wa[kChunk], wb[kChunk];
                widen<BF16>(load_chunk<BF16>(r.weight, part.a), wa);
                widen<BF16>(load_chunk<BF16>(r.weight, part.b), wb);
#pragma unroll
                for (int i = 0; i < kChunk; ++i) {
                    a[i] = a[i] * inv * wa[i];
                    b[i] = b[i] * inv * wb[i];
                }
            }
        }
        if (!mine) continue;
        if (part.turned) rotate(a, b, g, rope.pairs != 0);
        char* out = static_cast<char*>(r.out) + (t * r.out_stride + row) * kBytes;
        store_chunk<BF16>(out, part.a, a);
        store_chunk<BF16>(out, part.b, b);
    }
}

hipError_t launch_norm_rope(const HeadRows& q, const HeadRows& k, bool bf16, int32_t head_dim,
                            int32_t T_max, const int32_t* pos, const int32_t* T_valid, float eps,
                            const RopeIn& rope, hipStream_t stream) {
    const TokenThreads n = token_threads(head_dim, q.n + k.n, T_max);
    hipLaunchKernelGGL(bf16 ? norm_rope_kernel<true> : norm_rope_kernel<false>, n.grid, dim3(kHeadThreads), 0,
                       stream, q, k, head_dim, n.lanes_log2, n.threads_log2, T_max, pos, T_valid, eps, rope);
    return hipGetLastError();
}

// x / scale held to what the 8-bit type can represent (the conversion itself
// turns larger values into NaN); NaN stays NaN.
__device__ __forceinline__ float to_e4m3_range(float y) {
    const float held = __builtin_amdgcn_fmed3f(y, -448.0f, 448.0f);
    return y == y ? held : y;
}
// The rounded quotient x / s in four instructions: with the rounded reciprocal `inv`, a
// quotient that its remainder corrects once is the rounded one (Markstein's theorem),
// where neither leaves fp32's range: 2^-60 <= s <= 2^60, and what is far past +-448 or
// far below the type's least value ends there whatever its last bits are.
__device__ __forceinline__ float quotient(float x, float s, float inv) {
    const float q = x * inv;
    const float y = __builtin_copysignf(__builtin_fmaf(__builtin_fmaf(-q, s, x), inv, q), x);
    return fabsf(q) < 1024.0f ? y : q;
}
__device__ __forceinline__ void scale_down(float* a, float* b, float s) {
    if (__any(!(s >= 0x1p-60f && s <= 0x1p60f))) {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) {
            a[i] = to_e4m3_range(a[i] / s);
            b[i] = to_e4m3_range(b[i] / s);
        }
        return;
    }
    const float inv = 1.0f / s;
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
        a[i] = to_e4m3_range(quotient(a[i], s, inv));
        b[i] = to_e4m3_range(quotient(b[i], s, inv));
    }
}
__device__ __forceinline__ uint32_t pack4_e4m3(const float* x) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
}

// The threads that a token's heads need, a workgroup's at most: their lane groups take
// the token's key heads, rotated, and its value heads in turn, and store each into the token's slot.  Sixteen prompts'
// 9982 tokens of 8 heads of 128 into e4m3 pages: 14.6 us for 61 MB, 4.2 TB/s (in a trace
// 15.3; 15.9 when it was 17.0 with a full division a value, 19.3 with a workgroup for each
// token and half of its threads idle); 256 tokens into bf16 pages: 3.4 us, a chain of
// three round trips.
template <bool BF16, bool E4M3>
__global__ void __launch_bounds__(kHeadThreads)
kv_append_kernel(const void* __restrict__ k, int64_t k_stride, const void* __restrict__ v,
                 int64_t v_stride, int32_t lanes_log2, int32_t threads_log2, int32_t T_max,
                 const int32_t* __restrict__ req_of_token, const int32_t* __restrict__ pos_of_token,
                 const int32_t* __restrict__ T_valid, RopeIn rope, KvCacheIn cache,
                 uint32_t* __restrict__ err_word) {
    const int tid = threadIdx.x & ((1 << threads_log2) - 1);  // of the token's
    const int64_t at = (static_cast<int64_t>(grid_place()) * kHeadThreads + threadIdx.x) >> threads_log2;
    if (at >= T_max) return;
    const int32_t t = static_cast<int32_t>(at), hd = cache.head_dim;
    const int lanes = 1 << lanes_log2, u = tid & (lanes - 1), heads = (1 << threads_log2) >> lanes_log2;
    if (2 * kChunk * u >= hd) return;
    const HeadPart part = head_part(u, rope);
    auto load = [&](int h, Raw<BF16>* a, Raw<BF16>* b) {
        const bool is_k = h < cache.n_kv;
        const char* x = static_cast<const char*>(is_k ? k : v) +
                        (t * (is_k ? k_stride : v_stride) +
                         static_cast<int64_t>(is_k ? h : h - cache.n_kv) * hd) * (BF16 ? 2 : 4);
        *a = load_chunk<BF16>(x, part.a);
        *b = load_chunk<BF16>(x, part.b);
    };
    int h = tid >> lanes_log2;
    if (h >= 2 * cache.n_kv) return;
    Raw<BF16> ra, rb;
    load(h, &ra, &rb);  // on their way while the slot is looked up
    const int32_t req = req_of_token[t], pos = pos_of_token[t];
    if (req < 0 || pos < 0 || (T_valid && t >= *T_valid)) return;
    int32_t page = -1;
    const int32_t nth = pos >> cache.page_log2;
    if (req < cache.R_max && nth < cache.max_pages)
        page = page_at(cache, req, nth);
    if (!page_ok(cache, page)) {
        if (tid == 0) atomicOr(err_word, kErrKvSlot);
        return;
    }
    const int32_t slot = pos & ((1 << cache.page_log2) - 1);
    Angles g;
    if (part.turned) angles(g, rope, u, pos);
    for (;;) {
        const bool is_k = h < cache.n_kv;
        const int head = is_k ? h : h - cache.n_kv;
        float a[kChunk], b[kChunk];
        widen<BF16>(ra, a);
        widen<BF16>(rb, b);
        h += heads;
        if (h < 2 * cache.n_kv) load(h, &ra, &rb);
        if (is_k && part.turned) rotate(a, b, g, rope.pairs != 0);
        const int64_t row = page_row(cache, page, head, slot);
        char* out = static_cast<char*>(is_k ? cache.k : cache.v) + row * hd * (E4M3 ? 1 : 2);
        if constexpr (E4M3) {
            scale_down(a, b, (is_k ? cache.k_scale : cache.v_scale)[head]);
            *reinterpret_cast<uint2*>(out + part.a) = make_uint2(pack4_e4m3(a), pack4_e4m3(a + 4));
            *reinterpret_cast<uint2*>(out + part.b) = make_uint2(pack4_e4m3(b), pack4_e4m3(b + 4));
        } else {
            store_chunk<true>(out, part.a, a);
            store_chunk<true>(out, part.b, b);
        }
        if (h >= 2 * cache.n_kv) break;
    }
}

hipError_t launch_kv_append(const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                            bool bf16, int32_t T_max, const int32_t* req, const int32_t* pos,
                            const int32_t* T_valid, const RopeIn& rope, const KvCacheIn& cache,
                            bool e4m3, uint32_t* err_word, hipStream_t stream) {
    const TokenThreads n = token_threads(cache.head_dim, 2 * cache.n_kv, T_max);
    const auto kernel = bf16 ? (e4m3 ? kv_append_kernel<true, true> : kv_append_kernel<true, false>)
                             : (e4m3 ? kv_append_kernel<false, true> : kv_append_kernel<false, false>);
    hipLaunchKernelGGL(kernel, n.grid, dim3(kHeadThreads), 0, stream, k, k_stride, v, v_stride,
                       n.lanes_log2, n.threads_log2, T_max, req, pos, T_valid, rope, cache, err_word);
    return hipGetLastError();
}

void add_head_kernels(std::vector<KernelInfo>& t) {
    t.push_back(kernel_info(norm_rope_kernel<true>));
    t.push_back(kernel_info(norm_rope_kernel<false>));
    t.push_back(kernel_info(kv_append_kernel<true, true>));
    t.push_back(kernel_info(kv_append_kernel<true, false>));
    t.push_back(kernel_info(kv_append_kernel<false, true>));
    t.push_back(kernel_info(kv_append_kernel<false, false>));
}

}  // namespace xmix
