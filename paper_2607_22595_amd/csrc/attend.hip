// Attention of a step's tokens over the paged cache of their requests.
//
//   s_j = scale (q . k_j),  out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)
//
// over the keys j that the token sees, in one pass with the running maximum m and
// the running sum.  One wave per token and query head: a lane takes a key of each
// 64, then each lane its columns of the values.
#include "common.hpp"
#include "kernels.hpp"
#include "launch.hpp"
#include "paged.hpp"

namespace xmix {

template <>
struct ArgPointers<AttendIn> {
    static std::vector<uint16_t> offsets() {
        return {offsetof(AttendIn, q), offsetof(AttendIn, cu), offsetof(AttendIn, kv_len),
                offsetof(AttendIn, out), offsetof(AttendIn, lse), offsetof(AttendIn, err_word)};
    }
};

template <bool E4M3>
__device__ __forceinline__ float cached(const void* p, int64_t at) {
    if constexpr (E4M3)
        return __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(p)[at], 0);
    else
        return bf16_to_f32(static_cast<const uint16_t*>(p)[at]);
}

template <bool E4M3>
__global__ void __launch_bounds__(kWave)
attend_kernel(AttendIn in, KvCacheIn cache) {
    const int32_t r = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
    const int32_t lo = in.cu[r], hi = in.cu[r + 1], n = hi - lo, len = in.kv_len[r];
    if (n == 0 && lo >= 0 && lo <= in.T_max) return;
    if (lo < 0 || hi > in.T_max || n < 0 || n > in.max_q || len < 0 ||
        (len >> cache.page_log2) + ((len & ((1 << cache.page_log2) - 1)) != 0) > cache.max_pages) {
        if (lane == 0) atomicOr(in.err_word, kErrKvSpan);
        return;
    }
    const int32_t hd = cache.head_dim, head = h / (in.n_q / cache.n_kv);
    const float ks = E4M3 ? cache.k_scale[head] : 1.0f, vs = E4M3 ? cache.v_scale[head] : 1.0f;
    constexpr int kCols = 4;  // of 64 lanes: head_dim up to 256
    for (int32_t i = blockIdx.z; i < n; i += gridDim.z) {
        const int32_t p = len - n + i;
        const uint16_t* q = in.q + (lo + i) * in.q_stride + static_cast<int64_t>(h) * hd;
        float m = -INFINITY, l = 0.0f, acc[kCols] = {};
        const int32_t first = in.window > 0 && p >= in.window ? p - in.window + 1 : 0;
        for (int32_t j0 = first; j0 <= p; j0 += kWave) {
            const int32_t j = min(j0 + lane, p);
            const int32_t page = page_at(cache, r, j >> cache.page_log2);
            const bool ok = page_ok(cache, page);
            if (!ok) atomicOr(in.err_word, kErrKvPage);
            const int64_t row = page_row(cache, ok ? page : 0, head, j & ((1 << cache.page_log2) - 1)) * hd;
            float s = 0.0f;
            for (int c = 0; c < hd; ++c) s += bf16_to_f32(q[c]) * cached<E4M3>(cache.k, row + c);
            s *= in.scale * ks;
            if (j0 + lane > p || !ok) s = -INFINITY;
            float top = s;
            for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
            const float m2 = fmaxf(m, top), base = m2 == -INFINITY ? 0.0f : m2;
            const float e = expf(s - base), fade = expf(m - base);
            m = m2;
            l = l * fade + wave_sum(e);
            for (int c = 0; c < kCols; ++c) acc[c] *= fade;
            for (int k = 0; k < kWave; ++k) {
                const float w = __shfl(e, k);
                const int64_t at = __shfl(row, k);
                if (j0 + k > p || !__shfl(ok, k)) continue;
                for (int c = 0; c < kCols; ++c)
                    if (lane + c * kWave < hd) acc[c] += w * cached<E4M3>(cache.v, at + lane + c * kWave);
            }
        }
        uint16_t* out = in.out + (lo + i) * in.out_stride + static_cast<int64_t>(h) * hd;
        for (int c = 0; c < kCols; ++c)
            if (lane + c * kWave < hd)
                out[lane + c * kWave] = l == 0.0f ? 0 : f32_to_bf16_rne(acc[c] / l * vs);
        if (in.lse && lane == 0)
            in.lse[static_cast<int64_t>(h) * in.T_max + lo + i] = l == 0.0f ? -INFINITY : m + logf(l);
    }
}

size_t attend_workspace(int32_t, int32_t, const KvCacheIn&) { return 0; }

hipError_t launch_attend(const AttendIn& in, const KvCacheIn& cache, bool e4m3, void*,
                         hipStream_t stream) {
    const dim3 grid(cache.R_max, in.n_q, min(in.max_q, 256));
    if (e4m3)
        hipLaunchKernelGGL(attend_kernel<true>, grid, dim3(kWave), 0, stream, in, cache);
    else
        hipLaunchKernelGGL(attend_kernel<false>, grid, dim3(kWave), 0, stream, in, cache);
    return hipGetLastError();
}

void add_attend_kernels(std::vector<KernelInfo>& t) {
    t.push_back(kernel_info(attend_kernel<true>));
    t.push_back(kernel_info(attend_kernel<false>));
}

}  // namespace xmix
