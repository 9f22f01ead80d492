// Head rows in registers: loads and stores of a lane's part of a head, and the
// position rotation.
#pragma once

#include "common.hpp"
#include "launch.hpp"

namespace xmix {

constexpr int kChunk = 8;          // values of one 16-byte piece of bf16
constexpr int kMaxHeadDim = 256;

// How a head lies over lanes: a lane holds two chunks of eight values, chosen so
// that both values of every rotated pair are in one lane (no exchange between
// lanes, and the two loads of a lane group are contiguous).  Lane u of the head:
//   halves, 8 u < rot / 2: chunks u and u + rot / 16
//   otherwise:             two neighbouring chunks
// Either way the lane's angles are those of the frequencies 8 u .. 8 u + 7.
struct HeadPart {
    int32_t a, b;   // first value of each chunk
    bool turned;    // whether the rotation covers them
};
__device__ __forceinline__ HeadPart head_part(int u, const RopeIn& rope) {
    HeadPart p;
    const int half = rope.rot_dim >> 1;
    if (!rope.pairs && kChunk * u < half) {
        p.a = kChunk * u;
        p.b = p.a + half;
    } else {
        p.a = 2 * kChunk * u;
        p.b = p.a + kChunk;
    }
    p.turned = kChunk * u < half;
    return p;
}

// cos and sin of position * inv_freq.  The product is taken in fp64 and in
// revolutions, of which the fraction goes to the sine unit: its error there is
// at most 1.2e-7 over a whole revolution, where an fp32 product at position
// 100000 would be 0.006 radians off.
struct Angles {
    float c[kChunk], s[kChunk];
};
__device__ __forceinline__ void angles(Angles& g, const RopeIn& rope, int u, int32_t pos) {
    constexpr double kRevolutions = 0.15915494309189533577;  // 1 / (2 pi)
    const double turns = pos * kRevolutions;
    const double2* f = reinterpret_cast<const double2*>(rope.inv_freq + kChunk * u);
#pragma unroll
    for (int i = 0; i < kChunk / 2; ++i) {
        const double2 w = f[i];
        const float a = static_cast<float>(__builtin_amdgcn_fract(turns * w.x));
        const float b = static_cast<float>(__builtin_amdgcn_fract(turns * w.y));
        g.c[2 * i] = __builtin_amdgcn_cosf(a);
        g.s[2 * i] = __builtin_amdgcn_sinf(a);
        g.c[2 * i + 1] = __builtin_amdgcn_cosf(b);
        g.s[2 * i + 1] = __builtin_amdgcn_sinf(b);
    }
}

__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
    const float x = a * c - b * s;
    b = b * c + a * s;
    a = x;
}
__device__ __forceinline__ void rotate(float* a, float* b, const Angles& g, bool pairs) {
    if (pairs) {
#pragma unroll
        for (int i = 0; i < kChunk / 2; ++i) {
            turn(a[2 * i], a[2 * i + 1], g.c[i], g.s[i]);
            turn(b[2 * i], b[2 * i + 1], g.c[kChunk / 2 + i], g.s[kChunk / 2 + i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) turn(a[i], b[i], g.c[i], g.s[i]);
    }
}

// A chunk as it lies in memory, loaded whole and widened later.
template <bool BF16>
struct Raw {
    uint4 w[BF16 ? 1 : 2];
};
template <bool BF16>
__device__ __forceinline__ Raw<BF16> load_chunk(const void* row, int32_t at) {
    Raw<BF16> r;
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const char*>(row) +
                                                    static_cast<int64_t>(at) * (BF16 ? 2 : 4));
    r.w[0] = p[0];
    if constexpr (!BF16) r.w[1] = p[1];
    return r;
}
template <bool BF16>
__device__ __forceinline__ void widen(const Raw<BF16>& r, float* x) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(r.w);
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
        if constexpr (BF16) x[i] = i & 1 ? hi_bf16(w[i >> 1]) : lo_bf16(w[i >> 1]);
        else x[i] = __uint_as_float(w[i]);
    }
}
__device__ __forceinline__ uint4 pack8_bf16(const float* x) {
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]),
                      pack_bf16(x[6], x[7]));
}
template <bool BF16>
__device__ __forceinline__ void store_chunk(void* row, int32_t at, const float* x) {
    uint4* p = reinterpret_cast<uint4*>(static_cast<char*>(row) +
                                        static_cast<int64_t>(at) * (BF16 ? 2 : 4));
    if constexpr (BF16) {
        p[0] = pack8_bf16(x);
    } else {
        p[0] = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                          __float_as_uint(x[3]));
        p[1] = make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]),
                          __float_as_uint(x[7]));
    }
}

// Lanes that share a head: the power of two that holds head_dim / 16 parts.
inline int head_lanes(int32_t head_dim) {
    int n = 1;
    while (n * 2 * kChunk < head_dim) n *= 2;
    return n;
}

}  // namespace xmix
