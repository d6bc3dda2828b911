// Spans of consecutive elements as one access, and the 8-bit blocks of the activation checkpoints.
#pragma once

#include "moe_common.cuh"

namespace moe {

// ---------------------------------------------------------------- spans
// N consecutive elements of T as one access of sizeof(T) * N = 2, 4, 8 or 16 bytes.
template <typename T, int N> struct Span {
    static constexpr int BYTES = (int)sizeof(T) * N;
    static constexpr int WORDS = BYTES < 4 ? 1 : BYTES / 4;
    uint32_t w[WORDS];

    __device__ __forceinline__ void load(const T* p) {
        if constexpr (BYTES == 16) {
            const uint4 u = *reinterpret_cast<const uint4*>(p);
            w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
        } else if constexpr (BYTES == 8) {
            const uint2 u = *reinterpret_cast<const uint2*>(p);
            w[0] = u.x; w[1] = u.y;
        } else if constexpr (BYTES == 4) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else {
            w[0] = *reinterpret_cast<const uint16_t*>(p);
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void unpack(float (&f)[N]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = __uint_as_float(w[i]);
        } else if constexpr (N == 1) {
            f[0] = __uint_as_float(w[0] << 16);
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                f[2 * i] = __uint_as_float(w[i] << 16);
                f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
    // rounded to T, to nearest even
    __device__ __forceinline__ void pack(const float (&f)[N]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = __float_as_uint(f[i]);
        } else if constexpr (N == 1) {
            w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(f[0]));
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
    }
    // Largest magnitude of the elements as the bits of a float: unsigned order is that of the magnitudes, an
    // infinity above every number and a NaN above that.
    __device__ __forceinline__ uint32_t largest_bits() const {
        uint32_t m = 0;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) m = max(m, w[i] & 0x7fffffffu);
            return m;
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
            return max(m << 16, m & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void store(T* p) const {
        if constexpr (BYTES == 16) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (BYTES == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else if constexpr (BYTES == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
        else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    }
};

// ---------------------------------------------------------------- 8-bit blocks
// A checkpoint holds 128 columns of a row (fewer at its end) as int8 q with one fp32 scale:
//   a = max |x|, scale = a / 127, q = rint(x * (127 / a)), value = q * scale,
// so that a value is off by at most a / 254 and the arithmetic's own rounding. A block with
// a < 2^-100 (127 / a would overflow further down) holds zeros with scale 0; one with an infinity
// or a NaN gets scale NaN, so that all its values come back as NaN and none as a wrong number.
constexpr int CKPT_BLOCK = 128;

// The largest of LANES (a power of two) consecutive, aligned lanes
template <int LANES> __device__ __forceinline__ uint32_t lanes_max(uint32_t m) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}
__device__ __forceinline__ void block_scale(uint32_t bits, float& scale, float& inv) {
    const float a = __uint_as_float(bits);
    const bool zero = bits < 0x0d800000u /* 2^-100 */, bad = bits >= 0x7f800000u;
    scale = zero ? 0.f : bad ? __uint_as_float(0x7fffffffu) : __fdiv_rn(a, 127.f);
    inv = zero || bad ? 0.f : __fdiv_rn(127.f, a);
}
// Scales of U blocks of LANES lanes each: bits(u) is the lane's largest magnitude of block u. Lane u gets block u's
// scale, every lane all 127 / a: each lane does the divisions of one block (U of them in a lane cost more than the
// rest of its quantisation).
template <int LANES, int U, typename F> __device__ __forceinline__ void block_scales(F bits, float& scale, float (&inv)[U]) {
    static_assert(U <= LANES && LANES <= 32);
    const int lane = threadIdx.x % LANES;
    uint32_t mine = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t m = lanes_max<LANES>(bits(u));
        mine = lane % U == u ? m : mine;
    }
    float v;
    block_scale(mine, scale, v);
#pragma unroll
    for (int u = 0; u < U; ++u) inv[u] = __shfl_sync(0xffffffffu, v, (threadIdx.x & 31) - lane + u);
}
// Four values as int8 in a word. Adding 1.5 * 2^23 rounds the product to an integer (nearest, even)
// and leaves it in the low byte in two's complement; the product is rounded first, as x * inv is.
__device__ __forceinline__ uint32_t quant4(float a, float b, float c, float d, float inv) {
    constexpr float R = 12582912.f;
    const uint32_t ua = __float_as_uint(__fadd_rn(__fmul_rn(a, inv), R)), ub = __float_as_uint(__fadd_rn(__fmul_rn(b, inv), R));
    const uint32_t uc = __float_as_uint(__fadd_rn(__fmul_rn(c, inv), R)), ud = __float_as_uint(__fadd_rn(__fmul_rn(d, inv), R));
    return __byte_perm(__byte_perm(ua, ub, 0x0040), __byte_perm(uc, ud, 0x0040), 0x5410);
}
__device__ __forceinline__ int8_t quant1(float a, float inv) { return (int8_t)(quant4(a, 0.f, 0.f, 0.f, inv) & 0xffu); }

// int8 as floats: a byte plus 128 in the mantissa of 2^23, less 2^23 + 128 (exact)
__device__ __forceinline__ void unquant4(uint32_t q, float* f) {
    const uint32_t u = q ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7650u + (uint32_t)i)) - 8388736.f;
}
// N int8 (1, 2, 4 or 8) from p, aligned to N bytes
template <int N> __device__ __forceinline__ void load_q(const int8_t* p, uint32_t (&w)[(N + 3) / 4]) {
    if constexpr (N == 8) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        w[0] = u.x; w[1] = u.y;
    } else if constexpr (N == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
    else if constexpr (N == 2) w[0] = *reinterpret_cast<const uint16_t*>(p);
    else w[0] = (uint8_t)*p;
}
template <int N> __device__ __forceinline__ void unquant(const uint32_t (&w)[(N + 3) / 4], float scale, float (&f)[N]) {
    float t[4];
#pragma unroll
    for (int i = 0; i < (N + 3) / 4; ++i) {
        unquant4(w[i], t);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (4 * i + j < N) f[4 * i + j] = t[j] * scale;
    }
}

}  // namespace moe
