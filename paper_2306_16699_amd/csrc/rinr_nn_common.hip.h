// Operators for networks on decoded batches: types, loads and stores of any alignment, activations, 8-bit blocks.
#ifndef RINR_NN_COMMON_HIP_H
#define RINR_NN_COMMON_HIP_H

#include <hip/hip_runtime.h>
#include <cstdint>
#include "../../include/rinr_nn.h"

namespace rinr_nn {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
template <class E> struct VecOf;
template <> struct VecOf<bf16> { typedef bf16 x8 __attribute__((ext_vector_type(8))); typedef bf16 x4 __attribute__((ext_vector_type(4))); };
template <> struct VecOf<f16> { typedef f16 x8 __attribute__((ext_vector_type(8))); typedef f16 x4 __attribute__((ext_vector_type(4))); };
template <class E> using vec8 = typename VecOf<E>::x8;
template <class E> using vec4 = typename VecOf<E>::x4;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));          // of 16-bit values: at any of their addresses
constexpr int kBlock8 = 32;                   // columns that share a scale

// Workgroups of any number: a launch counts its threads along x in 32 bits, so more than kAcross of up to 1024 threads go on along y.  The last of these rows
// of workgroups may be longer than what is left.
constexpr int64_t kAcross = 1 << 21;
inline dim3 grid_of(int64_t blocks) { return dim3((uint32_t)(blocks < kAcross ? blocks : kAcross), (uint32_t)((blocks + kAcross - 1) / kAcross)); }
__device__ __forceinline__ int64_t block_of() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

template <class T> __device__ __forceinline__ T from_float(float v) { return (T)v; }

// At both ends of a branch whose accesses differ from the other branch's in nothing but where they are to be cached: else the compiler makes one access,
// of the other branch's kind, of the two
__device__ __forceinline__ void apart() { asm volatile(""); }

// N consecutive values at p, of which the first `have` exist (the others read as 0); N of them at once at any alignment of T.
template <class T, int N> __device__ __forceinline__ void load_n(const T *p, int64_t have, float (&v)[N]) {
    if (have >= N) {
        T t[N];
        __builtin_memcpy(t, p, sizeof t);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (float)t[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < have ? (float)p[i] : 0.0f;
    }
}
// ... as they are (`past`: not to be kept in the L2s)
template <class T, int N> __device__ __forceinline__ void load_raw(const T *p, int64_t have, T (&v)[N], bool past = false) {
    if (have >= N) {
        if (past) {
            apart();
#pragma unroll
            for (int i = 0; i < (int)sizeof v / 16; ++i) {
                const u32x4 w = __builtin_nontemporal_load((const u32x4 *)p + i);
                __builtin_memcpy((char *)v + i * 16, &w, 16);
            }
            apart();
        } else {
            __builtin_memcpy(v, p, sizeof v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < have ? p[i] : (T)0.0f;
    }
}
// A result that the L2s (8 of 4 MB) cannot hold goes past them (`past`): they keep what is read again, and lines that are written whole need not be
// fetched.  Measured, 134 M values: unpack 87 -> 59 us, through GELU 108 -> 86; norm's gradients of 32768 x 1024 62 -> 50; 32768 rows, 4096 <- 1024 with a
// slope 400 -> 345.  Results that fit stay: 64 x 1000 7.8 us, past the L2s 8.4.
constexpr int64_t kPastL2 = 32 << 20;
template <class T, int N> __device__ __forceinline__ void store_n(T *p, int64_t have, const float (&v)[N], bool past = false) {
    if (have >= N) {
        T t[N];
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = from_float<T>(v[i]);
        if (past) {
            apart();
#pragma unroll
            for (int i = 0; i < (int)sizeof t / 16; ++i) {
                u32x4 w;
                __builtin_memcpy(&w, (const char *)t + i * 16, 16);
                __builtin_nontemporal_store(w, (u32x4 *)p + i);
            }
            apart();
        } else {
            __builtin_memcpy(p, t, sizeof t);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < have) p[i] = from_float<T>(v[i]);
    }
}

// ---- 8-bit blocks ------------------------------------------------------------------------------------------------------------------

// Scale byte of a block whose largest magnitude has these bits: the least e in 1..254 with rint(largest / 2^(e-127)) <= 127.  Largest =
// f 2^k, 1 <= f < 2: k - 6 where 64 f < 127.5, that is where not all of the mantissa's first 7 bits are set, else k - 5; adding
// 2^16 carries into the exponent exactly there.  255 where the largest is no finite number.
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest_bits) {
    const int e = (int)((largest_bits + 0x10000u) >> 23) - 6;
    return largest_bits >= 0x7f800000u ? 255u : (uint32_t)(e < 1 ? 1 : e);
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }              // 255: in_range sees to it
__device__ __forceinline__ float inverse_of(uint32_t byte) { return byte == 255u ? 0.0f : __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// Four codes of a block: v * inverse is exact, and adding 1.5 2^23 rounds it to a whole number in the sum's low bits.  A block of 255: 0.
__device__ __forceinline__ uint32_t codes_of(const float *v, float inverse) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(__builtin_fmaf(v[i], inverse, 12582912.0f));
    const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
    return inverse == 0.0f ? 0u : lo | hi;
}
// The values of four codes (a signed byte converts in one instruction)
__device__ __forceinline__ void values_of(uint32_t word, float scale, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)(int)(int8_t)(word >> (8 * i)) * scale;
}

// Largest over four neighbouring lanes (quad_perm: lane ^ 1, lane ^ 2)
__device__ __forceinline__ uint32_t max_of_four(uint32_t m) {
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xb1, 0xf, 0xf, true);
    m = m > o ? m : o;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4e, 0xf, 0xf, true);
    return m > o ? m : o;
}

// Codes and scale of 8 values of a row that begin at column `col` (a multiple of 8); four neighbouring lanes hold a block, all of them
// here, with zeros behind the row's end.
__device__ __forceinline__ void store_packed(int8_t *codes, uint8_t *scales, int64_t row, int64_t ld, int64_t col, int64_t cols, const float (&v)[8], bool past) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t o = magnitude(v[i]);
        m = m > o ? m : o;
    }
    const uint32_t byte = scale_byte(max_of_four(m));
    const float inv = inverse_of(byte);
    if (col < (cols + kBlock8 - 1) / kBlock8 * kBlock8) {
        const u32x2 w = {codes_of(v, inv), codes_of(v + 4, inv)};
        u32x2 *const to = (u32x2 *)(codes + row * ld + col);
        if (past) {
            apart();
            __builtin_nontemporal_store(w, to);
            apart();
        } else {
            *to = w;
        }
        if ((threadIdx.x & 3) == 0) scales[row * (ld / kBlock8) + col / kBlock8] = (uint8_t)byte;
    }
}

// What a packed value beyond T's range stands for: T's largest finite number; in 32 bits bf16's, so that a product and an unpacked value are the same.  (A
// block whose largest is above 127.5 2^121 has codes of 64 and a scale of 2^122.)  Only scales from `first` on reach so far.  A block of 255 is NaN, whatever its codes.
template <class T> struct Reach { static constexpr float most = 0x1.fep127f; static constexpr uint32_t first = 249; };
template <> struct Reach<f16> { static constexpr float most = 65504.0f; static constexpr uint32_t first = 137; };
template <class T, int N> __device__ __forceinline__ void in_range(uint32_t byte, float (&v)[N]) {
    if (byte >= Reach<T>::first) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = byte == 255u ? __builtin_nanf("") : __builtin_amdgcn_fmed3f(v[i], -Reach<T>::most, Reach<T>::most);
    }
}

// ---- activations -------------------------------------------------------------------------------------------------------------------

struct Act {
    int kind;
    float w0, turn_hi, turn_lo;                                                  // w0 / 2 pi as a sum of two floats
};
inline Act make_act(int kind, float w0) {
    const double turn = (double)w0 * 0.15915494309189533577;
    const float hi = (float)turn;
    return {kind, w0, hi, (float)(turn - (double)hi)};
}

// The normal distribution's tail above |z|: e^(-z^2/2) times half of erfcx(|z| / sqrt 2), and that as a polynomial of t = 1 / (1 + p |z|).  The coefficients are
// fits of this framework's own (least squares, weighted anew until the largest error stops falling) up to |z| = 13.3, where the bell leaves 32 bits.  Of results of 16 bits
// the tail is held to 3.6e-8, and to 3.6e-5 of itself; of 32 bits to 1.5e-7 of itself from kGeluNear on, and below that the normal distribution's
// odd part, a polynomial of z^2, to 3e-10 of itself: so the error's norm for normal z is 3.1e-8 (elementary operations in 32 bits: 3.8e-8), the slope's 4.4e-8 (4.0e-8).  The bell is
// what the derivative needs too.
struct Gauss { float upper, bell; };
constexpr float kGeluNear = 1.25f;
template <int N> __device__ __forceinline__ float polynomial(const float (&c)[N], float t) {
    float v = c[N - 1];
#pragma unroll
    for (int i = N - 2; i >= 0; --i) v = __builtin_fmaf(v, t, c[i]);
    return v;
}
template <class T> __device__ __forceinline__ Gauss gauss_of(float z) {
    constexpr bool kWide = sizeof(T) == 4;
    constexpr float c16[] = {2.76409489e-4f, 0.154583347f, 0.195337404f, 0.00238212468f, 0.34939965f, -0.259232893f, 0.0572539932f};
    constexpr float c32[] = {1.37733018e-5f, 0.199068725f, 0.204343468f, 0.117957172f, 0.168213515f, -0.310400943f, 0.122242786f};
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(z), kWide ? 0.5f : 0.4f, 1.0f));
    const float bell = __builtin_amdgcn_exp2f(z * z * (-0.5f * 1.4426950408889634f));
    return {polynomial(kWide ? c32 : c16, t) * bell, bell};
}
// The distribution less a half, |z| < kGeluNear
__device__ __forceinline__ float gauss_near(float z) {
    constexpr float c[] = {0.39894228f, -0.0664903744f, 0.00997349993f, -0.00118710961f, 1.15032157e-4f, -9.05844081e-6f, 4.76074771e-7f};
    return z * polynomial(c, z * z);
}
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z)); }
// w0 z in turns, the unit of the hardware's sine, to the last bits of its fraction: one rounding of the product alone would cost
// 2^-24 of as many turns as there are
__device__ __forceinline__ float turns(float z, const Act &a) {
    const float r = z * a.turn_hi;
    return __builtin_amdgcn_fractf(r) + __builtin_fmaf(z, a.turn_lo, __builtin_fmaf(z, a.turn_hi, -r));
}

// Beyond these the bell and exp(-|z|) are 0 in 32 bits.  z itself is held to them wherever it is multiplied by what has vanished there, so that an infinity
// gives the limit and no NaN; a NaN stays one by the other factor.  (A z kept in f16 is infinite beyond 65504.)
constexpr float kGeluFlat = 16.0f, kSiluFlat = 128.0f;
__device__ __forceinline__ float held(float z, float low, float high) { return __builtin_amdgcn_fmed3f(z, low, high); }

template <class T> __device__ __forceinline__ float gelu(float z) {
    const float far = __builtin_fmaf(-__builtin_fabsf(held(z, -kGeluFlat, kGeluFlat)), gauss_of<T>(z).upper, __builtin_fmaxf(z, 0.0f));
    return sizeof(T) == 4 && __builtin_fabsf(z) < kGeluNear ? __builtin_fmaf(z, gauss_near(z), 0.5f * z) : far;
}
template <class T> __device__ __forceinline__ float gelu_slope(float z) {
    const Gauss g = gauss_of<T>(z);
    const float far = z > 0.0f ? 1.0f - g.upper : g.upper, below = sizeof(T) == 4 && __builtin_fabsf(z) < kGeluNear ? 0.5f + gauss_near(z) : far;
    return __builtin_fmaf(held(z, -kGeluFlat, kGeluFlat) * 0.39894228040143268f, g.bell, below);
}

// Eight values through an activation to results of T; eight gradients times its slopes at z
template <class T> __device__ __forceinline__ void act_all(float (&v)[8], const Act &a) {
    switch (a.kind) {
        case RINR_ACT_RELU:
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];        // a NaN stays one
            break;
        case RINR_ACT_GELU:
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = gelu<T>(v[i]);
            break;
        case RINR_ACT_SILU:
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = held(v[i], -kSiluFlat, __builtin_inff()) * sigmoid(v[i]);
            break;
        case RINR_ACT_SINE:
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __builtin_amdgcn_sinf(turns(v[i], a));
            break;
        default: break;
    }
}
template <class T> __device__ __forceinline__ void slope_all(float (&d)[8], const float (&z)[8], const Act &a) {
    switch (a.kind) {
        case RINR_ACT_RELU:
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] *= z[i] > 0.0f ? 1.0f : 0.0f;
            break;
        case RINR_ACT_GELU:
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] *= gelu_slope<T>(z[i]);
            break;
        case RINR_ACT_SILU:
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float g = sigmoid(z[i]);
                d[i] *= g * (1.0f + held(z[i], -kSiluFlat, kSiluFlat) * (1.0f - g));
            }
            break;
        case RINR_ACT_SINE:
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] *= a.w0 * __builtin_amdgcn_cosf(turns(z[i], a));
            break;
        default: break;
    }
}

// 8 values (from column `col` on, a multiple of 8; `have` of them exist) of a row kept as dtype T or packed: what memory gives, and the values.  A
// packed value beyond T's range is T's largest.
template <class T> struct Kept {
    T v[8];
    uint32_t w[2], byte;
    __device__ __forceinline__ void load(const void *p, const uint8_t *scales, int64_t ld, bool packed, int64_t row, int64_t col, int64_t have) {
        if (packed) {                                                            // whole blocks are there, whatever `have` is
            __builtin_memcpy(w, (const int8_t *)p + row * ld + col, 8);
            byte = scales[row * (ld / kBlock8) + col / kBlock8];
        } else {
            load_raw((const T *)p + row * ld + col, have, v);
        }
    }
    __device__ __forceinline__ void get(bool packed, float (&o)[8]) const {
        if (packed) {
            const float s = scale_of(byte);
            values_of(w[0], s, o);
            values_of(w[1], s, o + 4);
            in_range<T>(byte, o);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (float)v[i];
        }
    }
};

}  // namespace rinr_nn
#endif
