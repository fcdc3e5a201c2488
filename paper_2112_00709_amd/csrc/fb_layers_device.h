// Shared by the kernels of the network-side operators (fb_layers.h): element types, 16-byte pieces of rows that start at
// any element, sums and maxima over a wave.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>
#include <type_traits>

#include "../../include/fb_layers.h"
#include "fb_internal.h"

namespace fb {

int fail(int code, const std::string &msg);

namespace {

constexpr int kCUs = 256;   // compute units of the GPU

typedef __bf16 bf16;
typedef _Float16 f16;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));    // 16 bytes at any element: the hardware takes such addresses
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <class T>
struct Vec {                                            // one 16-byte piece
    static constexpr int kN = 16 / (int)sizeof(T);
};

// The piece as floats.
template <class T>
__device__ __forceinline__ void unpack(const u32x4 &r, float *v)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
    } else if constexpr (std::is_same<T, bf16>::value) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(r[i] << 16);
            v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = r[i];
            f16 h[2];
            __builtin_memcpy(h, &u, 4);
            v[2 * i] = (float)h[0];
            v[2 * i + 1] = (float)h[1];
        }
    }
}

template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const T h[2] = {(T)a, (T)b};
    uint32_t u;
    __builtin_memcpy(&u, h, 4);
    return u;
}

template <class T>
__device__ __forceinline__ u32x4 pack(const float *v)
{
    u32x4 r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
    }
    return r;
}

// Elements [0, n) of the piece at p, the others 0; n may be anything.  A piece that is whole is one load.
template <class T>
__device__ __forceinline__ u32x4 load_piece(const T *p, int n)
{
    constexpr int kN = Vec<T>::kN;
    u32x4 r = {0, 0, 0, 0};
    if (n >= kN) {
        r = *(const u32x4_any *)p;
    } else if (n > 0) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            if (i < n) {
                if constexpr (sizeof(T) == 4) {
                    r[i] = ((const uint32_t *)p)[i];
                } else {
                    r[i / 2] |= (uint32_t)((const uint16_t *)p)[i] << (16 * (i & 1));
                }
            }
        }
    }
    return r;
}

// Around a store past the caches: keeps the compiler from making one store of it and of the other branch's.
__device__ __forceinline__ void apart() { asm volatile(""); }

// Elements [0, n) of a piece to p; with `past` whole pieces go past the caches (see goes_past).
template <class T>
__device__ __forceinline__ void store_piece(T *p, int n, const u32x4 &r, bool past = false)
{
    constexpr int kN = Vec<T>::kN;
    if (n >= kN) {
        if (past) {
            apart();
            __builtin_nontemporal_store(r, (u32x4_any *)p);
            apart();
        } else {
            *(u32x4_any *)p = r;
        }
    } else if (n > 0) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            if (i < n) {
                if constexpr (sizeof(T) == 4) {
                    ((uint32_t *)p)[i] = r[i];
                } else {
                    ((uint16_t *)p)[i] = (uint16_t)(r[i / 2] >> (16 * (i & 1)));
                }
            }
        }
    }
}

// One element.
template <class T>
__device__ __forceinline__ float load_one(const T *p) { return (float)*p; }

template <int CTRL>
__device__ __forceinline__ uint32_t lane_move(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}

// op over all 64 lanes, in every lane, always in the same order: inside rows of 16 lanes by moves, across rows by the two
// exchanges of halves.
template <class Op>
__device__ __forceinline__ uint32_t over_wave(uint32_t v, Op op)
{
    v = op(v, lane_move<0xB1>(v));     // quad_perm [1,0,3,2]
    v = op(v, lane_move<0x4E>(v));     // quad_perm [2,3,0,1]
    v = op(v, lane_move<0x141>(v));    // row_half_mirror
    v = op(v, lane_move<0x140>(v));    // row_mirror
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = op(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return op(b[0], b[1]);
}
// op over the lane's row of 16 lanes, in each of them.
template <class Op>
__device__ __forceinline__ uint32_t over_row(uint32_t v, Op op)
{
    v = op(v, lane_move<0xB1>(v));
    v = op(v, lane_move<0x4E>(v));
    v = op(v, lane_move<0x141>(v));
    return op(v, lane_move<0x140>(v));
}
__device__ __forceinline__ float sum_row16(float v)
{
    return __uint_as_float(over_row(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ __forceinline__ float max_row16(float v)
{
    return __uint_as_float(over_row(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
__device__ __forceinline__ float sum_wave(float v)
{
    return __uint_as_float(over_wave(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
// NaN loses against any number.
__device__ __forceinline__ float max_wave(float v)
{
    return __uint_as_float(over_wave(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
__device__ __forceinline__ uint32_t max_wave_u(uint32_t v)
{
    return over_wave(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

}  // namespace

// Host side: argument checks that the calls share.
inline bool known_type(int t) { return t == FB_TYPE_F32 || t == FB_TYPE_BF16 || t == FB_TYPE_F16; }
inline size_t type_bytes(int t) { return t == FB_TYPE_F32 ? 4 : 2; }
constexpr int64_t kMostSize = (int64_t)1 << 31, kMostWidth = (int64_t)1 << 28;
inline bool bad_rows(int64_t n) { return n < 0 || n >= kMostSize; }
inline bool bad_width(int64_t n) { return n < 1 || n >= kMostWidth; }
inline bool bad_ld(int64_t ld, int64_t width) { return ld < width || ld >= kMostSize; }

// Outputs that the caches cannot keep for their reader are stored past them: nothing has to be written back first to make room.
// Called again and again on the same tensors: 69120 x 1024 in bfloat16, layer norm and its gradient, 45 and 72 us instead of 51
// and 83; 4095 x 32001, gradient of log probabilities, 89 instead of 107 (on other tensors each time 53, 81 and 104 instead of 55, 83 and 103); 69120 x 3000 products, 1024 long: 472 instead of 504.  Smaller ones are read from the caches:
// 20000 x 1024, layer norm, products and log probabilities one after the other, 97 us past them and 89 through them.
inline bool goes_past(int64_t rows, int64_t width, int type) { return rows * width * (int64_t)type_bytes(type) >= (int64_t)128 << 20; }

inline int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FB_OK : fail(FB_EHIP, std::string(what) + hipGetErrorString(e));
}

// f, with whatever it throws (memory for a message) turned into a code.
template <class F>
int guarded(F f) noexcept
{
    try {
        return f();
    } catch (...) {
        return FB_ENOMEM;
    }
}

}  // namespace fb
