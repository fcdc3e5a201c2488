// Shared by the files of the affine operator: what a product is, and what is done with its sums.
#pragma once

#include "fb_layers_device.h"

namespace fb {

// One factor of a product C[i][j] = sum over k of A[i][k] B[j][k].  `along`: the elements of a row (ld apart from the next)
// run along k; otherwise along i or j, and row k + 1 follows row k.
struct Factor {
    const void *p;
    int64_t ld;
    bool along;
};

// What becomes of the sums: y = act(sum + bias[j]) + residual, preact = sum + bias[j].
struct Finish {
    const float *bias;
    const void *residual;
    int64_t ldr;
    int act;
    void *y;
    int64_t ldy;
    int out_type;
    void *preact;        // of the factors' type
    int64_t ldp;
};

struct Product {
    Factor A, B;
    int64_t M, N, K;     // i < M, j < N, k < K
    int type;            // of the factors
    Finish f;
    float *part;         // split > 1: [split][M][N] sums of shares of k
    int split;
    int64_t share;       // length of a share
    int tile;            // 16-bit factors: 256 or 128, the side of the tiles
};

int launch_mfma_product(const Product &q, hipStream_t stream);   // 16-bit factors, see ready()

// Whether the matrix units' kernel can take a factor as it is: whole 16-byte pieces, at addresses and distances that are
// multiples of 16 bytes, and a tile's rows within the 2^31 bytes of a buffer.  `width`: the length of its rows in memory.
inline bool ready(const void *p, int64_t ld, int64_t width)
{
    return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && width % 8 == 0 && ld < (int64_t)1 << 21;
}

namespace {

__device__ __forceinline__ float act_of(float z, int act)
{
    if (act == FB_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
    if (act == FB_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752440f));
    if (act == FB_ACT_SILU) return z / (1.0f + __expf(-z));
    return z;
}

__device__ __forceinline__ float act_slope(float z, int act)
{
    if (act == FB_ACT_RELU) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
    if (act == FB_ACT_GELU)
        return fmaf(z * __expf(-0.5f * z * z), 0.39894228040143267794f, 0.5f * (1.0f + erff(z * 0.70710678118654752440f)));
    if (act == FB_ACT_SILU) {
        const float e = __expf(-z), s = 1.0f / (1.0f + e);
        return s * fmaf(z, e == __builtin_huge_valf() ? 1.0f : e * s, 1.0f);   // 1 - s = e s
    }
    return 1.0f;
}

template <class T>
__device__ __forceinline__ float load_as(const void *p, int type)
{
    return type == FB_TYPE_F32 ? *(const float *)p : (float)*(const T *)p;
}

// One sum finished and stored.  T: the factors' type.
template <class T>
__device__ __forceinline__ void finish_one(const Finish &f, int64_t i, int64_t j, float s)
{
    if (f.bias) s += f.bias[j];
    if (f.preact) ((T *)f.preact)[i * f.ldp + j] = (T)s;
    s = act_of(s, f.act);
    if (f.out_type == FB_TYPE_F32) {
        if (f.residual) s += ((const float *)f.residual)[i * f.ldr + j];
        ((float *)f.y)[i * f.ldy + j] = s;
    } else {
        if (f.residual) s += (float)((const T *)f.residual)[i * f.ldr + j];
        ((T *)f.y)[i * f.ldy + j] = (T)s;
    }
}

}  // namespace

}  // namespace fb
