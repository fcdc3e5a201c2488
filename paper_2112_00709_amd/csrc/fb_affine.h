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

// What becomes of the sums: y = act(sum + bias[j]) + residual, preact = sum + bias[j].  Sums of half-precision products whose first
// factor is dz are taken times *undo before that (see fb_peak_kernel).
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
    const float *undo;   // nullable
};

struct Product {
    Factor A, B;
    int64_t M, N, K;     // i < M, j < N, k < K
    int type;            // of the factors
    Finish f;
    bool parts;          // the sums of shares of k go to part, [split][M][N], to be joined and finished
    float *part;
    int split;
    int64_t share;       // length of a share
    int tile;            // 256, 128 or 64, the side of the tiles
    bool past;           // y goes past the caches (never parts: they are joined at once)
};

int launch_mfma_product(const Product &q, hipStream_t stream);   // factors as ready() wants them

// Both products of a gradient in one launch, if their workgroups fit the GPU together.
bool fits_as_pair(const Product &dx, const Product &dw);
int launch_mfma_pair(const Product &dx, const Product &dw, hipStream_t stream);

// Few rows of x (M <= kFewRows), both factors along k, at any address and distance.
constexpr int64_t kFewRows = 64;
int launch_few_rows(const Product &q, hipStream_t stream);

// Whether the matrix units' kernel can take a factor as it is: whole 16-byte pieces, at addresses and distances that are
// multiples of 16 bytes, and a tile's rows within the 2^31 bytes of a buffer.  `width`: the length of its rows in memory.
inline bool ready(const void *p, int64_t ld, int64_t width, int type)
{
    const int64_t piece = 16 / (int64_t)type_bytes(type);
    return ((uintptr_t)p & 15) == 0 && ld % piece == 0 && width % piece == 0 && ld * (int64_t)type_bytes(type) < (int64_t)1 << 22;
}

namespace {

constexpr float kLog2E = 1.44269504088896340736f;

// Phi(-|z|) and e^(-z^2/2).  Phi(-|z|) = e^(-z^2/2) P(t) / 2 with t = 1 / (1 + 0.4375 |z| / sqrt 2): P, of degree 8 and without a
// constant, is fitted to e^(x^2) erfc(x) over t in [1 / (1 + 0.4375 * 11), 1] by least squares with weights moved towards equal
// relative errors: 1.6e-7, with the roundings 5.6e-7 for |z| up to 2.  Further out the exponent's rounding counts, which grows as
// the exponent does: 1.5e-6 at 5.5, 7.4e-6 at 12.5, of values of 2e-8 and 4e-36.  (A library erf takes three times the
// instructions, and its difference from 1 has no digits left in the tail.)
__device__ __forceinline__ float normal_tail(float z, float &e)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.4375f * 0.70710678118654752440f, 1.0f));
    e = __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2E));
    float s = 0.5f * 0.07202345877885818f;
    s = fmaf(s, t, 0.5f * -0.2865780293941498f);
    s = fmaf(s, t, 0.5f * 0.3185701072216034f);
    s = fmaf(s, t, 0.5f * -0.036119312047958374f);
    s = fmaf(s, t, 0.5f * 0.22321322560310364f);
    s = fmaf(s, t, 0.5f * 0.2143726497888565f);
    s = fmaf(s, t, 0.5f * 0.24772194027900696f);
    s = fmaf(s, t, 0.5f * 0.24679607152938843f);
    return s * t * e;
}

__device__ __forceinline__ float act_of(float z, int act)
{
    if (act == FB_ACT_RELU) return z <= 0.0f ? 0.0f : z;         // (NaN stays)
    if (act == FB_ACT_GELU) {
        float e;
        const float h = normal_tail(z, e);
        return z * (z > 0.0f ? 1.0f - h : h);
    }
    if (act == FB_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -kLog2E));
    return z;
}

__device__ __forceinline__ float act_slope(float z, int act)
{
    if (act == FB_ACT_RELU) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
    if (act == FB_ACT_GELU) {                                    // Phi(z) + z e^(-z^2/2) / sqrt(2 pi)
        float e;
        const float h = normal_tail(z, e);
        return fmaf(z * e, 0.39894228040143267794f, z > 0.0f ? 1.0f - h : h);
    }
    if (act == FB_ACT_SILU) {                                    // s (1 + z (1 - s))
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -kLog2E));
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    return 1.0f;
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
