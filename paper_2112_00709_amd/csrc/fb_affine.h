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

// What becomes of the sums: y = act(sum + bias[j]) + residual, preact = sum + bias[j].  Sums of 16-bit products whose first
// factor is dz are taken times *undo before that (see fb_peak_kernel and scale_of).
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

// Log probabilities whose logits are the product's sums (see fb_vocabulary.hip).
struct Scores {
    const int32_t *tokens;   // [M]
    int first;               // the number of the product's first column as a token
    float *given;            // [M]: the tokens' logits
    float *stats;            // [tiles across][3][M]
    const void *rows;        // [M] fours of what the gradient takes of a row
    float *sums;             // [waves down][N]: shares of the sums of the gradient's columns, nullable
    const uint64_t *live;    // of a product over rows, bit k % 64 of word k / 64: row k of the second factor counts; one word more; nullable
    int64_t low;             // rows from a row of the gradient to the one with what it lacks, 0: none
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
    Scores s;
};

int launch_mfma_product(const Product &q, hipStream_t stream);   // factors as ready() wants them

// Both products of a gradient in one launch, if their workgroups fit the GPU together.
bool fits_as_pair(const Product &dx, const Product &dw);
int launch_mfma_pair(const Product &dx, const Product &dw, hipStream_t stream);

// Few rows of x (M <= kFewRows), both factors along k, at any address and distance.
constexpr int64_t kFewRows = 64;
int launch_few_rows(const Product &q, hipStream_t stream);

// Gated layers: B is the gate's N rows and the other factor's N behind them, N the outputs' width.
int launch_few_pairs(const Product &q, hipStream_t stream);

// Whether the matrix units' kernel can take a factor as it is: whole 16-byte pieces, at addresses and distances that are
// multiples of 16 bytes, and a tile's rows within the 2^31 bytes of a buffer.  `width`: the length of its rows in memory.
inline bool ready(const void *p, int64_t ld, int64_t width, int type)
{
    const int64_t piece = 16 / (int64_t)type_bytes(type);
    return ((uintptr_t)p & 15) == 0 && ld % piece == 0 && width % piece == 0 && ld * (int64_t)type_bytes(type) < (int64_t)1 << 22;
}

// Rows made before the products: dz = dy act'(z), or a copy in rows of whole pieces, and shares of the sums of their columns.
struct SlopeParams {
    const void *dy, *z;
    int64_t lddy, ldz, M, N, ldo;
    int act;
    void *out;           // dz as the products take it, nullable
    float *part;         // [down][N]: shares of the sums over rows, nullable
    int lanes;           // a row: a power of two, 64 where the rows are wider than that many pieces
    int wide, down;      // workgroups along the width and along the rows
    const uint32_t *peaks;   // half precision: shares of the largest |dy| that sets the power of two out is taken times, nullable
    int n_peaks;
    float *undo;         // its inverse, out
};

void lay_out(SlopeParams &p, int type);
int64_t sum_rows(int64_t M, int64_t N, int type);   // the shares of sums over M rows of N elements

// Up to three jobs that make rows, the first from rows of another type.
struct PrepareParams {
    SlopeParams job[3];
    int last[3];             // workgroups [last[i - 1], last[i]) have job i
};

// Jobs that make rows, in one launch; the first has rows of dy_type.
struct Prepare {
    PrepareParams p{};
    int n = 0, blocks = 0;
    void add(SlopeParams s, int type)
    {
        lay_out(s, type);
        p.job[n] = s;
        blocks += s.wide * s.down;
        p.last[n++] = blocks;
        for (int i = n; i < 3; ++i) p.last[i] = blocks;
    }
};

int launch_prepare(Prepare &j, int type, int dy_type, hipStream_t stream);

inline size_t aligned(size_t n) { return (n + 255) & ~(size_t)255; }

double plan(Product &q, int only_tile = 0, bool whole = false);   // tiles and shares of k (`whole`: one share); what it takes, in clocks
inline size_t product_bytes(const Product &q) { return q.parts ? aligned((size_t)q.split * (size_t)q.M * (size_t)q.N * sizeof(float)) : 0; }
bool plan_back(Product &dx, Product &dw);
int64_t rows_in_rounds(const Product &q, Product &last);          // rows that go in whole rounds of large tiles, before those of `last`; 0: all at once
int launch_dx(const Product &q, hipStream_t stream);              // by launch_mfma_product, perhaps in two
int launch_join(const Product *a, const Product *b, int type, const float *sums, int64_t rows, int64_t N, float *out, hipStream_t stream);

inline int64_t whole_pieces(int64_t width, int type)
{
    const int64_t piece = 16 / (int64_t)type_bytes(type);
    return (width + piece - 1) / piece * piece;
}

// The distance of rows that are made for the products: whole 128-byte lines, so that the 128 bytes of a step along k are one line and
// not parts of two (65536 x 3000 x 1024 in bfloat16, dx: 442 us at a distance of 3000 elements, 356 at 3008; dW 391 and 361).  Rows of
// less than 512 bytes are left at whole pieces: lines would be a quarter of them and more.
inline int64_t line_distance(int64_t width, int type)
{
    const int64_t line = 128 / (int64_t)type_bytes(type);
    return width < 4 * line ? whole_pieces(width, type) : (width + line - 1) / line * line;
}

// A matrix that the matrix units' kernel cannot take as it is, copied to rows of whole pieces (padded with zeros).
struct Packed {
    bool copy;
    int64_t ld;
    size_t bytes;
};

inline Packed packed(const void *p, int64_t ld, int64_t rows, int64_t width, int type, bool always = false)
{
    Packed k{};
    k.copy = always || !ready(p, ld, width, type);
    k.ld = k.copy ? line_distance(width, type) : ld;
    k.bytes = k.copy ? aligned((size_t)rows * (size_t)k.ld * type_bytes(type)) : 0;
    return k;
}

// The job that makes the copy (nothing if none is needed).
inline SlopeParams pack_job(const Packed &k, const void *p, int64_t ld, int64_t rows, int64_t width, void *to)
{
    return SlopeParams{p, nullptr, ld, 0, rows, width, k.ld, FB_ACT_NONE, to, nullptr, 0, 0, 0, nullptr, 0, nullptr};
}

// What the matrix units' kernel addresses in 32 bits: 64 or 128 rows of a factor, 16 rows of what it stores or adds.
inline bool too_long(int64_t width, int type) { return width * (int64_t)type_bytes(type) > (int64_t)1 << 22; }
inline bool too_far(int64_t ld) { return ld >= (int64_t)1 << 27; }

inline bool bad_sizes(int64_t M, int64_t N, int64_t K) { return bad_rows(M) || bad_width(N) || bad_width(K); }

// A dz that is rounded to 16 bits adds its roundings to those of the gradients: 2^0.5 of them on the average of many rows, but up to three times
// where few count (a row whose token has nearly all of its gradient).  Few rows cost little in the products, so their dz is kept as two
// numbers of 16 bits each, the second what the first lacks, M rows further down.  dx adds the sums of row i and row M + i, dW takes x twice.
// Bfloat16, log probabilities: 16 rows of 3000 x 1024 30 instead of 27 us, of 128000 x 1024 162 instead of 156; 64 rows 201 instead of 173; at
// 128 rows it would be 276 instead of 207.  Up to 128 rows (whose bits in Scores::live one workgroup sets) that are multiplied in less time than
// launches take have it too: 128 rows of 300 x 256 26.6 and 26.8 us, of 3000 x 1024 39 and 31.5.  (The host knows M, not how many of the rows count:
// see scale_of for what is done where few of many do.)
inline bool twice(int64_t M, int64_t N, int64_t K, int type)
{
    return type != FB_TYPE_F32 && M > 0 && (M <= 64 || (M <= 128 && N * K <= ((int64_t)1 << 24) / M));
}

// dx as launch_join takes it: the sums of the second M rows are further shares of the first.
inline Product joined_rows(const Product &dx, bool twice)
{
    Product q = dx;
    if (twice) {
        q.M /= 2;
        q.split *= 2;
    }
    return q;
}

// The two products of the gradient.
struct GradPlan {
    Product dx, dw;
    bool pair;            // in one launch
    bool slope;           // dz has to be made, or dy laid out anew
    bool scale;           // and is rounded to half precision: times a power of two
    bool twice;           // dz is two rows of 16 bits for each of M, see twice()
    int64_t ldz;
    Packed x, w;
    size_t dz, sums, range, part, bytes;
};

GradPlan grad_plan(const void *dy, int64_t lddy, int dy_type, const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N, int64_t K, int type,
                   int act);
int launch_grad(GradPlan &g, const Factor &d, const float *undo, void *dx, int64_t lddx, void *dweight, float *part, const float *sums, int64_t rows, float *dbias,
                hipStream_t stream);

// What the gradient of log probabilities from hidden frames is made of, for pieces of `width` of the vocabulary.
struct ScoreGradPlan {
    int64_t width, pieces, ldz;
    Product z, dx, dw;       // of a whole piece
    Packed x, w;
    bool pair;               // both products in one launch
    bool twice;              // dz is two rows of 16 bits for each of M, see twice()
    int64_t sum_rows;
    size_t dz, rows, picks, live, range, sums, acc, part_x, part_w, bytes;
};

ScoreGradPlan score_grad_plan(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t V, int64_t K, int type);

constexpr int kPeakGroups = kCUs;    // four peaks a lane for those who need the largest

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
    if (act == FB_ACT_SIGMOID) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -kLog2E));
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
    if (act == FB_ACT_SIGMOID) {                                 // s(z) s(-z), in which no digits cancel
        const float e = __builtin_amdgcn_exp2f(-fabsf(z) * kLog2E), s = __builtin_amdgcn_rcpf(1.0f + e);
        return e * s * s;
    }
    return 1.0f;
}

// act(z) and act'(z) together: they share their exponentials.
__device__ __forceinline__ void act_and_slope(float z, int act, float &value, float &slope)
{
    if (act == FB_ACT_GELU) {
        float e;
        const float h = normal_tail(z, e), p = z > 0.0f ? 1.0f - h : h;
        value = z * p;
        slope = fmaf(z * e, 0.39894228040143267794f, p);
    } else if (act == FB_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -kLog2E));
        value = z * s;
        slope = s * fmaf(z, 1.0f - s, 1.0f);
    } else {
        value = act_of(z, act);
        slope = act_slope(z, act);
    }
}

// A number that |act(z)| does not exceed, and is not far above it: z is where z > 0, and the least value of gelu is -0.17, of silu
// -0.2785.  NaN for NaN.
__device__ __forceinline__ float act_bound(float z, int act)
{
    if (act == FB_ACT_NONE) return fabsf(z);
    if (act == FB_ACT_SIGMOID) return z != z ? z : 1.0f;
    const float least = act == FB_ACT_RELU ? 0.0f : act == FB_ACT_GELU ? 0.171f : 0.279f;
    return z < least ? least : z;
}
// The same of |act'(z)|.
__device__ __forceinline__ float slope_bound(float z, int act)
{
    if (act == FB_ACT_NONE) return 1.0f;
    if (act == FB_ACT_SIGMOID) return 0.25f;
    if (act == FB_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    return z > 0.0f ? 1.13f : 0.51f;
}

// The power of two for a largest |dy|, and its inverse; both are normal numbers whatever the largest is.
__device__ __forceinline__ void range_of_peak(uint32_t peak, float &scale, float &undo)
{
    const uint32_t e = peak >> 23, up = peak == 0 ? 127 : e < 15 ? 253 : 268 - e;      // 2^(14 - (e - 127))
    scale = __uint_as_float(up << 23);
    undo = __uint_as_float((254 - up) << 23);
}
// The largest of shares of it.
__device__ __forceinline__ uint32_t largest_of(const uint32_t *peaks, int n)
{
    const int lane = threadIdx.x & 63;
    uint32_t peak = 0;
#pragma unroll
    for (int i = 0; i < kPeakGroups; i += 64) {
        const uint32_t one = i + lane < n ? peaks[i + lane] : 0;
        peak = one > peak ? one : peak;
    }
    return max_wave_u(peak);
}
__device__ __forceinline__ void range_of(const uint32_t *peaks, int n, float &scale, float &undo) { range_of_peak(largest_of(peaks, n), scale, undo); }

// dz = dy act'(z) (or a copy of dy in rows of whole pieces), rounded to the factors' type, and the sums of its columns before
// the rounding.  Bound by memory: 44160 x 2048 in bfloat16 with max(z, 0) take 100 us, 5.4 TB/s.  A thread has one piece of the
// width; `lanes` threads have a row side by side, so narrow rows fill the waves too, and kRowsAhead rows are asked for before the
// first is worked on.  The sums of a workgroup's threads over its rows are added in a fixed order.
constexpr int kRowsAhead = 4;

template <class T, class D>
__device__ __forceinline__ void make_rows(const SlopeParams &p, int block, float (*slots)[Vec<T>::kN + 1])
{
    constexpr int VE = Vec<T>::kN, VD = Vec<D>::kN;
    const int across = block % p.wide, down = block / p.wide;
    const int lane = threadIdx.x & (p.lanes - 1), sub = threadIdx.x / p.lanes, subs = 256 / p.lanes;
    const int64_t at = ((int64_t)across * p.lanes + lane) * VE;
    const int n = at >= p.N ? 0 : (int)(p.N - at < VE ? p.N - at : VE);
    float sum[VE] = {}, scale = 1.0f;
    if constexpr (std::is_same<T, f16>::value) {
        if (p.peaks) {
            float undo;
            range_of(p.peaks, p.n_peaks, scale, undo);
            if (block == 0 && threadIdx.x == 0) *p.undo = undo;
        }
    }
    if (n > 0) {
        const int64_t step = (int64_t)p.down * subs;
        for (int64_t r0 = (int64_t)down * subs + sub; r0 < p.M; r0 += kRowsAhead * step) {
            u32x4 rg[kRowsAhead][VE / VD], rz[kRowsAhead];
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u) {
                const int64_t r = r0 + u * step;
                const int here = r < p.M ? n : 0;
#pragma unroll
                for (int e = 0; e < VE / VD; ++e) rg[u][e] = load_piece((const D *)p.dy + r * p.lddy + at + e * VD, here - e * VD);
                if (p.act != FB_ACT_NONE) rz[u] = load_piece((const T *)p.z + r * p.ldz + at, here);
            }
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u) {
                const int64_t r = r0 + u * step;
                float g[VE];
#pragma unroll
                for (int e = 0; e < VE / VD; ++e) unpack<D>(rg[u][e], g + e * VD);
                if (p.act != FB_ACT_NONE) {
                    float z[VE];
                    unpack<T>(rz[u], z);
#pragma unroll
                    for (int e = 0; e < VE; ++e) g[e] = e < n && r < p.M ? g[e] * act_slope(z[e], p.act) : 0.0f;
                }
#pragma unroll
                for (int e = 0; e < VE; ++e) sum[e] += g[e];
                if constexpr (std::is_same<T, f16>::value) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) g[e] *= scale;
                }
                if (p.out && r < p.M) store_piece((T *)p.out + r * p.ldo + at, VE, pack<T>(g));   // (rows of whole pieces)
            }
        }
    }
    if (!p.part) return;
#pragma unroll
    for (int e = 0; e < VE; ++e) slots[threadIdx.x][e] = sum[e];
    __syncthreads();
    for (int c = threadIdx.x; c < p.lanes * VE; c += 256) {
        const int64_t col = (int64_t)across * p.lanes * VE + c;
        if (col >= p.N) continue;
        float s = 0.0f;
        for (int i = 0; i < subs; ++i) s += slots[i * p.lanes + c / VE][c % VE];
        p.part[(size_t)down * p.N + col] = s;
    }
}

// Workgroup `block` of the jobs'.
template <class T, class D>
__device__ __forceinline__ void prepare_block(const PrepareParams &p, int block, float (*slots)[Vec<T>::kN + 1])
{
    if (block < p.last[0])
        make_rows<T, D>(p.job[0], block, slots);
    else if (block < p.last[1])
        make_rows<T, T>(p.job[1], block - p.last[0], slots);
    else
        make_rows<T, T>(p.job[2], block - p.last[1], slots);
}

// Copies alone, in the launch of a kernel that they go with.
template <class T>
__device__ __forceinline__ void copy_block(const PrepareParams &p, int block, float (*slots)[Vec<T>::kN + 1])
{
    const int which = block < p.last[0] ? 0 : block < p.last[1] ? 1 : 2;
    SlopeParams job = p.job[0];
    if (which == 1) job = p.job[1];
    if (which == 2) job = p.job[2];
    make_rows<T, T>(job, block - (which == 0 ? 0 : which == 1 ? p.last[0] : p.last[1]), slots);
}

// What `high`, which is v rounded, lacks of v (nothing where they are not finite).
__device__ __forceinline__ float lacks(float v, float high)
{
    const float low = v - high;
    return fabsf(low) < __builtin_huge_valf() ? low : 0.0f;
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

// A pair of sums of a gated layer finished and stored: y = act(g + bias[j]) (u + bias[N + j]), preact both before that.
template <class T>
__device__ __forceinline__ void finish_pair(const Finish &f, int64_t N, int64_t i, int64_t j, float g, float u)
{
    if (f.bias) {
        g += f.bias[j];
        u += f.bias[N + j];
    }
    if (f.preact) {
        T *z = (T *)f.preact + i * f.ldp + j;
        z[0] = (T)g;
        z[N] = (T)u;
    }
    ((T *)f.y)[i * f.ldy + j] = (T)(act_of(g, f.act) * u);
}

}  // namespace

}  // namespace fb
