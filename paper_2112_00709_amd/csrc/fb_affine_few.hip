// The affine layer for few rows of x (single frames, small batches of them): bound by reading the weight once.
//
// A workgroup has 16 rows of the weight and all rows of x, up to 64; its waves share k, each taking every WAVES-th step of it, so
// that together they read runs of 256 bytes and more of a row.  What a lane loads (16 bytes of a row) is what the matrix
// instruction takes, rows of the weight against rows of x, so nothing passes through LDS but the waves' sums at the end, where
// they are added in the waves' order.  With 16 rows a workgroup all compute units have work from N = 4081 on.
// One row by 2048 x 2048 in bfloat16 takes 6 us (8.4 MB: 1.7 at a copy's rate; the rest is a launch and one trip to memory, with
// half of the compute units at work),
// 16 rows by 4096 x 4096 11 us, 64 rows by 2048 x 2048 12 us; 65 rows take 15 in the tiled kernel.
// A gated layer's workgroup has 8 rows of either factor: their sums are in the lower and the upper half of the lanes.
#include "fb_affine.h"

namespace fb {

namespace {

typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));

// sums of 4 * 16 / sizeof(T) k added: a, b hold 16 bytes of row lane % 16, from the (lane / 16)-th piece on
template <class T>
__device__ __forceinline__ f32x4 multiply_piece(const u32x4 &a, const u32x4 &b, f32x4 c)
{
    if constexpr (std::is_same<T, bf16>::value) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else if constexpr (std::is_same<T, f16>::value) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
        return c;
    }
}

// TILES: 16-row tiles of x; PAIRS: a gated layer
template <class T, int WAVES, int TILES, bool PAIRS>
__global__ __launch_bounds__(WAVES * 64) void fb_few_rows_kernel(Product q)
{
    constexpr int VE = Vec<T>::kN, kStep = 4 * VE, kAhead = TILES == 1 ? 8 : TILES == 2 ? 4 : 2;
    __shared__ f32x4 slots[WAVES][TILES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * (PAIRS ? 8 : 16);
    const int row = lane & 15, piece = lane >> 4;
    // (rows past the end are those of the last one: read, multiplied and not stored)
    int64_t of_w = n0 + (PAIRS ? row & 7 : row);
    of_w = (of_w < q.N ? of_w : q.N - 1) + (PAIRS && row >= 8 ? q.N : 0);
    const T *w = (const T *)q.B.p + of_w * q.B.ld + piece * VE;
    const T *x[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) x[t] = (const T *)q.A.p + (t * 16 + row < q.M ? t * 16 + row : q.M - 1) * q.A.ld + piece * VE;
    f32x4 acc[TILES] = {};
    const int64_t whole = q.K / kStep * kStep;
    int64_t k = (int64_t)wave * kStep;
    for (; k + (int64_t)(kAhead - 1) * WAVES * kStep < whole; k += (int64_t)kAhead * WAVES * kStep) {
        u32x4 a[kAhead], b[kAhead][TILES];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            a[u] = *(const u32x4_any *)(w + k + u * WAVES * kStep);
#pragma unroll
            for (int t = 0; t < TILES; ++t) b[u][t] = *(const u32x4_any *)(x[t] + k + u * WAVES * kStep);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int t = 0; t < TILES; ++t) acc[t] = multiply_piece<T>(a[u], b[u][t], acc[t]);
    }
    for (; k < q.K; k += WAVES * kStep) {
        const int n = (int)(q.K - k - piece * VE < VE ? q.K - k - piece * VE : VE);
        const u32x4 a = load_piece(w + k, n);
#pragma unroll
        for (int t = 0; t < TILES; ++t) acc[t] = multiply_piece<T>(a, load_piece(x[t] + k, n), acc[t]);
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) slots[wave][t][lane] = acc[t];
    __syncthreads();
    // sums of row m = lane % 16 of x and rows 4 (lane / 16) + 0 .. 3 of the weight, a tile a wave
    for (int t = wave; t < TILES; t += WAVES) {
        f32x4 s = slots[0][t][lane];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) s += slots[v][t][lane];
        const int64_t i = t * 16 + row;
        if constexpr (PAIRS) {
            if (lane >= 32) continue;
            f32x4 u = slots[0][t][lane + 32];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) u += slots[v][t][lane + 32];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t j = n0 + 4 * piece + e;
                if (i < q.M && j < q.N) finish_pair<T>(q.f, q.N, i, j, s[e], u[e]);
            }
            continue;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t j = n0 + 4 * piece + e;
            if (i < q.M && j < q.N) finish_one<T>(q.f, i, j, s[e]);
        }
    }
}

template <class T, int WAVES, bool PAIRS>
int launch_few(const Product &q, hipStream_t stream)
{
    constexpr int kRows = PAIRS ? 8 : 16;
    const dim3 grid((unsigned)((q.N + kRows - 1) / kRows)), block(WAVES * 64);
    if (q.M <= 16)
        hipLaunchKernelGGL((fb_few_rows_kernel<T, WAVES, 1, PAIRS>), grid, block, 0, stream, q);
    else if (q.M <= 32)
        hipLaunchKernelGGL((fb_few_rows_kernel<T, WAVES, 2, PAIRS>), grid, block, 0, stream, q);
    else
        hipLaunchKernelGGL((fb_few_rows_kernel<T, WAVES, 4, PAIRS>), grid, block, 0, stream, q);
    return launched("few-row product kernel launch: ");
}

template <class T, bool PAIRS>
int launch_few(const Product &q, hipStream_t stream)
{
    // steps of 64 bytes a row: with four waves up to 8 a wave are asked for at once; longer rows take eight waves
    return q.K * (int64_t)sizeof(T) <= 2048 ? launch_few<T, 4, PAIRS>(q, stream) : launch_few<T, 8, PAIRS>(q, stream);
}

template <bool PAIRS>
int launch_few(const Product &q, hipStream_t stream)
{
    if (q.type == FB_TYPE_F32) return launch_few<float, PAIRS>(q, stream);
    return q.type == FB_TYPE_BF16 ? launch_few<bf16, PAIRS>(q, stream) : launch_few<f16, PAIRS>(q, stream);
}

}  // namespace

int launch_few_rows(const Product &q, hipStream_t stream) { return launch_few<false>(q, stream); }
int launch_few_pairs(const Product &q, hipStream_t stream) { return launch_few<true>(q, stream); }

}  // namespace fb
