// Log probabilities and entropy straight from hidden frames, and their gradient (fb_layers.h): fb_token_logprobs of x W^T + bias,
// without the logits in memory.
//
// Forward, the product's sums never leave the registers as such: a tile leaves for each of its rows the maximum m, S = sum e^(z - m) and
// T = sum e^(z - m) (z - m), and a second launch joins the tiles of a row.  Backward, logits are formed once more, piece by piece of
// the vocabulary, and leave as their gradient in the factors' type; two products take that into dx and dweight.
//
// Bound by the matrix units.  Measured, bfloat16: 4095 x 128000 x 2048 forward 1864 us (1152 TFLOP/s; without the way out 1760), backward
// 5620 (under the profiler two pieces of 1015 for the logits, 852 for dx, 888 for dweight, 35 to join: 1146 TFLOP/s); 69120 x 3000 x 1024 backward 1258
// (logits 458, dx 403, dweight 364, rows and the largest gradient 10).
#include "fb_mfma.h"

namespace fb {

namespace {

constexpr float kInf = __builtin_huge_valf(), kLn2 = 0.69314718055994530942f;
constexpr float kOut = -1e38f;        // logits below are ruled out, as -inf is
constexpr float kFarOut = -1e4f;      // e^this is 0, and this times a finite number is finite

// S and T of one number more, or of another part: exponents are to base 2, m is as the logits are.
struct Part {
    float m, S, T;
};

__device__ __forceinline__ Part join(const Part &a, const Part &b)
{
    const float m = fmaxf(a.m, b.m);
    // (nothing: S = 0.  NaN in S or T stays: S is not 0 then)
    const float da = a.S == 0.0f ? 0.0f : (a.m - m) * kLog2E, db = b.S == 0.0f ? 0.0f : (b.m - m) * kLog2E;
    const float ea = __builtin_amdgcn_exp2f(da), eb = __builtin_amdgcn_exp2f(db);
    // (a part far below the other: 0 times a finite number)
    return Part{m, a.S * ea + b.S * eb, fmaf(a.S, fmaxf(da, kFarOut), a.T) * ea + fmaf(b.S, fmaxf(db, kFarOut), b.T) * eb};
}

__device__ __forceinline__ float other_half_max(float v)
{
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float other_half_sum(float v)
{
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The columns' operand of add_rank_one, asked for when a tile begins: the bias, -inf past the last column.
template <int FJ>
__device__ __forceinline__ void ask_columns(const Product &q, int64_t j0, int lane, f32x4 &of_columns)
{
#pragma unroll
    for (int y = 0; y < FJ; ++y) {
        const int64_t j = j0 + y * 32 + lane;
        of_columns[y] = lane >= 32 ? 1.0f : j >= q.N ? -kInf : q.f.bias ? q.f.bias[j] : 0.0f;
    }
}

// The bias of a lane's four columns, -inf past the last.
__device__ __forceinline__ void bias_or_out(const Product &q, int64_t j, f32x4 &four)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) four[e] = j + e < q.N ? (q.f.bias ? q.f.bias[j + e] : 0.0f) : -kInf;
}

// Which of a lane's FJ * 16 sums of a row is its token's (y 16 + k for acc[x][y][k]), -1 if it has none of them.  Few have: asked for
// once a fragment, by a ballot.
template <int FJ>
__device__ __forceinline__ int place_of(int token, int64_t j0, int lane)
{
    const int64_t far = (int64_t)token - j0;
    const int c = far >= 0 && far < FJ * 32 ? (int)far : -1;
    return c >= 0 && (c >> 2 & 1) == lane >> 5 ? (c >> 5) * 16 + (c >> 3 & 3) * 4 + (c & 3) : -1;
}

// Sums leave as each row's (m, S, T) over the tile's columns, and as the logits of given tokens.
struct Reduced {
    static constexpr bool kPaired = false, kNeverEmpty = true, kFolded = true;
    static constexpr int kEarly = 2;         // bias; tokens of the lane's rows

    template <int FI, int FJ>
    static __device__ __forceinline__ void early(const Product &q, const Where &where, int lane, f32x4 (&four)[2])
    {
        ask_columns<FJ>(q, where.j0 + where.wj * FJ * 32, lane, four[0]);
        const int64_t i = where.i0 + where.wi * FI * 32 + (lane & 31);
#pragma unroll
        for (int x = 0; x < FI; ++x) four[1][x] = __int_as_float(q.s.tokens[i + x * 32 < q.M ? i + x * 32 : q.M - 1]);
    }

    template <class T, int FI, int FJ>
    static __device__ __forceinline__ void leave(ProductArgs args, f32x16 (&acc)[FI][FJ], const f32x4 (&four)[2], float, const Where &where)
    {
        int lane = threadIdx.x & 63;
        asm volatile("" : "+s"(args), "+v"(lane));
        const int waves = blockDim.x / 64, across = FI == 4 ? 4 : 2, rows = waves / across * FI * 32;     // of the tile
        float *parts = where.room;
        const float upper = lane < 32 ? 0.0f : 1.0f;
        const f32x4 none = {upper, upper, upper, upper};
        const int64_t j0 = where.j0 + where.wj * FJ * 32;
#pragma unroll
        for (int x = 0; x < FI; ++x) {
            const int row = (where.wi * FI + x) * 32 + (lane & 31);
            add_rank_one<FJ>(acc[x], four[0], 0.0f, lane);
            const int place = where.i0 + row < args->M ? place_of<FJ>(__float_as_int(four[1][x]), j0, lane) : -1;
            if (__builtin_amdgcn_ballot_w64(place >= 0)) {
                float given = 0.0f;
#pragma unroll
                for (int k = 0; k < FJ * 16; ++k) given = place == k ? acc[x][k / 16][k % 16] : given;
                if (place >= 0) args->s.given[where.i0 + row] = given;
            }
            float m = acc[x][0][0];
#pragma unroll
            for (int y = 0; y < FJ; ++y)
#pragma unroll
                for (int k = 0; k < 16; ++k) m = fmaxf(m, acc[x][y][k]);
            m = other_half_max(m);
            add_rank_one<FJ>(acc[x], none, m < kOut ? 0.0f : -m, lane);      // (the difference first: a product with m has its rounding)
            float S = 0.0f, U = 0.0f;
#pragma unroll
            for (int y = 0; y < FJ; ++y)
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const float d = acc[x][y][k] * kLog2E, e = __builtin_amdgcn_exp2f(d);
                    S += e;
                    U = fmaf(e, fmaxf(d, kFarOut), U);
                }
            S = other_half_sum(S);
            U = other_half_sum(U);
            if (lane < 32) {
                float *p = parts + where.wj * 3 * rows + row;
                p[0] = m;
                p[rows] = S;
                p[2 * rows] = U;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // (the next tile's parts come behind further barriers)
        const int64_t i = where.i0 + threadIdx.x;
        if ((int)threadIdx.x < rows && i < args->M) {
            Part p{-kInf, 0.0f, 0.0f};
            for (int w = 0; w < across; ++w) {
                const float *o = parts + w * 3 * rows + threadIdx.x;
                p = join(p, Part{o[0], o[rows], o[2 * rows]});
            }
            float *out = args->s.stats + (size_t)(where.j0 / (across * FJ * 32)) * 3 * (size_t)args->M + i;
            out[0] = p.m;
            out[args->M] = p.S;
            out[2 * args->M] = p.T;
        }
    }
};

// Sums leave as the logits' gradient, rounded to the factors' type, and as shares of its column sums before that.  Of a row there
// are (-log Z, a, h, g):  dz = g [j = token] + p (a + h log2 p),  with a = -(g + h' entropy) and h = -h' ln 2 for the entropy's gradient h'.  Rows
// that do not count have log Z = inf and zeros.  A fragment's rows pass through LDS, in the factors' type, so that whole runs of a row
// are stored; rows of dz are whole 16-byte pieces.  There are whole 256 rows and tokens (those past M do not count): they are asked for when
// a tile begins, all at once: asked for at its end, with a condition each, each was waited for, and 69120 x 3000 x 1024 took 502 instead of 458 us.
struct Slopes {
    static constexpr bool kPaired = false, kNeverEmpty = true, kFolded = true;
    static constexpr int kEarly = 6;         // columns; rows, four at most; tokens of the lane's rows

    template <int FI, int FJ>
    static __device__ __forceinline__ void early(const Product &q, const Where &where, int lane, f32x4 (&four)[6])
    {
        const int64_t i = where.i0 + where.wi * FI * 32 + (lane & 31);
#pragma unroll
        for (int x = 0; x < FI; ++x) {
            four[1 + x] = ((const f32x4 *)q.s.rows)[i + x * 32];
            four[5][x] = __int_as_float(q.s.tokens[i + x * 32]);
        }
        ask_columns<FJ>(q, where.j0 + where.wj * FJ * 32, lane, four[0]);
    }

    template <class T, int FI, int FJ>
    static __device__ __forceinline__ void leave(ProductArgs args, f32x16 (&acc)[FI][FJ], const f32x4 (&four)[6], float undo, const Where &where)
    {
        int lane = threadIdx.x & 63;
        asm volatile("" : "+s"(args), "+v"(lane));
        const int64_t M = args->M, i0 = where.i0 + where.wi * FI * 32, j0 = where.j0 + where.wj * FJ * 32;
        const int64_t first = j0 + args->s.first, wide = (args->N + Vec<T>::kN - 1) / Vec<T>::kN * Vec<T>::kN;
        f32x16 sum[FJ] = {};
#pragma unroll
        for (int x = 0; x < FI; ++x) add_rank_one<FJ>(acc[x], four[0], four[1 + x][0], lane);
#pragma unroll
        for (int x = 0; x < FI; ++x) {
            f32x16(&v)[FJ] = acc[x];
            const f32x4 of_row = four[1 + x];
#pragma unroll
            for (int y = 0; y < FJ; ++y)
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const float d = fmaxf(v[y][k] * kLog2E, kFarOut);
                    v[y][k] = __builtin_amdgcn_exp2f(d) * fmaf(of_row[2], d, of_row[1]);
                }
            const int place = place_of<FJ>(__float_as_int(four[5][x]), first, lane);
            if (__builtin_amdgcn_ballot_w64(place >= 0)) {
#pragma unroll
                for (int k = 0; k < FJ * 16; ++k) v[k / 16][k % 16] += place == k ? of_row[3] : 0.0f;
            }
#pragma unroll
            for (int y = 0; y < FJ; ++y) sum[y] += v[y];
            store_fragments<T, FJ, true>(v, where.room + where.wave * 16 * FJ * 32, (T *)args->f.y, args->f.ldy, i0 + x * 32, j0, M, wide, lane,
                                         false);
            if constexpr (FI <= 2 && sizeof(T) == 2) {
                if (args->s.low) {
#pragma unroll
                    for (int y = 0; y < FJ; ++y)
#pragma unroll
                        for (int k = 0; k < 16; ++k) v[y][k] = lacks(v[y][k], (float)(T)v[y][k]);
                    store_fragments<T, FJ, true>(v, where.room + where.wave * 16 * FJ * 32, (T *)args->f.y + args->s.low * args->f.ldy, args->f.ldy,
                                                 i0 + x * 32, j0, M, wide, lane, false);
                }
            }
        }
        if (!args->s.sums) return;
        // 32 rows of a column added: two of a lane's columns at a time over the rows of 16 lanes, so that lanes 16 .. 31 and 48 .. 63 have
        // the second fragment's.
        f32x4 total[4];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const auto two = __builtin_amdgcn_permlane16_swap(__float_as_uint(sum[0][k]), __float_as_uint(sum[FJ - 1][k]), false, false);
            total[k / 4][k % 4] = sum_row16(__uint_as_float(two[0]) + __uint_as_float(two[1])) * undo;
        }
        const int64_t N = args->N, j = j0 + (FJ == 2 ? (lane >> 4 & 1) * 32 : 0) + (lane >> 5) * 4;
        float *out = args->s.sums + (size_t)(i0 / (FI * 32)) * (size_t)N + j;
        if ((lane & (FJ == 2 ? 15 : 31)) == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (j + 8 * e + 3 < N) {
                    *(f32x4_any *)(out + 8 * e) = total[e];
                } else {
#pragma unroll
                    for (int r = 0; r < 3; ++r)
                        if (j + 8 * e + r < N) out[8 * e + r] = total[e][r];
                }
            }
        }
    }
};

// Tiles of the logits' product: of 128 or 64 where a wave needs registers for a second set of sums (single precision; 256 would be 4 % faster) or
// leaves what dz lacks.
void plan_logits(Product &q, bool two = false)
{
    if (q.type != FB_TYPE_F32 && !two) {
        plan(q, 0, true);
        return;
    }
    Product small = q;
    const double cost = plan(small, 64, true);
    if (plan(q, 128, true) > cost) q = small;
}

template <class T, class WAY>
int launch_scores(const Product &q, hipStream_t stream)
{
    if constexpr (sizeof(T) == 2) {
        if (q.tile == 256) return launch<T, true, true, 2, 4, 4, 2, WAY>(q, stream);
    }
    return q.tile == 128 ? launch<T, true, true, 2, 2, 2, 2, WAY>(q, stream) : launch<T, true, true, 2, 2, 1, 1, WAY>(q, stream);
}

template <class WAY>
int launch_scores(const Product &q, hipStream_t stream)
{
    if (q.type == FB_TYPE_F32) return launch_scores<float, WAY>(q, stream);
    return q.type == FB_TYPE_BF16 ? launch_scores<bf16, WAY>(q, stream) : launch_scores<f16, WAY>(q, stream);
}

typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));

// Few rows of x: bound by reading the weight once, as fb_few_rows_kernel (262 MB in 42 us for one row of 128000 x 1024 in bfloat16, 6.2 TB/s,
// some of it from the last cache; 53 us a call on other inputs each time).  A workgroup takes 16 rows of the weight after the other, its
// waves share k and add their sums in their order; a lane keeps (m, S, T) of its row over the columns it has seen.
template <class T>
__device__ __forceinline__ f32x4 multiply_few(const u32x4 &a, const u32x4 &b, f32x4 c)
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

template <class T, int WAVES, int TILES>
__global__ __launch_bounds__(WAVES * 64) void fb_few_scores_kernel(Product q)
{
    constexpr int VE = Vec<T>::kN, kStep = 4 * VE, kAhead = TILES == 1 ? 8 : TILES == 2 ? 4 : 2;
    __shared__ f32x4 slots[2][WAVES][TILES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, piece = lane >> 4;
    // (rows past the end are those of the last one: read, multiplied and not counted)
    const T *x[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) x[t] = (const T *)q.A.p + (t * 16 + row < q.M ? t * 16 + row : q.M - 1) * q.A.ld + piece * VE;
    const int64_t whole = q.K / kStep * kStep, tiles = (q.N + 15) / 16, i = wave * 16 + row;
    const int token = wave < TILES && i < q.M ? q.s.tokens[i] : -1;
    Part part{-kInf, 0.0f, 0.0f};
    int turn = 0;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x, turn ^= 1) {
        const int64_t n0 = tile * 16;
        const T *w = (const T *)q.B.p + (n0 + row < q.N ? n0 + row : q.N - 1) * q.B.ld + piece * VE;
        f32x4 acc[TILES] = {};
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
                for (int t = 0; t < TILES; ++t) acc[t] = multiply_few<T>(a[u], b[u][t], acc[t]);
        }
        for (; k < q.K; k += WAVES * kStep) {
            const int n = (int)(q.K - k - piece * VE < VE ? q.K - k - piece * VE : VE);
            const u32x4 a = load_piece(w + k, n);
#pragma unroll
            for (int t = 0; t < TILES; ++t) acc[t] = multiply_few<T>(a, load_piece(x[t] + k, n), acc[t]);
        }
        f32x4 bias;
        bias_or_out(q, n0 + 4 * piece, bias);
#pragma unroll
        for (int t = 0; t < TILES; ++t) slots[turn][wave][t][lane] = acc[t];
        __syncthreads();
        if (wave < TILES) {                    // row `row` of the wave's 16, columns n0 + 4 piece + 0 .. 3
            f32x4 z = slots[turn][0][wave][lane];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) z += slots[turn][v][wave][lane];
            z += bias;
            Part here;
            here.m = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
            const float from = here.m < kOut ? 0.0f : here.m;
            here.S = here.T = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float d = (z[e] - from) * kLog2E, p = __builtin_amdgcn_exp2f(d);
                here.S += p;
                here.T = fmaf(p, fmaxf(d, kFarOut), here.T);
                if (token >= 0 && n0 + 4 * piece + e == token && token < q.N) q.s.given[i] = z[e];
            }
            part = join(part, here);
        }
    }
    if (wave >= TILES) return;
#pragma unroll
    for (int step = 16; step < 64; step *= 2) {
        const Part o{__shfl_xor(part.m, step), __shfl_xor(part.S, step), __shfl_xor(part.T, step)};
        part = lane & step ? join(o, part) : join(part, o);      // (one order in both)
    }
    if (lane < 16 && i < q.M) {
        float *out = q.s.stats + (size_t)blockIdx.x * 3 * (size_t)q.M + i;
        out[0] = part.m;
        out[q.M] = part.S;
        out[2 * q.M] = part.T;
    }
}

int few_groups(int64_t V) { return (int)std::min<int64_t>((V + 15) / 16, 8 * kCUs); }

template <class T, int WAVES>
int launch_few_scores(const Product &q, hipStream_t stream)
{
    const dim3 grid((unsigned)few_groups(q.N)), block(WAVES * 64);
    if (q.M <= 16)
        hipLaunchKernelGGL((fb_few_scores_kernel<T, WAVES, 1>), grid, block, 0, stream, q);
    else if (q.M <= 32)
        hipLaunchKernelGGL((fb_few_scores_kernel<T, WAVES, 2>), grid, block, 0, stream, q);
    else
        hipLaunchKernelGGL((fb_few_scores_kernel<T, WAVES, 4>), grid, block, 0, stream, q);
    return launched("few-row scores kernel launch: ");
}

template <class T>
int launch_few_scores(const Product &q, hipStream_t stream)
{
    return q.K * (int64_t)sizeof(T) <= 2048 ? launch_few_scores<T, 4>(q, stream) : launch_few_scores<T, 8>(q, stream);
}

struct EndParams {
    const float *stats;      // [parts][3][M]
    int64_t parts, M, V;
    const float *given;
    const int32_t *tokens;
    float *logprobs, *entropy, *logz;
};

// The parts of a row joined in a fixed order: COLS rows a workgroup, kPer threads a row with every kPer-th part each, four of them asked for
// at a time.  Bound by latency: a row of 2048 parts takes 4.8 us with 1024 threads, 13 with 64 that ask for one at a time.
template <int COLS>
__global__ __launch_bounds__(1024) void fb_scores_end_kernel(EndParams p)
{
    constexpr int kPer = 1024 / COLS, kAhead = 4;
    __shared__ Part slots[kPer][COLS + 1];
    const int col = threadIdx.x % COLS, g = threadIdx.x / COLS;
    const int64_t i = (int64_t)blockIdx.x * COLS + col;
    Part part{-kInf, 0.0f, 0.0f};
    int token = -1;
    float given = 0.0f;
    if (i < p.M) {
        if (g == 0) {
            token = p.tokens[i];
            if (token >= 0 && token < p.V) given = p.given[i];
        }
        for (int64_t k = g; k < p.parts; k += kAhead * kPer) {
            Part next[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const float *s = p.stats + (size_t)(k + u * kPer) * 3 * (size_t)p.M + i;
                next[u] = Part{-kInf, 0.0f, 0.0f};
                if (k + u * kPer < p.parts) next[u] = Part{s[0], s[p.M], s[2 * p.M]};
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) part = join(part, next[u]);
        }
    }
    slots[g][col] = part;
    __syncthreads();
    for (int n = kPer / 2; n > 0; n /= 2) {
        if (g < n) slots[g][col] = join(slots[g][col], slots[g + n][col]);
        __syncthreads();
    }
    if (g > 0 || i >= p.M) return;
    part = slots[0][col];
    float logz = 0.0f, entropy = 0.0f, logprob = 0.0f;
    if (token >= 0) {
        const float log_s = logf(part.S);
        logz = part.S == 0.0f ? -kInf : part.m + log_s;
        entropy = part.S == 0.0f ? 0.0f : log_s - part.T * kLn2 / part.S;
        logprob = token >= p.V ? __builtin_nanf("") : part.S == 0.0f ? -kInf : given - logz;
    }
    if (p.logz) p.logz[i] = logz;
    if (p.entropy) p.entropy[i] = entropy;
    if (p.logprobs) p.logprobs[i] = logprob;
}

int launch_end(const EndParams &p, hipStream_t stream)
{
    const auto grid = [&](int64_t rows) { return dim3((unsigned)((p.M + rows - 1) / rows)); };
    // (as many threads a row as have parts to ask for, as long as the workgroups fill the GPU)
    if (p.M <= 4 * kCUs && p.parts > 64)
        hipLaunchKernelGGL(fb_scores_end_kernel<1>, grid(1), dim3(1024), 0, stream, p);
    else if (p.parts > 64)
        hipLaunchKernelGGL(fb_scores_end_kernel<16>, grid(16), dim3(1024), 0, stream, p);
    else
        hipLaunchKernelGGL(fb_scores_end_kernel<64>, grid(64), dim3(1024), 0, stream, p);
    return launched("scores end kernel launch: ");
}

// What the gradient takes of a row, times the factor that dz is rounded with (see scale_of).
struct RowParams {
    const int32_t *tokens;
    const float *logz, *entropy, *g, *h;
    int64_t M;
    f32x4 *rows;
    uint32_t *peaks;         // shares of the largest finite bound of |dz| and, kPeakGroups further, of the largest finite |g|; nullable
    int n_peaks;
    float *undo;             // the factor's inverse, out; nullable (1)
    uint64_t *live;          // see Scores
    int32_t *picks;          // [whole 256 rows], as rows are: the tokens, -1 where a row does not count
    int low;                 // M where rows of x are there twice, see twice(); or 0
};

// What is known of a row (asked for whether it counts or not: all at once).
struct Row {
    int32_t token;
    float logz, g, h, entropy;
};

__device__ __forceinline__ Row ask_row(const RowParams &p, int64_t i)
{
    return Row{p.tokens[i], p.logz[i], p.g ? p.g[i] : 0.0f, p.h ? p.h[i] : 0.0f, p.h ? p.entropy[i] : 0.0f};
}

__device__ __forceinline__ f32x4 row_of(const RowParams &p, const Row &r)
{
    if (r.token < 0 || r.logz == -kInf) return f32x4{kInf, 0.0f, 0.0f, 0.0f};
    return f32x4{r.logz, r.logz != r.logz ? r.logz : p.h ? fmaf(r.h, r.entropy, r.g) : r.g, r.h, r.g};
}

// What no |dz| of the row exceeds, if it is finite, as a whole number that is larger where it is.
__device__ __forceinline__ uint32_t bound_of(const RowParams &p, const Row &row, const f32x4 &r)
{
    if (r[0] == kInf) return 0u;
    const uint32_t a = __float_as_uint(fabsf(r[3]) + (p.h ? fabsf(r[2]) * (0.37f + fabsf(row.entropy)) : 0.0f)) & 0x7fffffffu;
    return a < 0x7f800000u ? a : 0u;
}

// The largest bound and |g| of rows that count.
struct Peaks {
    uint32_t bound, g;
};

// Those of every `step`-th row from `from` on.
__device__ __forceinline__ Peaks peaks_of(const RowParams &p, int64_t from, int64_t step, uint32_t (&slots)[2][4])
{
    constexpr int kAhead = 8;
    Peaks peak{0, 0};
    for (int64_t i = from; i < p.M; i += kAhead * step) {
        Row row[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) row[u] = ask_row(p, i + u * step < p.M ? i + u * step : p.M - 1);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const f32x4 r = row_of(p, row[u]);
            const uint32_t a = bound_of(p, row[u], r);
            uint32_t b = __float_as_uint(r[3]) & 0x7fffffffu;
            b = b < 0x7f800000u ? b : 0u;
            peak.bound = a > peak.bound ? a : peak.bound;
            peak.g = b > peak.g ? b : peak.g;
        }
    }
    peak.bound = max_wave_u(peak.bound);
    peak.g = max_wave_u(peak.g);
    if ((threadIdx.x & 63) == 0) {
        slots[0][threadIdx.x >> 6] = peak.bound;
        slots[1][threadIdx.x >> 6] = peak.g;
    }
    __syncthreads();
    for (int w = 0; w < 4; ++w) {
        peak.bound = slots[0][w] > peak.bound ? slots[0][w] : peak.bound;
        peak.g = slots[1][w] > peak.g ? slots[1][w] : peak.g;
    }
    return peak;
}

__global__ __launch_bounds__(256) void fb_scores_peak_kernel(RowParams p)
{
    __shared__ uint32_t slots[2][4];
    const Peaks peak = peaks_of(p, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256, slots);
    if (threadIdx.x == 0) {
        p.peaks[blockIdx.x] = peak.bound;
        p.peaks[kPeakGroups + blockIdx.x] = peak.g;
    }
}

// The factor that dz is rounded with, and its inverse.  A row's largest entry is mostly its token's, g (1 - p) with a small p, and where g is one number in
// all rows, or few rows count, the rounding of that entry would be in every gradient (300 rows, g = -1 / 300, V 128000, in bfloat16: dx and dweight 2.6e-3
// off in the 2-norm, their own rounding is 1.7e-3).  Taken times 1 / m, where m is the mantissa of the largest |g|, 1 <= m < 2, such a g is a power of two
// and 1 - p rounds to 1; smaller ones lie in the halves of two powers of two where a step is less of the number.  In half precision times a power
// of two too, for the bound's sake.  Where dz is two numbers there is nothing to gain: m = 1.
template <class T>
__device__ __forceinline__ void scale_of(const Peaks &peak, bool twice, float &scale, float &undo)
{
    const float m = twice || peak.g < 0x00800000u ? 1.0f : __uint_as_float((peak.g & 0x007fffffu) | 0x3f800000u), part = 1.0f / m;
    scale = undo = 1.0f;
    if constexpr (std::is_same<T, f16>::value) range_of_peak(__float_as_uint(__uint_as_float(peak.bound) * part), scale, undo);
    scale *= part;
    undo *= m;
}

// Rows the way the gradient takes them, 256 a workgroup; in 16 bits few of them (kPeakAlone) are looked through for the largest bound and |g| by
// every workgroup.  Workgroups behind those copy what the products cannot take as it is.
template <class T>
__global__ __launch_bounds__(256) void fb_scores_rows_kernel(RowParams p, PrepareParams copies)
{
    __shared__ float slots[256][Vec<T>::kN + 1];
    const int blocks = (int)((p.M + 255) / 256);
    if ((int)blockIdx.x >= blocks) {
        copy_block<T>(copies, blockIdx.x - blocks, slots);
        return;
    }
    float scale = 1.0f;
    if (sizeof(T) == 2 && p.undo) {
        Peaks peak;
        if (p.peaks) {
            peak = Peaks{largest_of(p.peaks, p.n_peaks), largest_of(p.peaks + kPeakGroups, p.n_peaks)};
        } else {
            __shared__ uint32_t of_waves[2][4];
            peak = peaks_of(p, threadIdx.x, 256, of_waves);
        }
        float undo;
        scale_of<T>(peak, p.low != 0, scale, undo);
        if (blockIdx.x == 0 && threadIdx.x == 0) *p.undo = undo;
    }
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    Row row{-1, 0.0f, 0.0f, 0.0f, 0.0f};
    f32x4 r = {kInf, 0.0f, 0.0f, 0.0f};
    if (i < p.M) {
        row = ask_row(p, i);
        r = row_of(p, row);
    }
    const uint64_t live = __builtin_amdgcn_ballot_w64(r[0] != kInf);
    if (p.low) {                           // (up to 128 rows, in one workgroup: once more behind the last of them)
        __shared__ uint64_t once[4];
        if ((threadIdx.x & 63) == 0) once[threadIdx.x >> 6] = live;
        __syncthreads();
        if (threadIdx.x < 4) {
            const int back = p.low / 64, up = p.low % 64, w = (int)threadIdx.x - back;
            uint64_t word = once[threadIdx.x];
            if (w >= 0) word |= once[w] << up;
            if (w >= 1 && up) word |= once[w - 1] >> (64 - up);
            p.live[threadIdx.x] = word;
        }
    } else if ((threadIdx.x & 63) == 0) {
        p.live[i / 64] = live;
    }
    p.picks[i] = r[0] != kInf ? row.token : -1;
    r[0] = -r[0];
    r[1] *= -scale;
    r[2] *= -scale * kLn2;
    r[3] *= scale;
    p.rows[i] = r;
}

// (a launch less: 4095 rows, V 300, K 256 in bfloat16 28 instead of 30 us a call, 8000 rows 36 either way, 12000 43 and 40.5)
constexpr int64_t kPeakAlone = 8192;

int launch_rows(RowParams r, int type, const Prepare &copies, hipStream_t stream)
{
    const unsigned blocks = (unsigned)((r.M + 255) / 256);
    if (r.undo && r.M > kPeakAlone) {
        r.n_peaks = (int)std::min<int64_t>(kPeakGroups, blocks);
        hipLaunchKernelGGL(fb_scores_peak_kernel, dim3((unsigned)r.n_peaks), dim3(256), 0, stream, r);
        const int rc = launched("scores peak kernel launch: ");
        if (rc != FB_OK) return rc;
    } else {
        r.peaks = nullptr;
    }
    const dim3 grid(blocks + (unsigned)copies.blocks), block(256);
    if (type == FB_TYPE_F32)
        hipLaunchKernelGGL(fb_scores_rows_kernel<float>, grid, block, 0, stream, r, copies.p);
    else if (type == FB_TYPE_BF16)
        hipLaunchKernelGGL(fb_scores_rows_kernel<bf16>, grid, block, 0, stream, r, copies.p);
    else
        hipLaunchKernelGGL(fb_scores_rows_kernel<f16>, grid, block, 0, stream, r, copies.p);
    return launched("scores rows kernel launch: ");
}

// The sum over pieces of the vocabulary, rounded to dx.
struct RoundParams {
    const float *sums;       // [M][K]
    int64_t M, K, ld;
    void *out;
};

template <class T>
__global__ __launch_bounds__(256) void fb_scores_round_kernel(RoundParams p)
{
    constexpr int VE = Vec<T>::kN;
    const int64_t pieces = (p.K + VE - 1) / VE, n = p.M * pieces;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < n; at += (int64_t)gridDim.x * 256) {
        const int64_t r = at / pieces, c = (at - r * pieces) * VE;
        const int here = (int)(p.K - c < VE ? p.K - c : VE);
        float v[VE];
#pragma unroll
        for (int e = 0; e < VE; e += 4) unpack<float>(load_piece(p.sums + r * p.K + c + e, here - e), v + e);
        store_piece((T *)p.out + r * p.ld + c, here, pack<T>(v));
    }
}

int launch_round(const RoundParams &p, int type, hipStream_t stream)
{
    const int64_t ve = 16 / (int64_t)type_bytes(type);
    const dim3 grid((unsigned)std::min<int64_t>((p.M * ((p.K + ve - 1) / ve) + 255) / 256, 8 * kCUs)), block(256);
    if (type == FB_TYPE_F32)
        hipLaunchKernelGGL(fb_scores_round_kernel<float>, grid, block, 0, stream, p);
    else if (type == FB_TYPE_BF16)
        hipLaunchKernelGGL(fb_scores_round_kernel<bf16>, grid, block, 0, stream, p);
    else
        hipLaunchKernelGGL(fb_scores_round_kernel<f16>, grid, block, 0, stream, p);
    return launched("scores rounding kernel launch: ");
}

struct ScorePlan {
    Product q;
    bool few;
    Packed x, w;
    int64_t parts;
    size_t given, stats, bytes;
};

ScorePlan score_plan(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t V, int64_t K, int type)
{
    ScorePlan f{};
    f.q.M = M; f.q.N = V; f.q.K = K; f.q.type = type;
    f.few = M <= kFewRows;
    if (f.few) {
        f.parts = few_groups(V);
    } else {
        plan_logits(f.q);
        f.parts = (V + f.q.tile - 1) / f.q.tile;
        f.x = packed(x, ldx, M, K, type);
        f.w = packed(weight, ldw, V, K, type);
    }
    f.given = aligned((size_t)M * sizeof(float));
    f.stats = aligned((size_t)f.parts * 3 * (size_t)M * sizeof(float));
    f.bytes = f.x.bytes + f.w.bytes + f.given + f.stats + 256;
    return f;
}

// Alternatives of a piece of the vocabulary: the logits' gradient of a piece takes up to 512 MB (one piece for 69120 rows of 3000 in 16
// bits, two of 64000 for 4095 rows) in rows of less than 4 MB, and pieces are alike.
constexpr int64_t kPieceBytes = (int64_t)512 << 20;

}  // namespace

ScoreGradPlan score_grad_plan(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t V, int64_t K, int type)
{
    ScoreGradPlan g{};
    const int64_t size = (int64_t)type_bytes(type), longest = ((int64_t)1 << 22) / size - 256;
    const int64_t most = std::max<int64_t>(256, std::min(longest, kPieceBytes / std::max<int64_t>(1, M * size) / 256 * 256));
    g.pieces = (V + most - 1) / most;
    g.width = g.pieces == 1 ? V : ((V + g.pieces - 1) / g.pieces + 255) / 256 * 256;
    g.pieces = (V + g.width - 1) / g.width;
    g.ldz = line_distance(g.width, type);
    g.z.M = M; g.z.N = g.width; g.z.K = K; g.z.type = type;
    g.dx.M = M; g.dx.N = K; g.dx.K = g.width; g.dx.type = type;
    g.dw.M = g.width; g.dw.N = K; g.dw.K = M; g.dw.type = type;
    g.twice = twice(M, V, K, type);
    if (g.twice) g.dx.M = g.dw.K = 2 * M;
    plan_logits(g.z, g.twice);
    const bool pair = plan_back(g.dx, g.dw);
    g.pair = pair && g.pieces == 1;
    if (pair && !g.pair) {
        plan(g.dx);
        plan(g.dw);
    }
    if (g.twice) g.dx.parts = true;
    const int64_t rows = g.twice ? 2 * M : M;
    g.x = packed(x, ldx, rows, K, type, g.twice);
    g.w = packed(weight, ldw, V, K, type);
    const int64_t fragment = g.z.tile == 256 ? 128 : g.z.tile / 2;        // rows of a wave
    g.sum_rows = (M + g.z.tile - 1) / g.z.tile * (g.z.tile / fragment);
    g.dz = aligned((size_t)rows * (size_t)g.ldz * type_bytes(type));
    g.rows = aligned((size_t)((M + 255) / 256 * 256) * sizeof(f32x4));
    g.picks = aligned((size_t)((M + 255) / 256 * 256) * sizeof(int32_t));
    g.live = aligned((size_t)((M + 255) / 256 * 4 + 1) * sizeof(uint64_t));
    g.range = aligned((2 * kPeakGroups + 1) * sizeof(float));
    g.sums = aligned((size_t)g.sum_rows * (size_t)g.width * sizeof(float));
    g.acc = g.pieces > 1 ? aligned((size_t)M * (size_t)K * sizeof(float)) : 0;
    g.part_x = product_bytes(g.dx);
    g.part_w = product_bytes(g.dw);
    g.bytes = g.x.bytes + g.w.bytes + g.dz + g.rows + g.picks + g.live + g.range + g.sums + g.acc + g.part_x + g.part_w;
    return g;
}

namespace {

int check_scores(const char *who, const void *x, int64_t ldx, const void *weight, int64_t ldw, const int32_t *tokens, int64_t M, int64_t V, int64_t K, int type)
{
    const std::string w(who);
    if (!known_type(type)) return fail(FB_EINVAL, w + ": unknown type");
    if (bad_sizes(M, V, K)) return fail(FB_EINVAL, w + ": M must be 0 or more and below 2^31, V and K 1 or more and below 2^28");
    if (((!x || !tokens) && M > 0) || !weight) return fail(FB_EINVAL, w + ": x, weight or tokens is NULL");
    if (bad_ld(ldx, K) || bad_ld(ldw, K)) return fail(FB_EINVAL, w + ": rows of x or weight closer than K elements");
    if (too_long(K, type)) return fail(FB_EUNSUPPORTED, w + ": rows of x and weight longer than 4 MB");
    return FB_OK;
}

}  // namespace

}  // namespace fb

extern "C" {

size_t fb_affine_logprobs_workspace_bytes(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t V, int64_t K, int type)
{
    using namespace fb;
    if (bad_sizes(M, V, K) || !known_type(type)) return 0;
    return score_plan(x, ldx, weight, ldw, M, V, K, type).bytes;
}

int fb_affine_logprobs(const void *x, int64_t ldx, const void *weight, int64_t ldw, const float *bias, const int32_t *tokens, int64_t M, int64_t V,
                       int64_t K, int type, float *logprobs, float *entropy, float *logz, void *ws, size_t ws_bytes, fb_stream stream)
{
    using namespace fb;
    return guarded([&]() -> int {
        int rc = check_scores("fb_affine_logprobs", x, ldx, weight, ldw, tokens, M, V, K, type);
        if (rc != FB_OK) return rc;
        const ScorePlan f = score_plan(x, ldx, weight, ldw, M, V, K, type);
        if (!ws || ws_bytes < f.bytes) return fail(FB_EINVAL, "fb_affine_logprobs: workspace missing or too small");
        if (M == 0) return FB_OK;
        hipStream_t st = (hipStream_t)stream;
        char *xs = (char *)ws, *wts = xs + f.x.bytes, *given = wts + f.w.bytes, *stats = given + f.given;
        Product q = f.q;
        q.f.bias = bias;
        q.s.tokens = tokens;
        q.s.given = (float *)given;
        q.s.stats = (float *)stats;
        if (f.few) {
            q.A = {x, ldx, true};
            q.B = {weight, ldw, true};
            rc = type == FB_TYPE_F32 ? launch_few_scores<float>(q, st) : type == FB_TYPE_BF16 ? launch_few_scores<bf16>(q, st) : launch_few_scores<f16>(q, st);
        } else {
            Prepare jobs;
            if (f.x.copy) jobs.add(pack_job(f.x, x, ldx, M, K, xs), type);
            if (f.w.copy) jobs.add(pack_job(f.w, weight, ldw, V, K, wts), type);
            if ((rc = launch_prepare(jobs, type, type, st)) != FB_OK) return rc;
            q.A = {f.x.copy ? xs : x, f.x.ld, true};
            q.B = {f.w.copy ? wts : weight, f.w.ld, true};
            rc = launch_scores<Reduced>(q, st);
        }
        if (rc != FB_OK) return rc;
        const EndParams e{q.s.stats, f.parts, M, V, q.s.given, tokens, logprobs, entropy, logz};
        return launch_end(e, st);
    });
}

size_t fb_affine_logprobs_grad_workspace_bytes(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t V, int64_t K, int type)
{
    using namespace fb;
    if (bad_sizes(M, V, K) || !known_type(type)) return 0;
    return score_grad_plan(x, ldx, weight, ldw, M, V, K, type).bytes;
}

int fb_affine_logprobs_grad(const void *x, int64_t ldx, const void *weight, int64_t ldw, const float *bias, const int32_t *tokens, const float *logz,
                            const float *entropy, const float *g_logprobs, const float *g_entropy, int64_t M, int64_t V, int64_t K, int type,
                            void *dx, int64_t lddx, void *dweight, float *dbias, void *ws, size_t ws_bytes, fb_stream stream)
{
    using namespace fb;
    return guarded([&]() -> int {
        int rc = check_scores("fb_affine_logprobs_grad", x, ldx, weight, ldw, tokens, M, V, K, type);
        if (rc != FB_OK) return rc;
        if (M > 0 && (!logz || (g_entropy && !entropy))) return fail(FB_EINVAL, "fb_affine_logprobs_grad: logz or entropy is NULL");
        if (dx && bad_ld(lddx, K)) return fail(FB_EINVAL, "fb_affine_logprobs_grad: rows of dx closer than K elements");
        if (dx && too_far(lddx)) return fail(FB_EUNSUPPORTED, "fb_affine_logprobs_grad: rows of dx 2^27 elements apart");
        if (!dx && !dweight && !dbias) return FB_OK;
        const ScoreGradPlan g = score_grad_plan(x, ldx, weight, ldw, M, V, K, type);
        if (!ws || ws_bytes < g.bytes) return fail(FB_EINVAL, "fb_affine_logprobs_grad: workspace missing or too small");
        hipStream_t st = (hipStream_t)stream;
        char *xs = (char *)ws, *wts = xs + g.x.bytes, *dz = wts + g.w.bytes, *rows = dz + g.dz, *picks = rows + g.rows, *live = picks + g.picks;
        char *range = live + g.live, *sums = range + g.range;
        char *acc = sums + g.sums, *part_x = acc + g.acc, *part_w = part_x + g.part_x;
        const int64_t size = (int64_t)type_bytes(type);
        float *undo = M > 0 && (type == FB_TYPE_F16 || (type == FB_TYPE_BF16 && !g.twice)) ? (float *)range : nullptr;      // (no rows: nobody sets it)
        if (M > 0) {
            RowParams r{tokens, logz, entropy, g_logprobs, g_entropy, M, (f32x4 *)rows, undo ? (uint32_t *)(undo + 1) : nullptr, 0, undo,
                        (uint64_t *)live, (int32_t *)picks, g.twice ? (int)M : 0};
            Prepare copies;
            if (g.x.copy) copies.add(pack_job(g.x, x, ldx, M, K, xs), type);
            if (g.twice) copies.add(pack_job(g.x, x, ldx, M, K, xs + (size_t)M * (size_t)g.x.ld * type_bytes(type)), type);
            if (g.w.copy) copies.add(pack_job(g.w, weight, ldw, V, K, wts), type);
            if ((rc = launch_rows(r, type, copies, st)) != FB_OK) return rc;
        }
        const char *w = g.w.copy ? wts : (const char *)weight;
        const void *rows_of_x = g.x.copy ? xs : x;
        for (int64_t v0 = 0; v0 < V; v0 += g.width) {
            const int64_t n = std::min(g.width, V - v0);
            const bool first = v0 == 0, last = v0 + n == V;
            Product z = g.z, qx = g.dx, qw = g.dw;
            z.N = n; qx.K = n; qw.M = n;
            z.A = {rows_of_x, g.x.ld, true};
            z.B = {w + v0 * g.w.ld * size, g.w.ld, true};
            z.f.bias = bias ? bias + v0 : nullptr;
            z.f.y = dz; z.f.ldy = line_distance(n, type);
            z.f.undo = undo;
            z.s = {(const int32_t *)picks, (int)v0, nullptr, nullptr, rows, dbias ? (float *)sums : nullptr, nullptr, g.twice ? M : 0};
            if (M > 0 && (rc = launch_scores<Slopes>(z, st)) != FB_OK) return rc;
            qx.A = {dz, z.f.ldy, true};
            qx.B = {z.B.p, g.w.ld, false};
            qx.split = (int)((n + qx.share - 1) / qx.share);
            qx.f.undo = undo;
            qx.part = (float *)part_x;
            if (g.pieces > 1) {                     // pieces add up in single precision
                qx.f.y = acc; qx.f.ldy = K; qx.f.out_type = FB_TYPE_F32;
                qx.f.residual = first ? nullptr : acc; qx.f.ldr = K;
            } else {
                qx.f.y = dx; qx.f.ldy = lddx; qx.f.out_type = type;
            }
            qw.A = {dz, z.f.ldy, false};
            qw.B = {rows_of_x, g.x.ld, false};
            qw.s.live = (const uint64_t *)live;
            qw.f.y = dweight ? (char *)dweight + v0 * K * size : nullptr; qw.f.ldy = K; qw.f.out_type = type;
            qw.f.undo = undo;
            qw.part = (float *)part_w;
            const bool has_dx = dx && M > 0;
            if (g.pair && has_dx && dweight) {
                if ((rc = launch_mfma_pair(qx, qw, st)) != FB_OK) return rc;
            } else {
                if (has_dx && (rc = launch_dx(qx, st)) != FB_OK) return rc;
                if (dweight && (rc = launch_mfma_product(qw, st)) != FB_OK) return rc;
            }
            const Product joined = joined_rows(qx, g.twice);
            rc = launch_join(has_dx ? &joined : nullptr, dweight ? &qw : nullptr, type, (const float *)sums, M > 0 ? g.sum_rows : 0, n, dbias ? dbias + v0 : nullptr, st);
            if (rc != FB_OK) return rc;
            if (last && has_dx && g.pieces > 1 && (rc = launch_round(RoundParams{(const float *)acc, M, K, lddx, dx}, type, st)) != FB_OK) return rc;
        }
        return FB_OK;
    });
}

}  // extern "C"
