// Layer norm and its gradient (fb_layers.h).  Both are bound by memory: a row is read once into registers, everything that
// needs it whole is formed there, and it is written once.  69120 rows of 1024 in bfloat16 take 53 us forward (5.3 TB/s of the
// bytes that have to be moved; a large copy reaches 4.8) and 81 us backward (5.3 TB/s, 5 us of them the reduction of the
// weight's gradient), 8000 rows of 4096 floats 43 and 84; single rows 3 us of latency.
#include "fb_layers_device.h"

namespace fb {

namespace {

struct NormParams {
    const void *x, *dy, *weight, *bias;
    void *y;                       // y, or dx
    int64_t ldx, lddy, ldy, R, H;
    float eps;
    float *mean, *rstd;            // out; in for the gradient
    float *part;                   // gradient: [workgroup][2][H], shares of dweight and dbias
    bool past;                     // y goes past the caches
};

// EPL elements of a vector of [H] as floats, at the places a lane has of a row; `none` where there is no vector.
template <class W, int EPL, int VE>
__device__ __forceinline__ void load_vector(const void *w, int H, int step, int lane, float none, float *v)
{
    constexpr int kN = Vec<W>::kN;
#pragma unroll
    for (int i = 0; i < EPL / VE; ++i) {
        const int at = (i * step + lane) * VE;
#pragma unroll
        for (int j = 0; j < VE; j += kN) {
            float u[kN];
            unpack<W>(w ? load_piece((const W *)w + at + j, H - at - j) : u32x4{}, u);
#pragma unroll
            for (int e = 0; e < kN; ++e) v[i * VE + j + e] = w ? u[e] : none;
        }
    }
}

// Sums of N numbers a thread over the WAVES waves of a workgroup that share a row.  `slot` alternates, so that one barrier
// a call is enough: a wave writes a slot again only behind the next barrier, which every wave reaches when it has read it.
template <int WAVES, int N>
__device__ __forceinline__ void sum_row(float (&v)[N], float (*slots)[WAVES][N], int slot)
{
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = sum_wave(v[n]);
    if constexpr (WAVES > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int n = 0; n < N; ++n) slots[slot][wave][n] = v[n];
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) s += slots[slot][w][n];
            v[n] = s;
        }
    }
}

// y = (x - mean) rstd weight + bias.  WAVES waves of 64 lanes hold a row, EPL elements a lane; with one wave a row a
// workgroup has four rows at a time.  The next row is asked for before this one is worked on.  The variance is the mean of
// the squared distances from the mean, of the values in registers: no difference of large sums.
template <class T, class W, int WAVES, int EPL>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void fb_layer_norm_kernel(NormParams p)
{
    constexpr int VE = Vec<T>::kN, NV = EPL / VE, kStep = WAVES * 64;
    __shared__ float slots[2][WAVES][1];
    const int lane = WAVES == 1 ? (threadIdx.x & 63) : threadIdx.x;
    const int H = (int)p.H;
    const int64_t r0 = WAVES == 1 ? (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : (int64_t)blockIdx.x;
    const int64_t rstep = WAVES == 1 ? (int64_t)gridDim.x * 4 : (int64_t)gridDim.x;
    float w[EPL], b[EPL];
    load_vector<W, EPL, VE>(p.weight, H, kStep, lane, 1.0f, w);
    load_vector<W, EPL, VE>(p.bias, H, kStep, lane, 0.0f, b);
    const float inv = 1.0f / (float)H;
    u32x4 raw[NV];
    auto ask = [&](int64_t r) {
        const T *x = (const T *)p.x + r * p.ldx;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (i * kStep + lane) * VE;
            raw[i] = load_piece(x + at, (int)(H - at));
        }
    };
    if (r0 < p.R) ask(r0);
    for (int64_t r = r0; r < p.R; r += rstep) {
        float v[EPL];
#pragma unroll
        for (int i = 0; i < NV; ++i) unpack<T>(raw[i], v + i * VE);
        if (r + rstep < p.R) ask(r + rstep);
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < EPL; ++i) s[0] += v[i];
        sum_row<WAVES, 1>(s, slots, 0);
        const float mean = s[0] * inv;
        float q[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (i * kStep + lane) * VE;
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const float d = at + j < H ? v[i * VE + j] - mean : 0.0f;
                v[i * VE + j] = d;
                q[0] = fmaf(d, d, q[0]);
            }
        }
        sum_row<WAVES, 1>(q, slots, 1);
        const float rstd = 1.0f / sqrtf(q[0] * inv + p.eps);
        if (lane == 0) {
            if (p.mean) p.mean[r] = mean;
            if (p.rstd) p.rstd[r] = rstd;
        }
        T *y = (T *)p.y + r * p.ldy;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (i * kStep + lane) * VE;
            float o[VE];
#pragma unroll
            for (int j = 0; j < VE; ++j) o[j] = fmaf(v[i * VE + j] * rstd, w[i * VE + j], b[i * VE + j]);
            store_piece(y + at, H - at, pack<T>(o), p.past);
        }
    }
}

// Rows too long for the registers of a workgroup: read three times, from the caches when they are not too long for those.
template <class T, class W>
__global__ __launch_bounds__(1024) void fb_layer_norm_long_kernel(NormParams p)
{
    constexpr int VE = Vec<T>::kN;
    __shared__ float slots[2][16][1];
    const int64_t H = p.H;
    for (int64_t r = blockIdx.x; r < p.R; r += gridDim.x) {
        const T *x = (const T *)p.x + r * p.ldx;
        T *y = (T *)p.y + r * p.ldy;
        float s[1] = {0.0f}, q[1] = {0.0f};
        for (int64_t at = (int64_t)threadIdx.x * VE; at < H; at += 1024 * VE) {
            float v[VE];
            unpack<T>(load_piece(x + at, (int)(H - at)), v);
#pragma unroll
            for (int j = 0; j < VE; ++j) s[0] += v[j];
        }
        sum_row<16, 1>(s, slots, 0);
        const float mean = s[0] / (float)H;
        for (int64_t at = (int64_t)threadIdx.x * VE; at < H; at += 1024 * VE) {
            float v[VE];
            unpack<T>(load_piece(x + at, (int)(H - at)), v);
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const float d = at + j < H ? v[j] - mean : 0.0f;
                q[0] = fmaf(d, d, q[0]);
            }
        }
        sum_row<16, 1>(q, slots, 1);
        const float rstd = 1.0f / sqrtf(q[0] / (float)H + p.eps);
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[r] = mean;
            if (p.rstd) p.rstd[r] = rstd;
        }
        for (int64_t at = (int64_t)threadIdx.x * VE; at < H; at += 1024 * VE) {
            float v[VE], o[VE];
            unpack<T>(load_piece(x + at, (int)(H - at)), v);
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const bool in = at + j < H;
                const float w = p.weight && in ? (float)((const W *)p.weight)[at + j] : 1.0f;
                const float b = p.bias && in ? (float)((const W *)p.bias)[at + j] : 0.0f;
                o[j] = fmaf((v[j] - mean) * rstd, w, b);
            }
            store_piece(y + at, H - at, pack<T>(o), p.past);
        }
    }
}

// dx of a row, and the row's share of dweight and dbias added to sums that the lane keeps in registers for its places of
// the row over all rows it sees; they leave the kernel once, a row of sums a workgroup, for fb_column_sum_kernel.  The next row
// is asked for before this one is worked on and the weight kept in registers, except where 16 elements a lane in 16 waves
// leave no registers for either (65 to 94 of them would go to memory).
template <class T, class W, int WAVES, int EPL>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void fb_layer_norm_grad_kernel(NormParams p)
{
    constexpr int VE = Vec<T>::kN, NV = EPL / VE, kStep = WAVES * 64;
    constexpr bool kLean = WAVES * EPL >= 256;
    __shared__ float slots[2][WAVES][2];
    __shared__ float joined[WAVES == 1 ? 4 : 1][WAVES == 1 ? EPL * 64 : 1];
    const int lane = WAVES == 1 ? (threadIdx.x & 63) : threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int H = (int)p.H;
    const int64_t r0 = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
    const int64_t rstep = WAVES == 1 ? (int64_t)gridDim.x * 4 : (int64_t)gridDim.x;
    float w[kLean ? 1 : EPL], dw[EPL], db[EPL];
    if constexpr (!kLean) load_vector<W, EPL, VE>(p.weight, H, kStep, lane, 1.0f, w);
#pragma unroll
    for (int i = 0; i < EPL; ++i) dw[i] = db[i] = 0.0f;
    const float inv = 1.0f / (float)H;
    u32x4 rx[NV], rg[NV];
    float mean = 0.0f, rstd = 0.0f;
    auto ask = [&](int64_t r) {
        const T *x = (const T *)p.x + r * p.ldx, *dy = (const T *)p.dy + r * p.lddy;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (i * kStep + lane) * VE;
            rx[i] = load_piece(x + at, (int)(H - at));
            rg[i] = load_piece(dy + at, (int)(H - at));
        }
        mean = p.mean[r];
        rstd = p.rstd[r];
    };
    if (!kLean && r0 < p.R) ask(r0);
    int slot = 0;
    for (int64_t r = r0; r < p.R; r += rstep, slot ^= 1) {
        float xh[EPL], g[EPL];
        if (kLean) ask(r);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            unpack<T>(rx[i], xh + i * VE);
            unpack<T>(rg[i], g + i * VE);
        }
        const float m = mean, s = rstd;
        if (!kLean && r + rstep < p.R) ask(r + rstep);
        float t[2] = {0.0f, 0.0f};                      // (past the row's end dy is 0, and with it every share)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float wv[VE];
            if constexpr (kLean) load_vector<W, VE, VE>(p.weight, H, 0, v * kStep + lane, 1.0f, wv);
#pragma unroll
            for (int i = v * VE; i < (v + 1) * VE; ++i) {
                xh[i] = (xh[i] - m) * s;
                dw[i] = fmaf(g[i], xh[i], dw[i]);
                db[i] += g[i];
                g[i] *= kLean ? wv[i - v * VE] : w[kLean ? 0 : i];
                t[0] += g[i];
                t[1] = fmaf(g[i], xh[i], t[1]);
            }
        }
        if (p.y) {
            sum_row<WAVES, 2>(t, slots, slot);
            const float c0 = t[0] * inv, c1 = t[1] * inv;
            T *dx = (T *)p.y + r * p.ldy;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int at = (i * kStep + lane) * VE;
                float o[VE];
#pragma unroll
                for (int j = 0; j < VE; ++j) o[j] = s * (g[i * VE + j] - c0 - xh[i * VE + j] * c1);
                store_piece(dx + at, H - at, pack<T>(o), p.past);
            }
        }
    }
    if (!p.part) return;
    float *part = p.part + (size_t)blockIdx.x * 2 * H;
    if constexpr (WAVES == 1) {
        for (int k = 0; k < 2; ++k) {                   // the four waves' sums, added in their order
            __syncthreads();
#pragma unroll
            for (int i = 0; i < EPL; ++i) joined[wave][(i / VE * 64 + lane) * VE + i % VE] = k ? db[i] : dw[i];
            __syncthreads();
            for (int c = threadIdx.x; c < H; c += 256)
                part[(size_t)k * H + c] = (joined[0][c] + joined[1][c]) + (joined[2][c] + joined[3][c]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const int c = (i / VE * kStep + lane) * VE + i % VE;
            if (c < H) {
                part[c] = dw[i];
                part[(size_t)H + c] = db[i];
            }
        }
    }
}

// Long rows, dx: the sums of a row first, then the row again.
template <class T, class W>
__global__ __launch_bounds__(1024) void fb_layer_norm_long_dx_kernel(NormParams p)
{
    constexpr int VE = Vec<T>::kN;
    __shared__ float slots[2][16][2];
    const int64_t H = p.H;
    int slot = 0;
    for (int64_t r = blockIdx.x; r < p.R; r += gridDim.x, slot ^= 1) {
        const T *x = (const T *)p.x + r * p.ldx, *dy = (const T *)p.dy + r * p.lddy;
        T *dx = (T *)p.y + r * p.ldy;
        const float m = p.mean[r], s = p.rstd[r];
        float t[2] = {0.0f, 0.0f};
        for (int64_t at = (int64_t)threadIdx.x * VE; at < H; at += 1024 * VE) {
            float v[VE], g[VE];
            unpack<T>(load_piece(x + at, (int)(H - at)), v);
            unpack<T>(load_piece(dy + at, (int)(H - at)), g);
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const float w = p.weight && at + j < H ? (float)((const W *)p.weight)[at + j] : 1.0f;
                t[0] = fmaf(g[j], w, t[0]);
                t[1] = fmaf(g[j] * w, (v[j] - m) * s, t[1]);
            }
        }
        sum_row<16, 2>(t, slots, slot);
        const float c0 = t[0] / (float)H, c1 = t[1] / (float)H;
        for (int64_t at = (int64_t)threadIdx.x * VE; at < H; at += 1024 * VE) {
            float v[VE], g[VE], o[VE];
            unpack<T>(load_piece(x + at, (int)(H - at)), v);
            unpack<T>(load_piece(dy + at, (int)(H - at)), g);
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const float w = p.weight && at + j < H ? (float)((const W *)p.weight)[at + j] : 1.0f;
                o[j] = s * (g[j] * w - c0 - (v[j] - m) * s * c1);
            }
            store_piece(dx + at, H - at, pack<T>(o), p.past);
        }
    }
}

// Long rows, shares of dweight and dbias: a workgroup has 256 pieces of the rows' width and every gridDim.y-th row.  (Launched
// before dx is written, which may be where dy or x is.)
template <class T>
__global__ __launch_bounds__(256) void fb_layer_norm_long_dw_kernel(NormParams p)
{
    constexpr int VE = Vec<T>::kN;
    const int64_t H = p.H, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * VE;
    if (at >= H) return;
    float dw[VE] = {}, db[VE] = {};
    for (int64_t r = blockIdx.y; r < p.R; r += gridDim.y) {
        float v[VE], g[VE];
        unpack<T>(load_piece((const T *)p.x + r * p.ldx + at, (int)(H - at)), v);
        unpack<T>(load_piece((const T *)p.dy + r * p.lddy + at, (int)(H - at)), g);
        const float m = p.mean[r], s = p.rstd[r];
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            dw[j] = fmaf(g[j], (v[j] - m) * s, dw[j]);
            db[j] += g[j];
        }
    }
    float *part = p.part + (size_t)blockIdx.y * 2 * H;
#pragma unroll
    for (int j = 0; j < VE; ++j) {
        if (at + j < H) {
            part[at + j] = dw[j];
            part[(size_t)H + at + j] = db[j];
        }
    }
}

// out[k][c] = sum over i < P of part[i][k][c], in a fixed order: 16 threads share a column, each adding every 16th row.
__global__ __launch_bounds__(1024) void fb_column_sum_kernel(const float *part, int64_t P, int64_t C, float *out0, float *out1)
{
    __shared__ float slots[16][64];
    const int col = threadIdx.x & 63, g = threadIdx.x >> 6;
    const int k = blockIdx.y;
    float *out = k ? out1 : out0;
    if (!out) return;
    for (int64_t c0 = (int64_t)blockIdx.x * 64; c0 < C; c0 += (int64_t)gridDim.x * 64) {
        const int64_t c = c0 + col;
        float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
        if (c < C) {
            const float *q = part + (size_t)k * C + c;
            const int64_t step = (int64_t)gridDim.y * C;
            int64_t i = g;
            for (; i + 48 < P; i += 64) {
                s0 += q[i * step];
                s1 += q[(i + 16) * step];
                s2 += q[(i + 32) * step];
                s3 += q[(i + 48) * step];
            }
            for (; i < P; i += 16) s0 += q[i * step];
        }
        slots[g][col] = (s0 + s1) + (s2 + s3);
        __syncthreads();
        if (g == 0 && c < C) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) s += slots[i][col];
            out[c] = s;
        }
        __syncthreads();
    }
}

int launch_column_sum(const float *part, int64_t P, int64_t C, float *out0, float *out1, void *stream)
{
    // (2^22 workgroups of 1024 threads, those of the widest rows, are more threads than a launch may have)
    const int64_t groups = std::min<int64_t>((C + 63) / 64, (int64_t)1 << 21);
    hipLaunchKernelGGL(fb_column_sum_kernel, dim3((unsigned)groups, 2), dim3(1024), 0, (hipStream_t)stream, part, P, C, out0, out1);
    return launched("column sum kernel launch: ");
}

constexpr int64_t kRowMax = 16384;       // longest row that a workgroup holds in registers
// Workgroups of the gradient kernel: two a compute unit, one where it has 16 waves.  (Each leaves a row of sums to be added up:
// with 768 or 1024 of them 69120 rows of 1024 take 88 and 90 us instead of 84, with 256 20000 rows of 2048 59 instead of 48.)
constexpr int64_t kGradGroups = 512;
constexpr int64_t kLongRowGroups = 128;  // workgroups that share the rows of a piece of width

int64_t grad_groups(int64_t R, int64_t H)
{
    if (H > kRowMax) return std::min<int64_t>(R, kLongRowGroups);
    return std::min<int64_t>(H <= 1024 ? (R + 3) / 4 : R, H <= 4096 ? kGradGroups : kGradGroups / 2);
}

template <class T, class W, int WAVES, int EPL>
int launch_norm(const NormParams &p, bool grad, hipStream_t stream)
{
    const int64_t groups = WAVES == 1 ? (p.R + 3) / 4 : p.R;
    const dim3 block(WAVES == 1 ? 256 : WAVES * 64);
    if (grad) {
        hipLaunchKernelGGL((fb_layer_norm_grad_kernel<T, W, WAVES, EPL>), dim3((unsigned)grad_groups(p.R, p.H)), block, 0, stream, p);
    } else {
        const int64_t most = (int64_t)kCUs * (WAVES == 16 ? 2 : 8);
        hipLaunchKernelGGL((fb_layer_norm_kernel<T, W, WAVES, EPL>), dim3((unsigned)std::min(groups, most)), block, 0, stream, p);
    }
    return launched("layer norm kernel launch: ");
}

// One wave a row up to 1024 elements (no barrier), four up to 4096, sixteen beyond: at most 16 elements a lane.
template <class T, class W>
int launch_norm(const NormParams &p, bool grad, hipStream_t stream)
{
    const int64_t H = p.H;
    if (H <= 512) return launch_norm<T, W, 1, 8>(p, grad, stream);
    if (H <= 1024) return launch_norm<T, W, 1, 16>(p, grad, stream);
    if (H <= 2048) return launch_norm<T, W, 4, 8>(p, grad, stream);
    if (H <= 4096) return launch_norm<T, W, 4, 16>(p, grad, stream);
    if (H <= 8192) return launch_norm<T, W, 16, 8>(p, grad, stream);
    if (H <= kRowMax) return launch_norm<T, W, 16, 16>(p, grad, stream);
    if (!grad) {
        hipLaunchKernelGGL((fb_layer_norm_long_kernel<T, W>), dim3((unsigned)std::min<int64_t>(p.R, 2 * kCUs)), dim3(1024), 0, stream, p);
        return launched("layer norm kernel launch: ");
    }
    if (p.part) {
        constexpr int64_t wide = 256 * Vec<T>::kN;
        hipLaunchKernelGGL((fb_layer_norm_long_dw_kernel<T>), dim3((unsigned)((H + wide - 1) / wide), (unsigned)grad_groups(p.R, H)), dim3(256), 0,
                           stream, p);
        const int rc = launched("layer norm gradient kernel launch: ");
        if (rc != FB_OK) return rc;
    }
    if (p.y) {
        hipLaunchKernelGGL((fb_layer_norm_long_dx_kernel<T, W>), dim3((unsigned)std::min<int64_t>(p.R, 2 * kCUs)), dim3(1024), 0, stream, p);
        return launched("layer norm gradient kernel launch: ");
    }
    return FB_OK;
}

int dispatch_norm(const NormParams &p, int type, int wtype, bool grad, hipStream_t stream)
{
    if (type == FB_TYPE_F32) return launch_norm<float, float>(p, grad, stream);
    if (type == FB_TYPE_BF16)
        return wtype == FB_TYPE_F32 ? launch_norm<bf16, float>(p, grad, stream) : launch_norm<bf16, bf16>(p, grad, stream);
    return wtype == FB_TYPE_F32 ? launch_norm<f16, float>(p, grad, stream) : launch_norm<f16, f16>(p, grad, stream);
}

int check_norm(const char *who, const void *x, int64_t ldx, int wtype, int64_t R, int64_t H, int type)
{
    const std::string w(who);
    if (!known_type(type) || (wtype != FB_TYPE_F32 && wtype != type)) return fail(FB_EINVAL, w + ": unknown type, or a weight type that is neither float nor the rows'");
    if (bad_rows(R) || bad_width(H)) return fail(FB_EINVAL, w + ": R must be 0 or more, H 1 or more, both below 2^31");
    if (!x && R > 0) return fail(FB_EINVAL, w + ": x is NULL");
    if (bad_ld(ldx, H)) return fail(FB_EINVAL, w + ": rows closer than H elements");
    return FB_OK;
}

}  // namespace

}  // namespace fb

extern "C" {

int fb_layer_norm(const void *x, int64_t ldx, const void *weight, const void *bias, int wtype, int64_t R, int64_t H, int type,
                  float eps, void *y, int64_t ldy, float *mean, float *rstd, fb_stream stream)
{
    using namespace fb;
    return guarded([&]() -> int {
        const int rc = check_norm("fb_layer_norm", x, ldx, wtype, R, H, type);
        if (rc != FB_OK) return rc;
        if (!(eps >= 0.0f) || std::isinf(eps)) return fail(FB_EINVAL, "fb_layer_norm: eps must be finite and not negative");
        if (!y && R > 0) return fail(FB_EINVAL, "fb_layer_norm: y is NULL");
        if (bad_ld(ldy, H)) return fail(FB_EINVAL, "fb_layer_norm: rows closer than H elements");
        if (R == 0) return FB_OK;
        NormParams p{};
        p.x = x; p.ldx = ldx; p.weight = weight; p.bias = bias; p.R = R; p.H = H; p.eps = eps; p.y = y; p.ldy = ldy;
        p.past = goes_past(R, H, type);
        p.mean = mean; p.rstd = rstd;
        return dispatch_norm(p, type, wtype, false, (hipStream_t)stream);
    });
}

size_t fb_layer_norm_grad_workspace_bytes(int64_t R, int64_t H)
{
    using namespace fb;
    if (bad_rows(R) || bad_width(H)) return 0;
    return ((size_t)std::max<int64_t>(grad_groups(R, H), 1) * 2 * (size_t)H * sizeof(float) + 255) & ~(size_t)255;
}

int fb_layer_norm_grad(const void *dy, int64_t lddy, const void *x, int64_t ldx, const float *mean, const float *rstd,
                       const void *weight, int wtype, int64_t R, int64_t H, int type, void *dx, int64_t lddx, float *dweight,
                       float *dbias, void *ws, size_t ws_bytes, fb_stream stream)
{
    using namespace fb;
    return guarded([&]() -> int {
        int rc = check_norm("fb_layer_norm_grad", x, ldx, wtype, R, H, type);
        if (rc != FB_OK) return rc;
        if ((!dy || !mean || !rstd) && R > 0) return fail(FB_EINVAL, "fb_layer_norm_grad: dy, mean or rstd is NULL");
        if (bad_ld(lddy, H) || (dx && bad_ld(lddx, H))) return fail(FB_EINVAL, "fb_layer_norm_grad: rows closer than H elements");
        const bool sums = dweight || dbias;
        if (sums && (!ws || ws_bytes < fb_layer_norm_grad_workspace_bytes(R, H)))
            return fail(FB_EINVAL, "fb_layer_norm_grad: workspace missing or too small");
        NormParams p{};
        p.x = x; p.ldx = ldx; p.dy = dy; p.lddy = lddy; p.weight = weight; p.R = R; p.H = H; p.y = dx; p.ldy = lddx;
        p.past = goes_past(R, H, type);
        p.mean = const_cast<float *>(mean); p.rstd = const_cast<float *>(rstd);
        p.part = sums ? (float *)ws : nullptr;
        if (R > 0 && (dx || sums)) {
            rc = dispatch_norm(p, type, wtype, true, (hipStream_t)stream);
            if (rc != FB_OK) return rc;
        }
        return sums ? launch_column_sum((const float *)ws, R > 0 ? grad_groups(R, H) : 0, H, dweight, dbias, stream) : FB_OK;
    });
}

}  // extern "C"
