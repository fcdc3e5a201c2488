// The way from one block into the next (fb_layers.h): norm of what the block gives, gate, scale, residual, norm of their sum, in one
// pass, and its gradient.  Bound by memory: a row is read once into the registers of one to eight waves, everything that needs
// it whole is formed there, and it is written once.  Measured, bfloat16: 69120 x 1024 with both norms and a gate of one row 108 us (566 MB, 5.3
// TB/s), the gradient with a gate of rows and all seven outputs 205 us (1.13 GB, 5.5 TB/s), 6 of them the second launch; one row of 512 3.1 us on
// the GPU, 12.6 a call.
#include "fb_layers_device.h"

namespace fb {

namespace {

constexpr int kSums = 5;               // of columns: inner weight, inner bias, gate, weight, bias
enum { kInnerWeight, kInnerBias, kGate, kWeight, kBias };

struct ResidualParams {
    const void *h, *residual, *gate, *inner_weight, *inner_bias, *weight, *bias;
    int64_t ldh, ldr, ldg;             // ldg 0: gate is one row, of the weights' type
    int inner, outer;
    float scale, eps;
    int64_t R, H;
    void *s, *y;
    int64_t lds, ldy;
    float *stats;                      // [4][R]
    // gradient
    const void *ds, *dy;
    int64_t ldds, lddy;
    void *dh, *dresidual, *dgate;      // dgate: of rows
    int64_t lddh, lddr, lddg;
    float *part;                       // [sum][workgroup][H]
    int slot[kSums];                   // which sum in part, -1: not wanted
    bool past;                         // outputs go past the caches
};

// A piece without its first n elements (0 < n < kN), zeros behind the others.
template <class T>
__device__ __forceinline__ u32x4 drop(const u32x4 &r, int n)
{
    const int bits = n * 8 * (int)sizeof(T);
    uint64_t lo = (uint64_t)r[1] << 32 | r[0], hi = (uint64_t)r[3] << 32 | r[2];
    if (bits < 64) {
        lo = lo >> bits | hi << (64 - bits);
        hi >>= bits;
    } else {
        lo = hi >> (bits - 64);
        hi = 0;
    }
    return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// What the places of a lane in a row are: WAVES waves have a row, EPL elements a lane, a piece at a time.  A row's last piece, where it is not
// whole, is asked for as the whole piece that ends with the row, and what other lanes have of it is dropped when it has come (it may have been
// written in the meantime): element by element it was waited for at once, and 19904 x 2357 in bfloat16 took 182 instead of 130 us,
// backward 500 instead of 336.
enum Ends { kWhole, kEnding, kParts };     // rows are whole pieces; their last piece as above; element by element

template <class T, int WAVES, int EPL, Ends ENDS>
struct Places {
    static constexpr int kVE = Vec<T>::kN, kPieces = EPL / kVE, kStep = WAVES * 64;
    static constexpr int kThreads = WAVES < 4 ? 256 : WAVES * 64, kRows = kThreads / kStep;   // of a workgroup at a time
    int lane, sub, H;
    __device__ __forceinline__ explicit Places(int64_t width) : lane(threadIdx.x % kStep), sub(threadIdx.x / kStep), H((int)width) {}
    __device__ __forceinline__ int at(int i) const { return (i * kStep + lane) * kVE; }
    __device__ __forceinline__ bool in(int i, int j) const { return at(i) + j < H; }
    // (n elements of the row are there: H, or none)
    __device__ __forceinline__ void ask(const void *p, int64_t r, int64_t ld, int n, u32x4 (&raw)[kPieces]) const
    {
        const T *row = (const T *)p + (n ? r * ld : 0);
        if (ENDS == kWhole || (ENDS == kEnding && H >= kVE)) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int c = ENDS == kEnding && at(i) > H - kVE ? H - kVE : at(i);
                raw[i] = u32x4{0, 0, 0, 0};
                if (at(i) < n) raw[i] = *(const u32x4_any *)(row + c);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) raw[i] = load_piece(row + at(i), n - at(i));
        }
    }
    __device__ __forceinline__ void open(const u32x4 (&raw)[kPieces], float (&v)[EPL]) const
    {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int seen = at(i) - (H - kVE);
            u32x4 piece = raw[i];
            if (ENDS == kEnding && seen > 0 && seen < kVE && H >= kVE) piece = drop<T>(piece, seen);
            unpack<T>(piece, v + i * kVE);
        }
    }
    // A vector of [H], at the same places; `none` where there is no vector.
    template <class W>
    __device__ __forceinline__ void vector(const void *w, float none, float (&v)[EPL]) const
    {
        constexpr int kN = Vec<W>::kN;
        if constexpr (ENDS == kParts) {
            load_vector<W, EPL, kVE>(w, H, kStep, lane, none, v);
            return;
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
#pragma unroll
            for (int j = 0; j < kVE; j += kN) {
                const int c = at(i) + j;
                u32x4 piece = {0, 0, 0, 0};
                if (ENDS == kWhole) {
                    if (w && c < H) piece = *(const u32x4_any *)((const W *)w + c);
                } else if (ENDS == kEnding && H >= kN) {
                    if (w && c < H) piece = *(const u32x4_any *)((const W *)w + (c < H - kN ? c : H - kN));
                    if (c > H - kN && c < H) piece = drop<W>(piece, c - (H - kN));
                } else if (w) {
                    piece = load_piece((const W *)w + c, H - c);
                }
                float u[kN];
                unpack<W>(piece, u);
#pragma unroll
                for (int e = 0; e < kN; ++e) v[i * kVE + j + e] = w ? u[e] : none;
            }
        }
    }
    __device__ __forceinline__ void store(void *p, int64_t r, int64_t ld, const float (&v)[EPL], bool past) const
    {
        T *row = (T *)p + r * ld;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) store_piece(row + at(i), ENDS != kWhole ? H - at(i) : at(i) < H ? kVE : 0, pack<T>(v + i * kVE), past);
    }
};

// Mean and 1 / deviation of a row in registers, v turned into distances from the mean (0 past the row's end).  The variance is
// the mean of the squared distances: no difference of large sums.
template <class P, int WAVES, int EPL>
__device__ __forceinline__ void norm_row(const P &at, int kind, float eps, float inv, float (&v)[EPL], float (*slots)[WAVES][1], float &mean, float &rstd)
{
    mean = 0.0f;
    if (kind == FB_NORM_LAYER) {
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < EPL; ++i) s[0] += v[i];
        sum_row<WAVES, 1>(s, slots, 0);
        mean = s[0] * inv;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        v[i] = at.in(i / P::kVE, i % P::kVE) ? v[i] - mean : 0.0f;
        q[0] = fmaf(v[i], v[i], q[0]);
    }
    sum_row<WAVES, 1>(q, slots, 1);
    rstd = 1.0f / sqrtf(q[0] * inv + eps);
}

template <class T, class W, int WAVES, int EPL, Ends ENDS>
__global__ __launch_bounds__((Places<T, WAVES, EPL, ENDS>::kThreads)) void fb_residual_norm_kernel(ResidualParams p)
{
    typedef Places<T, WAVES, EPL, ENDS> P;
    constexpr int NV = P::kPieces;
    __shared__ float slots[2][P::kRows][4][WAVES][1];       // (by turns: a wave may be a row ahead of one that still reads)
    const P at(p.H);
    const bool gate_rows = p.gate && p.ldg, gate_vector = p.gate && !p.ldg;
    float w1[EPL], b1[EPL], w2[EPL], b2[EPL];
    at.template vector<W>(p.inner_weight, 1.0f, w1);
    at.template vector<W>(p.inner_bias, 0.0f, b1);
    at.template vector<W>(p.weight, 1.0f, w2);
    at.template vector<W>(p.bias, 0.0f, b2);
    {                                                       // a gate of one row, and the scale, go into the inner weights
        float g[EPL];
        at.template vector<W>(gate_vector ? p.gate : nullptr, 1.0f, g);
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            w1[i] *= g[i] * p.scale;
            if (p.inner_bias) b1[i] *= g[i] * p.scale;
        }
    }
    const float inv = 1.0f / (float)at.H;
    const int64_t rstep = (int64_t)gridDim.x * P::kRows;
    u32x4 rh[NV], rr[NV], rg[NV];
    auto ask = [&](int64_t r) {
        const int n = r < p.R ? at.H : 0;
        at.ask(p.h, r, p.ldh, n, rh);
        if (p.residual) at.ask(p.residual, r, p.ldr, n, rr);
        if (gate_rows) at.ask(p.gate, r, p.ldg, n, rg);
    };
    int turn = 0;
    int64_t base = (int64_t)blockIdx.x * P::kRows;
    ask(base + at.sub);
    for (; base < p.R; base += rstep, turn ^= 1) {
        const int64_t r = base + at.sub;
        float v[EPL], x[EPL];
        at.open(rh, v);
        float m1 = 0.0f, r1 = 1.0f, m2 = 0.0f, r2 = 1.0f;
        if (p.inner != FB_NORM_NONE) norm_row<P, WAVES, EPL>(at, p.inner, p.eps, inv, v, slots[turn][at.sub], m1, r1);
#pragma unroll
        for (int i = 0; i < EPL; ++i) v[i] = fmaf(v[i] * r1, w1[i], b1[i]);
        if (gate_rows) {
            at.open(rg, x);
#pragma unroll
            for (int i = 0; i < EPL; ++i) v[i] *= x[i];
        }
        if (p.residual) {
            at.open(rr, x);
#pragma unroll
            for (int i = 0; i < EPL; ++i) v[i] += x[i];
        }
        ask(r + rstep);
        if (r < p.R) at.store(p.s, r, p.lds, v, p.past);
        if (p.outer != FB_NORM_NONE) {
            norm_row<P, WAVES, EPL>(at, p.outer, p.eps, inv, v, slots[turn][at.sub] + 2, m2, r2);
            if (r < p.R) {
#pragma unroll
                for (int i = 0; i < EPL; ++i) v[i] = fmaf(v[i] * r2, w2[i], b2[i]);
                at.store(p.y, r, p.ldy, v, p.past);
            }
        }
        if (p.stats && at.lane == 0 && r < p.R) {
            p.stats[r] = m1;
            p.stats[p.R + r] = r1;
            p.stats[2 * p.R + r] = m2;
            p.stats[3 * p.R + r] = r2;
        }
    }
}

// With xh2 = (s - m2) r2, g2 = dy w2:  d = ds + r2 (g2 - sum g2 / H - xh2 sum(g2 xh2) / H) is the gradient of s and of the
// residual; du = scale d; with xh1 = (h - m1) r1, u = xh1 w1 + b1:  dgate = du u, and through the inner norm with
// du gate in the place of dy.  (rms: no sum g / H.)  Sums of columns stay in registers over all rows that a lane sees and leave
// once, a row of sums a workgroup (two workgroups a compute unit: with four, whose sums are twice as many, 4811 x 777 in single precision takes 38
// instead of 33.5 us and 69120 x 1024 220 instead of 207).  LEAN: weights are read again for every row, the next row is not asked for ahead.
template <class T, class W, int WAVES, int EPL, Ends ENDS, bool LEAN>
__global__ __launch_bounds__((Places<T, WAVES, EPL, ENDS>::kThreads)) void fb_residual_norm_grad_kernel(ResidualParams p)
{
    typedef Places<T, WAVES, EPL, ENDS> P;
    constexpr int VE = P::kVE, NV = P::kPieces;
    __shared__ float slots[2][P::kRows][2][WAVES][2];
    __shared__ float joined[P::kRows == 1 ? 1 : P::kRows * P::kStep * EPL];
    const P at(p.H);
    const bool gate_rows = p.gate && p.ldg, gate_vector = p.gate && !p.ldg, inner = p.inner != FB_NORM_NONE, outer = p.outer != FB_NORM_NONE;
    const bool need_h = inner || p.dgate || p.slot[kGate] >= 0;
    float w1[EPL], b1[EPL], w2[EPL], gv[EPL];
    auto vectors = [&]() {
        at.template vector<W>(p.inner_weight, 1.0f, w1);
        at.template vector<W>(p.inner_bias, 0.0f, b1);
        at.template vector<W>(p.weight, 1.0f, w2);
        at.template vector<W>(gate_vector ? p.gate : nullptr, 1.0f, gv);
    };
    if (!LEAN) vectors();
    float sum[kSums][EPL] = {};
    const float inv = 1.0f / (float)at.H;
    const int64_t rstep = (int64_t)gridDim.x * P::kRows;
    u32x4 rds[NV] = {}, rdy[NV] = {}, rs[NV] = {}, rh[NV] = {}, rg[NV] = {};
    float m1 = 0.0f, r1 = 1.0f, m2 = 0.0f, r2 = 1.0f;
    auto ask = [&](int64_t r) {
        const int n = r < p.R ? at.H : 0;
        if (p.ds) at.ask(p.ds, r, p.ldds, n, rds);
        if (outer) {
            at.ask(p.dy, r, p.lddy, n, rdy);
            at.ask(p.s, r, p.lds, n, rs);
        }
        if (need_h) at.ask(p.h, r, p.ldh, n, rh);
        if (gate_rows) at.ask(p.gate, r, p.ldg, n, rg);
        if (n && inner) {
            m1 = p.stats[r];
            r1 = p.stats[p.R + r];
        }
        if (n && outer) {
            m2 = p.stats[2 * p.R + r];
            r2 = p.stats[3 * p.R + r];
        }
    };
    int turn = 0;
    int64_t base = (int64_t)blockIdx.x * P::kRows;
    if (!LEAN) ask(base + at.sub);
    for (; base < p.R; base += rstep, turn ^= 1) {
        const int64_t r = base + at.sub;
        if (LEAN) {
            vectors();
            ask(r);
        }
        float d[EPL], g[EPL], xh[EPL], gr[EPL];
        at.open(rds, d);
        at.open(rdy, g);
        at.open(rs, xh);
        const float a1 = m1, c1 = r1, a2 = m2, c2 = r2;
        float t[2] = {0.0f, 0.0f};
        if (outer) {                                    // (past the row's end dy is 0, and with it every share)
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                xh[i] = (xh[i] - a2) * c2;
                sum[kWeight][i] = fmaf(g[i], xh[i], sum[kWeight][i]);
                sum[kBias][i] += g[i];
                g[i] *= w2[i];
                t[0] += g[i];
                t[1] = fmaf(g[i], xh[i], t[1]);
            }
            sum_row<WAVES, 2>(t, slots[turn][at.sub], 0);
            const float t0 = p.outer == FB_NORM_LAYER ? t[0] * inv : 0.0f, t1 = t[1] * inv;
#pragma unroll
            for (int i = 0; i < EPL; ++i) d[i] = at.in(i / VE, i % VE) ? fmaf(c2, g[i] - t0 - xh[i] * t1, d[i]) : 0.0f;
        }
        at.open(rh, xh);
        at.open(rg, gr);
        if (!LEAN) ask(r + rstep);
        if (p.dresidual && r < p.R) at.store(p.dresidual, r, p.lddr, d, p.past);
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            d[i] *= p.scale;
            xh[i] = (xh[i] - a1) * c1;
        }
        if (p.gate) {
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                g[i] = d[i] * fmaf(xh[i], w1[i], b1[i]);
                sum[kGate][i] += g[i];
                d[i] *= gate_vector ? gv[i] : gr[i];
            }
            if (p.dgate && r < p.R) at.store(p.dgate, r, p.lddg, g, p.past);
        }
        if (inner) {
            t[0] = t[1] = 0.0f;
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                sum[kInnerWeight][i] = fmaf(d[i], xh[i], sum[kInnerWeight][i]);
                sum[kInnerBias][i] += d[i];
                d[i] *= w1[i];
                t[0] += d[i];
                t[1] = fmaf(d[i], xh[i], t[1]);
            }
            if (p.dh) {
                sum_row<WAVES, 2>(t, slots[turn][at.sub], 1);
                const float t0 = p.inner == FB_NORM_LAYER ? t[0] * inv : 0.0f, t1 = t[1] * inv;
#pragma unroll
                for (int i = 0; i < EPL; ++i) d[i] = c1 * (d[i] - t0 - xh[i] * t1);
            }
        }
        if (p.dh && r < p.R) at.store(p.dh, r, p.lddh, d, p.past);
    }
    if (!p.part) return;
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if (p.slot[k] < 0) continue;
        float *part = p.part + ((size_t)p.slot[k] * gridDim.x + blockIdx.x) * (size_t)at.H;
        if constexpr (P::kRows == 1) {
#pragma unroll
            for (int i = 0; i < EPL; ++i)
                if (at.in(i / VE, i % VE)) part[at.at(i / VE) + i % VE] = sum[k][i];
        } else {                                        // what the workgroup's rows side by side have, added in their order
            __syncthreads();
#pragma unroll
            for (int i = 0; i < EPL; ++i) joined[at.sub * P::kStep * EPL + at.at(i / VE) + i % VE] = sum[k][i];
            __syncthreads();
            for (int c = threadIdx.x; c < at.H; c += P::kThreads) {
                float s = joined[c];
#pragma unroll
                for (int u = 1; u < P::kRows; ++u) s += joined[u * P::kStep * EPL + c];
                part[c] = s;
            }
        }
    }
}

struct SumParams {
    const float *part;                 // [sum][P][H]
    int64_t P, H;
    float *out[kSums];
};

// out[k][c] = sum over i < P of part[k][i][c], in a fixed order: 16 threads share a column, each adding every 16th row.
__global__ __launch_bounds__(1024) void fb_residual_norm_sum_kernel(SumParams p)
{
    __shared__ float slots[16][64];
    const int col = threadIdx.x & 63, g = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + col;
    const float *q = p.part + (size_t)blockIdx.y * p.P * p.H + c;
    float s[4] = {};
    if (c < p.H) {
        int64_t i = g;
        for (; i + 48 < p.P; i += 64) {
#pragma unroll
            for (int u = 0; u < 4; ++u) s[u] += q[(i + 16 * u) * p.H];
        }
        for (; i < p.P; i += 16) s[0] += q[i * p.H];
    }
    slots[g][col] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (g == 0 && c < p.H) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) t += slots[i][col];
        p.out[blockIdx.y][c] = t;
    }
}

constexpr int64_t kResidualWidth = 8192;   // the longest row that a workgroup holds in registers with its sums

int64_t rows_at_once(int64_t H) { return H <= 512 ? 4 : H <= 1024 ? 2 : 1; }
int64_t residual_groups(int64_t R, int64_t H)
{
    const int64_t rows = rows_at_once(H);
    return std::max<int64_t>(1, std::min<int64_t>((R + rows - 1) / rows, 2 * kCUs));
}

template <class T, class W, int WAVES, int EPL, Ends ENDS>
int launch_residual(const ResidualParams &p, bool grad, hipStream_t stream)
{
    typedef Places<T, WAVES, EPL, ENDS> P;
    if (grad) {
        // (few registers: a last piece is waited for at once, 13894 x 5094 in half precision 930 instead of 1212 us)
        constexpr bool kLean = EPL > 8;
        hipLaunchKernelGGL((fb_residual_norm_grad_kernel<T, W, WAVES, EPL, kLean ? kParts : ENDS, kLean>), dim3((unsigned)residual_groups(p.R, p.H)),
                           dim3(P::kThreads), 0, stream, p);
    } else {
        const int64_t groups = (p.R + P::kRows - 1) / P::kRows, most = (int64_t)kCUs * (P::kThreads > 256 ? 4 : 8);
        hipLaunchKernelGGL((fb_residual_norm_kernel<T, W, WAVES, EPL, ENDS>), dim3((unsigned)std::min(groups, most)), dim3(P::kThreads), 0, stream, p);
    }
    return launched("residual norm kernel launch: ");
}

template <class T, class W, int WAVES, int EPL>
int launch_residual(const ResidualParams &p, bool grad, hipStream_t stream)
{
    // (pieces of four elements: up to three single ones are no slower than what drops them, 4811 x 777 16 and 19 us)
    if (p.H % Vec<T>::kN == 0) return launch_residual<T, W, WAVES, EPL, kWhole>(p, grad, stream);
    return launch_residual<T, W, WAVES, EPL, sizeof(T) == 4 ? kParts : kEnding>(p, grad, stream);
}

template <class T, class W>
int launch_residual(const ResidualParams &p, bool grad, hipStream_t stream)
{
    if (p.H <= 512) return launch_residual<T, W, 1, 8>(p, grad, stream);
    if (p.H <= 1024) return launch_residual<T, W, 2, 8>(p, grad, stream);
    if (p.H <= 2048) return launch_residual<T, W, 4, 8>(p, grad, stream);
    if (p.H <= 4096) return launch_residual<T, W, 8, 8>(p, grad, stream);
    return launch_residual<T, W, 8, 16>(p, grad, stream);
}

int dispatch_residual(const ResidualParams &p, int type, int wtype, bool grad, hipStream_t stream)
{
    if (type == FB_TYPE_F32) return launch_residual<float, float>(p, grad, stream);
    if (type == FB_TYPE_BF16)
        return wtype == FB_TYPE_F32 ? launch_residual<bf16, float>(p, grad, stream) : launch_residual<bf16, bf16>(p, grad, stream);
    return wtype == FB_TYPE_F32 ? launch_residual<f16, float>(p, grad, stream) : launch_residual<f16, f16>(p, grad, stream);
}

bool known_norm(int kind) { return kind == FB_NORM_NONE || kind == FB_NORM_LAYER || kind == FB_NORM_RMS; }

int check_residual(const char *who, const void *gate, int64_t ldg, float scale, int inner, const void *inner_weight, const void *inner_bias, int outer,
                   const void *weight, const void *bias, int wtype, int64_t R, int64_t H, int type)
{
    const std::string w(who);
    if (!known_type(type) || (wtype != FB_TYPE_F32 && wtype != type)) return fail(FB_EINVAL, w + ": unknown type, or a weight type that is neither float nor the rows'");
    if (!known_norm(inner) || !known_norm(outer)) return fail(FB_EINVAL, w + ": unknown norm");
    if ((inner == FB_NORM_NONE && (inner_weight || inner_bias)) || (outer == FB_NORM_NONE && (weight || bias)))
        return fail(FB_EINVAL, w + ": weight or bias without a norm");
    if (bad_rows(R) || bad_width(H)) return fail(FB_EINVAL, w + ": R must be 0 or more, H 1 or more, both below 2^31");
    if (!std::isfinite(scale)) return fail(FB_EINVAL, w + ": scale must be finite");
    if (gate && ldg != 0 && bad_ld(ldg, H)) return fail(FB_EINVAL, w + ": rows of gate closer than H elements");
    if (H > kResidualWidth) return fail(FB_EUNSUPPORTED, w + ": H above 8192");
    return FB_OK;
}

}  // namespace

}  // namespace fb

extern "C" {

int fb_residual_norm(const void *h, int64_t ldh, const void *residual, int64_t ldr, const void *gate, int64_t ldg, float scale, int inner,
                     const void *inner_weight, const void *inner_bias, int outer, const void *weight, const void *bias, int wtype, int64_t R,
                     int64_t H, int type, float eps, void *s, int64_t lds, void *y, int64_t ldy, float *stats, fb_stream stream)
{
    using namespace fb;
    return guarded([&]() -> int {
        const int rc = check_residual("fb_residual_norm", gate, ldg, scale, inner, inner_weight, inner_bias, outer, weight, bias, wtype, R, H, type);
        if (rc != FB_OK) return rc;
        if (!(eps >= 0.0f) || std::isinf(eps)) return fail(FB_EINVAL, "fb_residual_norm: eps must be finite and not negative");
        if ((!h || !s || (!y && outer != FB_NORM_NONE)) && R > 0) return fail(FB_EINVAL, "fb_residual_norm: h, s or y is NULL");
        if (bad_ld(ldh, H) || bad_ld(lds, H) || (residual && bad_ld(ldr, H)) || (outer != FB_NORM_NONE && bad_ld(ldy, H)))
            return fail(FB_EINVAL, "fb_residual_norm: rows closer than H elements");
        if (R == 0) return FB_OK;
        ResidualParams p{};
        p.h = h; p.ldh = ldh; p.residual = residual; p.ldr = ldr; p.gate = gate; p.ldg = ldg; p.scale = scale; p.eps = eps;
        p.inner = inner; p.inner_weight = inner_weight; p.inner_bias = inner_bias; p.outer = outer; p.weight = weight; p.bias = bias;
        p.R = R; p.H = H; p.s = s; p.lds = lds; p.y = y; p.ldy = ldy; p.stats = stats;
        p.past = goes_past(R, H, type);
        return dispatch_residual(p, type, wtype, false, (hipStream_t)stream);
    });
}

size_t fb_residual_norm_grad_workspace_bytes(int64_t R, int64_t H)
{
    using namespace fb;
    if (bad_rows(R) || bad_width(H) || H > kResidualWidth) return 0;
    return ((size_t)residual_groups(R, H) * kSums * (size_t)H * sizeof(float) + 255) & ~(size_t)255;
}

int fb_residual_norm_grad(const void *ds, int64_t ldds, const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *s, int64_t lds,
                          const float *stats, const void *gate, int64_t ldg, float scale, int inner, const void *inner_weight, const void *inner_bias,
                          int outer, const void *weight, int wtype, int64_t R, int64_t H, int type, void *dh, int64_t lddh, void *dresidual,
                          int64_t lddr, void *dgate, int64_t lddg, float *dinner_weight, float *dinner_bias, float *dweight, float *dbias, void *ws,
                          size_t ws_bytes, fb_stream stream)
{
    using namespace fb;
    return guarded([&]() -> int {
        int rc = check_residual("fb_residual_norm_grad", gate, ldg, scale, inner, inner_weight, inner_bias, outer, weight, nullptr, wtype, R, H, type);
        if (rc != FB_OK) return rc;
        const bool in = inner != FB_NORM_NONE, out = outer != FB_NORM_NONE, rows = gate && ldg, vector = gate && !ldg;
        if ((!in && (dinner_weight || dinner_bias)) || (!out && (dweight || dbias)) || (!gate && dgate))
            return fail(FB_EINVAL, "fb_residual_norm_grad: a gradient of something that is not there");
        if (R > 0) {
            if (!ds && !out) return fail(FB_EINVAL, "fb_residual_norm_grad: neither ds nor an outer norm");
            if (out && (!dy || !s)) return fail(FB_EINVAL, "fb_residual_norm_grad: dy or s is NULL");
            if ((in || dgate) && !h) return fail(FB_EINVAL, "fb_residual_norm_grad: h is NULL");
            if ((in || out) && !stats) return fail(FB_EINVAL, "fb_residual_norm_grad: stats is NULL");
        }
        if ((ds && bad_ld(ldds, H)) || (out && (bad_ld(lddy, H) || bad_ld(lds, H))) || (h && bad_ld(ldh, H)) || (dh && bad_ld(lddh, H)) ||
            (dresidual && bad_ld(lddr, H)) || (dgate && rows && bad_ld(lddg, H)))
            return fail(FB_EINVAL, "fb_residual_norm_grad: rows closer than H elements");
        float *outs[kSums] = {dinner_weight, dinner_bias, vector ? (float *)dgate : nullptr, dweight, dbias};
        SumParams q{};
        ResidualParams p{};
        int n = 0;
        for (int k = 0; k < kSums; ++k) {
            p.slot[k] = outs[k] ? n : -1;
            if (outs[k]) q.out[n++] = outs[k];
        }
        if (n && (!ws || ws_bytes < fb_residual_norm_grad_workspace_bytes(R, H)))
            return fail(FB_EINVAL, "fb_residual_norm_grad: workspace missing or too small");
        p.ds = ds; p.ldds = ldds; p.dy = dy; p.lddy = lddy; p.h = h; p.ldh = ldh; p.s = const_cast<void *>(s); p.lds = lds;
        p.stats = const_cast<float *>(stats); p.gate = gate; p.ldg = ldg; p.scale = scale; p.inner = inner; p.inner_weight = inner_weight;
        p.inner_bias = inner_bias; p.outer = outer; p.weight = weight; p.R = R; p.H = H; p.dh = dh; p.lddh = lddh; p.dresidual = dresidual;
        p.lddr = lddr; p.dgate = rows ? dgate : nullptr; p.lddg = lddg;
        p.past = goes_past(R, H, type);
        p.part = n ? (float *)ws : nullptr;
        hipStream_t st = (hipStream_t)stream;
        if (R > 0 && (n || dh || dresidual || dgate) && (rc = dispatch_residual(p, type, wtype, true, st)) != FB_OK) return rc;
        if (!n) return FB_OK;
        q.part = (const float *)ws;
        q.P = R > 0 ? residual_groups(R, H) : 0;
        q.H = H;
        hipLaunchKernelGGL(fb_residual_norm_sum_kernel, dim3((unsigned)((H + 63) / 64), (unsigned)n), dim3(1024), 0, st, q);
        return launched("residual norm sum kernel launch: ");
    });
}

}  // extern "C"
