// Gated layer and its gradient (fb_layers.h): y = act(x G^T + a) (x U^T + b).
//
// Forward, both products are one, of x with G and U in turn 32 rows of each (see Side in fb_mfma.h): a wave's two fragments of the
// weight are the same rows of both, so that g and u of an output meet in one wave and y leaves alone.  44160 x 2048 x 1024 in bfloat16 with silu
// and both preactivations: 387 us (957 TFLOP/s); of these 305 are the products (1215), the rest the outputs' way through the registers and LDS, which
// nothing overlaps (543 MB; starting half of the chiplets later, so that they do not store all at once, changes nothing).
//
// Backward, dz is made in one pass over dy and preact, and is a factor of two products: 855 us for the same sizes, dz 163 (5.6 TB/s), dx 362 and
// dW 305 (1023 and 1215 TFLOP/s), shares of dW joined 20.
#include "fb_mfma.h"

namespace fb {

namespace {

// Sums of a wave leave as y = act(g) u, formed in the registers that have them, and as g and u.
struct Gated {
    static constexpr bool kPaired = true, kNeverEmpty = true, kFolded = false;
    static constexpr int kEarly = 1;

    template <int FI, int FJ>
    static __device__ __forceinline__ void early(const Product &q, const Where &where, int lane, f32x4 (&four)[1])
    {
        if (!q.f.bias) return;
#pragma unroll
        for (int y = 0; y < FJ; ++y) {
            const int64_t j = where.j0 + (where.wj * (FJ / 2) + y / 2) * 32 + lane;
            if (lane < 32 && j < q.N) four[0][y] = q.f.bias[(y & 1) * q.N + j];
        }
    }

    template <class T, int FI, int FJ>
    static __device__ __forceinline__ void leave(ProductArgs args, f32x16 (&acc)[FI][FJ], const f32x4 (&bias)[1], float, const Where &where)
    {
        constexpr int F = FJ / 2;
        int lane = threadIdx.x & 63;
        asm volatile("" : "+s"(args), "+v"(lane));
        const int64_t M = args->M, N = args->N, i0 = where.i0 + where.wi * FI * 32, j0 = where.j0 + where.wj * F * 32;
        const int act = args->f.act;
        const bool past = args->past;
        float *mine = where.room + where.wave * 16 * 2 * 32;
#pragma unroll
        for (int x = 0; x < FI; ++x) {
            const int64_t i = i0 + x * 32;
            if (args->f.bias) add_rank_one<FJ>(acc[x], bias[0], 0.0f, lane);
            f32x16 g[F], u[F];
#pragma unroll
            for (int f = 0; f < F; ++f) {
                g[f] = acc[x][2 * f];
                u[f] = acc[x][2 * f + 1];
            }
            if (args->f.preact) {
                store_fragments<T, F>(g, mine, (T *)args->f.preact, args->f.ldp, i, j0, M, N, lane, past);
                store_fragments<T, F>(u, mine, (T *)args->f.preact + N, args->f.ldp, i, j0, M, N, lane, past);
            }
            auto gate = [&](int which) {
#pragma unroll
                for (int f = 0; f < F; ++f)
#pragma unroll
                    for (int k = 0; k < 16; ++k) u[f][k] *= act_of(g[f][k], which);
            };
            if (act == FB_ACT_SILU) gate(FB_ACT_SILU);
            else if (act == FB_ACT_GELU) gate(FB_ACT_GELU);
            else if (act == FB_ACT_SIGMOID) gate(FB_ACT_SIGMOID);
            else if (act == FB_ACT_RELU) gate(FB_ACT_RELU);
            else gate(FB_ACT_NONE);
            store_fragments<T, F>(u, mine, (T *)args->f.y, args->f.ldy, i, j0, M, N, lane, past);
        }
    }
};

// Waves of 64 rows and 64 outputs: runs of 128 bytes of a row leave together.
template <class T>
int launch_gated(const Product &q, hipStream_t stream)
{
    return q.tile == 256 ? launch<T, true, true, 4, 2, 2, 4, Gated>(q, stream) : launch<T, true, true, 2, 2, 2, 2, Gated>(q, stream);
}

// Shares of k added in their order, pair by pair, and finished.
template <class T>
__global__ __launch_bounds__(256) void fb_gated_join_kernel(Product q)
{
    const int64_t N = q.N / 2, n = q.M * N;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < n; at += (int64_t)gridDim.x * 256) {
        const int64_t i = at / N, j = at - i * N;
        float g = 0.0f, u = 0.0f;
#pragma unroll 4
        for (int c = 0; c < q.split; ++c) {
            const float *part = q.part + ((size_t)c * q.M + i) * q.N + j;
            g += part[0];
            u += part[N];
        }
        finish_pair<T>(q.f, N, i, j, g, u);
    }
}

int launch_gated_join(const Product &q, hipStream_t stream)
{
    const dim3 grid((unsigned)std::min<int64_t>((q.M * (q.N / 2) + 255) / 256, 8 * kCUs)), block(256);
    if (q.type == FB_TYPE_F32)
        hipLaunchKernelGGL(fb_gated_join_kernel<float>, grid, block, 0, stream, q);
    else if (q.type == FB_TYPE_BF16)
        hipLaunchKernelGGL(fb_gated_join_kernel<bf16>, grid, block, 0, stream, q);
    else
        hipLaunchKernelGGL(fb_gated_join_kernel<f16>, grid, block, 0, stream, q);
    return launched("gated join kernel launch: ");
}

// dz = [dy u act'(g), dy act(g)], rounded to the factors' type, and the sums of its columns before the rounding.  Bound by memory.
// A thread has one piece of the width, of both halves; the layout of threads is that of rows of N (lay_out).  A row's last piece ends where
// the row does: what it has in common with the one before is formed and stored twice, alike, and summed once.
struct GatedSlopeParams {
    const void *dy, *z;
    int64_t lddy, ldz, M, N, ldo;
    int act;
    void *out;               // nullable
    int64_t low;             // rows from a row of out to the one with what it lacks, 0: none
    float *part;             // [down][2 N], nullable
    int lanes, wide, down;
    uint32_t *peaks;         // half precision: of the largest finite |dz|, see fb_affine_grad; nullable
    int n_peaks;
    float *undo;
};

constexpr int kPairsAhead = 2;

template <class T>
__device__ __forceinline__ void slopes_of(const u32x4 &rd, const u32x4 &rg, const u32x4 &ru, int act, float *dg, float *du)
{
    constexpr int VE = Vec<T>::kN;
    float d[VE], g[VE], u[VE];
    unpack<T>(rd, d);
    unpack<T>(rg, g);
    unpack<T>(ru, u);
    auto by = [&](int which) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            float value, slope;
            act_and_slope(g[e], which, value, slope);
            dg[e] = d[e] * u[e] * slope;
            du[e] = d[e] * value;
        }
    };
    if (act == FB_ACT_SILU) by(FB_ACT_SILU);
    else if (act == FB_ACT_GELU) by(FB_ACT_GELU);
    else if (act == FB_ACT_SIGMOID) by(FB_ACT_SIGMOID);
    else if (act == FB_ACT_RELU) by(FB_ACT_RELU);
    else by(FB_ACT_NONE);
}

template <class T>
__device__ __forceinline__ void make_pairs(const GatedSlopeParams &p, int block, float (*slots)[2 * Vec<T>::kN + 1])
{
    constexpr int VE = Vec<T>::kN;
    const int across = block % p.wide, down = block / p.wide;
    const int lane = threadIdx.x & (p.lanes - 1), sub = threadIdx.x / p.lanes, subs = 256 / p.lanes;
    const int64_t whole = p.N < VE ? 0 : p.N - VE, from = ((int64_t)across * p.lanes + lane) * VE, at = from < whole ? from : whole;
    const int n = from >= p.N ? 0 : (int)(p.N < VE ? p.N : VE), seen = (int)(from - at);
    float sum[2 * VE] = {}, scale = 1.0f;
    if constexpr (std::is_same<T, f16>::value) {
        if (p.peaks) {
            float undo;
            range_of(p.peaks, p.n_peaks, scale, undo);
            if (block == 0 && threadIdx.x == 0) *p.undo = undo;
        }
    }
    if (n > 0) {
        const int64_t step = (int64_t)p.down * subs;
        const int zeros = at == whole ? (int)((VE - 2 * p.N % VE) % VE) : 0;       // of the row's last piece, that the products read
        for (int64_t r0 = (int64_t)down * subs + sub; r0 < p.M; r0 += kPairsAhead * step) {
            u32x4 rd[kPairsAhead], rg[kPairsAhead], ru[kPairsAhead];
#pragma unroll
            for (int a = 0; a < kPairsAhead; ++a) {
                const int64_t r = r0 + a * step;
                const int here = r < p.M ? n : 0;
                rd[a] = load_piece((const T *)p.dy + r * p.lddy + at, here);
                rg[a] = load_piece((const T *)p.z + r * p.ldz + at, here);
                ru[a] = load_piece((const T *)p.z + r * p.ldz + p.N + at, here);
            }
#pragma unroll
            for (int a = 0; a < kPairsAhead; ++a) {
                const int64_t r = r0 + a * step;
                if (r >= p.M) break;
                float d[2 * VE];
                slopes_of<T>(rd[a], rg[a], ru[a], p.act, d, d + VE);
#pragma unroll
                for (int e = 0; e < 2 * VE; ++e) {
                    sum[e] += e % VE >= seen ? d[e] : 0.0f;
                    d[e] *= scale;
                }
                if (!p.out) continue;
                T *out = (T *)p.out + r * p.ldo;
                store_piece(out + at, n, pack<T>(d));
                store_piece(out + p.N + at, n, pack<T>(d + VE));
                for (int c = 0; c < zeros; ++c) out[2 * p.N + c] = (T)0.0f;
                if constexpr (sizeof(T) == 2) {
                    if (p.low) {
                        out += p.low * p.ldo;
                        float high[2 * VE];
                        unpack<T>(pack<T>(d), high);
                        unpack<T>(pack<T>(d + VE), high + VE);
#pragma unroll
                        for (int e = 0; e < 2 * VE; ++e) d[e] = lacks(d[e], high[e]);
                        store_piece(out + at, n, pack<T>(d));
                        store_piece(out + p.N + at, n, pack<T>(d + VE));
                        for (int c = 0; c < zeros; ++c) out[2 * p.N + c] = (T)0.0f;
                    }
                }
            }
        }
    }
    if (!p.part) return;
#pragma unroll
    for (int e = 0; e < 2 * VE; ++e) slots[threadIdx.x][e] = sum[e];
    __syncthreads();
    for (int c = threadIdx.x; c < p.lanes * VE * 2; c += 256) {
        const int half = c / (p.lanes * VE), k = c % (p.lanes * VE);
        const int64_t col = (int64_t)across * p.lanes * VE + k;
        if (col >= p.N) continue;
        float s = 0.0f;
        const int64_t first = col / VE * VE;
        const int e = (int)(col - (first < whole ? first : whole));
        for (int i = 0; i < subs; ++i) s += slots[i * p.lanes + k / VE][half * VE + e];
        p.part[(size_t)down * 2 * p.N + half * p.N + col] = s;
    }
}

// COPIES: workgroups behind those of dz copy what the products cannot take as it is (a launch less: 300 rows, N 501, K 203 in bfloat16 21.8
// instead of 25.0 us a call; nothing at 9601 x 1111 x 777, where both wait for memory).
template <class T, bool COPIES>
__global__ __launch_bounds__(256) void fb_gated_slope_kernel(GatedSlopeParams p, PrepareParams copies)
{
    __shared__ float slots[256][2 * Vec<T>::kN + 1];
    const int blocks = p.wide * p.down;
    if (!COPIES || (int)blockIdx.x < blocks)
        make_pairs<T>(p, blockIdx.x, slots);
    else
        copy_block<T>(copies, blockIdx.x - blocks, (float(*)[Vec<T>::kN + 1]) slots);
}

template <class T>
int launch_pairs(const GatedSlopeParams &p, const Prepare &copies, hipStream_t stream)
{
    const dim3 grid((unsigned)(p.wide * p.down + copies.blocks)), block(256);
    if (copies.n > 0)
        hipLaunchKernelGGL((fb_gated_slope_kernel<T, true>), grid, block, 0, stream, p, copies.p);
    else
        hipLaunchKernelGGL((fb_gated_slope_kernel<T, false>), grid, block, 0, stream, p, copies.p);
    return launched("gated slope kernel launch: ");
}

// The largest finite bound of |dz|, |dy| max(|u| slope_bound(g), act_bound(g)), a share a workgroup (half precision: what fb_affine_grad finds of dy,
// here with u and act(g), which are not bounded).  Bound by memory: 64 MB in 21 us; dz itself in the place of its bound 37.
__global__ __launch_bounds__(1024) void fb_gated_peak_kernel(GatedSlopeParams p)
{
    constexpr int VE = Vec<f16>::kN, kAhead = 2;
    __shared__ uint32_t slots[16];
    const int64_t pieces = (p.N + VE - 1) / VE, step = (int64_t)gridDim.x * 1024, down = step / pieces, across = step - down * pieces;
    const int64_t whole = p.N < VE ? 0 : p.N - VE, at = (int64_t)blockIdx.x * 1024 + threadIdx.x;
    int64_t r = at / pieces, c = at - r * pieces;
    uint32_t peak = 0;
    while (r < p.M) {
        u32x4 rd[kAhead], rg[kAhead], ru[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t j = c * VE < whole ? c * VE : whole;     // (a row's last piece ends with it)
            const int n = r < p.M ? (int)(p.N - j) : 0;
            rd[u] = load_piece((const f16 *)p.dy + r * p.lddy + j, n);
            rg[u] = load_piece((const f16 *)p.z + r * p.ldz + j, n);
            ru[u] = load_piece((const f16 *)p.z + r * p.ldz + p.N + j, n);
            r += down;
            c += across;
            if (c >= pieces) {
                c -= pieces;
                ++r;
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            float d[VE], g[VE], v[VE];
            unpack<f16>(rd[u], d);
            unpack<f16>(rg[u], g);
            unpack<f16>(ru[u], v);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float du = d[e] * act_bound(g[e], p.act), dg = d[e] * v[e] * slope_bound(g[e], p.act);
                uint32_t a = __float_as_uint(du) & 0x7fffffffu, b = __float_as_uint(dg) & 0x7fffffffu;
                a = a < 0x7f800000u ? a : 0u;
                b = b < 0x7f800000u ? b : 0u;
                a = a > b ? a : b;
                peak = a > peak ? a : peak;
            }
        }
    }
    peak = max_wave_u(peak);
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = peak;
    __syncthreads();
    if (threadIdx.x < 64) {
        peak = max_wave_u(threadIdx.x < 16 ? slots[threadIdx.x] : 0u);
        if (threadIdx.x == 0) p.peaks[blockIdx.x] = peak;
    }
}

void lay_out_pairs(GatedSlopeParams &p, int type)
{
    const int64_t ve = 16 / (int64_t)type_bytes(type), pieces = (p.N + ve - 1) / ve;
    for (p.lanes = 1; p.lanes < 64 && p.lanes < pieces;) p.lanes *= 2;
    p.wide = (int)((pieces + p.lanes - 1) / p.lanes);
    const int64_t rows = 256 / p.lanes * kPairsAhead;      // at a time
    p.down = (int)std::max<int64_t>(1, std::min<int64_t>((p.M + rows - 1) / rows, std::max<int64_t>(64, 8 * kCUs / p.wide)));
    p.n_peaks = (int)std::min<int64_t>(kPeakGroups, (p.M * pieces + 1023) / 1024);
}

struct GatedPlan {
    Product q;               // N: both factors' rows if the sums go through memory, else the outputs'
    bool few;
    Packed x, w;
    size_t bytes;
};

GatedPlan gated_plan(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N, int64_t K, int type)
{
    GatedPlan f{};
    f.q.M = M; f.q.N = 2 * N; f.q.K = K; f.q.type = type;
    f.few = M <= kFewRows;
    if (!f.few) {
        plan(f.q);
        // (tiles of 64 have one fragment a wave: their pairs meet in memory)
        f.q.parts = f.q.parts || f.q.tile == 64;
        f.x = packed(x, ldx, M, K, type);
        f.w = packed(weight, ldw, 2 * N, K, type);
        f.bytes = f.x.bytes + f.w.bytes + product_bytes(f.q);
    }
    if (!f.q.parts) f.q.N = N;
    return f;
}

struct GatedGradPlan {
    GradPlan g;
    GatedSlopeParams s;
};

GatedGradPlan gated_grad_plan(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N, int64_t K, int type)
{
    GatedGradPlan p{};
    const bool two = twice(M, 2 * N, K, type);
    p.g = grad_plan(nullptr, 2 * N, type, x, ldx, weight, ldw, two ? 2 * M : M, 2 * N, K, type, FB_ACT_SILU);   // (an activation: dz is made)
    p.g.twice = two;
    if (two) {
        p.g.bytes -= p.g.x.bytes + p.g.part;
        p.g.x = packed(nullptr, K, 2 * M, K, type, true);
        p.g.dx.parts = true;
        p.g.part = product_bytes(p.g.dx);
        p.g.bytes += p.g.x.bytes + p.g.part;
    }
    p.s.low = two ? M : 0;
    p.s.M = M; p.s.N = N; p.s.ldo = p.g.ldz;
    lay_out_pairs(p.s, type);
    const size_t sums = aligned((size_t)p.s.down * 2 * (size_t)N * sizeof(float));
    p.g.bytes += sums - p.g.sums;
    p.g.sums = sums;
    return p;
}

bool bad_pair_sizes(int64_t M, int64_t N, int64_t K) { return bad_sizes(M, N, K) || bad_width(2 * N); }

int check_gated(const char *who, const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N, int64_t K, int type, int act)
{
    const std::string w(who);
    if (!known_type(type)) return fail(FB_EINVAL, w + ": unknown type");
    if (act < FB_ACT_NONE || act > FB_ACT_SIGMOID) return fail(FB_EINVAL, w + ": unknown activation");
    if (bad_pair_sizes(M, N, K)) return fail(FB_EINVAL, w + ": M must be 0 or more and below 2^31, N and K 1 or more, 2 N and K below 2^28");
    if ((!x && M > 0) || !weight) return fail(FB_EINVAL, w + ": x or weight is NULL");
    if (bad_ld(ldx, K) || bad_ld(ldw, K)) return fail(FB_EINVAL, w + ": rows of x or weight closer than K elements");
    return FB_OK;
}

}  // namespace

}  // namespace fb

extern "C" {

size_t fb_gated_affine_workspace_bytes(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N, int64_t K, int type)
{
    using namespace fb;
    if (bad_pair_sizes(M, N, K) || !known_type(type)) return 0;
    return gated_plan(x, ldx, weight, ldw, M, N, K, type).bytes;
}

int fb_gated_affine(const void *x, int64_t ldx, const void *weight, int64_t ldw, const float *bias, int64_t M, int64_t N, int64_t K, int type, int act,
                    void *y, int64_t ldy, void *preact, int64_t ldp, void *ws, size_t ws_bytes, fb_stream stream)
{
    using namespace fb;
    return guarded([&]() -> int {
        int rc = check_gated("fb_gated_affine", x, ldx, weight, ldw, M, N, K, type, act);
        if (rc != FB_OK) return rc;
        if (!y && M > 0) return fail(FB_EINVAL, "fb_gated_affine: y is NULL");
        if (bad_ld(ldy, N) || (preact && bad_ld(ldp, 2 * N))) return fail(FB_EINVAL, "fb_gated_affine: rows closer than their width");
        if (M > kFewRows ? too_long(K, type) || too_far(ldy) || (preact && too_far(ldp)) : N >= (int64_t)1 << 25)
            return fail(FB_EUNSUPPORTED, "fb_gated_affine: rows of x and weight longer than 4 MB, rows of y or preact 2^27 elements apart, or (M <= 64) N of 2^25 and more");
        const GatedPlan f = gated_plan(x, ldx, weight, ldw, M, N, K, type);
        if (f.bytes && (!ws || ws_bytes < f.bytes)) return fail(FB_EINVAL, "fb_gated_affine: workspace missing or too small");
        if (M == 0) return FB_OK;
        hipStream_t st = (hipStream_t)stream;
        char *xs = (char *)ws, *wts = xs + f.x.bytes;
        Product q = f.q;
        q.f = {bias, nullptr, 0, act, y, ldy, type, preact, ldp, nullptr};
        if (f.few) {
            q.N = N;
            q.A = {x, ldx, true};
            q.B = {weight, ldw, true};
            return launch_few_pairs(q, st);
        }
        Prepare jobs;
        if (f.x.copy) jobs.add(pack_job(f.x, x, ldx, M, K, xs), type);
        if (f.w.copy) jobs.add(pack_job(f.w, weight, ldw, 2 * N, K, wts), type);
        if ((rc = launch_prepare(jobs, type, type, st)) != FB_OK) return rc;
        q.A = {f.x.copy ? xs : x, f.x.ld, true};
        q.B = {f.w.copy ? wts : weight, f.w.ld, true};
        q.part = (float *)(wts + f.w.bytes);
        if (q.parts) {
            if ((rc = launch_mfma_product(q, st)) != FB_OK) return rc;
            return launch_gated_join(q, st);
        }
        if (type == FB_TYPE_F32) return launch_gated<float>(q, st);
        return type == FB_TYPE_BF16 ? launch_gated<bf16>(q, st) : launch_gated<f16>(q, st);
    });
}

size_t fb_gated_affine_grad_workspace_bytes(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N, int64_t K, int type)
{
    using namespace fb;
    if (bad_pair_sizes(M, N, K) || !known_type(type)) return 0;
    return gated_grad_plan(x, ldx, weight, ldw, M, N, K, type).g.bytes;
}

int fb_gated_affine_grad(const void *dy, int64_t lddy, const void *x, int64_t ldx, const void *weight, int64_t ldw, const void *preact, int64_t ldp,
                         int64_t M, int64_t N, int64_t K, int type, int act, void *dx, int64_t lddx, void *dweight, float *dbias, void *ws,
                         size_t ws_bytes, fb_stream stream)
{
    using namespace fb;
    return guarded([&]() -> int {
        int rc = check_gated("fb_gated_affine_grad", x, ldx, weight, ldw, M, N, K, type, act);
        if (rc != FB_OK) return rc;
        if ((!dy || !preact) && M > 0) return fail(FB_EINVAL, "fb_gated_affine_grad: dy or preact is NULL");
        if (bad_ld(lddy, N) || bad_ld(ldp, 2 * N) || (dx && bad_ld(lddx, K))) return fail(FB_EINVAL, "fb_gated_affine_grad: rows closer than their width");
        if (!dx && !dweight && !dbias) return FB_OK;
        if (too_long(K, type) || too_long(2 * N, type) || (dx && too_far(lddx)))
            return fail(FB_EUNSUPPORTED, "fb_gated_affine_grad: rows of x, weight and dz longer than 4 MB, or rows of dx 2^27 elements apart");
        GatedGradPlan p = gated_grad_plan(x, ldx, weight, ldw, M, N, K, type);
        GradPlan &g = p.g;
        if (!ws || ws_bytes < g.bytes) return fail(FB_EINVAL, "fb_gated_affine_grad: workspace missing or too small");
        hipStream_t st = (hipStream_t)stream;
        char *dz = (char *)ws, *xs = dz + g.dz, *wts = xs + g.x.bytes;
        float *sums = (float *)(wts + g.w.bytes), *undo = (float *)(wts + g.w.bytes + g.sums);
        float *part = (float *)((char *)undo + g.range);
        const bool scale = g.scale && (dx || dweight) && M > 0;
        GatedSlopeParams s = p.s;
        s.dy = dy; s.lddy = lddy; s.z = preact; s.ldz = ldp; s.act = act;
        s.out = dx || dweight ? dz : nullptr;
        s.part = dbias ? sums : nullptr;
        s.undo = undo;
        s.peaks = scale ? (uint32_t *)(undo + 1) : nullptr;
        if (scale) {
            hipLaunchKernelGGL(fb_gated_peak_kernel, dim3((unsigned)s.n_peaks), dim3(1024), 0, st, s);
            if ((rc = launched("gated peak kernel launch: ")) != FB_OK) return rc;
        }
        if (M > 0) {
            Prepare copies;
            if (dx && g.w.copy) copies.add(pack_job(g.w, weight, ldw, 2 * N, K, wts), type);
            if (dweight && g.x.copy) copies.add(pack_job(g.x, x, ldx, M, K, xs), type);
            if (dweight && g.twice) copies.add(pack_job(g.x, x, ldx, M, K, xs + (size_t)M * (size_t)g.x.ld * type_bytes(type)), type);
            rc = type == FB_TYPE_F32 ? launch_pairs<float>(s, copies, st) : type == FB_TYPE_BF16 ? launch_pairs<bf16>(s, copies, st) : launch_pairs<f16>(s, copies, st);
            if (rc != FB_OK) return rc;
        }
        g.dx.B = {g.w.copy ? wts : weight, g.w.ld, false};
        g.dw.B = {g.x.copy ? xs : x, g.x.ld, false};
        return launch_grad(g, Factor{dz, g.ldz, true}, scale ? undo : nullptr, dx, lddx, dweight, part, sums, M > 0 ? s.down : 0, dbias, st);
    });
}

}  // extern "C"
