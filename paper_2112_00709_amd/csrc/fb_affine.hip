// Affine layer and its gradient (fb_layers.h): the calls, how their products are laid out, and what stands beside the products.
#include "fb_affine.h"

namespace fb {

namespace {

// What is left behind the products: shares of up to two of them added in their order and finished, and the sums of columns
// that fb_prepare_kernel has left a row a workgroup of (16 columns a workgroup, every sixteenth row a thread).
struct JoinParams {
    Product q[2];
    int last[2];             // workgroups [0, last[0]) have q[0], [last[0], last[1]) q[1], the others columns
    const float *sums;
    int64_t rows, N;
    float *out;
};

template <class T>
__global__ __launch_bounds__(256) void fb_join_kernel(JoinParams p)
{
    __shared__ float slots[16][16];
    const int block = blockIdx.x;
    if (block < p.last[1]) {
        const int which = block < p.last[0] ? 0 : 1, first = which ? p.last[0] : 0;
        const Product &q = p.q[which];
        const int64_t n = q.M * q.N;
        float undo = 1.0f;
        if constexpr (sizeof(T) == 2) undo = q.f.undo ? *q.f.undo : 1.0f;
        for (int64_t at = (int64_t)(block - first) * 256 + threadIdx.x; at < n; at += (int64_t)(p.last[which] - first) * 256) {
            float s = 0.0f;
#pragma unroll 8
            for (int c = 0; c < q.split; ++c) s += q.part[(size_t)c * n + at];
            finish_one<T>(q.f, at / q.N, at % q.N, s * undo);
        }
        return;
    }
    const int col = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int64_t c = (int64_t)(block - p.last[1]) * 16 + col;
    float s[4] = {};
    if (c < p.N) {
        int64_t i = g;
        for (; i + 48 < p.rows; i += 64) {
#pragma unroll
            for (int u = 0; u < 4; ++u) s[u] += p.sums[(i + 16 * u) * p.N + c];
        }
        for (; i < p.rows; i += 16) s[0] += p.sums[i * p.N + c];
    }
    slots[g][col] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (g == 0 && c < p.N) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) t += slots[i][col];
        p.out[c] = t;
    }
}

// The largest finite |dy|, as its bits, a share a workgroup.
//
// Half precision holds less than 6e-8 as 0 and more than 65504 as infinity, while a dy in single precision, or one times a slope,
// may be of any size and its products with x and W well inside half precision.  So dz goes into the products times the power of two
// that brings the largest |dy| into [2^14, 2^15) (slopes are at most 1.13), and the sums are taken times its inverse when they leave.
// What the largest exceeds by 2^29 and more loses digits, an error of at most 2^-39 of the largest; infinities and NaN do not
// count.  One more pass over dy, bound by memory, for half precision alone and only where dz has to be rounded: 36 of 529 us for the
// gradient of 44160 x 2048 x 1024 behind a gelu, 65 of 543 with dy in single precision (5 TB/s; 48 and 92 us where dy is new each
// time: with twice or four times the workgroups or the loads asked for ahead 50 and 80 to 92); 2 to 5 us in small ones.
struct PeakParams {
    const void *dy;
    int64_t ld, M, N;
    uint32_t *peaks;
};

template <class D>
__global__ __launch_bounds__(1024) void fb_peak_kernel(PeakParams p)
{
    constexpr int VD = Vec<D>::kN, kAhead = 4;
    __shared__ uint32_t slots[16];
    const int64_t pieces = (p.N + VD - 1) / VD, step = (int64_t)gridDim.x * 1024, down = step / pieces, across = step - down * pieces;
    const int64_t at = (int64_t)blockIdx.x * 1024 + threadIdx.x;
    int64_t r = at / pieces, c = at - r * pieces;
    uint32_t peak = 0;
    while (r < p.M) {
        u32x4 raw[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            raw[u] = load_piece((const D *)p.dy + r * p.ld + c * VD, r < p.M ? (int)(p.N - c * VD) : 0);
            r += down;
            c += across;
            if (c >= pieces) {
                c -= pieces;
                ++r;
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            float v[VD];
            unpack<D>(raw[u], v);
#pragma unroll
            for (int j = 0; j < VD; ++j) {
                const uint32_t a = __float_as_uint(v[j]) & 0x7fffffffu;
                peak = a < 0x7f800000u && a > peak ? a : peak;
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

int64_t peak_groups(int64_t M, int64_t N, int dy_type)
{
    const int64_t vd = 16 / (int64_t)type_bytes(dy_type), pieces = (N + vd - 1) / vd;
    return std::min<int64_t>(kPeakGroups, (M * pieces + 1023) / 1024);
}

int launch_peak(const PeakParams &p, int dy_type, hipStream_t stream)
{
    const dim3 grid((unsigned)peak_groups(p.M, p.N, dy_type)), block(1024);
    if (dy_type == FB_TYPE_F32)
        hipLaunchKernelGGL(fb_peak_kernel<float>, grid, block, 0, stream, p);
    else
        hipLaunchKernelGGL(fb_peak_kernel<f16>, grid, block, 0, stream, p);
    return launched("peak kernel launch: ");
}

template <class T, class D>
__global__ __launch_bounds__(256) void fb_prepare_kernel(PrepareParams p)
{
    __shared__ float slots[256][Vec<T>::kN + 1];
    prepare_block<T, D>(p, blockIdx.x, slots);
}

}  // namespace

void lay_out(SlopeParams &p, int type)
{
    const int64_t ve = 16 / (int64_t)type_bytes(type), pieces = (p.N + ve - 1) / ve;
    for (p.lanes = 1; p.lanes < 64 && p.lanes < pieces;) p.lanes *= 2;
    p.wide = (int)((pieces + p.lanes - 1) / p.lanes);
    const int64_t rows = 256 / p.lanes * kRowsAhead;      // at a time
    p.down = (int)std::max<int64_t>(1, std::min<int64_t>((p.M + rows - 1) / rows, std::max<int64_t>(64, 4 * kCUs / p.wide)));
}

// The shares of sums over M rows of N elements.
int64_t sum_rows(int64_t M, int64_t N, int type)
{
    SlopeParams p{};
    p.M = M;
    p.N = N;
    lay_out(p, type);
    return p.down;
}

// Tiles and shares of k, by estimated clocks of the busiest compute unit: its tiles' work, for every round of workgroups that
// it holds at a time (1, 2 or 4) a start, an end and the latency of every step, and, where k is shared, the sums' way through
// memory and a launch to join them.  In single precision a share is at most 4096 long, so that roundings do not pile up, as long as
// 128 shares are enough for that (k up to 524288); with k above 4096 the sums always go through memory then, split M N floats of it.
double plan(Product &q, int only_tile, bool whole)
{
    static constexpr int kSplits[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64, 96, 128};
    struct Shape {                          // (see fb_mfma.h)
        int tile, resident;
        double per_k16, per_k32;            // clocks of a compute unit on one k of a tile, measured
    };
    static constexpr Shape kShapes[] = {{256, 1, 62.0, 540.0}, {128, 2, 20.0, 140.0}, {64, 4, 9.0, 34.0}};
    constexpr double kEnds = 8000.0, kStep = 500.0, kJoin = 11000.0, kBytesPerClock = 1800.0;
    const bool wide = q.type == FB_TYPE_F32;
    const int64_t deep = wide ? 32 : 64;
    double best = 0.0;
    for (const Shape &sh : kShapes) {
        if (only_tile && sh.tile != only_tile) continue;
        const int64_t tiles = ((q.M + sh.tile - 1) / sh.tile) * ((q.N + sh.tile - 1) / sh.tile);
        for (const int64_t split : kSplits) {
            const int64_t share = std::max<int64_t>(deep, ((q.K + split - 1) / split + deep - 1) / deep * deep);
            if (split > 1 && (whole || (split - 1) * share >= q.K)) break;
            if (wide && share > 4096 && split < 128 && !whole) continue;
            const int64_t busiest = (tiles * split + kCUs - 1) / kCUs, rounds = (busiest + sh.resident - 1) / sh.resident;
            double cost = (double)rounds * (kEnds + (double)(share / deep) * kStep) + (double)busiest * (double)share * (wide ? sh.per_k32 : sh.per_k16);
            if (split > 1) cost += kJoin + (double)(split + 1) * (double)q.M * (double)q.N * 4.0 / kBytesPerClock;
            if (best == 0.0 || cost < best) {
                best = cost;
                q.tile = sh.tile;
                q.share = share;
                q.split = (int)((q.K + share - 1) / share);
            }
        }
    }
    q.split = std::max(q.split, 1);         // (K = 0, a gradient over no rows: sums of nothing)
    q.parts = !whole && (q.split > 1 || q.N < 4);       // (the kernel takes a residual by fours)
    return best;
}

// Tiles of 256 in whole rounds of workgroups, and the rows that would make a last round, which is mostly empty, by tiles that fit them:
// 69120 x 3000 x 1024 in bfloat16 has 1080 tiles for 256 compute units: 421 us, or 354 and 50.
int64_t rows_in_rounds(const Product &q, Product &last)
{
    const int64_t across = (q.N + 255) / 256, tiles = (q.M + 255) / 256 * across, rounds = (tiles + kCUs - 1) / kCUs;
    const int64_t rows = (rounds - 1) * kCUs / across * 256;
    last = q;
    if (q.parts || q.tile != 256 || rounds < 2 || rows <= 0 || rows >= q.M) return 0;
    Product whole = q;
    last.M = q.M - rows;
    whole.M = 256;
    whole.N = 256;
    constexpr double kLaunch = 5000.0;
    return plan(last, 0, true) + kLaunch >= plan(whole, 256, true) || last.tile == 256 ? 0 : rows;
}

int launch_dx(const Product &q, hipStream_t stream)
{
    Product first = q, last;
    const int64_t rows = rows_in_rounds(q, last);
    if (rows == 0) return launch_mfma_product(q, stream);
    first.M = rows;
    const auto skip = [&](const void *p, int64_t ld, int type) { return p ? (const char *)p + (size_t)rows * (size_t)ld * type_bytes(type) : nullptr; };
    last.A.p = skip(q.A.p, q.A.ld, q.type);
    last.f.y = (void *)skip(q.f.y, q.f.ldy, q.f.out_type);
    last.f.residual = skip(q.f.residual, q.f.ldr, q.f.out_type);
    const int rc = launch_mfma_product(first, stream);
    return rc == FB_OK ? launch_mfma_product(last, stream) : rc;
}

// Products whose shares are to be joined (at most two) and columns to be added up (out), in one launch.
int launch_join(const Product *a, const Product *b, int type, const float *sums, int64_t rows, int64_t N, float *out, hipStream_t stream)
{
    JoinParams p{};
    int blocks = 0, k = 0;
    for (const Product *q : {a, b}) {
        if (q && q->parts && q->M > 0) {
            p.q[k] = *q;
            blocks += (int)std::min<int64_t>((q->M * q->N + 255) / 256, 8 * kCUs);
            p.last[k++] = blocks;
        }
    }
    for (; k < 2; ++k) p.last[k] = blocks;
    if (out) {
        p.sums = sums;
        p.rows = rows;
        p.N = N;
        p.out = out;
        blocks += (int)((N + 15) / 16);
    }
    if (blocks == 0) return FB_OK;
    if (type == FB_TYPE_F32)
        hipLaunchKernelGGL(fb_join_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, stream, p);
    else if (type == FB_TYPE_BF16)
        hipLaunchKernelGGL(fb_join_kernel<bf16>, dim3((unsigned)blocks), dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL(fb_join_kernel<f16>, dim3((unsigned)blocks), dim3(256), 0, stream, p);
    return launched("product join kernel launch: ");
}

int launch_prepare(Prepare &j, int type, int dy_type, hipStream_t stream)
{
    if (j.n == 0) return FB_OK;
    for (int i = j.n; i < 3; ++i) j.p.last[i] = j.blocks;
    const dim3 grid((unsigned)j.blocks), block(256);
    if (type == FB_TYPE_F32)
        hipLaunchKernelGGL((fb_prepare_kernel<float, float>), grid, block, 0, stream, j.p);
    else if (type == FB_TYPE_BF16 && dy_type == type)
        hipLaunchKernelGGL((fb_prepare_kernel<bf16, bf16>), grid, block, 0, stream, j.p);
    else if (type == FB_TYPE_BF16)
        hipLaunchKernelGGL((fb_prepare_kernel<bf16, float>), grid, block, 0, stream, j.p);
    else if (dy_type == type)
        hipLaunchKernelGGL((fb_prepare_kernel<f16, f16>), grid, block, 0, stream, j.p);
    else
        hipLaunchKernelGGL((fb_prepare_kernel<f16, float>), grid, block, 0, stream, j.p);
    return launched("row preparation kernel launch: ");
}

namespace {

struct ForwardPlan {
    Product q;
    bool few;             // by launch_few_rows
    Packed x, w;
    size_t bytes;
};

ForwardPlan forward_plan(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N, int64_t K, int type)
{
    ForwardPlan f{};
    f.q.M = M; f.q.N = N; f.q.K = K; f.q.type = type;
    f.few = M <= kFewRows;
    if (f.few) return f;
    plan(f.q);
    f.x = packed(x, ldx, M, K, type);
    f.w = packed(weight, ldw, N, K, type);
    f.bytes = f.x.bytes + f.w.bytes + product_bytes(f.q);
    return f;
}

}  // namespace

// Both products of a gradient; whether they go in one launch: small ones do, by tiles of one size, as each alone would start and end by
// itself.
bool plan_back(Product &dx, Product &dw)
{
    plan(dx);
    plan(dw);
    if (fits_as_pair(dx, dw)) return true;
    if (dx.tile > 128 || dw.tile > 128 || dx.tile == dw.tile) return false;
    Product x = dx, w = dw;
    plan(x, 64);
    plan(w, 64);
    if (!fits_as_pair(x, w)) return false;
    dx = x;
    dw = w;
    return true;
}

GradPlan grad_plan(const void *dy, int64_t lddy, int dy_type, const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N,
                   int64_t K, int type, int act)
{
    GradPlan g{};
    g.dx.M = M; g.dx.N = K; g.dx.K = N; g.dx.type = type;
    g.dw.M = N; g.dw.N = K; g.dw.K = M; g.dw.type = type;
    g.pair = plan_back(g.dx, g.dw);
    g.slope = act != FB_ACT_NONE || dy_type != type || packed(dy, lddy, M, N, type).copy;
    g.scale = type == FB_TYPE_F16 && (dy_type != type || act > FB_ACT_RELU);
    g.ldz = line_distance(N, type);
    g.dz = g.slope ? aligned((size_t)M * (size_t)g.ldz * type_bytes(type)) : 0;
    g.x = packed(x, ldx, M, K, type);
    g.w = packed(weight, ldw, N, K, type);
    g.sums = aligned((size_t)sum_rows(M, N, type) * (size_t)N * sizeof(float));
    g.range = g.scale ? aligned((kPeakGroups + 1) * sizeof(float)) : 0;
    g.part = product_bytes(g.dx);
    g.bytes = g.dz + g.x.bytes + g.w.bytes + g.sums + g.range + g.part + product_bytes(g.dw);
    return g;
}

// dx = dz W and dweight = dz^T x, whose second factors are set, and what is left behind them; the sums of dz's columns are in `sums`.
int launch_grad(GradPlan &g, const Factor &d, const float *undo, void *dx, int64_t lddx, void *dweight, float *part, const float *sums, int64_t rows, float *dbias,
                hipStream_t st)
{
    const int64_t M = g.dx.M, N = g.dw.M, K = g.dx.N;
    const int type = g.dx.type;
    int rc;
    g.dx.A = d;
    g.dx.f.y = dx; g.dx.f.ldy = lddx; g.dx.f.out_type = type;
    g.dx.f.undo = g.dw.f.undo = undo;
    g.dx.part = part;
    g.dw.A = {d.p, d.ld, false};
    g.dw.f.y = dweight; g.dw.f.ldy = K; g.dw.f.out_type = type;
    g.dw.part = (float *)((char *)part + g.part);
    if (dx && dweight && g.pair) {
        if ((rc = launch_mfma_pair(g.dx, g.dw, st)) != FB_OK) return rc;
    } else {
        if (dx && M > 0 && (rc = launch_dx(g.dx, st)) != FB_OK) return rc;
        if (dweight && (rc = launch_mfma_product(g.dw, st)) != FB_OK) return rc;
    }
    const Product joined = joined_rows(g.dx, g.twice);
    return launch_join(dx ? &joined : nullptr, dweight ? &g.dw : nullptr, type, sums, rows, N, dbias, st);
}

namespace {

int check_affine(const char *who, const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N, int64_t K, int type, int act)
{
    const std::string w(who);
    if (!known_type(type)) return fail(FB_EINVAL, w + ": unknown type");
    if (act < FB_ACT_NONE || act > FB_ACT_SILU) return fail(FB_EINVAL, w + ": unknown activation");
    if (bad_sizes(M, N, K)) return fail(FB_EINVAL, w + ": M must be 0 or more, N and K 1 or more, all below 2^31");
    if ((!x && M > 0) || !weight) return fail(FB_EINVAL, w + ": x or weight is NULL");
    if (bad_ld(ldx, K) || bad_ld(ldw, K)) return fail(FB_EINVAL, w + ": rows of x or weight closer than K elements");
    return FB_OK;
}

}  // namespace

}  // namespace fb

extern "C" {

size_t fb_affine_workspace_bytes(const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M, int64_t N, int64_t K, int type)
{
    using namespace fb;
    if (bad_sizes(M, N, K) || !known_type(type)) return 0;
    return forward_plan(x, ldx, weight, ldw, M, N, K, type).bytes;
}

int fb_affine(const void *x, int64_t ldx, const void *weight, int64_t ldw, const float *bias, const void *residual, int64_t ldr,
              int64_t M, int64_t N, int64_t K, int type, int act, void *y, int64_t ldy, int out_type, void *preact, int64_t ldp,
              void *ws, size_t ws_bytes, fb_stream stream)
{
    using namespace fb;
    return guarded([&]() -> int {
        int rc = check_affine("fb_affine", x, ldx, weight, ldw, M, N, K, type, act);
        if (rc != FB_OK) return rc;
        if (out_type != type && out_type != FB_TYPE_F32) return fail(FB_EINVAL, "fb_affine: the output's type is neither float nor the factors'");
        if (!y && M > 0) return fail(FB_EINVAL, "fb_affine: y is NULL");
        if (bad_ld(ldy, N) || (residual && bad_ld(ldr, N)) || (preact && bad_ld(ldp, N))) return fail(FB_EINVAL, "fb_affine: rows closer than N elements");
        if (M > kFewRows ? too_long(K, type) || too_far(ldy) || (residual && too_far(ldr)) || (preact && too_far(ldp)) : N >= (int64_t)1 << 26)
            return fail(FB_EUNSUPPORTED, "fb_affine: rows of x and weight longer than 4 MB, rows of y, residual or preact 2^27 elements apart, or (M <= 64) N of 2^26 and more");
        const ForwardPlan f = forward_plan(x, ldx, weight, ldw, M, N, K, type);
        if (f.bytes && (!ws || ws_bytes < f.bytes)) return fail(FB_EINVAL, "fb_affine: workspace missing or too small");
        hipStream_t st = (hipStream_t)stream;
        char *xs = (char *)ws, *wts = xs + f.x.bytes;
        Product q = f.q;
        q.f = {bias, residual, ldr, act, y, ldy, out_type, preact, ldp, nullptr};
        if (f.few) {
            q.A = {x, ldx, true};
            q.B = {weight, ldw, true};
            return M > 0 ? launch_few_rows(q, st) : FB_OK;
        }
        if (M == 0) return FB_OK;
        Prepare jobs;
        if (f.x.copy) jobs.add(pack_job(f.x, x, ldx, M, K, xs), type);
        if (f.w.copy) jobs.add(pack_job(f.w, weight, ldw, N, K, wts), type);
        if ((rc = launch_prepare(jobs, type, type, st)) != FB_OK) return rc;
        q.A = {f.x.copy ? xs : x, f.x.ld, true};
        q.B = {f.w.copy ? wts : weight, f.w.ld, true};
        q.part = (float *)(wts + f.w.bytes);
        if ((rc = launch_mfma_product(q, st)) != FB_OK) return rc;
        return launch_join(&q, nullptr, type, nullptr, 0, 0, nullptr, st);
    });
}

size_t fb_affine_grad_workspace_bytes(const void *dy, int64_t lddy, int dy_type, const void *x, int64_t ldx, const void *weight, int64_t ldw, int64_t M,
                                      int64_t N, int64_t K, int type, int act)
{
    using namespace fb;
    if (bad_sizes(M, N, K) || !known_type(type) || (dy_type != type && dy_type != FB_TYPE_F32) || act < FB_ACT_NONE || act > FB_ACT_SILU) return 0;
    return grad_plan(dy, lddy, dy_type, x, ldx, weight, ldw, M, N, K, type, act).bytes;
}

int fb_affine_grad(const void *dy, int64_t lddy, int dy_type, const void *x, int64_t ldx, const void *weight, int64_t ldw,
                   const void *preact, int64_t ldp, int64_t M, int64_t N, int64_t K, int type, int act, void *dx, int64_t lddx,
                   void *dweight, float *dbias, void *ws, size_t ws_bytes, fb_stream stream)
{
    using namespace fb;
    return guarded([&]() -> int {
        int rc = check_affine("fb_affine_grad", x, ldx, weight, ldw, M, N, K, type, act);
        if (rc != FB_OK) return rc;
        if (dy_type != type && dy_type != FB_TYPE_F32) return fail(FB_EINVAL, "fb_affine_grad: the type of dy is neither float nor the factors'");
        if (!dy && M > 0) return fail(FB_EINVAL, "fb_affine_grad: dy is NULL");
        if (act != FB_ACT_NONE && !preact && M > 0) return fail(FB_EINVAL, "fb_affine_grad: this activation needs preact");
        if (bad_ld(lddy, N) || (act != FB_ACT_NONE && bad_ld(ldp, N)) || (dx && bad_ld(lddx, K))) return fail(FB_EINVAL, "fb_affine_grad: rows closer than their width");
        if (!dx && !dweight && !dbias) return FB_OK;
        if (too_long(K, type) || too_long(N, type) || (dx && too_far(lddx)))
            return fail(FB_EUNSUPPORTED, "fb_affine_grad: rows of x, weight and dy longer than 4 MB, or rows of dx 2^27 elements apart");
        GradPlan g = grad_plan(dy, lddy, dy_type, x, ldx, weight, ldw, M, N, K, type, act);
        if (!ws || ws_bytes < g.bytes) return fail(FB_EINVAL, "fb_affine_grad: workspace missing or too small");
        hipStream_t st = (hipStream_t)stream;
        char *dz = (char *)ws, *xs = dz + g.dz, *wts = xs + g.x.bytes;
        float *sums = (float *)(wts + g.w.bytes), *undo = (float *)(wts + g.w.bytes + g.sums);
        float *part = (float *)((char *)undo + g.range);
        const bool make = g.slope && (dx || dweight), scale = make && g.scale && M > 0;
        uint32_t *peaks = scale ? (uint32_t *)(undo + 1) : nullptr;
        if (scale && (rc = launch_peak(PeakParams{dy, lddy, M, N, peaks}, dy_type, st)) != FB_OK) return rc;
        Prepare jobs;                                             // (the first may have rows of another type: dy's)
        if (M > 0 && (make || dbias))
            jobs.add(SlopeParams{dy, preact, lddy, ldp, M, N, g.ldz, act, make ? dz : nullptr, dbias ? sums : nullptr, 0, 0, 0,
                                 peaks, scale ? (int)peak_groups(M, N, dy_type) : 0, undo},
                     type);
        else
            jobs.p.last[jobs.n++] = 0;
        if (M > 0 && dx && g.w.copy) jobs.add(pack_job(g.w, weight, ldw, N, K, wts), type);
        if (M > 0 && dweight && g.x.copy) jobs.add(pack_job(g.x, x, ldx, M, K, xs), type);
        if (jobs.blocks > 0 && (rc = launch_prepare(jobs, type, dy_type, st)) != FB_OK) return rc;
        const Factor d{make ? (const void *)dz : dy, make ? g.ldz : lddy, true};
        g.dx.B = {g.w.copy ? wts : weight, g.w.ld, false};
        g.dw.B = {g.x.copy ? xs : x, g.x.ld, false};
        return launch_grad(g, d, scale ? undo : nullptr, dx, lddx, dweight, part, sums, M > 0 ? sum_rows(M, N, type) : 0, dbias, st);
    });
}

}  // extern "C"
