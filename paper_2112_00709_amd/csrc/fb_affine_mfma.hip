// The affine operator's products on the matrix units: one at a time, or both of a small gradient in one launch (see fb_mfma.h).
#include "fb_mfma.h"

namespace fb {

namespace {

// Both products of a gradient, dx by the first `blocks` workgroups and dW by the others: small ones fill the GPU together.
template <class T, int WI, int WJ, int FI, int FJ, bool MASKED>
__global__ __launch_bounds__(WI * WJ * 64) void fb_mfma_pair_kernel(Task dx, Task dw, int blocks)
{
    const __attribute__((address_space(4))) char *args = (const __attribute__((address_space(4))) char *)__builtin_amdgcn_kernarg_segment_ptr();
    if ((int)blockIdx.x < blocks)
        run_tiles<T, true, false, WI, WJ, FI, FJ, Finished<kPlain>>(dx, (ProductArgs)args, blockIdx.x, blocks);
    else
        run_tiles<T, false, false, WI, WJ, FI, FJ, Finished<kPlain>, MASKED>(dw, (ProductArgs)(args + sizeof(Task)), blockIdx.x - blocks, gridDim.x - blocks);
}

template <class T, int WI, int WJ, int FI, int FJ, bool MASKED>
int launch_pair(const Product &dx, const Product &dw, hipStream_t stream)
{
    typedef Shape<WI, WJ, FI, FJ> S;
    const int64_t first = blocks_of<S>(dx);
    const auto kernel = fb_mfma_pair_kernel<T, WI, WJ, FI, FJ, MASKED>;
    const int rc = take_lds<S>(kernel);
    if (rc != FB_OK) return rc;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(first + blocks_of<S>(dw))), dim3(WI * WJ * 64), S::kBytes, stream, task_of<S>(dx), task_of<S>(dw), (int)first);
    return launched("matrix product kernel launch: ");
}

template <class T, bool MASKED>
int launch_pair(const Product &dx, const Product &dw, hipStream_t stream)
{
    return dx.tile == 128 ? launch_pair<T, 2, 2, 2, 2, MASKED>(dx, dw, stream) : launch_pair<T, 2, 2, 1, 1, MASKED>(dx, dw, stream);
}

template <class T>
int launch_pair(const Product &dx, const Product &dw, hipStream_t stream)
{
    return dw.s.live ? launch_pair<T, true>(dx, dw, stream) : launch_pair<T, false>(dx, dw, stream);
}

template <class T, bool ALONG_A, bool ALONG_B, class WAY, bool MASKED = false>
int launch_way(const Product &q, hipStream_t stream)
{
    if (q.tile == 256) return launch<T, ALONG_A, ALONG_B, 2, 4, 4, 2, WAY, MASKED>(q, stream);
    return q.tile == 128 ? launch<T, ALONG_A, ALONG_B, 2, 2, 2, 2, WAY, MASKED>(q, stream) : launch<T, ALONG_A, ALONG_B, 2, 2, 1, 1, WAY, MASKED>(q, stream);
}

template <class T, bool ALONG_A, bool ALONG_B, int KIND>
int launch(const Product &q, hipStream_t stream)
{
    return launch_way<T, ALONG_A, ALONG_B, Finished<KIND>>(q, stream);
}

// Products of a gradient: no bias, no activation.
template <class T, bool ALONG_A>
int launch_back(const Product &q, hipStream_t stream)
{
    if constexpr (ALONG_A) {
        if (q.f.residual && !q.parts) return launch<T, true, false, FB_ACT_NONE>(q, stream);      // (dx in pieces)
    }
    if constexpr (sizeof(T) == 2) {
        if (!q.parts && q.f.out_type == q.type) return launch_way<T, ALONG_A, false, Rounded>(q, stream);
    }
    return launch<T, ALONG_A, false, kPlain>(q, stream);
}

// dW where some rows do not count.
template <class T>
int launch_masked(const Product &q, hipStream_t stream)
{
    if constexpr (sizeof(T) == 2) {
        if (!q.parts && q.f.out_type == q.type) return launch_way<T, false, false, Rounded, true>(q, stream);
    }
    return launch_way<T, false, false, Finished<kPlain>, true>(q, stream);
}

template <class T>
int launch(const Product &q, hipStream_t stream)
{
    if (!q.A.along) return q.s.live ? launch_masked<T>(q, stream) : launch_back<T, false>(q, stream);
    if (!q.B.along) return launch_back<T, true>(q, stream);
    if (q.parts || (q.f.act <= FB_ACT_RELU && !q.f.residual && !q.f.preact)) return launch<T, true, true, kPlain>(q, stream);
    switch (q.f.act) {
    case FB_ACT_NONE: return launch<T, true, true, FB_ACT_NONE>(q, stream);
    case FB_ACT_RELU: return launch<T, true, true, FB_ACT_RELU>(q, stream);
    case FB_ACT_GELU: return launch<T, true, true, FB_ACT_GELU>(q, stream);
    default: return launch<T, true, true, FB_ACT_SILU>(q, stream);
    }
}

}  // namespace

bool fits_as_pair(const Product &dx, const Product &dw)
{
    // (beyond what the GPU holds at a time they are slower together: 9600 x 84 x 512 in single precision 50 instead of 39 us)
    if (dx.tile != dw.tile || dx.tile > 128 || dx.M == 0 || dw.K == 0) return false;
    if (dx.tile == 128) return blocks_of<Shape<2, 2, 2, 2>>(dx) + blocks_of<Shape<2, 2, 2, 2>>(dw) <= Shape<2, 2, 2, 2>::kSlots;
    return blocks_of<Shape<2, 2, 1, 1>>(dx) + blocks_of<Shape<2, 2, 1, 1>>(dw) <= Shape<2, 2, 1, 1>::kSlots;
}

int launch_mfma_pair(const Product &dx, const Product &dw, hipStream_t stream)
{
    if (dx.type == FB_TYPE_F32) return launch_pair<float>(dx, dw, stream);
    return dx.type == FB_TYPE_BF16 ? launch_pair<bf16>(dx, dw, stream) : launch_pair<f16>(dx, dw, stream);
}

int launch_mfma_product(const Product &q, hipStream_t stream)
{
    if (q.type == FB_TYPE_F32) return launch<float>(q, stream);
    return q.type == FB_TYPE_BF16 ? launch<bf16>(q, stream) : launch<f16>(q, stream);
}

}  // namespace fb
