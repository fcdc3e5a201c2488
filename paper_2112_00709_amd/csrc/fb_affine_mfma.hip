// Products of 16-bit factors on the matrix units (see fb_affine.h), for factors whose rows are whole 16-byte pieces.
//
// A workgroup forms a tile of C, 64 k at a time.  Both factors' shares of those k come into LDS by direct copies (16 bytes a
// lane, no registers in between), into one of two buffers while the other is worked on; a wave reads its 32-row fragments of
// 16 k from LDS one step ahead of the matrix instructions that use them.  A factor that runs along k is kept as [row][k], one
// that does not as [k][row] and is read by the transposing LDS read, so no factor is ever transposed in memory.
//
// LDS banks.  [row][64 k]: the 16-byte piece c of a row lies at piece c ^ (row & 7), so eight rows read at one c cover all
// banks.  [k][rows]: piece c of a k lies at c ^ ((k & 3) << 1): the four k that a transposing read takes at once lie in
// different quarters of the banks.  The copies write LDS in order of lanes, so the exchange is in the address a lane reads.
#include "fb_affine.h"

#ifndef FB_WI
#define FB_WI 2
#define FB_WJ 4
#define FB_FI 4
#define FB_FJ 2
#endif

namespace fb {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kDeep = 64;          // k of a step between barriers

template <class T>
__device__ __forceinline__ f32x16 multiply(const u32x4 &a, const u32x4 &b, const f32x16 &c)
{
    if constexpr (std::is_same<T, bf16>::value)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ u32x4 lds_read(uint32_t at) { return *(const __attribute__((address_space(3))) u32x4 *)(uintptr_t)at; }
__device__ __forceinline__ u32x2 lds_read_across(uint32_t at)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(uintptr_t)at));
}

// 16 bytes a lane from a buffer to LDS, lane by lane from `to` on; zeros where the address is past the buffer's end.
__device__ __forceinline__ void copy_to_lds(uint32_t to, uint32_t offset, const i32x4 &buffer)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(buffer) : "memory");
}

// One factor's way into LDS and out of it.  ROWS of the tile, NW waves that copy, F fragments of 32 rows a wave from row w0 on.
template <bool ALONG, int ROWS, int NW, int F>
struct Side {
    static constexpr int kBytes = ROWS * kDeep * 2, kCopies = kBytes / 1024 / NW;
    uint64_t base;           // of the tile's first element at the share's first k
    uint32_t ld2;            // bytes between rows
    int rows;                // rows of the factor from the tile's first on
    uint32_t from[2];        // a lane's offset in what a copy brings (two: even and odd copies)
    uint32_t lds;            // the first buffer
    uint32_t at[ALONG ? 4 : 2];
    int chunk;               // ALONG: a lane's piece along k

    __device__ __forceinline__ void start(const Factor &f, int64_t r0, int64_t n, int64_t k0, uint32_t lds_at, int wave, int w0)
    {
        const int lane = threadIdx.x & 63;
        ld2 = (uint32_t)f.ld * 2;
        rows = (int)(n - r0 < ROWS ? n - r0 : ROWS);
        base = (uint64_t)(uintptr_t)f.p + (uint64_t)(ALONG ? r0 * f.ld + k0 : k0 * f.ld + r0) * 2;
        lds = lds_at;
        const int l = lane & 31, h = lane >> 5;
        if constexpr (ALONG) {
            chunk = (lane & 7) ^ (lane >> 3);
            from[0] = from[1] = (uint32_t)(wave * kCopies * 8 + (lane >> 3)) * ld2 + chunk * 16;
#pragma unroll
            for (int s = 0; s < 4; ++s) at[s] = lds + (w0 + l) * 128 + (((s * 2 + h) ^ (l & 7)) * 16);
        } else {
            constexpr int kPer = ROWS / 8, kK = 64 / kPer;          // lanes a k, k a copy
            const int k = lane / kPer, p = lane % kPer;
            chunk = 0;
#pragma unroll
            for (int odd = 0; odd < 2; ++odd)
                from[odd] = (uint32_t)(wave * kCopies * kK + k) * ld2 + ((p ^ (((odd * kK + k) & 3) << 1)) * 16);
            const int g = lane >> 4, kq = (lane & 15) >> 2, c = (g & 1) * 2 + ((lane & 3) >> 1);
#pragma unroll
            for (int odd = 0; odd < 2; ++odd)
                at[odd] = lds + ((g >> 1) * 8 + kq) * (ROWS * 2) + w0 * 2 + (((c + odd * 4) ^ (kq << 1)) * 16) + (lane & 1) * 8;
        }
    }

    // The factor's share of the next 64 of `left` k, into buffer `b`.
    __device__ __forceinline__ void copy(int64_t left, int b, int wave)
    {
        i32x4 buffer;
        uint32_t bytes, past = 0;
        if constexpr (ALONG) {
            bytes = (uint32_t)(rows - 1) * ld2 + (uint32_t)(left < kDeep ? (left + 7) & ~7 : kDeep) * 2;   // (whole pieces)
            past = chunk * 8 < left ? 0u : 0x80000000u;                // (`bytes` is below 2^31)
        } else {
            bytes = (uint32_t)((left < kDeep ? left : kDeep) - 1) * ld2 + (uint32_t)((rows + 7) & ~7) * 2;
        }
        buffer[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)base);
        buffer[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32) & 0xffff);
        buffer[2] = __builtin_amdgcn_readfirstlane((int)bytes);
        buffer[3] = 0x00020000;
        const uint32_t to = lds + b * kBytes + wave * kCopies * 1024;
        constexpr int kStep = ALONG ? 8 : 64 / (ROWS / 8);
#pragma unroll
        for (int u = 0; u < kCopies; ++u)
            copy_to_lds(__builtin_amdgcn_readfirstlane(to + u * 1024), from[u & 1] + (uint32_t)(u * kStep) * ld2 + past, buffer);
        base += ALONG ? kDeep * 2 : (uint64_t)kDeep * ld2;
    }

    // Fragment f of step s (16 k) from buffer `b`: row lane % 32, k = 8 (lane / 32) + 0 .. 7.
    __device__ __forceinline__ u32x4 read(int b, int s, int f) const
    {
        if constexpr (ALONG) {
            return lds_read(at[s] + b * kBytes + f * 32 * 128);
        } else {
            const uint32_t a = at[f & 1] + b * kBytes + s * 16 * (ROWS * 2) + (f >> 1) * 128;
            const u32x2 lo = lds_read_across(a), hi = lds_read_across(a + 4 * (ROWS * 2));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }
};

// Four neighbouring sums of a row finished and stored; n of them exist.
template <class T>
__device__ __forceinline__ void finish_four(const Finish &f, int64_t i, int64_t j, int n, const f32x4 &sums, const f32x4 &bias)
{
    float s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = sums[e] + bias[e];
    auto put = [&](T *to) {
        const u32x2 v = {pack2<T>(s[0], s[1]), pack2<T>(s[2], s[3])};
        if (n == 4) {
            typedef u32x2 u32x2_any __attribute__((aligned(2)));
            *(u32x2_any *)to = v;
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < n) to[e] = (T)s[e];
        }
    };
    if (f.preact) put((T *)f.preact + i * f.ldp + j);
    if (f.act != FB_ACT_NONE) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = act_of(s[e], f.act);
    }
    if (f.out_type == FB_TYPE_F32) {
        typedef f32x4 f32x4_any __attribute__((aligned(4)));
        float *to = (float *)f.y + i * f.ldy + j;
        const float *from = (const float *)f.residual + i * f.ldr + j;
        if (n == 4) {
            f32x4 v = {s[0], s[1], s[2], s[3]};
            if (f.residual) v += *(const f32x4_any *)from;
            *(f32x4_any *)to = v;
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < n) to[e] = s[e] + (f.residual ? from[e] : 0.0f);
        }
    } else {
        if (f.residual) {
            const T *from = (const T *)f.residual + i * f.ldr + j;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < n) s[e] += (float)from[e];
        }
        put((T *)f.y + i * f.ldy + j);
    }
}

template <class T, bool ALONG_A, bool ALONG_B, int WI, int WJ, int FI, int FJ>
__global__ __launch_bounds__(WI * WJ * 64) void fb_mfma_product_kernel(Product q, int tiles_i, int tiles_j)
{
    constexpr int kI = WI * FI * 32, kJ = WJ * FJ * 32, kNW = WI * WJ;
    extern __shared__ char lds_raw[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds_raw;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wi = wave / WJ, wj = wave % WJ;

    // Workgroups go to the eight chiplets in turn: each chiplet gets a run of neighbouring tiles, so that its L2 holds what
    // they share; within a run eight tiles down, then one across.
    const int n = tiles_i * tiles_j * q.split, xcd = blockIdx.x % 8, in_xcd = blockIdx.x / 8;
    const int t = xcd * (n / 8) + (xcd < n % 8 ? xcd : n % 8) + in_xcd;
    const int share = t / (tiles_i * tiles_j), u = t - share * tiles_i * tiles_j;
    const int group = u / (8 * tiles_j), first = group * 8, down = tiles_i - first < 8 ? tiles_i - first : 8;
    const int v = u - group * 8 * tiles_j;
    const int64_t i0 = (int64_t)(first + v % down) * kI, j0 = (int64_t)(v / down) * kJ;
    const int64_t k0 = (int64_t)share * q.share, k1 = k0 + q.share < q.K ? k0 + q.share : q.K;
    const int steps = (int)((k1 - k0 + kDeep - 1) / kDeep);

    Side<ALONG_A, kI, kNW, FI> a;
    Side<ALONG_B, kJ, kNW, FJ> b;
    a.start(q.A, i0, q.M, k0, lds0, wave, wi * FI * 32);
    b.start(q.B, j0, q.N, k0, lds0 + 2 * a.kBytes, wave, wj * FJ * 32);

    f32x16 acc[FI][FJ] = {};
    u32x4 fa[2][FI], fb_[2][FJ];
    auto bring = [&](int step) {
        const int64_t left = k1 - k0 - (int64_t)step * kDeep;
        a.copy(left, step & 1, wave);
        b.copy(left, step & 1, wave);
    };
    auto read = [&](int buffer, int s, int set) {
#pragma unroll
        for (int f = 0; f < FI; ++f) fa[set][f] = a.read(buffer, s, f);
#pragma unroll
        for (int f = 0; f < FJ; ++f) fb_[set][f] = b.read(buffer, s, f);
    };
    // What has been asked for has come, in every wave; and every wave has read what it wanted of the other buffer.
    auto meet = [&]() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
    if (steps > 0) {
        bring(0);
        meet();
        if (steps > 1) bring(1);
        read(0, 0, 0);
    }
    for (int step = 0; step < steps; ++step) {
        const int cur = step & 1;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s < 3) {
                read(cur, s + 1, (s + 1) & 1);
            } else if (step + 1 < steps) {
                meet();
                if (step + 2 < steps) bring(step + 2);
                read(cur ^ 1, 0, 0);
            }
#pragma unroll
            for (int x = 0; x < FI; ++x)
#pragma unroll
                for (int y = 0; y < FJ; ++y) acc[x][y] = multiply<T>(fb_[s & 1][y], fa[s & 1][x], acc[x][y]);
        }
    }

    // The sums pass through LDS, 32 rows of C at a time and each wave in a region of its own, so that whole runs of a row are
    // stored: a lane's own are 4 neighbours of 4 rows 8 apart in every 32 columns.
    constexpr int kLd = FJ * 32 + 4, kPer = FJ * 8, kRows = 64 / kPer;
    __syncthreads();
    float *mine = (float *)lds_raw + wave * 32 * kLd;
    const int64_t j = j0 + wj * FJ * 32 + (lane % kPer) * 4;
    const int nj = (int)(q.N - j < 4 ? (q.N - j < 0 ? 0 : q.N - j) : 4);
    f32x4 bias = {};
    if (q.split == 1 && q.f.bias) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < nj) bias[e] = q.f.bias[j + e];
    }
#pragma unroll
    for (int x = 0; x < FI; ++x) {
#pragma unroll
        for (int y = 0; y < FJ; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x4 w = {acc[x][y][4 * e], acc[x][y][4 * e + 1], acc[x][y][4 * e + 2], acc[x][y][4 * e + 3]};
                *(f32x4 *)(mine + (lane & 31) * kLd + y * 32 + 8 * e + 4 * (lane >> 5)) = w;
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 4
        for (int r = 0; r < 32; r += kRows) {
            const int row = r + lane / kPer;
            const f32x4 w = *(const f32x4 *)(mine + row * kLd + (lane % kPer) * 4);
            const int64_t i = i0 + wi * FI * 32 + x * 32 + row;
            if (i < q.M && nj > 0) {
                if (q.split > 1) {
                    typedef f32x4 f32x4_any __attribute__((aligned(4)));
                    float *to = q.part + ((size_t)share * q.M + i) * q.N + j;
                    if (nj == 4) {
                        *(f32x4_any *)to = w;
                    } else {
#pragma unroll
                        for (int e = 0; e < 3; ++e)
                            if (e < nj) to[e] = w[e];
                    }
                } else {
                    finish_four<T>(q.f, i, j, nj, w, bias);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

template <class T, bool ALONG_A, bool ALONG_B, int WI, int WJ, int FI, int FJ>
int launch(const Product &q, hipStream_t stream)
{
    constexpr int kI = WI * FI * 32, kJ = WJ * FJ * 32;
    const int64_t ti = (q.M + kI - 1) / kI, tj = (q.N + kJ - 1) / kJ;
    if (ti * tj * q.split >= kMostSize) return fail(FB_EUNSUPPORTED, "affine product: more than 2^31 tiles");
    constexpr size_t copies = (size_t)2 * (kI + kJ) * kDeep * 2, sums = (size_t)WI * WJ * 32 * (FJ * 32 + 4) * 4;
    constexpr size_t bytes = copies > sums ? copies : sums;
    const void *k = (const void *)fb_mfma_product_kernel<T, ALONG_A, ALONG_B, WI, WJ, FI, FJ>;
    if (bytes > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != hipSuccess) return fail(FB_EHIP, std::string("hipFuncSetAttribute(LDS size): ") + hipGetErrorString(e));
    }
    hipLaunchKernelGGL((fb_mfma_product_kernel<T, ALONG_A, ALONG_B, WI, WJ, FI, FJ>), dim3((unsigned)(ti * tj * q.split)), dim3(WI * WJ * 64), bytes,
                       stream, q, (int)ti, (int)tj);
    return launched("matrix product kernel launch: ");
}

template <class T, bool ALONG_A, bool ALONG_B>
int launch(const Product &q, hipStream_t stream)
{
    return q.tile == 256 ? launch<T, ALONG_A, ALONG_B, FB_WI, FB_WJ, FB_FI, FB_FJ>(q, stream) : launch<T, ALONG_A, ALONG_B, 2, 2, 2, 2>(q, stream);
}

template <class T>
int launch(const Product &q, hipStream_t stream)
{
    if (q.A.along && q.B.along) return launch<T, true, true>(q, stream);
    if (q.A.along) return launch<T, true, false>(q, stream);
    return launch<T, false, false>(q, stream);
}

}  // namespace

int launch_mfma_product(const Product &q, hipStream_t stream)
{
    return q.type == FB_TYPE_BF16 ? launch<bf16>(q, stream) : launch<f16>(q, stream);
}

}  // namespace fb
