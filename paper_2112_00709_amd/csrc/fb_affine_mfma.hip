// Products on the matrix units (see fb_affine.h), for factors whose rows are whole 16-byte pieces.
//
// A workgroup forms a tile of C, 128 bytes along k at a time: 64 k of 16 bits, 32 of 32.  Both factors' shares of those k
// come into LDS by direct copies (16 bytes a lane, no registers in between), into one of two buffers while the other is worked
// on; a wave reads its 32-row fragments of 32 bytes along k from LDS one step ahead of the matrix instructions that use them.
// A factor that runs along k is kept as [row][k], one that does not as [k][row] and is read by the transposing LDS read (32
// bits: by single words), so no factor is ever transposed in memory.  Of 32 bytes along k a lane of the lower half has the
// first 16 and a lane of the upper half the others: in single precision, whose instruction takes 2 k, the four k of the one
// are multiplied beside those of the other.
//
// LDS banks.  [row][k]: the 16-byte piece c of a row lies at piece c ^ (row & 7), so eight rows read at one c share no bank
// of 32.  [k][rows] of 16 bits: piece c of a k lies at c ^ ((k & 3) << 1): the four k that a transposing read takes at once
// lie in different quarters of those.  The copies write LDS in order of lanes, so the exchange is in the address a lane reads.
// There are 64 banks, and the counters say that half of the passes are conflicts.  An exchange over all 64 (row >> 1 instead of
// row, k << 2 instead of k << 1) has none, and LDS is busy 26 % of the time instead of 43 %; the times stayed what they are
// (8192 cubed 875 and 875 us, 69120 x 3000 x 1024 446 and 446), for two more registers: LDS is not what bounds this.
//
// Measured, bfloat16: 8192 cubed 840 us forward (1310 TFLOP/s; the library's product on the same card 1376), 836 for dx, 816
// for dW (the library 1211 and 1069).  69120 x 3000 x 1024: 435 us, 471 with single-precision output (library, bfloat16 output:
// 483); of these some 370 are the products and the rest the sums' way out, which nothing overlaps: workgroups do it at the
// same time, and with one workgroup a compute unit (128 of 160 KB of LDS) a unit's matrix cores wait meanwhile.  Tiles of 128
// in two workgroups a unit overlap it but read LDS more: 534 us.  Four waves of 128 x 128 instead of eight of 128 x 64: the
// same at 8192 cubed, 460 instead of 438 here.  Single precision: 4096 cubed 966 us (142 TFLOP/s; library 912).
#include "fb_affine.h"

namespace fb {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));

template <class T>
constexpr int kDeepOf = 128 / (int)sizeof(T);          // k of a step between barriers

template <class T>
__device__ __forceinline__ f32x16 multiply(const u32x4 &a, const u32x4 &b, const f32x16 &c)
{
    if constexpr (sizeof(T) == 4) {
        f32x16 d = c;
#pragma unroll
        for (int e = 0; e < 4; ++e) d = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), d, 0, 0, 0);
        return d;
    } else if constexpr (std::is_same<T, bf16>::value)
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
template <class T, bool ALONG, int ROWS, int NW, int F>
struct Side {
    static constexpr int kSize = sizeof(T), kDeep = kDeepOf<T>, kPiece = 16 / kSize;
    static constexpr int kBytes = ROWS * 128, kCopies = kBytes / 1024 / NW;
    static constexpr int kPer = ROWS * kSize / 16, kK = 64 / kPer;      // not ALONG: lanes a k, k a copy
    uint64_t base;           // of the tile's first element at the share's first k
    uint32_t ldb;            // bytes between rows
    int rows;                // rows of the factor from the tile's first on
    uint32_t from[2];        // a lane's offset in what a copy brings (two: even and odd copies)
    uint32_t lds;            // the first buffer
    uint32_t at[ALONG ? 4 : 2];
    int chunk;               // ALONG: a lane's piece along k

    // What does not depend on the tile.
    __device__ __forceinline__ void start(const Factor &f, uint32_t lds_at, int wave, int w0)
    {
        const int lane = threadIdx.x & 63;
        ldb = (uint32_t)f.ld * kSize;
        lds = lds_at;
        const int l = lane & 31, h = lane >> 5;
        if constexpr (ALONG) {
            chunk = (lane & 7) ^ (lane >> 3);
            from[0] = from[1] = (uint32_t)(wave * kCopies * 8 + (lane >> 3)) * ldb + chunk * 16;
#pragma unroll
            for (int s = 0; s < 4; ++s) at[s] = lds + (w0 + l) * 128 + (((s * 2 + h) ^ (l & 7)) * 16);
        } else {
            const int k = lane / kPer, p = lane % kPer;
            chunk = 0;
#pragma unroll
            for (int odd = 0; odd < 2; ++odd)
                from[odd] = (uint32_t)(wave * kCopies * kK + k) * ldb + (kSize == 4 ? p : p ^ (((odd * kK + k) & 3) << 1)) * 16;
            if constexpr (kSize == 4) {
                at[0] = at[1] = lds + (h * 4 * ROWS + w0 + l) * 4;
                return;
            }
            const int g = lane >> 4, kq = (lane & 15) >> 2, c = (g & 1) * 2 + ((lane & 3) >> 1);
#pragma unroll
            for (int odd = 0; odd < 2; ++odd)
                at[odd] = lds + ((g >> 1) * 8 + kq) * (ROWS * 2) + (((w0 / 8 + c + odd * 4) ^ (kq << 1)) * 16) + (lane & 1) * 8;
        }
    }

    __device__ __forceinline__ void tile(const Factor &f, int64_t r0, int64_t n, int64_t k0)
    {
        rows = (int)(n - r0 < ROWS ? n - r0 : ROWS);
        base = (uint64_t)(uintptr_t)f.p + (uint64_t)(ALONG ? r0 * f.ld + k0 : k0 * f.ld + r0) * kSize;
    }

    // The copies that bring the factor's share of the next kDeep of `left` k into buffer `b`: where they read and write, then
    // each of the wave's kCopies.
    i32x4 buffer;
    uint32_t past, to;
    __device__ __forceinline__ void aim(int64_t left, int b, int wave)     // (left = 0: zeros, which nobody reads)
    {
        uint32_t bytes;
        past = 0;
        if constexpr (ALONG) {
            bytes = (uint32_t)(rows - 1) * ldb + (uint32_t)(left < kDeep ? (left + kPiece - 1) & ~(kPiece - 1) : kDeep) * kSize;   // (whole pieces)
            past = chunk * kPiece < left ? 0u : 0x80000000u;                // (`bytes` is below 2^31)
        } else {
            bytes = (uint32_t)((left < kDeep ? left : kDeep) - 1) * ldb + (uint32_t)((rows + kPiece - 1) & ~(kPiece - 1)) * kSize;
        }
        buffer[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)base);
        buffer[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32) & 0xffff);
        buffer[2] = __builtin_amdgcn_readfirstlane(left > 0 ? (int)bytes : 0);
        buffer[3] = 0x00020000;
        to = lds + b * kBytes + wave * kCopies * 1024;
        base += ALONG ? 128 : (uint64_t)kDeep * ldb;
    }
    __device__ __forceinline__ void copy(int u) const
    {
        constexpr int kStep = ALONG ? 8 : kK;
        copy_to_lds(__builtin_amdgcn_readfirstlane(to + u * 1024), from[u & 1] + (uint32_t)(u * kStep) * ldb + past, buffer);
    }

    // Fragment f of step s (32 bytes along k) from buffer `b`: row lane % 32, the (lane / 32)-th 16 bytes.
    __device__ __forceinline__ u32x4 read(int b, int s, int f) const
    {
        if constexpr (ALONG) {
            return lds_read(at[s] + b * kBytes + f * 32 * 128);
        } else if constexpr (kSize == 4) {
            u32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = *(const __attribute__((address_space(3))) uint32_t *)(uintptr_t)(at[0] + b * kBytes + ((s * 8 + e) * ROWS + f * 32) * 4);
            return v;
        } else {
            const uint32_t a = at[f & 1] + b * kBytes + s * 16 * (ROWS * 2) + (f >> 1) * 128;
            const u32x2 lo = lds_read_across(a), hi = lds_read_across(a + 4 * (ROWS * 2));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }
};

typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

template <class T>
__device__ __forceinline__ void store_four(T *p, const f32x4 &v, bool past)
{
    if constexpr (sizeof(T) == 4) {
        if (past) {
            apart();
            __builtin_nontemporal_store(v, (f32x4_any *)p);
            apart();
        } else {
            *(f32x4_any *)p = v;
        }
    } else {
        const u32x2 four = {pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3])};
        if (past) {
            apart();
            __builtin_nontemporal_store(four, (u32x2_any *)p);
            apart();
        } else {
            *(u32x2_any *)p = four;
        }
    }
}

// R times four neighbouring sums, `step` rows apart: those of a lane's row `row`, row + step, .. below `rows`, n of the four
// below N (1 .. 4).  The first of the tile's rows is at i, its first column at j, the lane's own `col` further: addresses are
// a wave's 64-bit base and a lane's 32-bit offset.  Each thing that may have to be done is asked for once for all R.
struct Spot {
    int64_t i, j;
    int row, col, rows, n;
};

template <class T, class O, int R, int STEP>
__device__ __forceinline__ void store_rows(O *p, int64_t ld, const Spot &at, const f32x4 (&w)[R], bool past)
{
    O *base = p + at.i * ld + at.j;
    const uint32_t off = (uint32_t)at.row * (uint32_t)ld + (uint32_t)at.col;
    if (at.n == 4 && past) {
#pragma unroll
        for (int r = 0; r < R; ++r, base += STEP * ld)
            if (at.row + r * STEP < at.rows) store_four(base + off, w[r], true);
    } else if (at.n == 4) {
#pragma unroll
        for (int r = 0; r < R; ++r, base += STEP * ld)
            if (at.row + r * STEP < at.rows) store_four(base + off, w[r], false);
    } else {
#pragma unroll 1
        for (int e = 0; e < at.n; ++e) {
            O *q = base + e;
#pragma unroll
            for (int r = 0; r < R; ++r, q += STEP * ld)
                if (at.row + r * STEP < at.rows) q[off] = (O)(e == 0 ? w[r][0] : e == 1 ? w[r][1] : w[r][2]);
        }
    }
}
// What a 16-bit residual has at the same places, as it is stored.  (At the right edge the last four of a row are read, so that
// such a lane waits no longer than the others; there are four, see Product::parts.)
template <class T, int R, int STEP>
__device__ __forceinline__ void ask_rows(const T *p, int64_t ld, const Spot &at, u32x2 (&raw)[R])
{
    const T *base = p + at.i * ld + at.j;
    const uint32_t off = (uint32_t)at.row * (uint32_t)ld + (uint32_t)at.col - (uint32_t)(4 - at.n);
#pragma unroll
    for (int r = 0; r < R; ++r, base += STEP * ld)
        if (at.row + r * STEP < at.rows && at.n > 0) raw[r] = *(const u32x2_any *)(base + (int32_t)off);
}
template <class T, int R>
__device__ __forceinline__ void add_rows(const Spot &at, const u32x2 (&raw)[R], f32x4 (&w)[R])
{
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint64_t four = __builtin_bit_cast(uint64_t, raw[r]) >> (16 * (4 - at.n));
        float v[8];
        unpack<T>(u32x4{(uint32_t)four, (uint32_t)(four >> 32), 0, 0}, v);
        w[r] += f32x4{v[0], v[1], v[2], v[3]};
    }
}
template <int R, int STEP>
__device__ __forceinline__ void add_rows(const float *p, int64_t ld, const Spot &at, f32x4 (&w)[R])
{
    const float *base = p + at.i * ld + at.j;
    const uint32_t off = (uint32_t)at.row * (uint32_t)ld + (uint32_t)at.col - (uint32_t)(4 - at.n);
    f32x4 v[R] = {};
#pragma unroll
    for (int r = 0; r < R; ++r, base += STEP * ld)
        if (at.row + r * STEP < at.rows) v[r] = *(const f32x4_any *)(base + (int32_t)off);
#pragma unroll
    for (int r = 0; r < R; ++r)
        w[r] += at.n == 4 ? v[r] : at.n == 3 ? f32x4{v[r][1], v[r][2], v[r][3], 0.0f} : at.n == 2 ? f32x4{v[r][2], v[r][3], 0.0f, 0.0f} : f32x4{v[r][3], 0.0f, 0.0f, 0.0f};
}

// How sums leave: as they are, with bias and perhaps max(z, 0); or with any of activation (one an instantiation), residual,
// preact: 720 us for 69120 x 3000 x 1024 with gelu, residual and preact, 1.24 GB to move.
constexpr int kPlain = -1;

// The sums of a wave's part of a tile finished and stored.  They pass through LDS, 16 rows of C at a time and each wave in a
// region of its own, so that whole runs of a row are stored: a lane's own are 4 neighbours, 8 apart in every 32 columns, of
// one row in 32.  Piece c of a row lies at c ^ row, as eight lanes that write or read at once are to cover all banks.
typedef const __attribute__((address_space(4))) Product *ProductArgs;

template <class T, int FI, int FJ, int KIND>
__device__ __forceinline__ void leave(ProductArgs args, const f32x16 (&acc)[FI][FJ], const f32x4 &bias, float undo, int share, int64_t i0, int64_t j0, float *mine)
{
    // What is needed here alone is fetched and computed here: kept over the loops before it costs registers that they need.
    int lane = threadIdx.x & 63;
    asm volatile("" : "+s"(args), "+v"(lane));
    constexpr int kPer = FJ * 8, kRows = 64 / kPer, kR = 16 / kRows;
    const int64_t M = args->M, N = args->N, j = j0 + (lane % kPer) * 4;
    const int nj = (int)(N - j < 4 ? (N - j < 0 ? 0 : N - j) : 4), in_row = lane / kPer;
    const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float *)mine + (lane & 15) * FJ * 128;
    const bool split = KIND == kPlain && args->parts, relu = KIND == FB_ACT_RELU || (KIND == kPlain && !split && args->f.act == FB_ACT_RELU);
    const int out_type = split ? FB_TYPE_F32 : args->f.out_type;
    const bool past = args->past;
    const int64_t ld = split ? N : args->f.ldy;
    void *y = split ? (void *)(args->part + (size_t)share * M * N) : args->f.y;
    const void *residual = KIND == kPlain ? nullptr : args->f.residual;
    auto spot = [&](int pass) {
        const int64_t i = i0 + pass * 16;
        return Spot{i, j0, in_row, (lane % kPer) * 4, (int)(M - i < 16 ? M - i : 16), nj};
    };
    auto put = [&](const f32x16 (&sums)[FJ]) {
#pragma unroll
        for (int y = 0; y < FJ; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x4 w = {sums[y][4 * e], sums[y][4 * e + 1], sums[y][4 * e + 2], sums[y][4 * e + 3]};
                const int c = (y * 8 + 2 * e + (lane >> 5)) ^ (lane & 15 & (kPer - 1));
                *(__attribute__((address_space(3))) f32x4 *)(uintptr_t)(to + c * 16) = w;
            }
    };
    auto get = [&](f32x4 (&w)[kR]) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            const int row = r * kRows + in_row;
            const f32x4 s = *(const f32x4 *)(mine + row * FJ * 32 + ((lane % kPer) ^ (row & (kPer - 1))) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[r][e] = fmaf(s[e], undo, bias[e]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    auto act = [&](f32x4 (&w)[kR], int which) {
#pragma unroll
        for (int r = 0; r < kR; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) w[r][e] = act_of(w[r][e], which);
    };
    auto store = [&](const Spot &at, const f32x4 (&w)[kR]) {
        if (out_type == FB_TYPE_F32)
            store_rows<T, float, kR, kRows>((float *)y, ld, at, w, past);
        else
            store_rows<T, T, kR, kRows>((T *)y, ld, at, w, past);
    };
    if constexpr (KIND == kPlain) {
#pragma unroll
        for (int pass = 0; pass < 2 * FI; ++pass) {
            if ((lane >> 4 & 1) == (pass & 1)) put(acc[pass / 2]);
            f32x4 w[kR];
            get(w);
            const Spot at = spot(pass);
            if (at.rows > in_row && nj > 0) {
                if (relu) act(w, FB_ACT_RELU);
                store(at, w);
            }
        }
    } else {
        // (A loop: unrolled, the addresses of three matrices in every pass take all scalar registers and more.)
        const T *res16 = out_type == FB_TYPE_F32 ? nullptr : (const T *)residual;
        const float *res32 = out_type == FB_TYPE_F32 ? (const float *)residual : nullptr;
        u32x2 next[kR] = {};
        if (res16) ask_rows<T, kR, kRows>(res16, args->f.ldr, spot(0), next);
#pragma unroll 1
        for (int pass = 0; pass < 2 * FI; ++pass) {
            if ((lane >> 4 & 1) == (pass & 1)) {
                if (pass < 2) put(acc[0]);
                else if (FI <= 2 || pass < 4) put(acc[1 % FI]);
                else if (pass < 6) put(acc[2 % FI]);
                else put(acc[3 % FI]);
            }
            u32x2 raw[kR];
#pragma unroll
            for (int r = 0; r < kR; ++r) raw[r] = next[r];
            if (res16 && pass + 1 < 2 * FI) ask_rows<T, kR, kRows>(res16, args->f.ldr, spot(pass + 1), next);
            f32x4 w[kR];
            get(w);
            const Spot at = spot(pass);
            if (at.rows > in_row && nj > 0) {
                if (args->f.preact) store_rows<T, T, kR, kRows>((T *)args->f.preact, args->f.ldp, at, w, past);
                act(w, KIND);
                if (res16) add_rows<T, kR>(at, raw, w);
                if (res32) add_rows<kR, kRows>(res32, args->f.ldr, at, w);
                store(at, w);
            }
        }
    }
}

// A product and its tiles, as a kernel gets it.
struct Task {
    Product q;
    int tiles_i, tiles_j;
};

// Workgroup `block` of `blocks`: they stay and take tile after tile, so that the copies for the next tile are under way while
// this one's sums leave.  `args`: where the kernel's argument with the product lies.
template <class T, bool ALONG_A, bool ALONG_B, int WI, int WJ, int FI, int FJ, int KIND>
__device__ __forceinline__ void run_tiles(const Task &task, ProductArgs args, int block, int blocks)
{
    const Product &q = task.q;
    const int tiles_i = task.tiles_i, tiles_j = task.tiles_j;
    constexpr int kI = WI * FI * 32, kJ = WJ * FJ * 32, kNW = WI * WJ;
    extern __shared__ char lds_raw[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds_raw;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wi = wave / WJ, wj = wave % WJ;

    // Workgroups go to the eight chiplets in turn: each chiplet has a run of neighbouring tiles, so that its L2 holds what
    // they share; within a run eight tiles down, then one across.
    const int n = tiles_i * tiles_j * q.split, xcd = block % 8, run = n / 8 + (xcd < n % 8 ? 1 : 0);
    const int run0 = xcd * (n / 8) + (xcd < n % 8 ? xcd : n % 8);
    struct Place {
        int share;
        int64_t i0, j0, length;
    };
    auto place = [&](int in_run) {
        const int t = run0 + in_run, share = t / (tiles_i * tiles_j), u = t - share * tiles_i * tiles_j;
        const int group = u / (8 * tiles_j), first = group * 8, down = tiles_i - first < 8 ? tiles_i - first : 8;
        const int v = u - group * 8 * tiles_j;
        const int64_t k0 = (int64_t)share * q.share;
        return Place{share, (int64_t)(first + v % down) * kI, (int64_t)(v / down) * kJ, k0 + q.share < q.K ? q.share : q.K - k0};
    };

    float undo = 1.0f;                     // (products of a half-precision gradient; shares of k leave as they are)
    if constexpr (std::is_same<T, f16>::value && !ALONG_B) {
        if (q.f.undo && !q.parts) undo = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(*q.f.undo)));
    }

    constexpr int kDeep = kDeepOf<T>;
    Side<T, ALONG_A, kI, kNW, FI> a;
    Side<T, ALONG_B, kJ, kNW, FJ> b;
    a.start(q.A, lds0, wave, wi * FI * 32);
    b.start(q.B, lds0 + 2 * a.kBytes, wave, wj * FJ * 32);
    // The copies run two steps ahead of the products, over the ends of tiles.
    constexpr int kCopies = a.kCopies + b.kCopies, kReads = FI + FJ, kSlots = FI * FJ;
    int ahead = block / 8;                 // the tile that they are at, and what is left of its k
    int64_t left = 0;
    auto enter = [&]() {
        if (ahead >= run) return;
        const Place p = place(ahead);
        a.tile(q.A, p.i0, q.M, (int64_t)p.share * q.share);
        b.tile(q.B, p.j0, q.N, (int64_t)p.share * q.share);
        left = p.length;
    };
    auto aim = [&](int buffer) {
        a.aim(left, buffer, wave);
        b.aim(left, buffer, wave);
        if (left > 0) {
            left = left > kDeep ? left - kDeep : 0;
            if (left == 0) {
                ahead += blocks / 8;
                enter();
            }
        }
    };
    auto copy = [&](int u) {
        if (u < a.kCopies)
            a.copy(u);
        else
            b.copy(u - a.kCopies);
    };
    u32x4 fa[2][FI], fb_[2][FJ];
    auto read = [&](int buffer, int s, int set, int f) {
        if (f < FI)
            fa[set][f] = a.read(buffer, s, f);
        else
            fb_[set][f - FI] = b.read(buffer, s, f - FI);
    };
    // What has been asked for has come, in every wave; and every wave has read what it wanted of the other buffer.
    auto meet = [&]() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    if (ahead >= run) return;
    if (q.K > 0) {
        enter();
        for (int buffer = 0; buffer < 2; ++buffer) {
            aim(buffer);
#pragma unroll
            for (int u = 0; u < kCopies; ++u) copy(u);
            if (buffer == 0) meet();
        }
    }
    int turn = 0;                               // the buffer that holds this step's share
    for (int in_run = block / 8; in_run < run; in_run += blocks / 8) {
        const Place p = place(in_run);
        const int steps = (int)((p.length + kDeep - 1) / kDeep);
        f32x16 acc[FI][FJ] = {};
        f32x4 bias = {};
        if (!q.parts && q.f.bias) {
            const int64_t j = p.j0 + wj * FJ * 32 + lane % (FJ * 8) * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j + e < q.N) bias[e] = q.f.bias[j + e];
        }
        // One matrix instruction at a time, and behind it a read for the next 32 bytes of k, and after the meeting also a copy: in this
        // order, which the compiler left to itself does not keep (it puts the reads right before their use).
        auto times = [&](int m, int set) {
            const int x = m / FJ, y = m % FJ;
            acc[x][y] = multiply<T>(fb_[set][y], fa[set][x], acc[x][y]);
        };
        if (steps > 0) {
#pragma unroll
            for (int f = 0; f < kReads; ++f) read(turn, 0, 0, f);
        }
        for (int step = 0; step < steps; ++step, turn ^= 1) {
#pragma unroll
            for (int s = 0; s < 3; ++s)
#pragma unroll
                for (int m = 0; m < kSlots; ++m) {
                    times(m, s & 1);
#pragma unroll
                    for (int f = 0; f < kReads; ++f)
                        if (f * kSlots / kReads == m) read(turn, s + 1, (s + 1) & 1, f);
                    __builtin_amdgcn_sched_barrier(0);
                }
            times(0, 1);
            __builtin_amdgcn_sched_barrier(0);
            meet();
            asm volatile("" : "+v"(bias));      // (it has come with the rest: no wait for it later, behind further copies)
            aim(turn);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kSlots == 1) {
#pragma unroll
                for (int f = 0; f < kReads; ++f) read(turn ^ 1, 0, 0, f);
#pragma unroll
                for (int u = 0; u < kCopies; ++u) copy(u);
            }
#pragma unroll
            for (int m = 1; m < kSlots; ++m) {  // (behind a tile's last step: of the next tile's first, and read again then)
                times(m, 1);
#pragma unroll
                for (int f = 0; f < kReads; ++f)
                    if (f * (kSlots - 1) / kReads == m - 1) read(turn ^ 1, 0, 0, f);
#pragma unroll
                for (int u = 0; u < kCopies; ++u)
                    if (u * (kSlots - 1) / kCopies == m - 1) copy(u);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        leave<T, FI, FJ, KIND>(args, acc, bias, undo, p.share, p.i0 + wi * FI * 32, p.j0 + wj * FJ * 32,
                               (float *)(lds_raw + 2 * (a.kBytes + b.kBytes)) + wave * 16 * FJ * 32);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (no copy into LDS outlives the workgroup)
}

template <class T, bool ALONG_A, bool ALONG_B, int WI, int WJ, int FI, int FJ, int KIND>
__global__ __launch_bounds__(WI * WJ * 64) void fb_mfma_product_kernel(Task task)
{
    run_tiles<T, ALONG_A, ALONG_B, WI, WJ, FI, FJ, KIND>(task, (ProductArgs)__builtin_amdgcn_kernarg_segment_ptr(), blockIdx.x, gridDim.x);
}

// Both products of a gradient, dx by the first `blocks` workgroups and dW by the others: small ones fill the GPU together.
template <class T, int WI, int WJ, int FI, int FJ>
__global__ __launch_bounds__(WI * WJ * 64) void fb_mfma_pair_kernel(Task dx, Task dw, int blocks)
{
    const __attribute__((address_space(4))) char *args = (const __attribute__((address_space(4))) char *)__builtin_amdgcn_kernarg_segment_ptr();
    if ((int)blockIdx.x < blocks)
        run_tiles<T, true, false, WI, WJ, FI, FJ, kPlain>(dx, (ProductArgs)args, blockIdx.x, blocks);
    else
        run_tiles<T, false, false, WI, WJ, FI, FJ, kPlain>(dw, (ProductArgs)(args + sizeof(Task)), blockIdx.x - blocks, gridDim.x - blocks);
}

// A kernel's tile, on-chip memory and the workgroups that the GPU holds.
template <int WI, int WJ, int FI, int FJ>
struct Shape {
    static constexpr int kI = WI * FI * 32, kJ = WJ * FJ * 32;
    static constexpr size_t kBytes = (size_t)2 * (kI + kJ) * 128 + (size_t)WI * WJ * 16 * FJ * 32 * 4;
    static constexpr int64_t kSlots = (int64_t)kCUs * (int64_t)(kLdsBytes / kBytes);
};

template <class S>
Task task_of(const Product &q)
{
    Task t{q, (int)((q.M + S::kI - 1) / S::kI), (int)((q.N + S::kJ - 1) / S::kJ)};
    t.q.past = !q.parts && goes_past(q.M, q.N, q.f.out_type);
    return t;
}
template <class S>
int64_t blocks_of(const Product &q)
{
    const int64_t n = ((q.M + S::kI - 1) / S::kI) * ((q.N + S::kJ - 1) / S::kJ) * q.split;
    return n >= kMostSize ? n : std::min(S::kSlots, (n + 7) / 8 * 8);
}

template <class S, class K>
int take_lds(K kernel)
{
    if (S::kBytes <= 64 * 1024) return FB_OK;
    const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)S::kBytes);
    return e == hipSuccess ? FB_OK : fail(FB_EHIP, std::string("hipFuncSetAttribute(LDS size): ") + hipGetErrorString(e));
}

template <class T, bool ALONG_A, bool ALONG_B, int WI, int WJ, int FI, int FJ, int KIND>
int launch(const Product &q, hipStream_t stream)
{
    typedef Shape<WI, WJ, FI, FJ> S;
    const int64_t blocks = blocks_of<S>(q);
    if (blocks >= kMostSize) return fail(FB_EUNSUPPORTED, "affine product: more than 2^31 tiles");
    const auto kernel = fb_mfma_product_kernel<T, ALONG_A, ALONG_B, WI, WJ, FI, FJ, KIND>;
    const int rc = take_lds<S>(kernel);
    if (rc != FB_OK) return rc;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(WI * WJ * 64), S::kBytes, stream, task_of<S>(q));
    return launched("matrix product kernel launch: ");
}

template <class T, int WI, int WJ, int FI, int FJ>
int launch_pair(const Product &dx, const Product &dw, hipStream_t stream)
{
    typedef Shape<WI, WJ, FI, FJ> S;
    const int64_t first = blocks_of<S>(dx);
    const auto kernel = fb_mfma_pair_kernel<T, WI, WJ, FI, FJ>;
    const int rc = take_lds<S>(kernel);
    if (rc != FB_OK) return rc;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(first + blocks_of<S>(dw))), dim3(WI * WJ * 64), S::kBytes, stream, task_of<S>(dx), task_of<S>(dw), (int)first);
    return launched("matrix product kernel launch: ");
}

template <class T>
int launch_pair(const Product &dx, const Product &dw, hipStream_t stream)
{
    return dx.tile == 128 ? launch_pair<T, 2, 2, 2, 2>(dx, dw, stream) : launch_pair<T, 2, 2, 1, 1>(dx, dw, stream);
}

template <class T, bool ALONG_A, bool ALONG_B, int KIND>
int launch(const Product &q, hipStream_t stream)
{
    if (q.tile == 256) return launch<T, ALONG_A, ALONG_B, 2, 4, 4, 2, KIND>(q, stream);
    return q.tile == 128 ? launch<T, ALONG_A, ALONG_B, 2, 2, 2, 2, KIND>(q, stream) : launch<T, ALONG_A, ALONG_B, 2, 2, 1, 1, KIND>(q, stream);
}

template <class T>
int launch(const Product &q, hipStream_t stream)
{
    if (!q.A.along) return launch<T, false, false, kPlain>(q, stream);
    if (!q.B.along) return launch<T, true, false, kPlain>(q, stream);
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
