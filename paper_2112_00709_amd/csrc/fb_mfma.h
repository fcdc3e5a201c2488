// Products on the matrix units (see fb_affine.h), for factors whose rows are whole 16-byte pieces; included by the files whose
// kernels are made of them.
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
#pragma once

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
// PAIRED: the factor is two of `n` rows, one behind the other, and the tile has as many rows of the one as of the other, 32 by 32 in
// turn, so that a wave's fragments are in twos the same rows of both.  A wave's copies are 32 rows, of one of them.
// MASKED: k whose bit in Product::live is 0 are zeros, whatever they hold.
template <class T, bool ALONG, int ROWS, int NW, int F, bool PAIRED = false, bool MASKED = false>
struct Side {
    static constexpr int kSize = sizeof(T), kDeep = kDeepOf<T>, kPiece = 16 / kSize;
    static constexpr int kBytes = ROWS * 128, kCopies = kBytes / 1024 / NW;
    static constexpr int kPer = ROWS * kSize / 16, kK = 64 / kPer;      // not ALONG: lanes a k, k a copy
    static_assert(!MASKED || !ALONG, "a lane copies pieces of one k");
    static_assert(!PAIRED || (ALONG && F % 2 == 0 && kCopies == 4), "a wave copies 32 rows and has as many fragments of each factor");
    uint64_t base;           // of the tile's first element at the share's first k
    uint32_t ldb;            // bytes between rows
    int rows;                // rows of the factor from the tile's first on
    uint32_t from[2];        // a lane's offset in what a copy brings (two: even and odd copies)
    uint32_t lds;            // the first buffer
    uint32_t at[ALONG ? 4 : 2];
    int chunk;               // ALONG: a lane's piece along k
    const __attribute__((address_space(4))) uint64_t *live;   // MASKED: of 64 k, and those of the next step
    uint64_t bits;
    int bit;                 // of the lane's first k, 32 k a step: in which half of `bits`
    uint32_t dead;           // bits of the step's k, from the lane's first, inverted

    // What does not depend on the tile.
    __device__ __forceinline__ void start(const Factor &f, uint32_t lds_at, int wave, int w0)
    {
        const int lane = threadIdx.x & 63;
        ldb = (uint32_t)f.ld * kSize;
        lds = lds_at;
        const int l = lane & 31, h = lane >> 5;
        if constexpr (ALONG) {
            chunk = (lane & 7) ^ (lane >> 3);
            from[0] = from[1] = (uint32_t)((PAIRED ? wave >> 1 : wave) * kCopies * 8 + (lane >> 3)) * ldb + chunk * 16;
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

    __device__ __forceinline__ void tile(const Factor &f, int64_t r0, int64_t n, int64_t k0, int wave, const uint64_t *mask)
    {
        if constexpr (MASKED) {
            live = (const __attribute__((address_space(4))) uint64_t *)(mask + k0 / 64);
            bit = (int)(k0 & 32);
            bits = *live;
        }
        constexpr int kMost = PAIRED ? ROWS / 2 : ROWS;
        rows = (int)(n - r0 < kMost ? n - r0 : kMost);
        if (PAIRED && (wave & 1)) r0 += n;
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
        if constexpr (MASKED) {
            const int lane = threadIdx.x & 63;
            dead = ~(uint32_t)(bits >> (bit + wave * kCopies * kK + lane / kPer));
            bit = kDeep == 64 ? 0 : bit ^ 32;
            if (bit == 0 && left > 0) bits = *++live;        // (one word more than there are k)
        }
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
        uint32_t offset = from[u & 1] + (uint32_t)(u * kStep) * ldb + past;
        if constexpr (MASKED) offset |= (dead << (31 - u * kK)) & 0x80000000u;     // (beyond the buffer's end)
        copy_to_lds(__builtin_amdgcn_readfirstlane(to + u * 1024), offset, buffer);
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

// Where a wave's sums belong: the tile's share of k, first row and column, the wave's place in the tile, and LDS for the way out (16
// rows of 32 or 64 sums a wave).
struct Where {
    int share;
    int64_t i0, j0;
    int wi, wj, wave;
    float *room;
};

// What a row has in common and what a column has go onto the sums by one matrix instruction a fragment, of two k in single
// precision: of_columns[y] lane % 32 1 + 1 of_row.  (`of_columns`: a column's in the lower lanes, 1 in the upper ones, or 0 if rows have nothing.)
template <int FJ>
__device__ __forceinline__ void add_rank_one(f32x16 (&acc)[FJ], const f32x4 &of_columns, float of_row, int lane)
{
#pragma unroll
    for (int y = 0; y < FJ; ++y) acc[y] = __builtin_amdgcn_mfma_f32_32x32x2f32(of_columns[y], lane < 32 ? 1.0f : of_row, acc[y], 0, 0, 0);
}

// F neighbouring fragments of 32 rows from i0 and 32 columns each from j0 on, stored as T: a lane has row lane % 32, columns
// 8 e + 4 (lane / 32) + 0 .. 3 of every 32.  They pass through the wave's LDS (`mine`, 16 rows of F fragments in single precision) as T, so that
// whole runs of a row are stored by 16 bytes a lane; piece c of a row lies at c ^ row there.  WHOLE: rows are whole pieces, kept in the caches.
template <class T, int F, bool WHOLE = false>
__device__ __forceinline__ void store_fragments(const f32x16 (&v)[F], float *mine, T *out, int64_t ld, int64_t i0, int64_t j0, int64_t M, int64_t N, int lane, bool past)
{
    constexpr int VE = Vec<T>::kN, kPieces = F * 32 / VE, kAll = 16 * F * 32 * 4 / (kPieces * 16), kAtOnce = 64 / kPieces, kR = kAll / kAtOnce;
    const int64_t j = j0 + lane % kPieces * VE;
    const int n = (int)(N - j < VE ? N - j : VE), in_row = lane / kPieces;
#pragma unroll
    for (int l0 = 0; l0 < 32; l0 += kAll) {
        const int l = (lane & 31) - l0;
        if (l >= 0 && l < kAll) {
            char *to = (char *)mine + l * kPieces * 16;
#pragma unroll
            for (int y = 0; y < F; ++y)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x4 four = {v[y][4 * e], v[y][4 * e + 1], v[y][4 * e + 2], v[y][4 * e + 3]};
                    if constexpr (sizeof(T) == 4)
                        *(f32x4 *)(to + ((y * 8 + 2 * e + (lane >> 5)) ^ (l & (kPieces - 1))) * 16) = four;
                    else
                        *(u32x2 *)(to + ((y * 4 + e) ^ (l & (kPieces - 1))) * 16 + (lane >> 5) * 8) = u32x2{pack2<T>(four[0], four[1]), pack2<T>(four[2], four[3])};
                }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        u32x4 w[kR];
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            const int row = r * kAtOnce + in_row;
            w[r] = *(const u32x4 *)((const char *)mine + row * kPieces * 16 + ((lane % kPieces) ^ (row & (kPieces - 1))) * 16);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        T *base = out + (i0 + l0) * ld + j0;
        const uint32_t off = (uint32_t)in_row * (uint32_t)ld + (uint32_t)(lane % kPieces * VE);
        const int rows = (int)(M - i0 - l0 < kAll ? M - i0 - l0 : kAll);
        if (n == VE) {
#pragma unroll
            for (int r = 0; r < kR; ++r, base += kAtOnce * ld)
                if (r * kAtOnce + in_row < rows) store_piece(base + off, VE, w[r], !WHOLE && past);
        } else if (!WHOLE && n > 0) {
#pragma unroll 1
            for (int e = 0; e < n; ++e) {
                T *p = base + off + e;
#pragma unroll
                for (int r = 0; r < kR; ++r, p += kAtOnce * ld) {
                    if (r * kAtOnce + in_row >= rows) continue;
                    if constexpr (sizeof(T) == 4)
                        *(uint32_t *)p = e == 0 ? w[r][0] : e == 1 ? w[r][1] : w[r][2];
                    else
                        *(uint16_t *)p = (uint16_t)((e < 2 ? w[r][0] : e < 4 ? w[r][1] : e < 6 ? w[r][2] : w[r][3]) >> (16 * (e & 1)));
                }
            }
        }
    }
}

__device__ __forceinline__ void bias_of(const float *bias, int64_t n, int64_t j, f32x4 &four)
{
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (j + e < n) four[e] = bias[j + e];
}

template <int KIND>
struct Finished {
    static constexpr bool kPaired = false, kNeverEmpty = false, kFolded = false;
    static constexpr int kEarly = 1;       // fours of numbers that a lane asks for when a tile begins: its columns' bias

    template <int FI, int FJ>
    static __device__ __forceinline__ void early(const Product &q, const Where &where, int lane, f32x4 (&four)[1])
    {
        if (!q.parts && q.f.bias) bias_of(q.f.bias, q.N, where.j0 + where.wj * FJ * 32 + lane % (FJ * 8) * 4, four[0]);
    }

    template <class T, int FI, int FJ>
    static __device__ __forceinline__ void leave(ProductArgs args, f32x16 (&acc)[FI][FJ], const f32x4 (&four)[1], float undo, const Where &where)
    {
        const f32x4 bias = four[0];
        const int share = where.share;
        const int64_t i0 = where.i0 + where.wi * FI * 32, j0 = where.j0 + where.wj * FJ * 32;
        float *mine = where.room + where.wave * 16 * FJ * 32;
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
};

// Sums leave rounded to the factors' 16 bits, as they are or times *undo: what gradients are.
struct Rounded {
    static constexpr bool kPaired = false, kNeverEmpty = false, kFolded = false;
    static constexpr int kEarly = 1;

    template <int FI, int FJ>
    static __device__ __forceinline__ void early(const Product &, const Where &, int, f32x4 (&)[1])
    {
    }

    template <class T, int FI, int FJ>
    static __device__ __forceinline__ void leave(ProductArgs args, f32x16 (&acc)[FI][FJ], const f32x4 (&)[1], float undo, const Where &where)
    {
        int lane = threadIdx.x & 63;
        asm volatile("" : "+s"(args), "+v"(lane));
        const int64_t i0 = where.i0 + where.wi * FI * 32, j0 = where.j0 + where.wj * FJ * 32;
#pragma unroll
        for (int x = 0; x < FI; ++x) {
            if (undo != 1.0f) {
#pragma unroll
                for (int y = 0; y < FJ; ++y) acc[x][y] *= undo;
            }
            store_fragments<T, FJ>(acc[x], where.room + where.wave * 16 * FJ * 32, (T *)args->f.y, args->f.ldy, i0 + x * 32, j0, args->M, args->N, lane, args->past);
        }
    }
};

// A product and its tiles, as a kernel gets it.
struct Task {
    Product q;
    int tiles_i, tiles_j;
};

// Whether there are registers for a second set of sums: not beside the 128 sums a lane of 16-bit tiles of 256, which are one chain over k.
template <class T, int FI, int FJ>
constexpr bool kFoldsOf = sizeof(T) == 4 || FI * FJ <= 4;

// Workgroup `block` of `blocks`: they stay and take tile after tile, so that the copies for the next tile are under way while
// this one's sums leave.  `args`: where the kernel's argument with the product lies.
template <class T, bool ALONG_A, bool ALONG_B, int WI, int WJ, int FI, int FJ, class WAY, bool MASKED = false>
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
        return Place{share, (int64_t)(first + v % down) * kI, (int64_t)(v / down) * (WAY::kPaired ? kJ / 2 : kJ), k0 + q.share < q.K ? q.share : q.K - k0};
    };

    float undo = 1.0f;                     // (products of a 16-bit gradient; shares of k leave as they are)
    if constexpr (sizeof(T) == 2 && (!ALONG_B || WAY::kNeverEmpty)) {
        if (q.f.undo && !q.parts) undo = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(*q.f.undo)));
    }

    constexpr int kDeep = kDeepOf<T>;
    Side<T, ALONG_A, kI, kNW, FI> a;
    Side<T, ALONG_B, kJ, kNW, FJ, WAY::kPaired, MASKED> b;
    a.start(q.A, lds0, wave, wi * FI * 32);
    b.start(q.B, lds0 + 2 * a.kBytes, wave, wj * FJ * 32);
    // The copies run two steps ahead of the products, over the ends of tiles.
    constexpr int kCopies = a.kCopies + b.kCopies, kReads = FI + FJ, kSlots = FI * FJ;
    int ahead = block / 8;                 // the tile that they are at, and what is left of its k
    int64_t left = 0;
    auto enter = [&]() {
        if (ahead >= run) return;
        const Place p = place(ahead);
        a.tile(q.A, p.i0, q.M, (int64_t)p.share * q.share, wave, nullptr);
        b.tile(q.B, p.j0, q.N, (int64_t)p.share * q.share, wave, q.s.live);
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
        if constexpr (WAY::kNeverEmpty) __builtin_assume(steps > 0);      // (or it would be waited for what `early` asks for)
        f32x16 acc[FI][FJ] = {};
        // Sums of kFold steps (256 k, of 16 bits 512) are added up apart, so that their roundings do not pile up over a long k (192 x 186 x 3769
        // in single precision: gradients 3.3e-7 off in the 2-norm instead of 1.4e-6, at the same time; 65 x 300 x 4096 in half precision: 31 and 41
        // instead of 29 and 39 us forward and backward, others unchanged).
        constexpr bool kFolds = WAY::kFolded && kFoldsOf<T, FI, FJ>;
        constexpr int kFold = 8;
        f32x16 folded[kFolds ? FI : 1][kFolds ? FJ : 1] = {};
        const Where where{p.share, p.i0, p.j0, wi, wj, wave, (float *)(lds_raw + 2 * (a.kBytes + b.kBytes))};
        f32x4 four[WAY::kEarly] = {};
        WAY::template early<FI, FJ>(q, where, lane, four);
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
        int done = 0;
        do {
            const int until = kFolds && steps - done > kFold ? done + kFold : steps;
            for (int step = done; step < until; ++step, turn ^= 1) {
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
#pragma unroll
                for (int e = 0; e < WAY::kEarly; ++e) asm volatile("" : "+v"(four[e]));   // (it has come with the rest: no wait for it later, behind further copies)
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
            if constexpr (kFolds) {
                done = until;
#pragma unroll
                for (int x = 0; x < FI; ++x)
#pragma unroll
                    for (int y = 0; y < FJ; ++y) {
                        folded[x][y] += acc[x][y];
                        acc[x][y] = done < steps ? f32x16{} : folded[x][y];
                    }
            }
        } while (kFolds && done < steps);
        WAY::template leave<T, FI, FJ>(args, acc, four, undo, where);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (no copy into LDS outlives the workgroup)
}

// (a second set of sums takes tiles of 128 two registers beyond what two workgroups a compute unit have, if they are not asked for)
template <class T, bool ALONG_A, bool ALONG_B, int WI, int WJ, int FI, int FJ, class WAY, bool MASKED>
__global__ __launch_bounds__(WI * WJ * 64, (WAY::kFolded && kFoldsOf<T, FI, FJ> && FI * FJ == 4 ? 2 : 1)) void fb_mfma_product_kernel(Task task)
{
    run_tiles<T, ALONG_A, ALONG_B, WI, WJ, FI, FJ, WAY, MASKED>(task, (ProductArgs)__builtin_amdgcn_kernarg_segment_ptr(), blockIdx.x, gridDim.x);
}

// A kernel's tile, on-chip memory and the workgroups that the GPU holds.
template <int WI, int WJ, int FI, int FJ>
struct Shape {
    static constexpr int kI = WI * FI * 32, kJ = WJ * FJ * 32;
    static constexpr size_t kBytes = (size_t)2 * (kI + kJ) * 128 + (size_t)WI * WJ * 16 * (FJ < 2 ? FJ : 2) * 32 * 4;
    static constexpr int64_t kSlots = (int64_t)kCUs * (int64_t)(kLdsBytes / kBytes);
};

template <class S>
Task task_of(const Product &q, bool paired = false)
{
    const int64_t across = paired ? S::kJ / 2 : S::kJ;
    Task t{q, (int)((q.M + S::kI - 1) / S::kI), (int)((q.N + across - 1) / across)};
    t.q.past = !q.parts && goes_past(q.M, q.N, q.f.out_type);
    return t;
}
template <class S>
int64_t blocks_of(const Product &q, bool paired = false)
{
    const int64_t across = paired ? S::kJ / 2 : S::kJ, n = ((q.M + S::kI - 1) / S::kI) * ((q.N + across - 1) / across) * q.split;
    return n >= kMostSize ? n : std::min(S::kSlots, (n + 7) / 8 * 8);
}

template <class S, class K>
int take_lds(K kernel)
{
    if (S::kBytes <= 64 * 1024) return FB_OK;
    const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)S::kBytes);
    return e == hipSuccess ? FB_OK : fail(FB_EHIP, std::string("hipFuncSetAttribute(LDS size): ") + hipGetErrorString(e));
}

template <class T, bool ALONG_A, bool ALONG_B, int WI, int WJ, int FI, int FJ, class WAY, bool MASKED = false>
int launch(const Product &q, hipStream_t stream)
{
    typedef Shape<WI, WJ, FI, FJ> S;
    const int64_t blocks = blocks_of<S>(q, WAY::kPaired);
    if (blocks >= kMostSize) return fail(FB_EUNSUPPORTED, "affine product: more than 2^31 tiles");
    const auto kernel = fb_mfma_product_kernel<T, ALONG_A, ALONG_B, WI, WJ, FI, FJ, WAY, MASKED>;
    const int rc = take_lds<S>(kernel);
    if (rc != FB_OK) return rc;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(WI * WJ * 64), S::kBytes, stream, task_of<S>(q, WAY::kPaired));
    return launched("matrix product kernel launch: ");
}

}  // namespace

}  // namespace fb
