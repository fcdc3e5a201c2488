// Log probabilities of given tokens, entropy and best alternatives, and their gradient (fb_layers.h).
//
// One pass over the logits.  A wave holds a piece of a row in registers (as stored, 16 bytes a piece and lane), takes its
// maximum m and with d = x - m the sums S = sum e^d and T = sum e^d d; then log Z = m + log S and H = log S - T / S.  Pieces
// of a row are joined by (m, S, T) -> (M, S e^(m-M), (T + S (m - M)) e^(m-M)), so a long row is split over as many waves
// and workgroups as it takes; of the logits only the few pieces that hold alternatives are read again.
//
// Many rows are bound by memory: 69120 rows of 3000 floats with 3 alternatives take 134 us, the tenth of them that is padding not
// read (5.6 TB/s of the others' bytes).  Few rows are a chain of latencies: one row of 128000 in bfloat16 takes 6 us in 32 workgroups and 5.5 to join
// them with 10 alternatives (5.5 in all without alternatives).
#include "fb_layers_device.h"

namespace fb {

namespace {

constexpr float kLog2E = 1.44269504088896340736f;
constexpr float kInf = __builtin_huge_valf();

struct TokenParams {
    const void *logits;
    int64_t ld, R, V;
    const int32_t *tokens;
    int top;
    float *logprobs, *entropy, *logz;
    int32_t *top_ids;
    float *top_logprobs;
    int split;                 // workgroups a row; beyond one, for each of their waves:
    int64_t chunk;             // (elements of the row that a workgroup has)
    float *part;               // [R][split * waves][3]: m, S, T
    uint64_t *part_top;        // [R][split * waves][top] keys, descending
};

// Total order of (value, number): larger values first, then smaller numbers.  -0 counts as 0.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o ^ ((o & 0x80000000u) ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ uint64_t key_of(float x, uint32_t j) { return (uint64_t)order_of(x) << 32 | (uint32_t)~j; }

// What a wave's lanes have written to LDS, its other lanes read from here on (LDS serves a wave in order: only the compiler
// is held).
__device__ __forceinline__ void lds_settled() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// Largest key of a wave; 0 stands for none.
__device__ __forceinline__ uint64_t max_wave_key(uint64_t k)
{
    const uint32_t hi = max_wave_u((uint32_t)(k >> 32));
    const uint32_t lo = max_wave_u((uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
    return (uint64_t)hi << 32 | lo;
}

struct Stats {
    float m, S, T;
};

__device__ __forceinline__ Stats join(const Stats &a, const Stats &b)
{
    const float M = fmaxf(a.m, b.m);
    if (M == -kInf) return {M, a.S + b.S, a.T + b.T};           // nothing but -inf so far (or NaN, which the sums carry on)
    const float da = a.m == -kInf ? 0.0f : a.m - M, db = b.m == -kInf ? 0.0f : b.m - M;   // (an empty side has no sums to scale)
    const float ea = __builtin_amdgcn_exp2f(da * kLog2E), eb = __builtin_amdgcn_exp2f(db * kLog2E);
    return {M, fmaf(a.S, ea, b.S * eb), fmaf(fmaf(a.S, da, a.T), ea, fmaf(b.S, db, b.T) * eb)};
}

// The rank of a key among `count` (at most 64) different ones, one a lane.
__device__ __forceinline__ int rank_in_wave(uint64_t mine, int count)
{
    int rank = 0;
    for (int c = 0; c < count; ++c) {
        const uint64_t k = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(mine >> 32), c) << 32 |
                           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, c);
        rank += k > mine ? 1 : 0;
    }
    return rank;
}

// The largest number that at least `top` lanes' `mine` reach, found bit by bit; 0 if there is none.
__device__ __forceinline__ uint32_t reached_by(uint32_t mine, int top)
{
    uint32_t least = 0;
#pragma unroll
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t with = least | 1u << bit;
        least = __popcll(__ballot(mine >= with)) >= top ? with : least;
    }
    return least;
}

// The best `top` keys of `lists` descending lists of `top` keys each (at most 64 * HEADS of them), descending, to `out`;
// missing ones are 0.  For one wave: a lane keeps the heads of up to HEADS lists.  What the lanes' largest heads bound from
// below is put on a list and ranked there; where that is more than 64 keys, the largest head of all is taken and its list
// moved on, once a place.  `keys` should lie in LDS: a list is moved on by a read that what follows waits for.
constexpr int kKeysInLds = 4096;

template <int HEADS>
__device__ __forceinline__ void merge_heads(const uint64_t *keys, int lists, int top, uint64_t *list, uint64_t *out)
{
    const int lane = threadIdx.x & 63;
    uint64_t head[HEADS], best = 0;
    int at[HEADS], end[HEADS];
    auto start = [&]() {
        best = 0;
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            at[h] = (h * 64 + lane) * top;
            end[h] = h * 64 + lane < lists ? at[h] + top : at[h];
            head[h] = at[h] < end[h] ? keys[at[h]] : 0;
            best = head[h] > best ? head[h] : best;
        }
    };
    auto move_on = [&](int h) {
        ++at[h];
        head[h] = at[h] < end[h] ? keys[at[h]] : 0;
    };
    start();
    const uint32_t least = reached_by((uint32_t)(best >> 32), top);
    int count = 0;
    if (least != 0) {
        for (bool any = true; any && count <= 64;) {
            any = false;
#pragma unroll
            for (int h = 0; h < HEADS; ++h) {
                const bool in = (uint32_t)(head[h] >> 32) >= least;
                const uint64_t hit = __ballot(in);
                const int to = count + __popcll(hit & ((1ull << lane) - 1));
                if (in && to < 64) list[to] = head[h];
                count += __popcll(hit);
                if (in) move_on(h);
                any = any || hit != 0;
            }
        }
        lds_settled();
    }
    if (least != 0 && count <= 64) {
        const uint64_t mine = lane < count ? list[lane] : 0;
        const int rank = rank_in_wave(mine, count);
        if (lane < count && rank < top) out[rank] = mine;
        return;                                                // (there are at least `top`)
    }
    start();
    for (int t = 0; t < top; ++t) {
        const uint64_t win = max_wave_key(best);
        if (lane == 0) out[t] = win;
        if (win != 0 && best == win) {                         // (keys are different: one lane)
            best = 0;
#pragma unroll
            for (int h = 0; h < HEADS; ++h) {
                if (head[h] == win) move_on(h);
                best = head[h] > best ? head[h] : best;
            }
        }
    }
}

__device__ __forceinline__ void merge_lists(const uint64_t *keys, int lists, int top, uint64_t *list, uint64_t *out)
{
    if (lists <= 64) return merge_heads<1>(keys, lists, top, list, out);
    if (lists <= 128) return merge_heads<2>(keys, lists, top, list, out);
    if (lists <= 512) return merge_heads<8>(keys, lists, top, list, out);
    const int lane = threadIdx.x & 63;
    uint64_t last = ~0ull;
    for (int t = 0; t < top; ++t) {
        uint64_t best = 0;
        for (int i = lane; i < lists * top; i += 64) {
            const uint64_t k = keys[i];
            if (k < last && k > best) best = k;
        }
        last = max_wave_key(best);
        if (lane == 0) out[t] = last;
    }
}

// The best `top` of the elements that a wave holds pieces of (in memory: piece i of a lane starts at element first + i * stride
// of n), as keys, descending, to out[0 .. top) in LDS; peak[i] is the largest element of the lane's piece i.  The top-th
// largest of the lanes' own maxima bounds the top-th best from below; what reaches it are few elements (about `top`) of few
// pieces, which are read once more, put on a list and ranked there, one a lane.  Where fewer than `top` lanes have an element
// above -inf, all such elements go to the list, and the places behind them to the first of the others.  Where ties make a
// list longer than 64 the elements are searched once per place.  (From memory: the pieces in registers, indexed at
// run time, would take a copy of all this per element; one of two is chosen by a select.)
template <class T, int NV>
__device__ __forceinline__ void best_of_wave(const T *row, const u32x4 (&raw)[NV], const float (&peak)[NV], float lane_max, int first, int stride, int n, int top, uint64_t *list, uint64_t *out)
{
    constexpr int VE = Vec<T>::kN;
    const int lane = threadIdx.x & 63;
    // few are taken one after the other; for more their order's bits are found one by one, a comparison and a count each
    float bound = -kInf;
    if (top <= 6) {
        float cur = lane_max;
        for (int found = 0; found < top;) {
            bound = max_wave(cur);
            const uint64_t hit = __ballot(cur == bound);
            if (bound == -kInf || hit == 0) break;
            found += __popcll(hit);
            if (cur == bound) cur = -kInf;
        }
    } else {
        bound = value_of(reached_by(order_of(lane_max), top));
    }
    const bool few = bound == -kInf;
    auto reaches = [&](float x) { return few ? x > -kInf : x >= bound; };
    uint32_t pieces = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) pieces |= reaches(peak[i]) ? 1u << i : 0u;
    int count = 0;
    while (count <= 64 && __ballot(pieces != 0) != 0) {
        const int at = first + (pieces ? __ffs(pieces) - 1 : 0) * stride;
        const int left = pieces ? n - at : 0;
        pieces &= pieces - 1;
        float v[VE];
        if constexpr (NV <= 2) {
            u32x4 piece = raw[0];
#pragma unroll
            for (int i = 1; i < NV; ++i) piece = at == first + i * stride ? raw[i] : piece;
            unpack<T>(piece, v);
        } else {
            unpack<T>(load_piece(row + at, left), v);
        }
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            const uint64_t hit = __ballot(j < left && reaches(v[j]));
            const int at_list = count + __popcll(hit & ((1ull << lane) - 1));
            if ((hit >> lane & 1) && at_list < 64) list[at_list] = key_of(v[j], (uint32_t)(at + j));
            count += __popcll(hit);
        }
    }
    lds_settled();
    if (count <= 64) {
        const uint64_t mine = lane < count ? list[lane] : 0;
        const int rank = rank_in_wave(mine, count);
        if (lane < count && rank < top) out[rank] = mine;
        if (lane >= count && lane < top) out[lane] = 0;
        if (few) {                                            // (a wave's first pieces lie side by side, 256 elements and more)
            const int start = __builtin_amdgcn_readfirstlane(first);
            int filled = count;
            for (int i = 0; i < 128 && filled < top && start + i < n; i += 64) {
                const int at = start + i + lane;
                const bool low = at < n && !(load_one(row + (at < n ? at : 0)) > -kInf);
                const uint64_t hit = __ballot(low);
                const int to = filled + __popcll(hit & ((1ull << lane) - 1));
                if (low && to < top) out[to] = key_of(-kInf, (uint32_t)at);
                filled += __popcll(hit);
            }
        }
        return;
    }
    uint64_t last = ~0ull;
    for (int t = 0; t < top; ++t) {
        uint64_t best = 0;
#pragma unroll 4
        for (int i = 0; i < NV; ++i) {
            float v[VE];
            const int at = first + i * stride;
            unpack<T>(load_piece(row + at, n - at), v);
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const uint64_t k = key_of(v[j], (uint32_t)(at + j));
                if (at + j < n && k < last && k > best) best = k;
            }
        }
        last = max_wave_key(best);
        if (lane == 0) out[t] = last;
    }
}

template <class T>
__device__ __forceinline__ float given_logit(const TokenParams &p, int64_t r, int32_t token)
{
    return token >= 0 && token < p.V ? load_one((const T *)p.logits + r * p.ld + token) : __builtin_nanf("");
}

// A row's results from its statistics and the keys of its best elements (one lane a place); given: the token's logit, asked
// for when the row is.
__device__ __forceinline__ void write_row(const TokenParams &p, int64_t r, int32_t token, float given, const Stats &st, const uint64_t *keys, int lane)
{
    const float ls = logf(st.S);
    const bool dead = st.m == -kInf && st.S == 0.0f;
    const float logz = dead ? -kInf : st.m + ls;
    if (lane == 0) {
        if (p.logz) p.logz[r] = logz;
        if (p.entropy) p.entropy[r] = dead ? 0.0f : ls - st.T / st.S;
        if (p.logprobs) {
            p.logprobs[r] = dead && token < p.V ? -kInf : given - logz;
        }
    }
    if (lane < p.top) {
        const uint64_t k = keys[lane];
        const float x = value_of((uint32_t)(k >> 32));
        p.top_ids[r * p.top + lane] = k ? (int32_t)~(uint32_t)k : -1;
        p.top_logprobs[r * p.top + lane] = !k ? __builtin_nanf("") : x == -kInf ? -kInf : x - logz;
    }
}

__device__ __forceinline__ void write_padding(const TokenParams &p, int64_t r, int lane)
{
    if (lane == 0) {
        if (p.logz) p.logz[r] = 0.0f;
        if (p.entropy) p.entropy[r] = 0.0f;
        if (p.logprobs) p.logprobs[r] = 0.0f;
    }
    if (lane < p.top) {
        p.top_ids[r * p.top + lane] = -1;
        p.top_logprobs[r * p.top + lane] = 0.0f;
    }
}

// Statistics of what a wave holds: elements first + i * stride + j < n.
template <class T, int NV>
__device__ __forceinline__ Stats wave_stats(u32x4 (&raw)[NV], int first, int stride, int n, float (&peak)[NV], float &lane_max)
{
    constexpr int VE = Vec<T>::kN;
    float m = -kInf;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float v[VE];
        unpack<T>(raw[i], v);
        const int at = first + i * stride;
        if (at + VE > n) {                                    // places past the end hold -inf from here on
#pragma unroll
            for (int j = 0; j < VE; ++j) v[j] = at + j < n ? v[j] : -kInf;
            raw[i] = pack<T>(v);
        }
        peak[i] = -kInf;
#pragma unroll
        for (int j = 0; j < VE; ++j) peak[i] = fmaxf(peak[i], v[j]);
        m = fmaxf(m, peak[i]);
    }
    lane_max = m;
    m = max_wave(m);
#pragma unroll
    for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(raw[i]));   // (unpacked anew below, not kept as floats in twice the registers)
    const float base = m == -kInf ? 0.0f : m;
    float S = 0.0f, U = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float v[VE];
        unpack<T>(raw[i], v);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            const float d = v[j] - base, e = __builtin_amdgcn_exp2f(d * kLog2E);
            S += e;
            U = fmaf(e, fmaxf(d, -1e30f), U);                 // (e is 0 where d is -inf)
        }
    }
    return {m, sum_wave(S), sum_wave(U)};
}

// WAVES waves hold a row, or a workgroup's chunk of one (SPLIT); with one wave a row a workgroup has four rows at a time.
template <class T, int WAVES, int NV, bool SPLIT>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64, NV * Vec<T>::kN <= 8 ? 8 : NV * Vec<T>::kN <= 16 ? 6 : 4) void fb_token_logprobs_kernel(TokenParams p)
{
    constexpr int VE = Vec<T>::kN, kRows = WAVES == 1 ? 4 : 1, kW = WAVES == 1 ? 4 : WAVES;
    __shared__ uint64_t list[kW][64], best[kW][FB_TOP_MAX];
    __shared__ Stats stats[kW];
    __shared__ uint64_t row_best[FB_TOP_MAX];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? wave : 0);
    const int64_t r = SPLIT ? item / p.split : item;
    const int c = SPLIT ? (int)(item - r * p.split) : 0;
    if (r >= p.R) return;                                     // (a whole wave; with WAVES > 1 the whole workgroup)
    const int32_t token = p.tokens[r];
    if (!SPLIT && token < 0) {
        if (WAVES == 1 || wave == 0) write_padding(p, r, lane);
        return;
    }
    const int64_t at0 = SPLIT ? c * p.chunk : 0;
    const int n = (int)((SPLIT ? (p.V - at0 < p.chunk ? p.V - at0 : p.chunk) : p.V));
    const T *row = (const T *)p.logits + r * p.ld + at0;
    const int first = ((WAVES == 1 ? 0 : wave) * 64 + lane) * VE;
    constexpr int kStride = WAVES * 64 * VE;                  // (waves take turns: all of them have a share of a short row)
    u32x4 raw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = load_piece(row + first + i * kStride, n - (first + i * kStride));
    if (SPLIT && token < 0) return;                           // (few rows: not waited for before the row is asked for)
    const float given = SPLIT ? 0.0f : given_logit<T>(p, r, token);
    float peak[NV], lane_max;
    Stats st = wave_stats<T, NV>(raw, first, kStride, n, peak, lane_max);
    if (p.top) best_of_wave<T, NV>(row, raw, peak, lane_max, first, kStride, n, p.top, list[wave], best[wave]);
    lds_settled();
    const uint64_t *keys = best[wave];
    if constexpr (SPLIT) {
        const size_t list = (size_t)item * WAVES + wave;
        float *q = p.part + list * 3;
        if (lane == 0) {
            q[0] = st.m;
            q[1] = st.S;
            q[2] = st.T;
        }
        if (lane < p.top) {
            const uint64_t k = keys[lane];                    // numbers in the row instead of the chunk
            p.part_top[list * p.top + lane] = k ? (k & 0xffffffff00000000ull) | (uint32_t)~(~(uint32_t)k + (uint32_t)at0) : 0;
        }
        return;
    }
    if constexpr (WAVES > 1) {
        if (lane == 0) stats[wave] = st;
        __syncthreads();
        if (wave != 0) return;
        st = stats[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) st = join(st, stats[w]);
        if (p.top) {
            uint64_t last = ~0ull;                            // (zeros are no keys)
            for (int t = 0; t < p.top; ++t) {
                uint64_t b = 0;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const uint64_t k = lane < p.top ? best[w][lane] : 0;
                    if (k < last && k > b) b = k;
                }
                last = max_wave_key(b);
                if (lane == 0) row_best[t] = last;
            }
            lds_settled();
            keys = row_best;
        }
    }
    write_row(p, r, token, given, st, keys, lane);
}

// Rows of up to 512 elements with more than kTakenInTurn alternatives: a wave a row at a time, element 64 j + lane in the lane's
// j-th register, the next row asked for before this one is worked on.  The top-th largest is found bit by bit of its order,
// exactly, and what lies above it and as many of its equals as there is room for, in ascending order of their numbers, are
// ranked one a lane.  Bound by instruction issue, the bits for the most part: a comparison and a count each and register.
template <class T, int E>
__global__ __launch_bounds__(256) void fb_token_short_kernel(TokenParams p)
{
    __shared__ uint64_t list[4][FB_TOP_MAX], best[4][FB_TOP_MAX];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = (int)p.V;
    const int64_t step = (int64_t)gridDim.x * 4;
    int32_t next_token = -1;
    float next[E];
    auto ask = [&](int64_t r) {
        next_token = p.tokens[r];
        const T *row = (const T *)p.logits + r * p.ld;
#pragma unroll
        for (int j = 0; j < E; ++j) next[j] = j * 64 + lane < n ? load_one(row + j * 64 + lane) : -kInf;
    };
    int64_t r = (int64_t)blockIdx.x * 4 + wave;
    if (r < p.R) ask(r);
    for (; r < p.R; r += step) {
        const int32_t token = __builtin_amdgcn_readfirstlane(next_token);
        float v[E], m = -kInf;
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = next[j];
        if (r + step < p.R) ask(r + step);
        if (token < 0) {
            write_padding(p, r, lane);
            continue;
        }
#pragma unroll
        for (int j = 0; j < E; ++j) m = fmaxf(m, v[j]);
        m = max_wave(m);
        const float base = m == -kInf ? 0.0f : m;
        float S = 0.0f, U = 0.0f;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float d = v[j] - base, e = __builtin_amdgcn_exp2f(d * kLog2E);
            S += e;
            U = fmaf(e, fmaxf(d, -1e30f), U);                 // (e is 0 where d is -inf)
        }
        const Stats st = {m, sum_wave(S), sum_wave(U)};
        float given = v[0];
#pragma unroll
        for (int j = 1; j < E; ++j) given = token >> 6 == j ? v[j] : given;
        given = token < n ? __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(given), token & 63)) : __builtin_nanf("");
        uint32_t order[E];
#pragma unroll
        for (int j = 0; j < E; ++j) order[j] = j * 64 + lane < n ? order_of(v[j]) : 0;   // (0: below every number)
        uint32_t least = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t with = least | 1u << bit;
            int count = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) count += __popcll(__ballot(order[j] >= with));
            least = count >= p.top ? with : least;
        }
        int filled = 0;
#pragma unroll
        for (int equal = 0; equal < 2; ++equal)
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const bool in = equal ? order[j] == least : order[j] > least;
                const uint64_t hit = __ballot(in);
                const int at = filled + __popcll(hit & ((1ull << lane) - 1));
                if (in && at < p.top) list[wave][at] = (uint64_t)order[j] << 32 | (uint32_t)~(uint32_t)(j * 64 + lane);
                filled += __popcll(hit);
            }
        lds_settled();
        const uint64_t mine = lane < p.top ? list[wave][lane] : 0;
        const int rank = rank_in_wave(mine, p.top);
        if (lane < p.top) best[wave][rank] = mine;
        lds_settled();
        write_row(p, r, token, given, st, best[wave], lane);
        lds_settled();
    }
}

// Rows of up to 512 elements otherwise: four rows a wave, 16 lanes a row, so that a reduction takes 4 steps for four rows instead
// of 6 for one.  Alternatives are taken one after the other: the largest order left, and among those that have it the lowest
// number.  Bound by issue still: 69120 rows of 84 floats take 6.5 us, 1.4 us more for each alternative (a row a wave at a time:
// 14.5 us, with 3 alternatives 23 where they are taken in turn).  In turn and by the bits, 40000 rows: of 84, 20 alternatives
// 24 and 27 us; of 140, 37 and 40; of 300, 63 and 68: kTakenInTurn.
constexpr int kTakenInTurn = 24;

// Without PIECES element 16 j + l is in lane l's j-th register.  With them a lane has 16 bytes of the row at a time, the
// 16 i + l-th; the last, where it is not whole, ends at the row's end, and what it has in common with the one before counts
// there.  (16-bit rows of 500, 40000 of them: 12 us, one element at a time 24.  Up to 128 elements both are alike.)
template <class T, int E, bool PIECES>
__global__ __launch_bounds__(256) void fb_token_tiny_kernel(TokenParams p)
{
    const int lane = threadIdx.x & 63, l = lane & 15, n = (int)p.V;
    const int64_t at = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * 4 + (lane >> 4);
    const bool real = at < p.R;                               // (a row past the end: the last one again, not stored)
    const int64_t r = real ? at : p.R - 1;
    const int32_t token = p.tokens[r];
    const T *row = (const T *)p.logits + r * p.ld;
    constexpr int VE = PIECES ? Vec<T>::kN : 1;
    auto piece = [&](int e) { return (e / VE * 16 + l) * VE; };
    auto number = [&](int e) { return !PIECES || piece(e) < n - VE ? piece(e) + e % VE : n - VE + e % VE; };
    auto there = [&](int e) { return piece(e) < n && (!PIECES || number(e) >= piece(e)); };
    float v[E], m = -kInf;
    if constexpr (PIECES) {
#pragma unroll
        for (int e = 0; e < E; e += VE) unpack<T>(piece(e) < n ? *(const u32x4_any *)(row + number(e)) : u32x4{0, 0, 0, 0}, v + e);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = there(e) ? load_one(row + number(e)) : -kInf;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = there(e) ? v[e] : -kInf;
#pragma unroll
    for (int j = 0; j < E; ++j) m = fmaxf(m, v[j]);
    m = max_row16(m);
    const float base = m == -kInf ? 0.0f : m;
    float S = 0.0f, U = 0.0f, pick = v[0];
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const float d = v[j] - base, e = __builtin_amdgcn_exp2f(d * kLog2E);
        S += e;
        U = fmaf(e, fmaxf(d, -1e30f), U);                     // (e is 0 where d is -inf)
        pick = there(j) && number(j) == token ? v[j] : pick;
    }
    S = sum_row16(S);
    U = sum_row16(U);
    const bool live = token >= 0, dead = m == -kInf && S == 0.0f, known = token < n;
    const float given = __shfl(pick, (lane & 48) | (token / VE & 15));
    const float ls = logf(S), logz = dead ? -kInf : m + ls;
    if (real && l == 0) {
        if (p.logz) p.logz[r] = live ? logz : 0.0f;
        if (p.entropy) p.entropy[r] = live && !dead ? ls - U / S : 0.0f;
        if (p.logprobs) p.logprobs[r] = !live ? 0.0f : !known ? __builtin_nanf("") : dead ? -kInf : given - logz;
    }
    if (p.top == 0) return;
    uint32_t order[E];
#pragma unroll
    for (int j = 0; j < E; ++j) order[j] = there(j) ? order_of(v[j]) : 0;   // (0: below every number)
    for (int t = 0; t < p.top; ++t) {
        uint32_t mine = 0;
#pragma unroll
        for (int j = 0; j < E; ++j) mine = order[j] > mine ? order[j] : mine;
        const uint32_t win = over_row(mine, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
        uint32_t lowest = ~0u;
#pragma unroll
        for (int j = E - 1; j >= 0; --j) lowest = order[j] == win ? (uint32_t)number(j) : lowest;
        const uint32_t first = over_row(lowest, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
        if (lowest == first) {                                // one lane of the row
#pragma unroll
            for (int j = 0; j < E; ++j) order[j] = (uint32_t)number(j) == first ? 0 : order[j];
            if (real) {
                const float x = value_of(win);
                p.top_ids[r * p.top + t] = live ? (int32_t)first : -1;
                p.top_logprobs[r * p.top + t] = !live ? 0.0f : x == -kInf ? -kInf : x - logz;
            }
        }
    }
}

// What the waves that share a row have found joined, one wave a row.
template <class T, int WAVES>
__global__ __launch_bounds__(64) void fb_token_join_kernel(TokenParams p)
{
    __shared__ uint64_t best[FB_TOP_MAX], list[64], near[kKeysInLds];
    const int lane = threadIdx.x;
    const int64_t r = blockIdx.x;
    const int32_t token = p.tokens[r];
    const int lists = p.split * WAVES, n = lists * p.top;
    const uint64_t *keys = p.part_top + (size_t)r * n;
    const float *q = p.part + (size_t)r * lists * 3;
    // (all that is needed is asked for before any of it is looked at, also for a padded row, where nothing was written)
    Stats st = {-kInf, 0.0f, 0.0f};
    if (lane < lists) st = {q[3 * lane], q[3 * lane + 1], q[3 * lane + 2]};
    if (n <= kKeysInLds) {
        for (int i = lane; i < n; i += 512) {
            uint64_t k[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) k[u] = i + u * 64 < n ? keys[i + u * 64] : 0;
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i + u * 64 < n) near[i + u * 64] = k[u];
        }
    }
    if (token < 0) {
        write_padding(p, r, lane);
        return;
    }
    const float given = given_logit<T>(p, r, token);
    for (int c = lane + 64; c < lists; c += 64) st = join(st, {q[3 * c], q[3 * c + 1], q[3 * c + 2]});
#pragma unroll
    for (int step = 1; step < 64; step <<= 1) {
        const Stats o = {__shfl_xor(st.m, step), __shfl_xor(st.S, step), __shfl_xor(st.T, step)};
        st = join(st, o);
    }
    lds_settled();
    if (p.top) merge_lists(n <= kKeysInLds ? near : keys, lists, p.top, list, best);
    lds_settled();
    write_row(p, r, token, given, st, best, lane);
}

struct TokenGradParams {
    const void *logits;
    int64_t ld, R, V, ldd;
    const int32_t *tokens;
    const float *logz, *entropy, *g_logprobs, *g_entropy;
    void *dlogits;
    bool past;                 // dlogits goes past the caches
    int64_t pieces, items;     // pieces of 64 * kGradPieces vectors a row, and of all rows
};

constexpr int kGradPieces = 4;

// p = e^lp is 0 in single precision below this, and p (g + h (lp + H)) then too: with lp held here the bracket is finite for every h
// below 10^36, also where lp is -inf.
constexpr float kLeastLog = -128.0f;

// One element at a time is all there is to it: bound by memory.  A wave has 4 KB of a row.  4095 rows of 32001 in bfloat16
// (rows at odd addresses) take 103 us, 5.1 TB/s.
template <class T>
__global__ __launch_bounds__(256) void fb_token_logprobs_grad_kernel(TokenGradParams p)
{
    constexpr int VE = Vec<T>::kN, kWide = 64 * VE * kGradPieces;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= p.items) return;
    const int64_t r = item / p.pieces;
    const int64_t at0 = (item - r * p.pieces) * kWide;
    const int n = (int)(p.V - at0 < kWide ? p.V - at0 : kWide);
    const int32_t token = p.tokens[r];
    const float logz = p.logz[r];
    const bool live = token >= 0 && logz != -kInf;
    const T *row = (const T *)p.logits + r * p.ld + at0;
    T *out = (T *)p.dlogits + r * p.ldd + at0;
    const float g = p.g_logprobs ? p.g_logprobs[r] : 0.0f, h = p.g_entropy ? p.g_entropy[r] : 0.0f, ent = p.g_entropy ? p.entropy[r] : 0.0f;
    const float a = fmaf(h, ent, g);                          // -p (g + h (log p + H)) = -p (a + h log p)
    const int64_t hit = (int64_t)token - at0;
    u32x4 raw[kGradPieces];
    if (live) {
#pragma unroll
        for (int i = 0; i < kGradPieces; ++i) raw[i] = load_piece(row + (i * 64 + lane) * VE, n - (i * 64 + lane) * VE);
    }
#pragma unroll
    for (int i = 0; i < kGradPieces; ++i) {
        const int at = (i * 64 + lane) * VE;
        float v[VE];
        if (live) {
            unpack<T>(raw[i], v);
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const float lp = v[j] - logz, q = __builtin_amdgcn_exp2f(lp * kLog2E);
                v[j] = -q * fmaf(h, fmaxf(lp, kLeastLog), a);
                if (at + j == hit) v[j] += g;
            }
        } else {
#pragma unroll
            for (int j = 0; j < VE; ++j) v[j] = 0.0f;
        }
        store_piece(out + at, n - at, pack<T>(v), p.past);
    }
}

// The same for rows of up to 128 pieces, a piece a lane: `lanes` lanes, a power of two, have a row, so short ones fill the waves
// too.  (69120 rows of 84 in bfloat16: 10 us, by the kernel above 64; 20000 of 1000: 16 and 22; of 2000, 250 pieces: 27 and 28.)
template <class T>
__global__ __launch_bounds__(256) void fb_token_short_grad_kernel(TokenGradParams p, int lanes)
{
    constexpr int VE = Vec<T>::kN;
    const int l = threadIdx.x & (lanes - 1);
    const int64_t r = (int64_t)blockIdx.x * (256 / lanes) + threadIdx.x / lanes;
    const int at = l * VE, n = (int)p.V - at;
    if (r >= p.R || n <= 0) return;
    const int32_t token = p.tokens[r];
    const float logz = p.logz[r];
    const bool live = token >= 0 && logz != -kInf;
    const float g = p.g_logprobs ? p.g_logprobs[r] : 0.0f, h = p.g_entropy ? p.g_entropy[r] : 0.0f, ent = p.g_entropy ? p.entropy[r] : 0.0f;
    const float a = fmaf(h, ent, g);
    float v[VE];
    unpack<T>(load_piece((const T *)p.logits + r * p.ld + at, n), v);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
        const float lp = v[j] - logz, q = __builtin_amdgcn_exp2f(lp * kLog2E);
        const float d = -q * fmaf(h, fmaxf(lp, kLeastLog), a) + (at + j == token ? g : 0.0f);
        v[j] = live ? d : 0.0f;
    }
    store_piece((T *)p.dlogits + r * p.ldd + at, n, pack<T>(v));
}

// How a call is laid out.  Rows of up to 512 elements have kernels of their own (waves = 0).  Otherwise a wave holds up to 64
// elements a lane: rows of up to 4096 elements go to a wave each where there are enough of them to fill the GPU, else to four; rows that four waves cannot hold are split over workgroups,
// and so are long rows that are few.
struct TokenPlan {
    int waves, nv, split;
    int64_t chunk;
};

constexpr int kSplitWaves = 4;      // of a workgroup that has a share of a row
constexpr int kMostElements = 64;   // of a row, in a lane's registers

TokenPlan token_plan(int64_t R, int64_t V, int type)
{
    const int64_t ve = 16 / (int64_t)type_bytes(type);
    const int64_t vecs = (V + ve - 1) / ve, most = kMostElements / ve;
    TokenPlan t{};
    t.split = 1;
    if (V <= 512) return t;
    const int64_t one = 64, four = 256;
    if (vecs <= one * 2 || (vecs <= one * most && R >= 4 * kCUs)) {
        t.waves = 1;
        t.nv = (int)((vecs + one - 1) / one);
    } else {
        t.waves = kSplitWaves;
        int64_t split = (vecs + four * most - 1) / (four * most);
        // few rows: as many workgroups as the GPU has compute units, as long as each has 2 vectors a lane
        const int64_t fill = (kCUs + R - 1) / std::max<int64_t>(R, 1);
        if (split < fill) split = std::max(split, std::min(fill, (vecs + four * 2 - 1) / (four * 2)));
        const int64_t each = (vecs + split - 1) / split;
        t.nv = (int)((each + four - 1) / four);
        t.split = (int)((vecs + each - 1) / each);
        t.chunk = each * ve;
    }
    t.nv = t.nv <= 1 ? 1 : t.nv <= 2 ? 2 : t.nv <= 4 ? 4 : t.nv <= 8 ? 8 : t.nv <= 12 ? 12 : 16;
    return t;
}

template <class T, int WAVES, int NV>
void launch_tokens(const TokenParams &p, hipStream_t stream)
{
    const int64_t items = p.R * p.split, groups = WAVES == 1 ? (items + 3) / 4 : items;
    const dim3 block(WAVES == 1 ? 256 : WAVES * 64);
    if constexpr (NV * Vec<T>::kN <= kMostElements) {
        if constexpr (WAVES > 1) {
            if (p.split > 1) {
                hipLaunchKernelGGL((fb_token_logprobs_kernel<T, WAVES, NV, true>), dim3((unsigned)groups), block, 0, stream, p);
                return;
            }
        }
        hipLaunchKernelGGL((fb_token_logprobs_kernel<T, WAVES, NV, false>), dim3((unsigned)groups), block, 0, stream, p);
    }
}

template <class T>
int launch_tokens(const TokenParams &p, const TokenPlan &t, hipStream_t stream)
{
    if (t.waves == 0) {
        const dim3 grid((unsigned)std::min<int64_t>((p.R + 3) / 4, 32 * kCUs)), block(256);   // (bound by issue: 8, 16, 32 a unit: 26, 25, 24 us)
        const dim3 tiny((unsigned)((p.R + 15) / 16));
        if (p.top > kTakenInTurn) {
            if (p.V <= 64)
                hipLaunchKernelGGL((fb_token_short_kernel<T, 1>), grid, block, 0, stream, p);
            else if (p.V <= 128)
                hipLaunchKernelGGL((fb_token_short_kernel<T, 2>), grid, block, 0, stream, p);
            else if (p.V <= 256)
                hipLaunchKernelGGL((fb_token_short_kernel<T, 4>), grid, block, 0, stream, p);
            else
                hipLaunchKernelGGL((fb_token_short_kernel<T, 8>), grid, block, 0, stream, p);
        } else if (p.V <= 32) {
            hipLaunchKernelGGL((fb_token_tiny_kernel<T, 2, false>), tiny, block, 0, stream, p);
        } else if (p.V <= 64) {
            hipLaunchKernelGGL((fb_token_tiny_kernel<T, 4, false>), tiny, block, 0, stream, p);
        } else if (p.V <= 128) {
            hipLaunchKernelGGL((fb_token_tiny_kernel<T, 8, false>), tiny, block, 0, stream, p);
        } else if (p.V <= 256) {
            hipLaunchKernelGGL((fb_token_tiny_kernel<T, 16, true>), tiny, block, 0, stream, p);
        } else {
            hipLaunchKernelGGL((fb_token_tiny_kernel<T, 32, true>), tiny, block, 0, stream, p);
        }
        return launched("token log probability kernel launch: ");
    }
#define FB_TOKENS(W, N) launch_tokens<T, W, N>(p, stream)
    if (t.waves == 1) {
        switch (t.nv) {
        case 1: FB_TOKENS(1, 1); break;
        case 2: FB_TOKENS(1, 2); break;
        case 4: FB_TOKENS(1, 4); break;
        case 8: FB_TOKENS(1, 8); break;
        case 12: FB_TOKENS(1, 12); break;
        default: FB_TOKENS(1, 16); break;
        }
    } else {
        switch (t.nv) {
        case 1: FB_TOKENS(4, 1); break;
        case 2: FB_TOKENS(4, 2); break;
        case 4: FB_TOKENS(4, 4); break;
        case 8: FB_TOKENS(4, 8); break;
        case 12: FB_TOKENS(4, 12); break;
        default: FB_TOKENS(4, 16); break;
        }
    }
#undef FB_TOKENS
    int rc = launched("token log probability kernel launch: ");
    if (rc == FB_OK && p.split > 1) {
        hipLaunchKernelGGL((fb_token_join_kernel<T, kSplitWaves>), dim3((unsigned)p.R), dim3(64), 0, stream, p);
        rc = launched("token join kernel launch: ");
    }
    return rc;
}

// A launch has fewer than 2^32 threads: more rows than that leaves are worked on in several launches.
constexpr int64_t kRowsALaunch = (int64_t)1 << 22, kPiecesALaunch = (int64_t)1 << 24;

template <class T>
T *from_row(T *p, int64_t elements) { return p ? p + elements : p; }
inline const void *from_row(const void *p, int64_t elements, int type) { return (const char *)p + (size_t)elements * type_bytes(type); }

int launch_tokens(const TokenParams &p, const TokenPlan &t, int type, hipStream_t stream)
{
    if (type == FB_TYPE_F32) return launch_tokens<float>(p, t, stream);
    return type == FB_TYPE_BF16 ? launch_tokens<bf16>(p, t, stream) : launch_tokens<f16>(p, t, stream);
}

size_t stats_bytes(int64_t R, int split) { return ((size_t)R * split * kSplitWaves * 3 * sizeof(float) + 255) & ~(size_t)255; }

int check_tokens(const char *who, const void *logits, int64_t ld, const int32_t *tokens, int64_t R, int64_t V, int type)
{
    const std::string w(who);
    if (!known_type(type)) return fail(FB_EINVAL, w + ": unknown type");
    if (bad_rows(R) || bad_width(V)) return fail(FB_EINVAL, w + ": R must be 0 or more, V 1 or more, both below 2^31");
    if ((!logits || !tokens) && R > 0) return fail(FB_EINVAL, w + ": logits or tokens is NULL");
    if (bad_ld(ld, V)) return fail(FB_EINVAL, w + ": rows closer than V elements");
    return FB_OK;
}

}  // namespace

}  // namespace fb

extern "C" {

size_t fb_token_logprobs_workspace_bytes(int64_t R, int64_t V, int type, int top)
{
    using namespace fb;
    if (bad_rows(R) || bad_width(V) || !known_type(type) || top < 0 || top > FB_TOP_MAX || top > V) return 0;
    const TokenPlan t = token_plan(R, V, type);
    return t.split == 1 ? 0 : stats_bytes(R, t.split) + (((size_t)R * t.split * kSplitWaves * top * sizeof(uint64_t) + 255) & ~(size_t)255);
}

int fb_token_logprobs(const void *logits, int64_t ld, const int32_t *tokens, int64_t R, int64_t V, int type, int top,
                      float *logprobs, float *entropy, float *logz, int32_t *top_ids, float *top_logprobs, void *ws,
                      size_t ws_bytes, fb_stream stream)
{
    using namespace fb;
    return guarded([&]() -> int {
        const int rc = check_tokens("fb_token_logprobs", logits, ld, tokens, R, V, type);
        if (rc != FB_OK) return rc;
        if (top < 0 || top > FB_TOP_MAX || top > V) return fail(FB_EINVAL, "fb_token_logprobs: top must lie in 0 .. min(FB_TOP_MAX, V)");
        if (top > 0 && (!top_ids || !top_logprobs) && R > 0) return fail(FB_EINVAL, "fb_token_logprobs: top_ids or top_logprobs is NULL");
        const size_t need = fb_token_logprobs_workspace_bytes(R, V, type, top);
        if (need && (!ws || ws_bytes < need)) return fail(FB_EINVAL, "fb_token_logprobs: workspace missing or too small");
        if (R == 0) return FB_OK;
        const TokenPlan t = token_plan(R, V, type);
        TokenParams p{};
        p.logits = logits; p.ld = ld; p.R = R; p.V = V; p.tokens = tokens; p.top = top;
        p.logprobs = logprobs; p.entropy = entropy; p.logz = logz; p.top_ids = top_ids; p.top_logprobs = top_logprobs;
        p.split = t.split; p.chunk = t.chunk;
        p.part = (float *)ws;
        p.part_top = (uint64_t *)((char *)ws + (t.split > 1 ? stats_bytes(R, t.split) : 0));
        if (t.split > 1 && R * t.split >= kPiecesALaunch) return fail(FB_EUNSUPPORTED, "fb_token_logprobs: more than 2^24 pieces of long rows");
        for (int64_t r = 0; r < R; r += t.split > 1 ? R : kRowsALaunch) {
            TokenParams q = p;
            if (t.split == 1) {
                q.R = std::min(R - r, kRowsALaunch);
                q.logits = from_row(logits, r * ld, type);
                q.tokens = from_row(tokens, r);
                q.logprobs = from_row(logprobs, r); q.entropy = from_row(entropy, r); q.logz = from_row(logz, r);
                q.top_ids = from_row(top_ids, r * top); q.top_logprobs = from_row(top_logprobs, r * top);
            }
            const int e = launch_tokens(q, t, type, (hipStream_t)stream);
            if (e != FB_OK) return e;
        }
        return FB_OK;
    });
}

int fb_token_logprobs_grad(const void *logits, int64_t ld, const int32_t *tokens, const float *logz, const float *entropy,
                           const float *g_logprobs, const float *g_entropy, int64_t R, int64_t V, int type, void *dlogits,
                           int64_t ldd, fb_stream stream)
{
    using namespace fb;
    return guarded([&]() -> int {
        const int rc = check_tokens("fb_token_logprobs_grad", logits, ld, tokens, R, V, type);
        if (rc != FB_OK) return rc;
        if ((!logz || !dlogits || (g_entropy && !entropy)) && R > 0) return fail(FB_EINVAL, "fb_token_logprobs_grad: logz, dlogits or entropy is NULL");
        if (bad_ld(ldd, V)) return fail(FB_EINVAL, "fb_token_logprobs_grad: rows closer than V elements");
        if (R == 0) return FB_OK;
        TokenGradParams p{};
        p.logits = logits; p.ld = ld; p.R = R; p.V = V; p.ldd = ldd; p.tokens = tokens; p.logz = logz; p.entropy = entropy;
        p.g_logprobs = g_logprobs; p.g_entropy = g_entropy; p.dlogits = dlogits;
        p.past = goes_past(R, V, type);
        const int64_t ve = 16 / (int64_t)type_bytes(type), wide = 64 * kGradPieces * ve;
        p.pieces = (V + wide - 1) / wide;
        const int64_t rows = std::max<int64_t>(1, kPiecesALaunch / p.pieces);
        for (int64_t r = 0; r < R; r += rows) {
            TokenGradParams q = p;
            q.R = std::min(R - r, rows);
            q.items = q.R * p.pieces;
            q.logits = from_row(logits, r * ld, type);
            q.dlogits = (void *)from_row((const void *)dlogits, r * ldd, type);
            q.tokens = from_row(tokens, r);
            q.logz = from_row(logz, r); q.entropy = from_row(entropy, r);
            q.g_logprobs = from_row(g_logprobs, r); q.g_entropy = from_row(g_entropy, r);
            const dim3 grid((unsigned)((q.items + 3) / 4)), block(256);
            const int64_t row_pieces = (V + ve - 1) / ve;
            if (row_pieces <= 128) {
                int lanes = 1;
                while (lanes < row_pieces) lanes *= 2;
                const dim3 few((unsigned)((q.R * lanes + 255) / 256));
                if (type == FB_TYPE_F32)
                    hipLaunchKernelGGL(fb_token_short_grad_kernel<float>, few, block, 0, (hipStream_t)stream, q, lanes);
                else if (type == FB_TYPE_BF16)
                    hipLaunchKernelGGL(fb_token_short_grad_kernel<bf16>, few, block, 0, (hipStream_t)stream, q, lanes);
                else
                    hipLaunchKernelGGL(fb_token_short_grad_kernel<f16>, few, block, 0, (hipStream_t)stream, q, lanes);
            } else if (type == FB_TYPE_F32)
                hipLaunchKernelGGL(fb_token_logprobs_grad_kernel<float>, grid, block, 0, (hipStream_t)stream, q);
            else if (type == FB_TYPE_BF16)
                hipLaunchKernelGGL(fb_token_logprobs_grad_kernel<bf16>, grid, block, 0, (hipStream_t)stream, q);
            else
                hipLaunchKernelGGL(fb_token_logprobs_grad_kernel<f16>, grid, block, 0, (hipStream_t)stream, q);
        }
        return launched("token log probability gradient kernel launch: ");
    });
}

}  // extern "C"
