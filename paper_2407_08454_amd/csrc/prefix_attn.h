// Building blocks of attention over shared prefixes and paged tails (prefix_attn.hip): which keys a query sees, key tiles
// of 32 rows in LDS, and the softmax-weighted sum over them on the matrix cores.
//
// A wave works on 32 queries (of one KV head) and takes keys 32 at a time.  Scores are formed transposed, S^T = K Q^T: in the 32x32
// result a lane holds sixteen keys of ONE query (its column), so maximum and sum of a softmax row stay inside the lane but
// for one exchange with the lane 32 above or below, and the weights, rounded, are already in the lanes in which the second product,
// O^T = V^T P^T, wants its right operand: its sixteen accumulators of key order 8 (i / 4) + 4 (l / 32) + i % 4 are two fragments of
// sixteen keys.  The left operand has to have the same keys in its lanes, one value row per lane: four keys of sixteen
// value columns at a time come out of LDS transposed (ds_read_b64_tr_b16; fp32: plain reads, its fragments hold one key).
#pragma once

#include "attn_tile.h"

namespace kvm {

constexpr float PX_NONE = -3.0e38f;      // maximum of no score: finite, so that no inf - inf arises

// Weights are exp2(score - reference).  The reference is put PX_LIFT below the maximum, and again when a score lies more than PX_SLACK above that,
// so that the accumulators are rarely scaled.  fp16: weights below 2^-25 are lost, and beside a first state that takes nearly all of the weight
// thousands of them are the output: with weights of up to 2^15 only what is below 2^-35 of the greatest is.
template <typename T> constexpr float PX_LIFT = Elem<T>::kDtype == KVM_F16 ? 10.f : 0.f;
template <typename T> constexpr float PX_SLACK = Elem<T>::kDtype == KVM_F16 ? 5.f : 8.f;

enum { PX_WIDE_NONE = 0, PX_WIDE_ROWS = 1, PX_WIDE_PREFIX = 2 };

struct PrefixAttnArgs {
    const void *q, *Kp, *Vp, *Kt, *Vt;
    const int32_t *lens, *row_start, *table, *new_lens, *kv_lens;
    void *out;
    float *lse;
    float *part, *stat;                   // split calls: accumulators (query rows, parts, d), maximum and sum (query rows, parts, 2)
    int64_t q_stride;
    int B, T, H, G, P, cap, n_pages, page_shift, max_pages;
    int tiles_p, tiles_t;                 // query tiles of all prompts (an upper bound with row_start), of one row
    int splits_p, splits_t;               // parts that a prefix and a tail are split into
    int wide;                             // which of the keys go to 128 queries at a time (PX_WIDE_*)
    int stream_p, stream_t;               // prefixes and tails of so many keys are read with the non-temporal hint
    float c;                              // log2(e) / sqrt(d): scores in base 2
};

// 16 bytes of zeros that stand for the rows behind a tile's last key and for missing pages: a key that nobody sees must not bring
// what lies in its memory into a product, where even a weight of zero would not take a NaN away.
static __device__ const u32x4 px_zeros = {0u, 0u, 0u, 0u};

// The prompt of row b, or -1, b the same for 32 lanes: the last whose first row is not behind b.  (The entries are counted, 32 at a time: a
// search would wait for one after the other.)
__device__ __forceinline__ int prefix_of(const PrefixAttnArgs &a, int b) {
    if (a.P == 0) return -1;
    if (!a.row_start) return b / (a.B / a.P);
    const int lane = threadIdx.x & 31;
    int starts = 0;
    for (int p = 0; p <= a.P; p += 32) {
        const uint64_t at = __ballot(p + lane <= a.P && a.row_start[min(p + lane, a.P)] <= b);
        starts += __popc((uint32_t)(at >> (threadIdx.x & 32)));
    }
    return starts >= 1 && starts <= a.P ? starts - 1 : -1;
}
__device__ __forceinline__ int prefix_len(const PrefixAttnArgs &a, int p, int h) {
    return p < 0 ? 0 : a.lens ? min(max(a.lens[(size_t)p * a.H + h], 0), a.cap) : a.cap;
}
__device__ __forceinline__ int tail_len(const PrefixAttnArgs &a, int b) {
    return a.table ? min(max(a.kv_lens[b], 0), a.max_pages << a.page_shift) : 0;
}
// keys of one of `splits` parts of n keys: whole tiles, two at least, so that a part has one to load while it works on another
__device__ __forceinline__ int part_keys(int n, int splits) { return max(((n + splits - 1) / splits + 31) & ~31, 64); }

// the same for the wide kernel, in tiles of 64 keys: those of the prefix, then those of the tail
__device__ __forceinline__ int wide_part(int n, int n_tail, int splits) {
    const int tiles = ((n + 63) >> 6) + ((n_tail + 63) >> 6);
    return max((tiles + splits - 1) / splits, 2);
}

// value of the lane 32 above or below
__device__ __forceinline__ float other_half(float v) {
    const uint32_t a = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? r0 : r1);
}

// ---- key tiles ------------------------------------------------------------------------------------

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// 32 rows of CH 16-byte chunks; chunk ch of row r sits at position ch ^ swz(r).  swz makes the sixteen rows that a score fragment
// reads at one chunk differ, and also the four rows of four chunks that a transposed read takes (fp32: the eight chunks of rows r and
// r + 4).
template <typename T> struct KeyTile {
    static constexpr int CH = Mma<T>::CHUNKS;
    static constexpr int SLOTS = 32 * CH;
    static constexpr int RPL = WAVE / CH;                     // rows per load instruction
    static constexpr int LOADS = 32 / RPL;
    static constexpr int ROWB = HEAD_DIM * (int)sizeof(T);
    static __device__ __forceinline__ int swz(int r) {
        return sizeof(T) == 2 ? ((r & 3) << 2) | ((r >> 2) & 3) : (r & 3) | ((r & 4) << 1) | ((r & 8) >> 1);
    }
};

// Byte offsets inside a tile that depend on the lane only.
template <typename T> struct TileLane {
    using KT = KeyTile<T>;
    static constexpr int VADDR = sizeof(T) == 2 ? 8 : 1;
    int src_row, src_pos;                                     // row (of RPL) and position that this lane's loads fill
    int kslot[8];                                             // score fragments: slots (fp32: the first eight of sixteen)
    int vaddr[VADDR];                                         // value fragments: bytes
    __device__ __forceinline__ TileLane(int lane) {
        src_row = lane / KT::CH;
        src_pos = lane % KT::CH;
        const int row = lane & 31, hf = lane >> 5;
#pragma unroll
        for (int f = 0; f < 8; ++f) kslot[f] = row * KT::CH + ((2 * f + hf) ^ KT::swz(row));
        if constexpr (sizeof(T) == 2) {
            const int k = (lane & 15) >> 2, col = (((lane >> 4) & 1) << 1) | ((lane >> 1) & 1);
#pragma unroll
            for (int i = 0; i < 8; ++i)                       // i = value block + 4 (row & 8)
                vaddr[i] = ((4 * hf + k) * KT::CH + ((((i & 3) ^ k) << 2) | (col ^ ((i >> 2) << 1) ^ hf))) * 16 + (lane & 1) * 8;
        } else {
            vaddr[0] = 0;
        }
    }
    __device__ __forceinline__ u32x4 kfrag(const u32x4 *tile, int f) const {
        // (fp32: chunks 16 .. 31 are the same positions sixteen further, as swz has four bits)
        return tile[kslot[f & 7] + (f >> 3) * 16];
    }
    // rows pos(lane) + 16-byte chunk of the source that load i of this lane fetches
    __device__ __forceinline__ int row_of(int i) const { return i * KT::RPL + src_row; }
    __device__ __forceinline__ int chunk_bytes(int i) const { return (src_pos ^ KT::swz(row_of(i))) * 16; }
};

// A row's page table, 64 entries at a time, one a lane.
struct PageWindow {
    const int32_t *table;
    int first = -(1 << 30), entry = -1, pages, n_pages;
    __device__ __forceinline__ PageWindow(const PrefixAttnArgs &a, int b) : table(a.table + (size_t)b * a.max_pages), pages(a.max_pages),
                                                                            n_pages(a.n_pages) {}
    __device__ __forceinline__ void load(int lo) {
        first = lo;
        const int i = lo + (int)(threadIdx.x & 63);
        entry = i < pages ? table[i] : -1;
        if (entry >= n_pages) entry = -1;
    }
    // entries of pages [lo, hi], hi - lo < 64 (wave-uniform)
    __device__ __forceinline__ void need(int lo, int hi) {
        if (lo < first || hi >= first + 64) load(lo);
    }
    __device__ __forceinline__ int page(int i) const { return __shfl(entry, i - first, WAVE); }
};

// Where the 32 rows of a tile are: `base`, the same for the wave, where they follow one another (a prefix, a page that holds all of
// them), else every lane has the place of row lane % 32.  In rows of the pool or the prefix.
template <typename T> struct TileRows {
    using KT = KeyTile<T>;
    uint64_t base;
    uint32_t lo, hi, there;                                   // there: which rows are there, one bit each
    bool in_order;
    __device__ __forceinline__ uint32_t of_prefix(uint64_t first, int j0, int n) {
        base = first + j0;
        there = n - j0 >= 32 ? 0xFFFFFFFFu : (1u << (n - j0)) - 1;
        in_order = n - j0 >= 32;
        lo = (uint32_t)(base + (threadIdx.x & 31));
        hi = (uint32_t)((base + (threadIdx.x & 31)) >> 32);
        return there;
    }
    // tokens [j0, j0 + 32) of a row's pages, below n
    __device__ __forceinline__ uint32_t of_tail(const PrefixAttnArgs &a, PageWindow &win, int h, int j0, int n) {
        const int shift = a.page_shift, mask = (1 << shift) - 1, last = min(j0 + 31, n - 1);
        win.need(j0 >> shift, last >> shift);
        const uint32_t below = n - j0 >= 32 ? 0xFFFFFFFFu : (1u << (n - j0)) - 1;
        const int j = min(j0 + (int)(threadIdx.x & 31), last);
        const int page = win.page(j >> shift);
        there = (uint32_t)__ballot(page >= 0) & below;
        in_order = shift >= 5 && there == 0xFFFFFFFFu;
        const uint64_t row = ((uint64_t)((int64_t)page * a.H + h) << shift) + (j & mask);
        lo = (uint32_t)row;
        hi = (uint32_t)(row >> 32);
        base = ((uint64_t)__builtin_amdgcn_readfirstlane(hi) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane(lo);
        return there;
    }
    // the tile of the keys or the values whose row 0 is at `src` -> LDS, asynchronously
    template <int HINT> __device__ __forceinline__ void load(const TileLane<T> &tl, const char *src, u32x4 *tile) const {
        if (in_order) {
            const char *first = src + base * KT::ROWB;
#pragma unroll
            for (int i = 0; i < KT::LOADS; ++i)
                __builtin_amdgcn_global_load_lds((gptr_t)(first + (uint32_t)(tl.row_of(i) * KT::ROWB + tl.chunk_bytes(i))), (lptr_t)(tile + i * WAVE), 16, 0, HINT);
        } else {
#pragma unroll
            for (int i = 0; i < KT::LOADS; ++i) {
                const int r = tl.row_of(i);
                const uint64_t row = ((uint64_t)(uint32_t)__shfl((int)hi, r, WAVE) << 32) | (uint32_t)__shfl((int)lo, r, WAVE);
                const char *at = (there >> r) & 1 ? src + row * KT::ROWB + tl.chunk_bytes(i) : (const char *)&px_zeros;
                __builtin_amdgcn_global_load_lds((gptr_t)at, (lptr_t)(tile + i * WAVE), 16, 0, HINT);
            }
        }
    }
};

// ---- 32 queries of a wave -------------------------------------------------------------------------

template <typename T> struct Queries {
    using M = Mma<T>;
    u32x4 q[M::FRAGS];
    f32x16 o[4];                          // O^T: value block, accumulator i = value 32 block + acc_row(i), column = query
    float m, l;                           // running reference (base 2) and this lane's part of the sum
    int sees;                             // tail tokens that this lane's query sees
    bool valid;
    int64_t row;                          // its row in out

    // query `lin` = (b T + t) G + g of head h, `end`: the first that is not this tile's
    __device__ __forceinline__ void init(const PrefixAttnArgs &a, int64_t lin, int64_t end, int h) {
        const int hf = (threadIdx.x >> 5) & 1;
        const int64_t token = lin / a.G;
        const int g = (int)(lin - token * a.G), b = (int)(token / a.T), t = (int)(token - (int64_t)b * a.T);
        valid = lin < end;
        sees = 0;
        if (valid) {
            const int n_new = clamp_len(a.new_lens, b, a.T), n_tail = tail_len(a, b);
            valid = t < n_new;
            sees = valid ? min(max(n_tail - n_new + t + 1, 0), n_tail) : 0;
        }
        row = token * (a.H * a.G) + h * a.G + g;
        const char *src = (const char *)((const T *)a.q + token * a.q_stride + (int64_t)(h * a.G + g) * HEAD_DIM);
#pragma unroll
        for (int f = 0; f < M::FRAGS; ++f) {
            u32x4 v = {0u, 0u, 0u, 0u};
            if (valid) v = *reinterpret_cast<const u32x4 *>(src + (2 * f + hf) * 16);
            q[f] = v;
        }
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        m = PX_NONE;
        l = 0.f;
    }

    __device__ __forceinline__ f32x16 scores(const TileLane<T> &tl, const u32x4 *kt) const {
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int f = 0; f < M::FRAGS; ++f) M::mma(s, tl.kfrag(kt, f), q[f]);
        return s;
    }

    // Keys that are not there, and the `left`-th and later ones, out of the scores.  (Bit by bit on the vector ALU: as conditions, sixteen
    // compares and selects, they took more scalar registers than there are.)
    __device__ __forceinline__ void mask(f32x16 &s, uint32_t there, int left) const {
        uint32_t seen = left >= 32 ? there : left <= 0 ? 0u : there & ((1u << left) - 1);
        seen >>= (threadIdx.x & 32) >> 3;                     // lanes from 32 on: keys four further
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float si = s[i];
            const uint32_t keep = (uint32_t)((int32_t)(seen << (31 - 8 * (i >> 2) - (i & 3))) >> 31);
            s[i] = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, si) & keep) | (0xFF800000u & ~keep));
        }
    }

    // the tile's weights, taken against a reference that lags behind the maximum
    __device__ __forceinline__ void weights(f32x16 &s, float c) {
        float top = max16(s);
        top = fmaxf(top, other_half(top)) * c;
        if (__ballot(top > m + (PX_LIFT<T> + PX_SLACK<T>))) {
            const float next = fmaxf(m, top - PX_LIFT<T>), scale = __builtin_amdgcn_exp2f(m - next);
            l *= scale;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= scale;
            m = next;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -m));
        float p0 = 0.f, p1 = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 2) { p0 += s[i]; p1 += s[i + 1]; }
        l += p0 + p1;
    }

    // the same for two tiles at once
    __device__ __forceinline__ void weights(f32x16 &s0, f32x16 &s1, float c) {
        float top = fmaxf(max16(s0), max16(s1));
        top = fmaxf(top, other_half(top)) * c;
        if (__ballot(top > m + (PX_LIFT<T> + PX_SLACK<T>))) {
            const float next = fmaxf(m, top - PX_LIFT<T>), scale = __builtin_amdgcn_exp2f(m - next);
            l *= scale;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= scale;
            m = next;
        }
        float p0 = 0.f, p1 = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) { s0[i] = __builtin_amdgcn_exp2f(fmaf(s0[i], c, -m)); p0 += s0[i]; }
#pragma unroll
        for (int i = 0; i < 16; ++i) { s1[i] = __builtin_amdgcn_exp2f(fmaf(s1[i], c, -m)); p1 += s1[i]; }
        l += p0 + p1;
    }

    // O^T += V^T P^T.  The weights go in as two numbers of the cache type, rounded and what the rounding left, so that all of the output's
    // error is its own rounding.  The rounded weight alone would add half a step of every weight: bf16, N(0, 1), 2.3e-3 of the output instead of
    // 1.7e-3, and which of the two a row gets must not hang on the others of its batch.  The second product costs nothing where keys and values are
    // waited for, 6 % where 128 queries share a prefix (64 rows 36.6 / 39.0 us), 27 % where the matrix cores are all there is (8 x 2048 tokens
    // 2.33 / 2.95 ms).
    __device__ __forceinline__ void values(const TileLane<T> &tl, const f32x16 &w, const u32x4 *vt) {
        if constexpr (sizeof(T) == 2) {
            const __attribute__((address_space(3))) char *base = (const __attribute__((address_space(3))) char *)(lptr_t)vt;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = w[8 * s + e];
                const typename Elem<T>::Raw p = Elem<T>::from_float(x);
                float y[8];
                Elem<T>::to_float(p, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] -= y[e];
                const u32x4 rest = __builtin_bit_cast(u32x4, Elem<T>::from_float(x));
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    typedef __attribute__((address_space(3))) s16x4 *tr_t;
                    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)(base + tl.vaddr[d] + (16 * s) * KeyTile<T>::ROWB)));
                    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)(base + tl.vaddr[4 + d] + (16 * s + 8) * KeyTile<T>::ROWB)));
                    const u32x4 v = {lo[0], lo[1], hi[0], hi[1]};
                    M::mma(o[d], v, __builtin_bit_cast(u32x4, p));
                    M::mma(o[d], v, rest);
                }
            }
        } else {
            const int lane = threadIdx.x & 63, hf = lane >> 5;
            const float *f = reinterpret_cast<const float *>(vt);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = 8 * (i >> 2) + (i & 3) + 4 * hf;
                const float wi = w[i];
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const float v = f[(r * KeyTile<T>::CH + ((8 * d + ((lane & 31) >> 2)) ^ KeyTile<T>::swz(r))) * 4 + (lane & 3)];
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, wi, o[d], 0, 0, 0);
                }
            }
        }
    }
};

// One key at a time, where infinities or NaN among the values must not meet a weight of zero (what a query does not see) or the rest of a
// rounded weight: every lane its own query and half of the dimensions; a query that does not see the key leaves it out altogether.  Rare, and a
// call of its own on a copy of the accumulators: inlined it took the registers of the tile loops (8 x 2048 new tokens 2.46 -> 2.97 ms).
struct LaneState { float o[4][16], m, l; };
struct KeySource { const void *K, *V; const int32_t *table; int n_pages, page_shift, H, h; float c; };   // table NULL: K and V are a list of rows
template <typename T>
static __device__ __attribute__((noinline)) void one_by_one(LaneState *st, KeySource src, const T *q, int sees, int first, int last)
{
    const int hf = (threadIdx.x >> 5) & 1;
    float o[4][16], m = st->m, l = st->l;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = st->o[d][i];
    for (int j = first; j < last; ++j) {
        size_t at = j;
        if (src.table) {
            const int page = src.table[j >> src.page_shift];
            if (page < 0 || page >= src.n_pages) continue;
            at = (((size_t)page * src.H + src.h) << src.page_shift) + (j & ((1 << src.page_shift) - 1));
        }
        const T *kr = (const T *)src.K + at * HEAD_DIM + 64 * hf, *vr = (const T *)src.V + at * HEAD_DIM + 4 * hf;
        float s = 0.f;
#pragma unroll
        for (int f = 0; f < 8; ++f) s += RowDot<T>::dot(Elem<T>::load(kr, f), Elem<T>::load(q + 64 * hf, f));
        s = (s + other_half(s)) * src.c;
        if (j >= sees) continue;
        const float next = fmaxf(m, s), scale = __builtin_amdgcn_exp2f(m - next), w = __builtin_amdgcn_exp2f(s - next);
        l = l * scale + (hf ? 0.f : w);                       // (the halves' sums are added in the end)
        m = next;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                T v[4];
                __builtin_memcpy(v, vr + 32 * d + 8 * i, sizeof(v));
#pragma unroll
                for (int e = 0; e < 4; ++e) o[d][4 * i + e] = o[d][4 * i + e] * scale + w * (float)v[e];
            }
    }
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) st->o[d][i] = o[d][i];
    st->m = m;
    st->l = l;
}
// tokens of row b or states of prefix (p, h)
template <typename T> __device__ __forceinline__ KeySource key_source(const PrefixAttnArgs &a, bool tail, int p, int b, int h) {
    const size_t at = ((size_t)max(p, 0) * a.H + h) * a.cap * HEAD_DIM;
    return {tail ? a.Kt : (const T *)a.Kp + at, tail ? a.Vt : (const T *)a.Vp + at, tail ? a.table + (size_t)b * a.max_pages : nullptr, a.n_pages,
            a.page_shift, a.H, h, a.c};
}
// states [first_p, last_p) of prefix (p, h) and tokens [first_t, last_t) of row b for a wave's queries; afresh: instead of what they have
template <typename T>
__device__ __forceinline__ void one_by_one(const PrefixAttnArgs &a, Queries<T> &qs, int p, int b, int h, int first_p, int last_p, int first_t, int last_t,
                                           bool afresh) {
    LaneState st;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) st.o[d][i] = afresh ? 0.f : qs.o[d][i];
    st.m = afresh ? PX_NONE : qs.m;
    st.l = afresh ? 0.f : qs.l;
    const int64_t HG = a.H * a.G, token = qs.valid ? qs.row / HG : 0, head = qs.valid ? qs.row - token * HG : 0;
    const T *q = (const T *)a.q + token * a.q_stride + head * HEAD_DIM;
#pragma unroll 1
    for (int tail = 0; tail < 2; ++tail) {                    // (a loop, so that the call stands here once)
        const int first = tail ? first_t : first_p, last = tail ? last_t : last_p;
        if (first >= last) continue;
        one_by_one<T>(&st, key_source<T>(a, tail, p, b, h), q, !qs.valid ? 0 : tail ? qs.sees : last, first, last);
    }
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) qs.o[d][i] = st.o[d][i];
    qs.m = st.m;
    qs.l = st.l;
}

// Infinities or NaN among the sums of weighted values of a wave's queries, whose weights themselves add up to a number: a value is infinite or NaN.  It
// may be behind a mask, or its weight may have been rounded, to zero or with a rest of the other sign, and have made a NaN of an
// infinity: the keys have to be taken one by one.
template <typename T>
__device__ __forceinline__ bool sums_broken(const Queries<T> &qs) {
    float finite = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) finite = fmaf(qs.o[d][i], 0.f, finite);
    const float l = qs.l + other_half(qs.l);
    return __ballot(qs.valid && finite != 0.f && l - l == 0.f) != 0;
}

// The infinities and NaN among values [first, last) of a list, added up: dimensions 2 lane and 2 lane + 1 (16-bit types).  A query that sees all of
// these keys has just that in such a dimension, whatever the weights.  One read of the values, where taking the keys one by one is a round trip each.
template <typename T>
static __device__ __forceinline__ void add_nonfinite(float sum[2], const KeySource &src, int first, int last) {
    for (int j = first, end; j < last; j = end) {
        size_t at = j;
        end = last;
        if (src.table) {
            const int page = src.table[j >> src.page_shift], mask = (1 << src.page_shift) - 1;
            end = min(last, (j | mask) + 1);
            if (page < 0 || page >= src.n_pages) continue;
            at = (((size_t)page * src.H + src.h) << src.page_shift) + (j & mask);
        }
        const T *row = (const T *)src.V + at * HEAD_DIM + 2 * (threadIdx.x & 63);
#pragma unroll 8
        for (int i = j; i < end; ++i, row += HEAD_DIM) {
            T v[2];
            __builtin_memcpy(v, row, sizeof(v));
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float x = (float)v[e];
                sum[e] += x - x == 0.f ? 0.f : x;
            }
        }
    }
}

// Does the value tile hold an infinity or a NaN?  Where some queries of a tile see a key that others do not (later tokens of the same
// step), a weight of zero would not keep it out of the others' sums.  (16-bit types: the wide kernel's.)
template <typename T>
__device__ __forceinline__ bool has_nonfinite(const u32x4 *vt) {
    constexpr uint32_t E = Elem<T>::kDtype == KVM_F16 ? 0x7C00u : 0x7F80u;
    const int lane = threadIdx.x & 63;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < KeyTile<T>::LOADS; ++i) {
        const u32x4 v = vt[i * WAVE + lane];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t x = v[k];
            bad |= (x & E) == E || ((x >> 16) & E) == E;
        }
    }
    return __ballot(bad) != 0;
}

}  // namespace kvm
