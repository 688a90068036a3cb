// Attention of new tokens over the compacted cache of their prompt and over their row's own pages:
//     out = sum_j w_j v_j,  w = softmax over all keys j that the query sees of q . k_j / sqrt(d).
// One pass over the keys with a running reference and sum (prefix_attn.h), the keys split into parts where there are few queries, a part's
// accumulators, reference and sum kept in fp32 in the workspace.
//
//   prefix_attn_split_kernel  32 queries and a part of their keys a wave.  The keys of a prefix are read once for 32 queries of
//                             all the prompt's rows; a row's own tail for the queries of that row.
//   prefix_attn_wide_kernel   128 queries a workgroup: many queries of one row, with all their keys, or the many rows of a prompt, with
//                             a part of their prefix (16-bit types)
//   prefix_attn_join_kernel   puts the parts of a query on one reference and adds them up
#include <algorithm>

#include "prefix_attn.h"

namespace kvm {

constexpr int PX_QUERIES = 32;           // of a wave
constexpr int PX_JOIN_ROWS = 8;          // query rows of a joining workgroup, 32 lanes each

// Query tile `tile` of `per_tile` queries of all prompts: its prompt and queries [lin, end) in the order (row, token, head of the group).
struct QueryTile { int p; int64_t lin, end; };
__device__ __forceinline__ QueryTile find_tile(const PrefixAttnArgs &a, int tile, int per_tile) {
    const int64_t per_row = (int64_t)a.T * a.G;
    QueryTile qt = {-1, 0, 0};
    if (!a.row_start) {
        const int64_t queries = (a.B / a.P) * per_row;
        const int tiles = (int)((queries + per_tile - 1) / per_tile);
        qt.p = tile / tiles;
        qt.lin = qt.p * queries + (int64_t)(tile - qt.p * tiles) * per_tile;
        qt.end = (qt.p + 1) * queries;
        return qt;
    }
    const int lane = threadIdx.x & 63;
    int before = 0;                                          // tiles of the prompts before these 64
    for (int p0 = 0; p0 < a.P; p0 += WAVE) {
        const int p = p0 + lane;
        int first = 0, last = 0;
        if (p < a.P) {
            first = min(max(a.row_start[p], 0), a.B);
            last = min(max(a.row_start[p + 1], first), a.B);
        }
        const int tiles = (int)(((last - first) * per_row + per_tile - 1) / per_tile);
        int sum = tiles;                                     // inclusive scan
#pragma unroll
        for (int d = 1; d < WAVE; d *= 2) {
            const int v = __shfl_up(sum, d, WAVE);
            if (lane >= d) sum += v;
        }
        const uint64_t reached = __ballot(before + sum > tile);
        if (reached) {
            const int at = __ffsll((unsigned long long)reached) - 1;
            qt.p = p0 + at;
            const int row0 = __shfl(first, at, WAVE), row1 = __shfl(last, at, WAVE);
            const int start = before + __shfl(sum - tiles, at, WAVE);
            qt.lin = row0 * per_row + (int64_t)(tile - start) * per_tile;
            qt.end = row1 * per_row;
            return qt;
        }
        before += __shfl(sum, WAVE - 1, WAVE);
    }
    return qt;
}

// A query's accumulators, maximum and sum into the workspace.
template <typename T>
__device__ __forceinline__ void store_part(const PrefixAttnArgs &a, const Queries<T> &qs, size_t at, float l) {
    const int lane = threadIdx.x & 63;
    float *dst = a.part + at * HEAD_DIM + 4 * (lane >> 5);
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 v = {qs.o[d][4 * i], qs.o[d][4 * i + 1], qs.o[d][4 * i + 2], qs.o[d][4 * i + 3]};
            *reinterpret_cast<f32x4 *>(dst + 32 * d + 8 * i) = v;
        }
    if (lane < 32) {
        a.stat[2 * at] = qs.m;
        a.stat[2 * at + 1] = l;
    }
}

// A query's output from the sum of its weighted values: four dimensions of lane `lane` of 32.
template <typename T>
__device__ __forceinline__ void store_out(const PrefixAttnArgs &a, int64_t row, int lane, float top, float total, const f32x4 &sum) {
    const float inv = total == 0.f ? 0.f : 1.f / total;
    T y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (T)(sum[i] * inv);
    __builtin_memcpy((T *)a.out + row * HEAD_DIM + lane * 4, y, sizeof(y));
    if (a.lse && lane == 0) a.lse[row] = total == 0.f ? -INFINITY : (top + __log2f(total)) * 0.69314718055994531f;
}

// parts that hold something of a prefix of n states
__device__ __forceinline__ int parts_of_prefix(const PrefixAttnArgs &a, int n) {
    const int part = a.wide ? wide_part(n, 0, a.splits_p) * 64 : part_keys(n, max(a.splits_p, 1));
    return (n + part - 1) / part;
}

// What bounds it: the read of the keys and values (fp32: the matrix cores, 8192 cycles a tile of 32 keys).  A wave has room for one tile of 32
// keys and one of their values in LDS: the next keys are asked for as soon as the scores are taken, the next values when they have been added
// up, so that one of the two is always on its way and mostly both; eight waves of a compute unit (fp32: four, of tiles twice as large) keep 128 KB
// on their way (two stages a wave, four waves: 37 rows over 2048 states and tails of up to 1000 tokens 88 us, this 72).  Nobody waits for anybody.  8 rows with tails of up to
// 16384 tokens, 1.76 GB: 284 us, 6.2 TB/s.
//   u: tail parts first (their keys are found by way of lengths and page table, and they may be the longer ones), then prefix parts.
template <typename T>
__device__ __forceinline__ void split_unit(const PrefixAttnArgs &a, int u, u32x4 *kt, u32x4 *vt)
{
    using KT = KeyTile<T>;
    const int lane = threadIdx.x & 63;
    const int units_t = a.B * a.tiles_t * a.H * a.splits_t;
    const bool tail = u < units_t;
    PageWindow win(a, 0);
    int h, s, b = 0, p = -1, j0, end, total, least = 0;       // least: tokens that every query of the tile sees
    int64_t lin, lin_end;
    if (!tail) {
        u -= units_t;
        // the query tiles of a part read the same keys: on one XCD
        const int groups = a.H * a.splits_p;
        int group, tile;
        if (groups % 8 == 0) {
            const int slot = u >> 3;
            group = slot / a.tiles_p * 8 + (u & 7);
            tile = slot % a.tiles_p;
        } else {
            group = u / a.tiles_p;
            tile = u % a.tiles_p;
        }
        h = group % a.H;
        s = group / a.H;
        const QueryTile qt = find_tile(a, tile, PX_QUERIES);
        p = qt.p;
        if (p < 0) return;
        lin = qt.lin;
        lin_end = qt.end;
        const int n = prefix_len(a, p, h), part = part_keys(n, a.splits_p);
        j0 = s * part;
        end = min(n, j0 + part);
        total = n;
    } else {
        s = u % a.splits_t;
        u /= a.splits_t;
        const int tile = u % a.tiles_t;
        u /= a.tiles_t;
        h = u % a.H;
        b = u / a.H;
        win = PageWindow(a, b);
        win.load(0);                                          // (on its way with the lengths)
        const int n_new = clamp_len(a.new_lens, b, a.T), n = tail_len(a, b), part = part_keys(n, a.splits_t);
        const int64_t row_lin = (int64_t)b * a.T * a.G;
        lin = row_lin + (int64_t)tile * PX_QUERIES;
        lin_end = row_lin + (int64_t)n_new * a.G;
        if (lin >= lin_end) return;
        const int t_first = (int)((lin - row_lin) / a.G), t_last = (int)((min(lin + PX_QUERIES, lin_end) - 1 - row_lin) / a.G);
        least = min(max(n - n_new + t_first + 1, 0), n);
        j0 = s * part;
        total = n;
        end = min(min(max(n - n_new + t_last + 1, 0), n), j0 + part);
    }
    if (j0 >= end) return;
    const bool stream = total >= (tail ? a.stream_t : a.stream_p);

    const TileLane<T> tl(lane);
    Queries<T> qs;
    TileRows<T> rows;                                        // of the tile that is loaded next
    const auto find = [&](int j) -> uint32_t {
        if (tail) return rows.of_tail(a, win, h, j, end);
        return rows.of_prefix(((size_t)p * a.H + h) * a.cap, j, end);
    };
    const char *K = (const char *)(tail ? a.Kt : a.Kp), *V = (const char *)(tail ? a.Vt : a.Vp);
    const auto load = [&](const char *src, u32x4 *tile) {
        if (stream) rows.template load<2>(tl, src, tile); else rows.template load<0>(tl, src, tile);
    };
    uint32_t next = find(j0);
    load(K, kt);
    load(V, vt);
    qs.init(a, lin + (lane & 31), lin_end, h);
    for (int j = j0; j < end; j += 32) {
        const uint32_t there = next;
        wait_vmcnt<KT::LOADS>();
        f32x16 x = qs.scores(tl, kt);
        wait_lds();
        if (j + 32 < end) {
            next = find(j + 32);
            load(K, kt);
            wait_vmcnt<KT::LOADS>();
        } else {
            wait_vmcnt<0>();
        }
        const bool mixed = tail && j + 32 > least;
        if (mixed || there != 0xFFFFFFFFu) {
            qs.mask(x, there, tail ? qs.sees - j : 32);
        }
        qs.weights(x, a.c);
        qs.values(tl, x, vt);
        wait_lds();
        if (j + 32 < end) load(V, vt);
    }
    wait_vmcnt<0>();
    if (sums_broken(qs)) one_by_one<T>(a, qs, p, b, h, tail ? 0 : j0, tail ? 0 : end, tail ? j0 : 0, tail ? end : 0, true);

    const float l = qs.l + other_half(qs.l);
    if (!qs.valid) return;
    store_part(a, qs, (size_t)qs.row * (a.splits_p + a.splits_t) + (tail ? a.splits_p + s : s), l);
}

template <typename T>
__global__ __launch_bounds__(WAVE, sizeof(T) == 2 ? 2 : 1) void prefix_attn_split_kernel(PrefixAttnArgs a)
{
    __shared__ u32x4 kt[KeyTile<T>::SLOTS], vt[KeyTile<T>::SLOTS];   // (two objects: see attn_lse_kernel)
    split_unit<T>(a, blockIdx.x, kt, vt);
}

// The same for many queries: a workgroup of four waves has 128 of them and takes 64 keys at a time, which its waves load together and share.
// What bounds it: matrix cores (49 % busy), vector ALU (48 %, their issue among it) and the fragments' way out of LDS beside one another: two
// workgroups a compute unit, two waves a SIMD, so one wave's exponentials meet the other's products by chance.  8 x 2048 tokens of 40 heads over
// 5734 states and their own: 2.8 ms, 680 TFLOP/s (1020 with the weights' second product), where a library product of 8192^3 reaches 1130.  Tried
// and slower, all without the second product, 2.1 ms: eight waves that change over between products and exponentials at barriers (2.35 ms:
// their LDS reads fall together), 64 queries a wave with a SIMD to itself (2.88), fragments read ahead (2.21), one half's exponentials written
// between the other's products (2.30).
//   ROWS: the queries of one row and all their keys, prefix and tail one after the other in tiles of 64, in one part or several;
//   else: the queries of a prompt's rows and a part of their prefix; the last workgroups have tail parts as above, one a wave.
constexpr int PX_WIDE = 128;

// A wave's share of a tile of 64 keys: rows r[0], r[1] of each half.
template <typename T> struct WideLoad {
    using KT = KeyTile<T>;
    static constexpr int N = KT::LOADS / 4;                   // load instructions of a wave per 32 rows of keys
    uint32_t off[N];
    int row[N], slot;
    __device__ __forceinline__ WideLoad(int wave, int lane) : slot(wave * N) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            row[i] = (wave * N + i) * KT::RPL + lane / KT::CH;
            off[i] = ((lane % KT::CH) ^ KT::swz(row[i])) * 16;
        }
    }
    // returns which keys are there
    __device__ __forceinline__ uint64_t prefix(const char *K, const char *V, int j0, int n, u32x4 *kt, u32x4 *vt) const {
        const char *kb = K + (size_t)j0 * KT::ROWB, *vb = V + (size_t)j0 * KT::ROWB;
        if (j0 + 64 <= n) {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const uint32_t at = (32 * s + row[i]) * KT::ROWB + off[i];
                    __builtin_amdgcn_global_load_lds((gptr_t)(kb + at), (lptr_t)(kt + s * KT::SLOTS + (slot + i) * WAVE), 16, 0, 0);
                    __builtin_amdgcn_global_load_lds((gptr_t)(vb + at), (lptr_t)(vt + s * KT::SLOTS + (slot + i) * WAVE), 16, 0, 0);
                }
            return ~0ull;
        }
        const uint64_t there = (1ull << (n - j0)) - 1;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t at = (32 * s + row[i]) * KT::ROWB + off[i];
                const bool ok = j0 + 32 * s + row[i] < n;
                const char *ks = ok ? kb + at : (const char *)&px_zeros, *vs = ok ? vb + at : (const char *)&px_zeros;
                __builtin_amdgcn_global_load_lds((gptr_t)ks, (lptr_t)(kt + s * KT::SLOTS + (slot + i) * WAVE), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((gptr_t)vs, (lptr_t)(vt + s * KT::SLOTS + (slot + i) * WAVE), 16, 0, 0);
            }
        return there;
    }
    __device__ __forceinline__ uint64_t tail(const PrefixAttnArgs &a, PageWindow &win, int h, int j0, int n, u32x4 *kt, u32x4 *vt) const {
        const int lane = threadIdx.x & 63, shift = a.page_shift, last = min(j0 + 63, n - 1);
        win.need(j0 >> shift, last >> shift);
        const int j = min(j0 + lane, last), page = win.page(j >> shift);
        uint64_t there = __ballot(page >= 0);
        if (n - j0 < 64) there &= (1ull << (n - j0)) - 1;
        const int64_t at_row = (((int64_t)page * a.H + h) << shift) + (j & ((1 << shift) - 1));
        const uint32_t lo = (uint32_t)at_row, hi = (uint32_t)(at_row >> 32);
        if (shift >= 6 && there == ~0ull) {                   // one page has them all, one after the other
            const uint64_t first = (((uint64_t)__builtin_amdgcn_readfirstlane(hi) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane(lo)) * KT::ROWB;
            return prefix((const char *)a.Kt + first, (const char *)a.Vt + first, 0, 64, kt, vt);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int r = 32 * s + row[i];
                const uint64_t at = (((uint64_t)(uint32_t)__shfl((int)hi, r, WAVE) << 32) | (uint32_t)__shfl((int)lo, r, WAVE)) * KT::ROWB + off[i];
                const bool ok = (there >> r) & 1;
                const char *ks = ok ? (const char *)a.Kt + at : (const char *)&px_zeros, *vs = ok ? (const char *)a.Vt + at : (const char *)&px_zeros;
                __builtin_amdgcn_global_load_lds((gptr_t)ks, (lptr_t)(kt + s * KT::SLOTS + (slot + i) * WAVE), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((gptr_t)vs, (lptr_t)(vt + s * KT::SLOTS + (slot + i) * WAVE), 16, 0, 0);
            }
        return there;
    }
};

template <typename T, bool ROWS>
__global__ __launch_bounds__(4 * WAVE, 2) void prefix_attn_wide_kernel(PrefixAttnArgs a)
{
    using KT = KeyTile<T>;
    __shared__ u32x4 k_a[2 * KT::SLOTS], v_a[2 * KT::SLOTS], k_b[2 * KT::SLOTS], v_b[2 * KT::SLOTS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = blockIdx.x;
    if (!ROWS && block >= a.tiles_p * a.H * a.splits_p) {
        const int u = __builtin_amdgcn_readfirstlane(4 * (block - a.tiles_p * a.H * a.splits_p) + wave), at = (wave & 1) * KT::SLOTS;
        if (u >= a.B * a.tiles_t * a.H * a.splits_t) return;
        if (wave < 2) split_unit<T>(a, u, k_a + at, v_a + at);
        else split_unit<T>(a, u, k_b + at, v_b + at);
        return;
    }
    const int tiles = ROWS ? a.B * a.tiles_t : a.tiles_p, splits = a.splits_p;
    const int groups = a.H * splits;
    int group, tile;
    if (groups % 8 == 0) {
        const int slot = block >> 3;
        group = slot / tiles * 8 + (block & 7);
        tile = slot % tiles;
    } else {
        group = block / tiles;
        tile = block % tiles;
    }
    const int h = group % a.H, part = group / a.H;
    int b = 0, p, n_tail = 0, n_new = 0;
    int64_t lin, lin_end, row_lin = 0;
    if (ROWS) {
        b = tile / a.tiles_t;
        tile = a.tiles_t - 1 - (tile - b * a.tiles_t);        // the last queries see most
        n_new = clamp_len(a.new_lens, b, a.T);
        n_tail = tail_len(a, b);
        row_lin = (int64_t)b * a.T * a.G;
        lin = row_lin + (int64_t)tile * PX_WIDE;
        lin_end = row_lin + (int64_t)n_new * a.G;
        if (lin >= lin_end) return;
        p = prefix_of(a, b);
    } else {
        const QueryTile qt = find_tile(a, tile, PX_WIDE);
        p = qt.p;
        if (p < 0) return;
        lin = qt.lin;
        lin_end = qt.end;
    }
    const int n = prefix_len(a, p, h), tiles_n = (n + 63) >> 6;
    // tail tokens that the first and the last query of these `count` see
    const auto sees = [&](int64_t q) { return min(max(n_tail - n_new + (int)((q - row_lin) / a.G) + 1, 0), n_tail); };
    const int most = ROWS ? sees(min(lin + PX_WIDE, lin_end) - 1) : 0;
    const int64_t first_q = lin + 32 * wave;
    const bool idle = first_q >= lin_end;
    const int wave_least = ROWS && !idle ? sees(first_q) : 0, wave_most = ROWS && !idle ? sees(min(first_q + 32, lin_end) - 1) : 0;
    const int per_part = wide_part(n, n_tail, splits);
    int v = part * per_part;
    const int v_end = min(v + per_part, tiles_n + ((most + 63) >> 6));
    Queries<T> qs;
    qs.init(a, first_q + (lane & 31), lin_end, h);
    int stop = n_tail;                                       // tail tokens from here on one at a time
    const int tail_end = min(wave_most, (v_end - tiles_n) * 64);
    if (v < v_end) {
        const TileLane<T> tl(lane);
        const WideLoad<T> wl(wave, lane);
        PageWindow win(a, b);
        const size_t at = ((size_t)max(p, 0) * a.H + h) * a.cap * KT::ROWB;
        const char *Kp = (const char *)a.Kp + at, *Vp = (const char *)a.Vp + at;
        auto load = [&](int v, u32x4 *kt, u32x4 *vt) -> uint64_t {
            if (!ROWS || v < tiles_n) return wl.prefix(Kp, Vp, 64 * v, n, kt, vt);
            return wl.tail(a, win, h, 64 * (v - tiles_n), most, kt, vt);
        };
        auto work = [&](int v, uint64_t there, const u32x4 *kt, const u32x4 *vt) {
            const bool tail = ROWS && v >= tiles_n;
            const int j = 64 * (v - tiles_n);
            if (idle || (tail && (j >= wave_most || stop < n_tail))) return;
            f32x16 x0 = qs.scores(tl, kt), x1 = qs.scores(tl, kt + KT::SLOTS);
            const bool mixed = tail && j + 64 > wave_least;
            if (mixed || there != ~0ull) {
                qs.mask(x0, (uint32_t)there, tail ? qs.sees - j : 64);
                qs.mask(x1, (uint32_t)(there >> 32), tail ? qs.sees - j - 32 : 64);
                if (mixed && a.T > 1 && (has_nonfinite<T>(vt) || has_nonfinite<T>(vt + KT::SLOTS))) { stop = j; return; }
            }
            qs.weights(x0, x1, a.c);
            qs.values(tl, x0, vt);
            qs.values(tl, x1, vt + KT::SLOTS);
        };
        uint64_t there_a = load(v, k_a, v_a), there_b = 0;
        for (;;) {
            wait_vmcnt<0>();
            wait_lds();
            barrier_no_fence();
            if (v + 1 < v_end) there_b = load(v + 1, k_b, v_b);
            work(v, there_a, k_a, v_a);
            if (++v >= v_end) break;
            wait_vmcnt<0>();
            wait_lds();
            barrier_no_fence();
            if (v + 1 < v_end) there_a = load(v + 1, k_a, v_a);
            work(v, there_b, k_b, v_b);
            if (++v >= v_end) break;
        }
    }
    // Sums that are not finite: of values that are not, which all of the wave's queries see (a tile that only some see has none), so
    // that each stands for itself in its dimension, or of finite ones beyond fp32: then all of the part once more.
    bool again = false;
    if (sums_broken(qs)) {
        const int first_p = 64 * part * per_part, last_p = min(n, 64 * v_end), first_t = 64 * max(part * per_part - tiles_n, 0);
        float sum[2] = {0.f, 0.f};
        add_nonfinite<T>(sum, key_source<T>(a, false, p, b, h), first_p, last_p);
        if (ROWS) add_nonfinite<T>(sum, key_source<T>(a, true, p, b, h), first_t, min(stop, tail_end));
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {                   // dimension 32 d + acc_row(i)
                const float own = qs.o[d][i], of_values = __shfl(sum[i & 1], 16 * d + 4 * (i >> 2) + 2 * (lane >> 5) + ((i & 3) >> 1), WAVE);
                if (of_values != 0.f) qs.o[d][i] = of_values;
                else again |= qs.valid && own - own != 0.f;
            }
        again = __ballot(again) != 0;
    }
    if (again || (ROWS && !idle && stop < tail_end)) {
        const int first_t = again ? 64 * max(part * per_part - tiles_n, 0) : stop;
        one_by_one<T>(a, qs, p, b, h, 64 * part * per_part, again ? min(n, 64 * v_end) : 0, first_t, ROWS ? tail_end : 0, again);
    }
    const float l = qs.l + other_half(qs.l);
    if (!qs.valid) return;
    if (ROWS && splits == 1) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T *dst = (T *)a.out + qs.row * HEAD_DIM + 4 * (lane >> 5);
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                T y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = (T)(qs.o[d][4 * i + e] * inv);
                __builtin_memcpy(dst + 32 * d + 8 * i, y, sizeof(y));
            }
        if (a.lse && lane < 32) a.lse[qs.row] = l == 0.f ? -INFINITY : (qs.m + __log2f(l)) * 0.69314718055994531f;
        return;
    }
    store_part(a, qs, (size_t)qs.row * (splits + a.splits_t) + part, l);
}

// ---- joining ---------------------------------------------------------------------------------------

// The parts of a query: GROUPS groups of 32 lanes a query row, four dimensions a lane, the parts dealt to the groups.  Bound by the way of
// a few bytes through the memory: each group's first JOIN_AHEAD parts are on their way before it is known which of them there are.
constexpr int JOIN_AHEAD = 4;
template <typename T, int GROUPS>
__global__ __launch_bounds__(PX_JOIN_ROWS * 32) void prefix_attn_join_kernel(PrefixAttnArgs a)
{
    __shared__ f32x4 sum_of[PX_JOIN_ROWS][32];
    __shared__ float top_of[PX_JOIN_ROWS], total_of[PX_JOIN_ROWS];
    const int HG = a.H * a.G, lane = threadIdx.x & 31, slot = threadIdx.x >> 5, g = slot % GROUPS;
    const int64_t row = (int64_t)blockIdx.x * (PX_JOIN_ROWS / GROUPS) + slot / GROUPS;
    const int64_t token = row / HG;
    const int b = (int)(token / a.T), t = (int)(token - (int64_t)b * a.T), h = (int)(row - token * HG) / a.G;
    const int parts = a.splits_p + a.splits_t;
    const size_t first = (size_t)row * parts;
    const bool there = b < a.B;
    f32x4 v[JOIN_AHEAD];
    float m[JOIN_AHEAD], l[JOIN_AHEAD];
#pragma unroll
    for (int i = 0; i < JOIN_AHEAD; ++i) {
        const int k = g + GROUPS * i;
        if (there && k < parts) {
            m[i] = a.stat[2 * (first + k)];
            l[i] = a.stat[2 * (first + k) + 1];
            v[i] = *reinterpret_cast<const f32x4 *>(a.part + (first + k) * HEAD_DIM + lane * 4);
        }
    }
    int used_p = 0, used_t = 0;
    bool valid = false;
    if (there) {
        const int n_new = clamp_len(a.new_lens, b, a.T);
        valid = t < n_new;
        const int n = prefix_len(a, prefix_of(a, b), h), n_tail = tail_len(a, b), sees = min(max(n_tail - n_new + t + 1, 0), n_tail);
        if (a.wide == PX_WIDE_ROWS) {
            const int part = wide_part(n, n_tail, a.splits_p);
            used_p = (((n + 63) >> 6) + ((sees + 63) >> 6) + part - 1) / part;
        } else {
            used_p = parts_of_prefix(a, n);
            const int part_t = part_keys(n_tail, max(a.splits_t, 1));
            used_t = (sees + part_t - 1) / part_t;
        }
    }
    const auto used = [&](int k) { return k < a.splits_p ? k < used_p : k - a.splits_p < used_t; };
    float top = PX_NONE;
#pragma unroll
    for (int i = 0; i < JOIN_AHEAD; ++i) {
        const int k = g + GROUPS * i;
        if (valid && k < parts && used(k)) top = fmaxf(top, m[i]);
        else m[i] = PX_NONE, l[i] = 0.f, v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    float total = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < JOIN_AHEAD; ++i) {
        const float scale = __builtin_amdgcn_exp2f(m[i] - top);
        total += l[i] * scale;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += v[i][e] * scale;
    }
    if (valid) {
        for (int k = g + GROUPS * JOIN_AHEAD; k < parts; k += GROUPS) {
            if (k >= used_p && k < a.splits_p) { k += (a.splits_p - 1 - k) / GROUPS * GROUPS; continue; }
            if (!used(k)) { if (k >= a.splits_p) break; continue; }
            const float mk = a.stat[2 * (first + k)], lk = a.stat[2 * (first + k) + 1];
            const f32x4 vk = *reinterpret_cast<const f32x4 *>(a.part + (first + k) * HEAD_DIM + lane * 4);
            const float next = fmaxf(top, mk), before = __builtin_amdgcn_exp2f(top - next), scale = __builtin_amdgcn_exp2f(mk - next);
            total = total * before + lk * scale;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = sum[e] * before + vk[e] * scale;
            top = next;
        }
    }
    if constexpr (GROUPS > 1) {
        sum_of[slot][lane] = sum;
        if (lane == 0) { top_of[slot] = top; total_of[slot] = total; }
        __syncthreads();
        if (g != 0) return;
        float all = top;
#pragma unroll
        for (int i = 1; i < GROUPS; ++i) all = fmaxf(all, top_of[slot + i]);
        const float own = __builtin_amdgcn_exp2f(top - all);
        total *= own;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] *= own;
#pragma unroll
        for (int i = 1; i < GROUPS; ++i) {
            const float scale = __builtin_amdgcn_exp2f(top_of[slot + i] - all);
            const f32x4 vi = sum_of[slot + i][lane];
            total += total_of[slot + i] * scale;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += vi[e] * scale;
        }
        top = all;
    }
    if (valid) store_out<T>(a, row, lane, top, total, sum);
}

// ---- host side ------------------------------------------------------------------------------------

// Parts of a list of keys that is `most` long at most, `units` of them at a time: as many as make `waves` of them, of 64 keys each at least;
// where there is more to read, four times as many, of 512 each, so that the last ones to end leave little of the chip idle.  (One row over 2048
// states, us, parts of 64 / 96 keys 9.0 / 12.7, 10 rows over 1433 in fp32 18.3 / 21.5; 8 rows with tails of up to 16384 tokens, 4 / 8 / 16 parts of a prefix 290 / 284 / 284.)
static int parts_for(int64_t units, int64_t most, int64_t waves)
{
    if (units <= 0 || most <= 0) return 0;
    const int64_t one_round = std::min<int64_t>(waves / units, (most + 63) / 64), rounds = std::min<int64_t>(4 * waves / units, most / 512);
    return (int)std::max<int64_t>(1, std::max(one_round, rounds));
}

static int tiles_of_prompts(const PrefixAttnArgs &a, int queries)
{
    const int64_t per_row = (int64_t)a.T * a.G;
    return (int)(a.row_start ? a.B * per_row / queries + a.P : a.P * (((int64_t)(a.B / a.P) * per_row + queries - 1) / queries));
}

// Keys and values that one wave reads carry the non-temporal hint where `rows` lists as long as theirs come to half the last-level cache: by
// a list's own length, as lengths are on the device.  (37 rows, 436 MB, us, without / with 89 / 73; 32 rows, 211 MB that the last-level cache
// still holds from the call before, 44 / 50.)
static int stream_keys(int64_t rows, const kvm_shape &sh)
{
    const int64_t per_key = rows * sh.H_kv * 2 * HEAD_DIM * (sh.dtype == KVM_F32 ? 4 : 2);
    return (int)std::min<int64_t>((LLC_BYTES / 2 + per_key - 1) / per_key, INT32_MAX);
}

static void plan(const kvm_shape &sh, const kvm_prefix *prefix, const kvm_pages *pages, PrefixAttnArgs &a)
{
    a.B = sh.B; a.T = sh.N; a.H = sh.H_kv; a.G = sh.G; a.new_lens = sh.seq_lens;
    const int64_t per_row = (int64_t)a.T * a.G;
    if (a.B * per_row == 0) return;                          // no query: nothing is launched, and below units are divided by
    if (prefix && prefix->P > 0 && prefix->capacity > 0) {
        a.Kp = prefix->K; a.Vp = prefix->V; a.lens = prefix->lens; a.row_start = prefix->row_start; a.P = prefix->P; a.cap = prefix->capacity;
    }
    if (pages && pages->n_pages > 0 && pages->max_pages > 0) {
        a.Kt = pages->K; a.Vt = pages->V; a.table = pages->table;
        a.n_pages = pages->n_pages; a.page_shift = __builtin_ctz((unsigned)pages->page_size); a.max_pages = pages->max_pages;
    }
    const int64_t tail_most = (int64_t)a.max_pages << a.page_shift;
    if (sh.dtype != KVM_F32) {
        const int64_t wide_rows = (int64_t)a.B * ((per_row + PX_WIDE - 1) / PX_WIDE) * a.H;
        const int64_t wide_prompts = a.P ? (a.B * per_row + PX_WIDE - 1) / PX_WIDE * a.H : 0;
        if (per_row >= PX_WIDE) {
            a.wide = PX_WIDE_ROWS;
            a.tiles_t = (int)((per_row + PX_WIDE - 1) / PX_WIDE);
            a.splits_p = (int)std::max<int64_t>(1, std::min<int64_t>(512 / wide_rows, (a.cap + tail_most) / 256));
            return;
        }
        // bf16, 8 KV heads, 6500 states, 64 tokens a tail, us both launches, by 32 / by 128 queries: 128 queries of a prompt share them 25.8 / 22.8,
        // 256 35.7 / 28.4, 1024 79 / 57
        if (a.P && a.B * per_row >= (int64_t)a.P * PX_WIDE) {
            a.wide = PX_WIDE_PREFIX;
            a.tiles_p = tiles_of_prompts(a, PX_WIDE);
            a.splits_p = (int)std::max<int64_t>(1, std::min<int64_t>(256 / wide_prompts, a.cap / 256));
        }
    }
    // A compute unit holds eight waves of the split kernel (fp32: four, by their registers and LDS, but it takes parts for eight all the same: half
    // as many, us, 16 rows of 4 tokens over 4000 states 87 instead of 48, 8 rows with tails of up to 2000 tokens 185 instead of 138, 4 rows with 8000
    // 71 instead of 77, one row 31 instead of 36).  The tails get parts for all of them, the prefixes for what the tails leave, a
    // quarter at least: their parts are joined for every one of their rows.  (32 rows of two prompts, us, both launches, prefixes and tails in 16
    // and 1 / 8 and 1 / 8 and 2 / 4 and 2 parts 57 / 52 / 44 / 47.)
    int64_t units_t = 0;
    if (a.table) {
        a.tiles_t = (int)((per_row + PX_QUERIES - 1) / PX_QUERIES);
        a.splits_t = parts_for((int64_t)a.B * a.tiles_t * a.H, tail_most, 2048);
        units_t = (int64_t)a.B * a.tiles_t * a.H * a.splits_t;
    }
    if (a.P && !a.wide) {
        const int64_t units = std::max<int64_t>((a.B * per_row + PX_QUERIES - 1) / PX_QUERIES, a.P) * a.H;
        a.tiles_p = tiles_of_prompts(a, PX_QUERIES);
        a.splits_p = parts_for(units, a.cap, std::max<int64_t>(512, std::min<int64_t>(2048 - units_t, 1024)));
        a.stream_p = a.B * per_row <= (int64_t)a.P * PX_QUERIES ? stream_keys(a.P, sh) : INT32_MAX;
    }
    a.stream_t = a.tiles_t == 1 ? stream_keys(a.B, sh) : INT32_MAX;
}

static int64_t query_rows(const PrefixAttnArgs &a) { return (int64_t)a.B * a.T * a.H * a.G; }
static bool direct(const PrefixAttnArgs &a) { return a.wide == PX_WIDE_ROWS && a.splits_p == 1; }

size_t prefix_attn_workspace_bytes(const kvm_shape &sh, const kvm_prefix *prefix, const kvm_pages *pages)
{
    PrefixAttnArgs a = {};
    plan(sh, prefix, pages, a);
    return (direct(a) ? 0 : (size_t)query_rows(a) * (a.splits_p + a.splits_t) * (HEAD_DIM + 2) * sizeof(float)) + 256;
}

template <typename T>
static kvm_status launch_t(const PrefixAttnArgs &a, hipStream_t st)
{
    kvm_status rc = KVM_OK;
    if constexpr (sizeof(T) == 2) {
        if (a.wide) {
            const int64_t units_t = (int64_t)a.B * a.tiles_t * a.H * a.splits_t;
            const int64_t blocks = a.wide == PX_WIDE_ROWS ? (int64_t)a.B * a.tiles_t * a.H * a.splits_p
                                                          : (int64_t)a.tiles_p * a.H * a.splits_p + (units_t + 3) / 4;
            ProfScope prof("prefix_attn_wide_kernel", st);
            if (a.wide == PX_WIDE_ROWS) hipLaunchKernelGGL((prefix_attn_wide_kernel<T, true>), dim3((unsigned)blocks), dim3(4 * WAVE), 0, st, a);
            else hipLaunchKernelGGL((prefix_attn_wide_kernel<T, false>), dim3((unsigned)blocks), dim3(4 * WAVE), 0, st, a);
            rc = check_launch("prefix_attn_wide_kernel");
            if (rc != KVM_OK || direct(a)) return rc;
        }
    }
    const int64_t units = a.wide ? 0 : (int64_t)a.tiles_p * a.H * a.splits_p + (int64_t)a.B * a.tiles_t * a.H * a.splits_t;
    if (units > 0) {
        ProfScope prof("prefix_attn_split_kernel", st);
        hipLaunchKernelGGL(prefix_attn_split_kernel<T>, dim3((unsigned)units), dim3(WAVE), 0, st, a);
        rc = check_launch("prefix_attn_split_kernel");
        if (rc != KVM_OK) return rc;
    }
    ProfScope prof("prefix_attn_join_kernel", st);
    const auto join = [&](auto kernel, int groups) {
        const int rows = PX_JOIN_ROWS / groups;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((query_rows(a) + rows - 1) / rows)), dim3(PX_JOIN_ROWS * 32), 0, st, a);
    };
    const int parts = a.splits_p + a.splits_t;
    if (parts <= JOIN_AHEAD) join(prefix_attn_join_kernel<T, 1>, 1);
    else if (parts <= 2 * JOIN_AHEAD) join(prefix_attn_join_kernel<T, 2>, 2);
    // (eight groups where rows are few, us by eight / four: 256 rows of 130 parts 12.8 / 20.7, 768 of 44 9.6 / 11.2, 1024 of 34 10.0 / 10.2, 1024 of 18
    // 8.4 / 8.2, 1280 of 18 9.3 / 8.7, 2048 of 20 11.3 / 10.6; by two groups 2048 rows take longer again)
    else if (parts <= 4 * JOIN_AHEAD || query_rows(a) > 1024) join(prefix_attn_join_kernel<T, 4>, 4);
    else join(prefix_attn_join_kernel<T, 8>, 8);
    return check_launch("prefix_attn_join_kernel");
}

kvm_status launch_prefix_attn(const kvm_shape &sh, const kvm_prefix *prefix, const kvm_pages *pages, const void *Q, int64_t q_stride,
                              const int32_t *kv_lens, void *out, float *lse, void *ws, hipStream_t st)
{
    PrefixAttnArgs a = {};
    plan(sh, prefix, pages, a);
    a.q = Q; a.q_stride = q_stride; a.kv_lens = kv_lens; a.out = out; a.lse = lse;
    a.part = (float *)ws;
    a.stat = a.part + (size_t)query_rows(a) * (a.splits_p + a.splits_t) * HEAD_DIM;
    a.c = (float)(1.4426950408889634 / sqrt((double)sh.d));
    switch (sh.dtype) {
    case KVM_F32: return launch_t<float>(a, st);
    case KVM_F16: return launch_t<half_t>(a, st);
    default: return launch_t<bf16_t>(a, st);
    }
}

}  // namespace kvm
