// Appending the tokens of a step to a paged cache, rotated to their positions on the way.
//
// Every pair (u, v) of a query or key head at position x turns by a = x f_i: (u cos a - v sin a, v cos a + u sin a); values are
// copied.  Each byte is read once and written once and a pair costs six operations, so the call is bound by memory, and
// by latency where few tokens come.
//
// A wave takes up to 8 * STEPS head rows of one token, eight rows at a time, eight lanes a row.  A lane holds the two 16-byte chunks
// that turn together: chunks u and u + rot/16 where dimensions i and i + rot/2 pair up, neighbouring chunks where 2i and
// 2i + 1 do; either way lane u of a row needs angles 8u .. 8u+7, the same for all rows of the token.  The wave's 64 lanes therefore
// work out one angle each, while the rows are on their way, and exchange them through LDS.  16384 tokens of 40 heads in fp16, 1.0 GB read and
// written: 172 us, 5.9 TB/s (a copy of 1 GiB runs at 5.2); one token 2.9 us, a launch.
#include "kvm_common.h"

namespace kvm {

constexpr int PA_BLOCK = 256;
constexpr int PA_WAVES = PA_BLOCK / WAVE;

struct AppendArgs {
    const void *q, *k, *v;
    void *q_out, *K, *V;
    const int32_t *new_lens, *past_lens, *pos_base, *table;
    const float *inv_freq;
    int32_t *kv_lens;
    int64_t q_stride, k_stride, v_stride;
    int B, T, H, HG, n_pages, page_shift, max_pages, rot, groups, token_blocks;
};

// cos and sin of x f, x an integer: in 64 bits down to a fraction of a turn, so that far positions keep their angle (x f in fp32 is off
// by 0.06 at x = 10^6).  From there fp32 caches go on in 64 bits, one rounding in the end: 2^-25 is all that a sine is off; with the fraction in
// fp32 it was 2^-23 (6 x 301 tokens 14.5 us either way).  16-bit types round 2^13 times as coarsely: the rest in fp32.
template <typename T> __device__ __forceinline__ float2 unit_at(int64_t x, float f) {
    double turns = (double)x * (double)f * 0.15915494309189533577;
    turns -= rint(turns);
    if constexpr (sizeof(T) == 4) {
        double s, c;
        sincospi(2.0 * turns, &s, &c);
        return make_float2((float)c, (float)s);
    } else {
        float s, c;
        sincospif((float)(2.0 * turns), &s, &c);
        return make_float2(c, s);
    }
}

template <typename T, int STEPS, bool INTERLEAVED, bool STREAM>
__global__ __launch_bounds__(PA_BLOCK) void paged_append_kernel(AppendArgs a)
{
    typedef typename Elem<T>::Raw Raw;
    __shared__ float2 units[PA_WAVES][WAVE];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int cap = a.max_pages << a.page_shift;
    if ((int)blockIdx.x >= a.token_blocks) {                  // the last workgroups add the lengths up
        const int b = ((int)blockIdx.x - a.token_blocks) * PA_BLOCK + (int)threadIdx.x;
        if (b < a.B) a.kv_lens[b] = (int)min((int64_t)min(max(a.past_lens[b], 0), cap) + clamp_len(a.new_lens, b, a.T), (int64_t)cap);
        return;
    }
    const int64_t index = (int64_t)blockIdx.x * PA_WAVES + wave;
    const int64_t token = index / a.groups;
    const int first = (int)(index - token * a.groups) * (8 * STEPS);
    if (token >= (int64_t)a.B * a.T) return;
    const int b = (int)(token / a.T), t = (int)(token - (int64_t)b * a.T);
    if (t >= clamp_len(a.new_lens, b, a.T)) return;

    const int rows = a.HG + 2 * a.H;                          // query heads, key heads, value heads
    const int u = lane & 7, half = a.rot >> 4;                // half: pairs of chunks that turn
    const bool turns = u < half;
    const int c0 = INTERLEAVED ? 2 * u : (turns ? u : 2 * u), c1 = INTERLEAVED || !turns ? 2 * u + 1 : u + half;

    Raw x0[STEPS], x1[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int r = first + i * 8 + (lane >> 3);
        if (r < rows) {
            const T *src = r < a.HG ? (const T *)a.q + token * a.q_stride + (int64_t)r * HEAD_DIM
                         : r < a.HG + a.H ? (const T *)a.k + token * a.k_stride + (int64_t)(r - a.HG) * HEAD_DIM
                                          : (const T *)a.v + token * a.v_stride + (int64_t)(r - a.HG - a.H) * HEAD_DIM;
            x0[i] = STREAM ? Elem<T>::load_stream(src, c0) : Elem<T>::load(src, c0);
            x1[i] = STREAM ? Elem<T>::load_stream(src, c1) : Elem<T>::load(src, c1);
        }
    }
    const int64_t slot = (int64_t)min(max(a.past_lens[b], 0), cap) + t;
    int page = -1;
    if (slot < cap) page = a.table[(int64_t)b * a.max_pages + (slot >> a.page_shift)];
    const int64_t x = slot + (a.pos_base ? a.pos_base[b] : 0);
    if (lane < a.rot / 2) units[wave][lane] = unit_at<T>(x, a.inv_freq[lane]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");    // (a wave's LDS operations stay in order: it holds the compiler)
    __builtin_amdgcn_wave_barrier();
    float2 w[8];
    if (turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = units[wave][8 * u + i];
    }

    const int64_t in_page = slot & ((1 << a.page_shift) - 1);
    const bool stored = page >= 0 && page < a.n_pages;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int r = first + i * 8 + (lane >> 3);
        if (r >= rows) continue;
        if (turns && r < a.HG + a.H) {
            float p[8], q[8], s[8], d[8];
            Elem<T>::to_float(x0[i], p);
            Elem<T>::to_float(x1[i], q);
            if (INTERLEAVED) {                                // pairs inside a chunk: p has angles 8u .. 8u+3, q the next four
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[2 * e] = p[2 * e] * w[e].x - p[2 * e + 1] * w[e].y;
                    s[2 * e + 1] = p[2 * e + 1] * w[e].x + p[2 * e] * w[e].y;
                    d[2 * e] = q[2 * e] * w[4 + e].x - q[2 * e + 1] * w[4 + e].y;
                    d[2 * e + 1] = q[2 * e + 1] * w[4 + e].x + q[2 * e] * w[4 + e].y;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[e] = p[e] * w[e].x - q[e] * w[e].y;
                    d[e] = q[e] * w[e].x + p[e] * w[e].y;
                }
            }
            x0[i] = Elem<T>::from_float(s);
            x1[i] = Elem<T>::from_float(d);
        }
        T *dst;
        if (r < a.HG) dst = (T *)a.q_out + (token * a.HG + r) * HEAD_DIM;
        else {
            if (!stored) continue;
            const int h = r < a.HG + a.H ? r - a.HG : r - a.HG - a.H;
            dst = (T *)(r < a.HG + a.H ? a.K : a.V) + ((((int64_t)page * a.H + h) << a.page_shift) + in_page) * HEAD_DIM;
        }
        if (STREAM) {
            Elem<T>::store_stream(dst, c0, x0[i]);
            Elem<T>::store_stream(dst, c1, x1[i]);
        } else {
            Elem<T>::store(dst, c0, x0[i]);
            Elem<T>::store(dst, c1, x1[i]);
        }
    }
}

template <typename T>
static kvm_status launch_t(AppendArgs &a, bool interleaved, hipStream_t st)
{
    const int rows = a.HG + 2 * a.H;
    ProfScope prof("paged_append_kernel", st);
    const auto run = [&](auto kernel, int steps) {
        a.groups = (rows + 8 * steps - 1) / (8 * steps);
        a.token_blocks = (int)(((int64_t)a.B * a.T * a.groups + PA_WAVES - 1) / PA_WAVES);
        hipLaunchKernelGGL(kernel, dim3((unsigned)(a.token_blocks + (a.B + PA_BLOCK - 1) / PA_BLOCK)), dim3(PA_BLOCK), 0, st, a);
    };
    // Steps that the last-level cache cannot hold carry the non-temporal hint, and a wave has eight rows instead of sixteen.  us, plain with 16 rows /
    // hint with 16 / hint with 8: 16384 tokens of 40 heads in fp16 (1.0 GB) 190 / 181 / 172, 8192 in fp32 194 / 202 / 179.  Plain with 8 rows, beside the
    // present choice: these two 176 / 169 and 179 / 181, 403 MB of fp16 74 / 70, 101 MB 17.9 / 17.3, 59 MB of fp32 13.6 / 13.7; where the
    // bytes are just the cache's (268 MB, and the same buffers every time) 42 / 51.
    if ((int64_t)a.B * a.T * rows * HEAD_DIM * (int)sizeof(T) * 2 >= LLC_BYTES)
        interleaved ? run(paged_append_kernel<T, 1, true, true>, 1) : run(paged_append_kernel<T, 1, false, true>, 1);
    else
        interleaved ? run(paged_append_kernel<T, 2, true, false>, 2) : run(paged_append_kernel<T, 2, false, false>, 2);
    return check_launch("paged_append_kernel");
}

kvm_status launch_paged_append(const kvm_shape &sh, const kvm_pages &pages, const kvm_rotation &rot, const void *q, int64_t q_stride,
                               const void *k, int64_t k_stride, const void *v, int64_t v_stride, const int32_t *past_lens,
                               const int32_t *pos_base, void *q_out, int32_t *kv_lens, hipStream_t st)
{
    AppendArgs a;
    a.q = q; a.k = k; a.v = v;
    a.q_out = q_out; a.K = pages.K; a.V = pages.V;
    a.new_lens = sh.seq_lens; a.past_lens = past_lens; a.pos_base = pos_base; a.table = pages.table;
    a.inv_freq = rot.inv_freq;
    a.kv_lens = kv_lens;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
    a.B = sh.B; a.T = sh.N; a.H = sh.H_kv; a.HG = q ? sh.H_kv * sh.G : 0;
    a.n_pages = pages.n_pages; a.page_shift = __builtin_ctz((unsigned)pages.page_size); a.max_pages = pages.max_pages;
    a.rot = rot.rot_dim;
    switch (sh.dtype) {
    case KVM_F32: return launch_t<float>(a, rot.interleaved != 0, st);
    case KVM_F16: return launch_t<half_t>(a, rot.interleaved != 0, st);
    default: return launch_t<bf16_t>(a, rot.interleaved != 0, st);
    }
}

}  // namespace kvm
