// Attention of new tokens over the compacted cache of their prompt and over their row's own pages.
//
//   prefix_attn_row_kernel  a workgroup per query row: the keys dealt to its sixteen groups of sixteen lanes, each with the
//                           running maximum and sum of its keys' softmax; joined through LDS at the end.
#include <algorithm>

#include "kvm_common.h"

namespace kvm {

constexpr int PX_BLOCK = 256;
constexpr float PX_NONE = -3.0e38f;      // maximum of no score: finite, so that no inf - inf arises

struct PrefixAttnArgs {
    const void *q, *Kp, *Vp, *Kt, *Vt;
    const int32_t *lens, *row_start, *table, *new_lens, *kv_lens;
    void *out;
    float *lse;
    int64_t q_stride;
    int B, T, H, G, P, cap, n_pages, page_shift, max_pages;
    float c;                              // log2(e) / sqrt(d): scores in base 2
};

// The prompt of row b, or -1.  (The largest p with row_start[p] <= b, so that empty prompts are passed over.)
__device__ __forceinline__ int prefix_of(const PrefixAttnArgs &a, int b) {
    if (a.P == 0) return -1;
    if (!a.row_start) return b / (a.B / a.P);
    int lo = -1, hi = a.P;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.row_start[mid] <= b) lo = mid; else hi = mid;
    }
    return lo >= 0 && b < a.row_start[lo + 1] ? lo : -1;
}
__device__ __forceinline__ int prefix_len(const PrefixAttnArgs &a, int p, int h) {
    return p < 0 ? 0 : a.lens ? min(max(a.lens[(size_t)p * a.H + h], 0), a.cap) : a.cap;
}
__device__ __forceinline__ int tail_len(const PrefixAttnArgs &a, int b) {
    return a.table ? min(max(a.kv_lens[b], 0), a.max_pages << a.page_shift) : 0;
}

template <typename T>
__global__ __launch_bounds__(PX_BLOCK) void prefix_attn_row_kernel(PrefixAttnArgs a)
{
    typedef typename Elem<T>::Raw Raw;
    constexpr int GROUPS = PX_BLOCK / 16;
    __shared__ float acc_of[GROUPS][HEAD_DIM], m_of[GROUPS], l_of[GROUPS];
    const int HG = a.H * a.G;
    for (int64_t row = blockIdx.x; row < (int64_t)a.B * a.T * HG; row += gridDim.x) {      // (b, t, head)
    const int64_t token = row / HG;
    const int head = (int)(row - token * HG), h = head / a.G;
    const int b = (int)(token / a.T), t = (int)(token - (int64_t)b * a.T);
    const int n_new = clamp_len(a.new_lens, b, a.T);
    if (t >= n_new) continue;
    const int p = prefix_of(a, b), n_prefix = prefix_len(a, p, h);
    const int n_tail = min(max(tail_len(a, b) - n_new + t + 1, 0), tail_len(a, b));
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    const Raw q = Elem<T>::load((const T *)a.q + token * a.q_stride + (int64_t)head * HEAD_DIM, lane);

    float m = PX_NONE, l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int j = group; j < n_prefix + n_tail; j += GROUPS) {
        const T *kr, *vr;
        if (j < n_prefix) {
            const size_t at = (((size_t)p * a.H + h) * a.cap + j) * HEAD_DIM;
            kr = (const T *)a.Kp + at;
            vr = (const T *)a.Vp + at;
        } else {
            const int s = j - n_prefix, page = a.table[(size_t)b * a.max_pages + (s >> a.page_shift)];
            if (page < 0 || page >= a.n_pages) continue;
            const size_t at = ((((size_t)page * a.H + h) << a.page_shift) + (s & ((1 << a.page_shift) - 1))) * HEAD_DIM;
            kr = (const T *)a.Kt + at;
            vr = (const T *)a.Vt + at;
        }
        const float x = row16_sum(RowDot<T>::dot(Elem<T>::load(kr, lane), q)) * a.c;
        float v[8];
        Elem<T>::to_float(Elem<T>::load(vr, lane), v);
        const float top = fmaxf(m, x), scale = __builtin_amdgcn_exp2f(m - top), w = __builtin_amdgcn_exp2f(x - top);
        l = l * scale + w;
        m = top;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = acc[i] * scale + w * v[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) acc_of[group][lane * 8 + i] = acc[i];
    if (lane == 0) { m_of[group] = m; l_of[group] = l; }
    __syncthreads();
    if (threadIdx.x < 16) {
    float top = PX_NONE, total = 0.f, sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int g = 0; g < GROUPS; ++g) top = fmaxf(top, m_of[g]);
    for (int g = 0; g < GROUPS; ++g) {
        const float scale = __builtin_amdgcn_exp2f(m_of[g] - top);
        total += l_of[g] * scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += acc_of[g][lane * 8 + i] * scale;
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] *= inv;
    Elem<T>::store((T *)a.out + row * HEAD_DIM, lane, Elem<T>::from_float(sum));
    if (a.lse && lane == 0) a.lse[row] = total == 0.f ? -INFINITY : (top + __log2f(total)) * 0.69314718055994531f;
    }
    __syncthreads();
    }
}

size_t prefix_attn_workspace_bytes(const kvm_shape &sh, const kvm_prefix *prefix, const kvm_pages *pages) { return 256; }

kvm_status launch_prefix_attn(const kvm_shape &sh, const kvm_prefix *prefix, const kvm_pages *pages, const void *Q, int64_t q_stride,
                              const int32_t *kv_lens, void *out, float *lse, void *ws, hipStream_t st)
{
    PrefixAttnArgs a = {};
    a.q = Q; a.q_stride = q_stride; a.out = out; a.lse = lse;
    a.B = sh.B; a.T = sh.N; a.H = sh.H_kv; a.G = sh.G; a.new_lens = sh.seq_lens;
    if (prefix) {
        a.Kp = prefix->K; a.Vp = prefix->V; a.lens = prefix->lens; a.row_start = prefix->row_start; a.P = prefix->P; a.cap = prefix->capacity;
    }
    if (pages) {
        a.Kt = pages->K; a.Vt = pages->V; a.table = pages->table; a.kv_lens = kv_lens;
        a.n_pages = pages->n_pages; a.page_shift = __builtin_ctz((unsigned)pages->page_size); a.max_pages = pages->max_pages;
    }
    a.c = (float)(1.4426950408889634 / sqrt((double)sh.d));
    const dim3 grid((unsigned)std::min((int64_t)a.B * a.T * a.H * a.G, (int64_t)1 << 23));
    ProfScope prof("prefix_attn_row_kernel", st);
    switch (sh.dtype) {
    case KVM_F32: hipLaunchKernelGGL(prefix_attn_row_kernel<float>, grid, dim3(PX_BLOCK), 0, st, a); break;
    case KVM_F16: hipLaunchKernelGGL(prefix_attn_row_kernel<half_t>, grid, dim3(PX_BLOCK), 0, st, a); break;
    default: hipLaunchKernelGGL(prefix_attn_row_kernel<bf16_t>, grid, dim3(PX_BLOCK), 0, st, a);
    }
    return check_launch("prefix_attn_row_kernel");
}

}  // namespace kvm
