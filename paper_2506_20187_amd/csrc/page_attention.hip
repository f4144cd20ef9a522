// page_attention_decode / page_attention_prefill: softmax(scale q K^T) V over a sequence's pages.
//
// The plain kernel: one workgroup per (query row, kv head) walks the row's tokens, a group of lanes per token, with a
// running maximum, sum and accumulator per query head; the groups' states are folded at the end.
#include "page_common.h"

namespace leoam {

struct PageAttArgs {
    const char *q, *k_pages, *v_pages;
    const float *k_scale, *v_scale;
    const int32_t *page_table, *seq_len;
    const int32_t *new_off;                  // prompts: whose row a query is (nullptr: row b is sequence b's last token)
    const int32_t *sel_idx, *sel_count;      // kept pages (nullptr: all)
    int k_max, n_rows;
    float scale_log2;
    char* out;
    float* lse;
    float* partial;
    int batch, n_kv_heads, n_pages, page_size, page_shift, max_pages;
};

// physical page of entry `i` of the walk over sequence b's pages (kept pages of (b, h), or all), -1 if there is none;
// `logical` is its place in the sequence
__device__ __forceinline__ int page_at(const PageAttArgs& a, int b, const int32_t* sel, int i, int& logical) {
    logical = sel ? sel[i] : i;
    if (logical < 0 || logical >= a.max_pages) return -1;
    const int id = a.page_table[(size_t)b * a.max_pages + logical];
    return id >= 0 && id < a.n_pages ? id : -1;
}

template <typename T, typename S, int G, bool kPrompt>
__global__ __launch_bounds__(kAttThreads) void page_attention_vector_kernel(PageAttArgs a) {
    constexpr int EPL = T::kEpl, LPR = Row<T>::kLanesPerRow, NG = kAttThreads / LPR;
    constexpr bool k8 = std::is_same<S, E4M3>::value;
    constexpr int ROWB = LEOAM_D * S::kBytes, QROWB = Row<T>::kRowBytes;
    __shared__ float xw[NG][G][kPartStride];

    const int row = blockIdx.x / a.n_kv_heads, h = blockIdx.x % a.n_kv_heads;
    const int tid = threadIdx.x, col = (tid % LPR) * EPL, grp = tid / LPR;
    const int cap = a.max_pages * a.page_size;
    int b = row, len;
    if (kPrompt && a.new_off) {
        b = wave_count_below(a.batch, row, [&](int i) { return a.new_off[i]; });
        if (b >= a.batch) return;
        const int r0 = a.new_off[b], r1 = a.new_off[b + 1];
        if (row < r0 || row >= r1) return;
        len = a.seq_len[b] - (r1 - 1 - row);
    } else {
        len = a.seq_len[b];
    }
    len = min(max(len, 0), cap);
    const size_t bh = (size_t)b * a.n_kv_heads + h;
    const int32_t* sel = a.sel_idx ? a.sel_idx + bh * (size_t)a.k_max : nullptr;
    const int n_entries = sel ? min(max(a.sel_count[bh], 0), a.k_max) : (len + a.page_size - 1) >> a.page_shift;

    float qs[G][EPL], acc[G][EPL], m_run[G], l_run[G];
    const size_t qhead = (size_t)row * a.n_kv_heads * G + (size_t)h * G;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        unpack<T>(load16(a.q, (qhead + g) * QROWB + (size_t)col * T::kBytes), qs[g]);
        m_run[g] = -INFINITY;
        l_run[g] = 0.f;
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
            qs[g][e] *= a.scale_log2;
            acc[g][e] = 0.f;
        }
    }
    for (int i = 0; i < n_entries; ++i) {
        int logical;
        const int id = page_at(a, b, sel, i, logical);
        if (id < 0) continue;
        const int n = min(len - logical * a.page_size, a.page_size);
        const size_t at = (size_t)id * a.n_kv_heads + h;
        const char* kp = a.k_pages + at * a.page_size * ROWB + (size_t)col * S::kBytes;
        const char* vp = a.v_pages + at * a.page_size * ROWB + (size_t)col * S::kBytes;
        float ks = 1.f, vs = 1.f;
        if (k8) {
            ks = a.k_scale[at];
            vs = a.v_scale[at];
        }
        for (int t = grp; t < n; t += NG) {
            float x[EPL], y[EPL];
            if constexpr (k8) {
                const uint2 kw = *reinterpret_cast<const uint2*>(kp + (size_t)t * ROWB);
                const uint2 vw = *reinterpret_cast<const uint2*>(vp + (size_t)t * ROWB);
                unpack_e4m3(kw.x, x);
                unpack_e4m3(kw.y, x + 4);
                unpack_e4m3(vw.x, y);
                unpack_e4m3(vw.y, y + 4);
            } else {
                unpack<T>(load16(kp, (size_t)t * ROWB), x);
                unpack<T>(load16(vp, (size_t)t * ROWB), y);
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float z = 0.f;
#pragma unroll
                for (int e = 0; e < EPL; ++e) z = fmaf(qs[g][e], x[e], z);
                z = row16_sum(z);
                if (LPR == 32) z += shfl_xor_f(z, 16);
                z *= ks;
                const float m = fmaxf(m_run[g], z);
                const float c = exp2_or_zero(m_run[g], m), p = exp2_or_zero(z, m);
                m_run[g] = m;
                l_run[g] = l_run[g] * c + p;
                const float pv = p * vs;
#pragma unroll
                for (int e = 0; e < EPL; ++e) acc[g][e] = fmaf(pv, y[e], acc[g][e] * c);
            }
        }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
#pragma unroll
        for (int e = 0; e < EPL; ++e) xw[grp][g][col + e] = acc[g][e];
        if (tid % LPR == 0) {
            xw[grp][g][LEOAM_D] = m_run[g];
            xw[grp][g][LEOAM_D + 1] = l_run[g];
        }
    }
    __syncthreads();
    for (int i = tid; i < G * LEOAM_D; i += kAttThreads) {
        const int g = i / LEOAM_D, d = i % LEOAM_D;
        float m = -INFINITY, l = 0.f, o = 0.f;
        for (int w = 0; w < NG; ++w) m = fmaxf(m, xw[w][g][LEOAM_D]);
        for (int w = 0; w < NG; ++w) {
            const float c = exp2_or_zero(xw[w][g][LEOAM_D], m);
            l += c * xw[w][g][LEOAM_D + 1];
            o += c * xw[w][g][d];
        }
        const float r = l == 0.f ? 0.f : o / l;      // (NaN stays)
        const size_t j = qhead + g;
        if (!kPrompt || T::kTag == LEOAM_F32) reinterpret_cast<float*>(a.out)[j * LEOAM_D + d] = r;
        else if (T::kTag == LEOAM_F16) reinterpret_cast<_Float16*>(a.out)[j * LEOAM_D + d] = (_Float16)r;
        else reinterpret_cast<__bf16*>(a.out)[j * LEOAM_D + d] = (__bf16)r;
        if (a.lse && d == 0) a.lse[j] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    }
}

template <typename T, typename S, bool kPrompt>
static hipError_t launch_vector(const PageAttArgs& a, int group, hipStream_t stream) {
    const long long units = (long long)a.n_rows * a.n_kv_heads;
    if (units > 0x7fffffffll) return hipErrorInvalidValue;
    const dim3 grid((unsigned)units), block(kAttThreads);
    switch (group) {
    case 1: hipLaunchKernelGGL((page_attention_vector_kernel<T, S, 1, kPrompt>), grid, block, 0, stream, a); break;
    case 2: hipLaunchKernelGGL((page_attention_vector_kernel<T, S, 2, kPrompt>), grid, block, 0, stream, a); break;
    case 4: hipLaunchKernelGGL((page_attention_vector_kernel<T, S, 4, kPrompt>), grid, block, 0, stream, a); break;
    default: hipLaunchKernelGGL((page_attention_vector_kernel<T, S, 8, kPrompt>), grid, block, 0, stream, a); break;
    }
    return hipGetLastError();
}

template <bool kPrompt> static hipError_t attention_of(const leoam_pages* s, const PageAttArgs& a, hipStream_t stream) {
    const int group = s->n_q_heads / s->n_kv_heads;
    const bool k8 = s->kv_dtype == LEOAM_E4M3;
    switch (s->q_dtype) {
    case LEOAM_F32: return launch_vector<F32, F32, kPrompt>(a, group, stream);
    case LEOAM_F16:
        return k8 ? launch_vector<F16, E4M3, kPrompt>(a, group, stream) : launch_vector<F16, F16, kPrompt>(a, group, stream);
    default:
        return k8 ? launch_vector<BF16, E4M3, kPrompt>(a, group, stream) : launch_vector<BF16, BF16, kPrompt>(a, group, stream);
    }
}

size_t page_decode_workspace_bytes(const leoam_pages*);
size_t page_decode_min_workspace_bytes(const leoam_pages*);
size_t page_workspace_bytes(const leoam_pages* s, int n_new) {
    return n_new <= 0 ? page_decode_workspace_bytes(s) : page_decode_min_workspace_bytes(s);
}
size_t page_min_workspace_bytes(const leoam_pages* s) { return page_decode_min_workspace_bytes(s); }

static PageAttArgs args_of(const leoam_pages* s, const void* q, const void* k_pages, const void* v_pages, const float* k_scale,
                           const float* v_scale, const int32_t* page_table, const int32_t* seq_len, float softmax_scale,
                           void* out, float* lse, void* workspace) {
    PageAttArgs a = {};
    a.q = (const char*)q; a.k_pages = (const char*)k_pages; a.v_pages = (const char*)v_pages;
    a.k_scale = k_scale; a.v_scale = v_scale; a.page_table = page_table; a.seq_len = seq_len;
    a.scale_log2 = softmax_scale * kLog2e;
    a.out = (char*)out; a.lse = lse; a.partial = (float*)workspace;
    a.batch = s->batch; a.n_kv_heads = s->n_kv_heads; a.n_pages = s->n_pages; a.page_size = s->page_size;
    a.page_shift = __builtin_ctz((unsigned)s->page_size); a.max_pages = s->max_pages;
    return a;
}

hipError_t page_prefill_dispatch(const leoam_pages* s, const void* q, int n_new, const int32_t* new_off, const void* k_pages,
                                 const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* page_table,
                                 const int32_t* seq_len, float softmax_scale, void* out, float* lse, void* workspace, size_t,
                                 hipStream_t stream) {
    PageAttArgs a = args_of(s, q, k_pages, v_pages, k_scale, v_scale, page_table, seq_len, softmax_scale, out, lse, workspace);
    a.new_off = new_off; a.n_rows = n_new;
    return attention_of<true>(s, a, stream);
}

}  // namespace leoam
