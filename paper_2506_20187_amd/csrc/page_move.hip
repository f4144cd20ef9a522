// kv_page_move: rows of the cache to other places of the same sequence and kv head, as page_evict_select lists them: keys, values,
// weights and the tokens' numbers; scales of 8-bit pages, abstracts and boundaries are kept up.
//
// Bytes-bound: a row is read once and written once.  With abstracts the pages that rows move to are read whole, since the key
// that was replaced may have been the page's largest or smallest.  A workgroup owns a (page that rows move to, kv head, tensor): an
// 8-bit page's scale may have to grow, and its codes with it.  The pairs are listed by their new place, so a page's pairs
// are neighbours; the workgroups of a (sequence, kv head) share its pairs equally and take the pages that begin in their share.
// Sources lie behind the kept length and are not written, but in the page that the kept length cuts: 8 bits leave that page to
// a second launch, when nobody reads it any more.
#include "page_common.h"

namespace leoam {

struct MoveArgs {
    const int32_t* moves;
    int m_max;
    const int32_t *move_count, *old_len, *new_len, *page_table;
    char *k_pages, *v_pages;
    float *k_scale, *v_scale, *weight;
    int32_t* token_id;
    char* abstract;
    int32_t *chunk_off, *n_chunks;
    int n_kv_heads, n_pages, page_shift, max_pages;
    int per_row;  // workgroups that share a (sequence, kv head) and tensor
    int cut;      // 1: only the page that the kept length cuts, 0: the others, -1: all
};

constexpr int kMoveThreads = 256, kMoveWaves = kMoveThreads / LEOAM_WAVE;

// eight channels (fp32: four) of a row as floats, of the stored type
template <typename T, typename S> __device__ __forceinline__ void stored_values(const uint4& w, float scale, float* y) {
    if constexpr (std::is_same<S, E4M3>::value) {
        unpack_e4m3(w.x, y);
        unpack_e4m3(w.y, y + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= scale;
    } else {
        unpack<T>(w, y);
    }
}

template <typename T, typename S> struct MoveShape {
    static constexpr bool k8 = std::is_same<S, E4M3>::value;
    static constexpr int EPL = T::kEpl, LPR = LEOAM_D / EPL, RPP = kMoveThreads / LPR;      // lanes to a row, rows to a pass
    static constexpr int LANEB = EPL * S::kBytes, ROWB = LEOAM_D * S::kBytes;
    static constexpr int BATCH = 4;                                                           // passes that are on their way together
};

template <typename S> __device__ __forceinline__ uint4 load_lane(const char* p) {
    if constexpr (std::is_same<S, E4M3>::value) {
        const uint2 w = *reinterpret_cast<const uint2*>(p);
        return make_uint4(w.x, w.y, 0, 0);
    } else {
        return load16(p, 0);
    }
}

// The smallest power of two s with amax <= 448 s, its exponent where s * code is a number of T (as an append has it).
template <typename T> __device__ __forceinline__ float move_scale_of(float amax) {
    if (!(amax > 0.f)) return 0.f;
    constexpr int kLow = T::kTag == LEOAM_F16 ? -15 : -100, kHigh = T::kTag == LEOAM_F16 ? 7 : 118;
    const uint32_t u = float_to_bits(amax);
    const int e = min(max((int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), kLow), kHigh);
    return bits_to_float((uint32_t)(e + 127) << 23);
}

template <typename T, typename S> __global__ __launch_bounds__(kMoveThreads) void page_move_kernel(MoveArgs a) {
    using M = MoveShape<T, S>;
    constexpr int EPL = M::EPL, LPR = M::LPR, RPP = M::RPP, BATCH = M::BATCH;
    constexpr bool k8 = M::k8;
    __shared__ int from[256];                            // the page's rows: which place moves there, -1: the row stays
    __shared__ int16_t rows[256];                        // the rows that are moved to, in order of the list (-1: left out)
    __shared__ float sh[kMoveWaves], sh_abs[kMoveWaves][2][LEOAM_D];
    __shared__ int sh_rows;
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE);
    const int col = (tid % LPR) * EPL, rg = tid / LPR, ps = 1 << a.page_shift, hkv = a.n_kv_heads;
    const int which = blockIdx.x & 1, unit = blockIdx.x >> 1, bh = unit / a.per_row, sharer = unit - bh * a.per_row;
    const int b = bh / hkv, h = bh - b * hkv;
    const int cap = a.max_pages << a.page_shift;
    const int old_len = uniform(min(max(a.old_len[b], 0), cap)), new_len = uniform(min(max(a.new_len[b], 0), old_len));
    if (new_len >= old_len) return;
    const int n = uniform(min(max(a.move_count[bh], 0), min(a.m_max, new_len)));
    const int32_t* moves = a.moves + (size_t)bh * a.m_max * 2;
    const int32_t* table = a.page_table + (size_t)b * a.max_pages;
    const int cut_page = new_len & (ps - 1) ? new_len >> a.page_shift : -1;
    const bool bounded = which == 0 && a.abstract;
    char* pool = which ? a.v_pages : a.k_pages;
    float* scales = which ? a.v_scale : a.k_scale;

    // page p, whose pairs begin at i0 (i0 == n: none)
    auto take = [&](int p, int i0) {
        const int id = uniform(table[p]);
        if ((uint32_t)id >= (uint32_t)a.n_pages) return;
        const size_t row_of_page = (size_t)id * hkv + h;
        if (tid < ps) {
            from[tid] = -1;
            rows[tid] = -1;      // (of a list that does not ascend the page's pairs may lie apart)
        }
        if (tid == 0) sh_rows = 0;
        __syncthreads();
        const int i = i0 + tid;
        if (i < n && tid < ps) {
            const int to = moves[2 * (size_t)i], src = moves[2 * (size_t)i + 1];
            if (to >> a.page_shift == p) {
                const bool fits = to < new_len && src >= new_len && src < old_len && (uint32_t)table[src >> a.page_shift] < (uint32_t)a.n_pages;
                if (fits) {
                    rows[tid] = (int16_t)(to & (ps - 1));
                    atomicMax(&sh_rows, tid + 1);
                    from[to & (ps - 1)] = src;
                    if (which == 0 && a.weight) a.weight[(size_t)bh * cap + to] = a.weight[(size_t)bh * cap + src];
                    if (which == 0 && a.token_id) a.token_id[(size_t)bh * cap + to] = a.token_id[(size_t)bh * cap + src];
                }
            }
        }
        __syncthreads();
        char* page = pool + (row_of_page << a.page_shift) * M::ROWB;
        const int n_rows = uniform(sh_rows);
        auto source = [&](int src, float& scale) {      // of a place behind the kept length
            const size_t row = (size_t)table[src >> a.page_shift] * hkv + h;
            if constexpr (k8) scale = scales[row];
            return pool + ((row << a.page_shift) + (src & (ps - 1))) * M::ROWB + col * S::kBytes;
        };
        float mx[EPL], mn[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
            mx[e] = -INFINITY;
            mn[e] = INFINITY;
        }
        auto extremes = [&](const float* y) {
#pragma unroll
            for (int e = 0; e < EPL; ++e) {
                mx[e] = fmaxf(mx[e], y[e]);
                mn[e] = fminf(mn[e], y[e]);
            }
        };
        if constexpr (!k8) {
            if (bounded) {      // every row of the page: from where it is or from where it comes
                const int valid = min(ps, new_len - (p << a.page_shift));
                for (int r0 = 0; r0 < valid; r0 += RPP * BATCH) {
                    uint4 w[BATCH];
                    int to[BATCH];
#pragma unroll
                    for (int u = 0; u < BATCH; ++u) {
                        const int r = min(r0 + u * RPP + rg, valid - 1), src = from[r];
                        float unused = 1.f;
                        to[u] = src < 0 ? -1 : r;
                        w[u] = load16(src < 0 ? page + (size_t)r * M::ROWB + col * S::kBytes : source(src, unused), 0);
                    }
#pragma unroll
                    for (int u = 0; u < BATCH; ++u) {
                        float y[EPL];
                        stored_values<T, S>(w[u], 1.f, y);
                        extremes(y);
                        if (to[u] >= 0) store16(page, (size_t)to[u] * M::ROWB + col * S::kBytes, w[u]);
                    }
                }
            } else {
                for (int j0 = 0; j0 < n_rows; j0 += RPP * BATCH) {
                    uint4 w[BATCH];
                    int to[BATCH];
#pragma unroll
                    for (int u = 0; u < BATCH; ++u) {
                        const int j = j0 + u * RPP + rg;
                        to[u] = j < n_rows ? rows[j] : -1;
                        float unused = 1.f;
                        if (to[u] >= 0) w[u] = load16(source(from[to[u]], unused), 0);
                    }
#pragma unroll
                    for (int u = 0; u < BATCH; ++u)
                        if (to[u] >= 0) store16(page, (size_t)to[u] * M::ROWB + col * S::kBytes, w[u]);
                }
            }
        } else {
            // All rows that move here, before anything is written: up to 256 of them, sixteen passes of sixteen.
            constexpr int PASSES = 256 / RPP;
            uint4 w[PASSES];
            float scale[PASSES], top = 0.f;
#pragma unroll
            for (int u = 0; u < PASSES; ++u) {
                scale[u] = -1.f;
                if (u * RPP >= ps) continue;
                const int src = from[u * RPP + rg];
                if (src >= 0) w[u] = load_lane<S>(source(src, scale[u]));
            }
#pragma unroll
            for (int u = 0; u < PASSES; ++u) {
                if (u * RPP >= ps || scale[u] < 0.f) continue;
                float y[EPL];
                stored_values<T, S>(w[u], scale[u], y);
#pragma unroll
                for (int e = 0; e < EPL; ++e) {
                    const float m = fabsf(y[e]);
                    top = fmaxf(top, m < INFINITY ? m : 0.f);
                }
            }
            const float old = scales[row_of_page];
            top = wave_extreme_f<true>(top);
            __syncthreads();
            if (lane == 0) sh[wave] = top;
            __syncthreads();
#pragma unroll
            for (int v = 0; v < kMoveWaves; ++v) top = fmaxf(top, sh[v]);
            const float now = fmaxf(old, move_scale_of<T>(top)), inv = now > 0.f ? 1.f / now : 0.f, f = old * inv;
            if (tid == 0 && now > old) scales[row_of_page] = now;
            const int valid = min(ps, new_len - (p << a.page_shift)), stored = min(ps, old_len - (p << a.page_shift));
#pragma unroll
            for (int u = 0; u < PASSES; ++u) {
                const int r = u * RPP + rg;
                if (u * RPP >= ps) continue;
                char* at = page + (size_t)r * M::ROWB + col;
                float y[EPL];
                if (scale[u] >= 0.f) {      // (448 * scale bounds it: an infinity is not stored in 8 bits)
                    stored_values<T, S>(w[u], scale[u], y);
#pragma unroll
                    for (int e = 0; e < EPL; ++e) y[e] = clamp_nan(y[e], 448.f * now) * inv;
                } else if (r < stored && (now > old || (bounded && r < valid))) {
                    const uint4 c = load_lane<S>(at);
                    unpack_e4m3(c.x, y);
                    unpack_e4m3(c.y, y + 4);
                    if (now > old) {
#pragma unroll
                        for (int e = 0; e < EPL; ++e) y[e] *= f;
                    }
                } else {
                    continue;
                }
                const uint2 c = make_uint2(pack_e4m3(y), pack_e4m3(y + 4));
                if (scale[u] >= 0.f || now > old) *reinterpret_cast<uint2*>(at) = c;
                if (bounded && r < valid) {
                    stored_values<T, S>(make_uint4(c.x, c.y, 0, 0), now, y);
                    extremes(y);
                }
            }
        }
        if (bounded) {
#pragma unroll
            for (int e = 0; e < EPL; ++e) {
#pragma unroll
                for (int msk = LPR; msk < LEOAM_WAVE; msk <<= 1) {
                    mx[e] = fmaxf(mx[e], shfl_xor_f(mx[e], msk));
                    mn[e] = fminf(mn[e], shfl_xor_f(mn[e], msk));
                }
                if (lane < LPR) {
                    sh_abs[wave][0][col + e] = mx[e];
                    sh_abs[wave][1][col + e] = mn[e];
                }
            }
            __syncthreads();
            if (tid < LPR) {
#pragma unroll
                for (int v = 1; v < kMoveWaves; ++v)
#pragma unroll
                    for (int e = 0; e < EPL; ++e) {
                        mx[e] = fmaxf(mx[e], sh_abs[v][0][col + e]);
                        mn[e] = fminf(mn[e], sh_abs[v][1][col + e]);
                    }
                char* row = a.abstract + ((size_t)bh * a.max_pages + p) * 2 * Row<T>::kRowBytes;
                store16(row, col * T::kBytes, round_pack<T>(mx));
                store16(row, Row<T>::kRowBytes + col * T::kBytes, round_pack<T>(mn));
            }
        }
        __syncthreads();      // (the lists have been read)
    };

    const int last_page = (new_len - 1) >> a.page_shift;      // -1: nothing is kept
    if (a.cut == 1) {
        if (cut_page < 0) return;
        // the page's pairs are the last ones: the first of them
        int i0 = n;
        for (int i1 = n; i1 > 0 && i0 == i1; i1 -= LEOAM_WAVE) {
            const int i = i1 - LEOAM_WAVE + lane;
            const uint64_t hit = __ballot(i >= 0 && moves[2 * (size_t)max(i, 0)] >> a.page_shift >= cut_page);
            // (ascending: the hits are the upper lanes)
            i0 = i1 - __popcll(hit);
            if (hit != ~0ull) break;
        }
        if (i0 < n || bounded) take(cut_page, i0);
        return;
    }
    const int share0 = (int)((long long)n * sharer / a.per_row), share1 = (int)((long long)n * (sharer + 1) / a.per_row);
    for (int base = share0; base < share1; base += LEOAM_WAVE) {
        const int i = min(base + lane, share1 - 1);
        const int p = moves[2 * (size_t)i] >> a.page_shift, before = i > 0 ? moves[2 * (size_t)i - 2] >> a.page_shift : -1;
        uint64_t heads = __ballot(base + lane < share1 && p != before && p >= 0 && p <= last_page && (a.cut < 0 || p != cut_page));
        while (heads) {
            const int l = __builtin_ctzll(heads);
            heads &= heads - 1;
            take(__builtin_amdgcn_readlane(p, l), base + l);
        }
    }
    if (sharer + 1 < a.per_row || which) return;
    // what the sequence loses beside the rows that moved: the last page holds fewer tokens
    if (bounded && last_page >= 0 && (a.cut < 0 || last_page != cut_page) &&
        (n == 0 || uniform(moves[2 * (size_t)(n - 1)]) >> a.page_shift != last_page))
        take(last_page, n);
    if (h == 0 && tid == 0) {
        if (a.chunk_off) a.chunk_off[(size_t)b * (a.max_pages + 1) + last_page + 1] = new_len;
        if (a.n_chunks) a.n_chunks[b] = last_page + 1;
    }
}

constexpr int kMoveGroups = 8192;

template <typename T, typename S> static hipError_t launch_move(MoveArgs a, int rows, hipStream_t stream) {
    a.per_row = kMoveGroups / (2 * rows);
    if (a.per_row > a.m_max) a.per_row = a.m_max;
    if (a.per_row < 1) a.per_row = 1;
    a.cut = std::is_same<S, E4M3>::value ? 0 : -1;
    hipLaunchKernelGGL((page_move_kernel<T, S>), dim3(2 * rows * a.per_row), dim3(kMoveThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.cut < 0) return e;
    a.cut = a.per_row = 1;
    hipLaunchKernelGGL((page_move_kernel<T, S>), dim3(2 * rows), dim3(kMoveThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t page_move_dispatch(const leoam_pages* s, const int32_t* moves, int m_max, const int32_t* move_count, const int32_t* old_len,
                              const int32_t* new_len, const int32_t* page_table, void* k_pages, void* v_pages, float* k_scale,
                              float* v_scale, float* weight, int32_t* token_id, void* abstract, int32_t* chunk_off, int32_t* n_chunks,
                              hipStream_t stream) {
    MoveArgs a;
    a.moves = moves; a.m_max = m_max; a.move_count = move_count; a.old_len = old_len; a.new_len = new_len; a.page_table = page_table;
    a.k_pages = (char*)k_pages; a.v_pages = (char*)v_pages; a.k_scale = k_scale; a.v_scale = v_scale;
    a.weight = weight; a.token_id = token_id; a.abstract = (char*)abstract; a.chunk_off = chunk_off; a.n_chunks = n_chunks;
    a.n_kv_heads = s->n_kv_heads; a.n_pages = s->n_pages; a.page_shift = __builtin_ctz((unsigned)s->page_size); a.max_pages = s->max_pages;
    a.cut = -1; a.per_row = 1;
    const int rows = s->batch * s->n_kv_heads;
    const bool k8 = s->kv_dtype == LEOAM_E4M3;
    switch (s->q_dtype) {
    case LEOAM_F32: return launch_move<F32, F32>(a, rows, stream);
    case LEOAM_F16: return k8 ? launch_move<F16, E4M3>(a, rows, stream) : launch_move<F16, F16>(a, rows, stream);
    default: return k8 ? launch_move<BF16, E4M3>(a, rows, stream) : launch_move<BF16, BF16>(a, rows, stream);
    }
}

}  // namespace leoam
