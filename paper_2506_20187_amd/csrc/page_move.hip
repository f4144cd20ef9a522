// kv_page_move: rows of the cache to other places of the same sequence and kv head, as page_evict_select lists them: keys, values,
// weights and the tokens' numbers; scales of 8-bit pages, abstracts and boundaries are kept up.
//
// Bytes-bound: a row is read once and written once.  With abstracts the pages that rows move to are read whole, since the key
// that was replaced may have been the page's largest or smallest.  A wave owns a (page that rows move to, kv head, tensor): an
// 8-bit page's scale may have to grow, and its codes with it.  The pairs are listed by their new place, so a page's pairs
// are neighbours; the waves of a (sequence, kv head) share its pairs equally and take the pages that begin in their share.  A wave
// first looks up all rows that come (a lane each), then has as many of them on their way as its registers hold.
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
    int n_rows, per_row;  // (sequence, kv head) pairs, waves that share one's list
    int cut;      // 1: only the page that the kept length cuts, 0: the others, -1: all
};

constexpr int kMoveThreads = 256, kMoveWaves = kMoveThreads / LEOAM_WAVE;
constexpr int kMostRows = 256;      // of a page

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

// The smallest power of two s with amax <= 448 s, its exponent where s * code is a number of T (as an append has it).
template <typename T> __device__ __forceinline__ float move_scale_of(float amax) {
    if (!(amax > 0.f)) return 0.f;
    constexpr int kLow = T::kTag == LEOAM_F16 ? -15 : -100, kHigh = T::kTag == LEOAM_F16 ? 7 : 118;
    const uint32_t u = float_to_bits(amax);
    const int e = min(max((int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), kLow), kHigh);
    return bits_to_float((uint32_t)(e + 127) << 23);
}

template <typename T, typename S> __global__ __launch_bounds__(kMoveThreads, 4) void page_move_kernel(MoveArgs a) {
    constexpr bool k8 = std::is_same<S, E4M3>::value;
    constexpr int EPL = T::kEpl, LPR = LEOAM_D / EPL, RPL = LEOAM_WAVE / LPR;      // lanes to a row, rows to a load
    constexpr int ROWB = LEOAM_D * S::kBytes, BATCH = 8;                             // loads that are on their way together
    // a wave's page: where each row comes from (bytes into the pool, -1: it stays), by which scale, and the rows that come
    __shared__ long long sh_from[kMoveWaves][kMostRows];
    __shared__ float sh_scale[k8 ? kMoveWaves : 1][kMostRows];
    __shared__ int16_t sh_rows[kMoveWaves][kMostRows];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / LEOAM_WAVE);
    const int col = (lane % LPR) * EPL, rg = lane / LPR, ps = 1 << a.page_shift, hkv = a.n_kv_heads;
    const int which = blockIdx.x & 1, task = (int)(blockIdx.x >> 1) * kMoveWaves + wave, bh = task / a.per_row, sharer = task - bh * a.per_row;
    if (bh >= a.n_rows) return;
    const int b = bh / hkv, h = bh - b * hkv;
    const int cap = a.max_pages << a.page_shift;
    const int old_len = uniform(min(max(a.old_len[b], 0), cap)), new_len = uniform(min(max(a.new_len[b], 0), old_len));
    if (new_len >= old_len) return;
    const int n = uniform(min(max(a.move_count[bh], 0), min(a.m_max, new_len)));
    const int2* moves = reinterpret_cast<const int2*>(a.moves) + (size_t)bh * a.m_max;
    const int32_t* table = a.page_table + (size_t)b * a.max_pages;
    const int cut_page = new_len & (ps - 1) ? new_len >> a.page_shift : -1;
    const bool bounded = which == 0 && a.abstract;
    char* pool = (which ? a.v_pages : a.k_pages) + col * S::kBytes;
    float* scales = which ? a.v_scale : a.k_scale;
    long long* from = sh_from[wave];
    float* from_scale = sh_scale[k8 ? wave : 0];
    int16_t* rows = sh_rows[wave];

    // page p, whose pairs begin at i0 (i0 == n: none)
    auto take = [&](int p, int i0) {
        const int entry = table[p];
        int2 pair = moves[min(i0 + lane, max(n - 1, 0))];      // (m_max >= 1: there is an entry)
        for (int r = lane; r < ps; r += LEOAM_WAVE) from[r] = -1;
        const int id = uniform(entry);
        if ((uint32_t)id >= (uint32_t)a.n_pages) return;
        const size_t row_of_page = (size_t)id * hkv + h;
        const float old = k8 ? scales[row_of_page] : 1.f;
        int n_rows = 0;
        for (int j0 = 0; j0 < ps; j0 += LEOAM_WAVE) {
            const int i = i0 + j0 + lane;
            if (j0 > 0) pair = moves[min(i, n - 1)];
            const bool mine = i < n && j0 + lane < ps && pair.x >> a.page_shift == p, inside = mine && pair.x < new_len && pair.y >= new_len && pair.y < old_len;
            const int src_id = table[inside ? pair.y >> a.page_shift : p];
            const bool fits = inside && (uint32_t)src_id < (uint32_t)a.n_pages;
            const uint64_t hit = __ballot(fits);
            if (fits) {
                const size_t row = (size_t)src_id * hkv + h;
                const int to = pair.x & (ps - 1);
                from[to] = (long long)(((row << a.page_shift) + (pair.y & (ps - 1))) * ROWB);
                if constexpr (k8) from_scale[to] = scales[row];
                rows[n_rows + __popcll(hit & ((1ull << lane) - 1))] = (int16_t)to;
                if (which) {      // (the keys' waves have the abstracts to see to)
                    const size_t at = (size_t)bh * cap;
                    const float moved_weight = a.weight ? a.weight[at + pair.y] : 0.f;
                    const int moved_id = a.token_id ? a.token_id[at + pair.y] : 0;
                    if (a.weight) a.weight[at + pair.x] = moved_weight;
                    if (a.token_id) a.token_id[at + pair.x] = moved_id;
                }
            }
            n_rows += __popcll(hit);
            if (__ballot(mine) != ~0ull) break;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // (the lists are the wave's own)
        char* page = pool + (row_of_page << a.page_shift) * ROWB;
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
        const int valid = min(ps, new_len - (p << a.page_shift));
        if constexpr (!k8) {
            // every row of the page, from where it is or from where it comes; without abstracts the rows that come
            const int count = bounded ? valid : n_rows;
            for (int j0 = 0; j0 < count; j0 += RPL * BATCH) {
                uint4 w[BATCH];
                int to[BATCH];
#pragma unroll
                for (int u = 0; u < BATCH; ++u) {      // (rows past the last repeat it)
                    const int j = min(j0 + u * RPL + rg, count - 1), r = bounded ? j : rows[j];
                    const long long src = from[r];
                    to[u] = src < 0 ? -1 : r;
                    w[u] = load16(src < 0 ? page + (size_t)r * ROWB : pool + src, 0);
                }
#pragma unroll
                for (int u = 0; u < BATCH; ++u) {
                    if (bounded) {
                        float y[EPL];
                        unpack<T>(w[u], y);
                        extremes(y);
                    }
                    if (to[u] >= 0) store16(page, (size_t)to[u] * ROWB, w[u]);
                }
            }
        } else {
            // The scale comes before the codes: rows that come are read for their largest magnitude, and again if they are more than
            // the registers hold (from the cache).
            uint2 w[2 * BATCH];
            auto fetch = [&](int j0) {
#pragma unroll
                for (int u = 0; u < 2 * BATCH; ++u) {
                    const int r = rows[min(j0 + u * RPL + rg, n_rows - 1)];
                    w[u] = *reinterpret_cast<const uint2*>(pool + from[r]);
                }
            };
            auto value = [&](int u, int r, float* y) {
                unpack_e4m3(w[u].x, y);
                unpack_e4m3(w[u].y, y + 4);
                const float f = from_scale[r];
#pragma unroll
                for (int e = 0; e < EPL; ++e) y[e] *= f;
            };
            constexpr int kHeld = RPL * 2 * BATCH;
            float top = 0.f;
            for (int j0 = 0; j0 < n_rows; j0 += kHeld) {
                fetch(j0);
#pragma unroll
                for (int u = 0; u < 2 * BATCH; ++u) {
                    float y[EPL];
                    value(u, rows[min(j0 + u * RPL + rg, n_rows - 1)], y);
#pragma unroll
                    for (int e = 0; e < EPL; ++e) {
                        const float m = fabsf(y[e]);
                        top = fmaxf(top, m < INFINITY ? m : 0.f);
                    }
                }
            }
            const float now = fmaxf(old, move_scale_of<T>(wave_extreme_f<true>(top))), inv = now > 0.f ? 1.f / now : 0.f, f = old * inv;
            const bool grows = now > old;
            if (lane == 0 && grows) scales[row_of_page] = now;
            auto put = [&](int r, const float* y, bool store) {
                const uint2 c = make_uint2(pack_e4m3(y), pack_e4m3(y + 4));
                if (store) *reinterpret_cast<uint2*>(page + (size_t)r * ROWB) = c;
                if (bounded && r < valid) {
                    float z[EPL];
                    stored_values<T, S>(make_uint4(c.x, c.y, 0, 0), now, z);
                    extremes(z);
                }
            };
            for (int j0 = 0; j0 < n_rows; j0 += kHeld) {
                if (n_rows > kHeld) fetch(j0);
#pragma unroll
                for (int u = 0; u < 2 * BATCH; ++u) {
                    const int j = j0 + u * RPL + rg, r = rows[min(j, n_rows - 1)];
                    float y[EPL];
                    value(u, r, y);
#pragma unroll
                    for (int e = 0; e < EPL; ++e) y[e] = clamp_nan(y[e], 448.f * now) * inv;
                    put(r, y, j < n_rows);
                }
            }
            // the rows that stay (those behind the kept length, too, that others may have been read from)
            const int count = grows ? min(ps, old_len - (p << a.page_shift)) : bounded ? valid : 0;
            for (int r0 = 0; r0 < count; r0 += kHeld) {
#pragma unroll
                for (int u = 0; u < 2 * BATCH; ++u) w[u] = *reinterpret_cast<const uint2*>(page + (size_t)min(r0 + u * RPL + rg, count - 1) * ROWB);
#pragma unroll
                for (int u = 0; u < 2 * BATCH; ++u) {
                    const int r = r0 + u * RPL + rg;
                    if (r >= count || from[r] >= 0) continue;
                    float y[EPL];
                    unpack_e4m3(w[u].x, y);
                    unpack_e4m3(w[u].y, y + 4);
                    if (grows) {
#pragma unroll
                        for (int e = 0; e < EPL; ++e) y[e] *= f;
                    }
                    put(r, y, grows);
                }
            }
        }
        if (bounded) {
#pragma unroll
            for (int e = 0; e < EPL; ++e)
#pragma unroll
                for (int msk = LPR; msk < LEOAM_WAVE; msk <<= 1) {
                    mx[e] = fmaxf(mx[e], shfl_xor_f(mx[e], msk));
                    mn[e] = fminf(mn[e], shfl_xor_f(mn[e], msk));
                }
            if (lane < LPR) {
                char* row = a.abstract + ((size_t)bh * a.max_pages + p) * 2 * Row<T>::kRowBytes;
                store16(row, col * T::kBytes, round_pack<T>(mx));
                store16(row, Row<T>::kRowBytes + col * T::kBytes, round_pack<T>(mn));
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // (the lists have been read)
    };

    const int last_page = (new_len - 1) >> a.page_shift;      // -1: nothing is kept
    if (a.cut == 1) {
        if (cut_page < 0) return;
        // the page's pairs are the last ones: the first of them
        int i0 = n;
        for (int i1 = n; i1 > 0 && i0 == i1; i1 -= LEOAM_WAVE) {
            const int i = i1 - LEOAM_WAVE + lane;
            const uint64_t hit = __ballot(i >= 0 && moves[max(i, 0)].x >> a.page_shift >= cut_page);
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
        const int p = moves[i].x >> a.page_shift, before = i > 0 ? moves[i - 1].x >> a.page_shift : -1;
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
        (n == 0 || uniform(moves[n - 1].x) >> a.page_shift != last_page))
        take(last_page, n);
    if (h == 0 && lane == 0) {
        if (a.chunk_off) a.chunk_off[(size_t)b * (a.max_pages + 1) + last_page + 1] = new_len;
        if (a.n_chunks) a.n_chunks[b] = last_page + 1;
    }
}

constexpr int kMoveTasks = 16384;      // waves of a tensor

template <typename T, typename S> static hipError_t launch_move(MoveArgs a, hipStream_t stream) {
    a.per_row = (kMoveTasks + a.n_rows - 1) / a.n_rows;
    if (a.per_row > a.m_max) a.per_row = a.m_max;
    a.cut = std::is_same<S, E4M3>::value ? 0 : -1;
    auto grid = [&] { return dim3(2 * (unsigned)(((long long)a.n_rows * a.per_row + kMoveWaves - 1) / kMoveWaves)); };
    hipLaunchKernelGGL((page_move_kernel<T, S>), grid(), dim3(kMoveThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.cut < 0) return e;
    a.cut = a.per_row = 1;
    hipLaunchKernelGGL((page_move_kernel<T, S>), grid(), dim3(kMoveThreads), 0, stream, a);
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
    a.n_rows = s->batch * s->n_kv_heads; a.per_row = 1; a.cut = -1;
    const bool k8 = s->kv_dtype == LEOAM_E4M3;
    switch (s->q_dtype) {
    case LEOAM_F32: return launch_move<F32, F32>(a, stream);
    case LEOAM_F16: return k8 ? launch_move<F16, E4M3>(a, stream) : launch_move<F16, F16>(a, stream);
    default: return k8 ? launch_move<BF16, E4M3>(a, stream) : launch_move<BF16, BF16>(a, stream);
    }
}

}  // namespace leoam
