// kv_page_move: rows of the cache to other places of the same sequence and kv head, as page_evict_select lists them: keys, values,
// weights and the tokens' numbers; scales of 8-bit pages, abstracts and boundaries are kept up.
//
// Bytes-bound: a row is read once and written once.  With abstracts the pages that rows move to are read whole, since the key
// that was replaced may have been the page's largest or smallest.  A wave owns a (page that rows move to, kv head): an
// 8-bit page's scale may have to grow, and its codes with it.  The pairs are listed by their new place, so a page's pairs
// are neighbours; the waves of a (sequence, kv head) share its pairs equally and take the pages that begin in their share.  A wave
// first looks up all rows that come (a lane each), then has as many of them on their way as its registers hold, keys and values.
// Sources lie behind the kept length and are not written, but in the page that the kept length cuts: 8 bits leave that page to
// a second launch, when nobody reads it any more.
// 40 sequences of 4.2K in bf16 (265 MB) 64 us, 4.1 TB/s; six of 60K in 8 bits (295 MB) 103 us: round trips, list -> page ->
// rows -> scales -> codes for a wave at a time, and the largest magnitudes, codes to numbers for the abstracts and, where scales
// differ, new codes (vector ALU 41 %).
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

// (Waves for each SIMD, and loads of a wave's that are on their way together in 8 bits: 12000 pairs of six sequences behind 48000, 8
// heads: 3 and 16 182 us, 3 and 8 164, 4 and 8 161, 4 and 4 154, 6 and 4 153 but in 16 bits 40 x 4.2K 73 instead of 64.)
template <typename T, typename S> __global__ __launch_bounds__(kMoveThreads, 4) void page_move_kernel(MoveArgs a) {
    constexpr bool k8 = std::is_same<S, E4M3>::value;
    constexpr int EPL = T::kEpl, LPR = LEOAM_D / EPL, RPL = LEOAM_WAVE / LPR;      // lanes to a row, rows to a load
    constexpr int ROWB = LEOAM_D * S::kBytes, BATCH = 8;                             // loads that are on their way together
    // a wave's page: where each row comes from (bytes into a pool, -1: it stays), by which scales, and the rows that come
    __shared__ long long sh_from[kMoveWaves][kMostRows];
    __shared__ float sh_scale[k8 ? 2 : 1][k8 ? kMoveWaves : 1][kMostRows];
    __shared__ int16_t sh_rows[kMoveWaves][kMostRows];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / LEOAM_WAVE);
    const int col = (lane % LPR) * EPL, rg = lane / LPR, ps = 1 << a.page_shift, hkv = a.n_kv_heads;
    const int task = (int)blockIdx.x * kMoveWaves + wave, bh = task / a.per_row, sharer = task - bh * a.per_row;
    if (bh >= a.n_rows) return;
    const int b = bh / hkv, h = bh - b * hkv;
    const int cap = a.max_pages << a.page_shift;
    const int old_len = min(max(scalar_at(a.old_len, b), 0), cap), new_len = min(max(scalar_at(a.new_len, b), 0), old_len);
    const int n = min(max(scalar_at(a.move_count, bh), 0), min(a.m_max, new_len));
    if (new_len >= old_len) return;
    const int2* moves = reinterpret_cast<const int2*>(a.moves) + (size_t)bh * a.m_max;
    const int32_t* table = a.page_table + (size_t)b * a.max_pages;
    const int cut_page = new_len & (ps - 1) ? new_len >> a.page_shift : -1;
    const bool bounded = a.abstract != nullptr;
    char* const pools[2] = {a.k_pages + col * S::kBytes, a.v_pages + col * S::kBytes};
    float* const scales[2] = {a.k_scale, a.v_scale};
    long long* from = sh_from[wave];
    float* const from_scale[2] = {sh_scale[0][k8 ? wave : 0], sh_scale[k8 ? 1 : 0][k8 ? wave : 0]};
    int16_t* rows = sh_rows[wave];

    // page p, whose pairs begin at i0 (i0 == n: none)
    auto take = [&](int p, int i0) {
        const int id = scalar_at(table, p);
        int2 pair = moves[min(i0 + lane, max(n - 1, 0))];      // (m_max >= 1: there is an entry)
        if ((uint32_t)id >= (uint32_t)a.n_pages) return;
        const size_t row_of_page = (size_t)id * hkv + h;
        float old[2] = {1.f, 1.f};
        if constexpr (k8) {
            old[0] = a.k_scale[row_of_page];
            old[1] = a.v_scale[row_of_page];
        }
        for (int r = lane; r < ps; r += LEOAM_WAVE) from[r] = -1;
        int n_rows = 0;
        for (int j0 = 0; j0 < ps; j0 += LEOAM_WAVE) {
            const int i = i0 + j0 + lane;
            if (j0 > 0) pair = moves[min(i, n - 1)];
            const bool mine = i < n && j0 + lane < ps && pair.x >> a.page_shift == p;
            const bool inside = mine && pair.x < new_len && pair.y >= new_len && pair.y < old_len;
            const int src_id = table[inside ? pair.y >> a.page_shift : p];
            const bool fits = inside && (uint32_t)src_id < (uint32_t)a.n_pages;
            const uint64_t hit = __ballot(fits);
            if (fits) {
                const size_t row = (size_t)src_id * hkv + h, at = (size_t)bh * cap;
                const int to = pair.x & (ps - 1);
                from[to] = (long long)(((row << a.page_shift) + (pair.y & (ps - 1))) * ROWB);
                rows[n_rows + __popcll(hit & ((1ull << lane) - 1))] = (int16_t)to;
                const float moved_weight = a.weight ? a.weight[at + pair.y] : 0.f;
                const int moved_id = a.token_id ? a.token_id[at + pair.y] : 0;
                if constexpr (k8) {
                    from_scale[0][to] = a.k_scale[row];
                    from_scale[1][to] = a.v_scale[row];
                }
                if (a.weight) a.weight[at + pair.x] = moved_weight;
                if (a.token_id) a.token_id[at + pair.x] = moved_id;
            }
            n_rows += __popcll(hit);
            if (__ballot(mine) != ~0ull) break;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // (the lists are the wave's own)
        char* const page[2] = {pools[0] + (row_of_page << a.page_shift) * ROWB, pools[1] + (row_of_page << a.page_shift) * ROWB};
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
            // the rows that come; with abstracts every key of the page, from where it is or from where it comes
            auto move_rows = [&](auto tensor) __attribute__((always_inline)) {
                constexpr int W = decltype(tensor)::value;
                const bool all = W == 0 && bounded;
                const int count = all ? valid : n_rows;
                for (int j0 = 0; j0 < count; j0 += RPL * BATCH) {
                    uint4 w[BATCH];
                    int to[BATCH];
#pragma unroll
                    for (int u = 0; u < BATCH; ++u) {      // (rows past the last repeat it)
                        const int j = min(j0 + u * RPL + rg, count - 1), r = all ? j : rows[j];
                        const long long src = from[r];
                        to[u] = src < 0 ? -1 : r;
                        w[u] = load16(src < 0 ? page[W] + (size_t)r * ROWB : pools[W] + src, 0);
                    }
#pragma unroll
                    for (int u = 0; u < BATCH; ++u) {
                        if (all) {
                            float y[EPL];
                            unpack<T>(w[u], y);
                            extremes(y);
                        }
                        if (to[u] >= 0) store16(page[W], (size_t)to[u] * ROWB, w[u]);
                    }
                }
            };
            move_rows(std::integral_constant<int, 1>{});
            move_rows(std::integral_constant<int, 0>{});
        } else {
            // The scale comes before the codes: rows that come are read for their largest magnitude, and again if they are more than
            // the registers hold (from the cache).
            constexpr int HELD = 4, kHeld = RPL * HELD;
            uint2 held[2][HELD];
            auto row_of = [&](int j) { return (int)rows[min(j, n_rows - 1)]; };
            auto fetch = [&](auto tensor, int j0) __attribute__((always_inline)) {
                constexpr int W = decltype(tensor)::value;
#pragma unroll
                for (int u = 0; u < HELD; ++u) {
                    if (j0 + u * RPL >= n_rows) break;
                    held[W][u] = *reinterpret_cast<const uint2*>(pools[W] + from[row_of(j0 + u * RPL + rg)]);
                }
            };
            auto encode_rows = [&](auto tensor) __attribute__((always_inline)) {
                constexpr int W = decltype(tensor)::value;
                const bool keys = W == 0 && bounded;
                float top = 0.f;
                for (int j0 = 0; j0 < n_rows; j0 += kHeld) {
                    if (j0 > 0) fetch(tensor, j0);
#pragma unroll
                    for (int u = 0; u < HELD; ++u) {      // (a code's magnitude, NaN left out by the maximum, and 8 bits have no infinity)
                        if (j0 + u * RPL >= n_rows) break;
                        float y[8];
                        unpack_e4m3(held[W][u].x, y);
                        unpack_e4m3(held[W][u].y, y + 4);
                        float m = fmaxf(fabsf(y[0]), fabsf(y[1]));
#pragma unroll
                        for (int e = 2; e < 8; ++e) m = fmaxf(m, fabsf(y[e]));
                        top = fmaxf(top, m * from_scale[W][row_of(j0 + u * RPL + rg)]);
                    }
                }
                const float now = fmaxf(old[W], scale_of<T>(wave_extreme_f<true>(top))), inv = now > 0.f ? 1.f / now : 0.f;
                const bool grows = now > old[W];
                if (lane == 0 && grows) scales[W][row_of_page] = now;
                // (what is stored is at most 448 of the new scale, and the quotient of two scales a power of two: mostly 1, and codes
                // stay what they are)
                auto put = [&](int r, uint2 c, float f, bool store) __attribute__((always_inline)) {
                    float y[8];
                    if (__ballot(f != 1.f)) {
                        unpack_e4m3(c.x, y);
                        unpack_e4m3(c.y, y + 4);
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] *= f;
                        c = make_uint2(pack_e4m3(y), pack_e4m3(y + 4));
                    }
                    if (store) *reinterpret_cast<uint2*>(page[W] + (size_t)r * ROWB) = c;
                    if (keys && r < valid) {      // (of codes: the scale comes at the end)
                        unpack_e4m3(c.x, y);
                        unpack_e4m3(c.y, y + 4);
                        extremes(y);
                    }
                };
                for (int j0 = 0; j0 < n_rows; j0 += kHeld) {
                    if (n_rows > kHeld) fetch(tensor, j0);
#pragma unroll
                    for (int u = 0; u < HELD; ++u) {
                        const int j = j0 + u * RPL + rg, r = row_of(j);
                        if (j0 + u * RPL >= n_rows) break;
                        put(r, held[W][u], fminf(from_scale[W][r] * inv, 0x1p30f), j < n_rows);      // (more: a row of zeros)
                    }
                }
                // the rows that stay (those behind the kept length, too, that others may have been read from)
                const int count = grows ? min(ps, old_len - (p << a.page_shift)) : keys ? valid : 0;
                const float f = grows ? old[W] * inv : 1.f;
                for (int r0 = 0; r0 < count; r0 += kHeld) {
#pragma unroll
                    for (int u = 0; u < HELD; ++u)
                        held[W][u] = *reinterpret_cast<const uint2*>(page[W] + (size_t)min(r0 + u * RPL + rg, count - 1) * ROWB);
#pragma unroll
                    for (int u = 0; u < HELD; ++u) {
                        const int r = r0 + u * RPL + rg;
                        if (r0 + u * RPL >= count) break;
                        if (r < count && from[r] < 0) put(r, held[W][u], f, grows);
                    }
                }
                if (keys) {
#pragma unroll
                    for (int e = 0; e < EPL; ++e) {      // (infinite: the lane saw no number)
                        mx[e] = mx[e] == -INFINITY ? mx[e] : mx[e] * now;
                        mn[e] = mn[e] == INFINITY ? mn[e] : mn[e] * now;
                    }
                }
            };
            if (n_rows > 0) {
                fetch(std::integral_constant<int, 0>{}, 0);
                fetch(std::integral_constant<int, 1>{}, 0);
            }
            encode_rows(std::integral_constant<int, 0>{});
            encode_rows(std::integral_constant<int, 1>{});
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
    if (sharer + 1 < a.per_row) return;
    // what the sequence loses beside the rows that moved: the last page holds fewer tokens
    if (bounded && last_page >= 0 && (a.cut < 0 || last_page != cut_page) &&
        (n == 0 || uniform(moves[n - 1].x) >> a.page_shift != last_page))
        take(last_page, n);
    if (h == 0 && lane == 0) {
        if (a.chunk_off) a.chunk_off[(size_t)b * (a.max_pages + 1) + last_page + 1] = new_len;
        if (a.n_chunks) a.n_chunks[b] = last_page + 1;
    }
}

constexpr int kMoveTasks = 16384;      // waves

template <typename T, typename S> static hipError_t launch_move(MoveArgs a, hipStream_t stream) {
    a.per_row = (kMoveTasks + a.n_rows - 1) / a.n_rows;
    if (a.per_row > a.m_max) a.per_row = a.m_max;
    a.cut = std::is_same<S, E4M3>::value ? 0 : -1;
    auto grid = [&] { return dim3((unsigned)(((long long)a.n_rows * a.per_row + kMoveWaves - 1) / kMoveWaves)); };
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
