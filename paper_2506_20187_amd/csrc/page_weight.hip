// page_weight_add: what every cached token got of the attention of the call's rows, added to what it got before:
// weight[t] = decay weight[t] + sum over the rows that see t and the group's heads of exp(scale q.k_t - lse).
//
// S = K Q^T on the matrix cores, keys as the first operand: a wave holds its keys in registers (64; fp32: 32) and goes through the
// rows sixteen (row, head) columns at a time, so the sums of a token stay in registers too and nothing is added by atomics.  One row
// for each sequence: every key is read once, bound by that; the four waves of a workgroup take four stretches of keys.
// Many rows: bound by the exponentials; the four waves share the keys and take every fourth block of columns each, their sums are
// added in order at the end.
#include "page_common.h"

namespace leoam {

struct PageWeightArgs {
    const char *q, *k_pages;
    const float* k_scale;
    const int32_t *page_table, *seq_len, *new_off;
    int n_new;
    float scale_log2;
    const float *lse, *before;
    float decay;
    float* weight;
    const int32_t* n_seen;
    int32_t* token_id;
    int batch, n_kv_heads, n_pages, page_shift, max_pages;
    int total;      // (block of keys, sequence, kv head) triples of a full table
};

template <typename T> constexpr int kWeightTiles = T::kTag == LEOAM_F32 ? 2 : 4;      // 16-key tiles of a wave

template <typename T, typename S, int G, bool kSplitRows> __global__ __launch_bounds__(kAttThreads) void page_weight_kernel(PageWeightArgs a) {
    constexpr bool k8 = std::is_same<S, E4M3>::value, k32 = T::kTag == LEOAM_F32;
    constexpr int ROWB = LEOAM_D * S::kBytes, QROWB = Row<T>::kRowBytes, NT = kWeightTiles<T>, KEYS = 16 * NT, NQ = k32 ? 8 : 4;
    constexpr int BLOCK = kSplitRows ? KEYS : kAttWaves * KEYS;
    __shared__ float sh[kAttWaves][KEYS];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / LEOAM_WAVE), grp = lane >> 4, l16 = lane & 15;
    const int hkv = a.n_kv_heads, rows_bh = a.batch * hkv;

    // A grid that goes round several times stops behind the longest sequence.
    int longest = 0x7fffffff;
    if ((int)gridDim.x < a.total) {
        longest = 0;
        for (int i = lane; i < a.batch; i += LEOAM_WAVE) longest = max(longest, a.seq_len[i]);
        longest = (int)wave_max_u32((uint32_t)longest);
    }
    for (int unit = blockIdx.x; unit < a.total; unit += gridDim.x) {
        const int bh = unit % rows_bh, b = bh / hkv, h = bh - b * hkv;
        const long long block0 = (long long)(unit / rows_bh) * BLOCK;
        if (block0 >= longest) return;
        const int len = uniform(min(max(a.seq_len[b], 0), a.max_pages << a.page_shift));
        const int t0 = (int)block0 + (kSplitRows ? 0 : wave * KEYS);
        if (t0 >= len) continue;      // (kSplitRows: all waves)
        int row0 = b, m = 1;
        if (a.new_off) {
            row0 = uniform(a.new_off[b]);
            m = uniform(a.new_off[b + 1]) - row0;
            if (row0 < 0 || m < 0 || m > a.n_new - row0) m = 0;
        }
        const int first = len - m;      // place of the first row's token

        // ---- keys: tile j, token l16; a token that does not count re-reads the last one that does --------------
        uint4 kb[NT * NQ];
        uint32_t have = 0;      // bit j: the tile has a page
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int t = min(t0 + 16 * j, len - 1), valid = min(len - (t0 + 16 * j), 16);
            const int id = uniform(a.page_table[(size_t)b * a.max_pages + (t >> a.page_shift)]);
            const bool ok = (uint32_t)id < (uint32_t)a.n_pages && valid > 0;
            have |= (ok ? 1u : 0u) << j;
            const size_t row = (size_t)(ok ? id : 0) * hkv + h;
            const char* kp = a.k_pages + (row << a.page_shift) * ROWB;
            const uint32_t at = (uint32_t)((t & ((1 << a.page_shift) - 1) & ~15) + min(l16, max(valid - 1, 0))) * ROWB;
            if constexpr (k8) {
                const float ks = a.k_scale[row];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint4 w = load16(kp, at + 64 * c + 16 * grp);
                    kb[NQ * j + 2 * c] = widen8<T>(w.x, w.y, ks);
                    kb[NQ * j + 2 * c + 1] = widen8<T>(w.z, w.w, ks);
                }
            } else {
#pragma unroll
                for (int s = 0; s < NQ; ++s) kb[NQ * j + s] = load16(kp, at + 64 * s + 16 * grp);
            }
        }

        float w[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) w[j][r] = 0.f;

        // ---- columns: (row, head) pairs from the first row that sees a key of this wave on ---------------------
        const int i0 = max(0, t0 - first), n_cols = (m - i0) * G, n_blocks = (n_cols + 15) / 16;
        const int last_key = min(t0 + KEYS, len) - 1;
        struct Columns {
            uint4 q[NQ];
            float base;      // lse, log2 domain
            int pos;         // the row's place, -1: no column, or a row that attended to nothing
        };
        auto fetch = [&](int cb, Columns& c) {
            const int col = min(16 * cb + l16, n_cols - 1), i = i0 + col / G;
            const size_t at = ((size_t)(row0 + i) * hkv + h) * G + col % G;
#pragma unroll
            for (int s = 0; s < NQ; ++s) {
                // 16-byte pieces in the order in which a key row's registers hold the channels
                const int byte = k32 ? 64 * s + 16 * grp : k8 ? 128 * (s >> 1) + 32 * grp + 16 * (s & 1) : 64 * s + 16 * grp;
                c.q[s] = load16(a.q, at * QROWB + byte);
            }
            const float lse = a.lse[at];
            c.base = lse * kLog2e;
            c.pos = 16 * cb + l16 < n_cols && lse != -INFINITY ? first + i : -1;
        };
        auto add = [&](const Columns& c) {
            const bool masked = __ballot(c.pos < last_key) != 0;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                f32x4_t s = {0.f, 0.f, 0.f, 0.f};
                if constexpr (k32) {
                    f32x4_t chain[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) chain[e] = s;
#pragma unroll
                    for (int i = 0; i < NQ; ++i) {
                        float kx[4], qx[4];
                        unpack<F32>(kb[NQ * j + i], kx);
                        unpack<F32>(c.q[i], qx);
#pragma unroll
                        for (int e = 0; e < 4; ++e) chain[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[e], qx[e], chain[e], 0, 0, 0);
                    }
                    s = (chain[0] + chain[1]) + (chain[2] + chain[3]);
                } else {
#pragma unroll
                    for (int i = 0; i < NQ; ++i) s = mfma_16x16x32<T>(kb[NQ * j + i], c.q[i], s);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float p = exp2_raw(fmaf(s[r], a.scale_log2, -c.base));
                    if (masked && t0 + 16 * j + 4 * grp + r > c.pos) p = 0.f;
                    w[j][r] += p;
                }
            }
        };
        constexpr int kStep = kSplitRows ? kAttWaves : 1;
        const int begin = kSplitRows ? wave : 0;
        if (begin < n_blocks) {
            Columns c[2];
            fetch(begin, c[0]);
            for (int cb = begin; cb < n_blocks; cb += 2 * kStep) {
                fetch(min(cb + kStep, n_blocks - 1), c[1]);
                add(c[0]);
                if (cb + kStep >= n_blocks) break;
                fetch(min(cb + 2 * kStep, n_blocks - 1), c[0]);
                add(c[1]);
            }
        }

        // ---- the columns' sums; lane l16 keeps that of register l16 % 4 of tile l16 / 4 ------------------------
        float mine = 0.f;
        bool counts = false;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float sum = row16_sum(w[j][r]);
                if (l16 == 4 * j + r) {
                    mine = have >> j & 1 ? sum : 0.f;      // (no page: nobody attended to it)
                    counts = true;
                }
            }
        const int slot = 16 * (l16 >> 2) + 4 * grp + (l16 & 3), t = t0 + slot;
        if constexpr (kSplitRows) {
            if (counts) sh[wave][slot] = mine;
            __syncthreads();
            if (wave == 0 && counts) {
                mine = sh[0][slot];
#pragma unroll
                for (int v = 1; v < kAttWaves; ++v) mine += sh[v][slot];
            }
        }
        if ((!kSplitRows || wave == 0) && counts && t < len) {
            const size_t at = (size_t)bh * ((size_t)a.max_pages << a.page_shift) + t;
            a.weight[at] = t < first && a.before ? fmaf(a.decay, a.before[at], mine) : mine;
            if (a.token_id && t >= first) a.token_id[at] = a.n_seen[b] - (len - t);
        }
        if constexpr (kSplitRows) __syncthreads();      // (the sums have been read)
    }
}

// Four or more blocks of columns for each sequence on average: the waves share keys.
constexpr int kManyColumns = 64;
constexpr int kMostWeightGroups = 8192;

template <typename T, typename S, int G> static hipError_t launch_weight(PageWeightArgs a, hipStream_t stream) {
    const bool split = (long long)a.n_new * G >= (long long)kManyColumns * a.batch;
    const long long block = 16 * kWeightTiles<T> * (split ? 1 : kAttWaves), capacity = (long long)a.max_pages << a.page_shift;
    const long long total = (capacity + block - 1) / block * a.batch * a.n_kv_heads;
    if (total > 0x7fffffffll - kMostWeightGroups) return hipErrorInvalidValue;
    a.total = (int)total;
    const dim3 grid((unsigned)(total < kMostWeightGroups ? total : kMostWeightGroups)), threads(kAttThreads);
    if (split) hipLaunchKernelGGL((page_weight_kernel<T, S, G, true>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((page_weight_kernel<T, S, G, false>), grid, threads, 0, stream, a);
    return hipGetLastError();
}
template <typename T, typename S> static hipError_t weight_of(const PageWeightArgs& a, int group, hipStream_t stream) {
    switch (group) {
    case 1: return launch_weight<T, S, 1>(a, stream);
    case 2: return launch_weight<T, S, 2>(a, stream);
    case 4: return launch_weight<T, S, 4>(a, stream);
    default: return launch_weight<T, S, 8>(a, stream);
    }
}

hipError_t page_weight_dispatch(const leoam_pages* s, const void* q, int n_new, const int32_t* new_off, const void* k_pages,
                                const float* k_scale, const int32_t* page_table, const int32_t* seq_len, float softmax_scale,
                                const float* lse, float decay, const float* before, float* weight, const int32_t* n_seen,
                                int32_t* token_id, hipStream_t stream) {
    PageWeightArgs a;
    a.q = (const char*)q; a.k_pages = (const char*)k_pages; a.k_scale = k_scale;
    a.page_table = page_table; a.seq_len = seq_len; a.new_off = new_off; a.n_new = n_new;
    a.scale_log2 = softmax_scale * kLog2e;
    a.lse = lse; a.before = before; a.decay = decay; a.weight = weight; a.n_seen = n_seen; a.token_id = token_id;
    a.batch = s->batch; a.n_kv_heads = s->n_kv_heads; a.n_pages = s->n_pages;
    a.page_shift = __builtin_ctz((unsigned)s->page_size); a.max_pages = s->max_pages;
    a.total = 0;
    const int group = s->n_q_heads / s->n_kv_heads;
    const bool k8 = s->kv_dtype == LEOAM_E4M3;
    switch (s->q_dtype) {
    case LEOAM_F32: return weight_of<F32, F32>(a, group, stream);
    case LEOAM_F16: return k8 ? weight_of<F16, E4M3>(a, group, stream) : weight_of<F16, F16>(a, group, stream);
    default: return k8 ? weight_of<BF16, E4M3>(a, group, stream) : weight_of<BF16, BF16>(a, group, stream);
    }
}

}  // namespace leoam
