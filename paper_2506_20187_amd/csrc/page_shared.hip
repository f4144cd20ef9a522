// page_attention_decode_shared: softmax(scale q K^T) V of one token per sequence where groups of sequences list the same leading
// pages: a group's prefix is read once for all of its members, each sequence's further pages by itself.
//
// HBM-bound up to some hundred (member, head) columns per kv head, by the matrix cores and the exponentials beyond.  A unit of work
// is (up to 128 columns of a group, kv head) over the group's prefix, or (sequence, kv head) over its own tokens.  The tiles of all
// units are laid end to end, each unit's beginning counted as some more, and shared out equally: the host does not know the
// lengths.  A unit cut by the ends of shares leaves its pieces, (acc[128], m, l) per column, in the workspace; a second
// kernel folds a head's pieces of its group's unit and of its own, in order, so results do not depend on scheduling.
//
// As in page_attention_decode everything runs on the matrix cores without passing through LDS: S^T = K Q^T, lane = column, registers =
// tokens, then O^T = V^T P^T with the weights in two fp16 or three bf16 parts.  Here a wave has two blocks of 16 columns, so what it
// fetches is used twice; up to 32 columns the four waves take a quarter of the tokens each, up to 64 two waves
// share tokens, up to 128 all four do, with a quarter of the columns each, and the first-level cache serves them.
#include <cfloat>

#include "page_common.h"

namespace leoam {

// Where the state of a (sequence, kv head) is: pieces in slots (count > 0), one whole state (kWhole), the result is final (kFinal),
// nothing (0).
constexpr int kWhole = -1, kFinal = -2;
struct SharedRow { int32_t own_count, own_slot, pre_count, pre_slot, pre_col; };

constexpr int kSharedTile = 128;          // unit of the partition, tokens
constexpr int kSharedColumns = 128;       // most columns of a unit
constexpr int kWaveColumns = 32;
constexpr int kGroupsInLds = 512;

struct PageSharedArgs {
    const char *q, *k_pages, *v_pages;
    const float *k_scale, *v_scale;
    const int32_t *page_table, *seq_len, *group_off, *group_pages;
    int n_groups;
    float scale_log2;      // of |softmax_scale|
    uint32_t flip;         // sign bits of the queries, turned if softmax_scale is negative
    float *out, *lse;
    SharedRow* rows;
    // States: 128 accumulators, and apart from them the maximum and the sum.  First the whole ones of each head over its own tokens, then
    // those over its group's prefix, then the slots of pieces, of kSharedColumns columns each.
    float *acc, *ml;
    int n_heads;
    int sharers;
    int batch, n_kv_heads, group_shift, n_pages, page_shift, max_pages;
};

// The reference of a column's weights may lag its maximum by 2^kSharedLag, so that the accumulators are rarely scaled; fp16 weights take
// it 2^7 lower, so that small ones stay clear of fp16's subnormals and the largest below its maximum.
constexpr float kSharedLag = 8.f;
template <typename T> constexpr int shared_bias() { return T::kTag == LEOAM_F16 ? 7 : 0; }

// a 16-token tile of the walk (wave-uniform)
struct SharedTile {
    uint32_t page;
    int row0, valid;
    float ks, vs;
};

// what a wave fetches at a time: 32 tokens (fp32: 16)
template <typename T, typename S> struct SharedStep {
    static constexpr bool k8 = std::is_same<S, E4M3>::value, k32 = T::kTag == LEOAM_F32;
    static constexpr int NT = k32 ? 1 : 2, NK = k32 ? 8 : k8 ? 2 : 4;      // tiles, loads of a key tile
    uint4 k[NT * NK];
    typename std::conditional<k8, uint2, uint4>::type v[8];
};

// What a tile costs a workgroup whose waves go `ways` over the columns, and what a unit's beginning does: shares are measured in that.
// (Every wave of a workgroup that goes four ways multiplies all of a tile.)
template <bool k8> __device__ __forceinline__ int tile_cost(int ways) { return ways == 1 ? 2 : ways == 2 ? (k8 ? 4 : 3) : (k8 ? 8 : 5); }
constexpr int kSharedStart = 4;
constexpr int kMostTileCost = 8;

__device__ __forceinline__ int shared_tiles(int tokens) { return max(1, (tokens + kSharedTile - 1) / kSharedTile); }
// of the waves, over a unit's columns
__device__ __forceinline__ int ways_of(int n_cols) { return n_cols <= kWaveColumns ? 1 : n_cols <= 2 * kWaveColumns ? 2 : 4; }

// Units of an entry (a group's prefix, or a sequence's own tokens): `full` ones of most columns, then `rest` of the others.
struct SharedEntry {
    int full, rest, tiles, cost_full, cost_rest;
    __device__ __forceinline__ long long length(int unit) const { return kSharedStart + (long long)tiles * cost(unit); }
    __device__ __forceinline__ int cost(int unit) const { return unit < full ? cost_full : cost_rest; }
    __device__ __forceinline__ long long total() const { return full * length(0) + rest * (kSharedStart + (long long)tiles * cost_rest); }
};

template <typename T, typename S>
__global__ __launch_bounds__(kAttThreads) __attribute__((amdgpu_waves_per_eu(2))) void page_shared_kernel(PageSharedArgs a) {
    using Step = SharedStep<T, S>;
    constexpr bool k8 = Step::k8, k32 = Step::k32;
    constexpr int ROWB = LEOAM_D * S::kBytes, QROWB = Row<T>::kRowBytes, NT = Step::NT, NK = Step::NK, STEP = 16 * NT, NQ = k32 ? 8 : 4;
    constexpr float kBias = shared_bias<T>();
    constexpr int kParts = T::kTag == LEOAM_F16 ? 2 : 3;
    constexpr int kStride = LEOAM_D + 4;      // of a column in LDS: its accumulators, maximum and sum
    __shared__ __align__(16) float xw[kAttWaves][kWaveColumns][kStride];
    __shared__ int sh_off[kGroupsInLds + 1], sh_pages[kGroupsInLds];
    __shared__ long long sh_sum[kAttWaves], sh_at;
    __shared__ int sh_entry;

    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE), grp = lane >> 4, l16 = lane & 15;
    const int hkv = a.n_kv_heads, group = 1 << a.group_shift, cap = a.max_pages << a.page_shift;
    const int most_members = kSharedColumns >> a.group_shift;

    // ---- groups, and this workgroup's share of the tiles -------------------------------------------------
    const bool in_lds = a.n_groups <= kGroupsInLds;
    if (in_lds) {
        for (int i = tid; i <= a.n_groups; i += kAttThreads) {
            sh_off[i] = a.group_off[i];
            if (i < a.n_groups) sh_pages[i] = a.group_pages[i];
        }
        __syncthreads();
    }
    auto off_of = [&](int g) { return min(max(in_lds ? sh_off[g] : a.group_off[g], 0), a.batch); };
    auto prefix_of = [&](int g) { return min(max(in_lds ? sh_pages[g] : a.group_pages[g], 0), a.max_pages) << a.page_shift; };
    auto length_of = [&](int b) { return min(max(a.seq_len[b], 0), cap); };
    // tokens of sequence b that its group's unit deals with
    auto before_of = [&](int b, int len) {
        int lo = 0, hi = a.n_groups;      // the last group that begins at or before b
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (off_of(mid) <= b) lo = mid + 1;
            else hi = mid;
        }
        if (lo == 0 || off_of(lo) <= b) return 0;
        const int shared = prefix_of(lo - 1);
        return len >= shared ? shared : 0;      // (a sequence that is shorter has all of its tokens to itself)
    };
    // entries: groups, then sequences
    auto entry_of = [&](int e) {
        if (e < a.n_groups) {
            const int members = off_of(e + 1) - off_of(e), tokens = prefix_of(e);
            if (members <= 0 || tokens == 0) return SharedEntry{0, 0, 0, 1, 1};
            const int full = members / most_members, rest = members - full * most_members;
            return SharedEntry{full * hkv, rest ? hkv : 0, shared_tiles(tokens), tile_cost<k8>(4), tile_cost<k8>(ways_of(rest << a.group_shift))};
        }
        const int b = e - a.n_groups, len = length_of(b);
        return SharedEntry{0, hkv, shared_tiles(len - before_of(b, len)), 1, tile_cost<k8>(1)};
    };
    const int n_entries = a.n_groups + a.batch;
    long long pos, end, share, off;      // off: how far into the unit pos is
    int entry, unit;
    {
        const int per = (n_entries + kAttThreads - 1) / kAttThreads, e0 = min(tid * per, n_entries), e1 = min(e0 + per, n_entries);
        long long mine = 0;
        for (int e = e0; e < e1; ++e) mine += entry_of(e).total();
        long long incl = mine;
#pragma unroll
        for (int d = 1; d < LEOAM_WAVE; d <<= 1) {
            const long long o = __shfl_up(incl, d, LEOAM_WAVE);
            if (lane >= d) incl += o;
        }
        if (lane == LEOAM_WAVE - 1) sh_sum[wave] = incl;
        __syncthreads();
        long long total = 0, before = incl - mine;
#pragma unroll
        for (int w = 0; w < kAttWaves; ++w) {
            if (w < wave) before += sh_sum[w];
            total += sh_sum[w];
        }
        share = max((total + a.sharers - 1) / a.sharers, (long long)kMostTileCost);      // (so that a tile begins in each)
        pos = share * blockIdx.x;
        end = min(total, pos + share);
        if (pos >= end) return;
        if (pos >= before && pos < before + mine) {
            int e = e0;
            for (;;) {
                const long long n = entry_of(e).total();
                if (pos < before + n) break;
                before += n;
                ++e;
            }
            sh_entry = e;
            sh_at = pos - before;
        }
        __syncthreads();
        entry = uniform(sh_entry);
        const SharedEntry x = entry_of(entry);
        const long long at = sh_at, full = x.full * x.length(0), in = at < full ? at : at - full, length = at < full ? x.length(0) : x.length(x.full);
        unit = uniform((int)(in / length));
        off = in - unit * length;
        if (at >= full) unit += x.full;
    }

    // One stretch of a unit: tokens [t_begin, t_end) of row b_table, for this wave's columns, NB blocks of 16; `col_row`: the lane's
    // row of q in each block, < 0: none.
    auto walk = [&](auto blocks, int b_table, int h, int t_begin, int t_end, int way, int ways, int n_cols, const long long* col_row, auto&& leave) {
        constexpr int NB = decltype(blocks)::value;
        uint4 qb[NB][NQ];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int s = 0; s < NQ; ++s) {
                // 16-byte pieces in the order in which a key row's loads hold the channels
                const int byte = k32 ? 64 * s + 16 * grp : k8 ? 128 * (s >> 1) + 32 * grp + 16 * (s & 1) : 64 * s + 16 * grp;
                qb[n][s] = make_uint4(0, 0, 0, 0);
                if (col_row[n] >= 0) qb[n][s] = load16(a.q, (size_t)col_row[n] * QROWB + byte);
                qb[n][s].x ^= a.flip; qb[n][s].y ^= a.flip; qb[n][s].z ^= a.flip; qb[n][s].w ^= a.flip;
            }
        const int n_streams = kAttWaves / ways, stream = wave / ways;
        const int n_steps = (t_end - t_begin + STEP - 1) / STEP, per = (n_steps + n_streams - 1) / n_streams;
        const int s0 = min(n_steps, stream * per), s1 = min(n_steps, s0 + per);

        // lane i holds entry held0 + i of the row's pages (-1: none)
        int held0 = -(1 << 30), held_page = -1;
        const int n_listed = (t_end + (1 << a.page_shift) - 1) >> a.page_shift;
        auto where = [&](int step, SharedTile* at) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int t = t_begin + step * STEP + 16 * j, e = t >> a.page_shift;
                if (e - held0 >= LEOAM_WAVE || e < held0) {
                    held0 = e;
                    const int id = e + lane < n_listed ? a.page_table[(size_t)b_table * a.max_pages + e + lane] : -1;
                    held_page = (uint32_t)id < (uint32_t)a.n_pages ? id : -1;
                }
                const int id = __builtin_amdgcn_readlane(held_page, e - held0);
                at[j].page = id < 0 ? 0u : (uint32_t)id;
                at[j].row0 = t & ((1 << a.page_shift) - 1);
                at[j].valid = id < 0 ? 0 : min(max(t_end - t, 0), 16);
                at[j].ks = at[j].vs = 1.f;
                if (k8) {
                    const size_t row = (size_t)at[j].page * hkv + h;
                    at[j].ks = a.k_scale[row];
                    at[j].vs = a.v_scale[row];
                }
            }
        };
        // Loads are unconditional; a token that does not count re-reads the tile's last one that does (what stands behind the last
        // token may be NaN, which a weight of zero would not silence).
        auto fetch_keys = [&](const SharedTile* at, Step& st) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const char* kp = a.k_pages + (((size_t)at[j].page * hkv + h) << a.page_shift) * ROWB;
                const uint32_t krow = (uint32_t)(at[j].row0 + min(l16, max(at[j].valid - 1, 0))) * ROWB;
#pragma unroll
                for (int s = 0; s < NK; ++s) st.k[NK * j + s] = load16(kp, krow + 64 * s + 16 * grp);
            }
        };
        auto fetch_values = [&](const SharedTile* at, Step& st) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const char* vp = a.v_pages + (((size_t)at[j].page * hkv + h) << a.page_shift) * ROWB;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t vrow = (uint32_t)(at[j].row0 + min(4 * grp + r, max(at[j].valid - 1, 0))) * ROWB;
                    if constexpr (k32) {
                        st.v[2 * r] = load16(vp, vrow + 16 * l16);
                        st.v[2 * r + 1] = load16(vp, vrow + 256 + 16 * l16);
                    } else if constexpr (k8) {
                        st.v[4 * j + r] = *reinterpret_cast<const uint2*>(vp + vrow + 8 * l16);
                    } else {
                        st.v[4 * j + r] = load16(vp, vrow + 16 * l16);
                    }
                }
            }
        };

        // lane (grp, column): running maximum (log2 domain) and this lane's part of the sum, accumulators of 32 channels
        float m_run[NB], l_run[NB];
        f32x4_t acc[NB][8];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            m_run[n] = -INFINITY;
            l_run[n] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[n][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }

        auto products = [&](const Step& st, const SharedTile* at, float (*x)[4 * NT]) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                uint4 ka[NQ];
#pragma unroll
                for (int i = 0; i < NQ; ++i) {
                    if constexpr (k8) {
                        const uint4 w = st.k[NK * j + i / 2];
                        ka[i] = i & 1 ? widen8<T>(w.z, w.w, at[j].ks) : widen8<T>(w.x, w.y, at[j].ks);
                    } else {
                        ka[i] = st.k[NK * j + i];
                    }
                }
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
                    if constexpr (k32) {
                        f32x4_t chain[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) chain[e] = s;
#pragma unroll
                        for (int i = 0; i < NQ; ++i) {
                            float kx[4], qx[4];
                            unpack<F32>(ka[i], kx);
                            unpack<F32>(qb[n][i], qx);
#pragma unroll
                            for (int e = 0; e < 4; ++e) chain[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[e], qx[e], chain[e], 0, 0, 0);
                        }
                        s = (chain[0] + chain[1]) + (chain[2] + chain[3]);
                    } else {
#pragma unroll
                        for (int i = 0; i < NQ; ++i) s = mfma_16x16x32<T>(ka[i], qb[n][i], s);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[n][4 * j + r] = s[r];
                }
            }
        };
        auto weigh = [&](float (*x)[4 * NT], const SharedTile* at) {      // products become weights
            bool partial = false;      // some tile has tokens that do not count
#pragma unroll
            for (int j = 0; j < NT; ++j) partial |= at[j].valid < 16;
            if (partial) {
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int i = 0; i < 4 * NT; ++i)
                        if (4 * grp + i % 4 >= at[i / 4].valid) x[n][i] = -INFINITY;
            }
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                float mt = x[n][0];
#pragma unroll
                for (int i = 1; i < 4 * NT; ++i) mt = fmaxf(mt, x[n][i]);
                mt = rows_max4(mt) * a.scale_log2 - kBias;
                if (__ballot(mt > m_run[n] + kSharedLag)) {
                    const float m = fmaxf(m_run[n], mt), c = exp2_or_zero(m_run[n], m);
                    m_run[n] = m;
                    l_run[n] *= c;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[n][i][r] *= c;
                }
                const float ref = m_run[n] == -INFINITY ? 0.f : m_run[n];
#pragma unroll
                for (int i = 0; i < 4 * NT; ++i) {
                    x[n][i] = exp2_raw(fmaf(x[n][i], a.scale_log2, -ref));
                    l_run[n] += x[n][i];
                }
            }
        };
        auto weighted = [&](Step& st, SharedTile* at, float (*p)[4 * NT]) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
                if (at[j].valid == 0) {      // nothing was read that counts: values must not matter either
                    at[j].vs = 1.f;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if constexpr (k32) st.v[2 * r] = st.v[2 * r + 1] = make_uint4(0, 0, 0, 0);
                        else if constexpr (k8) st.v[4 * j + r] = make_uint2(0, 0);
                        else st.v[4 * j + r] = make_uint4(0, 0, 0, 0);
                    }
                }
            if constexpr (k32) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float vx[4];
                        unpack<F32>(st.v[2 * r + c], vx);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
#pragma unroll
                            for (int n = 0; n < NB; ++n)
                                acc[n][4 * c + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vx[e], p[n][r], acc[n][4 * c + e], 0, 0, 0);
                    }
            } else {
                uint4 parts[NB][kParts];
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int k = 0; k < kParts; ++k) {
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float u, v;
                            w[i] = pair_of(T{}, p[n][2 * i], p[n][2 * i + 1]);
                            pair_back(T{}, w[i], u, v);
                            p[n][2 * i] -= u;      // (exact: what is left has fewer bits)
                            p[n][2 * i + 1] -= v;
                        }
                        parts[n][k] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                uint32_t v[8][4];      // [token slot][two channels each]
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    uint4 w;
                    if constexpr (k8) w = widen8<T>(st.v[t].x, st.v[t].y, at[t / 4].vs);
                    else w = st.v[t];
                    v[t][0] = w.x; v[t][1] = w.y; v[t][2] = w.z; v[t][3] = w.w;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t pick = e & 1 ? 0x07060302u : 0x05040100u;
                    uint4 col;      // channel 8 l16 + e of the eight tokens
                    col.x = __builtin_amdgcn_perm(v[1][e / 2], v[0][e / 2], pick);
                    col.y = __builtin_amdgcn_perm(v[3][e / 2], v[2][e / 2], pick);
                    col.z = __builtin_amdgcn_perm(v[5][e / 2], v[4][e / 2], pick);
                    col.w = __builtin_amdgcn_perm(v[7][e / 2], v[6][e / 2], pick);
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int k = 0; k < kParts; ++k) acc[n][e] = mfma_16x16x32<T>(col, parts[n][k], acc[n][e]);
                }
            }
        };

        if (s0 < s1) {
            // the next step's keys are on their way while the weights are computed, its values while the next products are
            Step st;
            SharedTile at[NT], next[NT];
            where(s0, at);
            fetch_keys(at, st);
            fetch_values(at, st);
            for (int s = s0; s < s1; ++s) {
                float x[NB][4 * NT];
                where(min(s + 1, s1 - 1), next);
                products(st, at, x);
                fetch_keys(next, st);
                weigh(x, at);
                weighted(st, at, x);
                fetch_values(next, st);
#pragma unroll
                for (int j = 0; j < NT; ++j) at[j] = next[j];
            }
        }
        // ---- the columns' states: leave(column, first of four channels, accumulators, maximum, sum) ------------
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            l_run[n] += shfl_xor_f(l_run[n], 16);
            l_run[n] += shfl_xor_f(l_run[n], 32);
        }
        // accumulator i, row 4 grp + r: its channel is 8 (4 grp + r) + i (fp32: 64 (i / 4) + 4 (4 grp + r) + i % 4)
        auto four = [&](int n, int r, int half) {
            return make_float4(acc[n][4 * half][r], acc[n][4 * half + 1][r], acc[n][4 * half + 2][r], acc[n][4 * half + 3][r]);
        };
        auto channel = [&](int r, int half) { return k32 ? 64 * half + 4 * (4 * grp + r) : 8 * (4 * grp + r) + 4 * half; };
        if (n_streams == 1) {      // a wave has all of its columns' tokens
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const int c = kWaveColumns * way + 16 * n + l16;
                if (c >= n_cols) continue;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int half = 0; half < 2; ++half) leave(c, channel(r, half), four(n, r, half), m_run[n], l_run[n]);
            }
            return;
        }
        __syncthreads();      // (the previous stretch's states have been read)
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            float* x = xw[wave][16 * n + l16];
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int half = 0; half < 2; ++half) *reinterpret_cast<float4*>(x + channel(r, half)) = four(n, r, half);
            if (grp == 0) {
                x[LEOAM_D] = m_run[n];
                x[LEOAM_D + 1] = l_run[n];
            }
        }
        __syncthreads();
        for (int i = tid; i < n_cols * (LEOAM_D / 4); i += kAttThreads) {
            const int c = i / (LEOAM_D / 4), d = 4 * (i % (LEOAM_D / 4)), w0 = c / kWaveColumns, in = c % kWaveColumns;
            float ms[kAttWaves], m = -INFINITY;
#pragma unroll
            for (int k = 0; k < kAttWaves; ++k) {      // (two ways: waves w0 and w0 + 2)
                ms[k] = k < n_streams ? xw[w0 + k * ways][in][LEOAM_D] : -INFINITY;
                m = fmaxf(m, ms[k]);
            }
            float l = 0.f;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kAttWaves; ++k) {
                if (k >= n_streams) break;
                const float f = exp2_or_zero(ms[k], m);
                const float4 x = *reinterpret_cast<const float4*>(&xw[w0 + k * ways][in][d]);
                l += f * xw[w0 + k * ways][in][LEOAM_D + 1];
                v.x += f * x.x; v.y += f * x.y; v.z += f * x.z; v.w += f * x.w;
            }
            leave(c, d, v, m, l);
        }
    };

    bool first_piece = true;
    while (pos < end) {
        const SharedEntry x = entry_of(entry);
        const int units = uniform(x.full + x.rest);
        if (units == 0) {      // (a group without a prefix)
            ++entry;
            continue;
        }
        const int tiles = uniform(x.tiles), cost = uniform(x.cost(unit));
        const long long length = kSharedStart + (long long)tiles * cost, take = min(length - off, end - pos);
        // tiles that begin in the share
        auto tiles_before = [&](long long at) { return at <= kSharedStart ? 0 : (int)((at - kSharedStart + cost - 1) / cost); };
        const int tile0 = uniform(tiles_before(off)), tile1 = uniform(min(tiles, tiles_before(off + take)));
        if (tile0 < tile1) {
            const int h = unit % hkv;
            const bool prefix = entry < a.n_groups, whole = tile1 - tile0 == tiles;
            const int slot = 2 * (int)blockIdx.x + (first_piece ? 0 : 1);      // opens the share, or closes it
            // pieces of the unit, and where the first lies, if it begins here
            const int count = whole ? kWhole : (int)((pos - off + kSharedStart + (long long)(tiles - 1) * cost) / share - blockIdx.x) + 1;
            int n_cols, b0, tokens, before = 0, b_table;
            bool work = true;
            if (prefix) {
                b0 = off_of(entry) + unit / hkv * most_members;
                const int members = min(off_of(entry + 1) - b0, most_members);
                n_cols = members << a.group_shift;
                tokens = prefix_of(entry);
                b_table = -1;      // the first member that has the whole prefix
                for (int i = 0; i < members && b_table < 0; i += LEOAM_WAVE) {
                    const uint64_t has = __ballot(i + lane < members && length_of(b0 + i + lane) >= tokens);
                    if (has) b_table = b0 + i + __builtin_ctzll(has);
                }
                b0 = uniform(b0);
                n_cols = uniform(n_cols);
                b_table = uniform(b_table);
                work = b_table >= 0;
                if (tile0 == 0 && tid < members && length_of(b0 + tid) >= tokens) {
                    SharedRow* r = a.rows + (size_t)(b0 + tid) * hkv + h;
                    r->pre_count = count;
                    r->pre_slot = slot;
                    r->pre_col = tid << a.group_shift;
                }
            } else {
                b0 = b_table = entry - a.n_groups;
                n_cols = group;
                const int len = uniform(length_of(b0));
                before = uniform(before_of(b0, len));
                tokens = len - before;
            }
            tokens = uniform(tokens);
            const bool final_ = !prefix && before == 0 && whole;
            if (!prefix && tile0 == 0 && tid == 0) {
                SharedRow* r = a.rows + (size_t)b0 * hkv + h;
                r->own_count = final_ ? kFinal : tokens == 0 ? 0 : count;
                r->own_slot = slot;
                if (before == 0) r->pre_count = 0;
            }
            if (work && (tokens > 0 || final_)) {
                const int ways = ways_of(n_cols);
                const int way = wave & (ways - 1);
                long long col_row[2];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const int c = kWaveColumns * way + 16 * n + l16, b = b0 + (c >> a.group_shift);
                    const bool counts = c < n_cols && (!prefix || length_of(b) >= tokens);
                    col_row[n] = counts ? (((long long)b * hkv + h) << a.group_shift) + (c & (group - 1)) : -1;
                }
                const int t_begin = before + tile0 * kSharedTile, t_end = before + min(tokens, tile1 * kSharedTile);
                auto leave = [&](int c, int d, const float4& v, float m, float l) {
                    const size_t j = (((size_t)(b0 + (c >> a.group_shift)) * hkv + h) << a.group_shift) + (c & (group - 1));
                    if (final_) {
                        const float inv = l == 0.f ? 0.f : 1.f / l;      // (NaN stays)
                        *reinterpret_cast<float4*>(a.out + j * LEOAM_D + d) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
                        if (d == 0 && a.lse) a.lse[j] = log_sum_exp(m, l, shared_bias<T>());
                        return;
                    }
                    const size_t at = !whole ? 2 * (size_t)a.n_heads + (size_t)slot * kSharedColumns + c : prefix ? a.n_heads + j : j;
                    *reinterpret_cast<float4*>(a.acc + at * LEOAM_D + d) = v;
                    if (d == 0) *reinterpret_cast<float2*>(a.ml + 2 * at) = make_float2(m, l);
                };
                if (n_cols <= 16) walk(std::integral_constant<int, 1>{}, b_table, h, t_begin, t_end, way, ways, n_cols, col_row, leave);
                else walk(std::integral_constant<int, 2>{}, b_table, h, t_begin, t_end, way, ways, n_cols, col_row, leave);
            }
            first_piece = false;
        }
        pos += take;
        off = 0;
        if (++unit == units) {
            unit = 0;
            ++entry;
        }
    }
}

// A head's pieces: those of its group's unit, then its own.  128 threads take eight at a time, all on their way together.
__global__ __launch_bounds__(2 * LEOAM_D) void page_shared_merge_kernel(const SharedRow* __restrict__ rows, const float* __restrict__ acc,
                                                                       const float* __restrict__ ml, int group_shift, int n_heads, int sharers, int bias,
                                                                       float* __restrict__ out, float* __restrict__ lse) {
    constexpr int kBatch = 8;
    const int d = threadIdx.x % LEOAM_D, j = 2 * blockIdx.x + threadIdx.x / LEOAM_D;
    if (j >= n_heads) return;
    const SharedRow r = rows[j >> group_shift];
    if (r.own_count == kFinal) return;
    // (counts and slots that no kernel wrote - lists of groups that overlap - stay within the workspace)
    const int g = j & ((1 << group_shift) - 1), last = 2 * sharers - 1;
    const int n_pre = r.pre_count == kWhole ? 1 : min(max(r.pre_count, 0), sharers), n_own = r.own_count == kWhole ? 1 : min(max(r.own_count, 0), sharers);
    auto state = [&](int i) {
        const bool mine = i >= n_pre;
        const int k = mine ? i - n_pre : i, count = mine ? r.own_count : r.pre_count;
        if (count == kWhole) return (size_t)(mine ? j : n_heads + j);
        // (each further piece opens the next workgroup's share)
        const int slot0 = mine ? r.own_slot : r.pre_slot, slot = min(max(k == 0 ? slot0 : 2 * (slot0 / 2 + k), 0), last);
        const int col = min(max(mine ? 0 : r.pre_col, 0), kSharedColumns - (1 << group_shift)) + g;
        return 2 * (size_t)n_heads + (size_t)slot * kSharedColumns + col;
    };
    float m = -INFINITY, l = 0.f, o = 0.f;
    for (int i0 = 0; i0 < n_pre + n_own; i0 += kBatch) {
        float ms[kBatch], ls[kBatch], os[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const size_t at = state(min(i0 + u, n_pre + n_own - 1));
            const float2 x = *reinterpret_cast<const float2*>(ml + 2 * at);
            ms[u] = x.x;
            ls[u] = x.y;
            os[u] = acc[at * LEOAM_D + d];
        }
        float mb = m;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i0 + u >= n_pre + n_own) ms[u] = -INFINITY;
            mb = fmaxf(mb, ms[u]);
        }
        const float c = exp2_or_zero(m, mb);
        m = mb;
        l *= c;
        o *= c;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i0 + u >= n_pre + n_own) continue;
            const float w = exp2_or_zero(ms[u], m);
            l += w * ls[u];
            o += w * os[u];
        }
    }
    out[(size_t)j * LEOAM_D + d] = l == 0.f ? 0.f : o / l;      // (NaN stays)
    if (lse && d == 0) lse[j] = log_sum_exp(m, l, bias);
}

constexpr int kSharedGroups = 512;      // workgroups: two fill a compute unit

static size_t shared_rows_bytes(const leoam_pages* s) { return ((size_t)s->batch * s->n_kv_heads * sizeof(SharedRow) + 255) / 256 * 256; }
constexpr size_t kStateBytes = (LEOAM_D + 2) * sizeof(float);
static size_t shared_fixed_bytes(const leoam_pages* s) { return shared_rows_bytes(s) + 2 * (size_t)s->batch * s->n_q_heads * kStateBytes; }
static size_t shared_slot_bytes() { return 2 * (size_t)kSharedColumns * kStateBytes; }      // of a workgroup
size_t page_shared_workspace_bytes(const leoam_pages* s, int) { return shared_fixed_bytes(s) + kSharedGroups * shared_slot_bytes(); }
size_t page_shared_min_workspace_bytes(const leoam_pages* s) { return shared_fixed_bytes(s) + shared_slot_bytes(); }

template <typename T, typename S> static hipError_t launch_shared(const PageSharedArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((page_shared_kernel<T, S>), dim3(a.sharers), dim3(kAttThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(page_shared_merge_kernel, dim3((a.n_heads + 1) / 2), dim3(2 * LEOAM_D), 0, stream, a.rows, a.acc, a.ml,
                       a.group_shift, a.n_heads, a.sharers, shared_bias<T>(), a.out, a.lse);
    return hipGetLastError();
}

hipError_t page_shared_dispatch(const leoam_pages* s, const void* q, const void* k_pages, const void* v_pages, const float* k_scale,
                                const float* v_scale, const int32_t* page_table, const int32_t* seq_len, int n_groups,
                                const int32_t* group_off, const int32_t* group_pages, float softmax_scale, float* out, float* lse,
                                void* workspace, size_t workspace_bytes, hipStream_t stream) {
    PageSharedArgs a;
    a.q = (const char*)q; a.k_pages = (const char*)k_pages; a.v_pages = (const char*)v_pages;
    a.k_scale = k_scale; a.v_scale = v_scale; a.page_table = page_table; a.seq_len = seq_len;
    a.group_off = group_off; a.group_pages = group_pages; a.n_groups = n_groups;
    // (tokens that do not count have -inf before it is scaled: a scale of zero is the smallest there is instead)
    a.scale_log2 = fmaxf(fabsf(softmax_scale) * kLog2e, FLT_MIN);
    a.flip = softmax_scale < 0.f ? (s->q_dtype == LEOAM_F32 ? 0x80000000u : 0x80008000u) : 0u;
    a.out = out; a.lse = lse;
    char* ws = (char*)workspace;
    a.rows = (SharedRow*)ws;
    const size_t fit = (workspace_bytes - shared_fixed_bytes(s)) / shared_slot_bytes();
    a.sharers = (int)(fit < (size_t)kSharedGroups ? fit : (size_t)kSharedGroups);
    a.n_heads = s->batch * s->n_q_heads;
    a.acc = (float*)(ws + shared_rows_bytes(s));
    a.ml = a.acc + (2 * (size_t)a.n_heads + 2 * (size_t)a.sharers * kSharedColumns) * LEOAM_D;
    a.batch = s->batch; a.n_kv_heads = s->n_kv_heads; a.group_shift = __builtin_ctz((unsigned)(s->n_q_heads / s->n_kv_heads));
    a.n_pages = s->n_pages; a.page_shift = __builtin_ctz((unsigned)s->page_size); a.max_pages = s->max_pages;
    const bool k8 = s->kv_dtype == LEOAM_E4M3;
    switch (s->q_dtype) {
    case LEOAM_F32: return launch_shared<F32, F32>(a, stream);
    case LEOAM_F16: return k8 ? launch_shared<F16, E4M3>(a, stream) : launch_shared<F16, F16>(a, stream);
    default: return k8 ? launch_shared<BF16, E4M3>(a, stream) : launch_shared<BF16, BF16>(a, stream);
    }
}

}  // namespace leoam
