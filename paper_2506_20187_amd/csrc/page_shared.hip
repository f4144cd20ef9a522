// page_attention_decode_shared: softmax(scale q K^T) V of one token per sequence where groups of sequences list the same leading
// pages: a group's prefix is read once for all of its members, each sequence's further pages by itself.
//
// HBM-bound up to some 64 (member, head) columns per kv head.  Beyond, nothing is at its limit (48 behind 32768: 3.9 TB/s, matrix cores
// 26 %, vector ALU 38 %): a wave's tile is staged, multiplied, weighed, split and multiplied in turn, with a barrier each.  A unit of work
// is (up to 128 columns of a group, kv head) over the group's prefix, or (sequence, kv head) over its own tokens.  The tiles of all
// units are laid end to end, each unit's beginning counted as some more, and shared out equally: the host does not know the
// lengths.  A unit cut by the ends of shares leaves its pieces, (acc[128], m, l) per column, in the workspace; a second
// kernel folds a head's pieces of its group's unit and of its own, in order, so results do not depend on scheduling.
//
// Up to 64 columns everything runs on the matrix cores without passing through LDS, as in page_attention_decode: S^T = K Q^T, lane =
// column, registers = tokens, then O^T = V^T P^T.  A wave has one or two blocks of 16 columns, so what it fetches is used twice; beyond 32
// columns two waves share tokens, with half of the columns each.  Beyond 64 the waves have 32 columns each and tiles of 64 keys go
// through LDS, with 32x32 products as in page_attention_prefill: a key row from the caches is 16 bytes of 16 rows a load, which
// the first-level cache serves at a quarter of its rate, four times over.  Weights go in as two fp16 or three bf16 numbers that add up to
// them (22 or 24 bits), so the float output keeps its precision, at twice the cost of rounded ones beyond 64 columns.
//
// 48 sequences behind 32768 tokens, 32 of 8 heads, bf16: 91 us (221 MB and 26 GFLOP; each by itself, as page_attention_decode has it,
// would read 6.6 GB); 70 of 64 heads in nine groups behind 9000, 8 bits: 88; four of 8 heads behind 1024, fp32: 16, launches and
// dependent round trips.
#include <cfloat>

#include "page_common.h"

namespace leoam {

// Where the state of a (sequence, kv head) is: pieces in slots (count > 0), one whole state (kWhole), the result is final (kFinal),
// nothing (0).
constexpr int kWhole = -1, kFinal = -2;
struct SharedRow { int32_t own_count, own_slot, pre_count, pre_slot, pre_col; };

constexpr int kSharedTile = 64;           // unit of the partition, tokens
constexpr int kSharedColumns = 128;       // most columns of a unit
constexpr int kWaveColumns = 32;
constexpr int kGroupsInLds = 512;

constexpr int kSharedStart = 6, kMostTileCost = 6;
// Most pieces of a unit: a head's are folded one batch after another, which lasts longer than what more workgroups save (us with 64,
// 128, 192 and as many as there are workgroups: 8 heads of one kv head behind 65536 tokens, 8 sequences 46, 34, 31, 47, 4 of 4 heads 28,
// 23, 25, 33).
constexpr int kMostPieces = 128;

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
// (us for 48 sequences behind 32K in bf16, 70 in nine groups in 8 bits, 128 behind 8000, 19 of 16 heads in four groups in fp32: 91, 89, 68,
// 24; with beginnings of 4 99, 100, 72, 24, of 8 92, 91, 70, 24; two and four ways at 3 and 4 95, 89, 73, 26; tiles of 128 93, 88, 77, 34.)
__device__ __forceinline__ int tile_cost(int ways) { return ways == 1 ? 2 : ways == 2 ? 4 : kMostTileCost; }

__device__ __forceinline__ int shared_tiles(int tokens) { return max(1, (tokens + kSharedTile - 1) / kSharedTile); }
// A sequence's own tokens that are this few: where there are more (sequence, kv head) pairs than half the workgroups, a unit is four of
// its heads, one to a wave, and is not cut.  (Us, a head to a unit : four: 126 sequences with a token of their own, 32 kv heads, in 8
// bits 65 : 35, 128 behind 1000 with 100 to 120, 8 heads, bf16 30.2 : 29.9, 93 of up to 71, 4 heads, fp32 35 : 25; with 64 tokens at most
// 31.5 and 31 of the latter two, with 256 nothing more.)
constexpr int kBundleTokens = 128;
__device__ __forceinline__ int bundle_cost(int tokens) { return 1 + 2 * ((tokens + 31) / 32); }

// of the waves, over a unit's columns
__device__ __forceinline__ int ways_of(int n_cols) { return n_cols <= kWaveColumns ? 1 : n_cols <= 2 * kWaveColumns ? 2 : 4; }

// a / b of numbers that are not negative; a division in 64 bits takes a microsecond, and they rarely need it
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return (unsigned long long)(a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}

// a 64-bit value that is the same in all lanes, to scalar registers
__device__ __forceinline__ long long uniform64(long long v) {
    return (long long)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}

// A value that the compiler takes for a new one, so that what is computed from it stays where it is used: what depends on the lane
// alone it would compute for all walks ahead of the loop over units, in more registers than there are (51 of them in scratch memory,
// 27 MB a launch).
__device__ __forceinline__ int here(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// Units of an entry (a group's prefix, or a sequence's own tokens): `full` ones of most columns, then `rest` of the others.
struct SharedEntry {
    int full, rest, tiles, cost_full, cost_rest;
    // (fewer than 2^23 tiles)
    __device__ __forceinline__ int length(int unit) const { return kSharedStart + tiles * cost(unit); }
    __device__ __forceinline__ int cost(int unit) const { return unit < full ? cost_full : cost_rest; }
    __device__ __forceinline__ long long total() const {
        return (long long)full * length(0) + (long long)rest * (kSharedStart + tiles * cost_rest);
    }
};

template <typename T, typename S>
__global__ __launch_bounds__(kAttThreads) __attribute__((amdgpu_waves_per_eu(2))) void page_shared_kernel(PageSharedArgs a) {
    using Step = SharedStep<T, S>;
    constexpr bool k8 = Step::k8, k32 = Step::k32;
    constexpr int ROWB = LEOAM_D * S::kBytes, QROWB = Row<T>::kRowBytes, NT = Step::NT, NK = Step::NK, STEP = 16 * NT, NQ = k32 ? 8 : 4;
    constexpr float kBias = shared_bias<T>();
    constexpr int kParts = T::kTag == LEOAM_F16 ? 2 : 3;
    constexpr int kStride = LEOAM_D + 4;      // of a column in LDS: its accumulators, maximum and sum
    constexpr int KEYS = k32 ? 32 : 64, KSTR = kKeyStride<T>, VSTR = kValueStride<T>;      // of a tile in LDS
    constexpr int kTilesBytes = 2 * KEYS * (KSTR + VSTR), kStatesBytes = kAttWaves * kWaveColumns * kStride * (int)sizeof(float);
    __shared__ __align__(16) char smem[kTilesBytes > kStatesBytes ? kTilesBytes : kStatesBytes];
    float (*xw)[kWaveColumns][kStride] = reinterpret_cast<float (*)[kWaveColumns][kStride]>(smem);
    __shared__ int sh_off[kGroupsInLds + 1], sh_pages[kGroupsInLds];
    __shared__ long long sh_sum[kAttWaves], sh_at;
    __shared__ int sh_entry, sh_longest[kAttWaves];

    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE);
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
    const bool bundles = hkv > 1 && (long long)a.batch * hkv > a.sharers / 2;
    auto bundled = [&](int tokens) { return bundles && tokens <= kBundleTokens; };
    // entries: groups, then sequences
    auto entry_of = [&](int e) {
        if (e < a.n_groups) {
            const int members = off_of(e + 1) - off_of(e), tokens = prefix_of(e);
            if (members <= 0 || tokens == 0) return SharedEntry{0, 0, 0, 1, 1};
            const int full = members / most_members, rest = members - full * most_members;
            return SharedEntry{full * hkv, rest ? hkv : 0, shared_tiles(tokens), tile_cost(4), tile_cost(ways_of(rest << a.group_shift))};
        }
        const int b = e - a.n_groups, len = length_of(b), tokens = len - before_of(b, len);
        if (bundled(tokens)) return SharedEntry{0, (hkv + kAttWaves - 1) / kAttWaves, 1, 1, bundle_cost(tokens)};
        return SharedEntry{0, hkv, shared_tiles(tokens), 1, tile_cost(1)};
    };
    const int n_entries = a.n_groups + a.batch;
    long long pos, end, share, first;      // its places on the line of all costs, [first, end), and where on it the work is
    int entry, unit, off;                   // off: how far into the unit
    {
        const int per = (n_entries + kAttThreads - 1) / kAttThreads, e0 = min(tid * per, n_entries), e1 = min(e0 + per, n_entries);
        long long mine = 0;
        int longest = 0;      // unit of them
        for (int e = e0; e < e1; ++e) {
            const SharedEntry x = entry_of(e);
            mine += x.total();
            longest = max(longest, x.full ? x.length(0) : x.length(x.full));
        }
        long long incl = mine;
#pragma unroll
        for (int d = 1; d < LEOAM_WAVE; d <<= 1) {
            const long long o = __shfl_up(incl, d, LEOAM_WAVE);
            if (lane >= d) incl += o;
        }
#pragma unroll
        for (int d = 1; d < LEOAM_WAVE; d <<= 1) longest = max(longest, __shfl_xor(longest, d, LEOAM_WAVE));
        if (lane == LEOAM_WAVE - 1) {
            sh_sum[wave] = incl;
            sh_longest[wave] = longest;
        }
        __syncthreads();
        long long total = 0, before = incl - mine;
#pragma unroll
        for (int w = 0; w < kAttWaves; ++w) {
            if (w < wave) before += sh_sum[w];
            total += sh_sum[w];
            longest = max(longest, sh_longest[w]);
        }
        total = uniform64(total);
        longest = uniform(longest);
        // (a tile begins in each, and a unit is not cut into more pieces than pay)
        share = max(quotient(total + a.sharers - 1, a.sharers), (long long)max(kMostTileCost, (longest + kMostPieces - 1) / kMostPieces));
        pos = first = share * blockIdx.x;
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
        const long long at = sh_at, full = (long long)x.full * x.length(0), in = at < full ? at : at - full;
        const int length = at < full ? x.length(0) : x.length(x.full);
        unit = uniform((int)quotient(in, length));
        off = uniform((int)(in - (long long)unit * length));
        if (at >= full) unit += uniform(x.full);
    }

    // a piece of a query as it takes part: with its sign turned, or zero
    auto settle = [&](uint4& q, bool counts) {
        q = counts ? make_uint4(q.x ^ a.flip, q.y ^ a.flip, q.z ^ a.flip, q.w ^ a.flip) : make_uint4(0, 0, 0, 0);
    };
    // One stretch of a unit: tokens [t_begin, t_end) of row b_table, for this wave's columns, NB blocks of 16, WAYS of the four waves on
    // columns of their own (four: each on those of a head, h).  rows, counts: the lane's row of q in each block, and whether the column
    // is one.
    auto walk = [&](auto blocks, auto apart, int b_table, int h, int t_begin, int t_end, int n_cols, const size_t* rows, const bool* counts,
                    auto&& leave) {
        const int lane = here(lane_id()), tid = here(threadIdx.x), grp = lane >> 4, l16 = lane & 15;
        constexpr int NB = decltype(blocks)::value, WAYS = decltype(apart)::value, STREAMS = kAttWaves / WAYS;
        uint4 qb[NB][NQ];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int s = 0; s < NQ; ++s) {
                // 16-byte pieces in the order in which a key row's loads hold the channels
                const int byte = k32 ? 64 * s + 16 * grp : k8 ? 128 * (s >> 1) + 32 * grp + 16 * (s & 1) : 64 * s + 16 * grp;
                qb[n][s] = load16(a.q, rows[n] * QROWB + byte);
            }
        const int n_steps = (t_end - t_begin + STEP - 1) / STEP, per = (n_steps + STREAMS - 1) / STREAMS;
        const int s0 = min(n_steps, wave / WAYS * per), s1 = min(n_steps, s0 + per);

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
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int s = 0; s < NQ; ++s) settle(qb[n][s], counts[n]);
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
        __syncthreads();      // (what the previous stretch left in LDS has been read)
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
            const int c = i / (LEOAM_D / 4), d = 4 * (i % (LEOAM_D / 4)), in = WAYS == 4 ? c & (group - 1) : c % kWaveColumns;
            const int w0 = WAYS == 1 ? 0 : WAYS == 4 ? c >> a.group_shift : c / kWaveColumns;
            float ms[STREAMS], ls[STREAMS], m = -INFINITY, l = 0.f;
            float4 x[STREAMS], v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < STREAMS; ++k) {
                const float* state = xw[w0 + k * WAYS][in];
                x[k] = *reinterpret_cast<const float4*>(state + d);
                ms[k] = state[LEOAM_D];
                ls[k] = state[LEOAM_D + 1];
                m = fmaxf(m, ms[k]);
            }
#pragma unroll
            for (int k = 0; k < STREAMS; ++k) {
                const float f = exp2_or_zero(ms[k], m);
                l += f * ls[k];
                v.x += f * x[k].x; v.y += f * x[k].y; v.z += f * x[k].z; v.w += f * x[k].w;
            }
            leave(c, d, v, m, l);
        }
    };

    // The same for more than 64 columns, 32 of them a wave's: the workgroup's tiles of 64 keys (fp32: 32) go through LDS, the next (8 bits:
    // the next two) on its way to registers.
    auto walk_tiles = [&](int b_table, int h, int t_begin, int t_end, int n_cols, size_t my_row, bool counts, auto&& leave) {
        constexpr int KB = KEYS / 32, PIECES = ROWB / 16, LOADS = KEYS * PIECES / kAttThreads, ROWS_PER_LOAD = kAttThreads / PIECES;
        constexpr int GROUPS = KEYS / 16, AHEAD = k8 ? 2 : 1, NQ32 = k32 ? 16 : 8;      // (16 keys never straddle a page)
        constexpr uint32_t kAllOk = (1u << GROUPS) - 1;
        char *sh_k = smem, *sh_v = smem + 2 * KEYS * KSTR;
        const int lane = here(lane_id()), tid = here(threadIdx.x), half = lane >> 5, l32 = lane & 31;
        const int32_t* table = a.page_table + (size_t)b_table * a.max_pages;
        const uint32_t head_bytes = (uint32_t)ROWB << a.page_shift, page_bytes = head_bytes * (uint32_t)hkv;
        const uint32_t in_page = (1u << a.page_shift) - 1;
        const char *kh = a.k_pages + (size_t)h * head_bytes, *vh = a.v_pages + (size_t)h * head_bytes;
        const int n_tiles = (t_end - t_begin + KEYS - 1) / KEYS;
        // lane l looks after 16-key group l % GROUPS of a tile; groups behind the end have no page
        auto pages_of = [&](int j) {
            const int t = t_begin + j * KEYS + 16 * (lane % GROUPS);
            return t < t_end ? table[t >> a.page_shift] : -1;
        };
        int id = pages_of(0);
        uint4 qb[NQ32];
#pragma unroll
        for (int s = 0; s < NQ32; ++s) qb[s] = load16(a.q, my_row * QROWB + 32 * s + 16 * half);
        struct Tile {
            uint4 k[LOADS], v[LOADS];
            float ks[LOADS], vs[LOADS];
            uint32_t ok;      // bit g: group g has a page
        };
        // id: the lane's page in tile j; afterwards - on its way ahead of the rows - in the tile behind it
        auto fetch = [&](int j, int& id, Tile& t) {
            const bool ok = (uint32_t)id < (uint32_t)a.n_pages;
            t.ok = (uint32_t)__ballot(ok) & kAllOk;
            const uint32_t page = ok ? (uint32_t)id : 0u;
            const uint64_t begin = (uint64_t)page * page_bytes;
            const int lo = (int)(uint32_t)begin, hi = (int)(uint32_t)(begin >> 32);
            id = pages_of(min(j + 1, n_tiles - 1));
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                // a load's 16-key group is the same for the wave
                constexpr int kPerLoad = ROWS_PER_LOAD > 16 ? ROWS_PER_LOAD / 16 : 1;      // groups of one load: waves differ
                const int r = i * ROWS_PER_LOAD + tid / PIECES;
                const int g = i * ROWS_PER_LOAD / 16 + (kPerLoad > 1 ? wave * (LEOAM_WAVE / PIECES) / 16 : 0);
                const uint32_t at = ((uint32_t)(t_begin + j * KEYS + r) & in_page) * ROWB + 16 * (tid % PIECES);
                const uint64_t base =
                    (uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, g) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, g);
                t.k[i] = load16(kh + base, at);
                t.v[i] = load16(vh + base, at);
                if (k8) {
                    const size_t row = (size_t)(uint32_t)__builtin_amdgcn_readlane((int)page, g) * hkv + h;
                    t.ks[i] = a.k_scale[row];
                    t.vs[i] = a.v_scale[row];
                }
            }
        };
        auto stage = [&](int buf, Tile& t) {
            if (t.ok != kAllOk) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    if (t.ok >> ((i * ROWS_PER_LOAD + tid / PIECES) / 16) & 1) continue;
                    t.v[i] = make_uint4(0, 0, 0, 0);      // nothing there: no value may matter
                    t.vs[i] = 1.f;
                }
            }
            char *kt = sh_k + buf * KEYS * KSTR, *vt = sh_v + buf * KEYS * VSTR;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int r = i * ROWS_PER_LOAD + tid / PIECES, piece = tid % PIECES;
                if constexpr (k8) {
                    store16(kt, r * KSTR + 32 * piece, widen8<T>(t.k[i].x, t.k[i].y, t.ks[i]));
                    store16(kt, r * KSTR + 32 * piece + 16, widen8<T>(t.k[i].z, t.k[i].w, t.ks[i]));
                    store16(vt, r * VSTR + 32 * piece, widen8<T>(t.v[i].x, t.v[i].y, t.vs[i]));
                    store16(vt, r * VSTR + 32 * piece + 16, widen8<T>(t.v[i].z, t.v[i].w, t.vs[i]));
                } else {
                    store16(kt, r * KSTR + 16 * piece, t.k[i]);
                    store16(vt, r * VSTR + 16 * piece, t.v[i]);
                }
            }
        };

        f32x16_t acc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
        float m_run = -INFINITY, l_run = 0.f;
        const uint32_t k_lane = l32 * KSTR + 16 * half;
        const uint32_t v_lane = k32 ? 4 * half * VSTR + 4 * l32
                                    : (4 * half + (lane & 15) / 4) * VSTR + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
        // lane = column, register r of key block kb = key 32 kb + 8 (r / 4) + 4 half + r % 4
        auto work = [&](int buf, uint32_t ok) {
            constexpr int NB = KB;
            const char *kt = sh_k + buf * KEYS * KSTR + k_lane, *vt = sh_v + buf * KEYS * VSTR + v_lane;
            f32x16_t s[NB];
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
                for (int i = 0; i < NQ32; ++i) {
                    const uint4 ka = load16(kt, 32 * kb * KSTR + 32 * i);
                    if constexpr (k32) {
                        float kx[4], qx[4];
                        unpack<F32>(ka, kx);
                        unpack<F32>(qb[i], qx);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(kx[e], qx[e], s[kb], 0, 0, 0);
                    } else {
                        s[kb] = mfma_32x32x16<T>(ka, qb[i], s[kb]);
                    }
                }
            }
            if (ok != kAllOk) {
#pragma unroll
                for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (!(ok >> (2 * kb + r / 8) & 1)) s[kb][r] = -INFINITY;
            }
            float mt = s[0][0];
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) mt = fmaxf(mt, s[kb][r]);
            {
                float x = mt, y = mt;
                permlane32_swap(x, y);
                mt = fmaxf(x, y) * a.scale_log2 - kBias;
            }
            if (__ballot(mt > m_run + kSharedLag)) {
                const float m = fmaxf(m_run, mt), c = exp2_or_zero(m_run, m);
                m_run = m;
                l_run *= c;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][r] *= c;
            }
            const float ref = m_run == -INFINITY ? 0.f : m_run;
            if constexpr (k32) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[0][r] = exp2_raw(fmaf(s[0][r], a.scale_log2, -ref));
                    l_run += s[0][r];
#pragma unroll
                    for (int db = 0; db < 4; ++db) {
                        const float v = *reinterpret_cast<const float*>(vt + (8 * (r / 4) + r % 4) * VSTR + 128 * db);
                        acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[0][r], acc[db], 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int t = 0; t < 2 * NB; ++t) {      // 16 keys
                    float p[8];
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        p[r] = exp2_raw(fmaf(s[t / 2][8 * (t % 2) + r], a.scale_log2, -ref));
                        l_run += p[r];
                    }
                    uint4 parts[kParts];
#pragma unroll
                    for (int k = 0; k < kParts; ++k) {
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float u, v;
                            w[i] = pair_of(T{}, p[2 * i], p[2 * i + 1]);
                            pair_back(T{}, w[i], u, v);
                            p[2 * i] -= u;      // (exact: what is left has fewer bits)
                            p[2 * i + 1] -= v;
                        }
                        parts[k] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
#pragma unroll
                    for (int db = 0; db < 4; ++db) {
                        // the lane's address is that of 4 channels of one key; what it gets is one channel of 4 keys
                        const uint2 w0 = transposed(vt + 16 * t * VSTR + 64 * db), w1 = transposed(vt + (16 * t + 8) * VSTR + 64 * db);
#pragma unroll
                        for (int k = 0; k < kParts; ++k) acc[db] = mfma_32x32x16<T>(make_uint4(w0.x, w0.y, w1.x, w1.y), parts[k], acc[db]);
                    }
                }
            }
        };

        const bool idle = kWaveColumns * wave >= n_cols;      // none of the wave's columns is one
        __syncthreads();                                       // (what the previous stretch left in LDS has been read)
        {
            Tile even, odd;
            fetch(0, id, even);
            if constexpr (AHEAD == 2) fetch(min(1, n_tiles - 1), id, odd);
#pragma unroll
            for (int s = 0; s < NQ32; ++s) settle(qb[s], counts);
            stage(0, even);
            uint32_t ok = even.ok;
            __syncthreads();
            // Tile j is worked on, then `in` is staged; `to` takes in tile j + AHEAD.  (No branch around the loads and none that leads
            // back, or the compiler has everybody wait for the second tile too.)
            int j = 0;
            auto step = [&](Tile& in, Tile& to) {
                if (AHEAD == 2 || j + 1 < n_tiles) fetch(min(j + AHEAD, n_tiles - 1), id, to);
                if (!idle) work(j & 1, ok);
                if (++j == n_tiles) return false;
                stage(j & 1, in);
                ok = in.ok;
                __syncthreads();
                return true;
            };
            if constexpr (AHEAD == 1) {
                while (step(even, even)) {}
            } else {
                while (step(odd, even) && step(even, odd)) {}
            }
        }
        l_run += shfl_xor_f(l_run, 32);
        const int c = kWaveColumns * wave + l32;
        if (c >= n_cols) return;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                leave(c, 32 * db + 2 * r + 4 * half, make_float4(acc[db][r], acc[db][r + 1], acc[db][r + 2], acc[db][r + 3]), m_run, l_run);
    };

    bool first_piece = true;
    while (pos < end) {
        const int lane = here(lane_id()), tid = here(threadIdx.x), l16 = lane & 15;
        const SharedEntry x = entry_of(entry);
        const int units = uniform(x.full + x.rest);
        if (units == 0) {      // (a group without a prefix)
            ++entry;
            continue;
        }
        const int tiles = uniform(x.tiles), cost = uniform(x.cost(unit));
        const int take = uniform((int)min((long long)(kSharedStart + tiles * cost - off), end - pos));
        // tiles that begin in the share
        auto tiles_before = [&](int at) {
            return at <= kSharedStart ? 0 : (int)((uint32_t)(at - kSharedStart + cost - 1) / (uint32_t)cost);
        };
        const int tile0 = tiles_before(off), tile1 = min(tiles, tiles_before(off + take));
        if (tile0 < tile1) {
            int h = unit % hkv;
            const bool prefix = entry < a.n_groups, whole = tile1 - tile0 == tiles;
            const int slot = 2 * (int)blockIdx.x + (first_piece ? 0 : 1);      // opens the share, or closes it
            // pieces of the unit, and where the first lies, if it begins here
            const long long last_at = pos - first - off + kSharedStart + (long long)(tiles - 1) * cost;
            const int count = whole ? kWhole : tile0 ? 1 : (int)quotient(last_at, share) + 1;
            int n_cols, b0, tokens, before = 0, b_table;
            bool work = true, bundle = false;
            if (prefix) {
                b0 = off_of(entry) + unit / hkv * most_members;
                const int members = min(off_of(entry + 1) - b0, most_members);
                n_cols = members << a.group_shift;
                tokens = prefix_of(entry);
                b0 = uniform(b0);
                n_cols = uniform(n_cols);
                // the first member that has the whole prefix (at most 128 members, two a lane)
                const int len0 = lane < members ? length_of(b0 + lane) : -1;
                const int len1 = lane + LEOAM_WAVE < members ? length_of(b0 + lane + LEOAM_WAVE) : -1;
                const uint64_t has0 = __ballot(len0 >= tokens), has1 = __ballot(len1 >= tokens);
                b_table = has0 ? b0 + __builtin_ctzll(has0) : has1 ? b0 + LEOAM_WAVE + __builtin_ctzll(has1) : -1;
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
                bundle = bundled(tokens);
                if (bundle) {
                    h = kAttWaves * unit;
                    n_cols = min(kAttWaves, hkv - h) << a.group_shift;
                }
            }
            tokens = uniform(tokens);
            const bool final_ = !prefix && before == 0 && whole;
            if (!prefix && tile0 == 0 && tid < (bundle ? n_cols >> a.group_shift : 1)) {
                SharedRow* r = a.rows + (size_t)b0 * hkv + h + tid;
                r->own_count = final_ ? kFinal : tokens == 0 ? 0 : count;
                r->own_slot = slot;
                if (before == 0) r->pre_count = 0;
            }
            if (work && (tokens > 0 || final_)) {
                // (columns past the last repeat it; what is asked for does not wait for whether it counts)
                auto row_of = [&](int c) {
                    c = min(c, n_cols - 1);
                    if (bundle) return (((size_t)b0 * hkv + h) << a.group_shift) + c;
                    return (((size_t)(b0 + (c >> a.group_shift)) * hkv + h) << a.group_shift) + (c & (group - 1));
                };
                auto counts_of = [&](int c) { return c < n_cols && (!prefix || length_of(b0 + (c >> a.group_shift)) >= tokens); };
                const int t_begin = before + tile0 * kSharedTile, t_end = before + (bundle ? tokens : min(tokens, tile1 * kSharedTile));
                auto leave = [&](int c, int d, const float4& v, float m, float l) {
                    const size_t j = row_of(c);
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
                constexpr std::integral_constant<int, 1> one{};
                constexpr std::integral_constant<int, 2> two{};
                constexpr std::integral_constant<int, 4> four{};
                if (bundle) {
                    const bool has = wave << a.group_shift < n_cols;
                    const size_t rows[1] = {row_of((wave << a.group_shift) + min(l16, group - 1))};
                    const bool counts[1] = {has && l16 < group};
                    walk(one, four, b_table, min(h + wave, hkv - 1), t_begin, has ? t_end : t_begin, n_cols, rows, counts, leave);
                } else if (n_cols <= 2 * kWaveColumns) {
                    const int c0 = (n_cols <= kWaveColumns ? 0 : kWaveColumns * (wave & 1)) + l16;
                    const size_t rows[2] = {row_of(c0), row_of(c0 + 16)};
                    const bool counts[2] = {counts_of(c0), counts_of(c0 + 16)};
                    if (n_cols <= 16) walk(one, one, b_table, h, t_begin, t_end, n_cols, rows, counts, leave);
                    else if (n_cols <= kWaveColumns) walk(two, one, b_table, h, t_begin, t_end, n_cols, rows, counts, leave);
                    else walk(two, two, b_table, h, t_begin, t_end, n_cols, rows, counts, leave);
                } else {
                    const int c = kWaveColumns * wave + (lane & 31);
                    walk_tiles(b_table, h, t_begin, t_end, n_cols, row_of(c), counts_of(c), leave);
                }
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

// A head's pieces: those of its group's unit, then its own.  32 threads take four channels each of eight pieces at a time, all on their
// way together; four such groups share a head's pieces, in order.
constexpr int kMergeParts = 4, kMergeHeads = 2;
constexpr int kMergeThreads = kMergeHeads * kMergeParts * 32;
__global__ __launch_bounds__(kMergeThreads) void page_shared_merge_kernel(const SharedRow* __restrict__ rows, const float* __restrict__ acc,
                                                                          const float* __restrict__ ml, int group_shift, int n_heads,
                                                                          int sharers, int bias, float* __restrict__ out,
                                                                          float* __restrict__ lse) {
    constexpr int kBatch = 8;
    __shared__ float sh_m[kMergeHeads][kMergeParts], sh_l[kMergeHeads][kMergeParts];
    __shared__ __align__(16) float sh_o[kMergeHeads][kMergeParts][LEOAM_D];
    const int t = threadIdx.x % 32, part = threadIdx.x / 32 % kMergeParts, mine = threadIdx.x / (32 * kMergeParts), d = 4 * t;
    const int j = min(kMergeHeads * (int)blockIdx.x + mine, n_heads - 1);      // (the last one twice)
    const SharedRow r = rows[j >> group_shift];
    const bool done = r.own_count == kFinal;
    // (counts and slots that no kernel wrote - lists of groups that overlap - stay within the workspace)
    const int g = j & ((1 << group_shift) - 1), last = 2 * sharers - 1;
    const int n_pre = r.pre_count == kWhole ? 1 : min(max(r.pre_count, 0), sharers);
    const int n_own = r.own_count == kWhole ? 1 : min(max(r.own_count, 0), sharers);
    const int n = done ? 0 : n_pre + n_own;
    auto state = [&](int i) {
        const bool own = i >= n_pre;
        const int k = own ? i - n_pre : i, count = own ? r.own_count : r.pre_count;
        if (count == kWhole) return (size_t)(own ? j : n_heads + j);
        // (each further piece opens the next workgroup's share)
        const int slot0 = own ? r.own_slot : r.pre_slot, slot = min(max(k == 0 ? slot0 : 2 * (slot0 / 2 + k), 0), last);
        const int col = min(max(own ? 0 : r.pre_col, 0), kSharedColumns - (1 << group_shift)) + g;
        return 2 * (size_t)n_heads + (size_t)slot * kSharedColumns + col;
    };
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = part * kBatch; i0 < n; i0 += kMergeParts * kBatch) {
        float ms[kBatch], ls[kBatch];
        float4 os[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const size_t at = state(min(i0 + u, n - 1));
            const float2 x = *reinterpret_cast<const float2*>(ml + 2 * at);
            ms[u] = i0 + u < n ? x.x : -INFINITY;
            ls[u] = x.y;
            os[u] = *reinterpret_cast<const float4*>(acc + at * LEOAM_D + d);
        }
        float mb = m;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) mb = fmaxf(mb, ms[u]);
        const float c = exp2_or_zero(m, mb);
        m = mb;
        l *= c;
        o.x *= c; o.y *= c; o.z *= c; o.w *= c;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i0 + u >= n) continue;
            const float w = exp2_or_zero(ms[u], m);
            l += w * ls[u];
            o.x += w * os[u].x; o.y += w * os[u].y; o.z += w * os[u].z; o.w += w * os[u].w;
        }
    }
    if (t == 0) {
        sh_m[mine][part] = m;
        sh_l[mine][part] = l;
    }
    *reinterpret_cast<float4*>(&sh_o[mine][part][d]) = o;
    __syncthreads();
    if (part || done) return;
    for (int p = 1; p < kMergeParts; ++p) m = fmaxf(m, sh_m[mine][p]);
    // (A part without pieces adds zeros.  One whose logits are all NaN has a maximum of -inf as well, and its NaN stays.)
    l = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int p = 0; p < kMergeParts; ++p) {
        const float w = exp2_or_zero(sh_m[mine][p], m);
        const float4 x = *reinterpret_cast<const float4*>(&sh_o[mine][p][d]);
        l += w * sh_l[mine][p];
        o.x += w * x.x; o.y += w * x.y; o.z += w * x.z; o.w += w * x.w;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;      // (NaN stays)
    *reinterpret_cast<float4*>(out + (size_t)j * LEOAM_D + d) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (lse && t == 0) lse[j] = log_sum_exp(m, l, bias);
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
    hipLaunchKernelGGL(page_shared_merge_kernel, dim3((a.n_heads + kMergeHeads - 1) / kMergeHeads), dim3(kMergeThreads), 0, stream, a.rows,
                       a.acc, a.ml, a.group_shift, a.n_heads, a.sharers, shared_bias<T>(), a.out, a.lse);
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
