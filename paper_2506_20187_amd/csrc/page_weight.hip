// page_weight_add: what every cached token got of the attention of the call's rows, added to what it got before:
// weight[t] = decay weight[t] + sum over the rows that see t and the group's heads of exp(scale q.k_t - lse).
//
// S = K Q^T on the matrix cores, keys as the first operand: a wave holds its keys in registers and goes through the rows sixteen
// (row, head) columns at a time, so the sums of a token stay in registers too and nothing is added by atomics.
// Few rows for each sequence: every key is read once, bound by that.  The stretches of 64 keys (fp32: 32) of all sequences and heads
// are laid end to end and shared out equally to the waves; a wave works on half of one while the next half's keys are on their
// way.  They come as whole rows, which the caches serve at four times the rate of an operand's 16 bytes of 16 rows, and become
// operands in LDS.  Sixteen tokens of sequences to 33001 (617 MB): 125 us, 4.9 TB/s; with operands straight from the loads and no
// equal shares 187; with weights written for 32 keys at a time 134; with lengths and pages looked up when the keys are fetched 129.
// Many rows: the vector ALU (an exponential, a multiply-add, a sum and the mask for each weight) is busy 57 % of the time, the rest goes to
// uneven work: the first stretches have all rows, the last ones few.  The waves of a workgroup share 64 keys (fp32: 32; half as
// many where keys are few) and go through the blocks of columns in turn; their sums are added in order at the end.  Queries, too,
// come as whole rows.  A prompt of 4096 with 32 heads: 114 us (268 M exponentials, 69 GFLOP); with operands straight from the
// loads 191.
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

// tiles of 16 keys that a wave has in registers: few rows; many rows
template <typename T> constexpr int kFewTiles = T::kTag == LEOAM_F32 ? 1 : 2;
template <typename T> constexpr int kManyTiles = T::kTag == LEOAM_F32 ? 2 : 4;

// A stretch of keys: (sequence, kv head), its first key, the sequence's length, its rows of the call and the place of the first
// one's token.
struct WeightUnit { int bh, b, h, t0, len, row0, m, first; };

// 16 (row, head) columns
template <typename T> struct WeightColumns {
    static constexpr int NQ = T::kTag == LEOAM_F32 ? 8 : 4;
    uint4 q[NQ];
    float base;      // lse, log2 domain
    int pos;         // the row's place, -1: no column, or a row that attended to nothing
};

// TILES: of 16 keys, that a wave has in registers
template <typename T, typename S, int G, bool kSplitRows, int TILES> struct Weighing {
    static constexpr bool k8 = std::is_same<S, E4M3>::value, k32 = T::kTag == LEOAM_F32;
    static constexpr int ROWB = LEOAM_D * S::kBytes, QROWB = Row<T>::kRowBytes, NT = TILES, KEYS = 16 * NT;
    static constexpr int NQ = WeightColumns<T>::NQ, NK = k32 ? 8 : k8 ? 2 : 4;
    // Tile j, token l16; a token that does not count re-reads the last one that does.  (Few rows: as they lie in the page, a row by
    // kPieces neighbouring lanes.)
    static constexpr int kPieces = ROWB / 16, kRowsOfLoad = LEOAM_WAVE / kPieces;
    static constexpr int kQPieces = QROWB / 16, kColumnsOfLoad = LEOAM_WAVE / kQPieces;
    struct Keys {
        uint4 k[NT * NK];
        float ks[NT];
        uint32_t have;      // bit j: the tile has a page
    };

    static __device__ __forceinline__ WeightUnit unit_at(const PageWeightArgs& a, int bh, int t0) {
        WeightUnit u;
        u.bh = bh;
        u.b = bh / a.n_kv_heads;
        u.h = bh - u.b * a.n_kv_heads;
        u.len = min(max(scalar_at(a.seq_len, u.b), 0), a.max_pages << a.page_shift);
        u.t0 = t0;
        u.row0 = u.b;
        u.m = 1;
        if (a.new_off) {
            u.row0 = scalar_at(a.new_off, u.b);
            u.m = scalar_at(a.new_off, u.b + 1) - u.row0;
            if (u.row0 < 0 || u.m < 0 || u.m > a.n_new - u.row0) u.m = 0;
        }
        u.first = u.len - u.m;
        return u;
    }
    // columns from the first row that sees a key of the stretch on
    // (few rows: all of them, so that a wave's columns stay what they are)
    static __device__ __forceinline__ int first_row(const WeightUnit& u) { return kSplitRows ? max(0, u.t0 - u.first) : 0; }
    static __device__ __forceinline__ int columns(const WeightUnit& u) { return (u.m - first_row(u)) * G; }

    struct PageIds { int id[NT]; };
    static __device__ __forceinline__ PageIds pages_of(const PageWeightArgs& a, const WeightUnit& u) {
        PageIds p;
#pragma unroll
        for (int j = 0; j < NT; ++j)
            p.id[j] = scalar_at(a.page_table, (size_t)u.b * a.max_pages + (min(u.t0 + 16 * j, u.len - 1) >> a.page_shift));
        return p;
    }
    static __device__ __forceinline__ void fetch_keys(const PageWeightArgs& a, const WeightUnit& u, const PageIds& p, Keys& x) {
        const int lane = lane_id(), grp = lane >> 4, l16 = lane & 15;
        x.have = 0;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int t = min(u.t0 + 16 * j, u.len - 1), valid = min(u.len - (u.t0 + 16 * j), 16), page = p.id[j];
            const bool ok = (uint32_t)page < (uint32_t)a.n_pages && valid > 0;
            x.have |= (ok ? 1u : 0u) << j;
            const size_t row = (size_t)(ok ? page : 0) * a.n_kv_heads + u.h;
            const char* kp = a.k_pages + (row << a.page_shift) * ROWB;
            const uint32_t row0 = t & ((1 << a.page_shift) - 1) & ~15, last = max(valid - 1, 0);
            if constexpr (k8) x.ks[j] = scalar_at(a.k_scale, row);
#pragma unroll
            for (int s = 0; s < NK; ++s) {
                const uint32_t r = kSplitRows ? l16 : s * kRowsOfLoad + lane / kPieces;
                const uint32_t piece = kSplitRows ? 4 * s + grp : lane % kPieces;
                x.k[NK * j + s] = load16(kp, (row0 + min(r, last)) * ROWB + 16 * piece);
            }
        }
    }
    static __device__ __forceinline__ void fetch_columns(const PageWeightArgs& a, const WeightUnit& u, int cb, WeightColumns<T>& c) {
        const int lane = lane_id(), grp = lane >> 4, l16 = lane & 15, n_cols = columns(u);
        const int i0 = first_row(u);
        auto row_of = [&](int col) {      // (columns past the last repeat it)
            col = max(min(16 * cb + col, n_cols - 1), 0);
            return n_cols > 0 ? ((size_t)(u.row0 + i0 + col / G) * a.n_kv_heads + u.h) * G + col % G : 0;
        };
#pragma unroll
        for (int s = 0; s < NQ; ++s) {
            if constexpr (kSplitRows) c.q[s] = load16(a.q, row_of(s * kColumnsOfLoad + lane / kQPieces) * QROWB + 16 * (lane % kQPieces));
            else c.q[s] = load16(a.q, row_of(l16) * QROWB + 16 * query_piece(s, grp));
        }
        const int i = i0 + max(min(16 * cb + l16, n_cols - 1), 0) / G;
        c.base = a.lse[row_of(l16)];
        c.pos = 16 * cb + l16 < n_cols ? u.first + i : -1;
    }
    // Rows into a wave's LDS, and out again as operands: 16-byte piece p of row r lies at p ^ r (low bits), so that a piece of 16 rows is
    // in banks of its own.
    static __device__ __forceinline__ uint32_t lds_at(int r, int p) { return r * ROWB + 16 * (p ^ (r & (kPieces - 1))); }
    static __device__ __forceinline__ void turn(Keys& x, char* lds) {
        const int lane = lane_id(), grp = lane >> 4, l16 = lane & 15;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int s = 0; s < NK; ++s) store16(lds, lds_at(16 * j + s * kRowsOfLoad + lane / kPieces, lane % kPieces), x.k[NK * j + s]);
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int s = 0; s < NK; ++s) x.k[NK * j + s] = load16(lds, lds_at(16 * j + l16, 4 * s + grp));
    }
    // the 16-byte piece of a query that goes with register i of a key's
    static __device__ __forceinline__ int query_piece(int i, int grp) { return k8 ? 8 * (i >> 1) + 2 * grp + (i & 1) : 4 * i + grp; }
    // queries that came as rows, by a wave's LDS (of 16 of them) to operands
    static __device__ __forceinline__ void turn(WeightColumns<T>& c, char* lds) {
        const int lane = lane_id(), grp = lane >> 4, l16 = lane & 15;
        auto at = [&](int r, int p) { return r * QROWB + 16 * (p ^ r); };
#pragma unroll
        for (int s = 0; s < NQ; ++s) store16(lds, at(s * kColumnsOfLoad + lane / kQPieces, lane % kQPieces), c.q[s]);
#pragma unroll
        for (int s = 0; s < NQ; ++s) c.q[s] = load16(lds, at(l16, query_piece(s, grp)));
    }
    // the operand's eight channels (fp32: four) of register i of tile j
    static __device__ __forceinline__ uint4 key(const Keys& x, int j, int i) {
        if constexpr (k8) {
            const uint4 w = x.k[NK * j + i / 2];
            return i & 1 ? widen8<T>(w.z, w.w, x.ks[j]) : widen8<T>(w.x, w.y, x.ks[j]);
        } else {
            return x.k[NK * j + i];
        }
    }
    // One block of columns onto the sums: p = exp2(s q.k - base) where the column sees the key; one that attended to nothing adds 0.
    template <typename K>
    static __device__ __forceinline__ void add(const PageWeightArgs& a, const WeightUnit& u, K&& key_of, const WeightColumns<T>& c,
                                               float (*w)[4]) {
        const int pos = c.base != -INFINITY ? c.pos : -1;
        const float base = c.base * kLog2e;
        if (__ballot(pos < min(u.t0 + KEYS, u.len) - 1)) add_products<true>(a, u, key_of, c, pos, base, w);
        else add_products<false>(a, u, key_of, c, pos, base, w);
    }
    template <bool kMasked, typename K>
    static __device__ __forceinline__ void add_products(const PageWeightArgs& a, const WeightUnit& u, K&& key_of,
                                                        const WeightColumns<T>& c, int pos, float base, float (*w)[4]) {
        const int grp = lane_id() >> 4;
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
                    unpack<F32>(key_of(j, i), kx);
                    unpack<F32>(c.q[i], qx);
#pragma unroll
                    for (int e = 0; e < 4; ++e) chain[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[e], qx[e], chain[e], 0, 0, 0);
                }
                s = (chain[0] + chain[1]) + (chain[2] + chain[3]);
            } else {
#pragma unroll
                for (int i = 0; i < NQ; ++i) s = mfma_16x16x32<T>(key_of(j, i), c.q[i], s);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float p = exp2_raw(fmaf(s[r], a.scale_log2, -base));
                if (kMasked && u.t0 + 16 * j + 4 * grp + r > pos) p = 0.f;
                w[j][r] += p;
            }
        }
    }
    // The columns' sums of N tiles: lane l16 keeps that of register l16 % 4 of tile l16 / 4, token `slot` of the stretch.
    static __device__ __forceinline__ int slot() { return 16 * ((lane_id() & 15) >> 2) + 4 * (lane_id() >> 4) + (lane_id() & 3); }
    static __device__ __forceinline__ bool keeps(const WeightUnit& u, int tiles) {
        return (lane_id() & 15) < 4 * tiles && u.t0 + slot() < u.len;
    }
    static __device__ __forceinline__ size_t place(const PageWeightArgs& a, const WeightUnit& u) {
        return (size_t)u.bh * ((size_t)a.max_pages << a.page_shift) + min(u.t0 + slot(), u.len - 1);
    }
    template <int N> static __device__ __forceinline__ float sums(uint32_t have, const float (*w)[4]) {
        float mine = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float sum = row16_sum(w[j][r]);
                if ((lane_id() & 15) == 4 * j + r && have >> j & 1) mine = sum;      // (no page: nobody attended to it)
            }
        return mine;
    }
    static __device__ __forceinline__ void store(const PageWeightArgs& a, const WeightUnit& u, float was, float mine) {
        const int t = u.t0 + slot();
        const size_t at = place(a, u);
        a.weight[at] = t < u.first && a.before ? fmaf(a.decay, was, mine) : mine;
        if (a.token_id && t >= u.first) a.token_id[at] = a.n_seen[u.b] - (u.len - t);
    }
};

// ---- few rows for each sequence -------------------------------------------------------------------------------
// Workgroups of a compute unit: two (three, with fewer registers each: 150 against 136 us, 16 sequences to 33001), in 8 bits three (16
// sequences of 33001 125 us, two 135).
template <typename S> constexpr int kFewPerUnit = std::is_same<S, E4M3>::value ? 3 : 2;
template <typename T, typename S, int G>
__global__ __launch_bounds__(kAttThreads, kFewPerUnit<S>) void page_weight_few_kernel(PageWeightArgs a) {
    using W = Weighing<T, S, G, false, kFewTiles<T>>;
    __shared__ long long sh_sum[kAttWaves], sh_in[kAttWaves];
    __shared__ int sh_entry[kAttWaves];
    __shared__ __align__(16) char sh_keys[kAttWaves][W::KEYS * W::ROWB];
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE), hkv = a.n_kv_heads;
    constexpr int STRETCH = 2 * W::KEYS;
    auto blocks_of = [&](int len) { return (min(max(len, 0), a.max_pages << a.page_shift) + STRETCH - 1) / STRETCH; };

    // ---- this wave's share of the stretches: `left` of them, from stretch `block` of head h of sequence b on -------
    int b, h, block, left;
    {
        const int per = (a.batch + kAttThreads - 1) / kAttThreads, b0 = min(tid * per, a.batch), b1 = min(b0 + per, a.batch);
        long long mine = 0;
        for (int i = b0; i < b1; ++i) mine += (long long)blocks_of(a.seq_len[i]) * hkv;
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
        // (the first `more` waves take one more than the others)
        const int waves = gridDim.x * kAttWaves, each = (int)(total / waves), more = (int)(total - (long long)each * waves);
        auto begin_of = [&](int w) { return (long long)w * each + min(w, more); };
        long long at = before;
        for (int i = b0; i < b1; ++i) {
            const long long n = (long long)blocks_of(a.seq_len[i]) * hkv;
#pragma unroll
            for (int w = 0; w < kAttWaves; ++w) {
                const long long p = begin_of(blockIdx.x * kAttWaves + w);
                if (p >= at && p < at + n) {
                    sh_entry[w] = i;
                    sh_in[w] = p - at;
                }
            }
            at += n;
        }
        __syncthreads();
        const int w = blockIdx.x * kAttWaves + wave;
        left = each + (w < more ? 1 : 0);
        if (left == 0) return;
        b = uniform(sh_entry[wave]);
        const int n = blocks_of(scalar_at(a.seq_len, b));
        h = uniform((int)(sh_in[wave] / n));
        block = uniform((int)(sh_in[wave] - (long long)h * n));
    }

    // half `half` of stretch `block`
    auto half_at = [&](int half) __attribute__((always_inline)) { return W::unit_at(a, b * hkv + h, block * STRETCH + half * W::KEYS); };
    typename W::Keys even, odd;
    WeightColumns<T> cols;
    int cols_of = -1;      // which (sequence, kv head) they are of
    // (what is looked up - lengths, pages - is looked up a half ahead of the keys that wait for it)
    WeightUnit u = half_at(0), v = half_at(1);      // (the second may lie behind the last token)
    W::fetch_keys(a, u, W::pages_of(a, u), even);
    typename W::PageIds v_pages = W::pages_of(a, v);
    while (left > 0) {
        if (u.bh != cols_of) {
            cols_of = u.bh;
            W::fetch_columns(a, u, 0, cols);
        }
        W::fetch_keys(a, v, v_pages, odd);
        const float was = a.before ? a.before[W::place(a, u)] : 0.f;
        // to the next stretch (behind the share's last: that one again, from the caches)
        if (--left > 0 && ++block * STRETCH >= u.len) {
            block = 0;
            if (++h == hkv) {
                h = 0;
                do ++b;
                while (blocks_of(scalar_at(a.seq_len, b)) == 0);      // (there is one: the share is not at its end)
            }
        }
        const WeightUnit next = half_at(0);
        const typename W::PageIds next_pages = W::pages_of(a, next);
        float w[2 * W::NT][4];
#pragma unroll
        for (int j = 0; j < 2 * W::NT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) w[j][r] = 0.f;
        auto work = [&](const WeightUnit& x, typename W::Keys& keys, float (*sums)[4]) __attribute__((always_inline)) {
            W::turn(keys, sh_keys[wave]);
            auto key_of = [&](int j, int i) { return W::key(keys, j, i); };
            const int n_cols = W::columns(x);
            if (n_cols > 0) W::add(a, x, key_of, cols, sums);
            for (int cb = 1; 16 * cb < n_cols; ++cb) {
                WeightColumns<T> more;
                W::fetch_columns(a, x, cb, more);
                W::add(a, x, key_of, more, sums);
            }
        };
        work(u, even, w);
        const uint32_t have = even.have;
        W::fetch_keys(a, next, next_pages, even);
        const WeightUnit next_v = half_at(1);
        v_pages = W::pages_of(a, next_v);
        work(v, odd, w + W::NT);
        const float mine = W::template sums<2 * W::NT>(have | odd.have << W::NT, w);
        if (W::keeps(u, 2 * W::NT)) W::store(a, u, was, mine);
        u = next;
        v = next_v;
    }
}

// ---- many rows ------------------------------------------------------------------------------------------------
template <typename T, typename S, int G, int TILES, int WAVES>
__global__ __launch_bounds__(WAVES * LEOAM_WAVE, 2) void page_weight_many_kernel(PageWeightArgs a) {
    using W = Weighing<T, S, G, true, TILES>;
    __shared__ float sh[WAVES][W::KEYS];
    __shared__ __align__(16) char sh_queries[WAVES][16 * W::QROWB];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / LEOAM_WAVE), rows_bh = a.batch * a.n_kv_heads;
    for (int unit = blockIdx.x; unit < a.total; unit += gridDim.x) {
        const int block = unit / rows_bh;
        const WeightUnit u = W::unit_at(a, unit - block * rows_bh, block * W::KEYS);
        if (u.t0 >= u.len) continue;
        typename W::Keys keys;
        W::fetch_keys(a, u, W::pages_of(a, u), keys);
        const float was = a.before ? a.before[W::place(a, u)] : 0.f;
        uint4 wide[W::NT * W::NQ];      // (8 bits: widened once)
#pragma unroll
        for (int j = 0; j < W::NT; ++j)
#pragma unroll
            for (int i = 0; i < W::NQ; ++i) wide[W::NQ * j + i] = W::key(keys, j, i);
        auto key_of = [&](int j, int i) { return wide[W::NQ * j + i]; };
        float w[W::NT][4];
#pragma unroll
        for (int j = 0; j < W::NT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) w[j][r] = 0.f;
        const int n_cols = W::columns(u), n_blocks = n_cols > 0 ? (n_cols + 15) / 16 : 0;
        if (wave < n_blocks) {
            // (two blocks a turn, of which the second may be behind the last column and add nothing: were there a branch, the loads would
            // be moved behind it, where they are waited for at once)
            WeightColumns<T> even, odd;
            W::fetch_columns(a, u, wave, even);
            for (int cb = wave; cb < n_blocks; cb += 2 * WAVES) {
                W::fetch_columns(a, u, cb + WAVES, odd);
                W::turn(even, sh_queries[wave]);
                W::add(a, u, key_of, even, w);
                W::fetch_columns(a, u, cb + 2 * WAVES, even);
                W::turn(odd, sh_queries[wave]);
                W::add(a, u, key_of, odd, w);
            }
        }
        float mine = W::template sums<W::NT>(keys.have, w);
        if ((lane_id() & 15) < 4 * W::NT) sh[wave][W::slot()] = mine;
        __syncthreads();
        if (wave == 0 && W::keeps(u, W::NT)) {
            mine = sh[0][W::slot()];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) mine += sh[v][W::slot()];
            W::store(a, u, was, mine);
        }
        __syncthreads();      // (the sums have been read)
    }
}

// More than a block of columns for each sequence on average: many rows.  (On average: the host does not know new_off.  A prompt's chunk
// beside many single tokens is taken for few rows, and each stretch's wave goes through all of its columns: 700 rows and 255 tokens
// behind 1000, 32 of 8 heads, bf16 2690 us, in calls of their own 18 and 105.)
constexpr int kFewColumns = 16;
constexpr int kManyGroups = 65536;

// Waves that share a stretch of many rows: one, where the stretches by themselves fill the card (a workgroup of eight is alone on its
// compute unit, and its loads are waited for at each stretch: 64 rows behind 32001 tokens 39 us, four waves 58, eight 110); more,
// where few stretches would leave it idle (256 rows behind 2000 36, 14, 13; prompt of 4096 530, 168, 129).  Prompts without much
// before them take more: the last stretches have few rows, the first ones all (8 prompts of 4096 1078, 865, 888).  Very few stretches
// are halved as well (prompt of 1024 with 8 kv heads 134, 41, 31 and 24 us; two of 1250 with 4 163, 51, 38, 29; of 4096, which has
// enough of them, 124 and 172), and with fewer columns four waves share those (50 rows behind 1000, one wave and four: 11.1, 6.2; of
// two sequences 11.0, 7.6; fp32 24, 12.6).
// The stretches are those that the table has room for, since the host does not know the lengths: the figures are of tables a page wider
// than the sequences.  In much wider ones prompts are taken for rows behind long histories and get a wave (prompt of 4096
// in a table of 16384 tokens 528 us, of 131072 546; of 1024 in either 134; two of 1250 with 4 heads 164).
struct ManyShape { int waves; bool half; };
static ManyShape many_shape(long long stretches, long long columns, bool prompts) {
    if (columns < 64) return {1, false};
    if (columns < 256) return stretches <= 512 ? ManyShape{4, true} : ManyShape{1, false};
    if (stretches <= 256) return {8, true};
    if (columns >= 512 && prompts && stretches <= 1024) return {8, false};
    return {prompts || stretches <= 1024 ? 4 : 1, false};
}

template <typename T, typename S, int G> static hipError_t launch_weight(PageWeightArgs a, hipStream_t stream) {
    const long long capacity = (long long)a.max_pages << a.page_shift, columns = (long long)a.n_new * G;
    const bool many = columns > (long long)kFewColumns * a.batch;
    const int block = 16 * (many ? kManyTiles<T> : 2 * kFewTiles<T>);
    const long long total = (capacity + block - 1) / block * a.batch * a.n_kv_heads;
    if (total > 0x7fffffffll - kManyGroups) return hipErrorInvalidValue;
    a.total = (int)total;
    if (!many) {
        constexpr int most = 256 * kFewPerUnit<S>;
        const long long groups = (total + kAttWaves - 1) / kAttWaves;
        const dim3 grid((unsigned)(groups < most ? groups : most));
        hipLaunchKernelGGL((page_weight_few_kernel<T, S, G>), grid, dim3(kAttThreads), 0, stream, a);
        return hipGetLastError();
    }
    auto many_rows = [&](auto tiles, auto waves) {
        constexpr int TILES = decltype(tiles)::value, WAVES = decltype(waves)::value;
        const long long units = (capacity + 16 * TILES - 1) / (16 * TILES) * a.batch * a.n_kv_heads;
        a.total = (int)units;
        hipLaunchKernelGGL((page_weight_many_kernel<T, S, G, TILES, WAVES>), dim3((unsigned)(units < kManyGroups ? units : kManyGroups)),
                           dim3(WAVES * LEOAM_WAVE), 0, stream, a);
    };
    constexpr std::integral_constant<int, kManyTiles<T>> wide{};
    constexpr std::integral_constant<int, kManyTiles<T> / 2> half{};
    constexpr std::integral_constant<int, 8> eight{};
    constexpr std::integral_constant<int, 4> four{};
    const ManyShape shape = many_shape(total, columns / a.batch, 2ll * a.n_new >= a.batch * capacity);
    if (shape.half && shape.waves == 8) many_rows(half, eight);
    else if (shape.half) many_rows(half, four);
    else if (shape.waves == 8) many_rows(wide, eight);
    else if (shape.waves == 4) many_rows(wide, four);
    else many_rows(wide, std::integral_constant<int, 1>{});
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
