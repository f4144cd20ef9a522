// page_attention_decode: softmax(scale q K^T) V of one token per sequence over its pages, all of them or the kept ones.
//
// HBM-bound: every stored key and value is read once.  The work of a call is the tokens of all (sequence, kv head)
// rows laid end to end in tiles; every workgroup takes an equal, contiguous share of the tiles (and of the rows' beginnings,
// kRowStart), whatever the lengths are (the host does not know them), and its four waves take a quarter of each stretch.  A share covers whole rows,
// whose results are final, and at most two pieces of rows, which leave (acc[128], m, l) per head in the
// workspace; a second small kernel folds a row's pieces in order, so results do not depend on scheduling.
//
// Where rows are short (uncut_row_tiles) a workgroup takes a row instead, and nothing is cut.
//
// Everything runs on the matrix cores without passing through LDS.  S^T = K Q^T: lane = token takes the 16-byte
// loads of its key row as they are.  The result has lane = query head, registers = tokens, which is what the second
// product O^T = V^T P^T wants of P; and because the order of the tokens in a contraction and of the channels
// among the rows of a product is free, lane l of a 16-lane group loads channels 8l..8l+7 of the four tokens 4g..4g+3 whose
// weights its group holds, and the operand (eight tokens of one channel) is put together from them by byte permutes.
// P goes in as two fp16 or three bf16 numbers that add up to it (22 or 24 bits), so the float output keeps its precision;
// the matrix cores are idle otherwise.  fp32 keys are contracted in four chains, whose sums are rounded less often.
#include "page_common.h"

namespace leoam {

// merge directory of a row (b, h): pieces (0: its result is final) and where the first lies
struct RowPieces { int32_t count, first_slot; };

constexpr int kTileTokens = 128;          // unit of the partition: 32 tokens for each wave

template <typename T, typename S> struct StepOf;      // what a wave fetches at a time, in registers
template <typename T> struct StepOf<T, T> {           // 16 bits, 32 tokens: K 2 x 4 loads, V 2 x 4 rows
    static constexpr int kTiles = 2;
    uint4 k[8], v[8];
};
template <typename T> struct StepOf<T, E4M3> {        // 8 bits, 32 tokens
    static constexpr int kTiles = 2;
    uint4 k[4];
    uint2 v[8];
};
template <> struct StepOf<F32, F32> {                 // 16 tokens: K 8 loads, V 4 rows x 2
    static constexpr int kTiles = 1;
    uint4 k[8], v[8];
};

// a 16-token tile of the walk (wave-uniform)
struct TileAt {
    uint32_t page;      // physical page, 0 if there is none
    int row0, valid;    // its first token's row in the page; how many of its tokens count
    float ks, vs;       // (loaded with the tile: only its weights and products wait for them)
};

// A row to a workgroup, or shares?  Cutting costs a second start, a fold and a piece per cut, not cutting lets the longest row
// decide.  Rows of at most this many tiles are not cut.  (us, shares against rows, lengths spread from 1 to the given, 8 bits / bf16:
// 160 rows to 900 tokens 15 / 18 : 14 / 14, to 1900 20 / 26 : 22 / 23, to 4000 25 / 38 : 39 / 50; 512 rows to 900 25 / 32 : 20 / 28, to
// 1900 34 / 60 : 32 / 57, to 4000 65 / 110 : 70 / 116; 8 rows to 900 10.6 : 13.5.  fp32: 64 rows to 400 13.5 : 15.0.)
__host__ __device__ __forceinline__ int uncut_row_tiles(int rows, bool k32) { return k32 ? min(max(rows / 32, 1), 32) : min(max(rows / 8, 4), 16); }

// What a row's beginning costs a workgroup, in tiles: its page, query, first keys and the fold.  A share is measured in tiles and
// beginnings, or the workgroup that short rows fall to ends last.  (us with 0, 1, 2, 4: 40 sequences of 1 to 9001 tokens, 8 heads,
// 8 bits 90, 84, 80, 80, bf16 144, 137, 135, 137; 1280 rows to 9000 tokens 308, 302, 286, 288; rows of one length the same.  fp32, whose
// tiles take four times as long, 0: 8 rows of 32 tiles 15.0, with 1 18.6.)
constexpr int kRowStart = 2;

// fp16 weights: the row's maximum is taken 2^15 lower, so that small weights stay clear of fp16's subnormals
template <typename T> constexpr int decode_bias() { return T::kTag == LEOAM_F16 ? 15 : 0; }

struct PageDecodeArgs {
    const char *q, *k_pages, *v_pages;
    const float *k_scale, *v_scale;
    const int32_t *page_table, *seq_len, *sel_idx, *sel_count;
    int k_max;
    float scale_log2;
    float *out, *lse, *partial;
    RowPieces* pieces;       // nullptr: a row to a workgroup, none is cut
    int sharers;             // workgroups that share the tiles if rows are cut
    int batch, n_kv_heads, n_pages, page_shift, max_pages;
};

// tokens of row (b, h)'s walk
__device__ __forceinline__ int walk_of(const PageDecodeArgs& a, int b, int h) {
    if (a.sel_idx) return min(max(a.sel_count[(size_t)b * a.n_kv_heads + h], 0), a.k_max) << a.page_shift;
    return min(max(a.seq_len[b], 0), a.max_pages << a.page_shift);
}
__device__ __forceinline__ int tiles_of(int tokens) { return max(1, (tokens + kTileTokens - 1) / kTileTokens); }

template <typename T, typename S, int G>
__global__ __launch_bounds__(kAttThreads) __attribute__((amdgpu_waves_per_eu(2))) void page_decode_kernel(PageDecodeArgs a) {
    constexpr bool k8 = std::is_same<S, E4M3>::value, k32 = T::kTag == LEOAM_F32;
    constexpr int ROWB = LEOAM_D * S::kBytes, QROWB = Row<T>::kRowBytes, NT = StepOf<T, S>::kTiles;
    constexpr int STEP = 16 * NT, NV = 4 * NT;
    constexpr int kStart = k32 ? 0 : kRowStart;
    constexpr float kBias = decode_bias<T>();
    constexpr int kParts = T::kTag == LEOAM_F16 ? 2 : 3;      // of a weight
    __shared__ float xw[kAttWaves][G][kPartStride];
    __shared__ long long sh_sum[kAttWaves];
    __shared__ long long sh_at;
    __shared__ int sh_entry, sh_tokens, sh_most[kAttWaves];

    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE), grp = lane >> 4, l16 = lane & 15;
    const int hkv = a.n_kv_heads;

    // ---- this workgroup's share of the tiles, or its rows -------------------------------------------------
    const int rows = a.batch * hkv;
    bool whole_rows = a.pieces == nullptr;      // (no row can be long)
    int b = 0, h = 0, off = 0;                   // the row, and the tile in it
    long long share = 1, pos = 0, end = 0;
    int next_tokens = 0;
    if (!whole_rows) {
        // entries: sequences (each hkv rows of the same length), or rows if a selection gives each its own
        const int n_entries = a.sel_idx ? rows : a.batch, weight = a.sel_idx ? 1 : hkv;
        const int per = (n_entries + kAttThreads - 1) / kAttThreads, e0 = min(tid * per, n_entries), e1 = min(e0 + per, n_entries);
        auto entry_tokens = [&](int e) { return a.sel_idx ? walk_of(a, e / hkv, e % hkv) : walk_of(a, e, 0); };
        long long mine = 0;
        int most = 0;
        for (int e = e0; e < e1; ++e) {
            const int n = tiles_of(entry_tokens(e));
            mine += (long long)weight * (n + kStart);
            most = max(most, n);
        }
        long long incl = mine;
#pragma unroll
        for (int d = 1; d < LEOAM_WAVE; d <<= 1) {
            const long long o = __shfl_up(incl, d, LEOAM_WAVE);
            if (lane >= d) incl += o;
        }
        most = (int)wave_max_u32((uint32_t)most);
        if (lane == LEOAM_WAVE - 1) {
            sh_sum[wave] = incl;
            sh_most[wave] = most;
        }
        __syncthreads();
        long long total = 0, before = incl - mine;
#pragma unroll
        for (int w = 0; w < kAttWaves; ++w) {
            if (w < wave) before += sh_sum[w];
            total += sh_sum[w];
            most = max(most, sh_most[w]);
        }
        whole_rows = uniform(most) <= uncut_row_tiles(rows, k32);
        if (!whole_rows) {
            share = (total + a.sharers - 1) / a.sharers;
            pos = share * blockIdx.x;
            end = min(total, pos + share);
            if ((int)blockIdx.x >= a.sharers || pos >= end) return;
            if (pos >= before && pos < before + mine) {
                int e = e0;
                for (;;) {
                    const int tokens = entry_tokens(e);
                    const long long n = (long long)weight * (tiles_of(tokens) + kStart);
                    sh_tokens = tokens;
                    if (pos < before + n) break;
                    before += n;
                    ++e;
                }
                sh_entry = e;
                sh_at = pos - before;
            }
            __syncthreads();
            const int e = uniform(sh_entry);
            const long long at = sh_at;
            next_tokens = sh_tokens;
            if (a.sel_idx) {
                b = e / hkv;
                h = e % hkv;
                off = uniform((int)at);
            } else {
                const int n = tiles_of(uniform(next_tokens)) + kStart;
                b = e;
                h = uniform((int)(at / n));
                off = uniform((int)(at - (long long)h * n));
            }
        }
    }
    if (whole_rows) {
        if ((int)blockIdx.x >= rows) return;
        b = blockIdx.x / hkv;
        h = blockIdx.x % hkv;
        next_tokens = walk_of(a, b, h);
        end = tiles_of(next_tokens);
    }

    const int start = whole_rows ? 0 : kStart;
    bool first_piece = true;
    auto advance = [&](int taken) {
        pos += taken;
        off = 0;
        if (++h == hkv) {
            h = 0;
            ++b;
        }
    };
    while (pos < end) {
        const int tokens = uniform(next_tokens), n_tiles = tiles_of(tokens);
        const int take = uniform((int)min((long long)(start + n_tiles - off), end - pos));
        const int tile0 = max(off - start, 0), n_here = off + take - start - tile0;
        const size_t bh = (size_t)b * hkv + h;
        {
            const int nh = h + 1 < hkv ? h + 1 : 0, nb = h + 1 < hkv ? b : b + 1;
            if (pos + take < end) next_tokens = walk_of(a, nb, nh);      // (the share has a further row)
        }
        if (n_here <= 0) {      // (the share ends before the row's first tile)
            advance(take);
            continue;
        }
        const int len = a.sel_idx ? min(max(a.seq_len[b], 0), a.max_pages << a.page_shift) : tokens;
        const int32_t* sel = a.sel_idx ? a.sel_idx + bh * (size_t)a.k_max : nullptr;

        // ---- queries: the second operand of the first product, column = head ------------------------------
        uint4 qb[k32 ? 8 : 4];
#pragma unroll
        for (int s = 0; s < (k32 ? 8 : 4); ++s) {
            qb[s] = make_uint4(0, 0, 0, 0);
            // 16-byte pieces in the order in which a key row's loads hold the channels
            const int byte = k32 ? 64 * s + 16 * grp : k8 ? 128 * (s >> 1) + 32 * grp + 16 * (s & 1) : 64 * s + 16 * grp;
            if (l16 < G) qb[s] = load16(a.q, (bh * G + l16) * QROWB + byte);
        }

        // ---- this wave's part of the stretch, in steps ------------------------------------------------------
        const int t_begin = tile0 * kTileTokens, t_end = min(tokens, (tile0 + n_here) * kTileTokens);
        const int n_steps = (t_end - t_begin + STEP - 1) / STEP, per_wave = (n_steps + kAttWaves - 1) / kAttWaves;
        const int s0 = min(n_steps, wave * per_wave), s1 = min(n_steps, s0 + per_wave);

        // lane i holds entry held0 + i of the walk: its physical page (0 and no tokens if it has none)
        int held0 = -(1 << 30), held_page = 0, held_valid = 0;
        auto hold = [&](int e) {
            held0 = e;
            const int i = e + lane, most = sel ? tokens >> a.page_shift : (tokens + (1 << a.page_shift) - 1) >> a.page_shift;
            const int logical = i >= most ? -1 : sel ? sel[i] : i;
            int id = -1, valid = 0;
            if (logical >= 0 && logical < a.max_pages) {
                valid = min(max(len - (logical << a.page_shift), 0), 1 << a.page_shift);
                if (valid > 0) id = a.page_table[(size_t)b * a.max_pages + logical];
            }
            const bool ok = id >= 0 && id < a.n_pages;
            held_page = ok ? id : 0;
            held_valid = ok ? valid : 0;
        };
        auto tile_at = [&](int t) {      // the tile that begins at token t (a multiple of 16) of the walk
            TileAt at;
            const int e = t >> a.page_shift;
            if (e - held0 >= LEOAM_WAVE || e < held0) hold(e);
            const int i = e - held0;
            at.page = (uint32_t)__builtin_amdgcn_readlane(held_page, i);
            at.row0 = t & ((1 << a.page_shift) - 1);
            at.valid = min(max(__builtin_amdgcn_readlane(held_valid, i) - at.row0, 0), 16);
            at.ks = at.vs = 1.f;
            if (k8) {
                const size_t row = (size_t)at.page * hkv + h;
                at.ks = a.k_scale[row];
                at.vs = a.v_scale[row];
            }
            return at;
        };
        // Loads are unconditional; a token that does not count re-reads the tile's last one that does (what
        // stands behind the last token may be NaN, which a weight of zero would not silence).
        auto fetch = [&](int step, StepOf<T, S>& st, TileAt* at) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                at[j] = tile_at(t_begin + step * STEP + 16 * j);
                const size_t base = (((size_t)at[j].page * hkv + h) << a.page_shift) * ROWB;
                const char *kp = a.k_pages + base, *vp = a.v_pages + base;
                const int last = max(at[j].valid - 1, 0);
                const uint32_t krow = (uint32_t)(at[j].row0 + min(l16, last)) * ROWB;
#pragma unroll
                for (int s = 0; s < (k32 ? 8 : k8 ? 2 : 4); ++s)
                    st.k[(k32 ? 8 : k8 ? 2 : 4) * j + s] = load16(kp, krow + 64 * s + 16 * grp);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t vrow = (uint32_t)(at[j].row0 + min(4 * grp + r, last)) * ROWB;
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

        // lane (grp, head): running maximum (log2 domain) and this lane's part of the sum, accumulators of 32 channels
        float m_run = -INFINITY, l_run = 0.f;
        f32x4_t acc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

        auto consume = [&](StepOf<T, S>& st, TileAt* at) {
            float x[4 * NT], z[4 * NT];      // products, logits (log2 domain)
            bool partial = false;            // some tile has tokens that do not count
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                f32x4_t s = {0.f, 0.f, 0.f, 0.f};
                if constexpr (k32) {
                    f32x4_t chain[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) chain[e] = s;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float kx[4], qx[4];
                        unpack<F32>(st.k[i], kx);
                        unpack<F32>(qb[i], qx);
#pragma unroll
                        for (int e = 0; e < 4; ++e) chain[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[e], qx[e], chain[e], 0, 0, 0);
                    }
                    s = (chain[0] + chain[1]) + (chain[2] + chain[3]);
                } else if constexpr (k8) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const uint4 w = st.k[2 * j + c];
                        s = mfma_16x16x32<T>(widen8<T>(w.x, w.y, at[j].ks), qb[2 * c], s);
                        s = mfma_16x16x32<T>(widen8<T>(w.z, w.w, at[j].ks), qb[2 * c + 1], s);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) s = mfma_16x16x32<T>(st.k[4 * j + i], qb[i], s);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[4 * j + r] = s[r];
                    z[4 * j + r] = s[r] * a.scale_log2;
                }
                partial |= at[j].valid < 16;
                if (at[j].valid < 16) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (4 * grp + r >= at[j].valid) z[4 * j + r] = -INFINITY;
                    if (at[j].valid == 0) {      // nothing was read that counts: values must not matter either
                        at[j].vs = 1.f;
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            if constexpr (k32) st.v[2 * r] = st.v[2 * r + 1] = make_uint4(0, 0, 0, 0);
                            else if constexpr (k8) st.v[4 * j + r] = make_uint2(0, 0);
                            else st.v[4 * j + r] = make_uint4(0, 0, 0, 0);
                        }
                    }
                }
            }
            float mt = z[0];
#pragma unroll
            for (int i = 1; i < 4 * NT; ++i) mt = fmaxf(mt, z[i]);
            mt = rows_max4(mt) - kBias;
            if (__ballot(mt > m_run)) {
                const float m = fmaxf(m_run, mt), c = exp2_or_zero(m_run, m);
                m_run = m;
                l_run *= c;
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][r] *= c;
            }
            const float ref = m_run == -INFINITY ? 0.f : m_run;
            float p[4 * NT];
#pragma unroll
            for (int i = 0; i < 4 * NT; ++i) {
                p[i] = exp2_raw(fmaf(x[i], a.scale_log2, -ref));
                if (partial && z[i] == -INFINITY) p[i] = 0.f;
                l_run += p[i];
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
                            acc[4 * c + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vx[e], p[r], acc[4 * c + e], 0, 0, 0);
                    }
            } else {
                uint4 parts[kParts];
#pragma unroll
                for (int n = 0; n < kParts; ++n) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float u, v;
                        w[i] = pair_of(T{}, p[2 * i], p[2 * i + 1]);
                        pair_back(T{}, w[i], u, v);
                        p[2 * i] -= u;      // (exact: what is left has fewer bits)
                        p[2 * i + 1] -= v;
                    }
                    parts[n] = make_uint4(w[0], w[1], w[2], w[3]);
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
                    for (int n = 0; n < kParts; ++n) acc[e] = mfma_16x16x32<T>(col, parts[n], acc[e]);
                }
            }
        };

        if (s0 < s1) {
            StepOf<T, S> st[2];
            TileAt at[2][NT];
            fetch(s0, st[0], at[0]);
            for (int s = s0; s < s1; s += 2) {
                fetch(min(s + 1, s1 - 1), st[1], at[1]);
                consume(st[0], at[0]);
                if (s + 1 >= s1) break;
                fetch(min(s + 2, s1 - 1), st[0], at[0]);
                consume(st[1], at[1]);
            }
        }

        // ---- the four waves' states into one ---------------------------------------------------------------
        l_run += shfl_xor_f(l_run, 16);
        l_run += shfl_xor_f(l_run, 32);
        __syncthreads();      // (the previous stretch's states have been read)
        if (l16 < G) {
            float* x = xw[wave][l16];
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    // row 4 grp + r of accumulator i: its channel
                    const int d = k32 ? 64 * (i / 4) + 4 * (4 * grp + r) + (i & 3) : 8 * (4 * grp + r) + i;
                    x[d] = acc[i][r];
                }
            if (grp == 0) {
                x[LEOAM_D] = m_run;
                x[LEOAM_D + 1] = l_run;
            }
        }
        __syncthreads();
        const bool whole = n_here == n_tiles;
        // a piece that opens the workgroup's share, or closes it
        const size_t slot = 2 * (size_t)blockIdx.x + (first_piece ? 0 : 1);
        for (int i = tid; i < G * kPartStride; i += kAttThreads) {
            const int g = i / kPartStride, d = i % kPartStride;
            float m = -INFINITY;
#pragma unroll
            for (int w = 0; w < kAttWaves; ++w) m = fmaxf(m, xw[w][g][LEOAM_D]);
            float v = 0.f, l = 0.f;
#pragma unroll
            for (int w = 0; w < kAttWaves; ++w) {
                const float c = exp2_or_zero(xw[w][g][LEOAM_D], m);
                l += c * xw[w][g][LEOAM_D + 1];
                if (d < LEOAM_D) v += c * xw[w][g][d];
            }
            if (whole) {
                const size_t j = bh * G + g;
                if (d < LEOAM_D) a.out[j * LEOAM_D + d] = l == 0.f ? 0.f : v / l;      // (NaN stays)
                else if (d == LEOAM_D && a.lse) a.lse[j] = log_sum_exp(m, l, decode_bias<T>());
            } else {
                a.partial[(slot * G + g) * kPartStride + d] = d < LEOAM_D ? v : d == LEOAM_D ? m : l;
            }
        }
        if (a.pieces && tile0 == 0 && tid == 0) {
            RowPieces rp = {0, 0};
            if (!whole) {
                rp.count = (int)((pos - off + start + n_tiles - 1) / share - blockIdx.x) + 1;
                rp.first_slot = (int)slot;
            }
            a.pieces[bh] = rp;
        }
        if (whole_rows) break;
        first_piece = false;
        advance(take);
    }
}

// A row's pieces: the first at first_slot, each further one opens the next workgroup's share.  128 threads take eight pieces
// of a head at a time, all on their way together; PARTS groups of threads share a head's pieces, folded in order.  Four where
// rows are few and pieces many (32 heads of 32 pieces: 4.0 us against 5.9 with two), one where it is the other way round
// (2560 heads of 2 or 3: 5.2 against 7.9).
constexpr int kMergeGroups = 4;
constexpr int kManyRows = 64;
template <int PARTS>
__global__ __launch_bounds__(kMergeGroups * LEOAM_D) void page_decode_merge_kernel(const float* __restrict__ partial,
                                                                                   const RowPieces* __restrict__ pieces, int group,
                                                                                   int n_heads, int bias, float* __restrict__ out,
                                                                                   float* __restrict__ lse) {
    constexpr int HEADS = kMergeGroups / PARTS;
    constexpr int kBatch = 8;
    __shared__ float sm[PARTS], sl[PARTS], so[PARTS][LEOAM_D];
    const int d = threadIdx.x % LEOAM_D, tg = threadIdx.x / LEOAM_D, part = PARTS == 1 ? 0 : tg;
    const int j = blockIdx.x * HEADS + (PARTS == 1 ? tg : 0);
    if (j >= n_heads) return;
    const RowPieces rp = pieces[j / group];
    if (rp.count == 0) return;
    const int g = j % group;
    const size_t wg0 = rp.first_slot / 2;
    float m = -INFINITY, l = 0.f, o = 0.f;
    for (int i0 = part * kBatch; i0 < rp.count; i0 += PARTS * kBatch) {
        float ms[kBatch], ls[kBatch], os[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int i = min(i0 + u, rp.count - 1);
            const size_t slot = i == 0 ? (size_t)rp.first_slot : 2 * (wg0 + i);
            const float* p = partial + (slot * group + g) * kPartStride;
            ms[u] = p[LEOAM_D];
            ls[u] = p[LEOAM_D + 1];
            os[u] = p[d];
        }
        float mb = m;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i0 + u >= rp.count) ms[u] = -INFINITY;
            mb = fmaxf(mb, ms[u]);
        }
        const float c = exp2_or_zero(m, mb);
        m = mb;
        l *= c;
        o *= c;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i0 + u >= rp.count) continue;
            const float w = exp2_or_zero(ms[u], m);
            l += w * ls[u];
            o += w * os[u];
        }
    }
    if constexpr (PARTS > 1) {      // (one head to a workgroup: all its threads are here)
        if (d == 0) {
            sm[part] = m;
            sl[part] = l;
        }
        so[part][d] = o;
        __syncthreads();
        if (part) return;
        m = sm[0];
        l = o = 0.f;
#pragma unroll
        for (int p = 1; p < PARTS; ++p) m = fmaxf(m, sm[p]);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const float w = exp2_or_zero(sm[p], m);
            l += w * sl[p];
            o += w * so[p][d];
        }
    }
    out[(size_t)j * LEOAM_D + d] = l == 0.f ? 0.f : o / l;      // (NaN stays)
    if (lse && d == 0) lse[j] = log_sum_exp(m, l, bias);
}

// Workgroups of the attention kernel: two fill a compute unit's registers (three, with fewer registers each, measured 101 against
// 84 us for 40 sequences of up to 9000 tokens in 8 bits; one 111; twice as many shares 84.5 and more pieces).
constexpr int kDecodeGroups = 512;

static size_t piece_bytes(const leoam_pages* s) { return 2 * (size_t)(s->n_q_heads / s->n_kv_heads) * kPartStride * sizeof(float); }
static size_t directory_bytes(const leoam_pages* s) {
    return ((size_t)s->batch * s->n_kv_heads * sizeof(RowPieces) + 255) / 256 * 256;
}
size_t page_decode_workspace_bytes(const leoam_pages* s) { return (directory_bytes(s) + kDecodeGroups * piece_bytes(s) + 15) / 16 * 16; }
size_t page_decode_min_workspace_bytes(const leoam_pages* s) { return (directory_bytes(s) + piece_bytes(s) + 15) / 16 * 16; }

template <typename T, typename S> static hipError_t launch_decode(const PageDecodeArgs& a, int group, int n_groups, hipStream_t stream) {
    const dim3 grid(n_groups), block(kAttThreads);
    switch (group) {
    case 1: hipLaunchKernelGGL((page_decode_kernel<T, S, 1>), grid, block, 0, stream, a); break;
    case 2: hipLaunchKernelGGL((page_decode_kernel<T, S, 2>), grid, block, 0, stream, a); break;
    case 4: hipLaunchKernelGGL((page_decode_kernel<T, S, 4>), grid, block, 0, stream, a); break;
    default: hipLaunchKernelGGL((page_decode_kernel<T, S, 8>), grid, block, 0, stream, a); break;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.pieces) return e;
    const int n_heads = a.batch * a.n_kv_heads * group;
    if (a.batch * a.n_kv_heads >= kManyRows)
        hipLaunchKernelGGL(page_decode_merge_kernel<1>, dim3((n_heads + kMergeGroups - 1) / kMergeGroups), dim3(kMergeGroups * LEOAM_D), 0,
                           stream, a.partial, a.pieces, group, n_heads, decode_bias<T>(), a.out, a.lse);
    else
        hipLaunchKernelGGL(page_decode_merge_kernel<kMergeGroups>, dim3(n_heads), dim3(kMergeGroups * LEOAM_D), 0, stream, a.partial,
                           a.pieces, group, n_heads, decode_bias<T>(), a.out, a.lse);
    return hipGetLastError();
}

hipError_t page_decode_dispatch(const leoam_pages* s, const void* q, const void* k_pages, const void* v_pages,
                                const float* k_scale, const float* v_scale, const int32_t* page_table, const int32_t* seq_len,
                                const int32_t* sel_idx, const int32_t* sel_count, int k_max, float softmax_scale, float* out,
                                float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    PageDecodeArgs a;
    a.q = (const char*)q; a.k_pages = (const char*)k_pages; a.v_pages = (const char*)v_pages;
    a.k_scale = k_scale; a.v_scale = v_scale; a.page_table = page_table; a.seq_len = seq_len;
    a.sel_idx = sel_idx; a.sel_count = sel_count; a.k_max = k_max;
    a.scale_log2 = softmax_scale * kLog2e;
    a.out = out; a.lse = lse;
    a.pieces = (RowPieces*)workspace;
    a.partial = (float*)((char*)workspace + directory_bytes(s));
    a.batch = s->batch; a.n_kv_heads = s->n_kv_heads; a.n_pages = s->n_pages;
    a.page_shift = __builtin_ctz((unsigned)s->page_size); a.max_pages = s->max_pages;
    const int group = s->n_q_heads / s->n_kv_heads;
    const int rows = s->batch * s->n_kv_heads;
    const size_t fit = (workspace_bytes - directory_bytes(s)) / piece_bytes(s);
    a.sharers = (int)(fit < (size_t)kDecodeGroups ? fit : (size_t)kDecodeGroups);
    int n_groups = rows > a.sharers ? rows : a.sharers;      // the kernel may take a row to a workgroup, or leave the rest idle
    // Where even a full table's row is not long, neither the search for shares nor the second kernel are needed.
    const long long most = (long long)(sel_idx ? k_max : s->max_pages) * s->page_size;
    if (most <= (long long)uncut_row_tiles(rows, s->q_dtype == LEOAM_F32) * kTileTokens) {
        a.pieces = nullptr;
        n_groups = rows;
    }
    const bool k8 = s->kv_dtype == LEOAM_E4M3;
    switch (s->q_dtype) {
    case LEOAM_F32: return launch_decode<F32, F32>(a, group, n_groups, stream);
    case LEOAM_F16: return k8 ? launch_decode<F16, E4M3>(a, group, n_groups, stream) : launch_decode<F16, F16>(a, group, n_groups, stream);
    default: return k8 ? launch_decode<BF16, E4M3>(a, group, n_groups, stream) : launch_decode<BF16, BF16>(a, group, n_groups, stream);
    }
}

}  // namespace leoam
