// page_attention_prefill: causal softmax(scale q K^T) V of a call's new tokens over their sequences' pages.
//
// Bound by the matrix cores.  A workgroup takes 128 query rows of one kv head - a row is a (token, head of the
// group) pair, so the heads of a group share every key and value that is fetched - and walks the keys 64 at a time (fp32:
// 32): the next tile (8 bits: the next two) is on its way to registers while the current one is worked on in LDS.
// Each of the four waves owns 32 rows.  S^T = K Q^T (32x32 products) leaves lane = row, registers = keys: the row's
// maximum and sum need no exchange but one with the lane 32 away, and P is already the second operand of O^T = V^T P^T;
// the first operand, four keys of one channel at a time, comes out of LDS by the transposing read.  For that P is rounded to the
// model's type, as the stored values are; the row's sum takes it before.  P in two parts, as decoding has it where the matrix cores
// are idle, doubles the second product: 8192 tokens in bf16 589 -> 772 us, 8-bit prompts behind histories 361 -> 477, for an output of
// bf16 that is off by 4.9e-4 (its own rounding) instead of 6.6e-4, root mean square; fp16 6.5e-5 instead of 8.5e-5.
//
// A unit of work is (128 rows, kv head).  With enough units to fill the chip each takes a workgroup.  With few (a
// handful of rows behind a long context) the key tiles of all units are laid end to end, each unit's beginning counted as
// some more (kUnitStart), and shared out equally; a unit cut by the ends of shares leaves its pieces, (acc, m, l) per row, in
// the workspace, and a second kernel folds them.
#include <cfloat>

#include "page_common.h"

namespace leoam {

constexpr int kRows = 128;            // query rows of a workgroup, 32 a wave

// fp16 weights: the reference is taken 2^7 lower, so that small weights stay clear of fp16's subnormals
template <typename T> constexpr int prefill_bias() { return T::kTag == LEOAM_F16 ? 7 : 0; }

struct PagePrefillArgs {
    const char *q, *k_pages, *v_pages;
    const float *k_scale, *v_scale;
    const int32_t *page_table, *seq_len, *new_off;
    int n_new, n_slots;
    float scale_log2;      // of |softmax_scale|
    uint32_t flip;         // sign bits of the queries, turned if softmax_scale is negative
    char* out;
    float* lse;
    struct UnitPieces* pieces;      // shared out: directory of the units, then the pieces
    float* partial;
    int batch, n_kv_heads, n_pages, page_shift, max_pages;
};

// pieces of a unit (0: its result is final), where the first lies, its first row of the call, its rows
struct UnitPieces { int32_t count, first_slot, token0, rows; };

constexpr int kSharers = 512;         // workgroups that share the tiles: two fill a compute unit
constexpr int kMostUnits = 1024;      // more units than this are not shared out: two rounds of workgroups or more
constexpr int kMostSlots = 256;       // of as many slots: their tables stay in LDS
// If no unit has more tiles than this, none is cut: a cut costs a second start, a piece and a fold.  (32 rows behind a context in
// bf16, us, shares against whole units: 8 units of 11 tiles 15 : 22; 64 of 11 20 : 22, of 24 24 : 42; 256 of 11 32 : 27, of 24 42 : 47,
// of 46 65 : 92; 512 of 11 50 : 34, of 24 70 : 63, of 46 114 : 111, of 94 183 : 217.  A tile of fp32 takes four times as long.)
__host__ __device__ __forceinline__ int uncut_unit_tiles(int units, bool k32) {
    return k32 ? min(max(units / 40, 1), 16) : min(max(units / (units < kSharers ? 20 : 10), 6), 64);
}
// What a unit's beginning costs a workgroup, in tiles (fp32: 1): shares are measured in tiles and beginnings.  (us with 0, 1, 2, 4: 81
// rows of ten sequences behind 89 to 22116 tokens, 16 heads, 8 bits 148, 109, 96, 97; 32 sequences to 6000 in bf16 110, 102, 95, 94.)
constexpr int kUnitStart = 2;
// `total` of them among the workgroups, in order: the first `more` take each + 1, the others each.  (The first ones land on compute
// units of their own, so the units' loads differ by a tile at most; fp32, 1656 tiles of 8 us for 504: 55 -> 51 us against
// shares of equal size and a last one of what is left.)
struct Shares {
    int each, more;
    __device__ __forceinline__ Shares(int total, int workgroups) : each(total / workgroups), more(total % workgroups) {}
    __device__ __forceinline__ int begin(int w) const { return w * each + min(w, more); }
    __device__ __forceinline__ int owner(int tile) const {      // of one of the tiles
        const int t = more * (each + 1);
        return tile < t ? tile / (each + 1) : more + (tile - t) / each;
    }
};
// a piece: [32 groups of 4 channels][128 rows][4], maxima, sums
constexpr int kPieceFloats = kRows * (LEOAM_D + 2);

// the rows of a slot: sequence, its first row in the call, its number of rows, which tile of them, the sequence's length
struct Unit { int b, row0, m, local, len; };
__device__ __forceinline__ int first_slot_of(int row0, int i, int group) { return (int)((long long)row0 * group / kRows) + i; }

// the values of a register that are not finite become zero; whether there were any
template <typename T> __device__ __forceinline__ bool silence(uint32_t& w) {
    if constexpr (T::kTag == LEOAM_F32) {
        const bool bad = (w & 0x7f800000u) == 0x7f800000u;
        if (bad) w = 0;
        return bad;
    } else {
        constexpr uint32_t m = T::kTag == LEOAM_F16 ? 0x7c00u : 0x7f80u;
        const bool lo = (w & m) == m, hi = (w & (m << 16)) == (m << 16);
        if (lo) w &= 0xffff0000u;
        if (hi) w &= 0x0000ffffu;
        return lo || hi;
    }
}
template <typename T> __device__ __forceinline__ bool silence(uint4& w) {
    const bool a = silence<T>(w.x), b = silence<T>(w.y), c = silence<T>(w.z), d = silence<T>(w.w);
    return a || b || c || d;
}

// the same for 8-bit codes: 0x7f and 0xff are not finite
__device__ __forceinline__ bool silence_codes(uint32_t& w) {
    // (a byte of `full` is 0x80 where the code's lower seven bits are all ones)
    const uint32_t full = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    w &= ~((full >> 7) * 0xffu);
    return full != 0;
}
__device__ __forceinline__ bool silence_codes(uint4& w) {
    const bool a = silence_codes(w.x), b = silence_codes(w.y), c = silence_codes(w.z), d = silence_codes(w.w);
    return a || b || c || d;
}

template <typename T, typename S, int G, bool kShared>
__global__ __launch_bounds__(kAttThreads) __attribute__((amdgpu_waves_per_eu(2))) void page_prefill_kernel(PagePrefillArgs a) {
    constexpr bool k8 = std::is_same<S, E4M3>::value, k32 = T::kTag == LEOAM_F32;
    constexpr int ROWB = LEOAM_D * T::kBytes, SROWB = LEOAM_D * S::kBytes;      // a row in LDS, in the pages
    constexpr int KEYS = k32 ? 32 : 64, KB = KEYS / 32, KSTR = kKeyStride<T>, VSTR = kValueStride<T>, NQ = k32 ? 16 : 8;
    constexpr int LOADS = KEYS * SROWB / (kAttThreads * 16), PIECES = SROWB / 16, ROWS_PER_LOAD = kAttThreads / PIECES;
    constexpr int kStart = k32 ? 1 : kUnitStart;
    // (few rows are usual where tiles are shared.  8 bits, ten sequences of 22K, 64 heads, us without : with, 2 tokens each 225 : 181, 8 226 : 190,
    // 16 251 : 223; 16 bits wait for memory with 8 already, 319 : 319)
    constexpr bool kHalves = kShared && k8;
    constexpr int AHEAD = k8 ? 2 : 1;      // tiles on their way to registers (8 bits, one: 363 us against 357 behind histories of 4K)
    constexpr int GROUPS = KEYS / 16;      // 16 keys never straddle a page
    constexpr float kLag = 8.f, kBias = prefill_bias<T>();      // the reference may lag the maximum by 2^kLag
    __shared__ __align__(16) char sh_k[2][KEYS * KSTR];
    __shared__ __align__(16) char sh_v[2][KEYS * VSTR];
    __shared__ int sh_bad;

    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE);
    const int half = lane >> 5, l32 = lane & 31;
    const int hkv = a.n_kv_heads;

    // tiles [j0, j1) of a unit; j1 < 0: all.  slot: where to leave a piece, < 0: the result is final
    auto run = [&](const Unit& unit, int h, int j0, int j1, int piece_slot) {
    const int b = unit.b, row0 = unit.row0, m = unit.m, local = unit.local;
    const int first = unit.len - m;                                   // position of the sequence's first new token (may be negative)
    const int tok0 = local * (kRows / G), n_tok = min(m - tok0, kRows / G);
    const int keys = max(first + tok0 + n_tok, 0);               // keys that some row of the workgroup sees
    // Half the rows or fewer: waves 2 and 3 take the same rows as 0 and 1 and the second half of every tile's keys.
    const bool halves = kHalves && n_tok * G <= kRows / 2;
    const int rows_of = halves ? wave & 1 : wave;
    // this lane's row
    const int row = 32 * rows_of + l32, tok = min(tok0 + row / G, m - 1);
    const int my_pos = first + tok;
    const bool stored = row / G < n_tok;
    const bool idle = (32 * rows_of) / G >= n_tok;                   // none of the wave's rows is one
    const size_t q_row = ((size_t)(row0 + tok) * hkv + h) * G + row % G;
    const int wave_lo = first + tok0 + 32 * rows_of / G;             // the wave's rows see at least / at most
    const int wave_hi = min(first + tok0 + (32 * rows_of + 31) / G, first + m - 1);

    const int n_tiles = (keys + KEYS - 1) / KEYS, last = keys - 1;
    const int first_masked = max(first + tok0 + 1, 0) / KEYS;     // tiles from here on hide keys from some row
    const int32_t* table = a.page_table + (size_t)b * a.max_pages;
    // Rows of head h of page p begin p * page_bytes behind kh and vh.  Lane l looks after 16-key group l % GROUPS of a tile.
    const uint32_t head_bytes = (uint32_t)SROWB << a.page_shift, page_bytes = head_bytes * (uint32_t)hkv, in_page = (1u << a.page_shift) - 1;
    const char *kh = a.k_pages + (size_t)h * head_bytes, *vh = a.v_pages + (size_t)h * head_bytes;
    auto pages_of = [&](int j) { return table[min(j * KEYS + 16 * (lane % GROUPS), last) >> a.page_shift]; };
    const int id0 = n_tiles > 0 ? pages_of(min(j0, n_tiles - 1)) : 0;
    uint4 qb[NQ];
#pragma unroll
    for (int s = 0; s < NQ; ++s) qb[s] = load16(a.q, q_row * ROWB + 32 * s + 16 * half);
    if (a.flip) {
#pragma unroll
        for (int s = 0; s < NQ; ++s) {
            qb[s].x ^= a.flip; qb[s].y ^= a.flip; qb[s].z ^= a.flip; qb[s].w ^= a.flip;
        }
    }
    if (tid == 0) sh_bad = 0;
    __syncthreads();

    struct Tile {
        uint4 k[LOADS], v[LOADS];
        float ks[LOADS], vs[LOADS];
        uint32_t ok;      // bit g: group g has a page
    };
    constexpr uint32_t kAllOk = (1u << GROUPS) - 1;
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
            const uint32_t at = ((uint32_t)min(j * KEYS + r, last) & in_page) * SROWB + 16 * (tid % PIECES);
            const uint64_t base = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, g) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, g);
            t.k[i] = load16(kh + base, at);
            t.v[i] = load16(vh + base, at);
            if (k8) {
                const size_t row = (size_t)(uint32_t)__builtin_amdgcn_readlane((int)page, g) * hkv + h;
                t.ks[i] = a.k_scale[row];
                t.vs[i] = a.v_scale[row];
            }
        }
    };
    auto stage = [&](int j, int buf, Tile& t) {
        // A value that is not finite must not reach rows that its key is hidden from, which a weight of zero does not
        // prevent: from the first tile that hides keys on such values are left out here and added at the end.
        const bool look = j >= first_masked;
        bool bad = false;
        if (t.ok != kAllOk) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                if (t.ok >> ((i * ROWS_PER_LOAD + tid / PIECES) / 16) & 1) continue;
                t.v[i] = make_uint4(0, 0, 0, 0);      // nothing there: no value may matter
                t.vs[i] = 1.f;
            }
        }
        if (look) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                if constexpr (k8) bad |= silence_codes(t.v[i]);
                else bad |= silence<T>(t.v[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = i * ROWS_PER_LOAD + tid / PIECES, piece = tid % PIECES;
            if constexpr (k8) {
                const uint4 v0 = widen8<T>(t.v[i].x, t.v[i].y, t.vs[i]), v1 = widen8<T>(t.v[i].z, t.v[i].w, t.vs[i]);
                store16(sh_k[buf], r * KSTR + 32 * piece, widen8<T>(t.k[i].x, t.k[i].y, t.ks[i]));
                store16(sh_k[buf], r * KSTR + 32 * piece + 16, widen8<T>(t.k[i].z, t.k[i].w, t.ks[i]));
                store16(sh_v[buf], r * VSTR + 32 * piece, v0);
                store16(sh_v[buf], r * VSTR + 32 * piece + 16, v1);
            } else {
                store16(sh_k[buf], r * KSTR + 16 * piece, t.k[i]);
                store16(sh_v[buf], r * VSTR + 16 * piece, t.v[i]);
            }
        }
        if (bad) sh_bad = 1;
    };

    f32x16_t acc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
    float ref = -INFINITY, l_run = 0.f;

    // key of register r of key block kb in this lane
    auto key_of = [&](int kb, int r) { return 32 * kb + 8 * (r / 4) + 4 * half + r % 4; };

    const uint32_t k_lane = l32 * KSTR + 16 * half;
    const uint32_t v_lane = k32 ? 4 * half * VSTR + 4 * l32
                                : (4 * half + (lane & 15) / 4) * VSTR + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
    auto work = [&](auto half_tile, int j, int buf, uint32_t ok) {
        constexpr int NB = decltype(half_tile)::value ? KB / 2 : KB;      // key blocks, from block b0 on
        const int b0 = decltype(half_tile)::value ? (wave >> 1) * NB : 0;
        const char *kt = sh_k[buf] + k_lane + b0 * 32 * KSTR, *vt = sh_v[buf] + v_lane + b0 * 32 * VSTR;
        f32x16_t s[NB];
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
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
        if constexpr (!k32) {      // six reads ahead of the products
            then<kLdsRead, 6>();
            static_for<0, 8 * NB - 6>([](auto) {
                then<kMfma, 1>();
                then<kLdsRead, 1>();
            });
            then<kMfma, 6>();
        }
        const bool masked = j * KEYS + KEYS - 1 > wave_lo || ok != kAllOk;
        if (masked) {
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (j * KEYS + 32 * b0 + key_of(kb, r) > my_pos || !(ok >> (2 * (b0 + kb) + r / 8) & 1)) s[kb][r] = -INFINITY;
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
        // The reference is the maximum of some earlier tile; it moves only when the maximum has left it behind by 2^kLag.
        if (__ballot(mt > ref + kLag)) {
            const float now = fmaxf(ref, mt), c = exp2_or_zero(ref, now);
            ref = now;
            l_run *= c;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][r] *= c;
        }
        const float base = ref == -INFINITY ? 0.f : ref;
        auto weigh = [&](int kb, int r) {
            s[kb][r] = exp2_raw(fmaf(s[kb][r], a.scale_log2, -base));
            l_run += s[kb][r];
        };
        if constexpr (k32) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                weigh(0, r);
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                    // key_of(0, r), channel 32 db + l32
                    const float v = *reinterpret_cast<const float*>(vt + (8 * (r / 4) + r % 4) * VSTR + 128 * db);
                    acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[0][r], acc[db], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int t = 0; t < 2 * NB; ++t) {      // 16 keys
                const int kb = t / 2, r0 = 8 * (t % 2);
#pragma unroll
                for (int r = r0; r < r0 + 8; ++r) weigh(kb, r);
                const uint4 p = make_uint4(pair_of(T{}, s[kb][r0], s[kb][r0 + 1]), pair_of(T{}, s[kb][r0 + 2], s[kb][r0 + 3]),
                                           pair_of(T{}, s[kb][r0 + 4], s[kb][r0 + 5]), pair_of(T{}, s[kb][r0 + 6], s[kb][r0 + 7]));
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                    // the lane's address is that of 4 channels of one key; what it gets is one channel of 4 keys
                    const uint2 w0 = transposed(vt + 16 * t * VSTR + 64 * db), w1 = transposed(vt + (16 * t + 8) * VSTR + 64 * db);
                    acc[db] = mfma_32x32x16<T>(make_uint4(w0.x, w0.y, w1.x, w1.y), p, acc[db]);
                }
            }
            // the products of 16 keys run while the weights of the next 16 are computed and their values read
            then<kLdsRead, 8>();
            static_for<0, 8>([](auto) {
                then<kValu, 3>();
                then<kTrans, 1>();
            });
            static_for<0, 8 * NB - 4>([](auto) {
                then<kMfma, 1>();
                then<kLdsRead, 2>();
                then<kValu, 5>();
                then<kTrans, 2>();
            });
            then<kMfma, 4>();
        }
    };

    const int j_end = j1 < 0 ? n_tiles : min(j1, n_tiles);
    if (j0 < j_end) {
        Tile even, odd;      // (of the tiles from j0 on)
        int id = id0;
        fetch(j0, id, even);
        if constexpr (AHEAD == 2) fetch(min(j0 + 1, j_end - 1), id, odd);
        stage(j0, j0 & 1, even);
        uint32_t ok = even.ok;
        __syncthreads();
        // Tile j is worked on, then `in` is staged; `to` takes in tile j + AHEAD.  (Two tiles on their way: no branch around the
        // loads and none that leads back, or the compiler has everybody wait for the second tile too.)
        auto walk = [&](auto half_tile) {
            int j = j0;
            auto step = [&](Tile& in, Tile& to) {
                if (AHEAD == 2 || j + 1 < j_end) fetch(min(j + AHEAD, j_end - 1), id, to);
                if (!idle && j * KEYS <= wave_hi) work(half_tile, j, j & 1, ok);
                if (++j == j_end) return false;
                stage(j, j & 1, in);
                ok = in.ok;
                __syncthreads();
                return true;
            };
            if constexpr (AHEAD == 1) {
                while (step(even, even)) {}
            } else {
                while (step(odd, even) && step(even, odd)) {}
            }
        };
        if (kHalves && halves) walk(std::integral_constant<bool, kHalves>{});
        else walk(std::false_type{});
    }

    if (kHalves && halves) {      // the rows' two states become one
        float* x = reinterpret_cast<float*>(sh_k) + (wave & 1) * 66 * LEOAM_WAVE + lane;
        __syncthreads();
        if (wave >= 2) {
#pragma unroll
            for (int i = 0; i < 64; ++i) x[i * LEOAM_WAVE] = acc[i / 16][i % 16];
            x[64 * LEOAM_WAVE] = ref;
            x[65 * LEOAM_WAVE] = l_run;
        }
        __syncthreads();
        if (wave >= 2) return;
        const float other = x[64 * LEOAM_WAVE], now = fmaxf(ref, other), c = exp2_or_zero(ref, now), d = exp2_or_zero(other, now);
        ref = now;
        l_run = c * l_run + d * x[65 * LEOAM_WAVE];
#pragma unroll
        for (int i = 0; i < 64; ++i) {
            acc[i / 16][i % 16] = c * acc[i / 16][i % 16] + d * x[i * LEOAM_WAVE];
            if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);      // (no more registers than that for what is read)
        }
    }
    if (sh_bad) {      // values that were left out reach the rows that see their keys
        for (int t = max(j0, first_masked) * KEYS; t < min(j_end * KEYS, keys); ++t) {
            const int id = uniform(table[t >> a.page_shift]);
            if ((uint32_t)id >= (uint32_t)a.n_pages || t > my_pos) continue;
            const char* v = vh + (uint64_t)(uint32_t)id * page_bytes + (size_t)(t & ((1 << a.page_shift) - 1)) * SROWB;
#pragma unroll
            for (int db = 0; db < 4; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int d = 32 * db + 8 * (r / 4) + 4 * half + r % 4;
                    uint32_t w;
                    if constexpr (k32) w = *reinterpret_cast<const uint32_t*>(v + 4 * d);
                    else if constexpr (k8) w = (*reinterpret_cast<const uint8_t*>(v + d) & 0x7fu) == 0x7fu ? 0x7fc00000u : 0u;
                    else {
                        w = *reinterpret_cast<const uint16_t*>(v + 2 * d);
                        // (the sign, the exponent's ones and whether there is a fraction, as a float has them)
                        constexpr uint32_t m = T::kTag == LEOAM_F16 ? 0x7c00u : 0x7f80u;
                        w = (w & m) != m ? 0u : (w & 0x8000u) << 16 | 0x7f800000u | (w & 0x7fffu & ~m ? 0x400000u : 0u);
                    }
                    if ((w & 0x7f800000u) == 0x7f800000u) acc[db][r] += bits_to_float(w);
                }
        }
    }

    // ---- the rows' results -------------------------------------------------------------------------------
    const float l = l_run + shfl_xor_f(l_run, 32), inv = l == 0.f ? 0.f : 1.f / l;      // (NaN stays)
    if (!stored) return;
    if (kShared && piece_slot >= 0) {
        float* piece = a.partial + (size_t)piece_slot * kPieceFloats;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int d4 = 8 * db + r / 2 + half;
                store16(piece, ((size_t)d4 * kRows + row) * 16, make_uint4(float_to_bits(acc[db][r]), float_to_bits(acc[db][r + 1]),
                                                                           float_to_bits(acc[db][r + 2]), float_to_bits(acc[db][r + 3])));
            }
        if (half == 0) {
            piece[kRows * LEOAM_D + row] = ref;
            piece[kRows * (LEOAM_D + 1) + row] = l;
        }
        return;
    }
    if (a.lse && half == 0) a.lse[q_row] = log_sum_exp(ref, l, prefill_bias<T>());
    char* out = a.out + q_row * ROWB;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = 32 * db + 2 * r + 4 * half;
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = acc[db][r + e] * inv;
            if constexpr (k32) store16(out, 4 * d, pack<F32>(x));
            else *reinterpret_cast<uint2*>(out + 2 * d) = make_uint2(pair_of(T{}, x[0], x[1]), pair_of(T{}, x[2], x[3]));
        }
    };      // run

    if constexpr (!kShared) {
        const int h = blockIdx.x % hkv;
        // (later rows see more keys: they are started first)
        const int slot = a.n_slots - 1 - (int)(blockIdx.x / hkv);
        Unit u = {slot, slot, 1, 0, 0};
        if (a.new_off) {
            u.b = uniform(wave_count_below(a.batch, slot, [&](int i) { return first_slot_of(a.new_off[i], i, G); }));
            if (u.b >= a.batch) return;
            u.row0 = uniform(a.new_off[u.b]);
            u.m = uniform(a.new_off[u.b + 1]) - u.row0;
            u.local = slot - first_slot_of(u.row0, u.b, G);
            if (u.row0 < 0 || u.m < 0 || u.m > a.n_new - u.row0) return;
        }
        if (u.local < 0 || (long long)u.local * kRows >= (long long)u.m * G) return;
        u.len = min(max(uniform(a.seq_len[u.b]), 0), a.max_pages << a.page_shift);
        run(u, h, 0, -1, -1);
    } else {
        // ---- this workgroup's share (at most kMostSlots slots, and no more sequences than slots) -------------
        __shared__ int sh_off[kMostSlots + 1], sh_len[kMostSlots], sh_tiles[kMostSlots], sh_before[kMostSlots + 1];
        __shared__ int sh_most;
        for (int i = tid; i <= a.batch; i += kAttThreads) {
            sh_off[i] = a.new_off ? a.new_off[i] : i;
            if (i < a.batch) sh_len[i] = min(max(a.seq_len[i], 0), a.max_pages << a.page_shift);
        }
        if (tid == 0) sh_most = 0;
        __syncthreads();
        auto unit_of = [&](int slot) {
            Unit u;
            if (!a.new_off) return Unit{slot, slot, 1, 0, sh_len[slot]};
            int lo = 0, hi = a.batch;      // the last sequence whose slots begin at or before this one
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (first_slot_of(sh_off[mid], mid, G) <= slot) lo = mid;
                else hi = mid;
            }
            u.b = lo;
            u.row0 = sh_off[lo];
            u.len = sh_len[lo];
            u.m = sh_off[lo + 1] - u.row0;
            u.local = slot - first_slot_of(u.row0, lo, G);
            if (u.row0 < 0 || u.m < 0 || u.m > a.n_new - u.row0 || u.local < 0 || (long long)u.local * kRows >= (long long)u.m * G) u.m = 0;
            return u;
        };
        for (int slot = tid; slot < a.n_slots; slot += kAttThreads) {
            const Unit u = unit_of(slot);
            int tiles = 0;
            if (u.m > 0) {
                const int first = u.len - u.m, tok0 = u.local * (kRows / G);
                tiles = max(1, (max(first + tok0 + min(u.m - tok0, kRows / G), 0) + KEYS - 1) / KEYS);
                atomicMax(&sh_most, tiles);
            } else if (blockIdx.x == 0) {
                for (int h = 0; h < hkv; ++h) a.pieces[slot * hkv + h] = UnitPieces{0, 0, 0, 0};
            }
            sh_tiles[slot] = tiles;
        }
        __syncthreads();
        if (wave == 0) {      // tiles before each slot (every slot has hkv units)
            int run_sum = 0;
            for (int s0 = 0; s0 < a.n_slots; s0 += LEOAM_WAVE) {
                const int slot = s0 + lane;
                const uint32_t mine = slot < a.n_slots && sh_tiles[slot] ? (uint32_t)(sh_tiles[slot] + kStart) * hkv : 0u, incl = wave_incl_scan_u32(mine);
                if (slot < a.n_slots) sh_before[slot] = run_sum + (int)(incl - mine);
                run_sum += __builtin_amdgcn_readlane((int)incl, LEOAM_WAVE - 1);
            }
            if (lane == 0) sh_before[a.n_slots] = run_sum;
        }
        __syncthreads();
        const int total = uniform(sh_before[a.n_slots]), W = gridDim.x;
        const bool uncut = uniform(sh_most) <= uncut_unit_tiles(a.n_slots * hkv, k32);      // then workgroup w takes units w, w + W, ...
        const Shares shares(total, W);
        int slot = 0, h = 0, off = 0, pos = 0, end = 0;
        int next = blockIdx.x;
        auto whole_unit = [&] {
            while (next < a.n_slots * hkv) {
                slot = next / hkv;
                h = next % hkv;
                next += W;
                pos = 0;
                end = uniform(sh_tiles[slot]) + kStart;
                if (end > kStart) return;
            }
            pos = end = 0;
        };
        if (uncut) {
            whole_unit();
        } else {
            pos = shares.begin(blockIdx.x);
            end = shares.begin(blockIdx.x + 1);
            if (pos >= end) return;
            int lo = 0, hi = a.n_slots;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (sh_before[mid] <= pos) lo = mid;
                else hi = mid;
            }
            slot = uniform(lo);      // (of equal ones the last: the one that has tiles)
            const int n = uniform(sh_tiles[slot]) + kStart, in = pos - uniform(sh_before[slot]);
            h = in / n;
            off = in - h * n;
        }
        bool first_piece = true;
        while (pos < end) {
            const int n = uniform(sh_tiles[slot]), take = min(kStart + n - off, end - pos);
            const int tile0 = max(off - kStart, 0), tile1 = off + take - kStart;
            if (tile0 < tile1) {      // (a share may end before the unit's first tile)
                Unit u = unit_of(slot);
                u = Unit{uniform(u.b), uniform(u.row0), uniform(u.m), uniform(u.local), uniform(u.len)};
                const int id = slot * hkv + h;
                const bool whole = tile1 - tile0 == n;
                const int piece_slot = 2 * (int)blockIdx.x + (first_piece ? 0 : 1);      // opens the share, or closes it
                first_piece = false;
                if (tile0 == 0 && tid == 0) {
                    UnitPieces up = {0, 0, 0, 0};
                    if (!whole) {
                        const int tok0 = u.local * (kRows / G);
                        up.count = shares.owner(pos - off + kStart + n - 1) - (int)blockIdx.x + 1;
                        up.first_slot = piece_slot;
                        up.token0 = u.row0 + tok0;
                        up.rows = min(u.m - tok0, kRows / G) * G;
                    }
                    a.pieces[id] = up;
                }
                run(u, h, tile0, tile1, whole ? -1 : piece_slot);
                __syncthreads();
            }
            if (uncut) {
                whole_unit();
                continue;
            }
            pos += take;
            off = 0;
            if (++h == hkv) {
                h = 0;
                do ++slot;
                while (slot < a.n_slots && sh_tiles[slot] == 0);
            }
        }
    }
}

// 8 channels of a unit's rows: its pieces, in order.  Where rows are few, two or four groups of threads share the pieces.
template <typename T>
__global__ __launch_bounds__(256) void page_prefill_merge_kernel(PagePrefillArgs a, int group) {
    __shared__ float sh[6][2 * kRows];      // states: m, l, 4 sums
    const UnitPieces up = a.pieces[blockIdx.x];
    if (up.count == 0) return;
    const int parts = up.rows <= kRows / 4 ? 4 : up.rows <= kRows / 2 ? 2 : 1, n_rows = kRows / parts;
    const int t = threadIdx.x % kRows, row = t % n_rows, part = t / n_rows, d4 = 2 * blockIdx.y + threadIdx.x / kRows;
    const int rc = min(row, up.rows - 1);
    constexpr int kBatch = 8;      // pieces that are on their way together
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = part * kBatch; i0 < up.count; i0 += parts * kBatch) {
        float ms[kBatch], ls[kBatch];
        uint4 x4[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int i = min(i0 + u, up.count - 1);
            // (each further piece opens the next workgroup's share)
            const float* piece = a.partial + (size_t)(i == 0 ? up.first_slot : 2 * (up.first_slot / 2 + i)) * kPieceFloats;
            ms[u] = piece[kRows * LEOAM_D + rc];
            ls[u] = piece[kRows * (LEOAM_D + 1) + rc];
            x4[u] = load16(piece, ((size_t)d4 * kRows + rc) * 16);
        }
        float now = m;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i0 + u >= up.count) ms[u] = -INFINITY;
            now = fmaxf(now, ms[u]);
        }
        const float c = exp2_or_zero(m, now);
        m = now;
        l *= c;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] *= c;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i0 + u >= up.count) continue;
            const float w = exp2_or_zero(ms[u], m);
            float x[4];
            unpack<F32>(x4[u], x);
            l += w * ls[u];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += w * x[e];
        }
    }
    if (parts > 1) {
        sh[0][threadIdx.x] = m;
        sh[1][threadIdx.x] = l;
#pragma unroll
        for (int e = 0; e < 4; ++e) sh[2 + e][threadIdx.x] = o[e];
        __syncthreads();
        if (part) return;
        for (int p = 1; p < parts; ++p) m = fmaxf(m, sh[0][threadIdx.x + p * n_rows]);
        l = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = 0.f;
        for (int p = 0; p < parts; ++p) {
            const int i = threadIdx.x + p * n_rows;
            const float w = exp2_or_zero(sh[0][i], m);
            l += w * sh[1][i];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += w * sh[2 + e][i];
        }
    }
    if (row >= up.rows) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int h = blockIdx.x % a.n_kv_heads;
    const size_t q_row = ((size_t)(up.token0 + row / group) * a.n_kv_heads + h) * group + row % group;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= inv;
    char* out = a.out + q_row * LEOAM_D * T::kBytes;
    if constexpr (T::kTag == LEOAM_F32) store16(out, 16 * d4, pack<F32>(o));
    else *reinterpret_cast<uint2*>(out + 8 * d4) = make_uint2(pair_of(T{}, o[0], o[1]), pair_of(T{}, o[2], o[3]));
    if (a.lse && d4 == 0) a.lse[q_row] = log_sum_exp(m, l, prefill_bias<T>());
}

size_t page_decode_workspace_bytes(const leoam_pages*);
size_t page_decode_min_workspace_bytes(const leoam_pages*);

static long long prefill_slots(const leoam_pages* s, long long n_new) {
    return n_new * (s->n_q_heads / s->n_kv_heads) / kRows + s->batch;
}
static size_t prefill_directory_bytes(long long units) { return (size_t)(units * sizeof(UnitPieces) + 255) / 256 * 256; }

size_t page_min_workspace_bytes(const leoam_pages* s) { return page_decode_min_workspace_bytes(s); }
size_t page_workspace_bytes(const leoam_pages* s, int n_new) {
    if (n_new <= 0) return page_decode_workspace_bytes(s);
    const long long units = prefill_slots(s, n_new) * s->n_kv_heads;
    size_t bytes = 16;
    if (units <= kMostUnits && prefill_slots(s, n_new) <= kMostSlots)
        bytes = prefill_directory_bytes(units) + 2 * (size_t)kSharers * kPieceFloats * sizeof(float);
    const size_t least = page_min_workspace_bytes(s);
    return bytes > least ? bytes : least;
}

template <typename T, typename S, int G> static hipError_t launch_prefill(const PagePrefillArgs& a, int sharers, hipStream_t stream) {
    const long long units = (long long)a.n_slots * a.n_kv_heads;
    if (units > 0x7fffffffll) return hipErrorInvalidValue;
    const dim3 block(kAttThreads);
    if (sharers == 0) {
        hipLaunchKernelGGL((page_prefill_kernel<T, S, G, false>), dim3((unsigned)units), block, 0, stream, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((page_prefill_kernel<T, S, G, true>), dim3(sharers), block, 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((page_prefill_merge_kernel<T>), dim3((unsigned)units, LEOAM_D / 8), dim3(256), 0, stream, a, G);
    return hipGetLastError();
}
template <typename T, typename S> static hipError_t prefill_of(const PagePrefillArgs& a, int group, int sharers, hipStream_t stream) {
    switch (group) {
    case 1: return launch_prefill<T, S, 1>(a, sharers, stream);
    case 2: return launch_prefill<T, S, 2>(a, sharers, stream);
    case 4: return launch_prefill<T, S, 4>(a, sharers, stream);
    default: return launch_prefill<T, S, 8>(a, sharers, stream);
    }
}

hipError_t page_prefill_dispatch(const leoam_pages* s, const void* q, int n_new, const int32_t* new_off, const void* k_pages,
                                 const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* page_table,
                                 const int32_t* seq_len, float softmax_scale, void* out, float* lse, void* workspace,
                                 size_t workspace_bytes, hipStream_t stream) {
    PagePrefillArgs a;
    const int group = s->n_q_heads / s->n_kv_heads;
    const long long slots = new_off ? prefill_slots(s, n_new) : s->batch, units = slots * s->n_kv_heads;
    if (units > 0x7fffffffll) return hipErrorInvalidValue;
    a.q = (const char*)q; a.k_pages = (const char*)k_pages; a.v_pages = (const char*)v_pages;
    a.k_scale = k_scale; a.v_scale = v_scale; a.page_table = page_table; a.seq_len = seq_len; a.new_off = new_off;
    a.n_new = n_new;
    a.n_slots = (int)slots;
    // (hidden logits are -inf before they are scaled: a scale of zero is the smallest there is instead)
    a.scale_log2 = fabsf(softmax_scale) * kLog2e;
    if (a.scale_log2 < FLT_MIN) a.scale_log2 = FLT_MIN;
    a.flip = softmax_scale < 0.f ? (s->q_dtype == LEOAM_F32 ? 0x80000000u : 0x80008000u) : 0u;
    a.out = (char*)out; a.lse = lse;
    a.batch = s->batch; a.n_kv_heads = s->n_kv_heads; a.n_pages = s->n_pages;
    a.page_shift = __builtin_ctz((unsigned)s->page_size); a.max_pages = s->max_pages;
    // shared out if the units make less than two rounds of workgroups and the workspace holds two pieces for each of at least
    // as many sharers as there are units (or as fill half the chip)
    int sharers = 0;
    a.pieces = (UnitPieces*)workspace;
    a.partial = nullptr;
    const long long most_tiles = (((long long)s->max_pages * s->page_size + 31) / 32) * units;      // 32-bit sums
    // (nor if no sequence can have so many tiles that it would be cut)
    const bool k32 = s->q_dtype == LEOAM_F32;
    const long long capacity = (long long)s->max_pages * s->page_size;
    const bool cut = units <= kMostUnits && capacity > (long long)uncut_unit_tiles((int)units, k32) * (k32 ? 32 : 64);
    if (cut && slots <= kMostSlots && most_tiles < (1ll << 30)) {
        const size_t dir = prefill_directory_bytes(units), piece = kPieceFloats * sizeof(float);
        const long long fit = workspace_bytes > dir ? (long long)((workspace_bytes - dir) / (2 * piece)) : 0;
        if (fit >= (units < kSharers / 2 ? units : kSharers / 2)) sharers = (int)(fit < kSharers ? fit : kSharers);
        a.partial = (float*)((char*)workspace + dir);
    }
    const bool k8 = s->kv_dtype == LEOAM_E4M3;
    switch (s->q_dtype) {
    case LEOAM_F32: return prefill_of<F32, F32>(a, group, sharers, stream);
    case LEOAM_F16: return k8 ? prefill_of<F16, E4M3>(a, group, sharers, stream) : prefill_of<F16, F16>(a, group, sharers, stream);
    default: return k8 ? prefill_of<BF16, E4M3>(a, group, sharers, stream) : prefill_of<BF16, BF16>(a, group, sharers, stream);
    }
}

}  // namespace leoam
