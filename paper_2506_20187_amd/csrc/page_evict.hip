// page_evict_select: which tokens of a sequence's kv head stay, and which rows move to the places that become free.
//
// Order: protected tokens (the first ones and the most recent ones) before all others, those by weight, equal ones by place;
// the first `keep` stay.  A place t < keep whose token does not stay is free, a token at t >= keep that stays moves: there are as
// many of the one as of the other, the i-th moves to the i-th.  With kept(t) = tokens before t that stay, t < keep is free place
// number t - kept(t), and t >= keep is mover number kept(t) - kept(keep): one count in order gives both.
//
// A weight becomes a 32-bit key of the same order, protected ones the highest, and the lowest key that stays is found by histograms of
// 11, 11 and 10 of its bits.  What is read is 8 bytes a token; bound by latency, where there are many rows by the instructions for each
// key.  A workgroup holds the keys of a row in registers (16 rows of 4200 tokens 8.4 us, of 32000 31, 512 rows of 20000 52).  Longer
// rows are cut into parts of 4096 or 8192 places (at `keep`, too, so that what stays before it is a sum over parts): three launches make
// the parts' histograms, each beginning with the sums of the last one's, a fourth one lists (16 rows of 64000 24 us).
#include "page_common.h"

namespace leoam {

struct EvictArgs {
    const float* weight;
    const int32_t *token_id, *n_seen, *seq_len, *keep_len, *n_first;
    int n_recent;
    int32_t* moves;
    int m_max;
    int32_t *move_count, *new_len, *status;
    int n_kv_heads, capacity;
};

constexpr int kPartThreads = 512;      // of a part
constexpr int kEvictBins = 2048;
constexpr uint32_t kProtected = 0xffffffffu;       // above every weight's key

// keys compare as the weights do; NaN is below all of them, -0 is 0
__device__ __forceinline__ uint32_t key_of_weight(float w) {
    if (w != w) return 0u;
    const uint32_t u = w == 0.f ? 0u : float_to_bits(w);
    return u >> 31 ? ~u : u | 0x80000000u;
}

// What is asked of a row, and what has to be known of its tokens.
struct EvictRow {
    int n, keep, first;
    long long newest;      // numbers from here on are recent
    const float* weight;
    const int32_t* ids;
    bool none, bad;
    __device__ __forceinline__ EvictRow(const EvictArgs& a, int bh) {
        const int b = bh / a.n_kv_heads;
        n = uniform(a.seq_len[b]);
        keep = uniform(a.keep_len[b]);
        bad = n < 0 || n > a.capacity || keep < 0 || (keep < n && min(keep, n - keep) > a.m_max);
        none = bad || keep >= n || keep == 0;
        first = a.n_first ? a.n_first[b] : 0;
        weight = a.weight + (size_t)bh * a.capacity;
        ids = a.token_id ? a.token_id + (size_t)bh * a.capacity : nullptr;
        newest = (long long)(ids ? a.n_seen[b] : n) - a.n_recent;
    }
    __device__ __forceinline__ uint32_t key(int t, int id, float w) const {
        const uint32_t k = key_of_weight(w);
        return t < first || id >= newest ? kProtected : k;
    }
    __device__ __forceinline__ void report(const EvictArgs& a, int bh) const {
        const int b = bh / a.n_kv_heads;
        if (bh == b * a.n_kv_heads) {
            a.new_len[b] = bad || keep >= n ? n : keep;
            if (a.status) a.status[b] = bad ? 1 : 0;
        }
        if (none) a.move_count[bh] = 0;
    }
};

// Places [begin, end) of a row, dealt out to the waves in order, 64 at a time, with their keys.
template <int THREADS, int HELD> struct HeldKeys {
    uint32_t keys[HELD];
    int begin, end;
    __device__ __forceinline__ HeldKeys(const EvictRow& row, int lo, int hi) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / LEOAM_WAVE), seg = (hi - lo + THREADS - 1) / THREADS * LEOAM_WAVE;
        begin = min(hi, lo + wave * seg);
        end = min(hi, begin + seg);
        constexpr int TOGETHER = HELD < 16 ? HELD : 16;      // on their way together; places past the last repeat it
#pragma unroll
        for (int i0 = 0; i0 < HELD; i0 += TOGETHER) {
            if (begin + i0 * LEOAM_WAVE >= end) break;
            float w[TOGETHER];
            int id[TOGETHER];
#pragma unroll
            for (int i = 0; i < TOGETHER; ++i) {
                if (begin + (i0 + i) * LEOAM_WAVE >= end) break;
                const int t = min(begin + (i0 + i) * LEOAM_WAVE + lane_id(), end - 1);
                w[i] = row.weight[t];
                id[i] = row.ids ? row.ids[t] : t;
            }
#pragma unroll
            for (int i = 0; i < TOGETHER; ++i)
                keys[i0 + i] = row.key(min(begin + (i0 + i) * LEOAM_WAVE + lane_id(), end - 1), id[i], w[i]);
        }
    }
    template <typename F> __device__ __forceinline__ void each(F&& f) const {      // f(place, key, counts), by whole waves
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int t = begin + i * LEOAM_WAVE + lane_id();
            if (begin + i * LEOAM_WAVE < end) f(t, keys[i], t < end);
        }
    }
};

// the sum of the waves' words before this wave's
template <int WAVES> __device__ __forceinline__ int before_wave(const int* sh, int wave) {
    const uint32_t incl = wave_incl_scan_u32(lane_id() < WAVES ? (uint32_t)sh[lane_id()] : 0u);
    return wave ? __builtin_amdgcn_readlane((int)incl, wave - 1) : 0;
}

// The bin, from the top, in which the `need`-th entry of a histogram is: bin, entries above it, entries in it.  The workgroup's `sh`:
// waves + 3 words.
template <int THREADS> __device__ __forceinline__ int3 find_bin(int need, int* sh, const uint32_t* hist) {
    constexpr int PER = kEvictBins / THREADS, WAVES = THREADS / LEOAM_WAVE;
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE);
    const int first = kEvictBins - (tid + 1) * PER;
    uint32_t c[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) c[i] = hist[first + i];
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += c[i];
    const uint32_t incl = wave_incl_scan_u32(sum);
    if (lane == LEOAM_WAVE - 1) sh[wave] = (int)incl;
    __syncthreads();
    int before = before_wave<WAVES>(sh, wave) + (int)(incl - sum);
#pragma unroll
    for (int i = PER - 1; i >= 0; --i) {
        if (before < need && before + (int)c[i] >= need) {
            sh[WAVES] = first + i;
            sh[WAVES + 1] = before;
            sh[WAVES + 2] = (int)c[i];
        }
        before += (int)c[i];
    }
    __syncthreads();
    const int3 found = make_int3(sh[WAVES], sh[WAVES + 1], sh[WAVES + 2]);
    __syncthreads();
    return found;
}

// The histogram of a stage in LDS: stage 0: bits 31..21 of all keys; 1: bits 20..10 of those that begin as `prefix`; 2: bits 9..0.
// (Protected ones come by the wave, all of them into the last bin: counted by the wave.)
template <int STAGE, int THREADS, int HELD>
__device__ __forceinline__ void count_keys(const HeldKeys<THREADS, HELD>& held, uint32_t prefix, uint32_t* hist) {
    constexpr int kShift = STAGE == 0 ? 21 : STAGE == 1 ? 10 : 0, kKnown = STAGE == 1 ? 21 : 10;
    int guarded = 0;
    held.each([&](int, uint32_t k, bool in) {
        const bool last = in && k == kProtected;
        guarded += __popcll(__ballot(last));
        if (in && !last && (STAGE == 0 || (k ^ prefix) >> kKnown == 0)) atomicAdd(&hist[k >> kShift & (STAGE == 2 ? 1023u : 2047u)], 1u);
    });
    if (lane_id() == 0 && guarded && (STAGE == 0 || (kProtected ^ prefix) >> kKnown == 0))
        atomicAdd(&hist[STAGE == 2 ? 1023 : 2047], (uint32_t)guarded);
}

// The moves of places [begin, end): keys above `bound` stay, and the first `ties` of those equal to it.  above, equal: how many of either
// are before the wave's places; kept_low: how many stay below `keep`.
template <int THREADS, int HELD>
__device__ __forceinline__ void list_moves(const HeldKeys<THREADS, HELD>& held, int keep, uint32_t bound, int ties, int above, int equal,
                                           int kept_low, int32_t* moves) {
    const uint64_t below = (1ull << lane_id()) - 1;
    held.each([&](int t, uint32_t k, bool in) {
        const uint64_t ab = __ballot(in && k > bound), eq = __ballot(in && k == bound);
        const int equal_here = equal + __popcll(eq & below);
        const int kept = above + __popcll(ab & below) + min(equal_here, ties);
        const bool stays = k > bound || (k == bound && equal_here < ties);
        if (in && t < keep && !stays) moves[2 * (size_t)(t - kept)] = t;
        if (in && t >= keep && stays) moves[2 * (size_t)(kept - kept_low) + 1] = t;
        above += __popcll(ab);
        equal += __popcll(eq);
    });
}

// ---- a row to a workgroup ---------------------------------------------------------------------------------
template <int THREADS, int HELD>
__global__ __launch_bounds__(THREADS, HELD <= 16 ? 8 : 4) void page_evict_row_kernel(EvictArgs a) {
    constexpr int WAVES = THREADS / LEOAM_WAVE;
    __shared__ uint32_t hist[3][kEvictBins];
    __shared__ int sh_find[WAVES + 3], sh_above[WAVES], sh_equal[WAVES], sh_kept_low[2];
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE), bh = blockIdx.x;
    const EvictRow row(a, bh);
    if (tid == 0) row.report(a, bh);
    if (row.none) return;
    const HeldKeys<THREADS, HELD> held(row, 0, row.n);
    const int keep = row.keep;
    for (int i = tid; i < 3 * kEvictBins; i += THREADS) hist[0][i] = 0;
    if (tid < 2) sh_kept_low[tid] = 0;

    // ---- keys above `bound` stay, and `ties` of those equal to it
    uint32_t bound = 0;
    int ties = keep;
    auto stage = [&](auto which) {      // whether the bound is found: the key itself, or a bin that stays whole
        constexpr int STAGE = decltype(which)::value, kShift = STAGE == 0 ? 21 : STAGE == 1 ? 10 : 0;
        __syncthreads();
        count_keys<STAGE, THREADS, HELD>(held, bound, hist[STAGE]);
        __syncthreads();
        const int3 found = find_bin<THREADS>(ties, sh_find, hist[STAGE]);
        ties -= found.y;
        bound |= (uint32_t)found.x << kShift;
        if (STAGE < 2 && ties == found.z && bound > 0u) {
            bound -= 1u;
            ties = 0;
            return true;
        }
        return STAGE == 2;
    };
    if (!stage(std::integral_constant<int, 0>{}) && !stage(std::integral_constant<int, 1>{})) stage(std::integral_constant<int, 2>{});

    // ---- how many stay before each wave's places, and before `keep`
    {
        int above = 0, equal = 0, above_low = 0, equal_low = 0;
        held.each([&](int t, uint32_t k, bool in) {
            const uint64_t ab = __ballot(in && k > bound), eq = __ballot(in && k == bound), lo = __ballot(t < keep);
            above += __popcll(ab);
            equal += __popcll(eq);
            above_low += __popcll(ab & lo);
            equal_low += __popcll(eq & lo);
        });
        if (lane == 0) {
            sh_above[wave] = above;
            sh_equal[wave] = equal;
            atomicAdd(&sh_kept_low[0], above_low);
            atomicAdd(&sh_kept_low[1], equal_low);
        }
    }
    __syncthreads();
    const int above = before_wave<WAVES>(sh_above, wave), equal = before_wave<WAVES>(sh_equal, wave);
    const int kept_low = sh_kept_low[0] + min(sh_kept_low[1], ties);
    if (tid == 0) a.move_count[bh] = keep - kept_low;
    list_moves<THREADS, HELD>(held, keep, bound, ties, above, equal, kept_low, a.moves + (size_t)bh * a.m_max * 2);
}

// ---- a part of a row to a workgroup -------------------------------------------------------------------------
// Of each part: histograms of two stages in turn, and how many of its keys are above all bins that were found so far.  Of each row,
// stage by stage: the bits of the bound that are known, and how many entries of the bin are still needed.
constexpr int kCoarse = 64, kFine = kEvictBins / kCoarse;
struct EvictFound { uint32_t prefix; int need; };
struct EvictLong {
    uint32_t* hist;         // [2][row][part][kEvictBins]
    uint32_t* coarse;       // [2][row][part][kCoarse]: its bins by 32
    int* above;             // [2][row][part]
    EvictFound* found;      // [2][row]
    int rows, parts;
};

// the parts of a row: those below `keep`, then those from it on
template <int PART> struct PartOf {
    int n_low, n_parts, begin, end;
    __device__ __forceinline__ PartOf(const EvictRow& row, int p) {
        n_low = (row.keep + PART - 1) / PART;
        n_parts = n_low + (row.n - row.keep + PART - 1) / PART;
        const int lo = p < n_low ? 0 : row.keep, hi = p < n_low ? row.keep : row.n;
        begin = lo + (p < n_low ? p : p - n_low) * PART;
        end = min(hi, begin + PART);
    }
};

// The bin of a row's histogram, from the top, that holds the `need`-th entry, out of those of its parts: first among the coarse bins,
// then among the 32 that one is made of, so that little more is read than 384 bytes of each part.  of(q, k): whether part q belongs to
// set k of K.
constexpr int kPartWaves = kPartThreads / LEOAM_WAVE;
template <int K> struct PartSums { uint32_t x[2][kPartWaves][K + 1][LEOAM_WAVE]; };
template <int K> struct PartBin {
    int bin, above, above_of[K], equal_of[K];      // entries above the bin: of the row, of the sets; entries in it
    template <typename F>
    __device__ __forceinline__ PartBin(const uint32_t* hist, const uint32_t* coarse, int n_parts, int need, PartSums<K>& sh, F&& of) {
        const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / LEOAM_WAVE);
        above = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) above_of[k] = 0;
        auto look = [&](int level, int lanes_of_part, const uint32_t* from, int stride) __attribute__((always_inline)) {
            // lane i of a part's: its i-th bin from the top
            const int per = LEOAM_WAVE / lanes_of_part, i = lane % lanes_of_part;
            uint32_t sums[K + 1];
#pragma unroll
            for (int k = 0; k <= K; ++k) sums[k] = 0;
            for (int q0 = wave * per + lane / lanes_of_part; q0 < n_parts; q0 += 4 * kPartWaves * per) {
                uint32_t x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    x[u] = from[(size_t)min(q0 + u * kPartWaves * per, n_parts - 1) * stride + lanes_of_part - 1 - i];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int q = q0 + u * kPartWaves * per;
                    if (q >= n_parts) break;
#pragma unroll
                    for (int k = 0; k < K; ++k) sums[k] += of(q, k) ? x[u] : 0u;
                    sums[K] += x[u];
                }
            }
#pragma unroll
            for (int k = 0; k <= K; ++k) sh.x[level][wave][k][lane] = sums[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k <= K; ++k) {
                sums[k] = 0;
#pragma unroll
                for (int w = 0; w < kPartWaves; ++w)
                    for (int r = 0; r < per; ++r) sums[k] += sh.x[level][w][k][r * lanes_of_part + i];
                if (lane >= lanes_of_part) sums[k] = 0;
            }
            const uint32_t upto = wave_incl_scan_u32(sums[K]), left = (uint32_t)(need - above);
            const int hit = min(__builtin_ctzll(__ballot(upto >= left && upto - sums[K] < left) | 1ull << 63), lanes_of_part - 1);
            above += __builtin_amdgcn_readlane((int)(upto - sums[K]), hit);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                above_of[k] += __builtin_amdgcn_readlane((int)(wave_incl_scan_u32(sums[k]) - sums[k]), hit);
                equal_of[k] = __builtin_amdgcn_readlane((int)sums[k], hit);
            }
            return lanes_of_part - 1 - hit;
        };
        const int big = look(0, kCoarse, coarse, kCoarse);
        bin = big * kFine + look(1, kFine, hist + big * kFine, kEvictBins);
    }
};

template <int STAGE, int HELD> __global__ __launch_bounds__(kPartThreads, 4) void page_evict_hist_kernel(EvictArgs a, EvictLong s) {
    __shared__ __align__(16) uint32_t hist[kEvictBins];
    __shared__ PartSums<1> sh_find;
    const int tid = threadIdx.x, bh = blockIdx.x / s.parts, p = blockIdx.x % s.parts;
    const EvictRow row(a, bh);
    if (STAGE == 0 && tid == 0 && p == 0) row.report(a, bh);
    if (row.none) return;
    const PartOf<HELD * kPartThreads> part(row, p);
    if (p >= part.n_parts) return;
    const HeldKeys<kPartThreads, HELD> held(row, part.begin, part.end);
    const size_t here = ((size_t)(STAGE & 1) * s.rows + bh) * s.parts + p;
    for (int i = tid; i < kEvictBins; i += kPartThreads) hist[i] = 0;
    uint32_t prefix = 0;
    int above = 0;
    if constexpr (STAGE > 0) {
        constexpr int kKnown = STAGE == 1 ? 21 : 10;
        const size_t before = (size_t)((STAGE & 1) ^ 1) * s.rows + bh;      // the last stage's
        above = s.above[before * s.parts + p];
        int need = row.keep;
        if (STAGE == 2) {
            const EvictFound f = s.found[bh];
            need = f.need;
            prefix = f.prefix;
        }
        const PartBin<1> found(s.hist + before * s.parts * kEvictBins, s.coarse + before * s.parts * kCoarse, part.n_parts, need, sh_find,
                               [&](int q, int) { return q == p; });
        prefix |= (uint32_t)found.bin << kKnown;
        above += found.above_of[0];
        if (tid == 0 && p == 0) s.found[(size_t)(STAGE - 1) * s.rows + bh] = EvictFound{prefix, need - found.above};
    }
    __syncthreads();
    count_keys<STAGE, kPartThreads, HELD>(held, prefix, hist);
    __syncthreads();
    static_assert(kEvictBins == 4 * kPartThreads && kFine == 32, "a thread writes four bins, eight threads a coarse one");
    const uint4 mine = *reinterpret_cast<const uint4*>(hist + 4 * tid);
    *reinterpret_cast<uint4*>(s.hist + here * kEvictBins + 4 * tid) = mine;
    uint32_t sum = (mine.x + mine.y) + (mine.z + mine.w);
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) sum += __shfl_xor(sum, d, LEOAM_WAVE);
    if ((tid & 7) == 0) s.coarse[here * kCoarse + (tid >> 3)] = sum;
    if (tid == 0) s.above[here] = above;
}

template <int HELD> __global__ __launch_bounds__(kPartThreads, 4) void page_evict_list_kernel(EvictArgs a, EvictLong s) {
    constexpr int WAVES = kPartThreads / LEOAM_WAVE;
    __shared__ PartSums<2> sh_find;
    __shared__ int sh_above[WAVES], sh_equal[WAVES];
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE);
    const int bh = blockIdx.x / s.parts, p = blockIdx.x % s.parts;
    const EvictRow row(a, bh);
    if (row.none) return;
    const PartOf<HELD * kPartThreads> part(row, p);
    if (p >= part.n_parts) return;
    const HeldKeys<kPartThreads, HELD> held(row, part.begin, part.end);
    // of the parts before this one, and of those below `keep`: keys above the bound and equal to it
    const size_t first = (size_t)bh * s.parts;      // (stage 2's)
    const EvictFound before = s.found[s.rows + bh];
    const PartBin<2> found(s.hist + first * kEvictBins, s.coarse + first * kCoarse, part.n_parts, before.need, sh_find,
                           [&](int q, int k) { return q < (k == 0 ? p : part.n_low); });
    const uint32_t bound = before.prefix | (uint32_t)found.bin;
    const int ties = before.need - found.above;
    uint32_t above_of[2] = {0, 0};
    for (int q = lane; q < part.n_parts; q += LEOAM_WAVE) {
        const int x = s.above[first + q];
        above_of[0] += q < p ? x : 0;
        above_of[1] += q < part.n_low ? x : 0;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
        above_of[k] = __builtin_amdgcn_readlane((int)wave_incl_scan_u32(above_of[k]), LEOAM_WAVE - 1) + found.above_of[k];
    int above = 0, equal = 0;
    held.each([&](int, uint32_t k, bool in) {
        above += __popcll(__ballot(in && k > bound));
        equal += __popcll(__ballot(in && k == bound));
    });
    if (lane == 0) {
        sh_above[wave] = above;
        sh_equal[wave] = equal;
    }
    __syncthreads();
    above = above_of[0] + before_wave<WAVES>(sh_above, wave);
    equal = found.equal_of[0] + before_wave<WAVES>(sh_equal, wave);
    const int kept_low = above_of[1] + min(found.equal_of[1], ties);
    if (tid == 0 && p == 0) a.move_count[bh] = row.keep - kept_low;
    list_moves<kPartThreads, HELD>(held, row.keep, bound, ties, above, equal, kept_low, a.moves + (size_t)bh * a.m_max * 2);
}

// Into how many parts rows are cut at most; 0: a row to a workgroup.  That takes a microsecond for a thousand tokens, four launches take
// 22 to 26 if there are few rows (four of 40000 22.5, 16 of 64000 24; a workgroup 16 of 20000 24, of 32000 31, of 64000 60), but more
// work in all (128 rows of 32000, parts 57, a workgroup 33; of 60000 74 / 61, 512 of those 221 / 142).
// The width is the table's: short rows of a wide one get workgroups with registers for more keys, of which fewer share a compute unit, or
// the four launches, most of whose workgroups find nothing to do (320 rows of 4200 in tables of 4288 tokens 13.8, of 16384 16.6, of 32768
// 27.3; of 131072, four launches, 66.4).
// Keys of a part's thread: few for few rows (16 rows of 64000, 8 and 16 keys: 24, 29; 64 of those 47, 51; 256 of 130000 307, 232).
constexpr int kRowHeld = 64;      // keys of a thread, at most
static int part_held(int rows) { return rows <= 64 ? 8 : 16; }
static int evict_parts(const leoam_pages* s) {
    const int capacity = s->max_pages * s->page_size, rows = s->batch * s->n_kv_heads;
    return capacity <= (rows < 64 ? 16 : rows < 128 ? 32 : kRowHeld) * 1024 ? 0 : capacity / (part_held(rows) * kPartThreads) + 2;
}
static size_t evict_hist_bytes(const leoam_pages* s) {
    return 2 * (size_t)s->batch * s->n_kv_heads * evict_parts(s) * kEvictBins * sizeof(uint32_t);
}
static size_t evict_above_bytes(const leoam_pages* s) { return 2 * (size_t)s->batch * s->n_kv_heads * evict_parts(s) * sizeof(int); }
static size_t evict_coarse_bytes(const leoam_pages* s) { return evict_hist_bytes(s) / kFine; }
size_t page_evict_workspace_bytes(const leoam_pages* s) {
    return evict_hist_bytes(s) + evict_coarse_bytes(s) + evict_above_bytes(s) + 2 * (size_t)s->batch * s->n_kv_heads * sizeof(EvictFound);
}

hipError_t page_evict_dispatch(const leoam_pages* s, const float* weight, const int32_t* token_id, const int32_t* n_seen,
                               const int32_t* seq_len, const int32_t* keep_len, const int32_t* n_first, int n_recent, int32_t* moves,
                               int m_max, int32_t* move_count, int32_t* new_len, int32_t* status, void* workspace, hipStream_t stream) {
    EvictArgs a;
    a.weight = weight; a.token_id = token_id; a.n_seen = n_seen; a.seq_len = seq_len; a.keep_len = keep_len; a.n_first = n_first;
    a.n_recent = n_recent; a.moves = moves; a.m_max = m_max; a.move_count = move_count; a.new_len = new_len; a.status = status;
    a.n_kv_heads = s->n_kv_heads; a.capacity = s->max_pages * s->page_size;
    const int rows = s->batch * s->n_kv_heads, parts = evict_parts(s);
    if (parts == 0) {
        // (two workgroups of 1024 threads share a compute unit, four of 512: 16 rows of 4200 8.4 against 9.7 us, 512 of those 13.8 / 14.7,
        // 1024 25.9 / 22.0)
        if (a.capacity <= 8 * 1024 && rows <= 512)
            hipLaunchKernelGGL((page_evict_row_kernel<1024, 8>), dim3(rows), dim3(1024), 0, stream, a);
        else if (a.capacity <= 16 * 512) hipLaunchKernelGGL((page_evict_row_kernel<512, 16>), dim3(rows), dim3(512), 0, stream, a);
        else if (a.capacity <= 16 * 1024) hipLaunchKernelGGL((page_evict_row_kernel<1024, 16>), dim3(rows), dim3(1024), 0, stream, a);
        else if (a.capacity <= 32 * 1024) hipLaunchKernelGGL((page_evict_row_kernel<1024, 32>), dim3(rows), dim3(1024), 0, stream, a);
        else hipLaunchKernelGGL((page_evict_row_kernel<1024, kRowHeld>), dim3(rows), dim3(1024), 0, stream, a);
        return hipGetLastError();
    }
    if ((long long)rows * parts > 0x7fffffffll) return hipErrorInvalidValue;
    EvictLong l;
    l.hist = (uint32_t*)workspace;
    l.coarse = (uint32_t*)((char*)l.hist + evict_hist_bytes(s));
    l.above = (int*)((char*)l.coarse + evict_coarse_bytes(s));
    l.found = (EvictFound*)((char*)l.above + evict_above_bytes(s));
    l.rows = rows; l.parts = parts;
    const dim3 grid((unsigned)(rows * parts)), block(kPartThreads);
    auto launch = [&](auto held) {
        constexpr int HELD = decltype(held)::value;
        hipLaunchKernelGGL((page_evict_hist_kernel<0, HELD>), grid, block, 0, stream, a, l);
        hipLaunchKernelGGL((page_evict_hist_kernel<1, HELD>), grid, block, 0, stream, a, l);
        hipLaunchKernelGGL((page_evict_hist_kernel<2, HELD>), grid, block, 0, stream, a, l);
        hipLaunchKernelGGL(page_evict_list_kernel<HELD>, grid, block, 0, stream, a, l);
    };
    if (part_held(rows) == 8) launch(std::integral_constant<int, 8>{});
    else launch(std::integral_constant<int, 16>{});
    return hipGetLastError();
}

}  // namespace leoam
