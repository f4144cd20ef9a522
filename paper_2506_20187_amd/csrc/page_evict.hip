// page_evict_select: which tokens of a sequence's kv head stay, and which rows move to the places that become free.
//
// Order: protected tokens (the first ones and the most recent ones) before all others, those by weight, equal ones by place;
// the first `keep` stay.  A place t < keep whose token does not stay is free, a token at t >= keep that stays moves: there are as
// many of the one as of the other, the i-th moves to the i-th.  With kept(t) = tokens before t that stay, t < keep is free place
// number t - kept(t), and t >= keep is mover number kept(t) - kept(keep): one count in order gives both.
//
// A weight becomes a 32-bit key of the same order, and the lowest key that stays is found by histograms.  What is read is 8 bytes
// a token; bound by latency.  Where a row fits, one workgroup holds its keys in registers and narrows down their range, 11 bits at
// a time.  Longer rows are cut into parts of 16384 places (at `keep`, too, so that what stays before it is a sum over parts): three
// launches make histograms of the parts' keys by 11, 11 and 10 bits, each beginning with the sums of the last one's, a fourth one lists.
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

constexpr int kEvictThreads = 1024;
constexpr int kEvictHeld = 16;                     // keys of a thread
constexpr int kEvictPart = kEvictThreads * kEvictHeld;
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
    bool bad, none;
    __device__ __forceinline__ EvictRow(const EvictArgs& a, int bh) {
        const int b = bh / a.n_kv_heads;
        n = uniform(a.seq_len[b]);
        keep = uniform(a.keep_len[b]);
        bad = n < 0 || n > a.capacity || keep < 0 || (keep < n && min(keep, n - keep) > a.m_max);
        none = bad || keep >= n;
        first = a.n_first ? a.n_first[b] : 0;
        weight = a.weight + (size_t)bh * a.capacity;
        ids = a.token_id ? a.token_id + (size_t)bh * a.capacity : nullptr;
        newest = (long long)(ids ? a.n_seen[b] : n) - a.n_recent;
    }
    __device__ __forceinline__ uint32_t key(int t) const {
        const int id = ids ? ids[t] : t;
        const uint32_t k = key_of_weight(weight[t]);
        return t < first || id >= newest ? kProtected : k;
    }
    __device__ __forceinline__ void report(const EvictArgs& a, int bh) const {
        const int b = bh / a.n_kv_heads;
        if (bh == b * a.n_kv_heads) {
            a.new_len[b] = none ? n : keep;
            if (a.status) a.status[b] = bad ? 1 : 0;
        }
        if (none) a.move_count[bh] = 0;
    }
};

// Places [begin, end) of a row, dealt out to the waves in order, 64 at a time, with their keys.
template <int THREADS> struct HeldKeys {
    uint32_t keys[kEvictHeld];
    int begin, end;
    __device__ __forceinline__ HeldKeys(const EvictRow& row, int lo, int hi) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / LEOAM_WAVE), seg = (hi - lo + THREADS - 1) / THREADS * LEOAM_WAVE;
        begin = min(hi, lo + wave * seg);
        end = min(hi, begin + seg);
#pragma unroll
        for (int i = 0; i < kEvictHeld; ++i) {
            const int t = begin + i * LEOAM_WAVE + lane_id();
            keys[i] = t < end ? row.key(t) : 0u;
        }
    }
    template <typename F> __device__ __forceinline__ void each(F&& f) const {      // f(place, key, counts), by whole waves
#pragma unroll
        for (int i = 0; i < kEvictHeld; ++i) {
            const int t = begin + i * LEOAM_WAVE + lane_id();
            if (begin + i * LEOAM_WAVE < end) f(t, keys[i], t < end);
        }
    }
};

// The bin, from the top, in which the `need`-th entry of a histogram is: bin, entries above it, entries in it.  count(bin): by
// thread i the bins kEvictBins - 1 - i * PER - (0 .. PER - 1).  The workgroup's `sh`: waves + 3 words.
template <int THREADS, typename F> __device__ __forceinline__ int3 find_bin(int need, int* sh, F&& count) {
    constexpr int PER = kEvictBins / THREADS, WAVES = THREADS / LEOAM_WAVE;
    const int tid = threadIdx.x, lane = lane_id(), wave = tid / LEOAM_WAVE, top = kEvictBins - 1 - tid * PER;
    uint32_t c[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += c[i] = count(top - i);
    const uint32_t incl = wave_incl_scan_u32(sum);
    if (lane == LEOAM_WAVE - 1) sh[wave] = (int)incl;
    __syncthreads();
    int before = (int)(incl - sum);
    for (int w = 0; w < wave; ++w) before += sh[w];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (before < need && before + (int)c[i] >= need) {
            sh[WAVES] = top - i;
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

// The moves of places [begin, end): keys above `bound` stay, and the first `ties` of those equal to it.  above, equal: how many of either
// are before the wave's places; kept_low: how many stay below `keep`.
template <int THREADS>
__device__ __forceinline__ void list_moves(const HeldKeys<THREADS>& held, int keep, uint32_t bound, int ties, int above, int equal, int kept_low,
                                           int32_t* moves) {
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
// (Rows of up to 8192 places: 512 threads, so that four workgroups share a compute unit.)
template <int THREADS> __global__ __launch_bounds__(THREADS, THREADS == 512 ? 8 : 4) void page_evict_row_kernel(EvictArgs a) {
    constexpr int WAVES = THREADS / LEOAM_WAVE;
    __shared__ uint32_t hist[kEvictBins];
    __shared__ uint32_t sh_low, sh_high;
    __shared__ int sh_protected, sh_find[WAVES + 3], sh_above[WAVES], sh_equal[WAVES], sh_kept_low[2];
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE), bh = blockIdx.x;
    const EvictRow row(a, bh);
    if (tid == 0) row.report(a, bh);
    if (row.none) return;
    const HeldKeys<THREADS> held(row, 0, row.n);
    const int keep = row.keep;

    // ---- protected ones, and the range of the others' keys
    if (tid == 0) {
        sh_low = 0xffffffffu;
        sh_high = 0u;
        sh_protected = sh_kept_low[0] = sh_kept_low[1] = 0;
    }
    __syncthreads();
    {
        uint32_t low = 0xffffffffu, high = 0u;
        int count = 0;
        held.each([&](int, uint32_t k, bool in) {
            const bool guarded = in && k == kProtected;
            count += __popcll(__ballot(guarded));
            if (in && !guarded) {
                low = min(low, k);
                high = max(high, k);
            }
        });
        low = wave_min_u32(low);
        high = wave_max_u32(high);
        if (lane == 0) {
            atomicMin(&sh_low, low);
            atomicMax(&sh_high, high);
            atomicAdd(&sh_protected, count);
        }
    }
    __syncthreads();

    // ---- keys above `bound` stay, and `ties` of those equal to it
    uint32_t bound = kProtected, low = sh_low, high = sh_high;
    int ties = keep, need = keep - sh_protected;      // (all of the protected ones or more than fit: the first of them)
    while (need > 0) {
        const int shift = max(0, 21 - __builtin_clz((high - low) | 1u));
        for (int i = tid; i < kEvictBins; i += THREADS) hist[i] = 0;
        __syncthreads();
        held.each([&](int, uint32_t k, bool in) {
            if (in && k >= low && k <= high) atomicAdd(&hist[(k - low) >> shift], 1u);
        });
        __syncthreads();
        const int3 found = find_bin<THREADS>(need, sh_find, [&](int bin) { return hist[bin]; });
        need -= found.y;
        low += (uint32_t)found.x << shift;
        high = min(high, low + ((1u << shift) - 1u));
        if (shift == 0 || (need == found.z && low > 0u)) {      // the key itself, or the whole bin stays
            bound = shift == 0 ? low : low - 1u;
            ties = shift == 0 ? need : 0;
            break;
        }
    }

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
    int above = 0, equal = 0;
    for (int w = 0; w < wave; ++w) {
        above += sh_above[w];
        equal += sh_equal[w];
    }
    const int kept_low = sh_kept_low[0] + min(sh_kept_low[1], ties);
    if (tid == 0) a.move_count[bh] = keep - kept_low;
    list_moves<THREADS>(held, keep, bound, ties, above, equal, kept_low, a.moves + (size_t)bh * a.m_max * 2);
}

// ---- a part of a row to a workgroup -------------------------------------------------------------------------
// Of each part: histograms of two stages in turn, and how many of its keys are above all bins that were found so far (protected ones
// included).  Of each row, stage by stage: the bits of the bound that are known, and how many entries of the bin are still needed.
struct EvictPart { int above, guarded; };
struct EvictFound { uint32_t prefix; int need; };
struct EvictLong {
    uint32_t* hist;         // [2][row][part][kEvictBins]
    EvictPart* part;        // [2][row][part]
    EvictFound* found;      // [2][row]
    int rows, parts;
};

// the parts of a row: those below `keep`, then those from it on
struct PartOf {
    int n_low, n_parts, begin, end;
    __device__ __forceinline__ PartOf(const EvictRow& row, int p) {
        n_low = (row.keep + kEvictPart - 1) / kEvictPart;
        n_parts = n_low + (row.n - row.keep + kEvictPart - 1) / kEvictPart;
        const int lo = p < n_low ? 0 : row.keep, hi = p < n_low ? row.keep : row.n;
        begin = lo + (p < n_low ? p : p - n_low) * kEvictPart;
        end = min(hi, begin + kEvictPart);
    }
};

// stage 0: bits 31..21 of all keys; 1: bits 20..10 of those that the first stage's bin holds; 2: bits 9..0
template <int STAGE> __global__ __launch_bounds__(kEvictThreads, 4) void page_evict_hist_kernel(EvictArgs a, EvictLong s) {
    constexpr int kShift = STAGE == 0 ? 21 : STAGE == 1 ? 10 : 0, kLast = STAGE == 1 ? 21 : 10;
    __shared__ uint32_t hist[kEvictBins];
    __shared__ int sh_find[kEvictThreads / LEOAM_WAVE + 3], sh_guarded, sh_above;
    const int tid = threadIdx.x, bh = blockIdx.x / s.parts, p = blockIdx.x % s.parts;
    const EvictRow row(a, bh);
    if (STAGE == 0 && tid == 0 && p == 0) row.report(a, bh);
    if (row.none) return;
    const PartOf part(row, p);
    if (p >= part.n_parts) return;
    const HeldKeys<kEvictThreads> held(row, part.begin, part.end);
    uint32_t* mine = s.hist + (((size_t)(STAGE & 1) * s.rows + bh) * s.parts + p) * kEvictBins;
    const uint32_t* last = s.hist + ((size_t)((STAGE & 1) ^ 1) * s.rows + bh) * s.parts * kEvictBins;
    EvictPart* state = s.part + ((size_t)(STAGE & 1) * s.rows + bh) * s.parts;
    const EvictPart* was = s.part + ((size_t)((STAGE & 1) ^ 1) * s.rows + bh) * s.parts;
    for (int i = tid; i < kEvictBins; i += kEvictThreads) hist[i] = 0;
    if (tid == 0) sh_guarded = sh_above = 0;
    uint32_t prefix = 0;
    EvictPart now = {0, 0};
    if constexpr (STAGE > 0) {
        int need = row.keep;
        now = was[p];
        if (STAGE == 1)
            for (int i = 0; i < part.n_parts; ++i) need -= was[i].guarded;
        else need = s.found[(STAGE - 2) * s.rows + bh].need;
        if (need <= 0) {      // (the protected ones alone are as many as stay)
            if (tid == 0 && p == 0) s.found[(STAGE - 1) * s.rows + bh] = EvictFound{0u, need};
            if (tid == 0) state[p] = now;
            return;
        }
        const int3 found = find_bin<kEvictThreads>(need, sh_find, [&](int bin) {
            uint32_t sum = 0;
            for (int i = 0; i < part.n_parts; ++i) sum += last[(size_t)i * kEvictBins + bin];
            return sum;
        });
        need -= found.y;
        prefix = (STAGE == 2 ? s.found[bh].prefix : 0u) | (uint32_t)found.x << kLast;
        if (tid == 0 && p == 0) s.found[(STAGE - 1) * s.rows + bh] = EvictFound{prefix, need};
        int above = 0;
        for (int bin = found.x + 1 + tid; bin < kEvictBins; bin += kEvictThreads) above += (int)last[(size_t)p * kEvictBins + bin];
        if (above) atomicAdd(&sh_above, above);
    }
    __syncthreads();
    held.each([&](int, uint32_t k, bool in) {
        const bool guarded = in && k == kProtected;
        if (STAGE == 0) {
            const uint64_t g = __ballot(guarded);
            if (lane_id() == 0 && g) atomicAdd(&sh_guarded, (int)__popcll(g));
        }
        if (!in || guarded) return;
        if (STAGE > 0 && (k ^ prefix) >> kLast) return;
        atomicAdd(&hist[(k >> kShift) & (STAGE == 2 ? 1023u : 2047u)], 1u);
    });
    __syncthreads();
    for (int i = tid; i < kEvictBins; i += kEvictThreads) mine[i] = hist[i];
    if (tid == 0) state[p] = STAGE == 0 ? EvictPart{sh_guarded, sh_guarded} : EvictPart{now.above + sh_above, now.guarded};
}

__global__ __launch_bounds__(kEvictThreads, 4) void page_evict_list_kernel(EvictArgs a, EvictLong s) {
    constexpr int WAVES = kEvictThreads / LEOAM_WAVE;
    __shared__ int sh_find[WAVES + 3], sh_above[WAVES], sh_equal[WAVES], sh_sums[4];
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE);
    const int bh = blockIdx.x / s.parts, p = blockIdx.x % s.parts;
    const EvictRow row(a, bh);
    if (row.none) return;
    const PartOf part(row, p);
    if (p >= part.n_parts) return;
    const HeldKeys<kEvictThreads> held(row, part.begin, part.end);
    const uint32_t* last = s.hist + (size_t)bh * s.parts * kEvictBins;      // (stage 2's)
    const EvictPart* state = s.part + (size_t)bh * s.parts;
    if (tid < 4) sh_sums[tid] = 0;
    uint32_t bound = kProtected;
    int ties = row.keep, bin = kEvictBins;
    const EvictFound before = s.found[s.rows + bh];
    if (before.need > 0) {
        const int3 found = find_bin<kEvictThreads>(before.need, sh_find, [&](int i) {
            uint32_t sum = 0;
            for (int q = 0; q < part.n_parts; ++q) sum += last[(size_t)q * kEvictBins + i];
            return sum;
        });
        bin = found.x;
        bound = before.prefix | (uint32_t)bin;
        ties = before.need - found.y;
    }
    __syncthreads();
    // the parts' keys above the bound and equal to it: those of parts before this one, those of parts below `keep`; a wave to a part
    for (int q = wave; q < part.n_parts; q += WAVES) {
        if (q >= p && q >= part.n_low) continue;
        int above = 0, equal = 0;
        if (bin < kEvictBins) {
            for (int i = lane; i < 1024; i += LEOAM_WAVE) above += i > bin ? (int)last[(size_t)q * kEvictBins + i] : 0;
            for (int d = 32; d > 0; d >>= 1) above += __shfl_xor(above, d, LEOAM_WAVE);
            above += state[q].above;
            equal = (int)last[(size_t)q * kEvictBins + bin];
        } else {
            equal = state[q].guarded;
        }
        if (lane == 0) {
            if (q < p) {
                atomicAdd(&sh_sums[0], above);
                atomicAdd(&sh_sums[1], equal);
            }
            if (q < part.n_low) {
                atomicAdd(&sh_sums[2], above);
                atomicAdd(&sh_sums[3], equal);
            }
        }
    }
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
    above = sh_sums[0];
    equal = sh_sums[1];
    for (int w = 0; w < wave; ++w) {
        above += sh_above[w];
        equal += sh_equal[w];
    }
    const int kept_low = sh_sums[2] + min(sh_sums[3], ties);
    if (tid == 0 && p == 0) a.move_count[bh] = row.keep - kept_low;
    list_moves<kEvictThreads>(held, row.keep, bound, ties, above, equal, kept_low, a.moves + (size_t)bh * a.m_max * 2);
}

static int evict_parts(const leoam_pages* s) {
    const int capacity = s->max_pages * s->page_size;
    return capacity <= kEvictPart ? 0 : capacity / kEvictPart + 2;      // (0: a row to a workgroup)
}
static size_t evict_hist_bytes(const leoam_pages* s) {
    return 2 * (size_t)s->batch * s->n_kv_heads * evict_parts(s) * kEvictBins * sizeof(uint32_t);
}
static size_t evict_part_bytes(const leoam_pages* s) { return 2 * (size_t)s->batch * s->n_kv_heads * evict_parts(s) * sizeof(EvictPart); }
size_t page_evict_workspace_bytes(const leoam_pages* s) {
    return evict_hist_bytes(s) + evict_part_bytes(s) + 2 * (size_t)s->batch * s->n_kv_heads * sizeof(EvictFound);
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
        if (a.capacity <= 512 * kEvictHeld) hipLaunchKernelGGL(page_evict_row_kernel<512>, dim3(rows), dim3(512), 0, stream, a);
        else hipLaunchKernelGGL(page_evict_row_kernel<kEvictThreads>, dim3(rows), dim3(kEvictThreads), 0, stream, a);
        return hipGetLastError();
    }
    if ((long long)rows * parts > 0x7fffffffll) return hipErrorInvalidValue;
    EvictLong l;
    l.hist = (uint32_t*)workspace;
    l.part = (EvictPart*)((char*)workspace + evict_hist_bytes(s));
    l.found = (EvictFound*)((char*)workspace + evict_hist_bytes(s) + evict_part_bytes(s));
    l.rows = rows; l.parts = parts;
    const dim3 grid((unsigned)(rows * parts)), block(kEvictThreads);
    hipLaunchKernelGGL(page_evict_hist_kernel<0>, grid, block, 0, stream, a, l);
    hipLaunchKernelGGL(page_evict_hist_kernel<1>, grid, block, 0, stream, a, l);
    hipLaunchKernelGGL(page_evict_hist_kernel<2>, grid, block, 0, stream, a, l);
    hipLaunchKernelGGL(page_evict_list_kernel, grid, block, 0, stream, a, l);
    return hipGetLastError();
}

}  // namespace leoam
