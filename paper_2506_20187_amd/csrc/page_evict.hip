// page_evict_select: which tokens of a sequence's kv head stay, and which rows move to the places that become free.
//
// Order: protected tokens (the first ones and the most recent ones) before all others, those by weight, equal ones by place;
// the first `keep` stay.  A place t < keep whose token does not stay is free, a token at t >= keep that stays moves: there are as
// many of the one as of the other, the i-th moves to the i-th.  With kept(t) = tokens before t that stay, t < keep is free place
// number t - kept(t), and t >= keep is mover number kept(t) - kept(keep): one count in order gives both.
//
// One workgroup to a (sequence, kv head): a weight becomes a 32-bit key of the same order, and the lowest key that stays is found
// by histograms over the keys' range, 11 bits at a time.  Bound by latency: what is read is 8 bytes a token.
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

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / LEOAM_WAVE;
constexpr int kEvictHeld = 16;                     // keys of a thread that stay in registers
constexpr int kEvictBins = 2048;
constexpr uint32_t kProtected = 0xffffffffu;       // above every weight's key

// keys compare as the weights do; NaN is below all of them, -0 is 0
__device__ __forceinline__ uint32_t key_of_weight(float w) {
    if (w != w) return 0u;
    const uint32_t u = w == 0.f ? 0u : float_to_bits(w);
    return u >> 31 ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kEvictThreads) void page_evict_kernel(EvictArgs a) {
    __shared__ uint32_t hist[kEvictBins];
    __shared__ uint32_t sh_low, sh_high;
    __shared__ int sh_protected, sh_bin, sh_above, sh_in_bin, sh_wave[kEvictWaves], sh_tie[kEvictWaves], sh_kept_low[2];
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE);
    const int bh = blockIdx.x, b = bh / a.n_kv_heads, h = bh - b * a.n_kv_heads;
    const int n = uniform(a.seq_len[b]), keep = uniform(a.keep_len[b]);
    const bool bad = n < 0 || n > a.capacity || keep < 0 || (keep < n && min(keep, n - keep) > a.m_max);
    const bool none = bad || keep >= n;
    if (tid == 0) {
        if (h == 0) {
            a.new_len[b] = none ? n : keep;
            if (a.status) a.status[b] = bad ? 1 : 0;
        }
        if (none) a.move_count[bh] = 0;
    }
    if (none) return;

    const int first = a.n_first ? a.n_first[b] : 0;
    const float* weight = a.weight + (size_t)bh * a.capacity;
    const int32_t* ids = a.token_id ? a.token_id + (size_t)bh * a.capacity : nullptr;
    const long long newest = (long long)(ids ? a.n_seen[b] : n) - a.n_recent;      // numbers from here on are recent
    auto key_at = [&](int t) {
        const int id = ids ? ids[t] : t;
        const uint32_t k = key_of_weight(weight[t]);
        return t < first || id >= newest ? kProtected : k;
    };

    // a wave's stretch of places, 64 at a time
    const int seg = (n + kEvictThreads - 1) / kEvictThreads * LEOAM_WAVE, begin = min(n, wave * seg), end = min(n, begin + seg);
    const bool held = seg <= kEvictHeld * LEOAM_WAVE;
    uint32_t keys[kEvictHeld];
    if (held) {
#pragma unroll
        for (int i = 0; i < kEvictHeld; ++i) {
            const int t = begin + i * LEOAM_WAVE + lane;
            keys[i] = t < end ? key_at(t) : 0u;
        }
    }
    auto for_each = [&](auto&& f) {      // f(place, key, counts): by whole waves
        if (held) {
#pragma unroll
            for (int i = 0; i < kEvictHeld; ++i) {
                const int t0 = begin + i * LEOAM_WAVE;
                if (t0 < end) f(t0 + lane, keys[i], t0 + lane < end);
            }
        } else {
            for (int t0 = begin; t0 < end; t0 += LEOAM_WAVE) {
                const int t = t0 + lane;
                f(t, t < end ? key_at(t) : 0u, t < end);
            }
        }
    };

    // ---- protected ones, and the range of the others' keys ------------------------------------------------
    if (tid == 0) {
        sh_low = 0xffffffffu;
        sh_high = 0u;
        sh_protected = 0;
    }
    __syncthreads();
    {
        uint32_t low = 0xffffffffu, high = 0u;
        int count = 0;
        for_each([&](int, uint32_t k, bool in) {
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

    // ---- keys above `bound` stay, and `ties` of those equal to it --------------------------------------
    uint32_t bound = kProtected, low = sh_low, high = sh_high;
    int ties = keep, need = keep - sh_protected;      // (all of the protected ones or more than fit: the first of them)
    while (need > 0) {
        const uint32_t span = high - low;
        const int bits = 32 - __builtin_clz(span | 1u), shift = max(0, bits - 11);
        for (int i = tid; i < kEvictBins; i += kEvictThreads) hist[i] = 0;
        __syncthreads();
        for_each([&](int, uint32_t k, bool in) {
            if (in && k >= low && k <= high) atomicAdd(&hist[(k - low) >> shift], 1u);
        });
        __syncthreads();
        // bins from the top: thread i has bins 2047 - 2i and 2046 - 2i
        const uint32_t c0 = hist[kEvictBins - 1 - 2 * tid], c1 = hist[kEvictBins - 2 - 2 * tid];
        const uint32_t incl = wave_incl_scan_u32(c0 + c1);
        if (lane == LEOAM_WAVE - 1) sh_wave[wave] = (int)incl;
        __syncthreads();
        int before = (int)(incl - c0 - c1);
        for (int w = 0; w < wave; ++w) before += sh_wave[w];
        if (before < need && before + (int)(c0 + c1) >= need) {
            const bool upper = before + (int)c0 >= need;
            sh_bin = kEvictBins - 1 - 2 * tid - (upper ? 0 : 1);
            sh_above = before + (upper ? 0 : (int)c0);
            sh_in_bin = (int)(upper ? c0 : c1);
        }
        __syncthreads();
        need -= sh_above;
        low += (uint32_t)sh_bin << shift;
        high = min(high, low + ((1u << shift) - 1u));
        const int in_bin = sh_in_bin;
        if (need == in_bin) {      // the whole bin stays
            bound = low - 1u;      // (a key of 0: wraps round, see below)
            ties = 0;
            if (low == 0u) {
                bound = 0u;
                ties = need;
            }
            break;
        }
        if (shift == 0) {
            bound = low;
            ties = need;
            break;
        }
        __syncthreads();      // (the bin has been read)
    }

    // ---- how many stay before each wave's stretch, and before `keep` ---------------------------------------
    if (tid == 0) sh_kept_low[0] = sh_kept_low[1] = 0;
    __syncthreads();
    {
        int above = 0, equal = 0, above_low = 0, equal_low = 0;
        for_each([&](int t, uint32_t k, bool in) {
            const uint64_t ab = __ballot(in && k > bound), eq = __ballot(in && k == bound), lo = __ballot(t < keep);
            above += __popcll(ab);
            equal += __popcll(eq);
            above_low += __popcll(ab & lo);
            equal_low += __popcll(eq & lo);
        });
        if (lane == 0) {
            sh_wave[wave] = above;
            sh_tie[wave] = equal;
            atomicAdd(&sh_kept_low[0], above_low);
            atomicAdd(&sh_kept_low[1], equal_low);
        }
    }
    __syncthreads();
    int above = 0, equal = 0;      // before the place that the wave is at
    for (int w = 0; w < wave; ++w) {
        above += sh_wave[w];
        equal += sh_tie[w];
    }
    const int kept_low = sh_kept_low[0] + min(sh_kept_low[1], ties);
    if (tid == 0) a.move_count[bh] = keep - kept_low;
    int32_t* moves = a.moves + (size_t)bh * a.m_max * 2;
    const uint64_t below = (1ull << lane) - 1;
    for_each([&](int t, uint32_t k, bool in) {
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

size_t page_evict_workspace_bytes(const leoam_pages*) { return 16; }

hipError_t page_evict_dispatch(const leoam_pages* s, const float* weight, const int32_t* token_id, const int32_t* n_seen,
                               const int32_t* seq_len, const int32_t* keep_len, const int32_t* n_first, int n_recent, int32_t* moves,
                               int m_max, int32_t* move_count, int32_t* new_len, int32_t* status, void*, hipStream_t stream) {
    EvictArgs a;
    a.weight = weight; a.token_id = token_id; a.n_seen = n_seen; a.seq_len = seq_len; a.keep_len = keep_len; a.n_first = n_first;
    a.n_recent = n_recent; a.moves = moves; a.m_max = m_max; a.move_count = move_count; a.new_len = new_len; a.status = status;
    a.n_kv_heads = s->n_kv_heads; a.capacity = s->max_pages * s->page_size;
    hipLaunchKernelGGL(page_evict_kernel, dim3((unsigned)(s->batch * s->n_kv_heads)), dim3(kEvictThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace leoam
