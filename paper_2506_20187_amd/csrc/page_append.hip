// kv_page_append: new tokens' queries, keys and values, straight from the projection's output, with the position
// rotation applied on the way, into the pages of a pool.
//
// Rotation of channel pair (a, b) at a token's position: (a c - b s, b c + a s) with c, s from a table; every
// product and the sum is one binary32 operation (contraction is off there), then one
// rounding to the page's type: what a plain evaluation gives, bit for bit.  The position is the token's place in the sequence, or
// (kAt) what the caller gives for each row and axis.
//
// Bytes-bound (a row is read once and written once) for prompts, a chain of dependent round trips
// (length -> page -> old scale) for single tokens.  One workgroup owns a (touched page, kv head), of 8-bit prompts one of its
// tensors: the scale of an 8-bit page needs the largest magnitude over all that enters it, and the page's abstract row the
// maximum and minimum, so nobody else may touch them.
#include "page_common.h"

namespace leoam {

struct AppendArgs {
    const char *q, *k, *v;
    long long q_stride, k_stride, v_stride;      // bytes from one token's row to the next
    int n_new, n_slots;
    const int32_t *new_off, *seq_len, *page_table;
    const float* rope;
    char *q_out, *k_pages, *v_pages;
    float *k_scale, *v_scale;
    char* abstract;
    int32_t *chunk_off, *n_chunks, *status;
    int batch, n_q_heads, n_kv_heads, n_pages, page_size, max_pages, rot_dim, interleaved, rope_len;
    // positions that the caller gives (kAt): [n_axes][n_new], and the axis of each pair (nullptr: the first)
    const int32_t *position, *axis;
    int n_axes;
};

// what a sequence takes in: rows [row0, row0 + m) of the call become its tokens [n - m, n); status as reported
struct Taken { int row0, m, n, status; };

__device__ __forceinline__ Taken taken_by(const AppendArgs& a, int b) {
    const bool ragged = a.new_off != nullptr;
    const int n = a.seq_len[b], row0 = ragged ? a.new_off[b] : b, m = ragged ? a.new_off[b + 1] - row0 : n > 0 ? 1 : 0;
    const bool misfit = m < 0 || row0 < 0 || m > a.n_new - row0 || n < m || n > a.max_pages * a.page_size;
    return Taken{row0, m, n, misfit ? 1 : a.rot_dim && m && n > a.rope_len && !a.position ? 3 : 0};
}

// a row's position on an axis, as near to it as the table has one
__device__ __forceinline__ int position_of(const AppendArgs& a, int axis, int row) {
    return min(max(a.position[(size_t)axis * a.n_new + row], 0), a.rope_len - 1);
}

// The axes of the pairs that the EPL channels from `col` belong to, four bits each (kAt).  They are the lane's, whatever the row: looked
// up once, ahead of the rows' positions.
template <int EPL, bool kAt> struct Axes {
    uint32_t packed = 0;
    bool mixed = false;      // some lane of the wave has pairs of several axes
    __device__ __forceinline__ Axes(const AppendArgs& a, int col) {
        if constexpr (kAt) {
            if (!a.axis) return;
            constexpr int N = EPL / 2;
            const int half = a.rot_dim >> 1, at = a.interleaved ? col >> 1 : col < half ? col : col - half, more = a.interleaved ? 0 : N;
            if (col < a.rot_dim) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    packed |= (uint32_t)min(max(a.axis[at + e], 0), a.n_axes - 1) << 4 * e;
                    packed |= (uint32_t)min(max(a.axis[at + more + e], 0), a.n_axes - 1) << 4 * (e + N);
                }
            }
            constexpr uint32_t kAll = EPL == 8 ? 0x11111111u : 0x1111u;
            mixed = __ballot(packed != (packed & 15u) * kAll) != 0;
        }
    }
    // the row's position on the axis of the first of the pairs
    __device__ __forceinline__ int position(const AppendArgs& a, int row) const { return kAt ? position_of(a, packed & 15u, row) : 0; }
};

// The cosines and sines that the EPL channels from `col` need (channels from rot_dim on: none): those of place `pos`, or (kAt) of
// the positions that the call's row `row` was given, `pos` on the axis of the first pair.
template <int EPL, bool kAt> struct Turn {
    float c[EPL], s[EPL];
    __device__ __forceinline__ void load(const AppendArgs& a, int pos, int row, int col, const Axes<EPL, kAt>& axes) {
        if (col >= a.rot_dim) return;
        // pairs (2i, 2i+1): EPL / 2 angles from col / 2; pairs (i, i + half): EPL from col or col - half (half is a multiple of EPL)
        constexpr int N = EPL / 2;
        const int half = a.rot_dim >> 1, at = a.interleaved ? col >> 1 : col < half ? col : col - half, more = a.interleaved ? 0 : N;
        float c0[N], c1[N], s0[N], s1[N];
        auto of_position = [&](int p, float* c0, float* c1, float* s0, float* s1) {
            const float* angle = a.rope + (size_t)p * a.rot_dim + at;
            angles(angle, c0);
            angles(angle + more, c1);
            angles(angle + half, s0);
            angles(angle + half + more, s1);
        };
        of_position(pos, c0, c1, s0, s1);
        if (kAt && axes.mixed) {
            // The pieces of all axes, and each pair keeps its own.  (Where axes come in sections whose borders are multiples of EPL there
            // are no such pairs.)
            float k0[N], k1[N], t0[N], t1[N];
            for (int x = 0; x < a.n_axes; ++x) {
                of_position(position_of(a, x, row), k0, k1, t0, t1);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const bool first = (axes.packed >> 4 * e & 15u) == (uint32_t)x;
                    const bool second = (axes.packed >> 4 * (e + N) & 15u) == (uint32_t)x;
                    c0[e] = first ? k0[e] : c0[e];
                    s0[e] = first ? t0[e] : s0[e];
                    c1[e] = second ? k1[e] : c1[e];
                    s1[e] = second ? t1[e] : s1[e];
                }
            }
        }
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
            c[e] = a.interleaved ? c0[e / 2] : e < N ? c0[e % N] : c1[e % N];
            s[e] = a.interleaved ? s0[e / 2] : e < N ? s0[e % N] : s1[e % N];
        }
    }
    static __device__ __forceinline__ void angles(const float* p, float* x) {
        if constexpr (EPL == 8) {
            unpack<F32>(load16(p, 0), x);
        } else {
            const float2 v = *reinterpret_cast<const float2*>(p);
            x[0] = v.x;
            x[1] = v.y;
        }
    }
};

// x: this lane's EPL channels from `col` of a row that LPR neighbouring lanes hold (all of them are here)
template <int EPL, int LPR, bool kAt>
__device__ __forceinline__ void rotate(const AppendArgs& a, const Turn<EPL, kAt>& t, int col, float* x) {
#pragma clang fp contract(off)
    const int half = a.rot_dim >> 1;
    float other[EPL];
    if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < EPL; ++e) other[e] = x[e ^ 1];
    } else {
        const int lane = lane_id(), away = half / EPL;
        const int from = col < half ? lane + away : lane - away;
#pragma unroll
        for (int e = 0; e < EPL; ++e) other[e] = __shfl(x[e], col < a.rot_dim ? from : lane, LEOAM_WAVE);
    }
    if (col >= a.rot_dim) return;
    const bool first_half = col < half;
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
        const bool first = a.interleaved ? (e & 1) == 0 : first_half;
        const float own = x[e] * t.c[e], cross = other[e] * t.s[e];
        x[e] = first ? own - cross : own + cross;
    }
}

// maximum over the workgroup, in every lane
template <int THREADS> __device__ __forceinline__ float group_max(float v, float* sh) {
    v = wave_extreme_f<true>(v);
    if constexpr (THREADS == LEOAM_WAVE) return v;
    __syncthreads();
    if (lane_id() == 0) sh[threadIdx.x / LEOAM_WAVE] = v;
    __syncthreads();
    float m = sh[0];
#pragma unroll
    for (int w = 1; w < THREADS / LEOAM_WAVE; ++w) m = fmaxf(m, sh[w]);
    return m;
}

// Query rows: a token and 2 * (rows of a pass) of its heads.
template <typename T, int THREADS, bool kAt> __device__ __forceinline__ void append_queries(const AppendArgs& a, int unit) {
    constexpr int EPL = T::kEpl, LPR = Row<T>::kLanesPerRow, RPP = THREADS / LPR, ROWB = Row<T>::kRowBytes;
    const int tid = threadIdx.x, col = (tid % LPR) * EPL, rg = tid / LPR;
    const int per_token = (a.n_q_heads + 2 * RPP - 1) / (2 * RPP);
    const int row = unit / per_token, h0 = (unit % per_token) * 2 * RPP;
    const Axes<EPL, kAt> axes(a, col);
    const int given = axes.position(a, row);
    int b = row;
    if (a.new_off) b = wave_count_below(a.batch, row, [&](int i) { return a.new_off[i]; });
    if (b >= a.batch) return;
    const Taken t = taken_by(a, b);
    if (t.status || row < t.row0 || row >= t.row0 + t.m) return;
    Turn<EPL, kAt> turn;
    turn.load(a, kAt ? given : t.n - t.m + (row - t.row0), row, col, axes);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int h = h0 + i * RPP + rg, hc = min(h, a.n_q_heads - 1);
        float x[EPL];
        unpack<T>(load16(a.q, row * a.q_stride + (size_t)hc * ROWB + col * T::kBytes), x);
        rotate<EPL, LPR, kAt>(a, turn, col, x);
        if (h < a.n_q_heads) store16(a.q_out, ((size_t)row * a.n_q_heads + h) * ROWB + col * T::kBytes, round_pack<T>(x));
    }
}

template <typename T, int THREADS, bool kAt> __global__ __launch_bounds__(THREADS) void page_append_queries_kernel(AppendArgs a) {
    append_queries<T, THREADS, kAt>(a, blockIdx.x);
}

// A touched page of a sequence: logical page, the positions [p0, p1) that enter it, the row of the call that p0 is, how many
// tokens the page held, its number in the pool; count = 0: nothing to do.
struct TouchedPage { int b, p, p0, row0, held, count, id; };

// Slot of the first page that sequence i touches, in a ragged call (it touches at most m / ps + 2).
__device__ __forceinline__ int first_slot(const AppendArgs& a, int i) { return a.new_off[i] / a.page_size + 2 * i; }

// Whether the searches over new_off miss some of sequence b's pages or rows, as they may if it descends somewhere.  The number of
// sequences that begin at or before an element grows with the element: the first and the last speak for those between.
__device__ __forceinline__ bool misses(const AppendArgs& a, int b, const Taken& t) {
    const int ps = a.page_size, slot = first_slot(a, b);
    const int at[4] = {slot, slot + (t.n - 1) / ps - (t.n - t.m) / ps, t.row0, t.row0 + t.m - 1};
    int found[4] = {0, 0, 0, 0};
    bool more[4] = {true, true, true, true};
    for (int i0 = 1; i0 <= a.batch && (more[0] || more[1] || more[2] || more[3]); i0 += LEOAM_WAVE) {      // (as wave_count_below)
        const int i = i0 + lane_id(), row = a.new_off[min(i, a.batch)], s = row / ps + 2 * i;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint64_t hit = __ballot(i <= a.batch && (e < 2 ? s : row) <= at[e]);
            if (more[e]) found[e] += __popcll(hit);
            more[e] = more[e] && hit == ~0ull;
        }
    }
    return found[0] != b || found[1] != b || found[2] != b || found[3] != b;
}

// `slot` of the call's touched pages, by the whole workgroup
__device__ __forceinline__ TouchedPage touched_page(const AppendArgs& a, int slot, bool bounds) {
    const int tid = threadIdx.x, ps = a.page_size;
    TouchedPage x = {slot, 0, 0, 0, 0, 0, 0};
    int local = 0;
    if (a.new_off) {
        x.b = wave_count_below(a.batch, slot, [&](int i) { return first_slot(a, i); });
        if (x.b >= a.batch) return x;
        local = slot - first_slot(a, x.b);
    }
    const Taken t = taken_by(a, x.b);
    const bool none = t.status || t.m == 0;
    const int first = none ? 0 : (t.n - t.m) / ps, last = none ? -1 : (t.n - 1) / ps;
    x.p = first + local;
    if (local < 0 || x.p > last) return x;
    x.p0 = max(t.n - t.m, x.p * ps);
    const int p1 = min(t.n, (x.p + 1) * ps);
    if (bounds && tid == 0 && a.chunk_off) {
        int32_t* off = a.chunk_off + (size_t)x.b * (a.max_pages + 1);
        off[x.p + 1] = p1;
        if (x.p == 0) off[0] = 0;
    }
    x.id = a.page_table[(size_t)x.b * a.max_pages + x.p];
    if (x.id < 0 || x.id >= a.n_pages) return x;
    x.held = x.p0 - x.p * ps;
    x.count = p1 - x.p0;
    x.row0 = t.row0 + x.p0 - (t.n - t.m);
    return x;
}

template <int N> __device__ __forceinline__ void no_extremes(float* mx, float* mn) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
        mx[e] = -INFINITY;
        mn[e] = INFINITY;
    }
}

// The codes of a page whose scale grows by 1 / f, again; mx, mn (if wanted) take in the values that this thread's channels
// (col, of 16 threads to a row) then stand for.
template <int THREADS>
__device__ __forceinline__ void encode_again(char* page, int held, float f, float now, bool want, float* mx, float* mn) {
    for (int i = threadIdx.x; i < held * (LEOAM_D / 8); i += THREADS) {      // (THREADS is a multiple of a row's 16: same columns)
        uint2 w = *reinterpret_cast<uint2*>(page + 8 * (size_t)i);
        float y[8];
        unpack_e4m3(w.x, y);
        unpack_e4m3(w.y, y + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= f;      // (f < 1)
        w = make_uint2(pack_e4m3(y), pack_e4m3(y + 4));
        *reinterpret_cast<uint2*>(page + 8 * (size_t)i) = w;
        if (!want) continue;
        unpack_e4m3(w.x, y);
        unpack_e4m3(w.y, y + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            mx[e] = fmaxf(mx[e], y[e] * now);
            mn[e] = fminf(mn[e], y[e] * now);
        }
    }
}

// One token's channels of this lane into its page; mx, mn take in what is stored.  inv: 1 / scale, or 0 for a scale of 0 (8 bits).
// 448 * scale bounds what is stored before it is scaled, so that beside nothing but zeros infinities become 0 (infinity * 0 is NaN).
template <typename T, bool kStore8>
__device__ __forceinline__ void store_token(char* page, int slot, int col, const float* x, float scale, float inv, bool valid, float* mx,
                                            float* mn) {
    constexpr int EPL = T::kEpl;
    float y[EPL];
    if constexpr (kStore8) {
#pragma unroll
        for (int e = 0; e < EPL; ++e) y[e] = clamp_nan(x[e], 448.f * scale) * inv;
        const uint2 w = make_uint2(pack_e4m3(y), pack_e4m3(y + 4));
        if (valid) *reinterpret_cast<uint2*>(page + (size_t)slot * LEOAM_D + col) = w;
        unpack_e4m3(w.x, y);
        unpack_e4m3(w.y, y + 4);
#pragma unroll
        for (int e = 0; e < EPL; ++e) y[e] *= scale;
    } else {
        const uint4 w = round_pack<T>(x);
        if (valid) store16(page, (size_t)slot * Row<T>::kRowBytes + col * T::kBytes, w);
        unpack<T>(w, y);
    }
#pragma unroll
    for (int e = 0; e < EPL; ++e) {      // (a token that does not count repeats one that does)
        mx[e] = fmaxf(mx[e], y[e]);
        mn[e] = fminf(mn[e], y[e]);
    }
}

// mx, mn take in the keys that a page holds already, read from the page: what its abstract row says may be of tokens that were taken
// back since, or of whoever had this place in the batch before.  (us for a token each, row folded in : page read; one sequence, 8
// heads, pages of 64 in bf16 3.5 : 4.2; 96 sequences, pages of 32 in 8 bits 5.4 : 5.5, of 64 5.4 : 5.8, in bf16 4.0 : 4.7, and of 256, 25 MB,
// 4.0 : 9.4.  Sixteen loads on their way instead of eight: 8.8 for the last, 6.2 against 5.8 for pages of 32.)
template <typename T, bool kStore8, int THREADS, int BATCH>
__device__ __forceinline__ void take_in_held(const char* page, int held, float scale, int col, float* mx, float* mn) {
    constexpr int EPL = T::kEpl, LPR = Row<T>::kLanesPerRow, RPP = THREADS / LPR;
    constexpr int STOREB = kStore8 ? LEOAM_D : Row<T>::kRowBytes;
    const int rg = threadIdx.x % THREADS / LPR;
    for (int r0 = 0; r0 < held; r0 += RPP * BATCH) {
        uint4 raw[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {      // (rows past the last repeat it)
            const char* at = page + (size_t)min(r0 + u * RPP + rg, held - 1) * STOREB;
            if constexpr (kStore8) {
                const uint2 w = *reinterpret_cast<const uint2*>(at + col);
                raw[u] = make_uint4(w.x, w.y, 0, 0);
            } else {
                raw[u] = load16(at, col * T::kBytes);
            }
        }
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            float y[EPL];
            if constexpr (kStore8) {
                unpack_e4m3(raw[u].x, y);
                unpack_e4m3(raw[u].y, y + 4);
            } else {
                unpack<T>(raw[u], y);
            }
#pragma unroll
            for (int e = 0; e < EPL; ++e) {
                const float v = kStore8 ? y[e] * scale : y[e];
                mx[e] = fmaxf(mx[e], v);
                mn[e] = fminf(mn[e], v);
            }
        }
    }
}

// The page's maximum and minimum key, from the lanes' (lanes LPR apart hold the same channels) and the waves'.
template <typename T, int THREADS>
__device__ __forceinline__ void write_abstract(char* abs_row, int col, float* mx, float* mn, float (*sh)[2][LEOAM_D]) {
    constexpr int EPL = T::kEpl, LPR = Row<T>::kLanesPerRow, WAVES = THREADS / LEOAM_WAVE, ROWB = Row<T>::kRowBytes;
    const int tid = threadIdx.x % THREADS, lane = lane_id(), wave = tid / LEOAM_WAVE;
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
#pragma unroll
        for (int msk = LPR; msk < LEOAM_WAVE; msk <<= 1) {
            mx[e] = fmaxf(mx[e], shfl_xor_f(mx[e], msk));
            mn[e] = fminf(mn[e], shfl_xor_f(mn[e], msk));
        }
    }
    if constexpr (WAVES > 1) {
        __syncthreads();
        if (lane < LPR) {
#pragma unroll
            for (int e = 0; e < EPL; ++e) {
                sh[wave][0][col + e] = mx[e];
                sh[wave][1][col + e] = mn[e];
            }
        }
        __syncthreads();
        if (tid < LPR) {
#pragma unroll
            for (int w = 1; w < WAVES; ++w)
#pragma unroll
                for (int e = 0; e < EPL; ++e) {
                    mx[e] = fmaxf(mx[e], sh[w][0][col + e]);
                    mn[e] = fminf(mn[e], sh[w][1][col + e]);
                }
        }
    }
    if (tid >= LPR) return;
    store16(abs_row, col * T::kBytes, round_pack<T>(mx));
    store16(abs_row, ROWB + col * T::kBytes, round_pack<T>(mn));
}

__device__ __forceinline__ char* abstract_row(const AppendArgs& a, int b, int p, int h, int row_bytes) {
    return a.abstract + (((size_t)b * a.n_kv_heads + h) * a.max_pages + p) * 2 * row_bytes;
}

// What became of sequence b, and its full pages from `n_chunks` to the first that takes a token - others filled them, or nobody
// had rows for them - in the abstract and the boundaries.  One workgroup, since it alone reads and sets n_chunks; once for a
// sequence and its prefix, so it need not be fast: a wave takes a (page, kv head) at a time (4096 tokens of 8 heads in bf16, pages of 64:
// 0.3 ms in a prompt's call, 0.85 in a single token's; 64K 5 ms).
template <typename T, bool kStore8, int THREADS, bool kAt>
__device__ __forceinline__ void report(const AppendArgs& a, int b, float* sh_max) {
    constexpr int EPL = T::kEpl, LPR = Row<T>::kLanesPerRow, ROWB = Row<T>::kRowBytes, STOREB = kStore8 ? LEOAM_D : ROWB;
    const int tid = threadIdx.x, ps = a.page_size, hkv = a.n_kv_heads;
    const int32_t* table = a.page_table + (size_t)b * a.max_pages;
    const int known = a.n_chunks ? max(a.n_chunks[b], 0) : a.max_pages;
    Taken t = taken_by(a, b);
    if (t.status == 0 && a.new_off && t.m > 0 && misses(a, b, t)) t.status = 1;
    const bool none = t.status || t.m == 0;
    const int first = none ? 0 : (t.n - t.m) / ps, last = none ? -1 : (t.n - 1) / ps;
    int bad = 0;
    for (int p = first + tid; p <= last; p += THREADS) bad |= (uint32_t)table[p] >= (uint32_t)a.n_pages;
    if constexpr (kAt) {      // 1: a position that the table does not have, 2: a page that the pool does not have
        bad <<= 1;
        if (a.status && a.rot_dim && !none)
            for (int x = 0; x < a.n_axes; ++x) {
                const int32_t* position = a.position + (size_t)x * a.n_new + t.row0;
                for (int r = tid; r < t.m; r += THREADS) bad = max(bad, (uint32_t)position[r] >= (uint32_t)a.rope_len ? 1 : 0);
            }
    }
    bad = (int)(group_max<THREADS>((float)bad, sh_max));      // (everybody has n_chunks)
    if (tid == 0) {
        if (a.status) a.status[b] = t.status ? t.status : kAt && bad == 1 ? 3 : bad ? 2 : 0;
        if (a.n_chunks && (!none || (t.status == 0 && t.n == 0))) a.n_chunks[b] = last + 1;
    }
    if (known >= first) return;
    if (a.chunk_off) {
        int32_t* off = a.chunk_off + (size_t)b * (a.max_pages + 1);
        for (int p = known + tid; p < first; p += THREADS) off[p + 1] = (p + 1) * ps;
        if (known == 0 && tid == 0) off[0] = 0;
    }
    if (!a.abstract) return;
    const int lane = lane_id(), col = (lane % LPR) * EPL;
    for (long long i = tid / LEOAM_WAVE; i < (long long)(first - known) * hkv; i += THREADS / LEOAM_WAVE) {
        const int p = known + (int)(i / hkv), h = (int)(i % hkv), id = table[p];
        if ((uint32_t)id >= (uint32_t)a.n_pages) continue;
        const size_t at = (size_t)id * hkv + h;
        float mx[EPL], mn[EPL];
        no_extremes<EPL>(mx, mn);
        take_in_held<T, kStore8, LEOAM_WAVE, THREADS == LEOAM_WAVE ? 8 : 4>(a.k_pages + at * ps * STOREB, ps, kStore8 ? a.k_scale[at] : 1.f, col, mx, mn);
        write_abstract<T, LEOAM_WAVE>(abstract_row(a, b, p, h, ROWB), col, mx, mn, nullptr);
    }
}

// Prompts: a touched page and a kv head to a workgroup, behind one for each sequence that reports on it.
//   16 / 32 bits (PASSES = 0): keys, then values, a pass of THREADS / lanes-per-row rows at a time; further workgroups take the
//     queries.  9K tokens of 32 + 64 heads in fp16: 96 us, 4.6 TB/s (a large copy: 4.7).
//   8 bits: the scale comes before the codes, so the page's new rows stay in registers, PASSES passes of them; keys and
//     values are workgroups of their own, and so are the queries in a launch of their own.  16K tokens of 32 + 16 heads: 93 us
//     against 134 with the former's shape (the queries at a quarter of the occupancy).
// Workgroups of four heads, which would load the angles of a token once for them, were slower (144 against 93 us for the
// keys and values of the former, 78 against 58 for the latter): a page then takes longer than there are pages to overlap.
// Positions of the caller's: three prompts of 4097 of 5001 tokens, 32 / 8 heads, fp16 (285 MB), waves for each SIMD 4, 5, 6, 7: three axes
// in sections 94, 84, 83, 79 us, by turns 114, 105, 111, 116, one axis 82, 74, 73, 73 (63 without positions).
template <typename T, bool kStore8, int THREADS, int PASSES, bool kAt>
__global__ __launch_bounds__(THREADS, kAt && !kStore8 ? 5 : 1) void page_append_prompt_kernel(AppendArgs a) {
    constexpr int EPL = T::kEpl, LPR = Row<T>::kLanesPerRow, RPP = THREADS / LPR, WAVES = THREADS / LEOAM_WAVE;
    constexpr int ROWB = Row<T>::kRowBytes, STOREB = kStore8 ? LEOAM_D : ROWB;
    __shared__ float sh_max[WAVES];
    __shared__ float sh_abs[WAVES][2][LEOAM_D];
    const int tid = threadIdx.x, col = (tid % LPR) * EPL, rg = tid / LPR, ps = a.page_size, hkv = a.n_kv_heads;
    if ((int)blockIdx.x < a.batch) {
        report<T, kStore8, THREADS, kAt>(a, blockIdx.x, sh_max);
        return;
    }
    int unit = blockIdx.x - a.batch, first = 0, last = 1;      // tensors
    if constexpr (kStore8) {
        first = last = unit & 1;
        unit >>= 1;
    } else if (unit >= a.n_slots * hkv) {
        append_queries<T, THREADS, kAt>(a, unit - a.n_slots * hkv);
        return;
    }
    const int h = unit % hkv;
    const Axes<EPL, kAt> axes(a, col);
    const TouchedPage x = touched_page(a, unit / hkv, h == 0 && first == 0);
    if (x.count == 0) return;
    const size_t at = (size_t)x.id * hkv + h;
#pragma unroll kStore8 ? 1 : 2
    for (int which = first; which <= last; ++which) {
        const char* src = (which ? a.v : a.k) + (size_t)h * ROWB + col * T::kBytes;
        const long long stride = which ? a.v_stride : a.k_stride;
        char* page = (which ? a.v_pages : a.k_pages) + at * ps * STOREB;
        const bool turned = which == 0 && a.rot_dim > 0, bounded = which == 0 && a.abstract;
        float mx[EPL], mn[EPL];
        no_extremes<EPL>(mx, mn);
        // (rows past the last repeat it: rotation exchanges lanes, so all of them are here)
        auto row_of = [&](int r) { return load16(src, (x.row0 + min(r, x.count - 1)) * stride); };
        auto given = [&](int r) { return axes.position(a, x.row0 + min(r, x.count - 1)); };
        auto turn_row = [&](int r, int pos, float* y) {
            if (!turned) return;
            Turn<EPL, kAt> turn;
            turn.load(a, kAt ? pos : x.p0 + min(r, x.count - 1), x.row0 + min(r, x.count - 1), col, axes);
            rotate<EPL, LPR, kAt>(a, turn, col, y);
        };
        if constexpr (!kStore8) {
            if (bounded) take_in_held<T, false, THREADS, 4>(page, x.held, 1.f, col, mx, mn);
            int pos = kAt && turned ? given(rg) : 0;
            for (int r = rg; r < x.count + rg; r += RPP) {      // (uniform trip count)
                float y[EPL];
                const uint4 raw = row_of(r);
                const int next = kAt && turned ? given(r + RPP) : 0;      // (a row ahead of the angles that it leads to)
                unpack<T>(raw, y);
                turn_row(r, pos, y);
                pos = next;
                store_token<T, false>(page, x.held + min(r, x.count - 1), col, y, 1.f, 1.f, r < x.count, mx, mn);
            }
        } else {
            uint4 raw[PASSES];
            float y[PASSES][EPL], top = 0.f;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) raw[i] = row_of(i * RPP + rg);
            int pos = kAt && turned ? given(rg) : 0;
            float* scales = which ? a.v_scale : a.k_scale;
            const float old = x.held > 0 ? scales[at] : 0.f;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                unpack<T>(raw[i], y[i]);
                const int next = kAt && turned && i + 1 < PASSES ? given((i + 1) * RPP + rg) : 0;
                turn_row(i * RPP + rg, pos, y[i]);
                pos = next;
#pragma unroll
                for (int e = 0; e < EPL; ++e) {
                    const float m = fabsf(y[i][e]);
                    top = fmaxf(top, m < INFINITY ? m : 0.f);
                }
            }
            const float now = fmaxf(old, scale_of<T>(group_max<THREADS>(top, sh_max)));      // (everybody has the old scale)
            const float inv = now > 0.f ? 1.f / now : 0.f;                                   // a power of two: exact
            const bool grows = x.held > 0 && now > old;
            if (grows) encode_again<THREADS>(page, x.held, old * inv, now, bounded, mx, mn);
            if (tid == 0) scales[at] = now;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int r = i * RPP + rg;
                store_token<T, true>(page, x.held + min(r, x.count - 1), col, y[i], now, inv, r < x.count, mx, mn);
            }
            if (bounded && !grows) take_in_held<T, true, THREADS, 4>(page, x.held, now, col, mx, mn);      // (the rows' registers are free)
        }
        if (bounded) write_abstract<T, THREADS>(abstract_row(a, x.b, x.p, h, ROWB), col, mx, mn, sh_abs);
    }
}

// One token for each sequence: a wave to a (sequence, kv head), lanes of the first row's width hold the key and the value; further
// waves report (in the first of these, before its own work, that took 0.25 us longer) and take the queries.
template <typename T, bool kStore8, bool kAt> __global__ __launch_bounds__(LEOAM_WAVE) void page_append_token_kernel(AppendArgs a) {
    constexpr int EPL = T::kEpl, LPR = Row<T>::kLanesPerRow, ROWB = Row<T>::kRowBytes, STOREB = kStore8 ? LEOAM_D : ROWB;
    constexpr int THREADS = LEOAM_WAVE;
    const int hkv = a.n_kv_heads, ps = a.page_size, tid = threadIdx.x, col = (tid % LPR) * EPL;
    if ((int)blockIdx.x < a.batch) {
        report<T, kStore8, THREADS, kAt>(a, blockIdx.x, nullptr);
        return;
    }
    const int unit = blockIdx.x - a.batch;
    if (unit >= a.n_slots * hkv) {
        append_queries<T, THREADS, kAt>(a, unit - a.n_slots * hkv);
        return;
    }
    const int h = unit % hkv;
    const Axes<EPL, kAt> axes(a, col);
    const int given = kAt && a.rot_dim ? axes.position(a, unit / hkv) : 0;      // (a token each: its row is its sequence's)
    const TouchedPage x = touched_page(a, unit / hkv, h == 0);
    if (x.count == 0) return;
    const uint4 raw[2] = {load16(a.k, x.row0 * a.k_stride + (size_t)h * ROWB + col * T::kBytes),
                          load16(a.v, x.row0 * a.v_stride + (size_t)h * ROWB + col * T::kBytes)};
    Turn<EPL, kAt> turn;
    if (a.rot_dim) turn.load(a, kAt ? given : x.p0, x.row0, col, axes);
    const size_t at = (size_t)x.id * hkv + h;
    float old[2] = {0.f, 0.f};
    if (kStore8 && x.held > 0) {
        old[0] = a.k_scale[at];
        old[1] = a.v_scale[at];
    }
    float held_mx[EPL], held_mn[EPL];      // (read before anybody knows whether the scale grows: one round trip less)
    no_extremes<EPL>(held_mx, held_mn);
    if (a.abstract) take_in_held<T, kStore8, THREADS, 8>(a.k_pages + at * ps * STOREB, x.held, old[0], col, held_mx, held_mn);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        char* page = (which ? a.v_pages : a.k_pages) + at * ps * STOREB;
        const bool bounded = which == 0 && a.abstract;
        float y[EPL], mx[EPL], mn[EPL], scale = 1.f, inv = 1.f;
        unpack<T>(raw[which], y);
        if (which == 0 && a.rot_dim) rotate<EPL, LPR, kAt>(a, turn, col, y);
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
            mx[e] = held_mx[e];
            mn[e] = held_mn[e];
        }
        if constexpr (kStore8) {
            float top = 0.f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) {
                const float m = fabsf(y[e]);
                top = fmaxf(top, m < INFINITY ? m : 0.f);
            }
            scale = fmaxf(old[which], scale_of<T>(group_max<THREADS>(top, nullptr)));
            inv = scale > 0.f ? 1.f / scale : 0.f;
            if (x.held > 0 && scale > old[which]) {
                no_extremes<EPL>(mx, mn);
                encode_again<THREADS>(page, x.held, old[which] * inv, scale, bounded, mx, mn);
            }
            if (tid == 0) (which ? a.v_scale : a.k_scale)[at] = scale;
        }
        store_token<T, kStore8>(page, x.held, col, y, scale, inv, tid < LPR, mx, mn);
        if (bounded) write_abstract<T, THREADS>(abstract_row(a, x.b, x.p, h, ROWB), col, mx, mn, nullptr);
    }
}

template <typename T> constexpr int queries_per_unit(int threads) { return 2 * (threads / Row<T>::kLanesPerRow); }

template <typename T, bool kStore8, bool kAt> static hipError_t launch_tokens(const AppendArgs& a, hipStream_t stream) {
    const int per = queries_per_unit<T>(LEOAM_WAVE);
    const long long q_units = a.q ? (long long)a.n_new * ((a.n_q_heads + per - 1) / per) : 0;
    const long long units = a.batch + (long long)a.n_slots * a.n_kv_heads + q_units;
    if (units > 0x7fffffffll) return hipErrorInvalidValue;
    hipLaunchKernelGGL((page_append_token_kernel<T, kStore8, kAt>), dim3((unsigned)units), dim3(LEOAM_WAVE), 0, stream, a);
    return hipGetLastError();
}

constexpr int kPromptThreads = 256;
template <typename T, bool kStore8, int PASSES, bool kAt> static hipError_t launch_prompt(const AppendArgs& a, hipStream_t stream) {
    const int per = queries_per_unit<T>(kPromptThreads);
    const long long q_units = a.q ? (long long)a.n_new * ((a.n_q_heads + per - 1) / per) : 0, kv_units = (long long)a.n_slots * a.n_kv_heads;
    const long long units = a.batch + (kStore8 ? 2 * kv_units : kv_units + q_units);
    if (units > 0x7fffffffll || q_units > 0x7fffffffll) return hipErrorInvalidValue;
    hipLaunchKernelGGL((page_append_prompt_kernel<T, kStore8, kPromptThreads, PASSES, kAt>), dim3((unsigned)units), dim3(kPromptThreads), 0,
                       stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !kStore8 || q_units == 0) return e;
    hipLaunchKernelGGL((page_append_queries_kernel<T, kPromptThreads, kAt>), dim3((unsigned)q_units), dim3(kPromptThreads), 0, stream, a);
    return hipGetLastError();
}

template <typename T, bool kAt> static hipError_t append_of(const AppendArgs& a, bool store8, bool single, hipStream_t stream) {
    if constexpr (T::kTag != LEOAM_F32) {
        if (store8) {
            if (single) return launch_tokens<T, true, kAt>(a, stream);
            switch (a.page_size) {
            case 16: return launch_prompt<T, true, 1, kAt>(a, stream);
            case 32: return launch_prompt<T, true, 2, kAt>(a, stream);
            case 64: return launch_prompt<T, true, 4, kAt>(a, stream);
            case 128: return launch_prompt<T, true, 8, kAt>(a, stream);
            default: return launch_prompt<T, true, 16, kAt>(a, stream);
            }
        }
    }
    return single ? launch_tokens<T, false, kAt>(a, stream) : launch_prompt<T, false, 0, kAt>(a, stream);
}

hipError_t page_append_dispatch(const leoam_pages* s, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                const void* v, int64_t v_stride, int n_new, const int32_t* new_off, const int32_t* seq_len,
                                const int32_t* page_table, const float* rope, const int32_t* position, int n_axes,
                                const int32_t* axis, void* q_out, void* k_pages, void* v_pages, float* k_scale, float* v_scale,
                                void* abstract, int32_t* chunk_off, int32_t* n_chunks, int32_t* status, hipStream_t stream) {
    const int e = s->q_dtype == LEOAM_F32 ? 4 : 2;
    AppendArgs a;
    a.q = (const char*)q; a.k = (const char*)k; a.v = (const char*)v;
    a.q_stride = q_stride * e; a.k_stride = k_stride * e; a.v_stride = v_stride * e;
    a.n_new = n_new;
    a.n_slots = new_off ? n_new / s->page_size + 2 * s->batch : s->batch;
    a.new_off = new_off; a.seq_len = seq_len; a.page_table = page_table; a.rope = rope;
    a.q_out = (char*)q_out; a.k_pages = (char*)k_pages; a.v_pages = (char*)v_pages;
    a.k_scale = k_scale; a.v_scale = v_scale; a.abstract = (char*)abstract;
    a.chunk_off = chunk_off; a.n_chunks = n_chunks; a.status = status;
    a.batch = s->batch; a.n_q_heads = s->n_q_heads; a.n_kv_heads = s->n_kv_heads; a.n_pages = s->n_pages;
    a.page_size = s->page_size; a.max_pages = s->max_pages; a.rot_dim = s->rot_dim; a.interleaved = s->rope_interleaved;
    a.rope_len = s->rope_len;
    a.position = position; a.n_axes = n_axes; a.axis = n_axes > 1 ? axis : nullptr;
    const bool store8 = s->kv_dtype == LEOAM_E4M3, single = new_off == nullptr;
    switch (s->q_dtype) {
    case LEOAM_F32: return position ? append_of<F32, true>(a, store8, single, stream) : append_of<F32, false>(a, store8, single, stream);
    case LEOAM_F16: return position ? append_of<F16, true>(a, store8, single, stream) : append_of<F16, false>(a, store8, single, stream);
    default: return position ? append_of<BF16, true>(a, store8, single, stream) : append_of<BF16, false>(a, store8, single, stream);
    }
}

}  // namespace leoam
