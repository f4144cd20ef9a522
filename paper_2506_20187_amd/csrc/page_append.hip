// kv_page_append: new tokens' queries, keys and values, straight from the projection's output, with the position
// rotation applied on the way, into the pages of a pool.
//
// Rotation of channel pair (a, b) at a token's position: (a c - b s, b c + a s) with c, s from a table; every
// product and the sum is one binary32 operation (contraction is off there), then one
// rounding to the page's type: what a plain evaluation gives, bit for bit.
//
// Bytes-bound (a row is read once and written once) for prompts, a chain of dependent round trips
// (length -> page -> old scale) for single tokens.  A workgroup owns one (touched page, kv head): the scale of
// an 8-bit page needs the largest magnitude over all that enters it, and the page's abstract row the maximum and
// minimum, so nobody else may touch them.  Further workgroups rotate the queries.  A prompt's page takes 256
// threads, a single token 64.
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
};

// what a sequence takes in: rows [row0, row0 + m) of the call become its tokens [n - m, n); status as reported
struct Taken { int row0, m, n, status; };

__device__ __forceinline__ Taken taken_by(const AppendArgs& a, int b) {
    Taken t;
    t.n = a.seq_len[b];
    if (a.new_off) {
        t.row0 = a.new_off[b];
        t.m = a.new_off[b + 1] - t.row0;
    } else {
        t.row0 = b;
        t.m = t.n > 0 ? 1 : 0;
    }
    t.status = 0;
    if (t.m < 0 || t.row0 < 0 || t.m > a.n_new - t.row0 || t.n < t.m || t.n > a.max_pages * a.page_size) t.status = 1;
    else if (a.rot_dim && t.m && t.n > a.rope_len) t.status = 3;
    return t;
}

// The cosines and sines that the EPL channels from `col` need, 0-channel pairs beyond rot_dim left alone.
template <int EPL> struct Turn {
    float c[EPL], s[EPL];
    __device__ __forceinline__ void load(const AppendArgs& a, int pos, int col) {
        if (col >= a.rot_dim) return;
        const int half = a.rot_dim >> 1;
        const float* row = a.rope + (size_t)pos * a.rot_dim;
        if (a.interleaved) {      // pairs (2i, 2i+1)
#pragma unroll
            for (int e = 0; e < EPL; e += 2) {
                c[e] = c[e + 1] = row[(col + e) >> 1];
                s[e] = s[e + 1] = row[half + ((col + e) >> 1)];
            }
        } else {                  // pairs (i, i + half); half is a multiple of EPL
            const float* p = row + (col < half ? col : col - half);
#pragma unroll
            for (int e = 0; e < EPL; e += 4) {
                const uint4 cc = load16(p, 4 * e), ss = load16(p + half, 4 * e);
                unpack<F32>(cc, c + e);
                unpack<F32>(ss, s + e);
            }
        }
    }
};

// x: this lane's EPL channels from `col` of a row that LPR neighbouring lanes hold (all of them are here)
template <int EPL, int LPR>
__device__ __forceinline__ void rotate(const AppendArgs& a, const Turn<EPL>& t, int col, float* x) {
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

// the smallest power of two s with amax <= 448 s, as a float; its exponent stays where s * code is a number of T
template <typename T> __device__ __forceinline__ float scale_of(float amax) {
    if (!(amax > 0.f)) return 0.f;
    constexpr int kLow = T::kTag == LEOAM_F16 ? -15 : -100, kHigh = T::kTag == LEOAM_F16 ? 7 : 118;
    const uint32_t u = float_to_bits(amax);
    // amax = 1.f * 2^e, 448 = 1.75 * 2^8   (a subnormal amax is below the smallest exponent anyway)
    int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = min(max(e, kLow), kHigh);
    return bits_to_float((uint32_t)(e + 127) << 23);
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

// ROWS passes of THREADS / lanes-per-row tokens each
template <typename T, bool kStore8, int THREADS, int PASSES>
__global__ __launch_bounds__(THREADS) void page_append_kernel(AppendArgs a) {
    constexpr int EPL = T::kEpl, LPR = Row<T>::kLanesPerRow, RPP = THREADS / LPR, WAVES = THREADS / LEOAM_WAVE;
    constexpr int ROWB = Row<T>::kRowBytes, STOREB = kStore8 ? LEOAM_D : ROWB;
    __shared__ float sh_max[WAVES];
    __shared__ float sh_abs[WAVES][2][LEOAM_D];
    const int tid = threadIdx.x, lane = lane_id(), wave = tid / LEOAM_WAVE;
    const int col = (tid % LPR) * EPL, rg = tid / LPR;
    const int B = a.batch, ps = a.page_size;

    const int n_kv_units = a.n_slots * a.n_kv_heads;
    if ((int)blockIdx.x >= n_kv_units) {
        // ---- queries: a token and 2 * RPP of its heads --------------------------------------------------
        const int per_token = (a.n_q_heads + 2 * RPP - 1) / (2 * RPP);
        const int u = blockIdx.x - n_kv_units, row = u / per_token, h0 = (u % per_token) * 2 * RPP;
        int b = row;
        if (a.new_off) b = wave_count_below(B, row, [&](int i) { return a.new_off[i]; });
        if (b >= B) return;
        const Taken t = taken_by(a, b);
        if (t.status || row < t.row0 || row >= t.row0 + t.m) return;
        Turn<EPL> turn;
        turn.load(a, t.n - t.m + (row - t.row0), col);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int h = h0 + i * RPP + rg, hc = min(h, a.n_q_heads - 1);
            float x[EPL];
            unpack<T>(load16(a.q, row * a.q_stride + (size_t)hc * ROWB + col * T::kBytes), x);
            rotate<EPL, LPR>(a, turn, col, x);
            if (h < a.n_q_heads) store16(a.q_out, ((size_t)row * a.n_q_heads + h) * ROWB + col * T::kBytes, round_pack<T>(x));
        }
        return;
    }

    // ---- a touched page of a sequence, one kv head ------------------------------------------------------------
    const int h = blockIdx.x % a.n_kv_heads, slot = blockIdx.x / a.n_kv_heads;
    int b = slot, local = 0;
    if (a.new_off) {
        // sequence i's pages begin at slot new_off[i] / ps + 2 i: it touches at most m / ps + 2
        b = wave_count_below(B, slot, [&](int i) { return a.new_off[i] / ps + 2 * i; });
        if (b >= B) return;
        local = slot - (a.new_off[b] / ps + 2 * b);
    }
    const Taken t = taken_by(a, b);
    const int first = t.status || t.m == 0 ? 0 : (t.n - t.m) / ps, last = t.status || t.m == 0 ? -1 : (t.n - 1) / ps;
    if (local == 0 && h == 0) {
        int bad = 0;
        for (int p = first + tid; p <= last; p += THREADS) {
            const int id = a.page_table[(size_t)b * a.max_pages + p];
            bad |= id < 0 || id >= a.n_pages;
        }
        bad = (int)(group_max<THREADS>((float)bad, sh_max));
        if (tid == 0) {
            if (a.status) a.status[b] = t.status ? t.status : bad ? 2 : 0;
            if (a.n_chunks && !t.status && t.m) a.n_chunks[b] = (t.n + ps - 1) / ps;
        }
    }
    const int p = first + local;
    if (local < 0 || p > last) return;
    const int p0 = max(t.n - t.m, p * ps), p1 = min(t.n, (p + 1) * ps);      // positions that enter this page
    if (h == 0 && tid == 0 && a.chunk_off) {
        int32_t* off = a.chunk_off + (size_t)b * (a.max_pages + 1);
        off[p + 1] = p1;
        if (p == 0) off[0] = 0;
    }
    const int id = a.page_table[(size_t)b * a.max_pages + p];
    if (id < 0 || id >= a.n_pages) return;
    const int held = p0 - p * ps, count = p1 - p0;
    const int row0 = t.row0 + p0 - (t.n - t.m);
    const size_t at = ((size_t)id * a.n_kv_heads + h), base = at * ps * STOREB;
    char* abs_row = a.abstract ? a.abstract + (((size_t)b * a.n_kv_heads + h) * a.max_pages + p) * 2 * ROWB : nullptr;
    // (model type: a lane stores 16 bytes of a row; 8 bits: the 8 codes of its channels)

#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const char* src = which ? a.v + (size_t)h * ROWB : a.k + (size_t)h * ROWB;
        const long long stride = which ? a.v_stride : a.k_stride;
        char* page = (which ? a.v_pages : a.k_pages) + base;
        float mx[EPL], mn[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
            mx[e] = -INFINITY;
            mn[e] = INFINITY;
        }
        bool begun = held > 0;      // the abstract row counts
        auto fetch = [&](int r, float* x) {
            const int rc = min(r, count - 1);
            unpack<T>(load16(src, (row0 + rc) * stride + col * T::kBytes), x);
            if (which == 0 && a.rot_dim) {
                Turn<EPL> turn;
                turn.load(a, p0 + rc, col);
                rotate<EPL, LPR>(a, turn, col, x);
            }
        };
        if constexpr (!kStore8) {
            for (int r = rg; r < count + rg; r += RPP) {      // (uniform trip count: rotation exchanges lanes)
                float x[EPL];
                fetch(r, x);
                const uint4 w = round_pack<T>(x);
                unpack<T>(w, x);
#pragma unroll
                for (int e = 0; e < EPL; ++e) {
                    mx[e] = fmaxf(mx[e], x[e]);
                    mn[e] = fminf(mn[e], x[e]);
                }
                if (r < count) store16(page, (size_t)(held + r) * ROWB + col * T::kBytes, w);
            }
        } else {
            float x[PASSES][EPL], top = 0.f;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                fetch(i * RPP + rg, x[i]);
#pragma unroll
                for (int e = 0; e < EPL; ++e) {
                    const float m = fabsf(x[i][e]);
                    top = fmaxf(top, m < INFINITY ? m : 0.f);
                }
            }
            top = group_max<THREADS>(top, sh_max);
            float* scales = which ? a.v_scale : a.k_scale;
            const float old = held > 0 ? scales[at] : 0.f;
            const float now = fmaxf(old, scale_of<T>(top));
            const float inv = now > 0.f ? 1.f / now : 0.f;      // a power of two: exact
            if (held > 0 && now > old) {
                // the page's scale grew: its codes again, in the new scale
                const float f = old * inv;
                for (int i = tid; i < held * (LEOAM_D / 8); i += THREADS) {
                    uint2 w = *reinterpret_cast<uint2*>(page + 8 * (size_t)i);
                    float y[8];
                    unpack_e4m3(w.x, y);
                    unpack_e4m3(w.y, y + 4);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        y[e] *= f;
                    }
                    w = make_uint2(pack_e4m3(y), pack_e4m3(y + 4));
                    *reinterpret_cast<uint2*>(page + 8 * (size_t)i) = w;
                    if (which == 0 && abs_row) {      // (THREADS is a multiple of a row's 16 lanes: same columns)
                        unpack_e4m3(w.x, y);
                        unpack_e4m3(w.y, y + 4);
#pragma unroll
                        for (int e = 0; e < EPL; ++e) {
                            mx[e] = fmaxf(mx[e], y[e] * now);
                            mn[e] = fminf(mn[e], y[e] * now);
                        }
                    }
                }
                begun = false;
            }
            __syncthreads();      // everybody has the old scale
            if (tid == 0) scales[at] = now;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int r = i * RPP + rg;
                if (r >= count) continue;
                float y[EPL];
#pragma unroll
                for (int e = 0; e < EPL; ++e) y[e] = x[i][e] * inv;
                const uint2 w = make_uint2(pack_e4m3(y), pack_e4m3(y + 4));
                *reinterpret_cast<uint2*>(page + (size_t)(held + r) * LEOAM_D + col) = w;
                unpack_e4m3(w.x, y);
                unpack_e4m3(w.y, y + 4);
#pragma unroll
                for (int e = 0; e < EPL; ++e) {
                    mx[e] = fmaxf(mx[e], y[e] * now);
                    mn[e] = fminf(mn[e], y[e] * now);
                }
            }
        }
        if (which == 1 || !abs_row) continue;
        // the page's maximum and minimum key: row groups of the wave, then the waves, then what the row held
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
                    sh_abs[wave][0][col + e] = mx[e];
                    sh_abs[wave][1][col + e] = mn[e];
                }
            }
            __syncthreads();
            if (tid < LPR) {
#pragma unroll
                for (int w = 1; w < WAVES; ++w)
#pragma unroll
                    for (int e = 0; e < EPL; ++e) {
                        mx[e] = fmaxf(mx[e], sh_abs[w][0][col + e]);
                        mn[e] = fminf(mn[e], sh_abs[w][1][col + e]);
                    }
            }
        }
        if (tid < LPR) {
            if (begun) {
                float y[EPL];
                unpack<T>(load16(abs_row, col * T::kBytes), y);
#pragma unroll
                for (int e = 0; e < EPL; ++e) mx[e] = fmaxf(mx[e], y[e]);
                unpack<T>(load16(abs_row, ROWB + col * T::kBytes), y);
#pragma unroll
                for (int e = 0; e < EPL; ++e) mn[e] = fminf(mn[e], y[e]);
            }
            store16(abs_row, col * T::kBytes, round_pack<T>(mx));
            store16(abs_row, ROWB + col * T::kBytes, round_pack<T>(mn));
        }
    }
}

template <typename T, bool kStore8, int THREADS, int PASSES>
static hipError_t launch_append(const AppendArgs& a, hipStream_t stream) {
    constexpr int RPP = THREADS / Row<T>::kLanesPerRow;
    const long long q_units = a.q ? (long long)a.n_new * ((a.n_q_heads + 2 * RPP - 1) / (2 * RPP)) : 0;
    const long long units = (long long)a.n_slots * a.n_kv_heads + q_units;
    if (units > 0x7fffffffll) return hipErrorInvalidValue;
    hipLaunchKernelGGL((page_append_kernel<T, kStore8, THREADS, PASSES>), dim3((unsigned)units), dim3(THREADS), 0, stream, a);
    return hipGetLastError();
}

template <typename T> static hipError_t append_of(const AppendArgs& a, bool store8, bool single, hipStream_t stream) {
    if constexpr (T::kTag != LEOAM_F32) {
        if (store8) {
            if (single) return launch_append<T, true, LEOAM_WAVE, 1>(a, stream);
            switch (a.page_size) {
            case 16: return launch_append<T, true, 256, 1>(a, stream);
            case 32: return launch_append<T, true, 256, 2>(a, stream);
            case 64: return launch_append<T, true, 256, 4>(a, stream);
            case 128: return launch_append<T, true, 256, 8>(a, stream);
            default: return launch_append<T, true, 256, 16>(a, stream);
            }
        }
    }
    return single ? launch_append<T, false, LEOAM_WAVE, 1>(a, stream) : launch_append<T, false, 256, 1>(a, stream);
}

hipError_t page_append_dispatch(const leoam_pages* s, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                const void* v, int64_t v_stride, int n_new, const int32_t* new_off, const int32_t* seq_len,
                                const int32_t* page_table, const float* rope, void* q_out, void* k_pages, void* v_pages,
                                float* k_scale, float* v_scale, void* abstract, int32_t* chunk_off, int32_t* n_chunks,
                                int32_t* status, hipStream_t stream) {
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
    const bool store8 = s->kv_dtype == LEOAM_E4M3, single = new_off == nullptr;
    switch (s->q_dtype) {
    case LEOAM_F32: return append_of<F32>(a, store8, single, stream);
    case LEOAM_F16: return append_of<F16>(a, store8, single, stream);
    default: return append_of<BF16>(a, store8, single, stream);
    }
}

}  // namespace leoam
