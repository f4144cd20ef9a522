// page_attention_prefill: causal softmax(scale q K^T) V of a call's new tokens over their sequences' pages.
//
// Bound by the matrix cores.  A workgroup takes 128 query rows of one kv head - a row is a (token, head of the
// group) pair, so the heads of a group share every key and value that is fetched - and walks the keys 64 at a time (fp32:
// 32): the tile after the current one is on its way to registers while the current one is worked on in LDS.
// Each of the four waves owns 32 rows.  S^T = K Q^T (32x32 products) leaves lane = row, registers = keys: the row's
// maximum and sum need no exchange but one with the lane 32 away, and P is already the second operand of O^T = V^T P^T;
// the first operand, four keys of one channel at a time, comes out of LDS by the transposing read.
#include "page_common.h"

namespace leoam {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;

constexpr int kRows = 128;            // query rows of a workgroup, 32 a wave

struct PagePrefillArgs {
    const char *q, *k_pages, *v_pages;
    const float *k_scale, *v_scale;
    const int32_t *page_table, *seq_len, *new_off;
    int n_new, n_slots;
    float scale_log2;      // of |softmax_scale|
    uint32_t flip;         // sign bits of the queries, turned if softmax_scale is negative
    char* out;
    float* lse;
    int batch, n_kv_heads, n_pages, page_shift, max_pages;
};

template <typename T> __device__ __forceinline__ f32x16_t mfma_32x32x16(const uint4& a, const uint4& b, f32x16_t c);
template <> __device__ __forceinline__ f32x16_t mfma_32x32x16<BF16>(const uint4& a, const uint4& b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16_t mfma_32x32x16<F16>(const uint4& a, const uint4& b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

// Where 16-byte piece `piece` of row `row` lies in a tile: the pieces of a row are permuted by the row so that neither
// eight rows at one piece (keys) nor four rows at four neighbouring pieces (values) meet in the banks.
__device__ __forceinline__ uint32_t tile_at(int row, int piece, int row_bytes) {
    return (uint32_t)(row * row_bytes + ((piece ^ (((row & 3) << 2) | ((row >> 2) & 3))) << 4));
}

template <typename T> __device__ __forceinline__ uint32_t not_finite(uint32_t w) {      // of a value in the register
    if (T::kTag == LEOAM_F32) return (w & 0x7f800000u) == 0x7f800000u;
    const uint32_t m = T::kTag == LEOAM_F16 ? 0x7c00u : 0x7f80u;
    return (w & m) == m || (w & (m << 16)) == (m << 16);
}

template <typename T, typename S, int G>
__global__ __launch_bounds__(kAttThreads) __attribute__((amdgpu_waves_per_eu(2))) void page_prefill_kernel(PagePrefillArgs a) {
    constexpr bool k8 = std::is_same<S, E4M3>::value, k32 = T::kTag == LEOAM_F32;
    constexpr int ROWB = LEOAM_D * T::kBytes, SROWB = LEOAM_D * S::kBytes;      // a row in LDS, in the pages
    constexpr int KEYS = k32 ? 32 : 64, KB = KEYS / 32, TILE_BYTES = KEYS * ROWB, NQ = k32 ? 16 : 8;
    constexpr int LOADS = KEYS * SROWB / (kAttThreads * 16), PIECES = SROWB / 16, ROWS_PER_LOAD = kAttThreads / PIECES;
    constexpr int GROUPS = KEYS / 16;      // 16 keys never straddle a page
    // fp16: small weights stay clear of fp16's subnormals; the reference may lag the maximum by 2^kLag
    constexpr float kLag = 8.f, kBias = T::kTag == LEOAM_F16 ? 7.f : 0.f;
    __shared__ __align__(16) char sh_k[2][TILE_BYTES];
    __shared__ __align__(16) char sh_v[2][TILE_BYTES];
    __shared__ int sh_bad;

    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / LEOAM_WAVE);
    const int half = lane >> 5, l32 = lane & 31;
    const int hkv = a.n_kv_heads, h = blockIdx.x % hkv;
    // (later rows see more keys: they are started first)
    const int slot = a.n_slots - 1 - (int)(blockIdx.x / hkv);
    int b, local = 0, row0 = 0, m = 1;
    if (a.new_off) {
        // sequence i's tiles begin at slot new_off[i] G / 128 + i
        b = uniform(wave_count_below(a.batch, slot, [&](int i) { return (int)((long long)a.new_off[i] * G / kRows) + i; }));
        if (b >= a.batch) return;
        row0 = uniform(a.new_off[b]);
        m = uniform(a.new_off[b + 1]) - row0;
        local = slot - ((int)((long long)row0 * G / kRows) + b);
        if (row0 < 0 || m < 0 || m > a.n_new - row0) return;
    } else {
        b = slot;
        row0 = b;
    }
    if (local < 0 || (long long)local * kRows >= (long long)m * G) return;
    const int len = min(max(uniform(a.seq_len[b]), 0), a.max_pages << a.page_shift);
    const int first = len - m;                                   // position of the sequence's first new token (may be negative)
    const int tok0 = local * (kRows / G), n_tok = min(m - tok0, kRows / G);
    const int keys = max(first + tok0 + n_tok, 0);               // keys that some row of the workgroup sees
    // this lane's row
    const int row = 32 * wave + l32, tok = min(tok0 + row / G, m - 1);
    const int my_pos = first + tok;
    const bool stored = row / G < n_tok;
    const size_t q_row = ((size_t)(row0 + tok) * hkv + h) * G + row % G;
    const int wave_lo = first + tok0 + 32 * wave / G;             // the wave's rows see at least / at most
    const int wave_hi = min(first + tok0 + (32 * wave + 31) / G, first + m - 1);

    uint4 qb[NQ];
#pragma unroll
    for (int s = 0; s < NQ; ++s) {
        qb[s] = load16(a.q, q_row * ROWB + 32 * s + 16 * half);
        qb[s].x ^= a.flip; qb[s].y ^= a.flip; qb[s].z ^= a.flip; qb[s].w ^= a.flip;
    }
    if (tid == 0) sh_bad = 0;
    __syncthreads();

    const int n_tiles = (keys + KEYS - 1) / KEYS, last = keys - 1;
    const int first_masked = max(first + tok0 + 1, 0) / KEYS;     // tiles from here on hide keys from some row
    const int32_t* table = a.page_table + (size_t)b * a.max_pages;
    auto pages_of = [&](int j, int* id) {      // physical page of each 16-key group of tile j
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) id[g] = uniform(table[min(j * KEYS + 16 * g, last) >> a.page_shift]);
    };
    uint4 kr[LOADS], vr[LOADS];
    float ks[LOADS], vs[LOADS];
    uint32_t ok_next = 0;      // bit g: group g of the tile in registers has a page
    auto fetch = [&](int j, const int* id) {
        ok_next = 0;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) ok_next |= (id[g] >= 0 && id[g] < a.n_pages ? 1u : 0u) << g;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = i * ROWS_PER_LOAD + tid / PIECES;      // (a load's 16-key group is the same for the wave)
            const int g = uniform(r / 16);
            int page = id[0];
#pragma unroll
            for (int u = 1; u < GROUPS; ++u) page = g == u ? id[u] : page;
            if (!(ok_next >> g & 1)) page = 0;
            const size_t base = ((size_t)page * hkv + h);
            const int e = min(j * KEYS + 16 * g, last) >> a.page_shift;
            const uint32_t at = (uint32_t)(min(j * KEYS + r, last) - (e << a.page_shift)) * SROWB + 16 * (tid % PIECES);
            kr[i] = load16(a.k_pages + (base << a.page_shift) * SROWB, at);
            vr[i] = load16(a.v_pages + (base << a.page_shift) * SROWB, at);
            if (k8) {
                ks[i] = a.k_scale[base];
                vs[i] = a.v_scale[base];
            }
        }
    };
    auto stage = [&](int j, int buf) {
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = i * ROWS_PER_LOAD + tid / PIECES, piece = tid % PIECES;
            if (!(ok_next >> (r / 16) & 1)) {      // nothing there: no value may matter
                vr[i] = make_uint4(0, 0, 0, 0);
                vs[i] = 1.f;
            }
            if constexpr (k8) {
                const uint4 k0 = widen8<T>(kr[i].x, kr[i].y, ks[i]), k1 = widen8<T>(kr[i].z, kr[i].w, ks[i]);
                uint4 v0 = widen8<T>(vr[i].x, vr[i].y, vs[i]), v1 = widen8<T>(vr[i].z, vr[i].w, vs[i]);
                store16(sh_k[buf], tile_at(r, 2 * piece, ROWB), k0);
                store16(sh_k[buf], tile_at(r, 2 * piece + 1, ROWB), k1);
                store16(sh_v[buf], tile_at(r, 2 * piece, ROWB), v0);
                store16(sh_v[buf], tile_at(r, 2 * piece + 1, ROWB), v1);
                if (j >= first_masked)
                    bad |= not_finite<T>(v0.x) | not_finite<T>(v0.y) | not_finite<T>(v0.z) | not_finite<T>(v0.w) |
                           not_finite<T>(v1.x) | not_finite<T>(v1.y) | not_finite<T>(v1.z) | not_finite<T>(v1.w);
            } else {
                store16(sh_k[buf], tile_at(r, piece, ROWB), kr[i]);
                store16(sh_v[buf], tile_at(r, piece, ROWB), vr[i]);
                if (j >= first_masked)
                    bad |= not_finite<T>(vr[i].x) | not_finite<T>(vr[i].y) | not_finite<T>(vr[i].z) | not_finite<T>(vr[i].w);
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

    auto work = [&](int j, int buf, uint32_t ok) {
        f32x16_t s[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                const uint4 ka = load16(sh_k[buf], tile_at(32 * kb + l32, 2 * i + half, ROWB));
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
        const bool masked = j * KEYS + KEYS - 1 > wave_lo || ok != (1u << GROUPS) - 1;
        if (masked) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (j * KEYS + key_of(kb, r) > my_pos || !(ok >> (2 * kb + r / 8) & 1)) s[kb][r] = -INFINITY;
        }
        float mt = s[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) mt = fmaxf(mt, s[kb][r]);
        {
            float x = mt, y = mt;
            permlane32_swap(x, y);
            mt = fmaxf(x, y) * a.scale_log2 - kBias;
        }
        // The reference is the maximum of some earlier tile; it moves only when the maximum has left it behind by 2^kLag.
        if (__ballot(mt > ref + kLag || (ref == -INFINITY && mt > ref))) {
            const float now = fmaxf(ref, mt), c = exp2_or_zero(ref, now);
            ref = now;
            l_run *= c;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][r] *= c;
        }
        const float base = ref == -INFINITY ? 0.f : ref;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[kb][r] = exp2_raw(fmaf(s[kb][r], a.scale_log2, -base));
                l_run += s[kb][r];
            }
        const bool careful = masked && sh_bad;      // a hidden key may have a value that is not finite
        if constexpr (k32) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                    const int key = key_of(0, r), d = 32 * db + l32;
                    uint32_t v = *reinterpret_cast<const uint32_t*>(sh_v[buf] + tile_at(key, d / 4, ROWB) + 4 * (d % 4));
                    if (careful && not_finite<T>(v)) v = 0;
                    acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(bits_to_float(v), s[0][r], acc[db], 0, 0, 0);
                }
        } else {
#pragma unroll
            for (int t = 0; t < 2 * KB; ++t) {      // 16 keys
                const int kb = t / 2, r0 = 8 * (t % 2);
                const uint4 p = make_uint4(pair_of(T{}, s[kb][r0], s[kb][r0 + 1]), pair_of(T{}, s[kb][r0 + 2], s[kb][r0 + 3]),
                                           pair_of(T{}, s[kb][r0 + 4], s[kb][r0 + 5]), pair_of(T{}, s[kb][r0 + 6], s[kb][r0 + 7]));
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                    uint2 w[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int key = 16 * t + 8 * u + 4 * half + (lane & 15) / 4, d = 32 * db + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
                        char* at = sh_v[buf] + tile_at(key, d / 8, ROWB) + 2 * (d % 8);
                        w[u] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                             (__attribute__((address_space(3))) s16x4_t*)at));
                    }
                    uint4 v = make_uint4(w[0].x, w[0].y, w[1].x, w[1].y);
                    if (careful) {
                        const uint32_t mk = T::kTag == LEOAM_F16 ? 0x7c00u : 0x7f80u;
                        auto clean = [&](uint32_t x) {
                            if ((x & mk) == mk) x &= 0xffff0000u;
                            if ((x & (mk << 16)) == (mk << 16)) x &= 0xffffu;
                            return x;
                        };
                        v = make_uint4(clean(v.x), clean(v.y), clean(v.z), clean(v.w));
                    }
                    acc[db] = mfma_32x32x16<T>(v, p, acc[db]);
                }
            }
        }
        if (careful) {
            // values that are not finite were left out: they reach the rows that see their key
            for (int key = 0; key < KEYS; ++key) {
                const bool sees = j * KEYS + key <= my_pos && (ok >> (key / 16) & 1);
#pragma unroll
                for (int db = 0; db < 4; ++db)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int d = 32 * db + 8 * (r / 4) + 4 * half + r % 4;
                        const char* at = sh_v[buf] + tile_at(key, d * T::kBytes / 16, ROWB) + (d * T::kBytes) % 16;
                        float v;
                        if constexpr (k32) v = *reinterpret_cast<const float*>(at);
                        else if constexpr (T::kTag == LEOAM_F16) v = (float)*reinterpret_cast<const _Float16*>(at);
                        else v = bits_to_float((uint32_t) * reinterpret_cast<const uint16_t*>(at) << 16);
                        if (sees && not_finite<F32>(float_to_bits(v))) acc[db][r] += v;
                    }
            }
        }
    };

    if (n_tiles > 0) {
        int id[GROUPS];
        pages_of(0, id);
        fetch(0, id);
        pages_of(min(1, n_tiles - 1), id);
        stage(0, 0);
        uint32_t ok = ok_next;
        __syncthreads();
        for (int j = 0; j < n_tiles; ++j) {
            const bool more = j + 1 < n_tiles;
            if (more) {
                fetch(j + 1, id);
                pages_of(min(j + 2, n_tiles - 1), id);
            }
            if (j * KEYS <= wave_hi) work(j, j & 1, ok);
            if (more) stage(j + 1, (j + 1) & 1);
            ok = ok_next;
            __syncthreads();
        }
    }

    // ---- the rows' results -------------------------------------------------------------------------------
    const float l = l_run + shfl_xor_f(l_run, 32), inv = l == 0.f ? 0.f : 1.f / l;      // (NaN stays)
    if (!stored) return;
    if (a.lse && half == 0) a.lse[q_row] = l == 0.f ? -INFINITY : (ref + log2f(l)) * kLn2;
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
}

size_t page_decode_workspace_bytes(const leoam_pages*);
size_t page_decode_min_workspace_bytes(const leoam_pages*);
size_t page_workspace_bytes(const leoam_pages* s, int n_new) {
    return n_new <= 0 ? page_decode_workspace_bytes(s) : page_decode_min_workspace_bytes(s);
}
size_t page_min_workspace_bytes(const leoam_pages* s) { return page_decode_min_workspace_bytes(s); }

template <typename T, typename S> static hipError_t launch_prefill(const PagePrefillArgs& a, int group, hipStream_t stream) {
    const long long units = (long long)a.n_slots * a.n_kv_heads;
    if (units > 0x7fffffffll) return hipErrorInvalidValue;
    const dim3 grid((unsigned)units), block(kAttThreads);
    switch (group) {
    case 1: hipLaunchKernelGGL((page_prefill_kernel<T, S, 1>), grid, block, 0, stream, a); break;
    case 2: hipLaunchKernelGGL((page_prefill_kernel<T, S, 2>), grid, block, 0, stream, a); break;
    case 4: hipLaunchKernelGGL((page_prefill_kernel<T, S, 4>), grid, block, 0, stream, a); break;
    default: hipLaunchKernelGGL((page_prefill_kernel<T, S, 8>), grid, block, 0, stream, a); break;
    }
    return hipGetLastError();
}

hipError_t page_prefill_dispatch(const leoam_pages* s, const void* q, int n_new, const int32_t* new_off, const void* k_pages,
                                 const void* v_pages, const float* k_scale, const float* v_scale, const int32_t* page_table,
                                 const int32_t* seq_len, float softmax_scale, void* out, float* lse, void*, size_t,
                                 hipStream_t stream) {
    PagePrefillArgs a;
    const int group = s->n_q_heads / s->n_kv_heads;
    a.q = (const char*)q; a.k_pages = (const char*)k_pages; a.v_pages = (const char*)v_pages;
    a.k_scale = k_scale; a.v_scale = v_scale; a.page_table = page_table; a.seq_len = seq_len; a.new_off = new_off;
    a.n_new = n_new;
    a.n_slots = new_off ? (int)((long long)n_new * group / kRows) + s->batch : s->batch;
    a.scale_log2 = fabsf(softmax_scale) * kLog2e;
    a.flip = softmax_scale < 0.f ? (s->q_dtype == LEOAM_F32 ? 0x80000000u : 0x80008000u) : 0u;
    a.out = (char*)out; a.lse = lse;
    a.batch = s->batch; a.n_kv_heads = s->n_kv_heads; a.n_pages = s->n_pages;
    a.page_shift = __builtin_ctz((unsigned)s->page_size); a.max_pages = s->max_pages;
    const bool k8 = s->kv_dtype == LEOAM_E4M3;
    switch (s->q_dtype) {
    case LEOAM_F32: return launch_prefill<F32, F32>(a, group, stream);
    case LEOAM_F16: return k8 ? launch_prefill<F16, E4M3>(a, group, stream) : launch_prefill<F16, F16>(a, group, stream);
    default: return k8 ? launch_prefill<BF16, E4M3>(a, group, stream) : launch_prefill<BF16, BF16>(a, group, stream);
    }
}

}  // namespace leoam
