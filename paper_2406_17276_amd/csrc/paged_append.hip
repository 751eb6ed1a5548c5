// Rows join a paged K/V cache, keys turned by their position on the way (opttree.h: ot_kv_append_paged).
//
// What bounds it: rows are read once (f32 or bf16) and written once (bf16, or bytes); single tokens and branches are launch
// latency and a chain length -> page -> older exponent -> store.  Table entries are read anew for every page (kKnownPages).
//
// The unit of work is a page that receives rows, because an 8-bit page has one exponent per head: its new rows' largest
// magnitude has to be known before the first of them is stored.  A workgroup takes one such page of one sequence and a share
// of the heads; half of its threads carry the keys and half the values, so that both are in flight together (pages of more
// than 16384 elements: all of them the keys, then the values).  A row is LPR lanes of sixteen columns (rope.hpp); a head's new
// rows of the page stay in registers between the pass that finds their largest magnitude and the pass that stores them.  The
// angles of a page's rows are the same for all heads: their cosines and sines are computed once per workgroup and kept in
// LDS, where the lanes of a row read them side by side.
// Measured: 8 prompts of 6144 to 8192 rows x 8 heads of 128, bf16 into 8 bits 83.7 us (4.2 TB/s read and written; a copy of 4 GiB
// reaches 4.76); 64 single tokens 6 us of which the host's part is 4.7.
#include <algorithm>

#include "common.hpp"
#include "internal.h"
#include "paged.hpp"
#include "rope.hpp"

namespace ot {
namespace {

struct AppendArgs {
    const void *K, *V;
    unsigned char *kp, *vp;
    unsigned char *k_exp, *v_exp;
    const int32_t *table, *cache_len, *count, *rows;
    int32_t* new_len;
    Rotary rot;
    int batch, n, heads, share;          // heads per workgroup
    int num_pages, max_pages, ps_log2;
    int shift, count_shift;
    int base;                            // first sequence of this launch
    int lengths_known;                   // new_len holds what this call stores
    long long ks[3], vs[3], kps[3], vps[3];
};

// Smallest exponent byte e with top <= 448 * 2^(e - 127): 448 = 1.75 * 2^8, so the float's exponent less 8, and one more
// where its mantissa is over 1.75's (0x600000 of 0x7fffff: the sum carries).  At least 1.
__device__ __forceinline__ int exponent_for(float top) {
    return max(1, (int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 8);
}
__device__ __forceinline__ float power_of(int e) { return __uint_as_float((unsigned)e << 23); }   // 2^(e - 127), e in 1..254

// Largest magnitude of values taken one by one, on their bits: as signed numbers the positive ones lie in order, as unsigned ones
// the negative ones above all others.  (A floating-point maximum forgets what it had when it meets a signalling NaN.)
struct Largest {
    int pos = 0;
    unsigned neg = 0;
    __device__ __forceinline__ void take(float x, float y) {
        pos = max(max(pos, __float_as_int(x)), __float_as_int(y));
        neg = max(max(neg, __float_as_uint(x)), __float_as_uint(y));
    }
    __device__ __forceinline__ float magnitude() const {                 // infinity if there was one, or a NaN
        return __uint_as_float(min(max((unsigned)pos, neg & 0x7fffffffu), 0x7f800000u));
    }
};
// |x| of finite x, 0 otherwise
__device__ __forceinline__ float finite_abs(float x) {
    const unsigned u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? __uint_as_float(u) : 0.f;
}
// E4M3 bytes, to nearest even; NaNs stay NaNs
__device__ __forceinline__ unsigned pack_e4m3(float x, float y, float z, float w) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(z, w, r, true);
}
__device__ __forceinline__ float saturate(float x) { return x > 448.f ? 448.f : (x < -448.f ? -448.f : x); }

// Rows of sequence b before the call, and those asked for, less what the capacity drops
struct Span {
    int len, cnt;
};
__device__ __forceinline__ Span span_of(const AppendArgs& a, int b) {
    const int cap = a.max_pages << a.ps_log2, len = min(max(a.cache_len[b], 0), cap);
    const long long want = a.count ? (long long)a.count[b] + a.count_shift : (long long)a.n;
    return Span{len, (int)min((long long)min(a.n, cap - len), max(want, 0LL))};
}
// new_len of sequence b, by a workgroup: rows are stored up to the first table entry that is no page
template <int NT>
__device__ __forceinline__ void write_new_len(const AppendArgs& a, int b, const Span& x) {
    __shared__ int s_stop[NT / 64];
    const int32_t* const table = a.table + (long long)b * a.max_pages;
    const int tid = threadIdx.x, p_first = x.len >> a.ps_log2, p_last = (x.len + x.cnt - 1) >> a.ps_log2;
    int stop = p_last + 1;
#pragma unroll 4
    for (int p = p_first + tid; p <= p_last; p += NT)
        if ((unsigned)table[p] >= (unsigned)a.num_pages) stop = min(stop, p);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) stop = min(stop, __shfl_xor(stop, o));
    if ((tid & 63) == 0) s_stop[tid >> 6] = stop;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < NT / 64; ++w) stop = min(stop, s_stop[w]);
        a.new_len[b] = x.cnt == 0 ? x.len : (stop > p_last ? x.len + x.cnt : max(x.len, stop << a.ps_log2));
    }
}
// Ahead of an append of many pages (kKnownPages)
__global__ __launch_bounds__(1024) void paged_new_len_kernel(const AppendArgs a) { write_new_len<1024>(a, blockIdx.x, span_of(a, blockIdx.x)); }
// A workgroup looks at its sequence's table entries from the first new page to its own, since rows behind one that is no page are
// dropped: P^2 / 2 reads for P pages, nothing beside the rows of a thousand pages and more than them beyond.  With more pages than this
// a launch ahead finds the new lengths once.  us without it and with it, pages of 16, 2 heads of 64: 7.0 and 8.1 for 1024 pages, 9.6 and
// 9.7 for 1536, 24.0 and 16.4 for 4096, 1875 and 252 for 65536; 8 heads of 128: 22.4 and 20.6, 32.0 and 27.3, 140 and 83 for 4096.
constexpr int kKnownPages = 1536;

template <int DT, bool KV8, int D, int NT, bool TOGETHER>
__global__ __launch_bounds__(NT) void kv_append_paged_kernel(const AppendArgs a) {
    constexpr int LPR = D / 16;                // lanes per row
    constexpr int PASSES = 2;
    constexpr int HALF = TOGETHER ? NT / 2 : NT;       // threads of the keys, and of the values
    constexpr int RPP = HALF / LPR;            // rows per pass
    // a page has at most PASSES * RPP rows (host)
    extern __shared__ __attribute__((aligned(16))) float2 s_cs[];               // [page rows][R / 2]
    __shared__ float s_top[NT / 64];
    const int tid = threadIdx.x, wave = tid >> 6;
    const int ht = tid % HALF, t = ht % LPR, r_first = ht / LPR;
    const int b = a.base + blockIdx.z;
    const int ps = 1 << a.ps_log2;
    Span x = span_of(a, b);
    if (a.lengths_known) x.cnt = a.new_len[b] - x.len;
    const int len = x.len, cnt = x.cnt;
    const int p_first = len >> a.ps_log2, p_last = (len + cnt - 1) >> a.ps_log2;      // (cnt = 0: p_last <= p_first)
    const int page_slot = p_first + blockIdx.x;
    const int32_t* const table = a.table + (long long)b * a.max_pages;
    if (!a.lengths_known && blockIdx.x == 0 && blockIdx.y == 0) write_new_len<NT>(a, b, x);
    if (cnt == 0 || page_slot > p_last) return;
    if (!a.lengths_known) {
        bool bad = false;
        for (int p = p_first + tid; p <= page_slot; p += NT) bad |= (unsigned)table[p] >= (unsigned)a.num_pages;
        if (__syncthreads_or(bad)) return;
    }
    const int page = table[page_slot];
    const int row0 = max(0, len - (page_slot << a.ps_log2)), row1 = min(ps, len + cnt - (page_slot << a.ps_log2));
    const int j0 = (page_slot << a.ps_log2) - len;                 // list position of the page's row 0
    const int half = a.rot.dim / 2;
    if (half) {
        for (int i = tid; i < (row1 - row0) * half; i += NT) {
            const int r = i / half, j = i - r * half;
            const long long pos = ((long long)page_slot << a.ps_log2) + row0 + r + a.shift;
            s_cs[(row0 + r) * half + angle_at(j, half / 8)] = cos_sin((double)pos * a.rot.inv_freq[j]);
        }
        __syncthreads();
    }
    const int h1 = min(a.heads, (int)(blockIdx.y + 1) * a.share);
    // keys and values side by side, or one after the other
    for (int turn_of = 0; turn_of < (TOGETHER ? 1 : 2); ++turn_of) {
    const bool val = TOGETHER ? tid >= HALF : turn_of == 1;
    const bool turns = !val && 16 * t < a.rot.dim;
    const int ca = val ? 16 * t : run_a(a.rot, t), cb = val ? 16 * t + 8 : run_b(a.rot, t);
    const long long ss[3] = {val ? a.vs[0] : a.ks[0], val ? a.vs[1] : a.ks[1], val ? a.vs[2] : a.ks[2]};
    const long long ds[3] = {val ? a.vps[0] : a.kps[0], val ? a.vps[1] : a.kps[1], val ? a.vps[2] : a.kps[2]};
    const void* const src = val ? a.V : a.K;
    unsigned char* const dst = (val ? a.vp : a.kp);
    constexpr int ESZ = KV8 ? 1 : 2;
    long long from[PASSES];                    // element offset of each pass's source row, -1: a row of zeros
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int r = r_first + p * RPP;
        from[p] = -1;
        if (r >= row0 && r < row1) {
            const int j = j0 + r, i = a.rows ? a.rows[(long long)b * a.n + j] : j;
            if ((unsigned)i < (unsigned)a.n) from[p] = (long long)b * ss[0] + (long long)i * ss[2];
        }
    }
    for (int h = blockIdx.y * a.share; h < h1; ++h) {
        float xa[PASSES][8], xb[PASSES][8];
        Largest largest;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
#pragma unroll
            for (int e = 0; e < 8; ++e) xa[p][e] = xb[p][e] = 0.f;
            if (from[p] >= 0) {
                load8<DT>(src, from[p] + h * ss[1] + ca, xa[p]);
                load8<DT>(src, from[p] + h * ss[1] + cb, xb[p]);
            }
        }
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = r_first + p * RPP;
            if (turns && r >= row0 && r < row1) {
                float2 cs[8];
                read_angles(s_cs + r * half, t, half / 8, cs);
                turn(xa[p], xb[p], cs, a.rot.interleaved);
            }
            if constexpr (KV8) {
#pragma unroll
                for (int e = 0; e < 8; ++e) largest.take(xa[p][e], xb[p][e]);
            }
        }
        unsigned char* const row_base = dst + ((long long)page * ds[0] + (long long)h * ds[1]) * ESZ;
        float f = 1.f;
        bool not_finite = false;
        if constexpr (KV8) {
            // over the wavefronts of the keys or the values, and over all
            constexpr int HW = TOGETHER ? NT / 128 : NT / 64;
            auto over = [&](float v, float& all) {
                v = wave_max_f(v);
                __syncthreads();                                   // (what was in s_top has been read)
                if ((tid & 63) == 0) s_top[wave] = v;
                __syncthreads();
                float k = 0.f, w = 0.f;
#pragma unroll
                for (int i = 0; i < HW; ++i) { k = fmaxf(k, s_top[i]); if (TOGETHER) w = fmaxf(w, s_top[HW + i]); }
                all = fmaxf(k, w);
                return TOGETHER && val ? w : k;
            };
            float all, top = over(largest.magnitude(), all);
            not_finite = all > 3.402823466e38f;
            if (not_finite) {                                      // the exponent is that of the finite values
                top = 0.f;
#pragma unroll
                for (int p = 0; p < PASSES; ++p)
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = fmaxf(top, fmaxf(finite_abs(xa[p][e]), finite_abs(xb[p][e])));
                top = over(top, all);
            }
            unsigned char* const exp_at = (val ? a.v_exp : a.k_exp) + (long long)page * a.heads + h;
            int e = exponent_for(top);
            if (row0 > 0) {
                const int e_old = min(max((int)*exp_at, 1), 253);
                if (e > e_old) {                                   // older rows follow
                    const float g = e - e_old > 126 ? 0.f : power_of(127 + e_old - e);
                    for (int r = r_first; r < row0; r += RPP) {
                        u32x4* const w = (u32x4*)(row_base + r * ds[2] + 16 * t);
                        u32x4 v = *w;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[i], false);
                            const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[i], true);
                            v[i] = pack_e4m3(lo[0] * g, lo[1] * g, hi[0] * g, hi[1] * g);
                        }
                        *w = v;
                    }
                }
                e = max(e, e_old);
            }
            f = power_of(254 - e);
            if (not_finite) {
#pragma unroll
                for (int p = 0; p < PASSES; ++p)
#pragma unroll
                    for (int i = 0; i < 8; ++i) { xa[p][i] = saturate(xa[p][i] * f); xb[p][i] = saturate(xb[p][i] * f); }
                f = 1.f;
            }
            if (row0 > 0) __syncthreads();                         // every lane has read the old exponent
            if (ht == 0) *exp_at = (unsigned char)e;
        }
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = r_first + p * RPP;
            if (r < row0 || r >= row1) continue;
            if constexpr (KV8) {
                const float* x = xa[p];
                *(uint2*)(row_base + r * ds[2] + ca) = uint2{pack_e4m3(x[0] * f, x[1] * f, x[2] * f, x[3] * f), pack_e4m3(x[4] * f, x[5] * f, x[6] * f, x[7] * f)};
                x = xb[p];
                *(uint2*)(row_base + r * ds[2] + cb) = uint2{pack_e4m3(x[0] * f, x[1] * f, x[2] * f, x[3] * f), pack_e4m3(x[4] * f, x[5] * f, x[6] * f, x[7] * f)};
            } else {
                store8<OT_BF16>(row_base, r * ds[2] + ca, xa[p]);
                store8<OT_BF16>(row_base, r * ds[2] + cb, xb[p]);
            }
        }
    }
    }
}

int validate_append(const ot_append_params* p, const ot_paged_cache* c) {
    if (!p) return OT_ERR_INVALID_ARG;
    const int st = validate_cache(c, true);
    if (st != OT_OK) return st;
    if (p->batch < 1 || p->n < 1) return OT_ERR_INVALID_ARG;
    if (p->dtype != OT_F32 && p->dtype != OT_BF16) return OT_ERR_INVALID_ARG;
    if (p->interleaved != 0 && p->interleaved != 1) return OT_ERR_INVALID_ARG;
    if (p->rotary_dim < 0 || p->rotary_dim > c->head_dim) return OT_ERR_INVALID_ARG;
    if (p->rotary_dim % 16) return OT_ERR_UNSUPPORTED;
    for (const int64_t* pool : {c->k_strides, c->v_strides})
        if (overlaps(pool, c->num_pages, c->kv_heads, c->page_size, c->head_dim)) return OT_ERR_INVALID_ARG;
    if ((long long)p->batch * p->n > 0x7fffffffLL || p->n > OT_MAX_APPEND || c->kv_heads > 65535) return OT_ERR_UNSUPPORTED;
    const int vec = p->dtype == OT_BF16 ? 8 : 4;
    for (int i = 0; i < 3; ++i)
        if (p->k_strides[i] < 0 || p->k_strides[i] % vec || p->v_strides[i] < 0 || p->v_strides[i] % vec) return OT_ERR_INVALID_ARG;
    return OT_OK;
}

bool overlap(const void* x, size_t nx, const void* y, size_t ny) {
    return x && y && (uintptr_t)x < (uintptr_t)y + ny && (uintptr_t)y < (uintptr_t)x + nx;
}

template <int DT, bool KV8, int D, int NT, bool TOGETHER>
int launch(const AppendArgs& a, const dim3& grid, size_t lds, hipStream_t s) {
    if (lds > 64 * 1024)
        OT_HIP_CHECK(hipFuncSetAttribute((const void*)kv_append_paged_kernel<DT, KV8, D, NT, TOGETHER>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    hipLaunchKernelGGL((kv_append_paged_kernel<DT, KV8, D, NT, TOGETHER>), grid, dim3(NT), lds, s, a);
    return OT_OK;
}
// Threads by the page's elements: two passes over its rows, which leaves room for 16 wavefronts and more on a compute unit (four
// passes of half the threads: 12; 8 prompts of 8192 rows 107 us, not 83).
template <int DT, bool KV8>
int launch_for(const AppendArgs& a, int D, const dim3& grid, size_t lds, hipStream_t s) {
    const int elements = D << a.ps_log2;
    if (elements <= 4096) return D == 128 ? launch<DT, KV8, 128, 256, true>(a, grid, lds, s) : launch<DT, KV8, 64, 256, true>(a, grid, lds, s);
    if (elements <= 8192) return D == 128 ? launch<DT, KV8, 128, 512, true>(a, grid, lds, s) : launch<DT, KV8, 64, 512, true>(a, grid, lds, s);
    if (elements <= 16384) return D == 128 ? launch<DT, KV8, 128, 1024, true>(a, grid, lds, s) : launch<DT, KV8, 64, 1024, true>(a, grid, lds, s);
    return launch<DT, KV8, 128, 1024, false>(a, grid, lds, s);
}

}  // namespace
}  // namespace ot

using namespace ot;

extern "C" {

int ot_kv_append_paged(const ot_append_params* p, const ot_paged_cache* cache, const void* K, const void* V, const double* inv_freq,
                       const int32_t* cache_len, const int32_t* count, const int32_t* rows, int32_t* new_len, void* hip_stream) {
    const int st = validate_append(p, cache);
    if (st != OT_OK) return st;
    if (!K || !V || !cache_len || !new_len || (p->rotary_dim && !inv_freq)) return OT_ERR_INVALID_ARG;
    if ((uintptr_t)K % 16 || (uintptr_t)V % 16 || (uintptr_t)inv_freq % 8 || (uintptr_t)cache_len % 4 || (uintptr_t)count % 4 ||
        (uintptr_t)rows % 4 || (uintptr_t)new_len % 4)
        return OT_ERR_INVALID_ARG;
    // workgroups still read these while new_len is written
    const size_t nb = (size_t)p->batch * 4;
    if (overlap(new_len, nb, cache_len, nb) || overlap(new_len, nb, count, nb) || overlap(new_len, nb, rows, nb * p->n)) return OT_ERR_INVALID_ARG;
    // keys and values of one row at one address, or their exponents
    if (cache->k_pages == cache->v_pages || (cache->dtype == OT_E4M3 && cache->k_exp == cache->v_exp)) return OT_ERR_INVALID_ARG;
    AppendArgs a;
    a.K = K; a.V = V; a.kp = (unsigned char*)cache->k_pages; a.vp = (unsigned char*)cache->v_pages;
    a.k_exp = cache->k_exp; a.v_exp = cache->v_exp;
    a.table = cache->page_table; a.cache_len = cache_len; a.count = count; a.rows = rows; a.new_len = new_len;
    a.rot = Rotary{inv_freq, p->rotary_dim, p->interleaved};
    a.batch = p->batch; a.n = p->n; a.heads = cache->kv_heads;
    a.num_pages = cache->num_pages; a.max_pages = cache->max_pages; a.ps_log2 = log2_of(cache->page_size);
    a.shift = p->shift; a.count_shift = p->count_shift;
    for (int i = 0; i < 3; ++i) { a.ks[i] = p->k_strides[i]; a.vs[i] = p->v_strides[i]; a.kps[i] = cache->k_strides[i]; a.vps[i] = cache->v_strides[i]; }
    // pages that n rows can touch
    const int ps = cache->page_size;
    const long long pages = std::min<long long>(((long long)p->n + ps - 2) / ps + 1, cache->max_pages);
    // heads that share a workgroup's angles: as many as leave two workgroups per compute unit
    a.share = 1;
    if (p->rotary_dim) a.share = (int)std::max(1LL, std::min<long long>(a.heads, pages * p->batch * a.heads / 512));
    // (a grid holds fewer than 2^32 threads: a long append's workgroups take more heads, a large batch goes in several launches)
    a.share = (int)std::max<long long>(a.share, (pages * a.heads * 1024 + 0xfffffffeLL) / 0xffffffffLL);
    while (pages * ((a.heads + a.share - 1) / a.share) * 1024 > 0xffffffffLL) ++a.share;
    const unsigned shares = (unsigned)((a.heads + a.share - 1) / a.share);
    const size_t lds = (size_t)ps * (p->rotary_dim / 2) * sizeof(float2);
    hipStream_t s = (hipStream_t)hip_stream;
    a.lengths_known = pages > kKnownPages;
    if (a.lengths_known) {                                         // (batch * n < 2^31: fewer than 2^15 sequences)
        hipLaunchKernelGGL(paged_new_len_kernel, dim3((unsigned)p->batch), dim3(1024), 0, s, a);
        OT_HIP_CHECK(hipGetLastError());
    }
    const int per = std::min(65535, sequences_per_launch(p->batch, pages * shares * 1024LL));
    for (int base = 0; base < p->batch; base += per) {
        a.base = base;
        const dim3 grid((unsigned)pages, shares, (unsigned)std::min(per, p->batch - base));
        const int D = cache->head_dim;
        int r;
        if (p->dtype == OT_BF16) r = cache->dtype == OT_E4M3 ? launch_for<OT_BF16, true>(a, D, grid, lds, s) : launch_for<OT_BF16, false>(a, D, grid, lds, s);
        else r = cache->dtype == OT_E4M3 ? launch_for<OT_F32, true>(a, D, grid, lds, s) : launch_for<OT_F32, false>(a, D, grid, lds, s);
        if (r != OT_OK) return r;
        OT_HIP_CHECK(hipGetLastError());
    }
    return OT_OK;
}

}  // extern "C"
