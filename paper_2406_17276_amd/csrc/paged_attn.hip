// Tree-masked attention over a paged cache (opttree.h: ot_tree_verify_attention_paged).
//   O[i] = sum_j softmax_j(scale q_i . k_j) v_j,  j over cache rows (found through the page table) and visible tree rows
//
// The keys of a (sequence, KV head) are cut into 64-key tiles, cache first, then tree.  A job is a range of tiles for one block
// of packed query rows (GQA: the rows of the g query heads of a KV head are stacked, row = head * n + node); a workgroup is a job.
// Softmax in one pass: running reference and sum per query, fp32; a range leaves an un-normalised partial and the last job of
// a row block to finish merges them (tickets).
//
// Ranges are decided on the device, from the lengths as they are (find_job): a page table gives every sequence room for
// the longest context, so the host's bound on a length says little, and lengths in a serving batch differ.
#include <math.h>

#include <algorithm>

#include "common.hpp"
#include "internal.h"
#include "paged.hpp"
#include "rope.hpp"

namespace ot {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned long long u64;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kCounters = OT_PAGED_SYNC_BYTES / 4 - 1024;   // tickets, behind the kilo-word that ends with the status word
constexpr int kSplitBatch = 256;                             // sequences of a batch whose contexts are cut into ranges
constexpr int kTile = 64;
// reference of a row that has seen nothing: from it a masked score gives 0 and any score moves the reference
constexpr float kNoRef = -3.402823466e38f;
// The reference follows the row's maximum only when that is this far ahead: probabilities up to 2^8 lose nothing in fp32 or in
// bf16, and most tiles then rescale nothing.
constexpr float kSlack = 8.f;

struct PagedArgs {
    const void *Q, *Kt, *Vt;
    const unsigned char *kp, *vp;
    const unsigned char *k_exp, *v_exp;
    const int32_t *table, *prefix_len;
    const uint64_t* mask;
    void* O;
    unsigned int* sync;
    float* part;                 // [job][rows of a block][D], then [job][rows][2] (reference, sum)
    float* part_ml;
    int batch, kv_heads, g, n, tree_keys, W, row_blocks, units;   // units = kv_heads * row_blocks
    int num_pages, max_pages, ps_log2;
    int split, target, least;    // ranges allowed; jobs aimed at; fewest tiles of a range
    int slot_rows;               // rows of a partial
    float scale_log2;
    long long qs[3], kts[3], vts[3], os[3], kps[3], vps[3];
};

__device__ __forceinline__ float xhalf_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float xhalf_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ int wave_sum_i(int v) {
    v = wave_incl_scan(v, 0);
    return rl(v, 63);
}
__device__ __forceinline__ int wave_max_i(int v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = max(v, __shfl_xor(v, o));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

struct Job {
    int b, unit;          // sequence; KV head and row block
    int len;              // cache rows
    int t0, t1;           // tiles
    int splits, split;
    int slot;             // of its partial; its siblings' are `units` apart
    bool none;
};

// Which range of which unit workgroup `wg` computes; the same in every lane of the workgroup.  With more than one range to go
// round, tiles per range are the fewest (at least a.least) with which all jobs together are no more than a.target: each
// sequence takes ceil(tiles / share) ranges of equal length.  Lane j holds sequences j, j + 64, ...
__device__ __forceinline__ Job find_job(const PagedArgs& a, int wg) {
    const int lane = threadIdx.x & 63, cap = a.max_pages << a.ps_log2;
    const int ttiles = (a.tree_keys + kTile - 1) / kTile;
    Job j;
    j.none = false;
    if (!a.split) {
        j.b = wg / a.units;
        j.unit = wg - j.b * a.units;
        j.splits = 1; j.split = 0; j.slot = 0;
        if (j.b >= a.batch) { j.none = true; return j; }
    } else {
        constexpr int NL = kSplitBatch / 64;
        int T[NL], S[NL], total = 0, most = 0;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int b = lane + 64 * i;
            T[i] = b < a.batch ? (min(max(a.prefix_len[b], 0), cap) + kTile - 1) / kTile + ttiles : 0;
        }
#pragma unroll
        for (int i = 0; i < NL; ++i)
            if (i == 0 || a.batch > 64 * i) { total += wave_sum_i(T[i]); most = max(most, wave_max_i(T[i])); }
        const long long all = (long long)total * a.units;
        int share = max(a.least, (int)min((long long)most, (all + a.target - 1) / a.target));
        int jobs;
        while (true) {
            jobs = 0;
#pragma unroll
            for (int i = 0; i < NL; ++i)
                if (i == 0 || a.batch > 64 * i) {
                    S[i] = lane + 64 * i < a.batch ? max(1, (T[i] + share - 1) / share) : 0;
                    jobs += wave_sum_i(S[i]);
                }
            if ((long long)jobs * a.units <= a.target || share >= most) break;
            share += max(1, share >> 4);
        }
        const int u = wg / a.units;                      // which (sequence, range)
        if (u >= jobs) { j.none = true; return j; }
        j.unit = wg - u * a.units;
        int before = 0;
        j.b = 0; j.split = 0; j.splits = 1;
#pragma unroll
        for (int i = 0; i < NL; ++i)
            if (i == 0 || a.batch > 64 * i) {
                const int end = before + wave_incl_scan(S[i], lane);
                const u64 hit = __ballot(u >= end - S[i] && u < end);
                if (hit) {
                    const int l = (int)__builtin_ctzll(hit);
                    j.b = 64 * i + l;
                    j.splits = rl(S[i], l);
                    j.split = u - (rl(end, l) - j.splits);
                }
                before = rl(end, 63);
            }
        j.slot = wg - j.split * a.units;                 // of the unit's first range
    }
    const int raw = a.prefix_len[j.b];
    j.len = min(max(raw, 0), cap);
    if (j.len != raw && threadIdx.x == 0)
        __hip_atomic_fetch_or(a.sync + OT_ATTN_STATUS_OFFSET / 4, OT_ATTN_STATUS_PREFIX_CLAMPED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const long long Tb = (j.len + kTile - 1) / kTile + ttiles;
    j.t0 = (int)(Tb * j.split / j.splits);
    j.t1 = (int)(Tb * (j.split + 1) / j.splits);
    j.b = uniform(j.b); j.unit = uniform(j.unit); j.len = uniform(j.len); j.t0 = uniform(j.t0); j.t1 = uniform(j.t1);
    j.splits = uniform(j.splits); j.split = uniform(j.split); j.slot = uniform(j.slot);
    return j;
}

// Union over a sequence's queries of the mask words of tree tiles tt0 .. tt1 - 1: rows of V that no query sees enter the
// products as zeros, whatever they hold.
__device__ __forceinline__ void union_masks(const PagedArgs& a, int b, int tt0, int tt1, u64* s_union, int nthreads) {
    for (int i = threadIdx.x; i < tt1 - tt0; i += nthreads) s_union[i] = 0;
    __syncthreads();
    const int words = tt1 - tt0;
    for (int i = threadIdx.x; i < words * a.n; i += nthreads) {
        const int row = i / words, w = i - row * words;
        const u64 m = a.mask[((long long)b * a.n + row) * a.W + tt0 + w];
        if (m) atomicOr(s_union + w, m);
    }
    __syncthreads();
}

// Sixteen E4M3 values times a power of two as bf16, which holds each of them
__device__ __forceinline__ void widen16(const u32x4& w, float scale, u32x4& lo, u32x4& hi) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        lo[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false));
        lo[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true));
        hi[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 + i], scale, false));
        hi[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 + i], scale, true));
    }
}
__device__ __forceinline__ float exp_scale(int e) { return __uint_as_float((unsigned)min(max(e, 1), 253) << 23); }

typedef s16x4 __attribute__((address_space(3))) * lds_s16x4;
__device__ __forceinline__ bf16x8 column_of_8_rows(const unsigned short* seg, int second) {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)seg);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(seg + second));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// Where V's 32-byte segment g of key row r sits inside the row: at g ^ v_swizzle(r).  A transposed read touches, per 32
// lanes, four consecutive rows and the two halves of a 32-column block; the eight segments must fall into eight different
// 32-byte slots of a 256-byte window.
template <int D> __device__ __forceinline__ int v_swizzle(int r) { return D == 128 ? (r & 3) << 1 : ((r >> 1) & 1) << 1; }

// A 32-key block of scores (lane: query l32, keys 8 (v/4) + 4 h + v%4) becomes probabilities; returns them packed as the
// B operands of the two 16-key slabs, and rescales what the row has summed when the reference moves.
template <int NO>
__device__ __forceinline__ void softmax_block(f32x16& s, float c, float& ref, float& l, f32x16 (&o)[NO], u32x4 (&p)[2]) {
    float m = max3(s[0], s[1], s[2]);
#pragma unroll
    for (int v = 3; v < 15; v += 2) m = max3(m, s[v], s[v + 1]);
    m = xhalf_max(max2(m, s[15])) * c;
    if (__any(m > ref + kSlack)) {
        const float to = m > ref + kSlack ? m : ref, f = __builtin_amdgcn_exp2f(ref - to);
        l *= f;
#pragma unroll
        for (int d = 0; d < NO; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[d][v] *= f;
        ref = to;
    }
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, -ref));
        sum += s[v];
    }
    l += sum;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[u][i] = pack_bf16(s[8 * u + 2 * i], s[8 * u + 2 * i + 1]);
}
// scores of keys whose bit is not set
__device__ __forceinline__ void hide(f32x16& s, unsigned bits, int h) {
    bits >>= 4 * h;
#pragma unroll
    for (int v = 0; v < 16; ++v)
        if (!(bits >> (8 * (v >> 2) + (v & 3)) & 1)) s[v] = -INFINITY;
}

__device__ __forceinline__ u64 pack2(float x, float y) { return (u64)__float_as_uint(x) | ((u64)__float_as_uint(y) << 32); }
// Partials travel between workgroups on different XCDs: device-scope stores write through, device-scope loads read around
// the caches, and every wavefront waits for its stores before the workgroup takes its ticket.
__device__ __forceinline__ void put2(float* p, float x, float y) {
    __hip_atomic_store((u64*)p, pack2(x, y), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get2(const float* p) {
    const u64 w = __hip_atomic_load((const u64*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return float2{__uint_as_float((unsigned)w), __uint_as_float((unsigned)(w >> 32))};
}
__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }       // nothing seen: zeros

__device__ __forceinline__ unsigned short* out_row(const PagedArgs& a, int b, int hk, int rho) {
    const int head = rho / a.n, node = rho - head * a.n;
    return (unsigned short*)a.O + (long long)b * a.os[0] + (long long)(hk * a.g + head) * a.os[1] + (long long)node * a.os[2];
}

// After a workgroup has stored its partial: the last one of its row block adds all of them up, in the order of the ranges.
template <int D, int NT>
__device__ __forceinline__ void join_splits(const PagedArgs& a, const Job& j, int hk, int row0, int rows) {
    __shared__ int s_last;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    unsigned int* const ticket = a.sync + 1024 + j.b * a.units + j.unit;
    if (threadIdx.x == 0)
        s_last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)(j.splits - 1);
    __syncthreads();
    if (!s_last) return;
    if (threadIdx.x == 0) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int i = threadIdx.x; i < rows * (D / 8); i += NT) {
        const int row = i / (D / 8), col = i % (D / 8) * 8;
        float M = kNoRef, L = 0.f, o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.f;
        for (int s = 0; s < j.splits; ++s) {
            const size_t at = (size_t)(j.slot + s * a.units) * a.slot_rows + row;
            const float2 ml = get2(a.part_ml + at * 2);
            const float to = fmaxf(M, ml.x), f = __builtin_amdgcn_exp2f(M - to), w = __builtin_amdgcn_exp2f(ml.x - to);
            L = L * f + ml.y * w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 x = get2(a.part + at * D + col + 2 * e);
                o[2 * e] = o[2 * e] * f + x.x * w;
                o[2 * e + 1] = o[2 * e + 1] * f + x.y * w;
            }
            M = to;
        }
        const float inv = inverse(L);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= inv;
        store8<OT_BF16>(out_row(a, j.b, hk, row0 + row), col, o);
    }
}

// ---------------------------------------------------------------------------
// Few rows: 32 or 64 packed query rows per workgroup (QB blocks of 32).
// Bound by the cache's bytes.  Four wavefronts share a job's keys, 32 at a time, and never wait for each other inside the
// loop: a wavefront loads its 32 rows of K straight into the registers that feed the matrix instruction (S^T = K Q^T, the
// order of the contraction is free, so a lane's sixteen consecutive values serve two instructions), and its 32 rows of V into
// a corner of LDS of its own, from which the transposing read makes the operand of O^T += V^T P^T.  The next block's rows are
// requested before the present one is used.  Pages are multiples of sixteen rows, so a block's page numbers and exponents are
// two scalars each.  The four partial results meet in LDS at the end.
// ---------------------------------------------------------------------------
template <int D, bool KV8, int QB>
__global__ __launch_bounds__(256) void paged_rows_kernel(const PagedArgs a) {
    constexpr int DB = D / 32, NJ = D / 32;
    constexpr int KL = KV8 ? NJ : 2 * NJ;              // 16-byte loads of K per lane and block; the same of V
    constexpr int CPR = (KV8 ? D : 2 * D) / 16;        // 16-byte pieces per row of V in memory
    constexpr int RPL = 64 / CPR;                      // rows of V per load instruction
    constexpr int VW = 32 * D;                         // a wavefront's V in LDS, 2-byte elements
    constexpr int OST = 68;                            // row stride of the exchange at the end
    constexpr int kShared = 4 * VW * 2 > 4 * 32 * OST * 4 ? 4 * VW * 2 : 4 * 32 * OST * 4;
    __shared__ __attribute__((aligned(16))) unsigned char s_mem[kShared];
    __shared__ float s_ref[4][QB * 32], s_sum[4][QB * 32];
    __shared__ u64 s_union[OT_MAX_TREE_KEYS / 64];
    const Job j = find_job(a, blockIdx.x);
    if (j.none) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, h = lane >> 5;
    const int hk = j.unit / a.row_blocks, rb = j.unit - hk * a.row_blocks;
    const int rows_all = a.g * a.n, row0 = rb * QB * 32, rows = min(QB * 32, rows_all - row0);

    // Q: lane (query l32, half h) holds columns 32 i + 16 h .. + 15
    bf16x8 qf[QB][2 * NJ];
    long long mask_at[QB];
#pragma unroll
    for (int q = 0; q < QB; ++q) {
        const int rho = min(row0 + q * 32 + l32, rows_all - 1), head = rho / a.n, node = rho - head * a.n;
        const unsigned short* p = (const unsigned short*)a.Q + (long long)j.b * a.qs[0] + (long long)(hk * a.g + head) * a.qs[1] +
                                  (long long)node * a.qs[2] + 16 * h;
        mask_at[q] = ((long long)j.b * a.n + node) * a.W;
#pragma unroll
        for (int i = 0; i < NJ; ++i) {
            qf[q][2 * i] = __builtin_bit_cast(bf16x8, *(const u32x4*)(p + 32 * i));
            qf[q][2 * i + 1] = __builtin_bit_cast(bf16x8, *(const u32x4*)(p + 32 * i + 8));
        }
    }
    const float c = a.scale_log2;
    float ref[QB], l[QB];
    f32x16 o[QB][DB];
#pragma unroll
    for (int q = 0; q < QB; ++q) {
        ref[q] = kNoRef; l[q] = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[q][d][v] = 0.f;
    }

    unsigned short* const s_v = (unsigned short*)s_mem + wave * VW;
    const int tr_j = (lane & 15) >> 2, vx = ((lane >> 4) & 1) ^ v_swizzle<D>(tr_j);
    const unsigned short* const v_read = s_v + (4 * h + tr_j) * D + 4 * (lane & 3);

    // the products of a block: kf(i) the A operands of its keys, V in s_v
    auto block = [&](const bf16x8 (&kf)[2 * NJ], auto bits_of, bool all) {
        u32x4 p[QB][2];
#pragma unroll
        for (int q = 0; q < QB; ++q) {
            f32x16 s;
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
            for (int i = 0; i < 2 * NJ; ++i) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], qf[q][i], s, 0, 0, 0);
            if (!all) hide(s, bits_of(q), h);
            softmax_block<DB>(s, c, ref[q], l[q], o[q], p[q]);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const bf16x8 vf = column_of_8_rows(v_read + 16 * u * D + (((2 * d) ^ vx) << 4), 8 * D);
#pragma unroll
                for (int q = 0; q < QB; ++q)
                    o[q][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, p[q][u]), o[q][d], 0, 0, 0);
            }
    };
    auto wave_fence = [] {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };

    // ---- cache ----
    const int blocks = (j.len + 31) / 32, ptiles = (j.len + kTile - 1) / kTile;
    struct Raw {
        u32x4 k[KL], v[KL];
        int ke[2], ve[2];
        unsigned seen;
    };
    const int32_t* const table = a.table + (long long)j.b * a.max_pages;
    const int ps = 1 << a.ps_log2, page_last = max(j.len - 1, 0) >> a.ps_log2;
    constexpr int ESZ = KV8 ? 1 : 2;
    const unsigned k_lane = (unsigned)(l32 & 15) * (unsigned)(a.kps[2] * ESZ) + 16 * h * ESZ;
    bool bad = false;
    auto load = [&](int i, Raw& r) {                     // block i: cache rows 32 i .. 32 i + 31
        const int key0 = 32 * i, rem = j.len - key0;
        r.seen = rem >= 32 ? 0xffffffffu : (1u << rem) - 1;
        const unsigned char *kb[2], *vb[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            int page = table[min((key0 + 16 * e) >> a.ps_log2, page_last)];
            if ((unsigned)page >= (unsigned)a.num_pages) {
                if (key0 + 16 * e < j.len) bad = true;
                page = 0;
                r.seen &= e ? 0xffffu : 0xffff0000u;
            }
            const int row = (key0 + 16 * e) & (ps - 1);
            kb[e] = a.kp + ((long long)page * a.kps[0] + (long long)hk * a.kps[1] + (long long)row * a.kps[2]) * ESZ;
            vb[e] = a.vp + ((long long)page * a.vps[0] + (long long)hk * a.vps[1] + (long long)row * a.vps[2]) * ESZ;
            if constexpr (KV8) {
                r.ke[e] = a.k_exp[(long long)page * a.kv_heads + hk];
                r.ve[e] = a.v_exp[(long long)page * a.kv_heads + hk];
            }
        }
        const unsigned char* const km = (l32 & 16 ? kb[1] : kb[0]) + k_lane;
#pragma unroll
        for (int n = 0; n < KL; ++n) r.k[n] = *(const u32x4*)(km + (KV8 ? 32 * n : 64 * (n >> 1) + 16 * (n & 1)));
#pragma unroll
        for (int n = 0; n < KL; ++n) {
            const int row = n * RPL, e = row >> 4;       // rows row .. row + RPL - 1 of the block
            r.v[n] = *(const u32x4*)(vb[e] + (unsigned)((row & 15) + lane / CPR) * (unsigned)(a.vps[2] * ESZ) + 16 * (lane % CPR));
        }
    };
    auto use = [&](Raw& r) {
        bf16x8 kf[2 * NJ];
        if constexpr (KV8) {
            const float ks = exp_scale(l32 & 16 ? r.ke[1] : r.ke[0]);
#pragma unroll
            for (int i = 0; i < NJ; ++i) {
                u32x4 lo, hi;
                widen16(r.k[i], ks, lo, hi);
                kf[2 * i] = __builtin_bit_cast(bf16x8, lo);
                kf[2 * i + 1] = __builtin_bit_cast(bf16x8, hi);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2 * NJ; ++i) kf[i] = __builtin_bit_cast(bf16x8, r.k[i]);
        }
        const float vs[2] = {KV8 ? exp_scale(r.ve[0]) : 1.f, KV8 ? exp_scale(r.ve[1]) : 1.f};
        wave_fence();
#pragma unroll
        for (int n = 0; n < KL; ++n) {
            const int row = n * RPL + lane / CPR, at = lane % CPR;
            u32x4 w = r.v[n];
            if (r.seen != 0xffffffffu && !(r.seen >> row & 1)) w = u32x4{0, 0, 0, 0};
            if constexpr (KV8) {
                u32x4 lo, hi;
                widen16(w, vs[(n * RPL) >> 4], lo, hi);
                u32x4* const to = (u32x4*)(s_v + row * D + ((at ^ v_swizzle<D>(row)) << 4));
                to[0] = lo; to[1] = hi;
            } else {
                *(u32x4*)(s_v + row * D + (((at >> 1) ^ v_swizzle<D>(row)) << 4) + 8 * (at & 1)) = w;
            }
        }
        wave_fence();
        const unsigned seen = r.seen;
        block(kf, [&](int) { return seen; }, seen == 0xffffffffu);
    };
    {
        const int end = min(2 * j.t1, blocks);
        int i = 2 * j.t0 + wave;
        Raw r0, r1;
        if (i < end) load(i, r0);
        while (i < end) {
            if (i + 4 < end) load(i + 4, r1);
            use(r0);
            i += 4;
            if (i >= end) break;
            if (i + 4 < end) load(i + 4, r0);
            use(r1);
            i += 4;
        }
    }
    if (bad && lane == 0)
        __hip_atomic_fetch_or(a.sync + OT_ATTN_STATUS_OFFSET / 4, OT_ATTN_STATUS_BAD_PAGE, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);

    // ---- tree ----
    const int tt0 = max(j.t0 - ptiles, 0), tt1 = j.t1 - ptiles;
    if (tt1 > tt0) {
        union_masks(a, j.b, tt0, tt1, s_union, 256);
        const unsigned short* const kt = (const unsigned short*)a.Kt + (long long)j.b * a.kts[0] + (long long)hk * a.kts[1];
        const unsigned short* const vt = (const unsigned short*)a.Vt + (long long)j.b * a.vts[0] + (long long)hk * a.vts[1];
        for (int i = 2 * tt0 + wave; i < 2 * tt1 && 32 * i < a.tree_keys; i += 4) {
            const int last = a.tree_keys - 1;
            const unsigned any = (unsigned)(s_union[(i >> 1) - tt0] >> (32 * (i & 1)));
            const unsigned short* const kr = kt + (long long)min(32 * i + l32, last) * a.kts[2] + 16 * h;
            bf16x8 kf[2 * NJ];
#pragma unroll
            for (int n = 0; n < NJ; ++n) {
                kf[2 * n] = __builtin_bit_cast(bf16x8, *(const u32x4*)(kr + 32 * n));
                kf[2 * n + 1] = __builtin_bit_cast(bf16x8, *(const u32x4*)(kr + 32 * n + 8));
            }
            constexpr int P = D / 8, R = 64 / P;
            wave_fence();
#pragma unroll
            for (int n = 0; n < 32 / R; ++n) {
                const int row = n * R + lane / P, at = lane % P;
                u32x4 w = *(const u32x4*)(vt + (long long)min(32 * i + row, last) * a.vts[2] + 8 * at);
                if (!(any >> row & 1)) w = u32x4{0, 0, 0, 0};
                *(u32x4*)(s_v + row * D + (((at >> 1) ^ v_swizzle<D>(row)) << 4) + 8 * (at & 1)) = w;
            }
            wave_fence();
            const unsigned tail = 32 * i + 32 <= a.tree_keys ? 0xffffffffu : (1u << (a.tree_keys - 32 * i)) - 1;
            block(kf, [&](int q) { return (unsigned)(a.mask[mask_at[q] + (i >> 1)] >> (32 * (i & 1))) & tail; }, false);
        }
    }

    // ---- the four wavefronts' results ----
#pragma unroll
    for (int q = 0; q < QB; ++q) {
        const float sum = xhalf_sum(l[q]);
        if (h == 0) { s_ref[wave][q * 32 + l32] = ref[q]; s_sum[wave][q * 32 + l32] = sum; }
    }
    __syncthreads();
    float* const s_o = (float*)s_mem;
    const int row = tid >> 3, col = (tid & 7) * 8;
#pragma unroll
    for (int q = 0; q < QB; ++q) {
        const float M4 = fmaxf(fmaxf(s_ref[0][q * 32 + l32], s_ref[1][q * 32 + l32]), fmaxf(s_ref[2][q * 32 + l32], s_ref[3][q * 32 + l32]));
        const float f = __builtin_amdgcn_exp2f(ref[q] - M4);
        float M = kNoRef, L = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, s_ref[w][q * 32 + row]);
#pragma unroll
        for (int w = 0; w < 4; ++w) L += s_sum[w][q * 32 + row] * __builtin_amdgcn_exp2f(s_ref[w][q * 32 + row] - M);
        const bool live = q * 32 + row < rows;
#pragma unroll
        for (int part = 0; part < D / 64; ++part) {
            __syncthreads();
#pragma unroll
            for (int d = 0; d < 2; ++d)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const f32x16& x = o[q][2 * part + d];
                    *(f32x4*)(s_o + (wave * 32 + l32) * OST + 32 * d + 8 * v + 4 * h) =
                        f32x4{x[4 * v] * f, x[4 * v + 1] * f, x[4 * v + 2] * f, x[4 * v + 3] * f};
                }
            __syncthreads();
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const f32x4 lo = *(const f32x4*)(s_o + (w * 32 + row) * OST + col), hi = *(const f32x4*)(s_o + (w * 32 + row) * OST + col + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) { y[e] += lo[e]; y[4 + e] += hi[e]; }
            }
            if (!live) continue;
            if (j.splits == 1) {
                const float inv = inverse(L);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] *= inv;
                store8<OT_BF16>(out_row(a, j.b, hk, row0 + q * 32 + row), 64 * part + col, y);
            } else {
                const size_t at = (size_t)(j.slot + j.split * a.units) * a.slot_rows + q * 32 + row;
#pragma unroll
                for (int e = 0; e < 4; ++e) put2(a.part + at * D + 64 * part + col + 2 * e, y[2 * e], y[2 * e + 1]);
                if (part == 0 && col == 0) put2(a.part_ml + at * 2, M, L);
            }
        }
    }
    if (j.splits > 1) join_splits<D, 256>(a, j, hk, row0, rows);
}

// ---------------------------------------------------------------------------
// Many rows: 32 packed query rows per wavefront, NW wavefronts, all of them over every 64-key tile of the job.
// Bound by the matrix cores and the exponentials.  A tile is requested into registers two tiles ahead, widened to bf16 on its
// way into LDS one tile ahead, and read by all wavefronts (one barrier per tile).
//   K [64][D]: 16-byte piece c of row r at c ^ (r mod D/8);  V [64][D]: 32-byte segment g of row r at g ^ v_swizzle(r)
// ---------------------------------------------------------------------------
template <int D, bool KV8, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_tiles_kernel(const PagedArgs a) {
    constexpr int NT = 64 * NW, DB = D / 32, SL = D / 16, CPR = D / 8;
    constexpr int ESZ = KV8 ? 1 : 2;
    constexpr int CPM = D * ESZ / 16;                  // 16-byte pieces per row in memory
    constexpr int CH = kTile * CPM / NT;               // pieces of K per thread and tile, and of V
    constexpr int CHT = kTile * CPR / NT;              // the same of a tree tile
    static_assert(CH >= 1 && 64 / CPM <= 16, "a piece per thread; a wavefront's rows lie in one page");
    extern __shared__ __attribute__((aligned(16))) unsigned short s_kv[];       // [2][K, V][64][D]
    __shared__ u64 s_union[OT_MAX_TREE_KEYS / 64];
    constexpr int BUF = 2 * kTile * D;
    const Job j = find_job(a, blockIdx.x);
    if (j.none) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, h = lane >> 5;
    const int hk = j.unit / a.row_blocks, rb = j.unit - hk * a.row_blocks;
    const int rows_all = a.g * a.n, row0 = rb * 32 * NW, rows = min(32 * NW, rows_all - row0);

    bf16x8 qf[SL];
    long long mask_at;
    {
        const int rho = min(row0 + wave * 32 + l32, rows_all - 1), head = rho / a.n, node = rho - head * a.n;
        const unsigned short* p = (const unsigned short*)a.Q + (long long)j.b * a.qs[0] + (long long)(hk * a.g + head) * a.qs[1] +
                                  (long long)node * a.qs[2] + 8 * h;
        mask_at = ((long long)j.b * a.n + node) * a.W;
#pragma unroll
        for (int i = 0; i < SL; ++i) qf[i] = __builtin_bit_cast(bf16x8, *(const u32x4*)(p + 16 * i));
    }
    const float c = a.scale_log2;
    float ref = kNoRef, l = 0.f;
    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[d][v] = 0.f;
    const int tr_j = (lane & 15) >> 2, vx = ((lane >> 4) & 1) ^ v_swizzle<D>(tr_j), kx = l32 & (CPR - 1);

    const int ptiles = (j.len + kTile - 1) / kTile;
    const int32_t* const table = a.table + (long long)j.b * a.max_pages;
    const int ps = 1 << a.ps_log2, page_last = max(j.len - 1, 0) >> a.ps_log2;
    const int tt0 = max(j.t0 - ptiles, 0), tt1 = j.t1 - ptiles;
    if (tt1 > tt0) union_masks(a, j.b, tt0, tt1, s_union, NT);
    bool bad = false;

    struct Raw {
        u32x4 k[CHT], v[CHT];          // a cache tile uses the first CH of each
        int ke[CH], ve[CH];
        u64 seen;                      // rows of the tile that exist (V rows that enter the product)
        u64 mask;                      // tree tile: the words of this lane's query
    };
    const int m_row = tid / CPM, m_at = tid % CPM;       // row of the tile and piece of this thread's first request; CH apart NT / CPM rows
    auto load = [&](int t, Raw& r) {
        if (t < ptiles) {
            const int key0 = t * kTile, rem = j.len - key0;
            r.seen = rem >= kTile ? ~0ull : (1ull << rem) - 1;
            for (int i = 0; i < kTile >> min(a.ps_log2, 6); ++i) {          // pages of the tile that are none
                const int k0 = key0 + (i << min(a.ps_log2, 6));
                if (k0 < j.len && (unsigned)table[k0 >> a.ps_log2] >= (unsigned)a.num_pages) {
                    bad = true;
                    const u64 rows_of = ps >= 64 ? ~0ull : ((1ull << (ps & 63)) - 1) << (k0 - key0);
                    r.seen &= ~rows_of;
                }
            }
#pragma unroll
            for (int n = 0; n < CH; ++n) {
                const int first = uniform(wave * (64 / CPM)) + n * (NT / CPM);                    // of the wavefront's rows
                int page = table[min((key0 + first) >> a.ps_log2, page_last)];
                page = (unsigned)page < (unsigned)a.num_pages ? page : 0;
                const int row = (key0 + first) & (ps - 1);
                const unsigned char* const kb = a.kp + ((long long)page * a.kps[0] + (long long)hk * a.kps[1] + (long long)row * a.kps[2]) * ESZ;
                const unsigned char* const vb = a.vp + ((long long)page * a.vps[0] + (long long)hk * a.vps[1] + (long long)row * a.vps[2]) * ESZ;
                r.k[n] = *(const u32x4*)(kb + (unsigned)(lane / CPM) * (unsigned)(a.kps[2] * ESZ) + 16 * m_at);
                r.v[n] = *(const u32x4*)(vb + (unsigned)(lane / CPM) * (unsigned)(a.vps[2] * ESZ) + 16 * m_at);
                if constexpr (KV8) {
                    r.ke[n] = a.k_exp[(long long)page * a.kv_heads + hk];
                    r.ve[n] = a.v_exp[(long long)page * a.kv_heads + hk];
                }
            }
        } else {
            const int tt = t - ptiles, last = a.tree_keys - 1;
            const int rem = a.tree_keys - tt * kTile;
            const u64 tail = rem >= kTile ? ~0ull : (1ull << rem) - 1;
            r.seen = s_union[tt - tt0] & tail;
            r.mask = a.mask[mask_at + tt] & tail;
            const unsigned short* const kt = (const unsigned short*)a.Kt + (long long)j.b * a.kts[0] + (long long)hk * a.kts[1];
            const unsigned short* const vt = (const unsigned short*)a.Vt + (long long)j.b * a.vts[0] + (long long)hk * a.vts[1];
#pragma unroll
            for (int n = 0; n < CHT; ++n) {
                const int row = min(tt * kTile + tid / CPR + n * (NT / CPR), last);
                r.k[n] = *(const u32x4*)(kt + (long long)row * a.kts[2] + 8 * (tid % CPR));
                r.v[n] = *(const u32x4*)(vt + (long long)row * a.vts[2] + 8 * (tid % CPR));
            }
        }
    };
    auto stage = [&](int t, Raw& r, int buf) {
        unsigned short* const sk = s_kv + buf * BUF;
        unsigned short* const sv = sk + kTile * D;
        if (KV8 && t < ptiles) {
#pragma unroll
            for (int n = 0; n < CH; ++n) {
                const int row = m_row + n * (NT / CPM);
                u32x4 lo, hi, w = r.v[n];
                widen16(r.k[n], exp_scale(r.ke[n]), lo, hi);
                *(u32x4*)(sk + row * D + (((2 * m_at) ^ (row & (CPR - 1))) << 3)) = lo;
                *(u32x4*)(sk + row * D + (((2 * m_at + 1) ^ (row & (CPR - 1))) << 3)) = hi;
                if (r.seen != ~0ull && !(r.seen >> row & 1)) w = u32x4{0, 0, 0, 0};
                widen16(w, exp_scale(r.ve[n]), lo, hi);
                u32x4* const to = (u32x4*)(sv + row * D + ((m_at ^ v_swizzle<D>(row)) << 4));
                to[0] = lo; to[1] = hi;
            }
        } else {
#pragma unroll
            for (int n = 0; n < CHT; ++n) {
                const int row = tid / CPR + n * (NT / CPR), at = tid % CPR;
                u32x4 w = r.v[n];
                *(u32x4*)(sk + row * D + ((at ^ (row & (CPR - 1))) << 3)) = r.k[n];
                if (r.seen != ~0ull && !(r.seen >> row & 1)) w = u32x4{0, 0, 0, 0};
                *(u32x4*)(sv + row * D + (((at >> 1) ^ v_swizzle<D>(row)) << 4) + 8 * (at & 1)) = w;
            }
        }
    };
    auto compute = [&](int t, u64 visible, int buf) {
        const unsigned short* const sk = s_kv + buf * BUF;
        const unsigned short* const sv = sk + kTile * D;
        u32x4 p[2][2];
        f32x16 s[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int v = 0; v < 16; ++v) s[kb][v] = 0.f;
#pragma unroll
            for (int i = 0; i < SL; ++i) {
                const bf16x8 kf = __builtin_bit_cast(bf16x8, *(const u32x4*)(sk + (32 * kb + l32) * D + (((2 * i + h) ^ kx) << 3)));
                s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[i], s[kb], 0, 0, 0);
            }
        }
        if (t >= ptiles || visible != ~0ull) {
            hide(s[0], (unsigned)visible, h);
            hide(s[1], (unsigned)(visible >> 32), h);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            softmax_block<DB>(s[kb], c, ref, l, o, p[kb]);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const bf16x8 vf = column_of_8_rows(sv + (32 * kb + 16 * u + 4 * h + tr_j) * D + (((2 * d) ^ vx) << 4) + 4 * (lane & 3), 8 * D);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, p[kb][u]), o[d], 0, 0, 0);
                }
        }
    };

    if (j.t0 < j.t1) {
        Raw ra, rb_;
        u64 vis[2];
        auto visible_of = [&](int t, const Raw& r) { return t < ptiles ? r.seen : r.mask; };
        load(j.t0, ra);
        if (j.t0 + 1 < j.t1) load(j.t0 + 1, rb_);
        stage(j.t0, ra, 0);
        vis[0] = visible_of(j.t0, ra);
        int t = j.t0;
        while (true) {                                   // tile t is staged in buffer 0, tile t + 1 on its way in rb_
            __syncthreads();
            if (t + 2 < j.t1) load(t + 2, ra);
            if (t + 1 < j.t1) { stage(t + 1, rb_, 1); vis[1] = visible_of(t + 1, rb_); }
            compute(t, vis[0], 0);
            if (++t >= j.t1) break;
            __syncthreads();
            if (t + 2 < j.t1) load(t + 2, rb_);
            if (t + 1 < j.t1) { stage(t + 1, ra, 0); vis[0] = visible_of(t + 1, ra); }
            compute(t, vis[1], 1);
            if (++t >= j.t1) break;
        }
    }
    if (bad && lane == 0)
        __hip_atomic_fetch_or(a.sync + OT_ATTN_STATUS_OFFSET / 4, OT_ATTN_STATUS_BAD_PAGE, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);

    const float L = xhalf_sum(l);
    const int row = wave * 32 + l32;
    if (j.splits == 1) {
        if (row >= rows) return;
        const float inv = inverse(L);
        unsigned short* const to = out_row(a, j.b, hk, row0 + row);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                *(uint2*)(to + 32 * d + 8 * v + 4 * h) = uint2{pack_bf16(o[d][4 * v] * inv, o[d][4 * v + 1] * inv),
                                                               pack_bf16(o[d][4 * v + 2] * inv, o[d][4 * v + 3] * inv)};
        return;
    }
    if (row < rows) {
        const size_t at = (size_t)(j.slot + j.split * a.units) * a.slot_rows + row;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int v = 0; v < 8; ++v) put2(a.part + at * D + 32 * d + 8 * (v >> 1) + 4 * h + 2 * (v & 1), o[d][2 * v], o[d][2 * v + 1]);
        if (h == 0) put2(a.part_ml + at * 2, ref, L);
    }
    join_splits<D, NT>(a, j, hk, row0, rows);
}

__global__ __launch_bounds__(256) void clear_words_kernel(unsigned int* w) { w[blockIdx.x * 256 + threadIdx.x] = 0; }

struct PagedPlan {
    int rows, row_blocks, units, split, target, least, grid, slot_rows;
    size_t bytes;
};

PagedPlan plan_paged(const ot_paged_attn_params& p, const ot_paged_cache& c) {
    PagedPlan pl;
    const int R = p.q_heads / c.kv_heads * p.n;
    // (an 8-bit tile of 64-wide heads is 256 pieces of 16 bytes: four wavefronts)
    pl.rows = R <= 32 ? 32 : R <= 64 ? 64 : R <= 128 || (c.head_dim == 64 && c.dtype == OT_E4M3) ? 128 : 256;
    pl.row_blocks = (R + pl.rows - 1) / pl.rows;
    pl.units = c.kv_heads * pl.row_blocks;
    const long long all = (long long)p.batch * pl.units;
    pl.split = p.batch <= kSplitBatch && all <= kCounters;
    pl.target = pl.rows == 32 || pl.rows == 128 ? 512 : 256;
    pl.least = pl.rows <= 64 ? 2 : 4;
    const long long tiles = ((long long)c.max_pages * c.page_size + kTile - 1) / kTile + (p.tree_keys + kTile - 1) / kTile;
    const long long most = std::max<long long>(all, pl.target);
    pl.grid = (int)(pl.split ? std::min(most, all * ((tiles + pl.least - 1) / pl.least)) : all);
    pl.slot_rows = std::min(R, pl.rows);
    pl.bytes = OT_PAGED_SYNC_BYTES + (pl.split ? (size_t)pl.grid * pl.slot_rows * (c.head_dim + 2) * 4 : 0);
    return pl;
}

int validate_paged(const ot_paged_attn_params* p, const ot_paged_cache* c, bool pointers) {
    if (!p) return OT_ERR_INVALID_ARG;
    const int st = validate_cache(c, pointers);
    if (st != OT_OK) return st;
    if (p->batch < 1 || p->q_heads < 1 || p->n < 1 || p->tree_keys < 0 || p->q_heads % c->kv_heads) return OT_ERR_INVALID_ARG;
    if (!(p->softmax_scale >= 0.f) || p->softmax_scale > 3.402823466e38f) return OT_ERR_INVALID_ARG;
    if (p->n > OT_MAX_NODES || p->tree_keys > OT_MAX_TREE_KEYS) return OT_ERR_UNSUPPORTED;
    if ((long long)p->batch * p->q_heads > 65535) return OT_ERR_UNSUPPORTED;
    const int64_t* st4[4] = {p->q_strides, p->o_strides, p->kt_strides, p->vt_strides};
    for (int t = 0; t < (p->tree_keys ? 4 : 2); ++t)
        for (int i = 0; i < 3; ++i)
            if (st4[t][i] < 0 || st4[t][i] % 8) return OT_ERR_INVALID_ARG;
    return OT_OK;
}

template <int D, bool KV8>
int launch_paged(const PagedArgs& a, const PagedPlan& pl, hipStream_t s) {
    constexpr size_t lds = (size_t)2 * 2 * kTile * D * 2;
    if (pl.rows == 32) hipLaunchKernelGGL((paged_rows_kernel<D, KV8, 1>), dim3(pl.grid), dim3(256), 0, s, a);
    else if (pl.rows == 64) hipLaunchKernelGGL((paged_rows_kernel<D, KV8, 2>), dim3(pl.grid), dim3(256), 0, s, a);
    else if (pl.rows == 128) {
        OT_HIP_CHECK(hipFuncSetAttribute((const void*)paged_tiles_kernel<D, KV8, 4>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        hipLaunchKernelGGL((paged_tiles_kernel<D, KV8, 4>), dim3(pl.grid), dim3(256), lds, s, a);
    } else if constexpr (!(D == 64 && KV8)) {
        OT_HIP_CHECK(hipFuncSetAttribute((const void*)paged_tiles_kernel<D, KV8, 8>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        hipLaunchKernelGGL((paged_tiles_kernel<D, KV8, 8>), dim3(pl.grid), dim3(512), lds, s, a);
    }
    OT_HIP_CHECK(hipGetLastError());
    return OT_OK;
}

}  // namespace
}  // namespace ot

using namespace ot;

extern "C" {

size_t ot_paged_attn_workspace_bytes(const ot_paged_attn_params* p, const ot_paged_cache* cache) {
    return validate_paged(p, cache, false) == OT_OK ? plan_paged(*p, *cache).bytes : 0;
}

int ot_paged_attn_workspace_prepare(void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!workspace || (uintptr_t)workspace % 16) return OT_ERR_INVALID_ARG;
    if (workspace_bytes < OT_PAGED_SYNC_BYTES) return OT_ERR_WORKSPACE_TOO_SMALL;
    hipLaunchKernelGGL(clear_words_kernel, dim3(OT_PAGED_SYNC_BYTES / 4 / 256), dim3(256), 0, (hipStream_t)hip_stream, (unsigned int*)workspace);
    OT_HIP_CHECK(hipGetLastError());
    return OT_OK;
}

int ot_tree_verify_attention_paged(const ot_paged_attn_params* p, const ot_paged_cache* cache, const void* Q, const void* K_tree,
                                   const void* V_tree, const int32_t* prefix_len, const uint64_t* mask, void* O, void* workspace,
                                   size_t workspace_bytes, void* hip_stream) {
    const int st = validate_paged(p, cache, true);
    if (st != OT_OK) return st;
    if (!Q || !O || !prefix_len || !workspace) return OT_ERR_INVALID_ARG;
    if (p->tree_keys && (!K_tree || !V_tree || !mask || (uintptr_t)K_tree % 16 || (uintptr_t)V_tree % 16 || (uintptr_t)mask % 8)) return OT_ERR_INVALID_ARG;
    if ((uintptr_t)Q % 16 || (uintptr_t)O % 16 || (uintptr_t)workspace % 16 || (uintptr_t)prefix_len % 4) return OT_ERR_INVALID_ARG;
    const PagedPlan pl = plan_paged(*p, *cache);
    if (workspace_bytes < pl.bytes) return OT_ERR_WORKSPACE_TOO_SMALL;
    PagedArgs a;
    a.Q = Q; a.Kt = K_tree; a.Vt = V_tree; a.O = O;
    a.kp = (const unsigned char*)cache->k_pages; a.vp = (const unsigned char*)cache->v_pages;
    a.k_exp = cache->k_exp; a.v_exp = cache->v_exp; a.table = cache->page_table;
    a.prefix_len = prefix_len; a.mask = mask;
    a.sync = (unsigned int*)workspace;
    a.part = (float*)((char*)workspace + OT_PAGED_SYNC_BYTES);
    a.part_ml = a.part + (size_t)pl.grid * pl.slot_rows * cache->head_dim;
    a.batch = p->batch; a.kv_heads = cache->kv_heads; a.g = p->q_heads / cache->kv_heads; a.n = p->n;
    a.tree_keys = p->tree_keys; a.W = OT_MASK_WORDS(p->tree_keys);
    a.row_blocks = pl.row_blocks; a.units = pl.units;
    a.num_pages = cache->num_pages; a.max_pages = cache->max_pages; a.ps_log2 = log2_of(cache->page_size);
    a.split = pl.split; a.target = pl.target; a.least = pl.least; a.slot_rows = pl.slot_rows;
    a.scale_log2 = (p->softmax_scale != 0.f ? p->softmax_scale : 1.0f / sqrtf((float)cache->head_dim)) * kLog2e;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = p->q_strides[i]; a.kts[i] = p->kt_strides[i]; a.vts[i] = p->vt_strides[i]; a.os[i] = p->o_strides[i];
        a.kps[i] = cache->k_strides[i]; a.vps[i] = cache->v_strides[i];
    }
    hipStream_t s = (hipStream_t)hip_stream;
    if (cache->dtype == OT_E4M3) return cache->head_dim == 128 ? launch_paged<128, true>(a, pl, s) : launch_paged<64, true>(a, pl, s);
    return cache->head_dim == 128 ? launch_paged<128, false>(a, pl, s) : launch_paged<64, false>(a, pl, s);
}

}  // extern "C"
