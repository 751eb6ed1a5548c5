// Tree-masked attention over a paged cache (opttree.h: ot_tree_verify_attention_paged).
//   O[i] = sum_j softmax_j(scale q_i . k_j) v_j,  j over cache rows (found through the page table) and visible tree rows
//
// The keys of a (sequence, KV head) are cut into 64-key tiles, cache first, then tree.  A job is a range of tiles for one block
// of packed query rows (GQA: the rows of the g query heads of a KV head are stacked, row = head * n + node); a workgroup is a job.
// Softmax in one pass: running reference and sum per query, fp32; a range leaves an un-normalised partial and the last job of
// a row block to finish merges them (tickets).
//
// Ranges are decided on the device, from the lengths as they are (find_job): a page table gives every sequence room for
// the longest context, so the host's bound on a length says little, and lengths in a serving batch differ.  Batches whose (sequence, KV
// head, row block) triples fill the card by themselves are not cut, whatever their lengths (plan_paged).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "internal.h"
#include "paged.hpp"
#include "rope.hpp"

namespace ot {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned long long u64;

constexpr float kLog2e = 1.4426950408889634f;
// Page numbers are read through the scalar cache (nothing writes the table while a call runs): as vector loads they would
// queue behind the K and V rows in flight, and waiting for one would wait for all of those.
typedef const int32_t __attribute__((address_space(4))) * scalar_int;
// Byte i of the array p, likewise: a scalar load has at least four bytes, those of the aligned word around it (p is aligned).
__device__ __forceinline__ int scalar_byte(const unsigned char* p, unsigned i) {
    return ((scalar_int)p)[i >> 2] >> (8 * (i & 3)) & 255;
}
constexpr int kTicketRows = 16;                              // up to so many rows of a block are joined by its last workgroup
constexpr int kSplitBatch = 256;                             // sequences of a batch whose contexts are cut into ranges
constexpr int kTile = 64;
// reference of a row that has seen nothing: from it a masked score gives 0 and any score moves the reference
constexpr float kNoRef = -3.402823466e38f;
// The reference follows the row's maximum only when that is this far ahead: probabilities up to 2^8 lose nothing in fp32 or in
// bf16, and most tiles then rescale nothing.
constexpr float kSlack = 8.f;

// What the first loads of a workgroup wait for, as leading scalar arguments: the hardware hands these over in registers at
// wavefront start (kernel-argument preload).
struct Lead {
    const int32_t *prefix_len, *table;
    int batch, kv_heads, row_blocks, max_pages, ps_log2, tiles_tree;
    int target;                  // jobs aimed at; 0: every sequence in one piece
    float apart;                 // what another range costs, in tiles
};
#define OT_LEAD_PARAMS const int32_t *l_prefix_len, const int32_t *l_table, const int l_batch, const int l_kv_heads, const int l_row_blocks, \
                       const int l_max_pages, const int l_ps_log2, const int l_tiles_tree, const int l_target, const float l_apart
#define OT_LEAD Lead{l_prefix_len, l_table, l_batch, l_kv_heads, l_row_blocks, l_max_pages, l_ps_log2, l_tiles_tree, l_target, l_apart}

struct PagedArgs {
    const void *Q, *Kt, *Vt;
    const unsigned char *k_exp, *v_exp;
    const uint64_t* mask;
    void* O;
    unsigned int* sync;
    float* part;                 // [job][rows of a block][D], then [job][rows][2] (reference, sum)
    float* part_ml;
    int2* joins;                 // [sequence][unit] (first job, ranges), for the launch that joins; null: the last job joins
    int kv_heads, g, n, tree_keys, W, row_blocks, units;          // units = kv_heads * row_blocks
    int num_pages;
    int block_rows, slot_rows;   // rows of a block, and of a partial
    float scale_log2;
    long long qs[3], kts[3], vts[3], os[3];
    unsigned k_page, v_page;     // page strides in units of 16 bytes
    unsigned k_row, v_row;       // row strides in bytes
    const unsigned char *kp, *vp;        // page 0
    long long k_head, v_head;    // head strides in bytes
};
// Rows `row` .. of a page, as an address that is the same in all lanes
__device__ __forceinline__ const unsigned char* row_of(const unsigned char* head, unsigned page, unsigned page_stride, unsigned row, unsigned row_stride) {
    return head + ((u64)page * page_stride << 4) + row * row_stride;
}

__device__ __forceinline__ float xhalf_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float xhalf_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ int wave_sum_i(int v) { return rl(wave_incl_scan(v, 0), 63); }
__device__ __forceinline__ int wave_max_i(int v) {
    v = max(v, dpp_i<DPP_QUAD_XOR1>(v, v));
    v = max(v, dpp_i<DPP_QUAD_XOR2>(v, v));
    v = max(v, dpp_i<DPP_ROW_HALF_MIRROR>(v, v));
    v = max(v, dpp_i<DPP_ROW_MIRROR>(v, v));
    return max(max(rl(v, 0), rl(v, 16)), max(rl(v, 32), rl(v, 48)));
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

// Which range of which unit workgroup `wg` computes; the same in every lane of the workgroup.  Tiles per range are about the
// fewest with which all jobs together are no more than `target`, and at least sqrt(T apart), T the tiles of the longest
// sequence: S ranges take T / S tiles and S joins of `apart` tiles each, which is least there.  Each sequence takes
// ceil(tiles / share) ranges of equal length.  Lane j holds sequences j, j + 64, ...
// Workgroups go to XCD wg % 8 in order; the row blocks of a KV head and range, which read the same rows, take consecutive
// places on one XCD, whose L2 they share (16 x 8 KV heads x 4 row blocks over 8192 keys: 322 MB fetched, not 1179; 535 us, not 545).
__device__ __forceinline__ Job find_job(const Lead& a, unsigned int* sync, int wg) {
    const int lane = threadIdx.x & 63, cap = a.max_pages << a.ps_log2;
    const int units = a.kv_heads * a.row_blocks, place = wg >> 3, group = place / a.row_blocks;
    const int pair = group * 8 + (wg & 7), u = pair / a.kv_heads;        // KV head of u: a sequence, or a (sequence, range)
    Job j;
    j.none = false;
    j.unit = (pair - u * a.kv_heads) * a.row_blocks + place - group * a.row_blocks;
    int raw;
    if (!a.target) {
        j.b = u;
        j.splits = 1; j.split = 0; j.slot = 0;
        if (j.b >= a.batch) { j.none = true; return j; }
        raw = a.prefix_len[j.b];
    } else {
        constexpr int NL = kSplitBatch / 64;
        const int target = a.target;
        int len[NL], T[NL], S[NL], most = 0;
        float total = 0.f;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int b = lane + 64 * i;
            len[i] = b < a.batch ? a.prefix_len[b] : 0;
        }
#pragma unroll
        for (int i = 0; i < NL; ++i)
            if (i == 0 || a.batch > 64 * i) {
                T[i] = lane + 64 * i < a.batch ? (min(max(len[i], 0), cap) + kTile - 1) / kTile + a.tiles_tree : 0;
                total += (float)wave_sum_i(T[i]);
                most = max(most, wave_max_i(T[i]));
            }
        int share = max(1, min(most, (int)ceilf(fmaxf(total * (float)units / (float)target, sqrtf((float)most * a.apart)))));
        int jobs;
        while (true) {
            jobs = 0;
#pragma unroll
            for (int i = 0; i < NL; ++i)
                if (i == 0 || a.batch > 64 * i) {
                    S[i] = lane + 64 * i < a.batch ? max(1, (int)((unsigned)(T[i] + share - 1) / (unsigned)share)) : 0;
                    jobs += wave_sum_i(S[i]);
                }
            if (jobs <= target / units || share >= most) break;
            share += max(1, share >> 4);
        }
        if (u >= jobs) { j.none = true; return j; }
        int before = 0;
        j.b = 0; j.split = 0; j.splits = 1; raw = 0;
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
                    raw = rl(len[i], l);
                }
                before = rl(end, 63);
            }
        j.slot = (u - j.split) * units + j.unit;         // of the unit's first range
    }
    raw = uniform(raw);
    j.len = min(max(raw, 0), cap);
    if (j.len != raw && threadIdx.x == 0)
        __hip_atomic_fetch_or(sync + OT_ATTN_STATUS_OFFSET / 4, OT_ATTN_STATUS_PREFIX_CLAMPED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    j.b = uniform(j.b); j.unit = uniform(j.unit); j.splits = uniform(j.splits); j.split = uniform(j.split); j.slot = uniform(j.slot);
    // the first ranges take a tile more each where the tiles do not divide
    const unsigned Tb = (unsigned)((j.len + kTile - 1) / kTile + a.tiles_tree), each = Tb / (unsigned)j.splits, over = Tb - each * (unsigned)j.splits;
    j.t0 = uniform((int)(each * (unsigned)j.split + min((unsigned)j.split, over)));
    j.t1 = uniform(j.t0 + (int)(each + ((unsigned)j.split < over ? 1u : 0u)));
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

// NB 32-key blocks of scores (lane: query l32, keys 8 (v/4) + 4 h + v%4 of a block) become probabilities; returns them packed as the
// B operands of the blocks' 16-key slabs, and rescales what the row has summed when the reference moves.
// A probability is rounded to bf16, the type that the matrix cores multiply V by; the sum is taken of the rounded ones, so that the
// weights of a row add up to one and equal values average to themselves.  Four sums side by side: two make a chain (8 x 8 KV heads of 64
// x 200 queries over 4000 keys 43.5 us, not 42.9).
template <int NB, int NO>
__device__ __forceinline__ void softmax_blocks(f32x16 (&s)[NB], float c, float& ref, float& l, f32x16 (&o)[NO], u32x4 (&p)[2 * NB]) {
    // (compiler-made maxima: an assembly one would not wait for the matrix instruction that makes its operand)
    float m = s[0][0];
#pragma unroll
    for (int i = 1; i + 1 < 16 * NB; i += 2) m = fmaxf(fmaxf(m, s[i / 16][i % 16]), s[(i + 1) / 16][(i + 1) % 16]);
    m = xhalf_max(fmaxf(m, s[NB - 1][15])) * c;
    if (__any(m > ref + kSlack)) {
        const float to = m > ref + kSlack ? m : ref, f = __builtin_amdgcn_exp2f(ref - to);
        l *= f;
#pragma unroll
        for (int d = 0; d < NO; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[d][v] *= f;
        ref = to;
    }
    const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int v = 0; v < 16; v += 2) {
            const bf16x2 pair = {(__bf16)__builtin_amdgcn_exp2f(fmaf(s[i][v], c, -ref)), (__bf16)__builtin_amdgcn_exp2f(fmaf(s[i][v + 1], c, -ref))};
            sum[v >> 1 & 3] = __builtin_amdgcn_fdot2_f32_bf16(pair, ones, sum[v >> 1 & 3], false);
            p[2 * i + (v >> 3)][v >> 1 & 3] = __builtin_bit_cast(unsigned, pair);
        }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    asm volatile("" : "+v"(l));                          // (here, not after the next products)
}
// STEPS products whose operands come from LDS, each requested AHEAD products before it is needed and held in that order (left to
// itself the compiler reads an operand right before its product, and every product waits for LDS).  read(i) returns the
// operands of product i, multiply(i, operands) does it; i is a constant in both.
template <int STEPS, int AHEAD, typename Read, typename Multiply>
__device__ __forceinline__ void pipelined(Read read, Multiply multiply) {
    decltype(read(0)) ring[AHEAD + 1];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ring[i] = read(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        if (i + AHEAD < STEPS) ring[(i + AHEAD) % (AHEAD + 1)] = read(i + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
        multiply(i, ring[i % (AHEAD + 1)]);
        __builtin_amdgcn_sched_barrier(0);
    }
}
// scores of keys whose bit is not set
__device__ __forceinline__ void hide(f32x16& s, unsigned bits, int h) {
    bits >>= 4 * h;
#pragma unroll
    for (int v = 0; v < 16; ++v)
        if (!(bits >> (8 * (v >> 2) + (v & 3)) & 1)) s[v] = -INFINITY;
}

// A float4 of a partial, past the caches either way
__device__ __forceinline__ __amdgpu_buffer_rsrc_t part_buffer(float* part) { return __builtin_amdgcn_make_buffer_rsrc(part, 0, 0x7fffffff, 0x00020000); }
constexpr int kDeviceScope = 16;             // cache policy of the buffer instructions: sc1
__device__ __forceinline__ void put4(__amdgpu_buffer_rsrc_t b, unsigned at, f32x4 v) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), b, (int)(at * 4), 0, kDeviceScope);
}
__device__ __forceinline__ f32x4 get4(__amdgpu_buffer_rsrc_t b, unsigned at) {
    return __builtin_bit_cast(f32x4, (u32x4)__builtin_amdgcn_raw_buffer_load_b128(b, (int)(at * 4), 0, kDeviceScope));
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

// Four columns of a row: all its ranges added up, in their order.  Everything a chunk of ranges needs is requested before the
// first of it is used.
template <int D, int CHUNK>
__device__ __forceinline__ f32x4 add_up(const PagedArgs& a, __amdgpu_buffer_rsrc_t part, int slot, int splits, int row, int col) {
    float M = kNoRef, L = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < splits; s0 += CHUNK) {
        float2 ml[CHUNK];
        f32x4 x[CHUNK];
#pragma unroll
        for (int s = 0; s < CHUNK; ++s) {
            const unsigned at = (unsigned)(slot + min(s0 + s, splits - 1) * a.units) * a.slot_rows + row;
            ml[s] = get2(a.part_ml + at * 2);
            x[s] = get4(part, at * D + col);
        }
        float to = M;
#pragma unroll
        for (int s = 0; s < CHUNK; ++s) to = fmaxf(to, ml[s].x);            // (a copy of the last range changes nothing)
        const float f = __builtin_amdgcn_exp2f(M - to);
        L *= f;
        o *= f;
#pragma unroll
        for (int s = 0; s < CHUNK; ++s) {
            const float w = s0 + s < splits ? __builtin_amdgcn_exp2f(ml[s].x - to) : 0.f;
            L += ml[s].y * w;
            o += x[s] * w;
        }
        M = to;
    }
    return o * inverse(L);
}
template <int D>
__device__ __forceinline__ void store_joined(const PagedArgs& a, int b, int hk, int rho, int col, f32x4 y) {
    *(uint2*)(out_row(a, b, hk, rho) + col) = uint2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
}

// After a workgroup has stored its partial.  Few rows: the last workgroup of a row block joins them (ticket).  Many: that would
// be one compute unit reading what all of them wrote (256 rows in 16 ranges: 50 us), so another launch joins, and the first
// range says where the partials are.
template <int D, int NT>
__device__ __forceinline__ void join_splits(const PagedArgs& a, const Job& j, int hk, int row0, int rows, int* s_last) {
    if (a.joins) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    unsigned int* const ticket = a.sync + 1024 + j.b * a.units + j.unit;
    if (threadIdx.x == 0)
        *s_last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)(j.splits - 1);
    __syncthreads();
    if (!*s_last) return;
    if (threadIdx.x == 0) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const auto part = part_buffer(a.part);
    for (int i = threadIdx.x; i < rows * (D / 4); i += NT) {
        const int row = i / (D / 4), col = i % (D / 4) * 4;
        store_joined<D>(a, j.b, hk, row0 + row, col, add_up<D, 16>(a, part, j.slot, j.splits, row, col));
    }
}
__device__ __forceinline__ void note_splits(const PagedArgs& a, const Job& j) {
    if (a.joins && j.split == 0 && threadIdx.x == 0) a.joins[j.b * a.units + j.unit] = int2{j.slot, j.splits};
}

// The launch that joins: a thread has four columns of a row
template <int D>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedArgs a) {
    const int2 from = a.joins[blockIdx.y];
    if (from.y == 1) return;
    const int b = blockIdx.y / a.units, unit = blockIdx.y - b * a.units, hk = unit / a.row_blocks, rb = unit - hk * a.row_blocks;
    const int row = blockIdx.x * (1024 / D) + threadIdx.x / (D / 4), col = threadIdx.x % (D / 4) * 4, rho = rb * a.block_rows + row;
    if (row >= a.slot_rows || rho >= a.g * a.n) return;
    store_joined<D>(a, b, hk, rho, col, add_up<D, 8>(a, part_buffer(a.part), from.x, from.y, row, col));
}

// ---------------------------------------------------------------------------
// Few rows: 32 packed query rows per wavefront, QW blocks of them per workgroup (1 or 2).
// Bound by the cache's bytes.  The four wavefronts are QW row blocks x KS streams of 32-key blocks and never wait for each
// other inside the loop: a wavefront requests its own 32 rows of K and V in whole rows, and passes them through a corner of LDS
// of its own, K as stored (a lane reads sixteen consecutive columns of its key and widens them; the order of the contraction
// in S^T = K Q^T is free, so they serve two instructions), V widened, in the layout that the transposing read turns into the
// operand of O^T += V^T P^T.  The next block is requested as soon as this one is in LDS; a deeper queue took registers that
// were not there and gained nothing (4 x 100000 keys: 172 us one block ahead, 177 two).  Pages are multiples of sixteen
// rows, so a block's page numbers and exponents are two scalars each, known a block earlier.  The streams' results meet in
// LDS at the end.
// Measured: 8 KV heads x 8 queries over 4 x 100000 keys in 8 bits (820 MB) 133 to 148 us, 5.5 to 6.2 TB/s; 8 KV heads x 4 over 1500 keys
// 10 us, a chain of eight trips to memory: length, page, exponents and rows, partial, ticket, partials.
// ---------------------------------------------------------------------------
template <int D, bool KV8, int QW>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_rows_kernel(OT_LEAD_PARAMS, const PagedArgs a) {
    constexpr int KS = 4 / QW;
    constexpr int DB = D / 32, NJ = D / 32;
    constexpr int ESZ = KV8 ? 1 : 2;
    constexpr int KL = KV8 ? NJ : 2 * NJ;              // 16-byte loads of K per lane and block; the same of V
    constexpr int CPR = D * ESZ / 16;                  // 16-byte pieces per row of V in memory
    constexpr int RPL = 64 / CPR;                      // rows of V per load instruction
    constexpr int VW = 32 * D;                         // a wavefront's V in LDS, 2-byte elements
    constexpr int KW = 32 * D * ESZ / 2;               // its K, as stored
    constexpr int OST = 68;                            // row stride of the exchange at the end
    constexpr int kLoop = 4 * (VW + KW) * 2, kEnd = 4 * 32 * OST * 4;
    // V and K of the four wavefronts, then Q.  The union of the masks takes the place of K once the cache is through, the
    // exchange that of V and K, its scalars that of Q: 80 KB at most, so that two workgroups share a compute unit.
    constexpr int kMem = kLoop > kEnd ? kLoop : kEnd;
    __shared__ __attribute__((aligned(16))) unsigned char s_mem[kMem + QW * 32 * D * 2];
    static_assert(sizeof(s_mem) <= 80 * 1024 && 4 * KW * 2 >= OT_MAX_TREE_KEYS / 8 && QW * 32 * D * 2 >= 4 * 32 * 8 + 4, "LDS");
    u64* const s_union = (u64*)(s_mem + 4 * VW * 2);
    float* const s_ref = (float*)(s_mem + kMem);                             // [4][32]
    float* const s_sum = s_ref + 4 * 32;
    int* const s_last = (int*)(s_sum + 4 * 32);
    const Job j = find_job(OT_LEAD, a.sync, blockIdx.x);
    if (j.none) return;
    note_splits(a, j);
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, h = lane >> 5;
    const int qb = wave % QW, ks = wave / QW;
    const int hk = j.unit / a.row_blocks, rb = j.unit - hk * a.row_blocks;
    const int rows_all = a.g * a.n, row0 = rb * QW * 32, rows = min(QW * 32, rows_all - row0);

    // Q in LDS, one copy per row block: lane (query l32, half h) reads columns 32 i + 16 h .. + 15, 16-byte piece p of query r at
    // p ^ (r mod D/8)
    unsigned short* const s_q = (unsigned short*)(s_mem + kMem);
    long long mask_at;
    {
        const int rho = min(row0 + qb * 32 + l32, rows_all - 1), head = rho / a.n, node = rho - head * a.n;
        mask_at = ((long long)j.b * a.n + node) * a.W;
        if (ks == 0) {
            const unsigned short* p = (const unsigned short*)a.Q + (long long)j.b * a.qs[0] + (long long)(hk * a.g + head) * a.qs[1] +
                                      (long long)node * a.qs[2];
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const int at = 2 * i + h;
                *(u32x4*)(s_q + (qb * 32 + l32) * D + ((at ^ (l32 & (D / 8 - 1))) << 3)) = *(const u32x4*)(p + 8 * at);
            }
        }
    }
    __syncthreads();
    const unsigned short* const q_row = s_q + (qb * 32 + l32) * D;
    auto q_frag = [&](int i) {                           // piece 4 (i / 2) + 2 h + i % 2
        return __builtin_bit_cast(bf16x8, *(const u32x4*)(q_row + (((4 * (i >> 1) + 2 * h + (i & 1)) ^ (l32 & (D / 8 - 1))) << 3)));
    };
    const float c = a.scale_log2;
    float ref = kNoRef, l = 0.f;
    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[d][v] = 0.f;

    unsigned short* const s_v = (unsigned short*)s_mem + wave * VW;
    // K rows in LDS: 16-byte piece c of row r at c ^ (the row's number among those that share a 256-byte line's place)
    unsigned short* const s_k = (unsigned short*)s_mem + 4 * VW + wave * KW;
    auto k_at = [](int row, int piece) { return row * (CPR * 8) + ((piece ^ ((row / (16 / CPR)) & (CPR - 1))) << 3); };
    const int tr_j = (lane & 15) >> 2, vx = ((lane >> 4) & 1) ^ v_swizzle<D>(tr_j);
    const unsigned short* const v_read = s_v + (4 * h + tr_j) * D + 4 * (lane & 3);
    // probabilities of a block's scores, times V in s_v
    auto finish = [&](f32x16& score) __attribute__((always_inline)) {
        u32x4 p[2];
        f32x16 s[1] = {score};
        softmax_blocks(s, c, ref, l, o, p);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const bf16x8 vf = column_of_8_rows(v_read + 16 * u * D + (((2 * d) ^ vx) << 4), 8 * D);
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, p[u]), o[d], 0, 0, 0);
            }
    };
    auto wave_fence = [] {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };

    // ---- cache ----
    const int blocks = (j.len + 31) / 32, ptiles = (j.len + kTile - 1) / kTile;
    const scalar_int table = (scalar_int)l_table + (long long)j.b * l_max_pages;
    const int ps = 1 << l_ps_log2, page_last = max(j.len - 1, 0) >> l_ps_log2;
    unsigned bad = 0;              // rows of pages that are none
    struct Pages {
        int page[2];               // of the block's first and second sixteen rows
        unsigned seen;             // its rows that exist
    };
    auto pages_of = [&](int i) {
        Pages r;
        const int key0 = 32 * i, rem = j.len - key0;
        r.seen = rem >= 32 ? 0xffffffffu : rem > 0 ? (1u << rem) - 1 : 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) r.page[e] = table[min((key0 + 16 * e) >> l_ps_log2, page_last)];
        return r;
    };
    auto check = [&](Pages& r) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const bool there = (unsigned)r.page[e] < (unsigned)a.num_pages;
            const unsigned rows = there ? 0u : 0xffffu << (16 * e);
            bad |= r.seen & rows;
            r.seen &= ~rows;
            r.page[e] = there ? r.page[e] : 0;
        }
    };
    u32x4 kr[KL], vr[KL];
    int ke[2], ve[2];                                    // exponents of either half of the block
    // Every instruction asks for whole rows, and says that they are read once: 16 bytes of 32 rows each instead, as the matrix
    // operand wants them, or without the hint, 64 heads over 4 x 100000 keys take 172 us, not 156.
    const unsigned k_lane = (unsigned)(lane / CPR) * a.k_row + 16 * (lane % CPR);
    const unsigned v_lane = (unsigned)(lane / CPR) * a.v_row + 16 * (lane % CPR);
    const unsigned char* const kh = a.kp + hk * a.k_head;
    const unsigned char* const vh = a.vp + hk * a.v_head;
    auto load_k = [&](int i, const Pages& r) {
        const unsigned char* b[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            b[e] = row_of(kh, r.page[e], a.k_page, (32 * i + 16 * e) & (ps - 1), a.k_row);
            if constexpr (KV8) ke[e] = scalar_byte(a.k_exp, (unsigned)r.page[e] * a.kv_heads + hk);
        }
#pragma unroll
        for (int n = 0; n < KL; ++n)                     // rows n RPL .. n RPL + RPL - 1 of the block
            kr[n] = __builtin_nontemporal_load((const u32x4*)(b[(n * RPL) >> 4] + ((n * RPL) & 15) * a.k_row + k_lane));
    };
    auto load_v = [&](int i, const Pages& r) {
        const unsigned char* b[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            b[e] = row_of(vh, r.page[e], a.v_page, (32 * i + 16 * e) & (ps - 1), a.v_row);
            if constexpr (KV8) ve[e] = scalar_byte(a.v_exp, (unsigned)r.page[e] * a.kv_heads + hk);
        }
#pragma unroll
        for (int n = 0; n < KL; ++n)
            vr[n] = __builtin_nontemporal_load((const u32x4*)(b[(n * RPL) >> 4] + ((n * RPL) & 15) * a.v_row + v_lane));
    };
    auto stage = [&](unsigned seen) {
        wave_fence();
#pragma unroll
        for (int n = 0; n < KL; ++n) *(u32x4*)(s_k + k_at(n * RPL + lane / CPR, lane % CPR)) = kr[n];
        const float vs[2] = {KV8 ? exp_scale(ve[0]) : 1.f, KV8 ? exp_scale(ve[1]) : 1.f};
#pragma unroll
        for (int n = 0; n < KL; ++n) {
            const int row = n * RPL + lane / CPR, at = lane % CPR;
            u32x4 w = vr[n];
            if (seen != 0xffffffffu && !(seen >> row & 1)) w = u32x4{0, 0, 0, 0};
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
    };
    auto scores = [&](int e0, int e1) {                  // exponents of the block's halves
        f32x16 s;
#pragma unroll
        for (int v = 0; v < 16; ++v) s[v] = 0.f;
        const float f = KV8 ? (l32 & 16 ? exp_scale(e1) : exp_scale(e0)) : 1.f;
#pragma unroll
        for (int i = 0; i < NJ; ++i) {
            u32x4 lo, hi;
            if constexpr (KV8) widen16(*(const u32x4*)(s_k + k_at(l32, 2 * i + h)), f, lo, hi);
            else {
                lo = *(const u32x4*)(s_k + k_at(l32, 4 * i + 2 * h));
                hi = *(const u32x4*)(s_k + k_at(l32, 4 * i + 2 * h + 1));
            }
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, lo), q_frag(2 * i), s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, hi), q_frag(2 * i + 1), s, 0, 0, 0);
        }
        return s;
    };
    {
        const int end = min(2 * j.t1, blocks);
        int i = 2 * j.t0 + ks;
        if (i < end) {
            // Requests past the last block read that one again: a load under a condition would make every wait for an older one
            // a wait for all.
            auto in_range = [&](int k) { return min(k, end - 1); };
            Pages now = pages_of(i), ahead = pages_of(in_range(i + KS));
            check(now);
            load_v(i, now);
            load_k(i, now);
            for (; i < end; i += KS) {
                const int to = in_range(i + KS);
                const Pages after = pages_of(in_range(i + 2 * KS));
                check(ahead);
                const unsigned seen = now.seen;
                const int e0 = KV8 ? ke[0] : 0, e1 = KV8 ? ke[1] : 0;
                stage(seen);
                __builtin_amdgcn_sched_barrier(0);
                load_v(to, ahead);
                load_k(to, ahead);
                __builtin_amdgcn_sched_barrier(0);
                f32x16 s = scores(e0, e1);
                if (seen != 0xffffffffu) hide(s, seen, h);
                finish(s);
                now = ahead;
                ahead = after;
            }
        }
    }
    if (bad && lane == 0)
        __hip_atomic_fetch_or(a.sync + OT_ATTN_STATUS_OFFSET / 4, OT_ATTN_STATUS_BAD_PAGE, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);

    // ---- tree ----
    const int tt0 = max(j.t0 - ptiles, 0), tt1 = j.t1 - ptiles;
    if (tt1 > tt0) {
        __syncthreads();                                 // no wavefront reads K from LDS any more
        union_masks(a, j.b, tt0, tt1, s_union, 256);
        const unsigned short* const kt = (const unsigned short*)a.Kt + (long long)j.b * a.kts[0] + (long long)hk * a.kts[1];
        const unsigned short* const vt = (const unsigned short*)a.Vt + (long long)j.b * a.vts[0] + (long long)hk * a.vts[1];
        for (int i = 2 * tt0 + ks; i < 2 * tt1 && 32 * i < a.tree_keys; i += KS) {
            const int last = a.tree_keys - 1;
            const unsigned tail = 32 * i + 32 <= a.tree_keys ? 0xffffffffu : (1u << (a.tree_keys - 32 * i)) - 1;      // rows that exist
            const unsigned any = (unsigned)(s_union[(i >> 1) - tt0] >> (32 * (i & 1))) & tail;
            const unsigned short* const k1 = kt + (long long)min(32 * i + l32, last) * a.kts[2] + 16 * h;
            u32x4 k[2 * NJ];
#pragma unroll
            for (int n = 0; n < NJ; ++n) {
                k[2 * n] = *(const u32x4*)(k1 + 32 * n);
                k[2 * n + 1] = *(const u32x4*)(k1 + 32 * n + 8);
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
            f32x16 s;
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
            for (int n = 0; n < 2 * NJ; ++n) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k[n]), q_frag(n), s, 0, 0, 0);
            hide(s, (unsigned)(a.mask[mask_at + (i >> 1)] >> (32 * (i & 1))) & tail, h);
            finish(s);
        }
    }

    // ---- the streams' results ----
    __syncthreads();                                     // no wavefront reads Q any more
    {
        const float sum = xhalf_sum(l);
        if (h == 0) { s_ref[wave * 32 + l32] = ref; s_sum[wave * 32 + l32] = sum; }
    }
    __syncthreads();
    float* const s_o = (float*)s_mem;
    const int row = tid >> 3, col = (tid & 7) * 8;
    float M4 = kNoRef;
#pragma unroll
    for (int w = 0; w < KS; ++w) M4 = fmaxf(M4, s_ref[(w * QW + qb) * 32 + l32]);
    const float f = __builtin_amdgcn_exp2f(ref - M4);
    float M[QW], L[QW];
#pragma unroll
    for (int q = 0; q < QW; ++q) {
        M[q] = kNoRef; L[q] = 0.f;
#pragma unroll
        for (int w = 0; w < KS; ++w) M[q] = fmaxf(M[q], s_ref[(w * QW + q) * 32 + row]);
#pragma unroll
        for (int w = 0; w < KS; ++w) L[q] += s_sum[(w * QW + q) * 32 + row] * __builtin_amdgcn_exp2f(s_ref[(w * QW + q) * 32 + row] - M[q]);
    }
#pragma unroll
    for (int part = 0; part < D / 64; ++part) {
        __syncthreads();
#pragma unroll
        for (int d = 0; d < 2; ++d)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const f32x16& x = o[2 * part + d];
                *(f32x4*)(s_o + (wave * 32 + l32) * OST + 32 * d + 8 * v + 4 * h) =
                    f32x4{x[4 * v] * f, x[4 * v + 1] * f, x[4 * v + 2] * f, x[4 * v + 3] * f};
            }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < QW; ++q) {
            if (q * 32 + row >= rows) continue;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = 0.f;
#pragma unroll
            for (int w = 0; w < KS; ++w) {
                const float* const x = s_o + ((w * QW + q) * 32 + row) * OST + col;
                const f32x4 lo = *(const f32x4*)x, hi = *(const f32x4*)(x + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) { y[e] += lo[e]; y[4 + e] += hi[e]; }
            }
            if (j.splits == 1) {
                const float inv = inverse(L[q]);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] *= inv;
                store8<OT_BF16>(out_row(a, j.b, hk, row0 + q * 32 + row), 64 * part + col, y);
            } else {
                const unsigned at = (unsigned)(j.slot + j.split * a.units) * a.slot_rows + q * 32 + row;
                put4(part_buffer(a.part), at * D + 64 * part + col, f32x4{y[0], y[1], y[2], y[3]});
                put4(part_buffer(a.part), at * D + 64 * part + col + 4, f32x4{y[4], y[5], y[6], y[7]});
                if (part == 0 && col == 0) put2(a.part_ml + at * 2, M[q], L[q]);
            }
        }
    }
    if (j.splits > 1) join_splits<D, 256>(a, j, hk, row0, rows, s_last);
}

// ---------------------------------------------------------------------------
// Many rows: 32 packed query rows per wavefront, NW wavefronts, all of them over every 64-key tile of the job.
// Bound by the matrix cores, the exponentials and the issue of what surrounds them.  A tile is requested into registers a tile
// ahead of its way into LDS, widened to bf16 there, and read by all wavefronts.
//   K [64][D]: 16-byte piece c of row r at c ^ (r mod D/8);  V [64][D]: 32-byte segment g of row r at g ^ v_swizzle(r)
// 256 rows take eight wavefronts, one workgroup to a compute unit; up to 128 rows four, two workgroups to a unit, which drift
// apart by themselves.
// Measured: 16 x 8 KV heads x 1024 queries over 8192 keys in 8 bits (550 GFLOP) 541 to 575 us, 0.96 to 1.02 PFLOP/s, where a large bf16
// matrix product of the library reaches 1.23; 16 x 8 x 480 over 4096 +-25 % 157 to 165 us (the longest sequence decides).
// ---------------------------------------------------------------------------
template <int D, bool KV8, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_tiles_kernel(OT_LEAD_PARAMS, const PagedArgs a) {
    constexpr int NT = 64 * NW, DB = D / 32, SL = D / 16, CPR = D / 8;
    constexpr int ESZ = KV8 ? 1 : 2;
    constexpr int CPM = D * ESZ / 16;                  // 16-byte pieces per row in memory
    constexpr int CH = kTile * CPM / NT;               // pieces of K per thread and tile, and of V
    constexpr int CHT = kTile * CPR / NT;              // the same of a tree tile
    static_assert(CH >= 1 && 64 / CPM <= 16, "a piece per thread; a wavefront's rows lie in one page");
    extern __shared__ __attribute__((aligned(16))) unsigned short s_kv[];       // tiles [64][D]
    __shared__ u64 s_union[OT_MAX_TREE_KEYS / 64];
    constexpr bool TURNS = NW == 8;                    // two wavefronts of a SIMD take turns, see below
    constexpr int TILE = kTile * D;                    // a tile of K or of V in LDS
    auto k_buf = [&](int i) { return s_kv + i * TILE; };                         // two of K,
    auto v_buf = [&](int i) { return s_kv + (2 + i) * TILE; };                   // two of V, three if the wavefronts take turns
    const Job j = find_job(OT_LEAD, a.sync, blockIdx.x);
    if (j.none) return;
    note_splits(a, j);
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
    const scalar_int table = (scalar_int)l_table + (long long)j.b * l_max_pages;
    const int ps = 1 << l_ps_log2, page_last = max(j.len - 1, 0) >> l_ps_log2;
    u64 bad = 0;                                         // rows of pages that are none
    const int e_wave = wave * (64 / CPM);                // first row of this wavefront's first request; the others NT / CPM rows on

    auto put_k = [&](unsigned short* sk, int row, int piece, const u32x4& w) { *(u32x4*)(sk + row * D + ((piece ^ (row & (CPR - 1))) << 3)) = w; };
    auto k_frag = [&](const unsigned short* sk, int kb, int i) {
        return __builtin_bit_cast(bf16x8, *(const u32x4*)(sk + (32 * kb + l32) * D + (((2 * i + h) ^ kx) << 3)));
    };
    auto v_frag = [&](const unsigned short* sv, int u, int d) {
        return column_of_8_rows(sv + (16 * u + 4 * h + tr_j) * D + (((2 * d) ^ vx) << 4) + 4 * (lane & 3), 8 * D);
    };
    f32x16 s[2];
    u32x4 p[4];
    auto clear_scores = [&] {
#pragma unroll
        for (int v = 0; v < 16; ++v) s[0][v] = s[1][v] = 0.f;
    };
    auto scores = [&](const unsigned short* sk) __attribute__((always_inline)) {
        clear_scores();
        pipelined<2 * SL, 4>([&](int i) { return k_frag(sk, i & 1, i >> 1); },
                             [&](int i, const bf16x8& k) { s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[i >> 1], s[i & 1], 0, 0, 0); });
    };
    auto weights = [&](u64 visible) __attribute__((always_inline)) {
        if (visible != ~0ull) {
            hide(s[0], (unsigned)visible, h);
            hide(s[1], (unsigned)(visible >> 32), h);
        }
        softmax_blocks(s, c, ref, l, o, p);
    };
    auto add_value = [&](int i, const bf16x8& v) __attribute__((always_inline)) {
        o[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, p[i / DB]), o[i % DB], 0, 0, 0);
    };
    auto values = [&](const unsigned short* sv) __attribute__((always_inline)) {
        pipelined<4 * DB, 3>([&](int i) { return v_frag(sv, i / DB, i % DB); }, add_value);
    };
    // values of one tile and scores of the next, 4 DB = 2 SL of either
    auto values_and_scores = [&](const unsigned short* sv, const unsigned short* sk) __attribute__((always_inline)) {
        struct Pair { bf16x8 v, k; };
        clear_scores();
        pipelined<2 * SL, 2>([&](int i) { return Pair{v_frag(sv, i / DB, i % DB), k_frag(sk, i & 1, i >> 1)}; },
                             [&](int i, const Pair& x) {
                                 add_value(i, x.v);
                                 s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.k, qf[i >> 1], s[i & 1], 0, 0, 0);
                             });
    };

    // ---- cache ----
    const int tp1 = min(j.t1, ptiles);
    if (j.t0 < tp1) {
        struct Pages {
            int page[4];                   // of the tile's four times sixteen rows
            u64 seen;                      // its rows that exist
        };
        auto in_range = [&](int t) { return min(t, tp1 - 1); };
        auto pages_of = [&](int t) {
            Pages r;
            const int key0 = t * kTile, rem = j.len - key0;
            r.seen = rem >= kTile ? ~0ull : (1ull << rem) - 1;
#pragma unroll
            for (int e = 0; e < 4; ++e) r.page[e] = table[min((key0 + 16 * e) >> l_ps_log2, page_last)];
            return r;
        };
        u32x4 kr[CH], vr[CH];
        int ke[CH], ve[CH];
        u64 next = 0;                      // rows of the tile in registers that exist
        const unsigned k_lane = (unsigned)(lane / CPM) * a.k_row + 16 * (lane % CPM);
        const unsigned v_lane = (unsigned)(lane / CPM) * a.v_row + 16 * (lane % CPM);
        const unsigned char* const kh = a.kp + hk * a.k_head;
        const unsigned char* const vh = a.vp + hk * a.v_head;
        auto load = [&](int t, Pages r) {                // past the last tile: that one again (a load under a condition makes waits longer)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool there = (unsigned)r.page[e] < (unsigned)a.num_pages;
                const u64 rows = there ? 0ull : 0xffffull << (16 * e);
                bad |= r.seen & rows;
                r.seen &= ~rows;
                r.page[e] = there ? r.page[e] : 0;
            }
            next = r.seen;
#pragma unroll
            for (int n = 0; n < CH; ++n) {
                const int first = e_wave + n * (NT / CPM), e = first >> 4;       // rows first .. first + 64 / CPM - 1
                const unsigned page = e == 0 ? r.page[0] : e == 1 ? r.page[1] : e == 2 ? r.page[2] : r.page[3];
                const unsigned row = (t * kTile + first) & (ps - 1);
                kr[n] = *(const u32x4*)(row_of(kh, page, a.k_page, row, a.k_row) + k_lane);
                vr[n] = *(const u32x4*)(row_of(vh, page, a.v_page, row, a.v_row) + v_lane);
                if constexpr (KV8) {
                    ke[n] = scalar_byte(a.k_exp, page * a.kv_heads + hk);
                    ve[n] = scalar_byte(a.v_exp, page * a.kv_heads + hk);
                }
            }
        };
        auto stage = [&](unsigned short* sk, unsigned short* sv) {
#pragma unroll
            for (int n = 0; n < CH; ++n) {
                const int row = tid / CPM + n * (NT / CPM), piece = tid % CPM;
                u32x4 w = vr[n];
                if (next != ~0ull && !(next >> row & 1)) w = u32x4{0, 0, 0, 0};
                if constexpr (KV8) {
                    u32x4 lo, hi;
                    widen16(kr[n], exp_scale(ke[n]), lo, hi);
                    put_k(sk, row, 2 * piece, lo);
                    put_k(sk, row, 2 * piece + 1, hi);
                    widen16(w, exp_scale(ve[n]), lo, hi);
                    u32x4* const v = (u32x4*)(sv + row * D + ((piece ^ v_swizzle<D>(row)) << 4));
                    v[0] = lo; v[1] = hi;
                } else {
                    put_k(sk, row, piece, kr[n]);
                    *(u32x4*)(sv + row * D + (((piece >> 1) ^ v_swizzle<D>(row)) << 4) + 8 * (piece & 1)) = w;
                }
            }
        };
        load(j.t0, pages_of(j.t0));
        Pages ahead = pages_of(in_range(j.t0 + 1));
        int x = j.t0;                                    // tile in registers
        u64 staged = 0, before = 0;                      // `next` of the last tile that was staged, and of the one before it
        int vb = 0;                                      // V buffer of tile x
        auto advance = [&]() __attribute__((always_inline)) {                    // tile x to LDS, tile x + 1 on its way
            stage(k_buf((x - j.t0) & 1), v_buf(vb));
            before = staged;
            staged = next;
            ++x;
            load(in_range(x), ahead);
            ahead = pages_of(in_range(x + 1));
            vb = vb == (TURNS ? 2 : 1) ? 0 : vb + 1;
        };
        advance();
        if constexpr (TURNS) {
            // The two wavefronts of a SIMD take turns: while wavefronts 0..3 have the matrix cores (values of tile t - 1, scores
            // of tile t), wavefronts 4..7 do the exponentials of tile t - 1 and bring a tile into LDS, and the other way
            // round; a barrier changes sides.  A tile of V is read half a turn into the next tile and written two turns
            // ahead: three buffers; K two.  Without turns both wavefronts would be at the same kind of work, since they meet
            // at every tile: 16 x 32 heads x 256 nodes over 8192 keys 649 us, not 576.
            const bool second = wave >= 4;
            __syncthreads();
            if (second) { advance(); __syncthreads(); }
            int va = 0;                                  // V buffer of tile t
            scores(k_buf(0));
            for (int t = j.t0;;) {
                __syncthreads();
                const u64 visible = second ? before : staged;
                advance();                               // (past the last tile: a copy of it, which nobody reads)
                weights(visible);
                __syncthreads();
                if (++t >= tp1) break;
                __builtin_amdgcn_s_setprio(1);           // (the matrix side is issued first: 582 -> 570 us)
                values_and_scores(v_buf(va), k_buf((t - j.t0) & 1));
                __builtin_amdgcn_s_setprio(0);
                va = va == 2 ? 0 : va + 1;
            }
            if (!second) __syncthreads();
            values(v_buf(va));
        } else {
            for (int t = j.t0; t < tp1; ++t) {
                const int now = (t - j.t0) & 1;
                __syncthreads();
                const u64 visible = staged;
                advance();
                scores(k_buf(now));
                weights(visible);
                values(v_buf(now));
            }
        }
    }

    // ---- tree ----
    {
        const int tt0 = max(j.t0 - ptiles, 0), tt1 = j.t1 - ptiles, last = a.tree_keys - 1;
        const unsigned short* const kt = (const unsigned short*)a.Kt + (long long)j.b * a.kts[0] + (long long)hk * a.kts[1];
        const unsigned short* const vt = (const unsigned short*)a.Vt + (long long)j.b * a.vts[0] + (long long)hk * a.vts[1];
        u32x4 kr[CHT], vr[CHT];
        u64 next = 0;
        int buf = 0;
        auto load = [&](int tt) {
            next = a.mask[mask_at + tt];
#pragma unroll
            for (int n = 0; n < CHT; ++n) {
                const int row = min(tt * kTile + tid / CPR + n * (NT / CPR), last);
                kr[n] = *(const u32x4*)(kt + (long long)row * a.kts[2] + 8 * (tid % CPR));
                vr[n] = *(const u32x4*)(vt + (long long)row * a.vts[2] + 8 * (tid % CPR));
            }
        };
        if (tt1 > tt0) {
            load(tt0);
            union_masks(a, j.b, tt0, tt1, s_union, NT);
        }
        for (int tt = tt0; tt < tt1; ++tt) {
            const int rem = a.tree_keys - tt * kTile;
            const u64 tail = rem >= kTile ? ~0ull : (1ull << rem) - 1, any = s_union[tt - tt0] & tail;
            unsigned short* const sk = k_buf(buf);
            unsigned short* const sv = v_buf(buf);
#pragma unroll
            for (int n = 0; n < CHT; ++n) {
                const int row = tid / CPR + n * (NT / CPR), piece = tid % CPR;
                u32x4 w = vr[n];
                put_k(sk, row, piece, kr[n]);
                if (!(any >> row & 1)) w = u32x4{0, 0, 0, 0};
                *(u32x4*)(sv + row * D + (((piece >> 1) ^ v_swizzle<D>(row)) << 4) + 8 * (piece & 1)) = w;
            }
            const u64 mask = next & tail;
            __syncthreads();
            load(min(tt + 1, tt1 - 1));
            scores(sk);
            weights(mask);
            values(sv);
            buf ^= 1;
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
        const unsigned at = (unsigned)(j.slot + j.split * a.units) * a.slot_rows + row;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                put4(part_buffer(a.part), at * D + 32 * d + 8 * v + 4 * h, f32x4{o[d][4 * v], o[d][4 * v + 1], o[d][4 * v + 2], o[d][4 * v + 3]});
        if (h == 0) put2(a.part_ml + at * 2, ref, L);
    }
    __shared__ int s_last;
    join_splits<D, NT>(a, j, hk, row0, rows, &s_last);
}

__global__ __launch_bounds__(256) void clear_words_kernel(unsigned int* w) { w[blockIdx.x * 256 + threadIdx.x] = 0; }

struct PagedPlan {
    int rows, row_blocks, units, target, grid, slot_rows;
    bool late;                // another launch joins
    float apart;
    size_t part_bytes, ml_bytes, bytes;
};

PagedPlan plan_paged(const ot_paged_attn_params& p, const ot_paged_cache& c) {
    PagedPlan pl;
    const int R = p.q_heads / c.kv_heads * p.n;
    // (an 8-bit tile of 64-wide heads is 256 pieces of 16 bytes: four wavefronts)
    pl.rows = R <= 32 ? 32 : R <= 64 ? 64 : R <= 128 || (c.head_dim == 64 && c.dtype == OT_E4M3) ? 128 : 256;
    pl.row_blocks = (R + pl.rows - 1) / pl.rows;
    pl.units = c.kv_heads * pl.row_blocks;
    pl.slot_rows = std::min(R, pl.rows);
    const long long all = (long long)p.batch * pl.units;
    const int resident = pl.rows <= 128 ? 512 : 256;           // workgroups that the card holds
    // As many triples as the card holds, or more than 256 sequences, stay in one piece each: cutting 16 x 8 KV heads x 480 rows over 4096
    // keys +-25 % into twice as many jobs took 199 us instead of 160, for the second round of workgroups.  The price is a batch that one
    // long context rules: 64 x 8 KV heads x 8 queries, 63 contexts of 1000 keys and one of 100000, 955 us (62 and one: 498, 31 and one:
    // 55; 64 of 2547, the same bytes: 55), 300 x 1 x 8 with one of 30000 288 us (256: 20).
    pl.target = p.batch <= kSplitBatch && all < resident ? resident : 0;
    // workgroups: whole rounds of eight XCDs (find_job); jobs, and partials, are `target` at most
    const long long pairs = pl.target ? pl.target / pl.row_blocks : (long long)p.batch * c.kv_heads;
    pl.grid = (int)((pairs + 7) / 8 * 8 * pl.row_blocks);
    pl.late = pl.target && pl.slot_rows > kTicketRows;
    // A range more costs a partial written and read by every unit, at 4 TB/s, or a trip to memory for a chunk of sixteen; a
    // tile of 64 keys takes (us, head_dim 128) 0.7 for up to 64 rows, 1.2 for 128, 2.2 for 256.  Over 14 shapes (1 to 500 rows a KV head, 700
    // to 30000 keys) a quarter, half, twice and four times this cost take 1.09, 1.03, 1.02 and 1.12 of the time in the mean, and no shape
    // is more than 13 % from its best of the five.
    const float tile = (pl.rows <= 64 ? 0.7f : pl.rows == 128 ? 1.2f : 2.2f) * (float)c.head_dim / 128.f;
    pl.apart = (pl.late ? (float)all * (float)pl.slot_rows * (float)c.head_dim * 8.f / 4e6f + 0.02f : 0.13f) / tile;
    const size_t jobs = (size_t)pl.target;
    pl.part_bytes = jobs * pl.slot_rows * c.head_dim * 4;
    pl.ml_bytes = jobs * pl.slot_rows * 8;
    pl.bytes = OT_PAGED_SYNC_BYTES + pl.part_bytes + pl.ml_bytes + (pl.late ? (size_t)all * sizeof(int2) : 0);
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
    if (overlaps(p->o_strides, p->batch, p->q_heads, p->n, c->head_dim)) return OT_ERR_INVALID_ARG;
    return OT_OK;
}

template <int D, bool KV8>
int launch_paged(const Lead& l, const PagedArgs& a, const PagedPlan& pl, hipStream_t s) {
#define OT_LEAD_ARGS l.prefix_len, l.table, l.batch, l.kv_heads, l.row_blocks, l.max_pages, l.ps_log2, l.tiles_tree, l.target, l.apart
    constexpr size_t tile = (size_t)kTile * D * 2;
    if (pl.rows == 32) hipLaunchKernelGGL((paged_rows_kernel<D, KV8, 1>), dim3(pl.grid), dim3(256), 0, s, OT_LEAD_ARGS, a);
    else if (pl.rows == 64) hipLaunchKernelGGL((paged_rows_kernel<D, KV8, 2>), dim3(pl.grid), dim3(256), 0, s, OT_LEAD_ARGS, a);
    else if (pl.rows == 128) {
        OT_HIP_CHECK(hipFuncSetAttribute((const void*)paged_tiles_kernel<D, KV8, 4>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(4 * tile)));
        hipLaunchKernelGGL((paged_tiles_kernel<D, KV8, 4>), dim3(pl.grid), dim3(256), 4 * tile, s, OT_LEAD_ARGS, a);
    } else if constexpr (!(D == 64 && KV8)) {
        OT_HIP_CHECK(hipFuncSetAttribute((const void*)paged_tiles_kernel<D, KV8, 8>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(5 * tile)));
        hipLaunchKernelGGL((paged_tiles_kernel<D, KV8, 8>), dim3(pl.grid), dim3(512), 5 * tile, s, OT_LEAD_ARGS, a);
    }
#undef OT_LEAD_ARGS
    OT_HIP_CHECK(hipGetLastError());
    if (!pl.late) return OT_OK;
    hipLaunchKernelGGL((paged_join_kernel<D>), dim3((unsigned)((pl.slot_rows + 1024 / D - 1) / (1024 / D)), (unsigned)(l.batch * pl.units)), dim3(256), 0, s, a);
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
    a.k_exp = cache->k_exp; a.v_exp = cache->v_exp; a.mask = mask;
    a.sync = (unsigned int*)workspace;
    a.part = (float*)((char*)workspace + OT_PAGED_SYNC_BYTES);
    a.part_ml = a.part + pl.part_bytes / 4;
    a.joins = pl.late ? (int2*)((char*)a.part_ml + pl.ml_bytes) : nullptr;
    a.kv_heads = cache->kv_heads; a.g = p->q_heads / cache->kv_heads; a.n = p->n;
    a.tree_keys = p->tree_keys; a.W = OT_MASK_WORDS(p->tree_keys);
    a.row_blocks = pl.row_blocks; a.units = pl.units;
    a.num_pages = cache->num_pages; a.block_rows = pl.rows; a.slot_rows = pl.slot_rows;
    const Lead lead{prefix_len, cache->page_table, p->batch, cache->kv_heads, pl.row_blocks, cache->max_pages, log2_of(cache->page_size),
                    (p->tree_keys + kTile - 1) / kTile, pl.target, pl.apart};
    a.scale_log2 = (p->softmax_scale != 0.f ? p->softmax_scale : 1.0f / sqrtf((float)cache->head_dim)) * kLog2e;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = p->q_strides[i]; a.kts[i] = p->kt_strides[i]; a.vts[i] = p->vt_strides[i]; a.os[i] = p->o_strides[i];
    }
    const long long esz = cache->dtype == OT_E4M3 ? 1 : 2;
    a.k_page = (unsigned)(cache->k_strides[0] * esz / 16); a.v_page = (unsigned)(cache->v_strides[0] * esz / 16);
    a.k_row = (unsigned)(cache->k_strides[2] * esz); a.v_row = (unsigned)(cache->v_strides[2] * esz);
    a.k_head = cache->k_strides[1] * esz; a.v_head = cache->v_strides[1] * esz;
    hipStream_t s = (hipStream_t)hip_stream;
    if (cache->dtype == OT_E4M3) return cache->head_dim == 128 ? launch_paged<128, true>(lead, a, pl, s) : launch_paged<64, true>(lead, a, pl, s);
    return cache->head_dim == 128 ? launch_paged<128, false>(lead, a, pl, s) : launch_paged<64, false>(lead, a, pl, s);
}

}  // extern "C"
