// Queries and keys of new tokens: root-mean-square norm of every head and position rotation in one pass.
//   y = x / sqrt(mean(x^2) + eps) * w;  pairs of columns turned by pos * inv_freq[j]          (opttree.h)
//
// What bounds it: every value is read once and written once (HBM); small calls are launch latency and one chain of
// position -> angle -> row.  A workgroup takes `tokens` consecutive tokens with all their heads (few tokens: one token and a share of
// its heads): the angles of a token are the same for all of its heads, so their cosines and sines are computed once, a
// thread each, and kept in LDS.  A row is eight lanes (head_dim 64: four) of sixteen columns, so its norm is three
// (two) exchanges inside a row of sixteen lanes and both partners of a pair are in one lane (rope.hpp).
// Measured: 15009 tokens x 40 heads of 128 in fp32 (615 MB) 130 us, 4.7 TB/s, the rate of a plain copy; 960 tokens x 72 heads in bf16
// (35 MB) 9.4 us; one token x 40 heads 2.8 us on the card, 5.7 a call.
#include <algorithm>

#include "common.hpp"
#include "internal.h"
#include "rope.hpp"

namespace ot {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 8;            // tokens per workgroup

struct QkKArgs {
    const void *Q, *K, *qw, *kw;
    void *Qo, *Ko;
    const int32_t *first, *offset;
    Rotary rot;
    int q_heads, heads;                  // heads = q_heads + kv_heads
    int n, all_tokens, tokens, share;    // tokens per workgroup; heads per workgroup (blockIdx.y counts shares)
    int base;                            // first token of this launch
    unsigned int inv_share;              // division by multiplication: ceil(2^32 / share), 0 for 1
    int shift;
    float eps;
    long long qs[3], ks[3], qos[3], kos[3];
};

template <int DT, int D>
__global__ __launch_bounds__(kThreads) void qk_rope_kernel(const QkKArgs a) {
    constexpr int LPR = D / 16;                       // lanes per row
    constexpr int RPP = kThreads / LPR;               // rows per pass
    __shared__ __attribute__((aligned(16))) float2 s_cs[kMaxTokens][D / 2];
    const int tid = threadIdx.x, t = tid % LPR;
    const int tok0 = a.base + (int)blockIdx.x * a.tokens, ntok = min(a.tokens, a.all_tokens - tok0);
    const int half = a.rot.dim / 2;
    const int h0 = blockIdx.y * a.share, hn = min(a.share, a.heads - h0);
    for (int i = tid; i < ntok * half; i += kThreads) {
        const int k = i / half, j = i - k * half, tok = tok0 + k, b = tok / a.n;
        const int step = a.offset ? a.offset[tok] : tok - b * a.n;
        const long long pos = (long long)a.first[b] + step + a.shift;
        s_cs[k][angle_at(j, a.rot.dim / 16)] = cos_sin((double)pos * a.rot.inv_freq[j]);
    }
    __syncthreads();
    const int ca = run_a(a.rot, t), cb = run_b(a.rot, t);
    const bool turns = 16 * t < a.rot.dim;
    for (int r = tid / LPR; r < ntok * hn; r += RPP) {
        const int k = hn == a.share ? (a.inv_share ? (int)__umulhi((unsigned)r, a.inv_share) : r) : r / hn;
        const int h = h0 + r - k * hn, tok = tok0 + k, b = tok / a.n, i = tok - b * a.n;
        const bool q = h < a.q_heads;
        const long long* const si = q ? a.qs : a.ks;
        const long long* const so = q ? a.qos : a.kos;
        const int hh = q ? h : h - a.q_heads;
        const long long in = b * si[0] + hh * si[1] + i * si[2], out = b * so[0] + hh * so[1] + i * so[2];
        float xa[8], xb[8];
        load8<DT>(q ? a.Q : a.K, in + ca, xa);
        load8<DT>(q ? a.Q : a.K, in + cb, xb);
        const void* const w = q ? a.qw : a.kw;
        if (w) {
            float wa[8], wb[8], ss = 0.f;
            load8<DT>(w, ca, wa);
            load8<DT>(w, cb, wb);
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(xa[e], xa[e], fmaf(xb[e], xb[e], ss));
            ss += __int_as_float(dpp_i<DPP_QUAD_XOR1>(__float_as_int(ss), __float_as_int(ss)));
            ss += __int_as_float(dpp_i<DPP_QUAD_XOR2>(__float_as_int(ss), __float_as_int(ss)));
            if constexpr (LPR == 8) ss += __int_as_float(dpp_i<DPP_ROW_HALF_MIRROR>(__float_as_int(ss), __float_as_int(ss)));
            const float f = 1.f / sqrtf(ss * (1.f / D) + a.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) { xa[e] = xa[e] * f * wa[e]; xb[e] = xb[e] * f * wb[e]; }
        }
        if (turns) {
            float2 cs[8];
            read_angles(s_cs[k], t, a.rot.dim / 16, cs);
            turn(xa, xb, cs, a.rot.interleaved);
        }
        store8<DT>(q ? a.Qo : a.Ko, out + ca, xa);
        store8<DT>(q ? a.Qo : a.Ko, out + cb, xb);
    }
}

int validate_qk(const ot_qk_params* p) {
    if (!p) return OT_ERR_INVALID_ARG;
    if (p->batch < 1 || p->q_heads < 0 || p->kv_heads < 0 || p->n < 1) return OT_ERR_INVALID_ARG;
    if ((long long)p->q_heads + p->kv_heads < 1) return OT_ERR_INVALID_ARG;
    if (p->dtype != OT_F32 && p->dtype != OT_BF16) return OT_ERR_INVALID_ARG;
    if (p->interleaved != 0 && p->interleaved != 1) return OT_ERR_INVALID_ARG;
    if (!(p->eps >= 0.f) || p->eps > 3.402823466e38f) return OT_ERR_INVALID_ARG;
    if (p->rotary_dim < 0 || p->rotary_dim > p->head_dim) return OT_ERR_INVALID_ARG;
    if (p->head_dim != 64 && p->head_dim != 128) return OT_ERR_UNSUPPORTED;
    if (p->rotary_dim % 16) return OT_ERR_UNSUPPORTED;
    if ((long long)p->batch * p->n > 0x7fffffffLL || (long long)p->q_heads + p->kv_heads > 65535) return OT_ERR_UNSUPPORTED;
    const int vec = p->dtype == OT_BF16 ? 8 : 4;
    const int64_t* st[4] = {p->q_strides, p->k_strides, p->qo_strides, p->ko_strides};
    for (int t = 0; t < 4; ++t) {
        if ((t % 2 == 0 ? p->q_heads : p->kv_heads) == 0) continue;
        for (int i = 0; i < 3; ++i)
            if (st[t][i] < 0 || st[t][i] % vec) return OT_ERR_INVALID_ARG;
        if (t >= 2 && overlaps(st[t], p->batch, t == 2 ? p->q_heads : p->kv_heads, p->n, p->head_dim)) return OT_ERR_INVALID_ARG;
    }
    return OT_OK;
}

}  // namespace
}  // namespace ot

using namespace ot;

extern "C" {

int ot_qk_norm_rope(const ot_qk_params* p, const void* Q, const void* K, const void* q_weight, const void* k_weight,
                    const double* inv_freq, const int32_t* first, const int32_t* offset, void* Q_out, void* K_out,
                    void* hip_stream) {
    const int st = validate_qk(p);
    if (st != OT_OK) return st;
    if ((p->q_heads && (!Q || !Q_out)) || (p->kv_heads && (!K || !K_out)) || !first) return OT_ERR_INVALID_ARG;
    if (p->rotary_dim && !inv_freq) return OT_ERR_INVALID_ARG;
    if (p->q_heads && p->kv_heads && Q_out == K_out) return OT_ERR_INVALID_ARG;
    const void* v[6] = {p->q_heads ? Q : nullptr, p->q_heads ? Q_out : nullptr, p->q_heads ? q_weight : nullptr,
                        p->kv_heads ? K : nullptr, p->kv_heads ? K_out : nullptr, p->kv_heads ? k_weight : nullptr};
    for (const void* x : v)
        if ((uintptr_t)x % 16) return OT_ERR_INVALID_ARG;
    if ((uintptr_t)inv_freq % 8 || (uintptr_t)first % 4 || (uintptr_t)offset % 4) return OT_ERR_INVALID_ARG;
    QkKArgs a;
    a.Q = Q; a.K = K; a.qw = q_weight; a.kw = k_weight; a.Qo = Q_out; a.Ko = K_out;
    a.first = first; a.offset = offset;
    a.rot = Rotary{inv_freq, p->rotary_dim, p->interleaved};
    a.q_heads = p->q_heads; a.heads = p->q_heads + p->kv_heads; a.n = p->n; a.all_tokens = p->batch * p->n;
    a.shift = p->shift; a.eps = p->eps;
    for (int i = 0; i < 3; ++i) { a.qs[i] = p->q_strides[i]; a.ks[i] = p->k_strides[i]; a.qos[i] = p->qo_strides[i]; a.kos[i] = p->ko_strides[i]; }
    const int rpp = kThreads * 16 / p->head_dim;
    // two passes of rows per workgroup (four: 149 us, not 130, at 15009 tokens x 40 heads in fp32)
    a.tokens = std::min(kMaxTokens, std::max(1, 2 * rpp / a.heads));
    a.share = a.heads;
    if (((long long)a.all_tokens + a.tokens - 1) / a.tokens < 512) {      // few tokens: a token each, heads over several workgroups
        a.tokens = 1;
        if (a.all_tokens < 512) a.share = std::min(a.heads, rpp);
    }
    a.inv_share = a.share > 1 ? (unsigned)((0x100000000ull + a.share - 1) / a.share) : 0;
    const unsigned shares = (unsigned)((a.heads + a.share - 1) / a.share);
    // a grid holds fewer than 2^32 threads: more tokens go in several launches
    const int groups = sequences_per_launch((int)(((long long)a.all_tokens + a.tokens - 1) / a.tokens), (long long)shares * kThreads);
    hipStream_t s = (hipStream_t)hip_stream;
    for (long long base = 0; base < a.all_tokens; base += (long long)groups * a.tokens) {
        a.base = (int)base;
        const dim3 grid((unsigned)std::min<long long>(groups, (a.all_tokens - base + a.tokens - 1) / a.tokens), shares);
        if (p->dtype == OT_BF16) {
            if (p->head_dim == 128) hipLaunchKernelGGL((qk_rope_kernel<OT_BF16, 128>), grid, dim3(kThreads), 0, s, a);
            else hipLaunchKernelGGL((qk_rope_kernel<OT_BF16, 64>), grid, dim3(kThreads), 0, s, a);
        } else {
            if (p->head_dim == 128) hipLaunchKernelGGL((qk_rope_kernel<OT_F32, 128>), grid, dim3(kThreads), 0, s, a);
            else hipLaunchKernelGGL((qk_rope_kernel<OT_F32, 64>), grid, dim3(kThreads), 0, s, a);
        }
    }
    OT_HIP_CHECK(hipGetLastError());
    return OT_OK;
}

}  // extern "C"
