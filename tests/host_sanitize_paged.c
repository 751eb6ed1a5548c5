/* Host-side paths of the operators around a paged cache under AddressSanitizer and UndefinedBehaviorSanitizer: sizes and
 * refusals over grids of shapes; nothing is launched.  Built and run by tests/test_host_sanitizers_paged.py. */
#include <stdio.h>
#include <string.h>
#include "opttree.h"

static int calls = 0, bad = 0;
#define EXPECT(expr, want)                                                              \
    do {                                                                                \
        const long long got_ = (long long)(expr);                                       \
        ++calls;                                                                        \
        if (got_ != (long long)(want)) {                                                \
            ++bad;                                                                      \
            fprintf(stderr, "line %d: %s = %lld, expected %lld\n", __LINE__, #expr, got_, (long long)(want)); \
        }                                                                               \
    } while (0)

int main(void) {
    void *const f = (void*)0x1000, *const far_away = (void*)0x10000000000;      /* never dereferenced on the host */
    const int batches[] = {1, 3, 255, 256, 257, 65535}, kvs[] = {1, 2, 8, 40}, gs[] = {1, 4, 8}, ns[] = {1, 4, 17, 50, 64, 256};
    const int pages[] = {16, 32, 64, 128, 256}, dims[] = {64, 128}, most[] = {1, 100, 100000, 4000000};
    for (int b = 0; b < 6; ++b) for (int k = 0; k < 4; ++k) for (int g = 0; g < 3; ++g) for (int n = 0; n < 6; ++n)
        for (int q = 0; q < 5; ++q) for (int d = 0; d < 2; ++d) for (int m = 0; m < 4; ++m) for (int t = 1; t < 3; ++t) {
            const int64_t D = dims[d], ps = pages[q], H = kvs[k];
            ot_paged_cache c;
            memset(&c, 0, sizeof c);
            c.num_pages = 1000; c.page_size = (int)ps; c.kv_heads = (int)H; c.head_dim = (int)D; c.dtype = t; c.max_pages = most[m];
            const int64_t s[3] = {H * ps * D, ps * D, D};
            memcpy(c.k_strides, s, sizeof s); memcpy(c.v_strides, s, sizeof s);
            c.k_pages = c.v_pages = f; c.k_exp = c.v_exp = f; c.page_table = f;
            ot_paged_attn_params p;
            memset(&p, 0, sizeof p);
            p.batch = batches[b]; p.q_heads = (int)H * gs[g]; p.n = ns[n]; p.tree_keys = ns[n];
            const int64_t qs[3] = {p.q_heads * (int64_t)p.n * D, p.n * D, D};
            memcpy(p.q_strides, qs, sizeof qs); memcpy(p.o_strides, qs, sizeof qs); memcpy(p.kt_strides, qs, sizeof qs); memcpy(p.vt_strides, qs, sizeof qs);
            const int ok = (int64_t)p.batch * p.q_heads <= 65535 && (int64_t)most[m] * ps < (1 << 30);
            const size_t need = ot_paged_attn_workspace_bytes(&p, &c);
            EXPECT(need != 0, ok);
            if (ok) {
                EXPECT(need >= OT_PAGED_SYNC_BYTES && need < ((size_t)1 << 28), 1);
                EXPECT(ot_tree_verify_attention_paged(&p, &c, f, f, f, f, f, f, f, need - 1, NULL), OT_ERR_WORKSPACE_TOO_SMALL);
            } else {
                EXPECT(ot_tree_verify_attention_paged(&p, &c, f, f, f, f, f, f, f, (size_t)1 << 40, NULL), OT_ERR_UNSUPPORTED);
            }
            ot_append_params a;
            memset(&a, 0, sizeof a);
            a.batch = batches[b]; a.n = ns[n]; a.dtype = OT_BF16; a.rotary_dim = (int)D;
            memcpy(a.k_strides, qs, sizeof qs); memcpy(a.v_strides, qs, sizeof qs);
            EXPECT(ot_kv_append_paged(&a, &c, f, f, f, f, f, f, f, NULL), (int64_t)most[m] * ps < (1 << 30) ? OT_ERR_INVALID_ARG : OT_ERR_UNSUPPORTED);
            a.n = OT_MAX_APPEND + 1;
            EXPECT(ot_kv_append_paged(&a, &c, f, f, f, f, f, f, far_away, NULL), OT_ERR_UNSUPPORTED);
        }
    ot_qk_params p;
    memset(&p, 0, sizeof p);
    EXPECT(ot_qk_norm_rope(&p, f, f, f, f, f, f, f, f, f, NULL), OT_ERR_INVALID_ARG);
    p.batch = 1 << 30; p.n = 2; p.q_heads = 1; p.head_dim = 64; p.dtype = OT_F32;
    EXPECT(ot_qk_norm_rope(&p, f, f, f, f, f, f, f, f, f, NULL), OT_ERR_UNSUPPORTED);
    if (!bad) printf("ok %d\n", calls);
    return bad != 0;
}
