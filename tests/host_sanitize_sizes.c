/* Host arithmetic of the operators around a paged cache at the largest sizes they take, under UndefinedBehaviorSanitizer.  No GPU may be
 * visible: the calls are valid up to their launches, which then fail.  Built and run by tests/test_host_sanitizers_sizes.py. */
#include <hip/hip_runtime_api.h>
#include <stdio.h>
#include <string.h>
#include "opttree.h"

static int bad = 0;
static void expect(const char* what, int got, int want) {
    if (got == want) return;
    ++bad;
    fprintf(stderr, "%s: %d, expected %d\n", what, got, want);
}

int main(void) {
    int devices = 0;
    if (hipGetDeviceCount(&devices) == hipSuccess && devices > 0) { printf("a GPU is visible\n"); return 2; }
    void* const f = (void*)0x1000;
    /* batch * n up to 2^31 - 1, in both dtypes and with few and many heads */
    const int batches[] = {1, 1, 1, 2147483647, 715827882, 65537, 46340}, ns[] = {2147483647, 2147483646, 2147483641, 1, 3, 32767, 46340};
    const int heads[] = {1, 2, 5, 40, 65535};
    for (int i = 0; i < 7; ++i) for (int h = 0; h < 5; ++h) for (int t = 0; t < 2; ++t) for (int D = 64; D <= 128; D += 64) {
        ot_qk_params p;
        memset(&p, 0, sizeof p);
        p.batch = batches[i]; p.n = ns[i]; p.q_heads = heads[h]; p.head_dim = D; p.dtype = t; p.rotary_dim = D;
        const int64_t s[3] = {(int64_t)p.q_heads * p.n * D, (int64_t)p.n * D, D};
        memcpy(p.q_strides, s, sizeof s); memcpy(p.qo_strides, s, sizeof s);
        expect("ot_qk_norm_rope", ot_qk_norm_rope(&p, f, NULL, NULL, NULL, f, f, f, (void*)0x2000, NULL, NULL), OT_ERR_HIP);
    }
    /* rows of an append up to OT_MAX_APPEND, batch * n up to 2^31 - 1 */
    const int many[] = {1, 127, 2147483647, 100}, rows[] = {OT_MAX_APPEND, OT_MAX_APPEND, 1, 1000000};
    for (int i = 0; i < 4; ++i) for (int ps = 16; ps <= 256; ps *= 4) for (int h = 1; h <= 65535; h = h * 40 + 15) for (int r = 0; r < 2; ++r) {
        ot_paged_cache c;
        memset(&c, 0, sizeof c);
        c.num_pages = 32767; c.page_size = ps; c.kv_heads = h; c.head_dim = 64; c.dtype = OT_E4M3; c.max_pages = (1 << 30) / ps - 1;
        const int64_t s[3] = {(int64_t)h * ps * 64, (int64_t)ps * 64, 64};
        memcpy(c.k_strides, s, sizeof s); memcpy(c.v_strides, s, sizeof s);
        c.k_pages = f; c.v_pages = (void*)0x100000; c.k_exp = f; c.v_exp = (void*)0x100000; c.page_table = f;
        ot_append_params a;
        memset(&a, 0, sizeof a);
        a.batch = many[i]; a.n = rows[i]; a.dtype = OT_BF16; a.rotary_dim = r * 64;
        const int64_t ks[3] = {0, 0, 64};
        memcpy(a.k_strides, ks, sizeof ks); memcpy(a.v_strides, ks, sizeof ks);
        expect("ot_kv_append_paged", ot_kv_append_paged(&a, &c, f, f, f, f, NULL, NULL, (void*)0x7f0000000000, NULL), OT_ERR_HIP);
    }
    if (!bad) printf("ok\n");
    return bad != 0;
}
