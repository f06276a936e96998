/* Sanitizer driver of the argument checks of the operators between a decoder's projections: as abi_check.c, calls that return
 * before anything is enqueued, against a build of libqii whose host half is instrumented.  Pointers such as 0x1000 are never
 * dereferenced by the host code.  Built and run by tests/test_sanitizers_decode.py.  Prints "decode abi: ok" and returns 0. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "../../include/qii.h"

static int fails = 0;
#define EXPECT(call, want)                                                                      \
    do {                                                                                        \
        const int got_ = (int)(call);                                                           \
        if (got_ != (int)(want)) {                                                              \
            fprintf(stderr, "line %d: %s returned %d (%s), expected %d\n", __LINE__, #call, got_, qii_last_error(), (int)(want)); \
            ++fails;                                                                            \
        }                                                                                       \
    } while (0)

#define P(x) ((void *)(uintptr_t)(x))

static const int64_t kBig = INT64_MAX;

static qii_status rotary(const qii_rotation *r, int64_t tokens, int64_t heads, int64_t dim, qii_dtype dt)
{
    return qii_rotary(P(0x1000), dt, tokens, heads, dim, 0, 0, P(0x2000), r, 0, NULL, 0, 0, NULL);   /* (y is missing) */
}

static qii_status append(const qii_kv_cache *c, const qii_page_table *t, const qii_rotation *r, qii_mode m, int64_t tokens)
{
    return qii_kv_append(NULL, P(0x1000), QII_BF16, tokens, 0, 0, 0, 0, P(0x2000), NULL, t, r, m, c, NULL);   /* (k is missing) */
}

static qii_status attend(const qii_kv_cache *c, const qii_page_table *t, int64_t seqs, int64_t heads, int64_t longest, int64_t window)
{
    return qii_paged_attention(NULL, QII_F32, seqs, heads, 0, 0, c, t, P(0x2000), longest, NULL, window, 1.0f, NULL, P(0x1000), 0, 0, NULL,
                               NULL, 0, NULL);   /* (q is missing) */
}

int main(void)
{
    /* tables */
    float *t = P(0x1000);
    EXPECT(qii_rotary_table(t, 4, 3, 1e4, QII_ROTARY_SCALING_NONE, 1, 0, 0, 0, 1, NULL), QII_BAD_SHAPE);
    EXPECT(qii_rotary_table(t, 4, 0, 1e4, QII_ROTARY_SCALING_NONE, 1, 0, 0, 0, 1, NULL), QII_BAD_SHAPE);
    EXPECT(qii_rotary_table(t, -1, 4, 1e4, QII_ROTARY_SCALING_NONE, 1, 0, 0, 0, 1, NULL), QII_BAD_SHAPE);
    EXPECT(qii_rotary_table(t, kBig, 4, 1e4, QII_ROTARY_SCALING_NONE, 1, 0, 0, 0, 1, NULL), QII_BAD_SHAPE);
    EXPECT(qii_rotary_table(t, 4, 4, 0.0, QII_ROTARY_SCALING_NONE, 1, 0, 0, 0, 1, NULL), QII_INVALID_ARG);
    EXPECT(qii_rotary_table(t, 4, 4, NAN, QII_ROTARY_SCALING_NONE, 1, 0, 0, 0, 1, NULL), QII_INVALID_ARG);
    EXPECT(qii_rotary_table(t, 4, 4, 1e4, QII_ROTARY_SCALING_NONE, 1, 0, 0, 0, INFINITY, NULL), QII_INVALID_ARG);
    EXPECT(qii_rotary_table(t, 4, 4, 1e4, (qii_rotary_scaling)4, 1, 0, 0, 0, 1, NULL), QII_INVALID_ARG);
    EXPECT(qii_rotary_table(t, 4, 4, 1e4, (qii_rotary_scaling)-1, 1, 0, 0, 0, 1, NULL), QII_INVALID_ARG);
    EXPECT(qii_rotary_table(t, 4, 4, 1e4, QII_ROTARY_SCALING_LINEAR, 0, 0, 0, 0, 1, NULL), QII_INVALID_ARG);
    EXPECT(qii_rotary_table(t, 4, 4, 1e4, QII_ROTARY_SCALING_BY_PARTS, 4, 0, 32, 1, 1, NULL), QII_INVALID_ARG);
    EXPECT(qii_rotary_table(t, 4, 4, 1e4, QII_ROTARY_SCALING_BY_PARTS, 4, 100, 1, 1, 1, NULL), QII_INVALID_ARG);
    EXPECT(qii_rotary_table(NULL, 4, 4, 1e4, QII_ROTARY_SCALING_NONE, 1, 0, 0, 0, 1, NULL), QII_INVALID_ARG);
    EXPECT(qii_rotary_table(P(0x1004), 4, 4, 1e4, QII_ROTARY_SCALING_NONE, 1, 0, 0, 0, 1, NULL), QII_INVALID_ARG);
    EXPECT(qii_rotary_table(NULL, 0, 4, 1e4, QII_ROTARY_SCALING_NONE, 1, 0, 0, 0, 1, NULL), QII_OK);
    /* rotations */
    qii_rotation r = {t, 100, 64, QII_ROTARY_HALF};
    EXPECT(rotary(&r, 4, 2, 64, QII_F32), QII_INVALID_ARG);
    EXPECT(rotary(&r, 0, 2, 64, QII_F32), QII_OK);
    EXPECT(rotary(&r, 4, 0, 64, QII_F32), QII_OK);
    EXPECT(rotary(&r, 4, 2, 62, QII_F32), QII_BAD_SHAPE);
    EXPECT(rotary(&r, 4, 2, 0, QII_F32), QII_BAD_SHAPE);
    EXPECT(rotary(&r, -1, 2, 64, QII_F32), QII_BAD_SHAPE);
    EXPECT(rotary(&r, kBig, 2, 64, QII_F32), QII_BAD_SHAPE);
    EXPECT(rotary(&r, 4, kBig, 64, QII_F32), QII_BAD_SHAPE);
    EXPECT(rotary(&r, 4, 2, kBig, QII_F32), QII_BAD_SHAPE);
    EXPECT(rotary(&r, 4, 2, 64, (qii_dtype)2), QII_INVALID_ARG);
    EXPECT(rotary(NULL, 4, 2, 64, QII_F32), QII_INVALID_ARG);
    EXPECT(qii_rotary(P(0x1000), QII_F32, 4, 2, 64, 128, 64, P(0x2000), &r, 0, P(0x1000), 256, 64, NULL), QII_INVALID_ARG);
    EXPECT(qii_rotary(P(0x1002), QII_F32, 4, 2, 64, 128, 64, P(0x2000), &r, 0, P(0x3000), 128, 64, NULL), QII_INVALID_ARG);
    EXPECT(qii_rotary(P(0x1000), QII_F32, 4, 2, 64, 128, 64, P(0x2002), &r, 0, P(0x3000), 128, 64, NULL), QII_INVALID_ARG);
    const qii_rotation bad[] = {{t, 0, 64, QII_ROTARY_HALF}, {t, kBig, 64, QII_ROTARY_HALF}, {t, 100, 63, QII_ROTARY_HALF}, {t, 100, 0, QII_ROTARY_HALF},
                                {t, 100, 66, QII_ROTARY_HALF}, {t, 100, -2, QII_ROTARY_HALF}, {NULL, 100, 64, QII_ROTARY_HALF},
                                {P(0x1008), 100, 64, QII_ROTARY_HALF}, {t, 100, 64, (qii_rotary_layout)2}};
    const qii_kv_cache cache = {P(0x1000), P(0x2000), P(0x3000), P(0x4000), P(0x5000), P(0x6000), 8, 2, 16, 64, QII_KV_NVFP4};
    const qii_page_table table = {P(0x7000), 4, 2, 2};
    for (unsigned i = 0; i < sizeof bad / sizeof bad[0]; ++i) {
        const qii_status want = i < 6 ? QII_BAD_SHAPE : QII_INVALID_ARG;
        EXPECT(rotary(&bad[i], 4, 2, 64, QII_BF16), want);
        EXPECT(append(&cache, &table, &bad[i], QII_RTN, 4), want);
    }
    /* the cache and its page table */
    EXPECT(append(&cache, &table, NULL, QII_RTN, 4), QII_INVALID_ARG);   /* k */
    EXPECT(append(&cache, &table, NULL, QII_RTN, 0), QII_OK);
    EXPECT(append(&cache, &table, NULL, QII_SR, 0), QII_INVALID_ARG);
    EXPECT(append(&cache, &table, NULL, (qii_mode)17, 0), QII_INVALID_ARG);
    EXPECT(append(&cache, &table, NULL, QII_RTN, -1), QII_BAD_SHAPE);
    EXPECT(append(&cache, &table, NULL, QII_RTN, kBig), QII_BAD_SHAPE);
    EXPECT(append(NULL, &table, NULL, QII_RTN, 0), QII_INVALID_ARG);
    EXPECT(append(&cache, NULL, NULL, QII_RTN, 0), QII_INVALID_ARG);
    for (int i = 0; i < 24; ++i) {
        qii_kv_cache c = cache;
        qii_status want = QII_BAD_SHAPE;
        switch (i) {
        case 0: c.head_dim = 0; break;
        case 1: c.head_dim = 24; break;
        case 2: c.head_dim = 272; break;
        case 3: c.head_dim = kBig; break;
        case 4: c.page_size = 0; break;
        case 5: c.page_size = 24; break;
        case 6: c.page_size = 65552; break;
        case 7: c.page_size = -16; break;
        case 8: c.kv_heads = 0; break;
        case 9: c.kv_heads = kBig; break;
        case 10: c.kv_heads = 1 << 21; break;
        case 11: c.pages = -1; break;
        case 12: c.pages = kBig; break;
        default:
            want = QII_INVALID_ARG;
            switch (i) {
            case 13: c.k = NULL; break;
            case 14: c.v = P(0x2008); break;
            case 15: c.k_scales = NULL; break;
            case 16: c.v_scales = P(0x4001); break;
            case 17: c.k_scale = NULL; break;
            case 18: c.v_scale = P(0x6002); break;
            case 19: c.kind = (qii_kv_kind)2; break;
            case 20: c.kind = (qii_kv_kind)-1; break;
            default: want = QII_OK; c.pages = 0; c.k = c.v = NULL; c.k_scales = c.v_scales = NULL; break;
            }
        }
        EXPECT(append(&c, &table, NULL, QII_RTN, 0), want);
        EXPECT(qii_kv_read(&c, &table, 0, NULL, NULL, NULL, NULL, QII_F32, 0, 0, 0, 0, NULL), want);
    }
    qii_kv_cache plain = cache;
    plain.kind = QII_KV_BF16;
    plain.k_scales = plain.v_scales = NULL;
    plain.k_scale = plain.v_scale = NULL;
    EXPECT(append(&plain, &table, NULL, QII_SR, 0), QII_OK);   /* (the mode is not looked at) */
    const qii_page_table tables[] = {{P(0x7000), -1, 2, 2}, {P(0x7000), 4, -1, 2}, {P(0x7000), 4, 2, 1}, {P(0x7000), kBig, 2, 2}, {P(0x7000), 4, kBig, kBig},
                                     {NULL, 4, 2, 2}, {P(0x7002), 4, 2, 2}};
    for (unsigned i = 0; i < sizeof tables / sizeof tables[0]; ++i)
        EXPECT(append(&cache, &tables[i], NULL, QII_RTN, 0), i < 5 ? QII_BAD_SHAPE : QII_INVALID_ARG);
    EXPECT(qii_kv_read(&cache, &table, 3, P(0x8000), NULL, NULL, NULL, QII_F32, 0, 0, 0, 0, NULL), QII_INVALID_ARG);
    EXPECT(qii_kv_read(&cache, &table, 3, NULL, NULL, P(0x9000), NULL, QII_F32, 0, 0, 0, 0, NULL), QII_INVALID_ARG);
    EXPECT(qii_kv_read(&cache, &table, 3, P(0x8000), P(0x8001), P(0x9000), NULL, QII_F32, 0, 0, 0, 0, NULL), QII_INVALID_ARG);
    EXPECT(qii_kv_read(&cache, &table, 3, P(0x8000), NULL, NULL, P(0x9002), QII_F32, 0, 0, 0, 0, NULL), QII_INVALID_ARG);
    EXPECT(qii_kv_read(&cache, &table, 3, P(0x8000), NULL, P(0x9000), NULL, (qii_dtype)9, 0, 0, 0, 0, NULL), QII_INVALID_ARG);
    /* attention */
    EXPECT(attend(&cache, &table, 4, 8, 32, 0), QII_INVALID_ARG);   /* q */
    EXPECT(attend(&cache, &table, 3, 8, 32, 0), QII_BAD_SHAPE);
    EXPECT(attend(&cache, &table, 4, 7, 32, 0), QII_BAD_SHAPE);
    EXPECT(attend(&cache, &table, 4, 0, 32, 0), QII_BAD_SHAPE);
    EXPECT(attend(&cache, &table, 4, kBig - 1, 32, 0), QII_BAD_SHAPE);
    EXPECT(attend(&cache, &table, 4, 1 << 21, 32, 0), QII_BAD_SHAPE);
    EXPECT(attend(&cache, &table, 4, 8, -1, 0), QII_BAD_SHAPE);
    EXPECT(attend(&cache, &table, 4, 8, 32, -1), QII_BAD_SHAPE);
    const qii_page_table none = {NULL, 0, 0, 0};
    EXPECT(attend(&cache, &none, 0, 8, 32, 0), QII_OK);
    EXPECT(qii_paged_attention(P(0x1000), QII_F32, 4, 8, 0, 0, &cache, &table, P(0x2000), 32, NULL, 0, 1.0f, NULL, P(0x1000), 0, 0, P(0x3002), NULL, 0, NULL), QII_INVALID_ARG);
    EXPECT(qii_paged_attention(P(0x1000), QII_F32, 4, 8, 0, 0, &cache, &table, P(0x2000), 32, NULL, 0, 1.0f, NULL, P(0x1000), 0, 0, NULL, P(0x3080), 1 << 20, NULL), QII_INVALID_ARG);
    EXPECT(qii_paged_attention(P(0x1000), QII_F32, 4, 8, 0, 0, &cache, &table, P(0x2000), 32, P(0x3001), 0, 1.0f, NULL, P(0x1000), 0, 0, NULL, NULL, 0, NULL), QII_INVALID_ARG);
    /* workspace sizes over small, large and impossible arguments */
    const int64_t n[] = {-5, 0, 1, 3, 16, 128, 1000, 131072, 1 << 30, INT32_MAX, kBig};
    const int count = (int)(sizeof n / sizeof n[0]);
    volatile size_t sink = 0;
    for (int a = 0; a < count; ++a)
        for (int b = 0; b < count; ++b)
            for (int c = 0; c < count; ++c)
                for (int d = 0; d < count; ++d) sink ^= qii_paged_attention_workspace_bytes(n[a], n[b], n[c], 128, n[d]) ^ qii_paged_attention_workspace_bytes(n[a], n[b], 1, 256, n[d]);
    if (qii_paged_attention_workspace_bytes(1, 3, 2, 128, 100) != 0) ++fails;
    if (fails) return 1;
    printf("decode abi: ok (%u)\n", (unsigned)(sink & 1u));
    return 0;
}
