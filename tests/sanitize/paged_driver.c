/* The paged cache's front end at the ends of its arguments' ranges, under sanitizers: sizes whose products overflow 32 bits, and what
 * reaches the launchers. */
#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include "../../include/ws_synapse.h"

extern int g_paged_launches;
extern double g_turns[64];
extern unsigned char g_axis[64];

#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

int main(void)
{
    void *fake = (void *)0x100000;
    const int32_t *ints = fake;
    float *floats = fake;
    const size_t big = (size_t)1 << 60;
    const int most = 2147483647;
    ws_paged_cache c = {fake, fake, ints, ints, WS_BF16, 100, 4, 16, 128, 3, 200};
    const ws_rows rows = {fake, (int64_t)1 << 60, 128};
    const int pairs[4] = {16, 24, 0, 24};

    CHECK(ws_synapse_paged_append(&c, &rows, &rows, 5, ints, ints, 4, pairs, 1e4f, &rows, 8, fake, ints, (int32_t *)fake, floats, NULL) == WS_OK);
    CHECK(g_paged_launches == 1);
    for (int p = 0; p < 64; ++p) {
        CHECK(g_axis[p] == (p < 16 ? 0 : p < 40 ? 1 : 3));
        CHECK(fabs(g_turns[p] * 6.283185307179586476925 / pow(1e4, -p / 64.0) - 1) < 1e-15);
    }
    CHECK(ws_synapse_paged_append(&c, &rows, &rows, 5, ints, NULL, most, NULL, NAN, NULL, -most, NULL, NULL, NULL, NULL, NULL) == WS_OK);
    CHECK(ws_synapse_paged_append(&c, &rows, &rows, most, ints, NULL, 0, NULL, 0, NULL, 0, NULL, NULL, NULL, NULL, NULL) == WS_ERR_UNSUPPORTED);
    {
        const int overflow[2] = {most, most};
        CHECK(ws_synapse_paged_append(&c, &rows, &rows, 5, ints, ints, 2, overflow, 1e4f, NULL, 0, NULL, NULL, NULL, NULL, NULL) == WS_ERR_INVALID_ARG);
    }
    const int launches = g_paged_launches;
    CHECK(ws_synapse_paged_attend(&c, fake, most - 3, 0, floats, floats, 1, floats, floats, fake, big, NULL) == WS_ERR_UNSUPPORTED);
    CHECK(ws_synapse_paged_evict(&c, most, 0, most, ints, floats, floats, ints, (int32_t *)fake, (int32_t *)fake, NULL, fake, big, NULL) == WS_ERR_UNSUPPORTED);
    CHECK(ws_synapse_paged_evict(&c, 5, most, most, ints, floats, floats, ints, (int32_t *)fake, (int32_t *)fake, NULL, fake, big, NULL) == WS_ERR_INVALID_ARG);
    /* sizes on the cache itself */
    for (int field = 0; field < 6; ++field)
        for (int v = 0; v < 3; ++v) {
            const int value = v == 0 ? most : v == 1 ? -most - 1 : 1 << 24;
            ws_paged_cache d = c;
            if (field == 0) d.Hkv = value;
            if (field == 1) d.S = value;
            if (field == 2) d.per_seq = value;
            if (field == 3) d.page = value;
            if (field == 4) d.d = value;
            if (field == 5) d.dt = value;
            CHECK(ws_synapse_paged_append(&d, &rows, &rows, 5, ints, NULL, 0, NULL, 0, NULL, 0, NULL, NULL, NULL, NULL, NULL) != WS_OK);
            CHECK(ws_synapse_paged_attend(&d, fake, 4, 0, floats, NULL, 1, NULL, NULL, fake, big, NULL) != WS_OK);
            CHECK(ws_synapse_paged_evict(&d, 5, 0, 0, ints, floats, floats, ints, (int32_t *)fake, (int32_t *)fake, NULL, fake, big, NULL) != WS_OK);
        }
    /* rows of very many sequences: more tiles than 31 bits count; logits of one head beyond 32 bits of offsets */
    ws_paged_cache wide = {fake, fake, ints, ints, WS_F32, 100, 1, 256, 64, 1 << 16, 65535};
    CHECK(ws_synapse_paged_attend(&wide, fake, 1, 0, floats, NULL, 1, NULL, NULL, fake, big, NULL) == WS_ERR_UNSUPPORTED);
    CHECK(ws_synapse_workspace_bytes(WS_OP_PAGED_ATTEND, WS_F32, 1, 65535 * 256, 64, 0, 1 << 16, 1) == (size_t)-1);
    wide.S = 1;
    CHECK(ws_synapse_paged_attend(&wide, fake, 64, 0, floats, NULL, 1, NULL, floats, fake, big, NULL) == WS_ERR_UNSUPPORTED);
    CHECK(ws_synapse_workspace_bytes(WS_OP_PAGED_ATTEND, WS_F32, 1, 65535 * 256, 64, 1, 1, 64) == (size_t)-1);
    CHECK(ws_synapse_workspace_bytes(WS_OP_PAGED_ATTEND, WS_F32, 1, 65535 * 256, 64, 0, 1, 64) != (size_t)-1);
    CHECK(g_paged_launches == launches);
    /* the reported size is enough and what is asked for; one byte less is not */
    for (int weights = 0; weights < 2; ++weights)
        for (int g = 1; g <= 40; g += 13) {
            const size_t n = ws_synapse_workspace_bytes(WS_OP_PAGED_ATTEND, WS_BF16, 4, 3200, 128, weights, 3, 4 * g);
            CHECK(n != (size_t)-1 && n > 0);
            CHECK(ws_synapse_paged_attend(&c, fake, 4 * g, 0, floats, NULL, 1, NULL, weights ? floats : NULL, fake, n, NULL) == WS_OK);
            CHECK(ws_synapse_paged_attend(&c, fake, 4 * g, 0, floats, NULL, 1, NULL, weights ? floats : NULL, fake, n - 1, NULL) == WS_ERR_WORKSPACE);
        }
    c.per_seq = 10;
    CHECK(ws_synapse_workspace_bytes(WS_OP_PAGED_ATTEND, WS_BF16, 4, 160, 128, 0, 3, 8) == 0);
    CHECK(ws_synapse_paged_attend(&c, fake, 8, 0, floats, NULL, 1, NULL, NULL, NULL, 0, NULL) == WS_OK);
    for (int keep = 1; keep < 100000; keep = keep * 7 + 1) {
        c.per_seq = keep % 2 ? 200 : 2000;
        const size_t n = ws_synapse_workspace_bytes(WS_OP_PAGED_EVICT, WS_BF16, 4, c.per_seq * 16, 128, keep, 3, 0);
        CHECK(n != (size_t)-1 && n > 0);
        CHECK(ws_synapse_paged_evict(&c, keep, 0, 0, ints, floats, floats, ints, (int32_t *)fake, (int32_t *)fake, NULL, fake, n, NULL) == WS_OK);
        CHECK(ws_synapse_paged_evict(&c, keep, 0, 0, ints, floats, floats, ints, (int32_t *)fake, (int32_t *)fake, NULL, fake, n - 1, NULL) == WS_ERR_WORKSPACE);
    }
    for (int op = 7; op <= 10; ++op)
        (void)ws_synapse_workspace_bytes((ws_op)op, WS_BF16, most, 16777215, 128, most, most, most);
    printf("all checks passed\n");
    return 0;
}
