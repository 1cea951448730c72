/* Drives the host half of the paged calls (sizes, plans and every check of the arguments) through planner handles, for a
 * build of the library with sanitizers on its host code.  No GPU: pointers are compared and tested for alignment, never read. */
#include <stdio.h>
#include <string.h>

#include "commvq.h"

#define P ((void *)(size_t)(1u << 20))

static int fails;
static void expect(commvq_status got, commvq_status want, const char *what)
{
    if (got != want) { printf("pages_driver: %s: %d, not %d\n", what, got, want); ++fails; }
}

int main(void)
{
    const int heads[] = {1, 2, 4, 8}, books[] = {16, 32};
    for (int gi = 0; gi < 4; ++gi)
        for (int mi = 0; mi < 4; ++mi)
            for (int f = 0; f < 2; ++f) {
                commvq_config c;
                memset(&c, 0, sizeof c);
                c.n_kv_heads = 8; c.n_q_heads = 8 * heads[gi]; c.head_dim = 128; c.m_key = books[mi & 1]; c.m_val = books[mi >> 1];
                c.k = 256; c.q_dtype = c.codebook_dtype = f; c.rope_base = 500000.0; c.max_position = 1 << 24;
                commvq_handle *h = NULL;
                expect(commvq_create_planner(&c, &h), COMMVQ_OK, "planner");
                const int lens[] = {0, 1, 15, 31, 33, 1000, 4097, 131072, 1 << 24}, nodes[] = {1, 3, 16, 64}, batches[] = {1, 3, 64, 1000};
                for (int l = 0; l < 9; ++l)
                    for (int n = 0; n < 4; ++n)
                        for (int b = 0; b < 4; ++b) {
                            size_t bytes = 0;
                            const int total = batches[b] * nodes[n];
                            expect(commvq_tree_workspace_bytes(h, batches[b], total, nodes[n], lens[l], &bytes), COMMVQ_OK, "workspace size");
                            commvq_pages p = {16, 1 << 24, 1 << 21, 3};
                            unsigned char axis[64];
                            for (int j = 0; j < 64; ++j) axis[j] = (unsigned char)(j % 3);
                            commvq_tree t;
                            memset(&t, 0, sizeof t);
                            t.batch = batches[b]; t.total_nodes = total; t.max_nodes = nodes[n]; t.max_seqlen = lens[l];
                            t.seq_lens = t.block_tables = t.cu_nodes = t.node_pos = t.key_pos = P;
                            t.pair_axis = axis;
                            const void *tables = f ? P : NULL;
                            expect(commvq_tree_attn(h, &p, &t, P, P, P, P, P, P, P, tables, P, P, bytes, NULL), COMMVQ_ERR_NO_DEVICE, "attention");
                            expect(commvq_tree_attn(h, &p, &t, P, P, P, P, P, P, P, tables, P, P, bytes - 1, NULL), COMMVQ_ERR_WORKSPACE, "attention, small workspace");
                            axis[63] = 3;
                            expect(commvq_tree_attn(h, &p, &t, P, P, P, P, P, P, P, tables, P, P, bytes, NULL), COMMVQ_ERR_SHAPE, "attention, axis");
                        }
                commvq_pages p = {32, 100, 4, 1};
                expect(commvq_store_pages(h, &p, 7, P, P, P, P, P, P, P, NULL), COMMVQ_ERR_NO_DEVICE, "store");
                expect(commvq_store_pages(h, &p, 7, P, P, P, NULL, P, P, P, NULL), COMMVQ_ERR_NULL, "store, positions");
                size_t bytes = 0;
                expect(commvq_tree_table_bytes(h, &bytes), f ? COMMVQ_OK : COMMVQ_ERR_CONFIG, "table size");
                expect(commvq_tree_prepare(h, P, P, P, NULL), f ? COMMVQ_ERR_NO_DEVICE : COMMVQ_ERR_CONFIG, "prepare");
                expect(commvq_destroy(h), COMMVQ_OK, "destroy");
            }
    expect(commvq_page_tables(NULL, 1, P, P, P, 1, P, P, P, P, P, 1, P, NULL), COMMVQ_ERR_NULL, "tables, no pages");
    expect(commvq_tree_attn(NULL, NULL, NULL, P, P, P, P, P, P, P, P, P, P, 0, NULL), COMMVQ_ERR_NULL, "attention, no handle");
    expect(commvq_tree_workspace_bytes(NULL, 1, 1, 1, 1, NULL), COMMVQ_ERR_NULL, "size, no handle");
    if (!fails) printf("pages_driver: ok\n");
    return fails != 0;
}
