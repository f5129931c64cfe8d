/* Drives the host side of the paged cache calls and of relax_token_logprobs -- everything they do before they enqueue anything -- against a build of
 * the library whose host code is compiled with -fsanitize=address,undefined (tests/test_paged_sanitizers.py).  No GPU: device pointers are fake
 * addresses that the host code must not dereference, host arrays have their exact size.  Every descriptor is refused late, for its
 * workspace, so that all of it has been read. */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "relax_mi355.h"

static int failures = 0;
#define EXPECT(call, want) do { relax_status got_ = (call); if (got_ != (want)) { \
    fprintf(stderr, "%s:%d: %s returned %d, expected %d\n", __FILE__, __LINE__, #call, (int)got_, (int)(want)); ++failures; } } while (0)

#define DEV ((void *)(uintptr_t)0x7f0000100000ull)

static int32_t *ints(int count, int32_t value)
{
    int32_t *p = malloc((size_t)count * sizeof(int32_t));
    for (int i = 0; i < count; ++i) p[i] = value;
    return p;
}

int main(void)
{
    const int sizes[] = {1, 16, 17, 127, 128, 129, 1000, 65535};
    for (unsigned i = 0; i < sizeof sizes / sizeof *sizes; ++i) {
        const int B = sizes[i];
        relax_layer_dims d = {256, 4, 2, 64, 688, 32, 1e-5f, 10000.0f, 4096, B};
        relax_paged_cache c = {DEV, DEV, DEV, DEV, DEV, NULL, 100, 64, 64};
        for (int slotted = 0; slotted < 2; ++slotted) {
            int32_t *q = ints(B, 1), *kv = ints(B, 300), *slots = slotted ? ints(B, B - 1) : NULL;
            q[B - 1] = 77;
            relax_seqs s = {B, q, kv, slots, NULL};
            const int32_t n = B - 1 + 77;
            const size_t bytes = relax_paged_workspace_bytes(&d, n, 300, B);
            EXPECT(relax_paged_append(DEV, 512, DEV, DEV, 512, DEV, &c, &s, &d, 1, DEV, bytes, NULL), RELAX_ERR_SHAPE);
            EXPECT(relax_paged_append(DEV, 256, DEV, DEV, 512, DEV, &c, &s, &d, n, DEV, bytes - 1, NULL), RELAX_ERR_WORKSPACE);
            EXPECT(relax_paged_append(DEV, 512, DEV, DEV, 512, DEV, &c, &s, &d, n, DEV, bytes, NULL), RELAX_ERR_SHAPE);
            EXPECT(relax_paged_attention(DEV, &c, &s, &d, DEV, n, DEV, bytes - 1, NULL), RELAX_ERR_WORKSPACE);
            EXPECT(relax_paged_read(&c, &s, &d, DEV, NULL, n, DEV, bytes - 1, NULL), RELAX_ERR_WORKSPACE);
            kv[B - 1] = 4097;
            EXPECT(relax_paged_attention(DEV, &c, &s, &d, DEV, n, DEV, bytes, NULL), RELAX_ERR_CAPACITY);
            free(q), free(kv), free(slots);
        }
    }
    /* sizes at the ends of their types */
    relax_layer_dims d = {256, 4, 2, 64, 688, 32, 1e-5f, 10000.0f, INT32_MAX, INT32_MAX};
    if (relax_paged_workspace_bytes(&d, INT32_MAX, INT32_MAX, INT32_MAX) == 0) ++failures;
    int32_t one = 1, far = INT32_MAX;
    relax_seqs s = {1, &one, &far, NULL, NULL};
    relax_paged_cache c = {DEV, DEV, DEV, DEV, DEV, NULL, 1 << 24, 256, 1 << 23};
    EXPECT(relax_paged_attention(DEV, &c, &s, &d, DEV, 1, DEV, 256, NULL), RELAX_ERR_WORKSPACE);
    c.n_pages = INT32_MAX;
    EXPECT(relax_paged_attention(DEV, &c, &s, &d, DEV, 1, DEV, 256, NULL), RELAX_ERR_UNSUPPORTED);
    if (relax_token_logprobs_workspace_bytes(INT32_MAX, 1 << 20, 32) == 0 || relax_token_logprobs_workspace_bytes(1, INT32_MAX, 32) != 0) ++failures;
    EXPECT(relax_token_logprobs(DEV, 99, DEV, DEV, NULL, NULL, NULL, 1, 100, 0, NULL, 0, NULL), RELAX_ERR_SHAPE);
    EXPECT(relax_token_logprobs(DEV, 100, NULL, NULL, NULL, NULL, NULL, 1, 100, 0, NULL, 0, NULL), RELAX_ERR_NULL);
    if (failures == 0) printf("paged driver ok\n");
    return failures != 0;
}
