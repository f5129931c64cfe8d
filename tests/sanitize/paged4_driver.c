/* Drives the host side of the paged 4-bit cache calls, of relax_head_norm_rope and of relax_rope_table_scaled -- argument checks, and how their launches are cut --
 * against a build of the library whose host code is compiled with -fsanitize=address,undefined (tests/test_paged4_sanitizers.py).  The process sees no
 * GPU, so that a launch is refused by the runtime: device pointers are fake addresses that the host code must not dereference, host arrays have their exact size. */
#define _POSIX_C_SOURCE 200112L
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "relax_mi355.h"

static int failures = 0;
#define EXPECT(call, want) do { relax_status got_ = (call); if (got_ != (want)) { \
    fprintf(stderr, "%s:%d: %s returned %d, expected %d\n", __FILE__, __LINE__, #call, (int)got_, (int)(want)); ++failures; } } while (0)

#define DEV ((void *)(uintptr_t)0x7f0000100000ull)

static uint32_t state = 1;
static int32_t upto(int32_t most)                                       /* 1 .. most */
{
    state = state * 1664525u + 1013904223u;
    return 1 + (int32_t)((uint64_t)(state >> 8) * (uint64_t)most >> 24);
}

/* One call of each kind, of rows and lengths that the functions give; every launch is refused. */
static void calls(const relax_layer_dims *d, int B, int32_t q_most, int32_t past_most, int slotted, int device_table)
{
    int32_t *q = malloc(sizeof *q * (size_t)B), *kv = malloc(sizeof *q * (size_t)B), *slots = slotted ? malloc(sizeof *q * (size_t)B) : NULL;
    int32_t n = 0, L = 0;
    for (int b = 0; b < B; ++b) {
        q[b] = upto(q_most), kv[b] = q[b] + upto(past_most) - 1, n += q[b];
        if (slots) slots[b] = B - 1 - b;
        if (kv[b] > L) L = kv[b];
    }
    relax_seqs s = {B, q, kv, slots, device_table ? DEV : NULL};
    relax_paged4_cache c = {DEV, DEV, DEV, DEV, DEV, 100, 64, (d->kv_capacity + 63) / 64};
    relax_head_prep p = {DEV, DEV, 1e-6f, DEV, 32, RELAX_ROPE_PAIRS};
    const size_t bytes = relax_paged4_workspace_bytes(d, n, L, B), head_bytes = relax_head_workspace_bytes(d, B);
    const int64_t width = (int64_t)d->n_heads * d->head_dim, kv_width = (int64_t)d->n_kv_heads * d->head_dim;
    EXPECT(relax_paged4_append(DEV, width, DEV, DEV, kv_width, DEV, &p, &c, &s, d, n, DEV, bytes, NULL), RELAX_ERR_HIP);
    EXPECT(relax_paged4_append(DEV, width - 8, DEV, DEV, kv_width, DEV, &p, &c, &s, d, n, DEV, bytes, NULL), RELAX_ERR_SHAPE);
    EXPECT(relax_paged4_append(NULL, 0, DEV, DEV, kv_width, NULL, NULL, &c, &s, d, n, DEV, bytes - 1, NULL), RELAX_ERR_WORKSPACE);
    EXPECT(relax_paged4_attention(DEV, &c, &s, d, DEV, n, DEV, bytes, NULL), RELAX_ERR_HIP);
    EXPECT(relax_paged4_attention(DEV, &c, &s, d, DEV, n, DEV, bytes - 1, NULL), RELAX_ERR_WORKSPACE);
    EXPECT(relax_paged4_attention(DEV, &c, &s, d, DEV, n + 1, DEV, bytes + 100000, NULL), RELAX_ERR_SHAPE);
    EXPECT(relax_paged4_read(&c, &s, d, DEV, NULL, n, DEV, bytes, NULL), RELAX_ERR_HIP);
    EXPECT(relax_head_norm_rope(DEV, width, DEV, kv_width, DEV, width, DEV, kv_width, &p, &s, d, n, DEV, head_bytes, NULL), RELAX_ERR_HIP);
    EXPECT(relax_head_norm_rope(DEV, width, NULL, 0, DEV, width, NULL, 0, &p, &s, d, n, DEV, head_bytes - 1, NULL), RELAX_ERR_WORKSPACE);
    free(q), free(kv), free(slots);
}

int main(void)
{
    setenv("HIP_VISIBLE_DEVICES", "-1", 1);
    static const struct { int32_t heads, kv_heads, d; } shapes[] = {{4, 4, 64}, {64, 8, 128}, {40, 40, 128}, {16, 2, 64}, {7, 1, 128}, {200, 200, 64}};
    static const int sizes[] = {1, 2, 16, 17, 127, 128, 129, 1000};
    static const int32_t most[][2] = {{1, 1}, {1, 120000}, {6, 3000}, {40, 100}, {900, 1}, {2043, 600}, {1, 1 << 30}};
    for (unsigned i = 0; i < sizeof shapes / sizeof *shapes; ++i)
        for (unsigned j = 0; j < sizeof sizes / sizeof *sizes; ++j)
            for (unsigned k = 0; k < sizeof most / sizeof *most; ++k) {
                const relax_layer_dims d = {shapes[i].heads * shapes[i].d, shapes[i].heads, shapes[i].kv_heads, shapes[i].d, 688, 32, 1e-5f, 10000.0f, 1 << 30, sizes[j]};
                calls(&d, sizes[j], most[k][0], most[k][1], (int)((i + j + k) % 2), (int)((j + k) % 3 == 0));
            }
    /* sizes at the ends of their types */
    const relax_layer_dims d = {256, 4, 2, 64, 688, 32, 1e-5f, 10000.0f, INT32_MAX, INT32_MAX};
    if (relax_paged4_workspace_bytes(&d, INT32_MAX, INT32_MAX, INT32_MAX) == 0 || relax_head_workspace_bytes(&d, INT32_MAX) == 0) ++failures;
    int32_t one = 1, far = INT32_MAX;
    relax_seqs s = {1, &one, &far, NULL, NULL};
    relax_paged4_cache c = {DEV, DEV, DEV, DEV, DEV, 1 << 24, 256, 1 << 23};
    EXPECT(relax_paged4_attention(DEV, &c, &s, &d, DEV, 1, DEV, 256, NULL), RELAX_ERR_WORKSPACE);
    EXPECT(relax_paged4_attention(DEV, &c, &s, &d, DEV, 1, DEV, (size_t)1 << 40, NULL), RELAX_ERR_UNSUPPORTED);
    for (int scaling = RELAX_ROPE_PLAIN; scaling <= RELAX_ROPE_WAVELENGTH_RAMP; ++scaling)
        for (int32_t R = 2; R <= 256; R += 2)
            for (int b = 0; b < 3; ++b) {
                const relax_rope_scaling sc = {scaling, R, b == 0 ? nextafter(1.0, 2.0) : b == 1 ? 10000.0 : 1e300, b == 1 ? 4.0 : 1e-300, b == 2 ? 1e300 : 1.0, 1e-300, b ? 4.0 : 2e-300, 0.0};
                EXPECT(relax_rope_table_scaled(&sc, b == 2 ? 1 << 30 : 1 + R, DEV, NULL), RELAX_ERR_HIP);
            }
    if (failures == 0) printf("paged4 driver ok\n");
    return failures != 0;
}
