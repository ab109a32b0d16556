/*
 * The host side of a block's operators under AddressSanitizer and UndefinedBehaviorSanitizer: id lists of exactly
 * their size, structs on the heap, sizes and strides at the ends of their types. No call reaches a launch: device
 * pointers are fabricated addresses that the checks reject, and nothing is dereferenced. Prints "ok <checks>".
 */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "rhymeflow.h"

static int checks = 0;

#define EXPECT(call, want)                                                                      \
    do {                                                                                        \
        const int got_ = (call);                                                                \
        ++checks;                                                                               \
        if (got_ != (want)) {                                                                   \
            printf("FAIL line %d: %s returned %d, expected %d (%s)\n", __LINE__, #call, got_,   \
                   (int)(want), rf_last_error());                                               \
            return 1;                                                                           \
        }                                                                                       \
    } while (0)

#define DEV(i) ((void *)(uintptr_t)(0x100000000000ull + (uint64_t)(i) * 0x10000000000ull))

int main(void) {
    int32_t *ids = (int32_t *)malloc(sizeof(int32_t) * RF_MAX_FRAMES);
    for (int i = 0; i < RF_MAX_FRAMES; ++i) ids[i] = i;
    rf_rotary_axes *ax = (rf_rotary_axes *)malloc(sizeof *ax);
    const int32_t whole[3] = {64, 96, 96};
    memcpy(ax->dims, whole, sizeof whole);
    for (int a = 0; a < 3; ++a) ax->theta[a] = 10000.0, ax->origin[a] = 0.0, ax->step[a] = 1.0;
#define ROTARY(q, qo, k, ko, M, T, H, W, hq, hk, d, s0, s1, s2, s3, fl, dt) \
    rf_rotary(q, qo, k, ko, ids, M, T, H, W, hq, hk, d, ax, s0, s1, s2, s3, fl, dt, NULL)
    /* every frame, every pair: rejected at the last check (an output over an input) */
    EXPECT(ROTARY(DEV(0), DEV(0), DEV(1), DEV(0), 256, 256, 8, 8, 2, 2, 256, 0, 0, 0, 0, 0, RF_BF16), RF_ERR_INVALID_ARG);
    EXPECT(ROTARY(DEV(0), DEV(0), DEV(1), DEV(0), 256, 256, 8, 8, 2, 2, 256, 0, 0, 0, 0, RF_ROTARY_INVERSE, RF_F32),
           RF_ERR_INVALID_ARG);
    EXPECT(ROTARY(DEV(0), DEV(1), NULL, NULL, 256, 256, 65536, 1024, 65535, 0, 256, INT64_MAX, 0, 0, 0, 0, RF_F32),
           RF_ERR_RANGE);
    EXPECT(ROTARY(DEV(0), DEV(1), NULL, NULL, 1, 1, 1, 1, 1, 0, 256, INT64_MIN, 0, 0, 0, 0, RF_F32), RF_ERR_INVALID_ARG);
    EXPECT(ROTARY(DEV(0), DEV(1), NULL, NULL, INT32_MAX, INT32_MAX, 1, 1, 1, 0, 256, 0, 0, 0, 0, 0, RF_F32), RF_ERR_RANGE);
    EXPECT(ROTARY(DEV(0), DEV(1), NULL, NULL, 1, 1, INT32_MAX, INT32_MAX, 1, 0, 256, 0, 0, 0, 0, 0, RF_F32), RF_ERR_RANGE);
    EXPECT(ROTARY(DEV(0), DEV(1), DEV(2), DEV(3), 1, 1, 1, 1, 1, INT32_MAX, 256, 0, 0, 0, 0, 0, RF_F32), RF_ERR_RANGE);
    for (int a = 0; a < 3; ++a) {
        ax->dims[a] = INT32_MAX - 1;
        EXPECT(ROTARY(DEV(0), DEV(1), NULL, NULL, 1, 1, 1, 1, 1, 0, 256, 0, 0, 0, 0, 0, RF_F32), RF_ERR_INVALID_ARG);
        ax->dims[a] = INT32_MIN;
        EXPECT(ROTARY(DEV(0), DEV(1), NULL, NULL, 1, 1, 1, 1, 1, 0, 256, 0, 0, 0, 0, 0, RF_F32), RF_ERR_INVALID_ARG);
        ax->dims[a] = whole[a];
        ax->step[a] = 1e300;
        EXPECT(ROTARY(DEV(0), DEV(1), NULL, NULL, 1, 1, 1, 1, 1, 0, 256, 0, 0, 0, 0, 0, RF_F32), RF_ERR_RANGE);
        ax->step[a] = NAN;
        EXPECT(ROTARY(DEV(0), DEV(1), NULL, NULL, 1, 1, 1, 1, 1, 0, 256, 0, 0, 0, 0, 0, RF_F32), RF_ERR_INVALID_ARG);
        ax->step[a] = 1.0;
    }

    rf_cross_layout *l = (rf_cross_layout *)malloc(sizeof *l);
#define CROSS(out, B, Lq, Lk, h, kh, d, lay, dt, ws, wb) \
    rf_cross_attention(DEV(0), DEV(1), DEV(2), out, NULL, NULL, B, Lq, Lk, h, kh, d, lay, dt, ws, wb, NULL)
    for (int i = 0; i < 3; ++i) l->q[i] = l->k[i] = l->v[i] = l->out[i] = INT64_MAX;
    EXPECT(CROSS(DEV(3), 2, 5, 7, 4, 2, 64, l, RF_BF16, NULL, 0), RF_ERR_RANGE);
    for (int i = 0; i < 3; ++i) l->q[i] = l->k[i] = l->v[i] = l->out[i] = INT64_MIN;
    EXPECT(CROSS(DEV(3), 2, 5, 7, 4, 2, 64, l, RF_BF16, NULL, 0), RF_ERR_INVALID_ARG);
    for (int i = 0; i < 3; ++i) l->q[i] = l->k[i] = l->v[i] = l->out[i] = 1000000000000000000LL;
    EXPECT(CROSS(DEV(3), 2, 5, 7, 4, 2, 64, l, RF_F32, NULL, 0), RF_ERR_UNSUPPORTED);
    EXPECT(CROSS(DEV(3), INT32_MAX, INT32_MAX, 1, INT32_MAX, 1, 64, NULL, RF_F32, NULL, 0), RF_ERR_RANGE);
    EXPECT(CROSS(DEV(3), INT32_MAX, 1, INT32_MAX, 1, 1, 64, NULL, RF_F32, NULL, 0), RF_ERR_RANGE);
    EXPECT(CROSS(DEV(3), 1, 1, INT32_MAX, 1, 1, 64, NULL, RF_F32, NULL, 0), RF_ERR_RANGE);
    EXPECT(CROSS(DEV(0), 1, 1 << 28, 1, 1, 1, 128, NULL, RF_F32, NULL, 0), RF_ERR_INVALID_ARG);
    EXPECT(CROSS(DEV(3), 1, 4, 9, 1, 1, 128, NULL, RF_F32, DEV(4), INT64_MIN), RF_ERR_INVALID_ARG);
    int64_t *bytes = (int64_t *)malloc(sizeof *bytes);
    EXPECT(rf_cross_attention_workspace(1, 1, 1 << 30, 1, 1, 128, RF_BF16, RF_MAX_COMPUTE_UNITS, bytes), RF_OK);
    EXPECT(rf_cross_attention_workspace(64, 1 << 18, 1 << 30, 32, 1, 64, RF_F32, 1, bytes), RF_OK);
    EXPECT(rf_cross_attention_workspace(1, 1, INT32_MAX, 1, 1, 128, RF_BF16, 256, bytes), RF_ERR_RANGE);

#define LINEAR(y, g, res, M, T, N, K, n, act, fl, dt, ws, wb) \
    rf_frame_linear(DEV(0), DEV(1), DEV(2), g, res, y, ids, M, T, N, K, n, act, fl, dt, ws, wb, NULL)
    EXPECT(LINEAR(DEV(0), NULL, NULL, 256, 256, 8388607, 2097144, 2147483640, 0, 0, RF_F32, NULL, 0), RF_ERR_RANGE);
    EXPECT(LINEAR(DEV(0), NULL, NULL, 256, 256, 8388607, 64, 64, 0, 0, RF_BF16, NULL, 0), RF_ERR_INVALID_ARG);
    EXPECT(LINEAR(DEV(5), NULL, NULL, 256, 256, INT64_MAX, 64, 64, 0, 0, RF_BF16, NULL, 0), RF_ERR_RANGE);
    EXPECT(LINEAR(DEV(5), NULL, NULL, 1, 1, INT64_MIN, 64, 64, 0, 0, RF_BF16, NULL, 0), RF_ERR_INVALID_ARG);
    EXPECT(LINEAR(DEV(5), NULL, NULL, 1, 1, 1, INT32_MAX - 7, 64, 0, 0, RF_BF16, NULL, 0), RF_ERR_UNSUPPORTED);
    EXPECT(LINEAR(DEV(5), DEV(3), DEV(4), 1, 256, 8, 64, 64, INT32_MAX, 0, RF_BF16, NULL, 0), RF_ERR_INVALID_ARG);
    EXPECT(LINEAR(DEV(3), DEV(3), DEV(4), 1, 256, 8, 64, 64, 3, RF_GATE_PER_FRAME | RF_ROWS_IN_FULL, RF_BF16, NULL, 0),
           RF_ERR_INVALID_ARG);
    EXPECT(LINEAR(DEV(4), NULL, DEV(4), 1, 256, 8, 64, 64, 3, 0, RF_BF16, DEV(4), 64), RF_ERR_INVALID_ARG);
    EXPECT(rf_frame_linear_workspace(256, 8388607, 4194296, 2147483640, RF_BF16, 256, bytes), RF_OK);
    EXPECT(rf_frame_linear_workspace(1, 1, 8, 8, RF_BF16, 1, bytes), RF_OK);
    EXPECT(rf_frame_linear_workspace(1, 100, 4194296, 8, RF_BF16, RF_MAX_COMPUTE_UNITS, bytes), RF_OK);
    EXPECT(rf_frame_linear_workspace(INT32_MAX, INT64_MAX, 64, 64, RF_F32, 256, bytes), RF_ERR_RANGE);

    free(ids);
    free(ax);
    free(l);
    free(bytes);
    printf("ok %d\n", checks);
    return 0;
}
