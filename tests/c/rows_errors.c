/*
 * The host side of group norm, rows in 8 bits and their products under AddressSanitizer and UndefinedBehaviorSanitizer:
 * id lists of exactly their size, sizes and strides at the ends of their types. No call reaches a launch: device
 * pointers are fabricated addresses that the checks reject, and nothing is dereferenced. Prints "ok <checks>".
 */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

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
    int64_t *bytes = (int64_t *)malloc(sizeof *bytes);

#define QUANTIZE(q, s, M, T, N, K, st, fl, dt) rf_frame_quantize(DEV(0), q, s, ids, M, T, N, K, st, fl, dt, NULL)
    EXPECT(QUANTIZE(DEV(1), DEV(2), 256, 256, INT64_MAX, 64, 0, 0, RF_BF16), RF_ERR_RANGE);
    EXPECT(QUANTIZE(DEV(1), DEV(2), 1, 1, INT64_MIN, 64, 0, 0, RF_BF16), RF_ERR_INVALID_ARG);
    EXPECT(QUANTIZE(DEV(1), DEV(2), 1, 1, 5, INT32_MAX, 0, 0, RF_BF16), RF_ERR_UNSUPPORTED);
    EXPECT(QUANTIZE(DEV(1), DEV(2), 1, 1, 5, INT32_MIN, 0, 0, RF_F32), RF_ERR_INVALID_ARG);
    EXPECT(QUANTIZE(DEV(1), DEV(2), 1, 1, 5, 64, INT64_MAX, 0, RF_F32), RF_ERR_RANGE);
    EXPECT(QUANTIZE(DEV(1), DEV(2), 1, 1, 5, 64, INT64_MIN, 0, RF_F32), RF_ERR_INVALID_ARG);
    EXPECT(QUANTIZE(DEV(0), DEV(2), 256, 256, 8388607, 65536, 0, RF_ROWS_IN_FULL, RF_F32), RF_ERR_INVALID_ARG);
    EXPECT(QUANTIZE(DEV(1), DEV(2), INT32_MAX, INT32_MAX, 5, 64, 0, 0, RF_F32), RF_ERR_RANGE);

#define LINEAR(y, M, T, N, K, n, fl, dt, ws, wb) \
    rf_frame_linear_i8(DEV(0), DEV(1), DEV(2), DEV(3), DEV(4), DEV(5), DEV(6), y, ids, M, T, N, K, n, 0, fl, dt, ws, wb, NULL)
    EXPECT(LINEAR(DEV(0), 256, 256, 8388607, 65536, 2147483640, 0, RF_F32, NULL, 0), RF_ERR_RANGE);
    EXPECT(LINEAR(DEV(0), 256, 256, 8388607, 64, 64, 0, RF_BF16, NULL, 0), RF_ERR_INVALID_ARG);
    EXPECT(LINEAR(DEV(7), 256, 256, INT64_MAX, 64, 64, 0, RF_BF16, NULL, 0), RF_ERR_RANGE);
    EXPECT(LINEAR(DEV(7), 1, 1, INT64_MIN, 64, 64, 0, RF_BF16, NULL, 0), RF_ERR_INVALID_ARG);
    EXPECT(LINEAR(DEV(7), 1, 1, 1, INT32_MAX - 15, 64, 0, RF_BF16, NULL, 0), RF_ERR_UNSUPPORTED);
    EXPECT(LINEAR(DEV(3), 1, 256, 8, 64, 64, RF_GATE_PER_FRAME | RF_ROWS_IN_FULL, RF_BF16, NULL, 0), RF_ERR_INVALID_ARG);
    EXPECT(LINEAR(DEV(6), 1, 256, 8, 64, 64, 0, RF_BF16, DEV(1), 64), RF_ERR_INVALID_ARG);
    EXPECT(LINEAR(DEV(7), 1, 1, 8, 64, 64, 0, RF_BF16, DEV(8), INT64_MIN), RF_ERR_INVALID_ARG);
    EXPECT(rf_frame_linear_i8_workspace(256, 8388607, 65536, 2147483640, RF_BF16, 256, bytes), RF_OK);
    EXPECT(rf_frame_linear_i8_workspace(1, 1, 16, 8, RF_BF16, 1, bytes), RF_OK);
    EXPECT(rf_frame_linear_i8_workspace(1, 100, 65536, 8, RF_F32, RF_MAX_COMPUTE_UNITS, bytes), RF_OK);
    EXPECT(rf_frame_linear_i8_workspace(INT32_MAX, INT64_MAX, 64, 64, RF_F32, 256, bytes), RF_ERR_RANGE);

#define NORM(y, ys, M, T, N, C, G, to, eps, xs, yst, fl, dt, ws, wb) \
    rf_frame_group_norm(DEV(0), DEV(1), DEV(2), y, ys, ids, M, T, N, C, G, to, eps, 0, xs, yst, fl, dt, ws, wb, NULL)
    EXPECT(NORM(DEV(3), NULL, 256, 256, INT64_MAX, 64, 8, 1, 1e-5, 0, 0, 0, RF_BF16, DEV(8), 64), RF_ERR_RANGE);
    EXPECT(NORM(DEV(3), NULL, 1, 1, INT64_MIN, 64, 8, 1, 1e-5, 0, 0, 0, RF_BF16, DEV(8), 64), RF_ERR_INVALID_ARG);
    EXPECT(NORM(DEV(3), NULL, 1, 1, 4, INT32_MAX, 1, 1, 1e-5, 0, 0, 0, RF_BF16, DEV(8), 64), RF_ERR_UNSUPPORTED);
    EXPECT(NORM(DEV(3), NULL, 1, 1, 4, 64, INT32_MAX, 1, 1e-5, 0, 0, 0, RF_BF16, DEV(8), 64), RF_ERR_INVALID_ARG);
    EXPECT(NORM(DEV(3), NULL, 1, 1, 4, 64, INT32_MIN, 1, 1e-5, 0, 0, 0, RF_BF16, DEV(8), 64), RF_ERR_INVALID_ARG);
    EXPECT(NORM(DEV(3), NULL, 4, 4, 4, 64, 8, INT32_MAX, 1e-5, 0, 0, 0, RF_BF16, DEV(8), 64), RF_ERR_INVALID_ARG);
    EXPECT(NORM(DEV(3), NULL, 4, 4, 4, 64, 8, 1, NAN, 0, 0, 0, RF_BF16, DEV(8), 64), RF_ERR_INVALID_ARG);
    EXPECT(NORM(DEV(3), NULL, 4, 4, 4, 64, 8, 1, 1e-5, INT64_MAX, INT64_MAX, 0, RF_BF16, DEV(8), 64), RF_ERR_RANGE);
    EXPECT(NORM(DEV(3), NULL, 4, 4, 4, 64, 8, 1, 1e-5, INT64_MIN, 0, 0, RF_BF16, DEV(8), 64), RF_ERR_INVALID_ARG);
    EXPECT(NORM(DEV(3), DEV(4), 4, 4, 4, 64, 8, 1, 1e-5, 0, INT64_MAX, 0, RF_BF16, DEV(8), 64), RF_ERR_INVALID_ARG);
    EXPECT(NORM(DEV(0), DEV(4), 256, 256, 8388607, 8192, 8, 256, 1e-5, 0, 0, 0, RF_F32, DEV(8), 64), RF_ERR_INVALID_ARG);
    EXPECT(NORM(DEV(3), NULL, 4, 4, 4, 64, 8, 1, 1e-5, 0, 0, 0, RF_BF16, DEV(8), INT64_MIN), RF_ERR_INVALID_ARG);
    EXPECT(rf_frame_group_norm_workspace(256, 8388607, 8192, 8192, 256, 1, RF_F32, RF_MAX_COMPUTE_UNITS, bytes), RF_OK);
    EXPECT(rf_frame_group_norm_workspace(1, 2147483647, 8, 1, 1, 0, RF_BF16, RF_MAX_COMPUTE_UNITS, bytes), RF_OK);
    EXPECT(rf_frame_group_norm_workspace(1, 1, 4, 4, 1, 0, RF_F32, 1, bytes), RF_OK);
    EXPECT(rf_frame_group_norm_workspace(INT32_MAX, INT64_MAX, 64, 8, 1, 0, RF_F32, 256, bytes), RF_ERR_RANGE);

    free(ids);
    free(bytes);
    printf("ok %d\n", checks);
    return 0;
}
