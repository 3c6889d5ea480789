/*
 * The host checks of the sequence operators under AddressSanitizer and
 * UndefinedBehaviorSanitizer (test infrastructure), as abi_fuzz.c drives the
 * other entry points: seeded random, extreme and defective arguments, every
 * call with at least one defect that the host must reject, so that none
 * reaches the device; workspace sizes are checked for consistency.
 *
 * Usage: sequence_fuzz [iterations]. Prints one summary line; exit status 0
 * when every check held.
 */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "mdlstm.h"

static uint64_t g_rng = 0x2545f4914f6cdd1dull;
static uint64_t next_u64(void) { /* xorshift64* (Vigna) */
    g_rng ^= g_rng >> 12;
    g_rng ^= g_rng << 25;
    g_rng ^= g_rng >> 27;
    return g_rng * 0x2545f4914f6cdd1dull;
}
static int64_t uniform(int64_t lo, int64_t hi) { /* inclusive, less than 2^63 - 1 apart */
    return lo + (int64_t)(next_u64() % ((uint64_t)(hi - lo) + 1));
}
static int chance(int percent) { return (int)(next_u64() % 100) < percent; }

static int32_t any32(int32_t typical) {
    switch (uniform(0, 9)) {
        case 0: return 0;
        case 1: return (int32_t)-uniform(1, 1000);
        case 2: return (int32_t)(INT32_MAX - uniform(0, 3));
        case 3: return (int32_t)(INT32_MIN + uniform(0, 3));
        default: return (int32_t)uniform(1, typical);
    }
}
static int64_t any64(int64_t typical) {
    switch (uniform(0, 11)) {
        case 0: return 0;
        case 1: return -uniform(1, 1000);
        case 2: return INT64_MAX - uniform(0, 3);
        case 3: return INT64_MIN + uniform(0, 3);
        case 4: return (int64_t)1 << uniform(30, 62);
        default: return uniform(1, typical);
    }
}
static void* any_ptr(void) { /* never dereferenced */
    return chance(10) ? NULL : (void*)(uintptr_t)(0x100000 + (chance(10) ? uniform(1, 15) : 0));
}

static long g_checks = 0, g_failures = 0, g_last = 0;
static void rejected(mdlstm_status st, const char* what) {
    ++g_checks;
    if (st == MDLSTM_ERR_WORKSPACE) ++g_last;
    if (st != MDLSTM_OK && st != MDLSTM_ERR_DEVICE) return;
    ++g_failures;
    fprintf(stderr, "%s: status %d (%s)\n", what, (int)st, mdlstm_last_error());
}

static mdlstm_attention_desc any_desc(void) {
    mdlstm_attention_desc d;
    d.kv_heads = chance(80) ? (int32_t)uniform(1, 8) : any32(64);
    d.heads = chance(80) && d.kv_heads > 0 && d.kv_heads < 1000 ? d.kv_heads * (int32_t)uniform(1, 4) : any32(64);
    d.dim_k = chance(80) ? (int32_t)uniform(1, 128) : any32(300);
    d.dim_v = chance(80) ? (int32_t)uniform(1, 128) : any32(300);
    d.dtype = chance(90) ? (int32_t)uniform(0, 1) : any32(5);
    d.scale = 0.5f;
    return d;
}
static mdlstm_heads any_view(void) {
    mdlstm_heads v;
    v.d_data = any_ptr();
    v.token_stride = chance(80) ? uniform(0, 4096) : any64(100000);
    v.head_stride = chance(80) ? uniform(0, 128) : any64(1000);
    return v;
}

static void fuzz_attention(void) {
    mdlstm_attention_desc d = any_desc();
    const int32_t n = chance(80) ? (int32_t)uniform(1, 1000) : any32(1000);
    const int64_t tokens = chance(80) ? uniform(0, 1 << 20) : any64(1 << 20);
    const int64_t longest = chance(80) && tokens > 0 ? uniform(0, tokens) : any64(1 << 16);
    mdlstm_heads v[4];
    for (int i = 0; i < 4; ++i) v[i] = any_view();
    const size_t f = mdlstm_attention_workspace_bytes(&d, n, tokens, longest, 0);
    const size_t b = mdlstm_attention_workspace_bytes(&d, n, tokens, longest, 1);
    ++g_checks;
    if ((f == 0) != (b == 0) || (f > 0 && f < 16)) {
        ++g_failures;
        fprintf(stderr, "workspace sizes %zu and %zu\n", f, b);
    }
    rejected(mdlstm_attention_forward(chance(2) ? NULL : &d, n, tokens, longest, any_ptr(), any_ptr(), any_ptr(), &v[0], &v[1],
                                      chance(2) ? NULL : &v[2], any_ptr(), any_ptr(), any_ptr(), any_ptr(),
                                      f > 0 ? f - 1 : 0, NULL), "attention_forward");
    rejected(mdlstm_attention_backward(&d, n, tokens, longest, any_ptr(), any_ptr(), any_ptr(), &v[0], &v[1], &v[2], any_ptr(), &v[3],
                                       any_ptr(), any_ptr(), any_ptr(), any_ptr(), any_ptr(), any_ptr(), b > 0 ? b - 1 : 0,
                                       NULL), "attention_backward");
    v[uniform(0, 2)].token_stride = -1; /* a defect for certain */
    rejected(mdlstm_attention_step(&d, chance(90) ? (int32_t)uniform(1, 100) : any32(100), any_ptr(), &v[0], &v[1], &v[2],
                                   any_ptr(), any64(1000), any_ptr(), any_ptr(), NULL), "attention_step");
}

static void fuzz_norm(void) {
    mdlstm_norm_desc d;
    d.cols = chance(80) ? (int32_t)uniform(1, 32768) : any32(40000);
    d.dtype = chance(90) ? (int32_t)uniform(0, 1) : any32(5);
    d.eps = chance(90) ? 1e-6f : chance(50) ? -1.0f : NAN;
    d.p = chance(80) ? 0.25 : chance(50) ? 1.5 : NAN;
    const int64_t rows = chance(80) ? uniform(1, 1 << 20) : any64(1 << 20), stride = chance(80) ? d.cols : any64(1 << 16);
    const size_t b = mdlstm_norm_workspace_bytes(&d, rows);
    void *y = any_ptr(), *y8 = y ? (void*)(uintptr_t)0x200000 : NULL; /* both or none: rejected */
    rejected(mdlstm_norm_forward(&d, rows > 0 ? rows : -1, any_ptr(), stride, any_ptr(), stride, any_ptr(), 1, 2, any_ptr(), y, y8,
                                 any_ptr(), any_ptr(), NULL), "norm_forward");
    rejected(mdlstm_norm_backward(&d, rows, any_ptr(), stride, any_ptr(), any_ptr(), any_ptr(), any_ptr(), 1, 2, any_ptr(),
                                  any_ptr(), any_ptr(), any_ptr(), b > 0 ? b - 1 : 0, NULL), "norm_backward");
    const int64_t cols = d.cols > 0 ? d.cols : 1;
    rejected(mdlstm_dropout(d.dtype, any64(1 << 20), any64(1 << 20), NULL, any64(1 << 20), d.p, 1, 2, any_ptr(), any64(1 << 20),
                            any_ptr(), NULL) == MDLSTM_OK /* nothing to do is no defect */ ? MDLSTM_ERR_INVALID_ARG :
             mdlstm_dropout(d.dtype, 7, cols, any_ptr(), cols - 1, d.p, 1, 2, any_ptr(), any64(1 << 20), any_ptr(), NULL),
             "dropout");
}

int main(int argc, char** argv) {
    const long iterations = argc > 1 ? atol(argv[1]) : 20000;
    for (long i = 0; i < iterations; ++i) {
        fuzz_attention();
        fuzz_norm();
    }
    printf("%ld checks, %ld failures, %ld reached the workspace size\n", g_checks, g_failures, g_last);
    return g_failures || g_last < iterations / 20 ? 1 : 0;
}
