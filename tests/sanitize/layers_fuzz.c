/*
 * The host checks of the gated recurrence, the group norm and the loss over a
 * vocabulary under AddressSanitizer and UndefinedBehaviorSanitizer (test
 * infrastructure), as sequence_fuzz.c drives the other sequence operators: every
 * call with at least one defect that the host must reject (a workspace of none, if
 * no other), so that none reaches the device.
 *
 * Usage: layers_fuzz [iterations]. Prints one summary line; exit status 0 when
 * every check held.
 */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "mdlstm.h"

static uint64_t g_rng = 0x9e3779b97f4a7c15ull;
static uint64_t next_u64(void) { /* xorshift64* (Vigna) */
    g_rng ^= g_rng >> 12;
    g_rng ^= g_rng << 25;
    g_rng ^= g_rng >> 27;
    return g_rng * 0x2545f4914f6cdd1dull;
}
static int64_t uniform(int64_t lo, int64_t hi) { return lo + (int64_t)(next_u64() % ((uint64_t)(hi - lo) + 1)); }
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
        case 4: return (int64_t)1 << uniform(20, 62);
        default: return uniform(1, typical);
    }
}
static void* any_ptr(void) { /* never dereferenced */
    return chance(5) ? NULL : (void*)(uintptr_t)(((uint64_t)uniform(1, 40) << 36) + (chance(5) ? uniform(1, 15) : 0));
}

static long g_checks = 0, g_failures = 0, g_last = 0;
static void rejected(mdlstm_status st, const char* what) {
    ++g_checks;
    if (st == MDLSTM_ERR_WORKSPACE) ++g_last;
    if (st != MDLSTM_OK && st != MDLSTM_ERR_DEVICE) return;
    ++g_failures;
    fprintf(stderr, "%s: status %d (%s)\n", what, (int)st, mdlstm_last_error());
}
static void sized(size_t small, size_t large, const char* what) { /* of fewer and of more tokens or rows */
    ++g_checks;
    if (!small || !large || small <= large) return;
    ++g_failures;
    fprintf(stderr, "%s: %zu bytes, %zu for more\n", what, small, large);
}

static void fuzz_packed(void) {
    const int32_t n = chance(80) ? (int32_t)uniform(1, 1000) : any32(1 << 24), channels = chance(80) ? (int32_t)uniform(1, 4096) : any32(1 << 20);
    const int64_t tokens = chance(80) ? uniform(1, 1000000) : any64((int64_t)1 << 35), longest = chance(80) && tokens > 0 ? uniform(1, tokens) : any64(1000);
    const int64_t s0 = chance(80) ? channels + uniform(0, 64) : any64(1 << 22), s1 = chance(80) ? channels + uniform(0, 64) : any64(1 << 22);
    const mdlstm_recurrence_desc r = {channels, chance(90) ? (int32_t)uniform(0, 1) : any32(4), chance(90) ? (int32_t)uniform(0, 1) : any32(4)};
    for (int b = 0; b < 2; ++b) {
        const size_t need = mdlstm_recurrence_workspace_bytes(&r, n, tokens, longest, b);
        ++g_checks;
        if (need && need < 16) ++g_failures;
    }
    if (tokens > 0 && tokens < (int64_t)1 << 34) sized(mdlstm_recurrence_marks_bytes(&r, tokens), mdlstm_recurrence_marks_bytes(&r, 2 * tokens), "marks");
    rejected(mdlstm_recurrence_forward(&r, n, tokens, longest, any_ptr(), any_ptr(), any_ptr(), s0, any_ptr(), s1, any_ptr(), any_ptr(), any_ptr(),
                                       any_ptr(), chance(50) ? NULL : any_ptr(), 0, NULL), "recurrence_forward");
    rejected(mdlstm_recurrence_backward(&r, n, tokens, longest, any_ptr(), any_ptr(), any_ptr(), s0, any_ptr(), s1, any_ptr(), any_ptr(), any_ptr(), s0,
                                        any_ptr(), any_ptr(), any_ptr(), any_ptr(), any_ptr(), 0, NULL), "recurrence_backward");
    void* same = (void*)(uintptr_t)0x10000000;
    rejected(mdlstm_recurrence_step(&r, n > 0 ? n : 1, same, s0, any_ptr(), s1, any_ptr(), any64(100), any_ptr(), same, NULL), "recurrence_step");
    const mdlstm_group_norm_desc g = {channels, chance(60) ? 1 : any32(64), r.dtype, chance(90) ? (int32_t)uniform(0, 2) : any32(9), chance(90) ? 1e-5f : 0.0f};
    for (int b = 0; b < 2; ++b) {
        const size_t need = mdlstm_group_norm_workspace_bytes(&g, n, tokens, longest, b);
        ++g_checks;
        if (need && need < 16) ++g_failures;
    }
    rejected(mdlstm_group_norm_forward(&g, n, tokens, longest, any_ptr(), any_ptr(), any_ptr(), s0, any_ptr(), any_ptr(), any_ptr(), any_ptr(), any_ptr(),
                                       any_ptr(), 0, NULL), "group_norm_forward");
    rejected(mdlstm_group_norm_backward(&g, n, tokens, longest, any_ptr(), any_ptr(), any_ptr(), s0, any_ptr(), any_ptr(), any_ptr(), any_ptr(), any_ptr(),
                                        s1, any_ptr(), any_ptr(), any_ptr(), any_ptr(), 0, NULL), "group_norm_backward");
}

static void fuzz_vocabulary(void) {
    const mdlstm_vocabulary_desc v = {chance(80) ? (int32_t)uniform(1, 4096) : any32(1 << 16), chance(80) ? (int32_t)uniform(1, 200000) : any32(1 << 24),
                                      chance(90) ? (int32_t)uniform(0, 1) : any32(4)};
    const int64_t rows = chance(80) ? uniform(0, 100000) : any64((int64_t)1 << 22);
    const int64_t s0 = chance(80) ? v.dim + uniform(0, 64) : any64(1 << 20), s1 = chance(80) ? v.dim + uniform(0, 64) : any64(1 << 20);
    for (int b = 0; b < 2; ++b) {
        const size_t need = mdlstm_vocabulary_workspace_bytes(&v, rows, b);
        ++g_checks;
        if (need && need < 16) ++g_failures;
    }
    rejected(mdlstm_vocabulary_forward(&v, rows, any_ptr(), s0, any_ptr(), s1, any_ptr(), any_ptr(), any_ptr(), any_ptr(), 0, NULL), "vocabulary_forward");
    rejected(mdlstm_vocabulary_backward(&v, rows, any_ptr(), s0, any_ptr(), s1, any_ptr(), any_ptr(), any_ptr(), any_ptr(), any_ptr(), any_ptr(), 0, NULL),
             "vocabulary_backward");
}

int main(int argc, char** argv) {
    const long iterations = argc > 1 ? atol(argv[1]) : 10000;
    for (long i = 0; i < iterations; ++i) {
        fuzz_packed();
        fuzz_vocabulary();
    }
    printf("%ld checks, %ld rejected at the workspace, %ld failures\n", g_checks, g_last, g_failures);
    return g_failures || !g_last ? 1 : 0;
}
