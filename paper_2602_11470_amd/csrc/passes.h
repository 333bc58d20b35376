// Several passes of scores-times-V (or of query-times-K on the key index) taken together (passes.hip).
#pragma once
#include "kv.h"

struct KvPasses {
    int P = 0, r_i = 0, r_o = 0, level = 0;        // passes of a turn
    int D = 0, B = 0, G = 0;                       // digit arrays; relinearisations and giant steps of a batch
    u64 *babies = nullptr;                         // [P][r_i] ciphertexts; the others are parts of the same allocation
    u64 *sums = nullptr, *inner = nullptr;         // [P][r_o] tensor sums of three components, [r_o][P] ciphertexts
    u64 *ksin = nullptr, *digits = nullptr;        // D polynomials and their digits
    u64 *acc = nullptr, *nxt = nullptr;            // [P] sums on the extended basis
    KsManyTables baby_tabs, relin_tabs, giant_tabs;
};
// room for turns of up to `passes` passes over caches of kv's shape and level; P = 0 where passes are taken one at a time instead (r_o > 8, more than six digits, no memory)
void kv_passes_create(cm_ctx *ctx, const cm_kv *kv, int passes, KvPasses *kp);
void kv_passes_destroy(KvPasses *kp);
inline bool kv_passes_fit(const KvPasses &kp, const cm_kv *kv) { return kp.P && kp.r_i == kv->r_i && kp.r_o == kv->r_o && kp.level == kv->level; }
// outs[p][2][level][n] = the un-replicated, un-reduced product (cm_vmm_kv) of the ciphertexts at babies[p][0] with array, p < m <= P.
// keys have been checked (kv_sv_keys)
cm_status kv_passes_run(cm_ctx *ctx, const cm_evk *evk, const cm_kv *kv, const KvPasses &kp, const u64 *array, int m, u64 *const *outs, hipStream_t st);
// dst[z] = src[z] (words each, a multiple of 512), z < m <= CM_KS_BATCH
void launch_copies(u64 *const *dst, const u64 *const *src, int m, size_t words, hipStream_t st);
