// The encrypted KV cache as the files that work on it see it (kv.hip: products and appends, pages.hip: forking and taking).
#pragma once
#include "kernels.h"

struct cm_kv {
    cm_ctx *ctx = nullptr;
    int S, H, E, t, r_i, r_o, level, max_tokens, ntok, nk_max;
    int pos = 0;                            // where the next append goes (ntok unless cm_kv_seek has set it)
    double scale;
    bool scale_set = false;
    u64 *d_k = nullptr, *d_v = nullptr;     // nk_max / E ciphertexts [2][level+1][n]
    u64 *d_mask_qk = nullptr;               // base: slots (0, h, tau) all h, tau; level-1; multiplier form
    u64 *d_mask_k = nullptr;                // base: slots with residue 0;         level+1
    u64 *d_mask_v = nullptr;                // base: slots (0, h, 0) all h;        level+1
    u64 *d_mask_kg = nullptr;               // every slot;                         level+1  (token-group append)
    u64 *d_mask_vg = nullptr;               // base: slots (0, h, tau) all h, tau; level+1  (token-group append)
    u64 *d_work = nullptr;
    size_t work_words = 0;
    // query-times-K runs CM_KS_BATCH key ciphertexts at a time: tables for raising the third
    // component of their tensor products (level) and the second of their rotated sums (level-1)
    KsManyTables relin_tabs, rot_tabs;
    // sum over the head dims of query-times-K in the extended basis: the ladder cut into runs, every run the hoisted
    // rotations by its subset sums
    bool unrolled = false;
    std::vector<std::vector<long long>> dim_groups;
    // scores-times-V in the same form: giant steps unrolled (one key per multiple of the giant step), the ladder over
    // the residues in runs; tables for raising the second components of up to CM_KS_BATCH inner sums at once
    std::vector<std::vector<long long>> res_groups;
    KsManyTables giant_tabs;
    // query-times-K with the copy mask applied before the last `shared` terms of the sum over the dims: the sums of
    // the key ciphertexts (d_T), their masked combinations A_k (d_A) and the E slot rotations of the mask (d_M)
    // d_Mhat: the transform of d_M along the copy index (the masked sums as a cyclic correlation), with its twiddles
    // the key index: E ciphertexts like d_v, copy b of ciphertext g r_i + j = dim (b + j) of key group b - g r_i;
    // query-times-K from it is the scores-times-V schedule with the query in the place of the scores.  Ciphertext
    // g r_i + j is stored at place j r_o + g: the r_o ciphertexts an append makes from ONE rotation of the new key are
    // then neighbours (one launch reads that rotation once)
    bool indexed = false;
    u64 *d_x = nullptr;
    int shared = 1;
    u64 *d_T = nullptr, *d_A = nullptr, *d_M = nullptr, *d_Mhat = nullptr, *d_tw = nullptr, *d_einv = nullptr;
};

inline int ilog2(int x) {
    int l = 0;
    while ((1 << l) < x) l++;
    return l;
}
inline bool pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }
inline size_t kv_ctw(const cm_kv *kv) { return 2 * (size_t)(kv->level + 1) * kv->ctx->n; }
// where index ciphertext k is stored
inline int x_place(const cm_kv *kv, int k) { return (k % kv->r_i) * kv->r_o + k / kv->r_i; }
inline u64 rot_g(const cm_kv *kv, long long step) {
    long long S = kv->S;
    return galois_of_step(kv->ctx, (int)(((step % S) + S) % S));
}
