// Rotary positions as the files that use them see them (rotary.hip; appends in kv.hip), and weighted rotations (tree.hip).
#pragma once
#include "kernels.h"

// plaintexts of all residues; with a split those of the residues from it on and of the residues below it
#define ROT_SETS 3
struct cm_rotary {
    cm_ctx *ctx = nullptr;
    int H, E, t, level, room;
    int low, high;                    // position = low * (high part) + low part
    int step, parts;                  // left rotation to the second dim of a pair; plaintexts of a set: 3, or 2 where both rotations are one
    int ma, mb;                       // indices of the two moduli
    u64 inv;                          // of the second under the first, multiplier form
    int batch;                        // ciphertexts raised together
    u64 *d_low = nullptr;             // [low][cos first, cos second, sin first, sin second][2][n]
    u64 *d_still = nullptr;           // [2][n], null where the whole head turns
    u64 *d_high = nullptr;            // [high][cos, sin][2][n], multiplier form
    u64 *d_v = nullptr, *d_p = nullptr;      // [set][part][2][n], [set][part][ext][n] (multiplier form)
    u64 *d_work = nullptr;            // two ciphertexts, then the second components, coefficients and digits of a batch
    int *d_mods = nullptr, *d_ext_mods = nullptr;
    KsManyTables tabs;
    std::vector<int32_t> pos;         // set last
    int split = 0;
    bool set = false;
};
// of up to r->batch ciphertexts, each with the plaintexts of `sets` sets from the first on: sums on the extended basis, us[z][set]; *rows_done: what
// weighted_down takes
cm_status rotary_sums(cm_ctx *ctx, const cm_evk *evk, const cm_rotary *r, int m, const u64 *const *xs, int first, int sets, u64 *us, bool *rows_done,
                      hipStream_t st);
// outs[z][2][level][n] = rescale(ModDown(us[z][2][ext][n])) for z < m <= CM_KS_BATCH; tmp: a ciphertext of the level (onto: two), used where it takes
// two steps; rows_done: the row pass of the inverse transforms has been done (launch_rows_weighted); onto: outs += instead
cm_status weighted_down(cm_ctx *ctx, u64 *us, int level, int m, u64 *const *outs, u64 *tmp, hipStream_t st, bool rows_done = false, bool onto = false);
// whether launch_rows_weighted applies, and is the faster form, for outputs of nsum items, m ModDowns following
bool weighted_rows(cm_ctx *ctx, int beta, int level, int nsum, int m);
// whether na words at a and nb at b share one
inline bool words_meet(const u64 *a, size_t na, const u64 *b, size_t nb) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + nb * 8 && y < x + na * 8;
}
