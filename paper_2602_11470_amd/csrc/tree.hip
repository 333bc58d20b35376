// Attention of a tree of drafted tokens over an encrypted cache.
//
// The drafted tokens stand behind the committed ones in the cache, the token of place a at residue a mod t_kv; their queries stand in one
// ciphertext, t = t_kv / group of them at the residues of their places.  The product with a page pairs equal residues, so it runs t_kv
// times, pass delta with the residues of every block moved by delta: from_delta Rot(q, -delta) + below_delta Rot(q, t_kv - delta), the
// residues from delta on and those below it.  All those rotations are of ONE ciphertext: one raise, one launch of weighted sums for eight
// passes, and ModDown and rescale in one.  The results of scores times V move back by t_kv - delta; as sums they stay on the
// extended basis until all passes are in, so that one ModDown and rescale ends them.
//
// What a query may not see takes the mask's value: the drafted places that it does not follow, those behind the last one in its page, places whose
// token has been dropped, and whole pages.  Every place is one slot row of the mask turned to its page and residue (an exact permutation), so a tree is data of the call.
#include <math.h>

#include <algorithm>

#include "passes.h"
#include "rotary.h"

#define TREE_ROWS 4
#define TREE_T 64                  // residues of a page, at most: a place is a bit of a word
struct cm_tree {
    cm_ctx *ctx = nullptr;
    int H, E, t_kv, G, level;
    double scale;
    u64 *d_q = nullptr, *d_v = nullptr;       // [from, below][t_kv - 1][ext][n]: for the queries (level + 1) and the results (level - 1)
    u64 *d_one = nullptr;                     // [level][n]: the mask's value at row 0, residue 0
    u64 *d_unseen = nullptr;                  // [E - 1][level][n]: entry m - 1: in the rows m .. E - 1
    u64 *d_work = nullptr;
    std::vector<u64> empty;                   // of every page, the places that hold no token (bits)
    KsManyTables tabs, q_tabs;                // raise of the second components of CM_KS_BATCH results, of the query's
    KvPasses passes;                          // for caches with the creating one's baby steps; others' passes run one at a time
};

struct TreeMask {
    u64 *score[CM_KS_BATCH];                   // first components
    u64 bits[TREE_ROWS][CM_KS_BATCH];          // hidden residues of a row for a pass
    unsigned row[TREE_ROWS], residue[TREE_T];  // Galois elements that take row 0 there, residue 0 there
};
// score[z] += the mask's value at every hidden place of up to TREE_ROWS rows, and unseen (nullable) through the map gu.  The masks are never formed:
// one polynomial that the caches hold is gathered once a hidden place.  Eight passes of four limbs, two pages with up to
// sixteen hidden places, 21 us, a third of it the scores' own words; n = 4096 5.3 us, a launch.  No query of the tree is left without a place: it sees itself.
__global__ __launch_bounds__(256) void k_tree_mask(TreeMask m, int rows, const u64 *__restrict__ one, const u64 *__restrict__ unseen, unsigned gu,
                                                   const ModC *__restrict__ modc, int n, int logn) {
    const unsigned i = blockIdx.x * 256 + threadIdx.x;
    const size_t at = (size_t)blockIdx.y * n;
    const u64 q = modc[blockIdx.y].q;
    u64 *p = m.score[blockIdx.z] + at + i;
    u64 v = *p;
    for (int r = 0; r < rows; r++)
        for (u64 left = m.bits[r][blockIdx.z]; left; left &= left - 1)
            v = addmod(v, one[at + perm_src(i, (m.row[r] * m.residue[__ffsll((unsigned long long)left) - 1]) & ((2u << logn) - 1u), logn)], q);
    if (unseen) v = addmod(v, unseen[at + perm_src(i, gu, logn)], q);
    *p = v;
}

// out[c][limbs][n] = a[c][limbs][n] + the first limbs of b[c][limbs + 1][n]
__global__ __launch_bounds__(256) void k_add_dropped(u64 *__restrict__ out, const u64 *__restrict__ a, const u64 *__restrict__ b, const ModC *__restrict__ modc,
                                                     int limbs, int n) {
    const size_t i = blockIdx.x * 256 + threadIdx.x;
    const int l = blockIdx.y, c = blockIdx.z;
    const size_t at = ((size_t)c * limbs + l) * n + i;
    out[at] = addmod(a[at], b[at + (size_t)c * n], modc[l].q);
}

extern "C" void cm_tree_destroy(cm_tree *tr) {
    if (!tr) return;
    ks_many_tables_destroy(&tr->tabs), ks_many_tables_destroy(&tr->q_tabs);
    kv_passes_destroy(&tr->passes);
    hipFree(tr->d_q), hipFree(tr->d_v), hipFree(tr->d_one), hipFree(tr->d_unseen), hipFree(tr->d_work);
    delete tr;
}
// work area of the passes: digits of the query, then CM_KS_BATCH ciphertexts (level + 1); or, of the results, CM_KS_BATCH of them with their
// coefficients and digits, two sums on the extended basis and three ciphertexts
static size_t tree_work_words(cm_ctx *ctx, int level) {
    const size_t n = ctx->n, B = CM_KS_BATCH;
    const KsLevel &up = ks_level(ctx, level + 1), &dn = ks_level(ctx, level - 1);
    const size_t qk = (size_t)up.beta * up.ext * n + (B + 1) * 2 * (size_t)(level + 2) * n;
    const size_t sv = B * 3 * (size_t)level * n + B * (size_t)dn.beta * dn.ext * n + 2 * 2 * (size_t)dn.ext * n + 3 * 2 * (size_t)level * n;
    return std::max(qk, sv);
}
extern "C" cm_status cm_tree_create(cm_ctx *ctx, const cm_kv *kv, int32_t group, double mask, double scale, const int64_t *coeffs, cm_tree **out) {
    (void)hipGetLastError();          // stale errors of earlier calls are not this call's
    if (!ctx || !kv || kv->ctx != ctx || !out || group < 1 || !isfinite(mask) || !isfinite(scale) || scale < 0) return CM_E_INVAL;
    if (!pow2(group) || kv->t % group || kv->t > TREE_T) return CM_E_LAYOUT;
    if (kv->level + 1 > ctx->L || kv->level < 2) return CM_E_LEVEL;
    if (scale == 0) scale = ctx->prm.scale * kv->scale / (double)ctx->mod[kv->level];
    if (fabs(mask) * scale >= 0x1p61) return CM_E_INVAL;
    cm_tree *tr = new (std::nothrow) cm_tree();
    if (!tr) return CM_E_NOMEM;
    cm_status status = CM_OK;
    u64 *row = nullptr, *d_coeffs = nullptr;
    int *d_mods = nullptr;
    try {
        const int t = kv->t, H = kv->H, E = kv->E, level = kv->level, S = kv->S, n = ctx->n;
        tr->ctx = ctx, tr->H = H, tr->E = E, tr->t_kv = t, tr->G = group, tr->level = level, tr->scale = scale;
        tr->empty.assign(E, 0);
        const size_t lw = (size_t)level * n;
        auto get = [&](u64 **p, size_t words) {
            if (status == CM_OK && words && hipMalloc((void **)p, words * 8) != hipSuccess) status = CM_E_NOMEM;
        };
        const int up = level + 2 + ctx->K, dn = level + ctx->K;
        get(&tr->d_q, 2 * (size_t)(t - 1) * up * n), get(&tr->d_v, 2 * (size_t)(t - 1) * dn * n);
        get(&tr->d_one, lw), get(&tr->d_unseen, (E - 1) * lw), get(&row, lw), get(&d_coeffs, n);
        get(&tr->d_work, tree_work_words(ctx, level));
        if (status == CM_OK && hipMalloc((void **)&d_mods, CM_MAX_LIMBS * 4) != hipSuccess) status = CM_E_NOMEM;
        if (status == CM_OK) status = ks_many_tables_create(ctx, level - 1, CM_KS_BATCH, &tr->tabs, 2, 1);
        if (status == CM_OK) status = ks_many_tables_create(ctx, level + 1, 1, &tr->q_tabs, 2, 1);
        // a plaintext on `limbs` limbs, the special ones of a level among them (mont), or the first ones alone
        auto put = [&](u64 *dst, const int64_t *c, int limbs, int lv, bool mont) {
            if (status != CM_OK) return;
            std::vector<int> mods;
            for (int l = 0; l < limbs; l++) mods.push_back(l <= lv ? l : ctx->L + l - lv);
            if (hipMemcpy(d_coeffs, c, (size_t)n * 8, hipMemcpyHostToDevice) != hipSuccess ||
                hipMemcpy(d_mods, mods.data(), mods.size() * 4, hipMemcpyHostToDevice) != hipSuccess) {
                status = CM_E_HIP;
                return;
            }
            launch_reduce_i64(ctx, dst, (const long long *)d_coeffs, d_mods, limbs, 0);
            launch_ntt(ctx, dst, d_mods, limbs, false, 0);
            if (mont) launch_to_mont(ctx, dst, d_mods, limbs, 0);
            if (hipDeviceSynchronize() != hipSuccess || hipGetLastError() != hipSuccess) status = CM_E_HIP;
        };
        if (status == CM_OK && hipDeviceSynchronize() != hipSuccess) status = CM_E_HIP;
        std::vector<double> m(S);
        std::vector<int64_t> c(n), own(n);
        auto coefficients = [&](size_t i, double sc) -> const int64_t * {
            if (coeffs) return coeffs + i * n;
            if (status == CM_OK) status = cm_encode_coeffs(ctx, m.data(), nullptr, S, sc, own.data());
            return own.data();
        };
        for (int dir = 0; dir < 2; dir++) {
            const int lv = dir == 0 ? level + 1 : level - 1, ext = lv + 1 + ctx->K;
            const u64 q = ctx->mod[lv];
            for (int d = 1; d < t && status == CM_OK; d++) {
                for (int i = 0; i < S; i++) m[i] = i % t >= d;
                const int64_t *from = coefficients((size_t)dir * (t - 1) + d - 1, (double)q);
                u64 *dst = (dir == 0 ? tr->d_q : tr->d_v) + (size_t)(d - 1) * ext * n;
                put(dst, from, ext, lv, true);
                for (int i = 0; i < n; i++) c[i] = (i == 0 ? (int64_t)q : 0) - from[i];      // the scale everywhere, less the mask
                put(dst + (size_t)(t - 1) * ext * n, c.data(), ext, lv, true);
            }
        }
        const size_t at = 2 * (size_t)(t - 1);
        for (int i = 0; i < S; i++) m[i] = i < H * t && i % t == 0 ? mask : 0.0;
        put(tr->d_one, coefficients(at, scale), level, level - 1, false);
        for (int i = 0; i < S; i++) m[i] = i < H * t ? mask : 0.0;
        put(row, coefficients(at + 1, scale), level, level - 1, false);
        if (status == CM_OK && E > 1) {
            rows_from_on(ctx, tr->d_unseen, row, H * t, E, level);
            if (hipDeviceSynchronize() != hipSuccess || hipGetLastError() != hipSuccess) status = CM_E_HIP;
        }
        // last, so that what the object cannot do without has its memory
        if (status == CM_OK) kv_passes_create(ctx, kv, t, &tr->passes);
    } catch (...) {
        status = CM_E_NOMEM;
    }
    hipFree(row), hipFree(d_coeffs), hipFree(d_mods);
    if (status != CM_OK) {
        cm_tree_destroy(tr);
        return status;
    }
    *out = tr;
    return CM_OK;
}
extern "C" cm_status cm_tree_set_empty(cm_tree *tr, const int32_t *places, int32_t count) {
    if (!tr || count < 0 || (count && !places)) return CM_E_INVAL;
    for (int i = 0; i < count; i++) if (places[i] < 0 || places[i] >= tr->E * tr->t_kv) return CM_E_LAYOUT;
    std::fill(tr->empty.begin(), tr->empty.end(), 0);
    for (int i = 0; i < count; i++) tr->empty[places[i] / tr->t_kv] |= 1ULL << (places[i] % tr->t_kv);
    return CM_OK;
}
extern "C" int32_t cm_tree_passes(const cm_tree *tr) { return tr ? tr->t_kv : 0; }
extern "C" int32_t cm_tree_steps(const cm_tree *tr, int32_t *steps, int32_t cap) {
    if (!tr) return 0;
    int32_t count = 0;
    for (int d = 1; d < tr->t_kv; d++)
        for (const int s : {-d, tr->t_kv - d}) {
            if (count < cap && steps) steps[count] = s;
            count++;
        }
    return count;
}
static cm_status tree_keys(const cm_evk *evk, const cm_tree *tr) {
    for (int s = 1; s < tr->t_kv; s++)
        for (const int step : {-s, s}) if (!find_key(evk, galois_of_step(tr->ctx, step))) return CM_E_NOKEY;
    return CM_OK;
}
static bool tree_fits(const cm_tree *tr, const cm_kv *kv) { return kv->t == tr->t_kv && kv->E == tr->E && kv->H == tr->H; }
// the residues of a block moved by delta: items 2 k and 2 k + 1 of an output
static void tree_moves(const cm_evk *evk, const cm_tree *tr, WrItem *it, const u64 *masks, size_t ptw, int delta, const u64 *dig, const u64 *c) {
    for (int s = 0; s < 2; s++) {
        it[s].g = (unsigned)galois_of_step(tr->ctx, s ? tr->t_kv - delta : -delta), it[s].key = find_key(evk, it[s].g);
        it[s].dig = dig, it[s].c = c, it[s].pt = masks + ((size_t)s * (tr->t_kv - 1) + delta - 1) * ptw;
    }
}
extern "C" cm_status cm_tree_qk(cm_ctx *ctx, const cm_evk *evk, const cm_tree *tr, const cm_kv *kv, const int32_t *parent, int32_t nodes, int32_t base,
                                int32_t node0, int32_t first, const cm_ct *q, cm_ct *scores, void *stream) {
    (void)hipGetLastError();          // stale errors of earlier calls are not this call's
    if (!ctx || !evk || !tr || !kv || tr->ctx != ctx || kv->ctx != ctx || !parent || !q || !q->dev || q->ncomp != 2 || !scores || !evk_fits(ctx, evk)) return CM_E_INVAL;
    if (!tree_fits(tr, kv) || nodes < 1 || base < 0 || nodes > kv->ntok || base > kv->ntok - nodes || node0 < 0 || node0 >= nodes) return CM_E_LAYOUT;
    if (first < 0 || first > base || first % kv->t) return CM_E_LAYOUT;
    for (int i = 0; i < nodes; i++) if (parent[i] < -1 || parent[i] >= i) return CM_E_INVAL;
    if (kv->level != tr->level || q->level != kv->level + 1) return CM_E_LEVEL;
    const int lv = kv->level, t = tr->t_kv, ls = kv->indexed ? lv - 1 : lv - 2;
    const size_t n = ctx->n, sw = 2 * (size_t)(ls + 1) * n, qw = 2 * (size_t)(lv + 2) * n;
    if (!(fabs(q->scale * kv->scale / (double)ctx->mod[lv] / tr->scale - 1) < 1e-9)) return CM_E_SCALE;
    for (int d = 0; d < t; d++) {
        if (!scores[d].dev || words_meet(scores[d].dev, sw, q->dev, qw)) return CM_E_INVAL;
        for (int e = 0; e < d; e++) if (words_meet(scores[d].dev, sw, scores[e].dev, sw)) return CM_E_INVAL;
    }
    CM_TRY
    CMCHK(tree_keys(evk, tr));
    CMCHK(kv->indexed ? kv_sv_keys(evk, kv, false, false) : kv_qk_keys(evk, kv, false));
    // which places of the tree's pages the query at every residue may see: itself and what it follows
    const int per = t / tr->G, page = base / t, start = base % t, rows = (start + nodes + t - 1) / t;
    std::vector<std::vector<u64>> seen(per, std::vector<u64>(rows, 0));
    for (int u = 0; u < per; u++) {
        const int node = node0 + ((u - base - node0) % per + per) % per;
        if (node < nodes)
            for (int k = node; k >= 0; k = parent[k]) seen[u][(start + k) / t] |= 1ULL << ((start + k) % t);
    }
    // pages with places to hide: the tree's, and those before it that are seen and have places without a token
    std::vector<int> masked;
    for (int r = 0; r < rows; r++) masked.push_back(page + r);
    for (int c = first / t; c < page; c++) if (tr->empty[c]) masked.push_back(c);
    hipStream_t st = (hipStream_t)stream;
    const KsLevel &up = ks_level(ctx, lv + 1);
    const size_t ctw = kv_ctw(kv);
    u64 *digits = tr->d_work, *x = digits + (size_t)up.beta * up.ext * n, *tmp = x + CM_KS_BATCH * ctw, *us = arena_batch_sums(ctx);
    if (t > 1 && n == 65536) CMCHK(ks_raise_apart(ctx, tr->q_tabs, &q->dev, x, digits, st, 1));
    else if (t > 1) CMCHK(ks_raise(ctx, q->dev + (size_t)(lv + 2) * n, lv + 1, digits, st));
    const u64 *unseen = nullptr;
    unsigned gu = 0;
    {
        const int from = first / t, many = page + rows - from;                // pages that are seen
        if (many < tr->E) unseen = tr->d_unseen + (size_t)(many - 1) * lv * n, gu = (unsigned)rot_g(kv, -(long long)from * kv->H * t);
    }
    const bool joint = kv->indexed && kv_passes_fit(tr->passes, kv);
    const int turn = joint ? tr->passes.P : CM_KS_BATCH;
    const size_t xw = joint ? tr->passes.r_i * ctw : ctw;                     // from one pass's ciphertext to the next one's
    if (joint) x = tr->passes.babies;
    for (int d0 = 0; d0 < t; d0 += turn) {
        const int m = std::min(turn, t - d0), skip = d0 == 0;
        if (skip) {                                                          // pass 0 does not move: a level drop
            u64 *dst[2] = {x, x + ctw / 2};
            const u64 *src[2] = {q->dev, q->dev + (size_t)(lv + 2) * n};
            launch_copies(dst, src, 2, ctw / 2, st);
        }
        if (m > skip) {
            WrBatch b;
            b.nz = m - skip, b.nsum = 2;
            u64 *outs[CM_KS_BATCH];
            for (int z = 0; z < b.nz; z++) {
                tree_moves(evk, tr, b.it + 2 * z, tr->d_q, (size_t)up.ext * n, d0 + skip + z, digits, q->dev);
                b.out[z] = us + z * 2 * (size_t)up.ext * n, outs[z] = x + (skip + z) * xw;
            }
            launch_weighted(ctx, b, up.beta, lv + 1, st);
            CMCHK(weighted_down(ctx, us, lv + 1, b.nz, outs, tmp, st));
        }
        if (joint) {
            u64 *outs[CM_KS_BATCH];
            for (int z = 0; z < m; z++) outs[z] = scores[d0 + z].dev;
            CMCHK(kv_passes_run(ctx, evk, kv, tr->passes, kv->d_x, m, outs, st));
        }
        for (int z = 0; z < m; z++) {
            cm_ct in{x + z * xw, lv, 2, q->scale}, &out = scores[d0 + z];
            if (joint) out.level = lv - 1, out.ncomp = 2, out.scale = in.scale * kv->scale / (double)ctx->mod[lv];
            else if (kv->indexed) CMCHK(kv_sv(ctx, evk, kv, &in, &out, st, false, kv->d_x, false));
            else CMCHK(kv_qk(ctx, evk, kv, &in, &out, st, false));
        }
        for (int r0 = 0; r0 < (int)masked.size(); r0 += TREE_ROWS) {
            TreeMask mk;
            const int mr = std::min(TREE_ROWS, (int)masked.size() - r0);
            for (int z = 0; z < CM_KS_BATCH; z++) mk.score[z] = scores[d0 + (z < m ? z : 0)].dev;
            for (int r = 0; r < TREE_ROWS; r++) {
                const int c = masked[r0 + (r < mr ? r : 0)];
                mk.row[r] = r < mr ? (unsigned)rot_g(kv, -(long long)c * kv->H * t) : 1;
                for (int z = 0; z < CM_KS_BATCH; z++) {
                    u64 bits = r < mr && z < m ? tr->empty[c] : 0;
                    for (int j = 0; j < t && r < mr && z < m && c >= page; j++) {
                        const int place = (c - page) * t + j, u = (j - (d0 + z) + t) % t % per;
                        if (place >= start && !(seen[u][c - page] >> j & 1)) bits |= 1ULL << j;
                    }
                    mk.bits[r][z] = bits;
                }
            }
            for (int j = 0; j < TREE_T; j++) mk.residue[j] = j < t ? (unsigned)galois_of_step(ctx, -j) : 1;
            Prof prof_(ctx, CM_K_ELEMENTWISE, (double)m * (ls + 1), st);
            hipLaunchKernelGGL(k_tree_mask, dim3(n / 256, ls + 1, m), dim3(256), 0, st, mk, mr, tr->d_one, r0 == 0 ? unseen : nullptr, gu, ctx->d_modc, (int)n, ctx->logn);
        }
    }
    RETURN_LAUNCH_STATUS();
    CM_CATCH
}
extern "C" cm_status cm_tree_sv(cm_ctx *ctx, const cm_evk *evk, const cm_tree *tr, const cm_kv *kv, const cm_ct *scores, cm_ct *out, void *stream) {
    (void)hipGetLastError();          // stale errors of earlier calls are not this call's
    if (!ctx || !evk || !tr || !kv || tr->ctx != ctx || kv->ctx != ctx || !scores || !out || !out->dev || !evk_fits(ctx, evk)) return CM_E_INVAL;
    if (!tree_fits(tr, kv)) return CM_E_LAYOUT;
    if (kv->level != tr->level) return CM_E_LEVEL;
    const int lv = kv->level, t = tr->t_kv, lp = lv - 1;
    for (int d = 0; d < t; d++) {
        if (!scores[d].dev || scores[d].ncomp != 2) return CM_E_INVAL;
        if (scores[d].level != lv) return CM_E_LEVEL;
        if (!(fabs(scores[d].scale / scores[0].scale - 1) < 1e-9)) return CM_E_SCALE;
    }
    CM_TRY
    CMCHK(tree_keys(evk, tr));
    CMCHK(kv_sv_keys(evk, kv, false, false));
    hipStream_t st = (hipStream_t)stream;
    const KsLevel &dn = ks_level(ctx, lp);
    const size_t n = ctx->n, B = CM_KS_BATCH, pw = 2 * (size_t)lv * n, dblk = (size_t)dn.beta * dn.ext * n, ublk = 2 * (size_t)dn.ext * n;
    u64 *parts = tr->d_work, *ksin = parts + B * pw, *digits = ksin + B * (size_t)lv * n, *acc = digits + B * dblk, *nxt = acc + ublk, *own = nxt + ublk,
        *res = own + pw, *tmp = res + pw;
    const double scale = scores[0].scale * kv->scale / (double)ctx->mod[lv];
    const bool joint = kv_passes_fit(tr->passes, kv);
    const int turn = joint ? tr->passes.P : CM_KS_BATCH;
    bool any = false;
    for (int d0 = 0; d0 < t; d0 += turn) {
        const int m = std::min(turn, t - d0), skip = d0 == 0;
        // the results, the one that does not move in a place of its own
        u64 *to[CM_KS_BATCH];
        for (int z = 0; z < m; z++) to[z] = d0 + z == 0 ? own : parts + (z - skip) * pw;
        if (joint) {
            u64 *dst[CM_KS_BATCH];
            const u64 *src[CM_KS_BATCH];
            for (int z = 0; z < m; z++) dst[z] = tr->passes.babies + z * tr->passes.r_i * kv_ctw(kv), src[z] = scores[d0 + z].dev;
            launch_copies(dst, src, m, kv_ctw(kv), st);
            CMCHK(kv_passes_run(ctx, evk, kv, tr->passes, kv->d_v, m, to, st));
        } else {
            for (int z = 0; z < m; z++) {
                cm_ct part{to[z], lp, 2, 0.0};
                CMCHK(kv_sv(ctx, evk, kv, &scores[d0 + z], &part, st, false, kv->d_v, false));
            }
        }
        if (m == skip) continue;
        if (n == 65536) CMCHK(ks_raise_apart(ctx, tr->tabs, to + skip, ksin, digits, st, m - skip));
        else CMCHK(ks_raise_many(ctx, tr->tabs, parts, ksin, digits, st, m - skip));
        WrBatch b;
        b.nz = 1, b.nsum = 2 * (m - skip);
        for (int z = skip; z < m; z++)
            tree_moves(evk, tr, b.it + 2 * (z - skip), tr->d_v, (size_t)dn.ext * n, t - (d0 + z), digits + (z - skip) * dblk, parts + (z - skip) * pw);
        b.extra[0] = any ? acc : nullptr, b.out[0] = nxt;
        launch_weighted(ctx, b, dn.beta, lp, st);
        std::swap(acc, nxt);
        any = true;
    }
    if (any) {
        CMCHK(weighted_down(ctx, acc, lp, 1, &res, tmp, st));
        hipLaunchKernelGGL(k_add_dropped, dim3(n / 256, lp, 2), dim3(256), 0, st, out->dev, res, own, ctx->d_modc, lp, (int)n);
    } else {
        u64 *dst[2] = {out->dev, out->dev + (size_t)lp * n};
        const u64 *src[2] = {own, own + (size_t)lv * n};
        launch_copies(dst, src, 2, (size_t)lp * n, st);
    }
    out->level = lp - 1, out->ncomp = 2, out->scale = scale;
    RETURN_LAUNCH_STATUS();
    CM_CATCH
}
