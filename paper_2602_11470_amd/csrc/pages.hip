// Pages of an encrypted cache: copies of a cache (cm_kv_fork) and the kept tokens of one moved into another (cm_kv_take).
//
// Page c of a cache is its tokens c t .. c t + t - 1.  With B = H t slots a row and E rows:
//   K ciphertext c              holds page c, dim e in row e;
//   V ciphertext k = g r_i + j  holds page c in row c - j, as dim c - j - g r_i         (rows and dims modulo E);
//   X ciphertext k = g r_i + j  (the key index) holds page c in row c + g r_i, as dim c + g r_i + j.
// So dropping tokens multiplies every V and X ciphertext by a rotation of ONE 0/1 mask M (the kept tokens, page c in row c): by
// Rot(M, j B) and Rot(M, -g r_i B).  A rescale follows: the result lies one level below.  A page that moves from c to c' = c + s
// keeps its dims, which says where it goes:
//   V: k' = k + s (mod E), its rows by (g' - g) r_i to the right;      X: k' = k - s (mod E), its rows by j - j' to the right.
// Every ciphertext therefore moves as a whole: to another place, and by one rotation by whole rows where the giant step (V) or
// the baby step (X) of the place is another one.  K ciphertexts move without any arithmetic, unless a page keeps some of its
// tokens only (a mask by residues).
#include <math.h>

#include <algorithm>

#include "kv.h"

typedef u64 u64x2 __attribute__((ext_vector_type(2)));

// One ciphertext of the result that is a masked product: where it comes from and goes to (array 0 K, 1 V, 2 X as stored), which mask, the
// Galois element that the mask is read through, the rows it turns by (left).
struct Move {
    int array, from, to, mask, rows;
    unsigned g;
};
struct cm_kv_sel {
    cm_ctx *ctx = nullptr;
    int H, E, t, r_i, level, ntok, shift, kept_end;     // level of the source; kept_end: one past the last kept token, after the move
    bool indexed = false, any = false;                  // any: a token is kept
    std::vector<Move> moves;                            // ordered by rows
    std::vector<int> rows;                              // the amounts other than 0, ascending
    u64 *d_masks = nullptr;                             // [1 + patterns][level+1][n], multiplier form
    int *d_from = nullptr;                              // [E] per page of the result: the page copied there, or -1
    KsManyTables tabs;                                  // raises of ks_batch_max moved ciphertexts, level - 1
};

static bool same_shape(const cm_kv *a, const cm_kv *b) {
    return a->H == b->H && a->E == b->E && a->r_i == b->r_i && a->indexed == b->indexed;
}

// ---- copies -----------------------------------------------------------------------------------------------------------
// A lane moves 16 bytes of a limb: to every destination that has the limb, reading them once.  Bound by memory: 2.6 GB read and written
// once 430 us (6.2 TB/s, the card's own copy 5.85), read once and written four times 13.5 GB 2.3 to 2.4 ms.  More words a lane: 2, 4 and 8 pairs
// 435, 444 and 485 us; plain instead of non-temporal loads and stores of 8 pairs 505.
#define LANES 256
#define LANE_WORDS (2 * LANES)                   // words a workgroup moves
#define MAX_Y 65534                              // workgroups along y, even: two components a ciphertext
#define FORK_MAX 8
struct ForkDst {
    u64 *k, *v, *x;
    int level, pages;
};
struct ForkArgs {
    const u64 *k, *v, *x;
    int level, top, used, cts, E, n, ndst;       // level of the source, highest level of a destination, pages in use, ciphertexts to copy
    ForkDst d[FORK_MAX];
};
// grid: x = piece of a limb, y = ciphertext and component from y0 on: pages in use, V, X, then the pages behind the last one, which are cleared
__global__ __launch_bounds__(LANES) void k_fork(ForkArgs a, int y0) {
    const int per = a.n / LANE_WORDS, l = blockIdx.x / per, y = blockIdx.y + y0, c = y & 1, z = y >> 1;
    const size_t at = (size_t)(blockIdx.x % per) * LANE_WORDS + 2 * threadIdx.x, limb = (size_t)c * (a.level + 1) + l;
    if (z >= a.cts) {
        const int page = a.used + z - a.cts;
        for (int d = 0; d < a.ndst; d++) {
            const ForkDst &t = a.d[d];
            if (l > t.level || page >= t.pages) continue;
            __builtin_nontemporal_store(u64x2{0, 0}, (u64x2 *)(t.k + (((size_t)page * 2 + c) * (t.level + 1) + l) * a.n + at));
        }
        return;
    }
    const int array = z < a.used ? 0 : z < a.used + a.E ? 1 : 2, i = z - (array ? a.used : 0) - (array == 2 ? a.E : 0);
    const u64 *src = (array == 0 ? a.k : array == 1 ? a.v : a.x) + (2 * (size_t)(a.level + 1) * i + limb) * a.n + at;
    const u64x2 w = __builtin_nontemporal_load((const u64x2 *)src);
    for (int d = 0; d < a.ndst; d++) {
        const ForkDst &t = a.d[d];
        if (l > t.level) continue;
        u64 *dst = (array == 0 ? t.k : array == 1 ? t.v : t.x) + (((size_t)i * 2 + c) * (t.level + 1) + l) * a.n + at;
        __builtin_nontemporal_store(w, (u64x2 *)dst);
    }
}

extern "C" cm_status cm_kv_view(const cm_kv *kv, int32_t which, int32_t idx, cm_ct *out) {
    if (!kv || !out) return CM_E_INVAL;
    if (which != CM_QK && which != CM_SV && !(which == CM_KV_INDEX && kv->indexed)) return CM_E_INVAL;
    if (idx < 0 || idx >= (which == CM_QK ? kv->nk_max : kv->E)) return CM_E_LAYOUT;
    out->dev = (which == CM_QK ? kv->d_k : which == CM_SV ? kv->d_v : kv->d_x) + (size_t)(which == CM_KV_INDEX ? x_place(kv, idx) : idx) * kv_ctw(kv);
    out->level = kv->level, out->ncomp = 2, out->scale = kv->scale;
    return CM_OK;
}
extern "C" cm_status cm_kv_seek(cm_kv *kv, int32_t token) {
    if (!kv || token < 0 || token > kv->max_tokens) return CM_E_INVAL;
    kv->pos = token;
    return CM_OK;
}
extern "C" cm_status cm_kv_fork(cm_ctx *ctx, const cm_kv *src, cm_kv *const *dsts, int32_t ndst, void *stream) {
    (void)hipGetLastError();          // stale errors of earlier calls are not this call's
    if (!ctx || !src || src->ctx != ctx || !dsts || ndst < 1) return CM_E_INVAL;
    for (int d = 0; d < ndst; d++) {
        if (!dsts[d] || dsts[d]->ctx != ctx || dsts[d] == src) return CM_E_INVAL;
        for (int e = 0; e < d; e++) if (dsts[e] == dsts[d]) return CM_E_INVAL;
        if (!same_shape(src, dsts[d]) || dsts[d]->max_tokens < src->ntok || dsts[d]->max_tokens < src->pos) return CM_E_LAYOUT;
        if (dsts[d]->level > src->level) return CM_E_LEVEL;
    }
    hipStream_t st = (hipStream_t)stream;
    const int used = (src->ntok + src->t - 1) / src->t, n = ctx->n;
    for (int d0 = 0; d0 < ndst; d0 += FORK_MAX) {
        ForkArgs a{src->d_k, src->d_v, src->d_x, src->level, 0, used, used + (src->indexed ? 2 : 1) * src->E, src->E, n, std::min(ndst - d0, FORK_MAX), {}};
        int clear = 0;
        for (int d = 0; d < a.ndst; d++) {
            const cm_kv *t = dsts[d0 + d];
            a.d[d] = {t->d_k, t->d_v, t->d_x, t->level, t->nk_max};
            a.top = std::max(a.top, t->level), clear = std::max(clear, t->nk_max - used);
        }
        const int rows = 2 * (a.cts + clear);
        Prof prof_(ctx, CM_K_ELEMENTWISE, (double)rows * (a.top + 1), st);
        for (int y = 0; y < rows; y += MAX_Y)
            hipLaunchKernelGGL(k_fork, dim3((a.top + 1) * (n / LANE_WORDS), std::min(rows - y, MAX_Y)), dim3(LANES), 0, st, a, y);
    }
    for (int d = 0; d < ndst; d++)
        dsts[d]->ntok = src->ntok, dsts[d]->pos = src->pos, dsts[d]->scale = src->scale, dsts[d]->scale_set = src->scale_set;
    RETURN_LAUNCH_STATUS();
}

// ---- kept tokens ----------------------------------------------------------------------------------------------------------
// V ciphertext k goes to place k + s, index ciphertext k to k - s (in the numbering of cm_kv_load)
static void sel_moves(cm_kv_sel *s, const cm_kv *kv) {
    const int E = s->E, r_i = s->r_i;
    const long long B = (long long)s->H * s->t;
    auto mod = [E](int a) { return (a % E + E) % E; };
    for (int to = 0; to < E; to++) {
        const int k = mod(to - s->shift);
        s->moves.push_back({1, k, to, 0, mod((k / r_i - to / r_i) * r_i), (unsigned)rot_g(kv, k % r_i * B)});
    }
    for (int p = 0; p < E && s->indexed; p++) {                   // by places, so that neighbours share their source's neighbourhood
        const int r_o = E / r_i, to = p % r_o * r_i + p / r_o, k = mod(to + s->shift);
        s->moves.push_back({2, x_place(kv, k), p, 0, mod(to % r_i - k % r_i), (unsigned)rot_g(kv, -(k / r_i * r_i) * B)});
    }
    std::stable_sort(s->moves.begin(), s->moves.end(), [](const Move &a, const Move &b) { return a.rows < b.rows; });
    for (const Move &m : s->moves)
        if (m.rows && (s->rows.empty() || s->rows.back() != m.rows)) s->rows.push_back(m.rows);
}
extern "C" void cm_kv_sel_destroy(cm_kv_sel *s) {
    if (!s) return;
    hipFree(s->d_masks), hipFree(s->d_from);
    ks_many_tables_destroy(&s->tabs);
    delete s;
}
// the kept residues of page c, and how many they are
static int page_pattern(const cm_kv *like, const uint8_t *keep, int ntok, int c, std::vector<uint8_t> &p) {
    int kept = 0;
    p.assign(like->t, 0);
    for (int r = 0; r < like->t && c * like->t + r < ntok; r++)
        if (keep[c * like->t + r]) p[r] = 1, kept++;
    return kept;
}
extern "C" int32_t cm_kv_sel_masks(const cm_kv *like, const uint8_t *keep, int32_t ntok) {
    if (!like || !keep || ntok < 0 || ntok > like->E * like->t) return 0;
    try {
        std::vector<std::vector<uint8_t>> patterns;
        std::vector<uint8_t> p;
        bool any = false;
        for (int c = 0; c * like->t < ntok; c++) {
            const int kept = page_pattern(like, keep, ntok, c, p);
            any = any || kept;
            if (kept && kept < std::min(like->t, ntok - c * like->t) && std::find(patterns.begin(), patterns.end(), p) == patterns.end()) patterns.push_back(p);
        }
        return any ? 1 + (int32_t)patterns.size() : 0;
    } catch (...) {
        return 0;
    }
}
extern "C" cm_status cm_kv_sel_create(cm_ctx *ctx, const cm_kv *like, const uint8_t *keep, int32_t ntok, int32_t shift, const int64_t *coeffs,
                                      cm_kv_sel **out) {
    (void)hipGetLastError();          // stale errors of earlier calls are not this call's
    if (!ctx || !like || like->ctx != ctx || !out || ntok < 0 || (ntok && !keep)) return CM_E_INVAL;
    if (like->level < 3) return CM_E_LEVEL;                      // the result is a cache, and those begin at level 2
    const int t = like->t, E = like->E, S = like->S;
    if (ntok > E * t || shift <= -E || shift >= E) return CM_E_LAYOUT;
    cm_kv_sel *s = new (std::nothrow) cm_kv_sel();
    if (!s) return CM_E_NOMEM;
    cm_status status = CM_OK;
    try {
        s->ctx = ctx, s->H = like->H, s->E = E, s->t = t, s->r_i = like->r_i, s->level = like->level, s->ntok = ntok, s->shift = shift, s->kept_end = 0;
        s->indexed = like->indexed;
        const int pages = (ntok + t - 1) / t;
        std::vector<std::vector<uint8_t>> patterns;
        std::vector<int> from(E, -1);
        for (int c = 0; c < pages && status == CM_OK; c++) {
            const int stored = std::min(t, ntok - c * t);
            std::vector<uint8_t> p;
            const int kept = page_pattern(like, keep, ntok, c, p);
            if (!kept) continue;
            for (int r = 0; r < stored; r++) if (p[r]) s->kept_end = (c + shift) * t + r + 1;
            if (c + shift < 0 || c + shift >= E) { status = CM_E_LAYOUT; break; }
            s->any = true;
            if (kept == stored) {
                from[c + shift] = c;
                continue;
            }
            const size_t i = std::find(patterns.begin(), patterns.end(), p) - patterns.begin();
            if (i == patterns.size()) patterns.push_back(p);
            s->moves.push_back({0, c, c + shift, 1 + (int)i, 0, 1});
        }
        if (s->any) sel_moves(s, like);
        if (status == CM_OK && s->any) {
            const int n = ctx->n, lv = s->level;
            const size_t words = (size_t)(lv + 1) * n;
            const double scale = (double)ctx->mod[lv];           // what the rescale divides by
            if (hipMalloc((void **)&s->d_masks, (1 + patterns.size()) * words * 8) != hipSuccess || hipMalloc((void **)&s->d_from, E * sizeof(int)) != hipSuccess)
                status = CM_E_NOMEM;
            else if (hipMemcpy(s->d_from, from.data(), E * sizeof(int), hipMemcpyHostToDevice) != hipSuccess)
                status = CM_E_HIP;
            std::vector<double> m(S);
            for (size_t i = 0; i <= patterns.size() && status == CM_OK; i++) {
                cm_pt pt;
                pt.dev = s->d_masks + i * words, pt.mont = 1;
                for (int a = 0; a < S; a++) {                    // slot (row, h, residue)
                    const int tok = a / (s->H * t) * t + a % t;
                    m[a] = i ? patterns[i - 1][a % t] : tok < ntok && keep[tok] ? 1.0 : 0.0;
                }
                status = coeffs ? cm_pt_from_coeffs(ctx, coeffs + i * n, lv, scale, &pt) : cm_encode(ctx, m.data(), nullptr, S, lv, scale, &pt);
            }
            if (status == CM_OK && !s->rows.empty() && !ks_batches_grow(ctx)) status = CM_E_NOMEM;
            if (status == CM_OK && !s->rows.empty()) status = ks_many_tables_create(ctx, lv - 1, ks_batch_max(ctx, lv - 1), &s->tabs, 2, 1);
            if (status == CM_OK) ks_level(ctx, lv), get_qlinv(ctx, lv), get_pinv(ctx, lv - 1);      // the per-level tables that a take reads
        }
    } catch (...) {
        status = CM_E_NOMEM;
    }
    if (status != CM_OK) {
        cm_kv_sel_destroy(s);
        return status;
    }
    *out = s;
    return CM_OK;
}
extern "C" int32_t cm_kv_sel_steps(const cm_kv_sel *s, int32_t *steps, int32_t cap) {
    if (!s) return 0;
    for (int i = 0; i < (int)s->rows.size() && i < cap && steps; i++) steps[i] = s->rows[i] * s->H * s->t;
    return (int32_t)s->rows.size();
}

// K pages of the result, grid as in k_fork: page (+)= the page from[page] of the source, a level above; zero, or nothing added, where there is none
template <bool ADD>
__global__ __launch_bounds__(LANES) void k_pages(u64 *out, const u64 *in, const int *from, const ModC *__restrict__ modc, int level, int n, int y0) {
    const int per = n / LANE_WORDS, l = blockIdx.x / per, y = blockIdx.y + y0, c = y & 1, page = y >> 1, src = from ? from[page] : -1;
    const size_t at = (size_t)(blockIdx.x % per) * LANE_WORDS + 2 * threadIdx.x;
    u64x2 *dst = (u64x2 *)(out + (((size_t)page * 2 + c) * (level + 1) + l) * n + at);
    u64x2 w = {0, 0};
    if (src >= 0) w = __builtin_nontemporal_load((const u64x2 *)(in + (((size_t)src * 2 + c) * (level + 2) + l) * n + at));
    if (ADD) {
        if (src < 0) return;
        const u64 q = modc[l].q;
        const u64x2 o = __builtin_nontemporal_load(dst);
        w = u64x2{addmod(w.x, o.x, q), addmod(w.y, o.y, q)};
    }
    __builtin_nontemporal_store(w, dst);
}
__global__ __launch_bounds__(LANES) void k_clear(u64 *p) { ((u64x2 *)p)[(size_t)blockIdx.x * LANES + threadIdx.x] = u64x2{0, 0}; }

extern "C" cm_status cm_kv_take(cm_ctx *ctx, const cm_evk *evk, const cm_kv_sel *s, const cm_kv *src, cm_kv *dst, int32_t add, void *stream) {
    (void)hipGetLastError();
    if (!ctx || !s || s->ctx != ctx || !src || src->ctx != ctx || !dst || dst->ctx != ctx || src == dst) return CM_E_INVAL;
    if (!s->rows.empty() && (!evk || !evk_fits(ctx, evk))) return CM_E_INVAL;
    if (!same_shape(src, dst) || s->H != src->H || s->E != src->E || s->r_i != src->r_i || s->indexed != src->indexed) return CM_E_LAYOUT;
    if (src->level != s->level || dst->level != s->level - 1) return CM_E_LEVEL;
    if (src->ntok != s->ntok || s->kept_end > dst->max_tokens) return CM_E_LAYOUT;
    if (add && src->scale_set && dst->scale_set && fabs(src->scale / dst->scale - 1) > 1e-9) return CM_E_SCALE;
    CM_TRY
    for (int rows : s->rows)
        if (!find_key(evk, rot_g(src, (long long)rows * s->H * s->t))) return CM_E_NOKEY;
    hipStream_t st = (hipStream_t)stream;
    const int lv = s->level, lo = lv - 1, n = ctx->n;
    const size_t ctw_in = kv_ctw(src), ctw = kv_ctw(dst);
    // K: pages kept whole are copied, the places without one cleared; then the pages that keep some of their tokens
    if (!add || s->any) {
        const int rows = 2 * dst->nk_max;
        Prof prof_(ctx, CM_K_ELEMENTWISE, (double)rows * lv, st);
        for (int y = 0; y < rows; y += MAX_Y)
            hipLaunchKernelGGL((add ? k_pages<true> : k_pages<false>), dim3(lv * (n / LANE_WORDS), std::min(rows - y, MAX_Y)), dim3(LANES), 0, st, dst->d_k,
                               src->d_k, s->d_from, ctx->d_modc, lo, n, y);
    }
    if (!s->any) {
        for (int i = 0; i < dst->E && !add; i++) {               // an empty cache
            hipLaunchKernelGGL(k_clear, dim3((unsigned)(ctw / LANE_WORDS)), dim3(LANES), 0, st, dst->d_v + i * ctw);
            if (dst->indexed) hipLaunchKernelGGL(k_clear, dim3((unsigned)(ctw / LANE_WORDS)), dim3(LANES), 0, st, dst->d_x + i * ctw);
        }
    } else {
        // K pages kept in part, V and X: masked products, rescaled, as many a batch as the work area has room for; those that turn
        // next to one another and then rotated, ks_batch_max at a time
        const KsLevel &kl = ks_level(ctx, lo);
        const size_t ln = (size_t)lv * n, dblk = (size_t)kl.beta * kl.ext * n, ublk = 2 * (size_t)kl.ext * n;
        const u64 *in[3] = {src->d_k, src->d_v, src->d_x};
        u64 *out[3] = {dst->d_k, dst->d_v, dst->d_x};
        const int fused = rescale_masked_batch(ctx, lv, dst->work_words);
        // those that turn: stacked in front of the masked product's last limbs and residues, and of what a batch of key switches takes;
        // the work area has room for CM_KS_BATCH of them (fused or in two steps)
        const int batch = ks_batch_max(ctx, lo);
        int turning = CM_KS_BATCH;
        while (fused && turning < CM_MASK_BATCH &&
               (turning + 1) * ctw + std::max(std::min(turning + 1, batch) * (ln + dblk), (turning + 1) * ctw_in) <= dst->work_words)
            turning++;
        for (size_t i = 0; i < s->moves.size();) {
            // what is left of those that turn by the same rows: in batches of the same size where they do not turn (257 products in nine batches
            // 1378 us, in eight of 32 and one 1388), else as many as fit (of 32 in batches of 24 and 8 1780 us, of 16 and 16 1817)
            const int rows = s->moves[i].rows, most = rows ? turning : fused ? fused : CM_KS_BATCH;
            int left = 0;
            while (i + left < s->moves.size() && s->moves[i + left].rows == rows) left++;
            const int batches = (left + most - 1) / most, cap = rows ? std::min(left, most) : (left + batches - 1) / batches;
            int m = 0;
            MulPtBatch mb;
            u64 *outs[CM_MASK_BATCH], *to[CM_MASK_BATCH];
            for (; m < cap; m++) {
                const Move &v = s->moves[i + m];
                mb.src[m] = in[v.array] + v.from * ctw_in, mb.g[m] = v.g, mb.at[m] = v.mask;
                to[m] = out[v.array] + v.to * ctw, outs[m] = rows ? dst->d_work + m * ctw : to[m];
            }
            u64 *work = dst->d_work + (rows ? m * ctw : 0), *last = work, *red = last + (size_t)m * 2 * n, *prods = red + (size_t)m * 2 * lv * n;
            const bool acc = add && !rows;
            if (!rescale_masked_into(ctx, mb, m, s->d_masks, lv, outs, st, last, red, acc)) {
                launch_mul_pt_rot_batch(ctx, prods, mb, m, s->d_masks, lv + 1, st);
                for (int r = 0; r < m; r++) CMCHK(rescale_into(ctx, prods + r * ctw_in, 2, lv, outs[r], st, last, red, acc));
            }
            for (int r0 = 0; r0 < m && rows; r0 += batch) {
                const u64 g = rot_g(src, (long long)rows * s->H * s->t), *key = find_key(evk, g);
                const int b = std::min(m - r0, batch);
                const bool half = rows_ip_fits(ctx, kl.beta, lo, b, 1);
                u64 *ksin = work, *digits = ksin + b * ln, *bu = arena_batch_sums(ctx);
                CMCHK(ks_raise_many(ctx, s->tabs, outs[r0], ksin, digits, st, b, g, half));
                IpBatch ip;
                ip.nz = b, ip.nsum = 1;
                const u64 *adds[CM_MASK_BATCH], *accs[CM_MASK_BATCH];
                for (int r = 0; r < b; r++) {
                    ip.it[r].dig = digits + r * dblk, ip.it[r].key = key, ip.out[r] = bu + r * ublk;
                    ip.it[r].own = outs[r0 + r] + ln, ip.it[r].own_g = (unsigned)g;
                    adds[r] = outs[r0 + r], accs[r] = add ? to[r0 + r] : nullptr;
                }
                // one key for all: its words stay in registers over the batch, except at n = 4096, where there are too few lanes for that
                // (ten ciphertexts 20.4 us against 6.8)
                if (half) launch_rows_ip(ctx, ip, kl.beta, lo, st, lo + 1);
                else if (n == 4096) launch_inner_product_batch(ctx, ip, kl.beta, lo, st);
                else launch_inner_product_shared_key(ctx, ip, kl.beta, lo, st);
                CMCHK(moddown_batch_into(ctx, bu, lo, b, adds, 1, g, accs, to + r0, st, half));
            }
            i += m;
        }
    }
    dst->ntok = add ? std::max(dst->ntok, s->kept_end) : s->kept_end;
    dst->pos = dst->ntok;
    if (!add) dst->scale = src->scale, dst->scale_set = src->scale_set && s->any;
    else if (s->any && src->scale_set && !dst->scale_set) dst->scale = src->scale, dst->scale_set = true;
    RETURN_LAUNCH_STATUS();
    CM_CATCH
}
