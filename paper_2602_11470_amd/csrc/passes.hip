// Several passes of scores-times-V (or of query-times-K on the key index) taken together.  Each is what kv_sv does with one: hoisted
// rotations by rows, products with the cache, relinearisations, giant steps, ModDown and rescale -- the same words.  Together a rotation's key is read
// and its uniform half drawn once for four passes, the cache is read once for four, relinearisations and ModDowns fill batches of up to
// CM_MASK_BATCH, and a turn has a quarter of the launches or fewer.
#include "passes.h"

#include <algorithm>

#define PS_TPB 256
#define PS_KEYS 16                 // keys of a launch
#define PS_GROUP 4                 // passes of a lane
typedef u64 u64x2 __attribute__((ext_vector_type(2)));

struct CopyBatch {
    u64 *dst[CM_KS_BATCH];
    const u64 *src[CM_KS_BATCH];
};
__global__ __launch_bounds__(PS_TPB) void k_copies(CopyBatch b) {
    const size_t i = 2 * ((size_t)blockIdx.x * PS_TPB + threadIdx.x);
    *reinterpret_cast<u64x2 *>(b.dst[blockIdx.y] + i) = *reinterpret_cast<const u64x2 *>(b.src[blockIdx.y] + i);
}
void launch_copies(u64 *const *dst, const u64 *const *src, int m, size_t words, hipStream_t st) {
    CopyBatch b;
    for (int z = 0; z < CM_KS_BATCH; z++) b.dst[z] = dst[z < m ? z : 0], b.src[z] = src[z < m ? z : 0];
    hipLaunchKernelGGL(k_copies, dim3(words / (2 * PS_TPB), m), dim3(PS_TPB), 0, st, b);
}

// Rotations of several ciphertexts by the same steps, before their ModDown: out[a][p] = sum_j sigma_a(dig_p,j) key_a,j for `per` keys a
// a workgroup and PS_GROUP passes p.  As in k_inner_product_fanout a lane keeps the digit words of two source positions and writes each result
// where the key's Galois map sends them; here it keeps those of PS_GROUP passes, so a key's words are read and drawn once for all.  seconds
// (nullable): the polynomials that were raised, `stride` words apart, where a digit's own limbs are read.
// Bound by its writes at n = 65536: four keys, eight passes, two digits, nine limbs 83 us (302 MB written, 3.7 TB/s), one digit, eight limbs 61 us (4.4).
// Eight, four and two keys a workgroup are equal there; at n = 4096, where a launch is as long as a workgroup's chain, one key 11.9 us, eight 23.7.
struct FanPasses {
    int n, per;                         // keys, of a workgroup
    const u64 *key[PS_KEYS];
    unsigned ginv[PS_KEYS];
};
template <bool SA, int NB>
__global__ __launch_bounds__(PS_TPB) void k_fan_passes(FanPasses f, u64 *__restrict__ out, const u64 *__restrict__ dig, const u64 *__restrict__ seconds,
                                                       size_t stride, int alpha, int passes, const ModC *__restrict__ modc,
                                                       int beta, int ext, int level, int L, int nmod, int n, int logn, EvkA eva, const u64 *__restrict__ ubound) {
    const int chunks = (f.n + f.per - 1) / f.per;
    const unsigned s2 = (blockIdx.x * PS_TPB + threadIdx.x) * 2;
    const int r = blockIdx.y, mi = r <= level ? r : L + 1 + (r - level - 1), p0 = (int)(blockIdx.z / chunks) * PS_GROUP;
    const int first = (int)(blockIdx.z % chunks) * f.per, end = min(f.n, first + f.per);
    const ModC m = modc[mi];
    const u64 bound = ubound[mi];
    const bool small = m.q < (1ULL << 50);
    const int own = r <= level ? r / alpha : -1;
    const size_t dblk = (size_t)beta * ext * n, ublk = 2 * (size_t)ext * n;
    ulonglong2 d[PS_GROUP][NB];
#pragma unroll
    for (int p = 0; p < PS_GROUP; p++)
#pragma unroll
        for (int j = 0; j < NB; j++)
            if (j < beta) {
                const int q = min(p0 + p, passes - 1);
                const u64 *w = seconds && j == own ? seconds + q * stride + (size_t)r * n : dig + q * dblk + ((size_t)j * ext + r) * n;
                d[p][j] = *reinterpret_cast<const ulonglong2 *>(w + s2);
            }
    for (int a = first; a < end; a++) {
        const unsigned dst = perm_src(s2, f.ginv[a], logn), base = dst & ~1u;
        const bool swap = dst & 1u;
        const u64 cg0 = ((u64)base + 1) * GOLD, cg1 = cg0 + GOLD;
        ulonglong2 eb[NB], ea[NB];
#pragma unroll
        for (int j = 0; j < NB; j++)
            if (j < beta) {
                const u64x2 w = __builtin_nontemporal_load(reinterpret_cast<const u64x2 *>(f.key[a] + ((size_t)j * nmod + mi) * n + base));
                eb[j] = make_ulonglong2(w.x, w.y);
                ea[j] = evk_a_words<SA>(f.key[a], eva, nmod, n, j, mi, base, cg0, cg1, bound);
            }
#pragma unroll
        for (int p = 0; p < PS_GROUP; p++) {
            if (p0 + p >= passes) break;
            u128 a0 = 0, a1 = 0, b0 = 0, b1 = 0;
            if (small) {
                Acc50 A0, A1, B0, B1;
#pragma unroll
                for (int j = 0; j < NB; j++)
                    if (j < beta) {
                        const u64 dx = swap ? d[p][j].y : d[p][j].x, dy = swap ? d[p][j].x : d[p][j].y;
                        const unsigned x0 = (unsigned)dx & LOW25, x1 = (unsigned)(dx >> 25), y0 = (unsigned)dy & LOW25, y1 = (unsigned)(dy >> 25);
                        B0.mac(x0, x1, eb[j].x), B1.mac(y0, y1, eb[j].y), A0.mac(x0, x1, ea[j].x), A1.mac(y0, y1, ea[j].y);
                    }
                a0 = A0.total(), a1 = A1.total(), b0 = B0.total(), b1 = B1.total();
            } else {
#pragma unroll
                for (int j = 0; j < NB; j++)
                    if (j < beta) {
                        const u64 dx = swap ? d[p][j].y : d[p][j].x, dy = swap ? d[p][j].x : d[p][j].y;
                        b0 += (u128)dx * eb[j].x, b1 += (u128)dy * eb[j].y, a0 += (u128)dx * ea[j].x, a1 += (u128)dy * ea[j].y;
                    }
            }
            u64 *o = out + ((size_t)a * passes + p0 + p) * ublk + (size_t)r * n + base;
            const u64x2 w0 = {redc(b0, m.q, m.qinv), redc(b1, m.q, m.qinv)}, w1 = {evk_a_reduce<SA>(a0, m), evk_a_reduce<SA>(a1, m)};
            *reinterpret_cast<u64x2 *>(o) = w0;
            *reinterpret_cast<u64x2 *>(o + (size_t)ext * n) = w1;
        }
    }
}
static void launch_fan_passes(cm_ctx *ctx, const FanPasses &f, u64 *out, const u64 *dig, const u64 *seconds, size_t stride, int passes, int beta, int level, hipStream_t st) {
    Prof prof_(ctx, CM_K_INNER_PRODUCT, f.n * passes, st);
    const int ext = level + 1 + ctx->K;
    const dim3 grid(ctx->n / (2 * PS_TPB), ext, (f.n + f.per - 1) / f.per * ((passes + PS_GROUP - 1) / PS_GROUP));
#define FANP(SA_, NB_)                                                                                                                                  \
    hipLaunchKernelGGL((k_fan_passes<SA_, NB_>), grid, dim3(PS_TPB), 0, st, f, out, dig, seconds, stride, ctx->alpha, passes, ctx->d_modc, beta, ext, level, ctx->L, ctx->nmod, ctx->n, \
                       ctx->logn, evk_a_of(ctx), ctx->d_ubound)
    if (ctx->evk_stored_a) {
        if (beta <= 2) FANP(true, 2);
        else FANP(true, 6);
    } else if (beta <= 1) FANP(false, 1);
    else if (beta <= 2) FANP(false, 2);
    else if (beta <= 4) FANP(false, 4);
    else FANP(false, 6);
#undef FANP
}

void kv_passes_destroy(KvPasses *kp) {
    ks_many_tables_destroy(&kp->baby_tabs), ks_many_tables_destroy(&kp->relin_tabs), ks_many_tables_destroy(&kp->giant_tabs);
    hipFree(kp->babies);
    *kp = KvPasses();
}
void kv_passes_create(cm_ctx *ctx, const cm_kv *kv, int passes, KvPasses *kp) {
    const KsLevel &kl = ks_level(ctx, kv->level);
    // More giant steps (a bound of the area, 20 ciphertexts each) or digits than k_fan_passes keeps: the passes run one at a time.  32 x 128 at level 4:
    // sixteen giant steps 8787 us for eight passes, eight (taken together) 4938.
    if (passes < 2 || kv->r_o > 8 || kl.beta > 6) return;
    const size_t n = ctx->n, ctw = kv_ctw(kv), ln = ctw / 2, dblk = (size_t)kl.beta * kl.ext * n, ublk = 2 * (size_t)kl.ext * n;
    ks_batches_grow(ctx);
    kp->P = std::min(passes, CM_KS_BATCH), kp->r_i = kv->r_i, kp->r_o = kv->r_o, kp->level = kv->level;
    // a turn's relinearisations at once where their digits stay below 1 GB.  Eight passes over (16, 8) at level 4, 32, 16 and 8 in a batch: 5162, 5242 and
    // 5405 us, at level 3 3811, 3844 and 3953; ModDowns of the rotations by rows in batches of 32, 16 and 8: 5162, 5273 and 5389
    kp->D = std::max<int>(kp->P, (int)std::min<size_t>(std::min(kp->P * kv->r_o, CM_MASK_BATCH), ((size_t)1 << 30) / (dblk * 8)));
    kp->B = std::min(kp->D, ks_batch_max(ctx, kv->level)), kp->G = std::max(1, kp->D / kp->P);
    const size_t words = kp->P * (kv->r_i * ctw + kv->r_o * (3 * ln + ctw) + 2 * ublk) + kp->D * (ln + dblk);
    bool ok = hipMalloc((void **)&kp->babies, words * 8) == hipSuccess;
    if (ok) {
        kp->sums = kp->babies + kp->P * kv->r_i * ctw, kp->inner = kp->sums + kp->P * kv->r_o * 3 * ln, kp->ksin = kp->inner + kp->P * kv->r_o * ctw;
        kp->digits = kp->ksin + kp->D * ln, kp->acc = kp->digits + kp->D * dblk, kp->nxt = kp->acc + kp->P * ublk;
        ok = ks_many_tables_create(ctx, kv->level, kp->P, &kp->baby_tabs, 2 * kv->r_i, 1) == CM_OK &&
             ks_many_tables_create(ctx, kv->level, kp->B, &kp->relin_tabs, 3, 2) == CM_OK &&
             ks_many_tables_create(ctx, kv->level, kp->P * kp->G, &kp->giant_tabs, 2, 1) == CM_OK;
    }
    if (ok) return;
    (void)hipGetLastError();
    kv_passes_destroy(kp);
}
cm_status kv_passes_run(cm_ctx *ctx, const cm_evk *evk, const cm_kv *kv, const KvPasses &kp, const u64 *array, int m, u64 *const *outs, hipStream_t st) {
    const int lv = kv->level, limbs = lv + 1, r_i = kv->r_i, r_o = kv->r_o;
    const KsLevel &kl = ks_level(ctx, lv);
    const size_t n = ctx->n, ctw = kv_ctw(kv), ln = (size_t)limbs * n, dblk = (size_t)kl.beta * kl.ext * n, ublk = 2 * (size_t)kl.ext * n;
    const long long Ht = (long long)kv->H * kv->t;
    const u64 *relin = find_key(evk, 0);
    u64 *us = arena_batch_sums(ctx);
    // rotations by rows: keys in groups whose results one ModDown takes
    if (r_i > 1) {
        const bool apart = n == 65536;                 // the digits' own limbs are read where they are
        const u64 *first[CM_KS_BATCH];
        for (int p = 0; p < m; p++) first[p] = kp.babies + p * r_i * ctw;
        if (apart) CMCHK(ks_raise_apart(ctx, kp.baby_tabs, first, kp.ksin, kp.digits, st, m));
        else CMCHK(ks_raise_many(ctx, kp.baby_tabs, kp.babies, kp.ksin, kp.digits, st, m));
        const int most = std::max(1, std::min({ks_batch_max(ctx, lv) / m, PS_KEYS, CM_MASK_BATCH / m}));
        for (int j0 = 1; j0 < r_i; j0 += most) {
            FanPasses f;
            f.n = std::min(most, r_i - j0), f.per = n == 4096 ? 1 : 8;
            u64 gs[CM_MASK_BATCH], *to[CM_MASK_BATCH];
            const u64 *adds[CM_MASK_BATCH];
            for (int a = 0; a < PS_KEYS; a++) {
                const u64 g = rot_g(kv, (j0 + (a < f.n ? a : 0)) * Ht);
                f.key[a] = find_key(evk, g), f.ginv[a] = (unsigned)rot_g(kv, -(j0 + (a < f.n ? a : 0)) * Ht);
                for (int p = 0; p < m && a < f.n; p++)
                    gs[a * m + p] = g, adds[a * m + p] = kp.babies + p * r_i * ctw, to[a * m + p] = kp.babies + (p * r_i + j0 + a) * ctw;
            }
            launch_fan_passes(ctx, f, us, kp.digits, apart ? kp.babies + ln : nullptr, r_i * ctw, m, kl.beta, lv, st);
            CMCHK(moddown_batch_turned(ctx, us, lv, f.n * m, adds, 1, gs, to, st));
        }
    }
    // products with the cache: eight passes over 128 ciphertexts of five limbs in one launch 513 us, four at a time 595
    const int gs = array == kv->d_x ? 1 : r_i, ts = array == kv->d_x ? r_o : 1;
    for (int p = 0; p < m;) {
        u64 *sum = kp.sums + p * r_o * 3 * ln;
        const u64 *a = kp.babies + p * r_i * ctw;
        const int joint = m - p >= TS_WIDE ? TS_WIDE : m - p >= TS_PASSES ? TS_PASSES : m - p >= 2 ? 2 : 1;
        if (joint > 1 && tensor_sum_passes_fits(ctx, r_i, r_o, limbs, joint)) {
            launch_tensor_sum_passes(ctx, sum, r_o * 3 * ln, a, r_i * ctw, joint, array, r_i, r_o, limbs, st, gs, ts);
            p += joint;
        } else {
            launch_tensor_sum(ctx, sum, a, array, r_i, r_o, limbs, st, gs, ts);
            p++;
        }
    }
    // relinearisations; result g of pass p at inner[g][p]
    for (int i0 = 0; i0 < m * r_o; i0 += kp.B) {
        const int cnt = std::min(kp.B, m * r_o - i0);
        const u64 *T = kp.sums + i0 * 3 * ln;
        const bool half = rows_ip_fits(ctx, kl.beta, lv, cnt, 1);
        CMCHK(ks_raise_many(ctx, kp.relin_tabs, T, kp.ksin, kp.digits, st, cnt, 0, half));
        IpBatch ip;
        ip.nz = cnt, ip.nsum = 1;
        const u64 *adds[CM_MASK_BATCH];
        u64 *to[CM_MASK_BATCH];
        for (int r = 0; r < cnt; r++) {
            const int p = (i0 + r) / r_o, g = (i0 + r) % r_o;
            adds[r] = T + r * 3 * ln, to[r] = kp.inner + (g * m + p) * ctw;
            ip.it[r].dig = kp.digits + r * dblk, ip.it[r].key = relin, ip.it[r].own = adds[r] + 2 * ln, ip.out[r] = us + r * ublk;
        }
        if (half) launch_rows_ip(ctx, ip, kl.beta, lv, st, lv + 1);
        else if (n == 4096) launch_inner_product_batch(ctx, ip, kl.beta, lv, st);       // lanes that walk over 32 items do not fill the chip: 70 us, 12 apart
        else launch_inner_product_shared_key(ctx, ip, kl.beta, lv, st);
        CMCHK(moddown_batch_into(ctx, us, lv, cnt, adds, 2, 0, nullptr, to, st, half));
    }
    if (kv->unrolled) {
        // sum_g Rot(inner_g, g G) on the extended basis; inner_0 joins behind the ModDown (ModDown(u + P x) = ModDown(u) + x, word for word), or as P inner_0
        const bool joins = r_o > 1 && ks_drop_fits(ctx, lv, 1, m);
        u64 *cur = kp.acc, *nxt = kp.nxt;
        if (!joins) launch_raise_by_P(ctx, cur, kp.inner, lv, st, m);
        const int most = std::max(1, std::min(kp.G, IP_MAX_ITEMS / m));
        for (int g0 = 1; g0 < r_o; g0 += most) {
            const int cnt = std::min(most, r_o - g0);
            const bool half = rows_ip_fits(ctx, kl.beta, lv, m, cnt);
            const u64 *c = kp.inner + g0 * m * ctw;
            CMCHK(ks_raise_many(ctx, kp.giant_tabs, c, kp.ksin, kp.digits, st, cnt * m, 0, half));
            IpBatch b;
            b.nz = m, b.nsum = cnt;
            for (int p = 0; p < m; p++) {
                for (int s = 0; s < cnt; s++) {
                    const u64 gal = rot_g(kv, (long long)(g0 + s) * r_i * Ht);
                    IpItem &it = b.it[p * cnt + s];
                    it.dig = kp.digits + (s * m + p) * dblk, it.key = find_key(evk, gal), it.g = (unsigned)gal;
                    it.c0 = c + (s * m + p) * ctw, it.own = it.c0 + ln;
                }
                b.out[p] = nxt + p * ublk, b.extra[p] = joins && g0 == 1 ? nullptr : cur + p * ublk;
            }
            if (half) launch_rows_ip(ctx, b, kl.beta, lv, st);
            else launch_inner_product_batch(ctx, b, kl.beta, lv, st);
            std::swap(cur, nxt);
        }
        if (joins) return ks_drop(ctx, cur, lv, 1, m, kp.inner, ctw, 2, 0, nullptr, 0, nullptr, st, false, outs);
        if (ks_drop_fits(ctx, lv, 1, m)) return ks_drop(ctx, cur, lv, 1, m, nullptr, 0, 0, 0, nullptr, 0, nullptr, st, false, outs);
        for (int p = 0; p < m; p++) CMCHK(moddown_rescale_into(ctx, cur + p * ublk, lv, kp.inner, outs[p], st));
        return CM_OK;
    }
    // nested: inner_g + Rot(acc, G), written over inner_g
    const u64 gg = r_o > 1 ? rot_g(kv, r_i * Ht) : 0;
    const u64 *key = r_o > 1 ? find_key(evk, gg) : nullptr;
    for (int g = r_o - 2; g >= 0; g--) {
        const u64 *from = kp.inner + (g + 1) * m * ctw;
        const bool half = rows_ip_fits(ctx, kl.beta, lv, m, 1);
        CMCHK(ks_raise_many(ctx, kp.giant_tabs, from, kp.ksin, kp.digits, st, m, gg, half));
        IpBatch ip;
        ip.nz = m, ip.nsum = 1;
        const u64 *adds[CM_MASK_BATCH], *accs[CM_MASK_BATCH];
        u64 *to[CM_MASK_BATCH];
        for (int p = 0; p < m; p++) {
            adds[p] = from + p * ctw, to[p] = kp.inner + (g * m + p) * ctw, accs[p] = to[p];
            ip.it[p].dig = kp.digits + p * dblk, ip.it[p].key = key, ip.out[p] = us + p * ublk;
            ip.it[p].own = adds[p] + ln, ip.it[p].own_g = (unsigned)gg;
        }
        if (half) launch_rows_ip(ctx, ip, kl.beta, lv, st, lv + 1);
        else launch_inner_product_shared_key(ctx, ip, kl.beta, lv, st);
        CMCHK(moddown_batch_into(ctx, us, lv, m, adds, 1, gg, accs, to, st, half));
    }
    u64 *rescaled = kp.sums;
    CMCHK(rescale_into(ctx, kp.inner, 2 * m, lv, rescaled, st, kp.ksin, kp.babies));      // scratch [2 m][n] and [2 m][level][n]
    const u64 *src[CM_KS_BATCH];
    for (int p = 0; p < m; p++) src[p] = rescaled + p * 2 * (size_t)lv * n;
    launch_copies(outs, src, m, 2 * (size_t)lv * n, st);
    return CM_OK;
}
