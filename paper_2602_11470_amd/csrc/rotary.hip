// Rotary positions that are given with the call (cm_rotary_*), and the weighted rotations that they and the tree's passes are.
//
// The two dims of a pair sit `step` slots apart: one row of B = H t slots (neighbours) or rot_dims / 2 rows (halves).  With the positions of
// its residues the dims of a ciphertext turn by
//     y = p0 x + p_up Rot(x, step) + p_dn Rot(x, -step),   p0 = cos,  p_up = -sin in the rows of the first dims,  p_dn = sin in those of the
// second ones, ones in p0 where a head is not turned, zeros where a residue holds no token.  The plaintexts multiply BEHIND the
// rotations: both share one raise of x, and nothing leaves the extended basis before the one ModDown, which the rescale joins.
//
// The plaintexts of a position follow from tables without encoding anything: p = R h + l, and
//     cos(p theta) = cos(l theta) cos(h R theta) - sin(l theta) sin(h R theta)
// holds slot by slot, so it holds for plaintext polynomials, whose products are exact integers.  The low table stands at residue 0 with
// the scale q_level; slot rotations (exact permutations) put every token's entry at its residue; the entries of one h are summed
// and multiplied by the high table, which stands in all slots with the scale m2.  The products are formed under two moduli m1, m2 and
// divided by m2 to the nearest integer, which leaves coefficients at the scale q_level, within one unit of those of an encoding.
#include <math.h>

#include <algorithm>

#include "kernels.h"
#include "rotary.h"

#define ROT_TPB 256
#define ROT_AHEAD 4               // entries whose words are requested together
// Tokens up to which the products are formed inside the inverse transform's row pass (launch_rotary_inv), whose lanes each do four words of them: one
// token 8.5 us joined, 10.9 apart; eight 24 and 18.
#define ROT_JOINED 4
static bool rot_pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }

// v[set][part][2][n] (+)= the products of the tables' entries; limb blockIdx.y under modulus ma or mb.  A lane has one word of all parts, so an entry's four
// words are read once.  Bound by the gathers' latency, up to some ten entries by the launch: one token at n = 4096 3.6 us; at n = 65536 (4 MB an entry) a
// group of eight 12 us, 21 tokens of a tree 25 us.
__global__ __launch_bounds__(ROT_TPB) void k_rotary_products(u64 *__restrict__ v, RotBatch b, int count, const u64 *__restrict__ low,
                                                             const u64 *__restrict__ still, const u64 *__restrict__ high, const ModC *__restrict__ modc,
                                                             int ma, int mb, int parts, int n, int logn, int accumulate) {
    const unsigned i = blockIdx.x * ROT_TPB + threadIdx.x;
    const int limb = blockIdx.y, set = blockIdx.z;
    const ModC m = modc[limb ? mb : ma];
    const size_t poly = 2 * (size_t)n, at = (size_t)limb * n;
    u64 here = 0, up = 0, dn = 0, c1 = 0, c2 = 0, s1 = 0, s2 = 0, st = 0;
    u64 *out = v + (size_t)set * parts * poly + at + i;
    if (accumulate) {
        here = out[0], up = out[poly];
        if (parts == 3) dn = out[2 * poly];
    }
    auto mul = [&](u64 x, u64 y) { return redc((u128)x * y, m.q, m.qinv); };
    for (int k0 = 0; k0 < count; k0 += ROT_AHEAD) {
        u64 w[ROT_AHEAD][5], h[ROT_AHEAD][2];
        auto ends = [&](int k) { return k + 1 >= count || b.e[k + 1].high != b.e[k].high; };
#pragma unroll
        for (int a = 0; a < ROT_AHEAD; a++) {
            const RotEntry e = b.e[k0 + a];
            if (k0 + a >= count) continue;
            const unsigned src = perm_src(i, e.g, logn);
            const u64 *p = low + (size_t)e.low * 4 * poly + at + src, *t = high + (size_t)e.high * 2 * poly + at + i;
#pragma unroll
            for (int q = 0; q < 4; q++) w[a][q] = p[q * poly];
            w[a][4] = still ? still[at + src] : 0;
            if (ends(k0 + a)) h[a][0] = t[0], h[a][1] = t[poly];
        }
#pragma unroll
        for (int a = 0; a < ROT_AHEAD; a++) {
            if (k0 + a >= count) continue;
            if (b.e[k0 + a].sets >> set & 1u)
                c1 = addmod(c1, w[a][0], m.q), c2 = addmod(c2, w[a][1], m.q), s1 = addmod(s1, w[a][2], m.q), s2 = addmod(s2, w[a][3], m.q), st = addmod(st, w[a][4], m.q);
            if (!ends(k0 + a)) continue;
            const u64 c = h[a][0], s = h[a][1];
            here = addmod(here, submod(mul(addmod(addmod(c1, c2, m.q), st, m.q), c), mul(addmod(s1, s2, m.q), s), m.q), m.q);
            up = submod(up, addmod(mul(s1, c), mul(c1, s), m.q), m.q);
            const u64 d = addmod(mul(s2, c), mul(c2, s), m.q);
            if (parts == 3) dn = addmod(dn, d, m.q);
            else up = addmod(up, d, m.q);
            c1 = c2 = s1 = s2 = st = 0;
        }
    }
    out[0] = here, out[poly] = up;
    if (parts == 3) out[2 * poly] = dn;
}
// out[z][limbs][n] = the second components of b.c[z]
__global__ __launch_bounds__(ROT_TPB) void k_second(u64 *__restrict__ out, SecondBatch b, int limbs, int n) {
    const size_t i = blockIdx.x * ROT_TPB + threadIdx.x, at = (size_t)blockIdx.y * n + i;
    out[(size_t)blockIdx.z * limbs * n + at] = b.c[blockIdx.z][(size_t)limbs * n + at];
}

// ---- weighted rotations -----------------------------------------------------------------------------------------------
// A lane has W neighbouring words of an output and runs over its items: the item's digits through the Galois map, its key's
// words, the sums reduced and multiplied by the item's plaintext.  All loads of an item are requested before the first is used (NB bounds its
// digits), keys and plaintexts past the caches; one word a lane at n = 4096, where a launch is as long as a lane's chain (two items, one digit 5.7 -> 4.7 us, four digits 9.5 -> 6.3).
// At n = 65536 bound by HBM and by drawing the keys' uniform halves: 14 items of two digits into seven outputs of ten limbs 77 us (0.3 GB: keys 147 MB,
// plaintexts and outputs 73 MB each; 3.9 TB/s), two ciphertexts at level 3 20 us.  Rotating first, each to its ModDown, and multiplying then would write and
// read every rotation and end in as many ModDowns.
// SPLIT waves share the items of 64 W words and join their sums in LDS (sums of more than two items at n = 4096, whose launch does not fill the
// chip: 14 items of four digits 24.9 -> 10.1 us).  Z: outputs of a lane, whose items have the same keys.
template <bool SA, int NB, int W, int SPLIT, int Z, bool WIDE>
__global__ __launch_bounds__(ROT_TPB) void k_weighted(WrBatch b, const ModC *__restrict__ modc, int beta, int ext, int level, int alpha, int L, int nmod, int n,
                                                      int logn, const u64 *__restrict__ pmont, EvkA eva, const u64 *__restrict__ ubound) {
    typedef u64 words __attribute__((ext_vector_type(W)));
    const int part = threadIdx.x / (ROT_TPB / SPLIT);
    const unsigned i0 = (blockIdx.x * (ROT_TPB / SPLIT) + threadIdx.x % (ROT_TPB / SPLIT)) * W;
    const int r = blockIdx.y, z0 = blockIdx.z * Z, mi = r <= level ? r : L + 1 + (r - level - 1);
    const ModC m = modc[mi];
    const size_t o = (size_t)r * n + i0;
    const u64 bound = ubound[mi], pm = r <= level ? pmont[r] : 0;
    const int own = r <= level ? r / alpha : -1;
    u64 r0[Z][W] = {}, r1[Z][W] = {};
    auto mul = [&](u64 x, u64 y) { return redc((u128)x * y, m.q, m.qinv); };
    auto load = [](const u64 *p) { return *reinterpret_cast<const words *>(p); };
#pragma unroll
    for (int zz = 0; zz < Z; zz++) {
        const int z = z0 + zz;
        if (part == 0 && b.extra[z]) {
            const words x = load(b.extra[z] + o), y = load(b.extra[z] + (size_t)ext * n + o);
#pragma unroll
            for (int k = 0; k < W; k++) r0[zz][k] = x[k], r1[zz][k] = y[k];
        }
        if (part == 0 && b.here[z] && r <= level) {
            const words w = load(b.here[z] + o), x = load(b.c_here[z] + o), y = load(b.c_here[z] + (size_t)(level + 1) * n + o);
#pragma unroll
            for (int k = 0; k < W; k++) {
                const u64 wp = mul(w[k], pm);
                r0[zz][k] = addmod(r0[zz][k], mul(x[k], wp), m.q), r1[zz][k] = addmod(r1[zz][k], mul(y[k], wp), m.q);
            }
        }
    }
    for (int s = part; s < b.nsum; s += SPLIT) {
        WrItem its[Z];                                           // of the same key and Galois map
#pragma unroll
        for (int zz = 0; zz < Z; zz++) its[zz] = b.it[(z0 + zz) * b.nsum + s];
        const WrItem &first = its[0];
        const unsigned src = perm_src(i0, first.g, logn), base = src & ~(unsigned)(W - 1), flip = src & (W - 1);      // word k is word k ^ flip of the pair
        words d[Z][NB], e[NB], c[Z], w[Z];
        u64 sk[NB];
#pragma unroll
        for (int j = 0; j < NB; j++)
            if (j < beta) {
                const size_t at = ((size_t)j * nmod + mi) * n + i0;
#pragma unroll
                for (int zz = 0; zz < Z; zz++)
                    d[zz][j] = load((j == own ? its[zz].c + (size_t)(level + 1 + r) * n : its[zz].dig + ((size_t)j * ext + r) * n) + base);
                e[j] = __builtin_nontemporal_load(reinterpret_cast<const words *>(first.key + at));
                if (!SA) sk[j] = first.key[(size_t)eva.kdig * nmod * n + (size_t)j * nmod + mi];
            }
#pragma unroll
        for (int zz = 0; zz < Z; zz++) {
            if (r <= level) c[zz] = load(its[zz].c + (size_t)r * n + base);
            w[zz] = __builtin_nontemporal_load(reinterpret_cast<const words *>(its[zz].pt + o));
        }
#pragma unroll
        for (int k = 0; k < W; k++) {
            u128 sa[Z] = {}, sb[Z] = {};
            const u64 cg = ((u64)i0 + k + 1) * GOLD;
#pragma unroll
            for (int j = 0; j < NB; j++)
                if (j < beta) {
                    const u64 a = SA ? __builtin_nontemporal_load(first.key + eva.a_off + ((size_t)j * nmod + mi) * n + i0 + k) : evk_a_draw(sk[j], cg, i0 + k, bound);
#pragma unroll
                    for (int zz = 0; zz < Z; zz++) {
                        const u64 x = W == 1 ? d[zz][j][0] : flip ? d[zz][j][W - 1 - k] : d[zz][j][k];
                        sb[zz] += (u128)x * e[j][k], sa[zz] += (u128)x * a;
                        if (WIDE && (j & 3) == 3) less_of_sum<false>(sb[zz], m.q), less_of_sum<!SA>(sa[zz], m.q);
                    }
                }
#pragma unroll
            for (int zz = 0; zz < Z; zz++) {
                if (r <= level) sb[zz] += (u128)(W == 1 ? c[zz][0] : flip ? c[zz][W - 1 - k] : c[zz][k]) * pm;
                if (WIDE) less_of_sum<false>(sb[zz], m.q);
                if (WIDE && SA) less_of_sum<false>(sa[zz], m.q);
                r0[zz][k] = addmod(r0[zz][k], mul(redc(sb[zz], m.q, m.qinv), w[zz][k]), m.q);
                r1[zz][k] = addmod(r1[zz][k], mul(evk_a_reduce<SA>(sa[zz], m), w[zz][k]), m.q);
            }
        }
    }
    if (SPLIT > 1) {
        __shared__ u64 sums[SPLIT][2 * W * Z][ROT_TPB / SPLIT];
        const int lane = threadIdx.x % (ROT_TPB / SPLIT);
#pragma unroll
        for (int k = 0; k < W * Z; k++) sums[part][k][lane] = r0[k / W][k % W], sums[part][W * Z + k][lane] = r1[k / W][k % W];
        __syncthreads();
        if (part) return;
#pragma unroll
        for (int q = 1; q < SPLIT; q++)
#pragma unroll
            for (int k = 0; k < W * Z; k++)
                r0[k / W][k % W] = addmod(r0[k / W][k % W], sums[q][k][lane], m.q), r1[k / W][k % W] = addmod(r1[k / W][k % W], sums[q][W * Z + k][lane], m.q);
    }
#pragma unroll
    for (int zz = 0; zz < Z; zz++) {
        words x, y;
#pragma unroll
        for (int k = 0; k < W; k++) x[k] = r0[zz][k], y[k] = r1[zz][k];
        *reinterpret_cast<words *>(b.out[z0 + zz] + o) = x;
        *reinterpret_cast<words *>(b.out[z0 + zz] + (size_t)ext * n + o) = y;
    }
}
template <int W, int SPLIT = 1, int Z = 1>
static void launch_weighted_words(cm_ctx *ctx, const WrBatch &b, int beta, int level, hipStream_t st) {
    const int ext = level + 1 + ctx->K;
    const dim3 grid(ctx->n * SPLIT / (W * ROT_TPB), ext, b.nz / Z);
#define WEIGHTED(SA_, NB_, WIDE_)                                                                                                                              \
    hipLaunchKernelGGL((k_weighted<SA_, NB_, W, SPLIT, Z, WIDE_>), grid, dim3(ROT_TPB), 0, st, b, ctx->d_modc, beta, ext, level, ctx->alpha, ctx->L, ctx->nmod, ctx->n, ctx->logn, \
                       ctx->d_pmont, evk_a_of(ctx), ctx->d_ubound)
    const bool sa = ctx->evk_stored_a;
    if (beta <= 1 && !sa) WEIGHTED(false, 1, false);
    else if (beta <= 2 && !sa) WEIGHTED(false, 2, false);
    else if (beta <= 4) {
        if (sa) WEIGHTED(true, 4, false);
        else WEIGHTED(false, 4, false);
    } else if constexpr (Z == 1) {
        if (beta > ctx->lazy_terms) {
            if (sa) WEIGHTED(true, CM_MAX_DIGITS, true);
            else WEIGHTED(false, CM_MAX_DIGITS, true);
        } else if (sa) WEIGHTED(true, CM_MAX_DIGITS, false);
        else if (beta <= 6) WEIGHTED(false, 6, false);
        else WEIGHTED(false, CM_MAX_DIGITS, false);
    }
#undef WEIGHTED
}
void launch_weighted(cm_ctx *ctx, const WrBatch &b, int beta, int level, hipStream_t st) {
    Prof prof_(ctx, CM_K_INNER_PRODUCT, b.nz * b.nsum, st);
    // Outputs of the same keys, two a lane: a key's words are read and drawn once for both.  Four ciphertexts turned at level 12 (four digits) 398 -> 381 us, two
    // 215 -> 208, at levels 3 and 7 1 % less; with six digits (176 registers) 426 -> 435.
    bool pairs = ctx->n == 65536 && b.nz % 2 == 0 && beta <= 4;
    for (int i = 0; i < b.nz * b.nsum && pairs; i++) pairs = b.it[i].key == b.it[i % b.nsum].key;
    if (ctx->n == 4096 && b.nsum > 2) launch_weighted_words<1, 4>(ctx, b, beta, level, st);
    else if (ctx->n == 4096) launch_weighted_words<1>(ctx, b, beta, level, st);
    else if (pairs) launch_weighted_words<2, 1, 2>(ctx, b, beta, level, st);
    else launch_weighted_words<2>(ctx, b, beta, level, st);
}
// The row pass of the digits inside the weighted sums (launch_rows_weighted) repeats it for every item: the faster form with one item an output.  Two
// ciphertexts at level 22, one rotation each: raise, sums and row passes 242 -> 218 us; with two rotations at level 12 143 -> 159, at level 3 39 -> 43.
bool weighted_rows(cm_ctx *ctx, int beta, int level, int nsum, int m) {
    return ctx->n == 65536 && !ctx->evk_stored_a && beta <= 7 && nsum == 1 && ks_drop_fits(ctx, level, 1, m);
}
cm_status weighted_down(cm_ctx *ctx, u64 *us, int level, int m, u64 *const *outs, u64 *tmp, hipStream_t st, bool rows_done, bool onto) {
    if (ks_drop_fits(ctx, level, 1, m)) return ks_drop(ctx, us, level, 1, m, nullptr, 0, 0, 0, nullptr, 0, nullptr, st, rows_done, outs, onto);
    const size_t ublk = 2 * (size_t)(level + 1 + ctx->K) * ctx->n;
    for (int z = 0; z < m; z++) {
        // tmp holds what the first step leaves and, onto, the result behind it
        u64 *to = onto ? tmp + 2 * (size_t)(level + 1) * ctx->n : outs[z];
        CMCHK(moddown_rescale_into(ctx, us + z * ublk, level, tmp, to, st));
        if (onto) launch_add(ctx, outs[z], outs[z], to, 2, level, st);
    }
    return CM_OK;
}

// ---- the tables ---------------------------------------------------------------------------------------------------------
extern "C" void cm_rotary_destroy(cm_rotary *r) {
    if (!r) return;
    ks_many_tables_destroy(&r->tabs);
    hipFree(r->d_low), hipFree(r->d_still), hipFree(r->d_high), hipFree(r->d_v), hipFree(r->d_p), hipFree(r->d_work), hipFree(r->d_mods), hipFree(r->d_ext_mods);
    delete r;
}
static void rotary_sizes(int room, int *low, int *high) {
    int bits = 0;
    while ((1LL << bits) < room) bits++;
    *low = 1 << ((bits + 1) / 2), *high = (room + *low - 1) / *low;
}
extern "C" int32_t cm_rotary_polys(int32_t room) {
    if (room < 1 || room > CM_ROTARY_ROOM) return 0;
    int low, high;
    rotary_sizes(room, &low, &high);
    return 4 * low + 1 + 2 * high;
}
extern "C" cm_status cm_rotary_freqs(int32_t rot_dims, double base, int32_t scaling, const double *par, double *out) {
    if (rot_dims < 2 || rot_dims % 2 || !(base > 1.0) || !isfinite(base) || !out) return CM_E_INVAL;
    if (scaling < CM_ROTARY_PLAIN || scaling > CM_ROTARY_BANDS || (scaling != CM_ROTARY_PLAIN && (!par || !(par[0] > 0) || !isfinite(par[0])))) return CM_E_INVAL;
    if (scaling == CM_ROTARY_BANDS && !(par[1] < par[2] && par[3] > 0 && isfinite(par[1]) && isfinite(par[2]) && isfinite(par[3]))) return CM_E_INVAL;
    if (scaling == CM_ROTARY_BASE && rot_dims > 2) base *= pow(par[0], (double)rot_dims / (rot_dims - 2));
    for (int m = 0; m < rot_dims / 2; m++) {
        double f = pow(base, -2.0 * m / rot_dims);
        if (scaling == CM_ROTARY_LINEAR) f /= par[0];
        if (scaling == CM_ROTARY_BANDS) {
            const double keep = fmin(1.0, fmax(0.0, (par[3] * f / (2 * M_PI) - par[1]) / (par[2] - par[1])));
            f = keep * f + (1 - keep) * f / par[0];
        }
        if (!isfinite(f)) return CM_E_INVAL;          // a factor too small for the base or the frequencies
        out[m] = f;
    }
    return CM_OK;
}
extern "C" cm_status cm_rotary_create(cm_ctx *ctx, int32_t heads, int32_t dim, int32_t level, int32_t rot_dims, const double *freq, double gain, int32_t room,
                                      uint32_t flags, const int64_t *coeffs, cm_rotary **out) {
    (void)hipGetLastError();          // stale errors of earlier calls are not this call's
    if (!ctx || !out || heads < 1 || dim < 2 || rot_dims < 2 || rot_dims % 2 || room < 1 || room > CM_ROTARY_ROOM || (flags & ~(uint32_t)CM_ROTARY_HALVES)) return CM_E_INVAL;
    if (level < 1 || level > ctx->L) return CM_E_LEVEL;
    const int S = ctx->n / 2;
    if (heads > S || dim > S || rot_dims > dim) return CM_E_LAYOUT;
    while (!rot_pow2(heads)) heads++;          // a head count that is not a power of two is padded to the next one
    if (!rot_pow2(dim) || (long long)heads * dim > S) return CM_E_LAYOUT;
    for (int m = 0; freq && m < rot_dims / 2; m++) if (!(fabs(freq[m]) * room < 0x1p53)) return CM_E_INVAL;
    // the plaintexts' coefficients are at most gain q_level in size: below half of the first special modulus, which they are rounded under, and
    // below the signed words of the encoding
    const double q = (double)ctx->mod[level], top = fmax(gain, 1.0) * q;
    if (!(gain > 0) || !isfinite(gain) || !(top < 0.49 * (double)ctx->mod[ctx->L + 1]) || !(top < 0x1p61)) return CM_E_INVAL;
    cm_rotary *r = new (std::nothrow) cm_rotary();
    if (!r) return CM_E_NOMEM;
    cm_status status = CM_OK;
    long long *d_coeffs = nullptr;
    try {
        r->ctx = ctx, r->H = heads, r->E = dim, r->t = S / (heads * dim), r->level = level, r->room = room;
        rotary_sizes(room, &r->low, &r->high);
        const bool halves = flags & CM_ROTARY_HALVES;
        r->step = (halves ? rot_dims / 2 : 1) * heads * r->t, r->parts = 2 * r->step == S ? 2 : 3;
        r->ma = ctx->L + 1, r->mb = ctx->K > 1 ? ctx->L + 2 : 0;
        const u64 m1 = ctx->mod[r->ma], m2 = ctx->mod[r->mb];
        r->inv = h_mulmod(h_invmod(m2 % m1, m1), (u64)(((u128)1 << 64) % m1), m1);
        const KsLevel &kl = ks_level(ctx, level);
        const size_t n = ctx->n, ln = (size_t)(level + 1) * n, dblk = (size_t)kl.beta * kl.ext * n;
        r->batch = (int)std::max<size_t>(1, std::min<size_t>(CM_KS_BATCH, (256u << 20) / (dblk * 8)));
        const size_t polys = (size_t)4 * r->low, chunk = 64;
        auto get = [&](u64 **p, size_t words) {
            if (status == CM_OK && hipMalloc((void **)p, words * 8) != hipSuccess) status = CM_E_NOMEM;
        };
        get(&r->d_low, polys * 2 * n), get(&r->d_high, (size_t)r->high * 4 * n);
        if (rot_dims < dim) get(&r->d_still, 2 * n);
        get(&r->d_v, (size_t)ROT_SETS * r->parts * 2 * n), get(&r->d_p, (size_t)ROT_SETS * r->parts * kl.ext * n);
        get(&r->d_work, 4 * ln + r->batch * (2 * ln + dblk));
        get((u64 **)&d_coeffs, chunk * n);
        std::vector<int> mods, ext_mods;
        for (size_t i = 0; i < chunk; i++) mods.push_back(r->ma), mods.push_back(r->mb);
        for (int i = 0; i < ROT_SETS * r->parts; i++)
            for (int l = 0; l < kl.ext; l++) ext_mods.push_back(l <= level ? l : ctx->L + l - level);
        if (status == CM_OK && (hipMalloc((void **)&r->d_mods, mods.size() * 4) != hipSuccess || hipMalloc((void **)&r->d_ext_mods, ext_mods.size() * 4) != hipSuccess)) status = CM_E_NOMEM;
        if (status == CM_OK && (hipMemcpy(r->d_mods, mods.data(), mods.size() * 4, hipMemcpyHostToDevice) != hipSuccess ||
                                hipMemcpy(r->d_ext_mods, ext_mods.data(), ext_mods.size() * 4, hipMemcpyHostToDevice) != hipSuccess)) status = CM_E_HIP;
        if (status == CM_OK) status = ks_many_tables_create(ctx, level, r->batch, &r->tabs, 1, 0);
        // the tables, a chunk of polynomials at a time: coefficients (given or encoded), residues under the two moduli, transforms
        std::vector<double> slots, theta(dim, 0.0);
        std::vector<int> cls(dim, 0);                       // 1, 2: first and second dims of the pairs; 0: not turned
        for (int e = 0; e < rot_dims; e++) {
            const int m = halves ? e % (rot_dims / 2) : e / 2;
            theta[e] = freq ? freq[m] : pow(10000.0, -2.0 * m / rot_dims);
            cls[e] = (halves ? e < rot_dims / 2 : e % 2 == 0) ? 1 : 2;
        }
        std::vector<int64_t> host;
        auto table = [&](u64 *dst, size_t count, size_t first, double scale, bool mont, auto value) {
            for (size_t k0 = 0; k0 < count && status == CM_OK; k0 += chunk) {
                const size_t m = std::min(chunk, count - k0);
                const int64_t *src = coeffs ? coeffs + (first + k0) * n : nullptr;
                if (!coeffs) {
                    host.assign(m * n, 0);
                    for (size_t k = 0; k < m && status == CM_OK; k++) {
                        slots.assign(S, 0.0);
                        for (int e = 0; e < dim; e++)
                            for (int i = 0; i < heads * r->t; i++)
                                if (mont || i % r->t == 0) slots[(size_t)e * heads * r->t + i] = value(k0 + k, e);
                        status = cm_encode_coeffs(ctx, slots.data(), nullptr, S, scale, host.data() + k * n);
                    }
                    src = host.data();
                }
                if (status != CM_OK) break;
                if (hipMemcpy(d_coeffs, src, m * n * 8, hipMemcpyHostToDevice) != hipSuccess) { status = CM_E_HIP; break; }
                u64 *at = dst + k0 * 2 * n;
                for (size_t k = 0; k < m; k++) launch_reduce_i64(ctx, at + k * 2 * n, d_coeffs + k * n, r->d_mods, 2, 0);
                launch_ntt(ctx, at, r->d_mods, 2 * (int)m, false, 0);
                if (mont) launch_to_mont(ctx, at, r->d_mods, 2 * (int)m, 0);
                if (hipDeviceSynchronize() != hipSuccess || hipGetLastError() != hipSuccess) status = CM_E_HIP;
            }
        };
        if (status == CM_OK && hipDeviceSynchronize() != hipSuccess) status = CM_E_HIP;
        table(r->d_low, polys, 0, q, false, [&](size_t k, int e) {
            const long double a = (long double)(k / 4) * theta[e];
            return cls[e] != (int)(k % 2) + 1 ? 0.0 : gain * (double)(k % 4 < 2 ? cosl(a) : sinl(a));
        });
        if (r->d_still) table(r->d_still, 1, polys, q, false, [&](size_t, int e) { return cls[e] ? 0.0 : 1.0; });
        table(r->d_high, 2 * (size_t)r->high, polys + 1, (double)m2, true, [&](size_t k, int e) {
            const long double a = (long double)(k / 2) * r->low * (long double)theta[e];
            return (double)(k % 2 ? sinl(a) : cosl(a));
        });
        r->pos.assign(r->t, -1);
    } catch (...) {
        status = CM_E_NOMEM;
    }
    hipFree(d_coeffs);
    if (status != CM_OK) {
        cm_rotary_destroy(r);
        return status;
    }
    *out = r;
    return CM_OK;
}
extern "C" int32_t cm_rotary_steps(const cm_rotary *r, int32_t *steps, int32_t cap) {
    if (!r) return 0;
    const int s[2] = {r->step, -r->step};
    for (int i = 0; i < r->parts - 1 && i < cap && steps; i++) steps[i] = s[i];
    return r->parts - 1;
}
extern "C" cm_status cm_rotary_set(cm_ctx *ctx, cm_rotary *r, const int32_t *pos, int32_t split, void *stream) {
    (void)hipGetLastError();          // stale errors of earlier calls are not this call's
    if (!ctx || !r || r->ctx != ctx || !pos) return CM_E_INVAL;
    if (split < 0 || split >= r->t) return CM_E_LAYOUT;
    for (int i = 0; i < r->t; i++) if (pos[i] < -1 || pos[i] >= r->room) return CM_E_LAYOUT;
    CM_TRY
    hipStream_t st = (hipStream_t)stream;
    const int n = ctx->n, sets = split ? ROT_SETS : 1;
    std::vector<RotEntry> entries;
    for (int i = 0; i < r->t; i++)
        if (pos[i] >= 0)
            entries.push_back({(unsigned short)(pos[i] % r->low), (unsigned short)(pos[i] / r->low), (unsigned)galois_of_step(ctx, -i),
                               1u | (i >= split ? 2u : 4u)});
    std::sort(entries.begin(), entries.end(), [](const RotEntry &a, const RotEntry &b) { return a.high < b.high; });
    std::vector<int32_t> kept(pos, pos + r->t);
    r->set = false;                     // until everything has been enqueued: a call that fails leaves no positions
    auto batch = [&](size_t k0, int m) {
        RotBatch b;
        for (int k = 0; k < ROT_ENTRIES; k++) b.e[k] = k < m ? entries[k0 + k] : RotEntry{0, 0, 1, 0};
        return b;
    };
    if (n == 65536 && entries.size() <= ROT_JOINED) {
        launch_rotary_inv(ctx, r->d_v, batch(0, (int)entries.size()), (int)entries.size(), r->d_low, r->d_still, r->d_high, r->ma, r->mb, r->parts, sets, r->d_mods, st);
    } else {
        for (size_t k0 = 0; k0 == 0 || k0 < entries.size(); k0 += ROT_ENTRIES) {
            const int m = (int)std::min<size_t>(ROT_ENTRIES, entries.size() - k0);
            Prof prof_(ctx, CM_K_ELEMENTWISE, sets * r->parts * 2, st);
            hipLaunchKernelGGL(k_rotary_products, dim3(n / ROT_TPB, 2, sets), dim3(ROT_TPB), 0, st, r->d_v, batch(k0, m), m, r->d_low, r->d_still, r->d_high,
                               ctx->d_modc, r->ma, r->mb, r->parts, n, ctx->logn, k0 > 0);
        }
        launch_ntt(ctx, r->d_v, r->d_mods, sets * r->parts * 2, true, st);
    }
    launch_rotary_fwd(ctx, r->d_p, r->d_v, r->ma, r->mb, r->inv, r->level, sets * r->parts, r->d_ext_mods, st);
    auto enqueued = [] { RETURN_LAUNCH_STATUS(); };
    CMCHK(enqueued());
    r->pos.swap(kept), r->split = split, r->set = true;
    return CM_OK;
    CM_CATCH
}
cm_status rotary_sums(cm_ctx *ctx, const cm_evk *evk, const cm_rotary *r, int m, const u64 *const *xs, int first, int sets, u64 *us, bool *rows_done,
                      hipStream_t st) {
    const int level = r->level;
    const KsLevel &kl = ks_level(ctx, level);
    const size_t n = ctx->n, ln = (size_t)(level + 1) * n, dblk = (size_t)kl.beta * kl.ext * n, ublk = 2 * (size_t)kl.ext * n;
    u64 *second = r->d_work + 4 * ln, *ksin = second + r->batch * ln, *digits = ksin + r->batch * ln;
    const u64 *keys[2];
    unsigned g[2];
    for (int s = 0; s < r->parts - 1; s++) {
        g[s] = (unsigned)galois_of_step(ctx, s ? -r->step : r->step), keys[s] = find_key(evk, g[s]);
        if (!keys[s]) return CM_E_NOKEY;
    }
    const bool half = weighted_rows(ctx, kl.beta, level, r->parts - 1, m * sets);
    if (n == 65536) {
        CMCHK(ks_raise_apart(ctx, r->tabs, xs, ksin, digits, st, m, half));
    } else {
        const u64 *d = xs[0] + ln;
        if (m > 1) {
            SecondBatch b;
            for (int z = 0; z < CM_KS_BATCH; z++) b.c[z] = xs[z < m ? z : 0];
            hipLaunchKernelGGL(k_second, dim3(n / ROT_TPB, level + 1, m), dim3(ROT_TPB), 0, st, second, b, level + 1, (int)n);
            d = second;
        }
        CMCHK(ks_raise_many(ctx, r->tabs, d, ksin, digits, st, m));
    }
    *rows_done = half;
    WrBatch b;
    b.nz = m * sets, b.nsum = r->parts - 1;
    for (int z = 0; z < m; z++)
        for (int k = 0; k < sets; k++) {
            const int o = z * sets + k;
            const u64 *p = r->d_p + (size_t)(first + k) * r->parts * kl.ext * n;
            b.here[o] = p, b.c_here[o] = xs[z], b.out[o] = us + o * ublk;
            for (int s = 0; s < b.nsum; s++) {
                WrItem &it = b.it[o * b.nsum + s];
                it.dig = digits + z * dblk, it.c = xs[z], it.key = keys[s], it.g = g[s], it.pt = p + (size_t)(1 + s) * kl.ext * n;
            }
        }
    if (half) launch_rows_weighted(ctx, b, kl.beta, level, st, level);
    else launch_weighted(ctx, b, kl.beta, level, st);
    return CM_OK;
}
extern "C" cm_status cm_rotary_apply(cm_ctx *ctx, const cm_evk *evk, const cm_rotary *r, int32_t count, const cm_ct *x, cm_ct *y, void *stream) {
    (void)hipGetLastError();          // stale errors of earlier calls are not this call's
    if (!ctx || !evk || !r || r->ctx != ctx || !x || !y || count < 1 || count > CM_ROTARY_MAX || !evk_fits(ctx, evk)) return CM_E_INVAL;
    const size_t n = ctx->n, in = 2 * (size_t)(r->level + 1) * n, res = 2 * (size_t)r->level * n;
    for (int i = 0; i < count; i++) {
        if (!x[i].dev || !y[i].dev || x[i].ncomp != 2) return CM_E_INVAL;
        if (x[i].level != r->level) return CM_E_LEVEL;
        for (int j = 0; j < count; j++)
            if (words_meet(y[i].dev, res, x[j].dev, in) || (j < i && words_meet(y[i].dev, res, y[j].dev, res))) return CM_E_INVAL;
    }
    if (!r->set) return CM_E_LAYOUT;
    for (int s = 0; s < r->parts - 1; s++) if (!find_key(evk, galois_of_step(ctx, s ? -r->step : r->step))) return CM_E_NOKEY;
    CM_TRY
    hipStream_t st = (hipStream_t)stream;
    u64 *us = arena_batch_sums(ctx);
    for (int i0 = 0; i0 < count; i0 += r->batch) {
        const int m = std::min(r->batch, count - i0);
        const u64 *xs[CM_KS_BATCH];
        u64 *outs[CM_KS_BATCH];
        for (int z = 0; z < m; z++) xs[z] = x[i0 + z].dev, outs[z] = y[i0 + z].dev;
        bool rows;
        CMCHK(rotary_sums(ctx, evk, r, m, xs, 0, 1, us, &rows, st));
        CMCHK(weighted_down(ctx, us, r->level, m, outs, r->d_work, st, rows));
    }
    for (int i = 0; i < count; i++) y[i].level = r->level - 1, y[i].ncomp = 2, y[i].scale = x[i].scale;      // plaintext scale = the prime just removed
    RETURN_LAUNCH_STATUS();
    CM_CATCH
}
