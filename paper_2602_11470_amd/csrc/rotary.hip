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

#define ROT_ENTRIES 64
#define ROT_TPB 256
struct RotEntry {
    unsigned short low, high;
    unsigned g, sets;              // Galois element that takes residue 0 to the token's; the sets (bits) it belongs to
};
struct RotBatch {
    RotEntry e[ROT_ENTRIES];       // in the order of their high parts
};
static bool rot_pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }

// v[set][part][2][n] (+)= the products of the tables' entries; limb blockIdx.y under modulus ma or mb
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
    for (int k = 0; k < count; k++) {
        const RotEntry e = b.e[k];
        if (e.sets >> set & 1u) {
            const u64 *p = low + (size_t)e.low * 4 * poly + at + perm_src(i, e.g, logn);
            c1 = addmod(c1, p[0], m.q), c2 = addmod(c2, p[poly], m.q), s1 = addmod(s1, p[2 * poly], m.q), s2 = addmod(s2, p[3 * poly], m.q);
            if (still) st = addmod(st, still[at + perm_src(i, e.g, logn)], m.q);
        }
        if (k + 1 < count && b.e[k + 1].high == e.high) continue;
        const u64 c = high[(size_t)e.high * 2 * poly + at + i], s = high[((size_t)e.high * 2 + 1) * poly + at + i];
        auto mul = [&](u64 x, u64 y) { return redc((u128)x * y, m.q, m.qinv); };
        here = addmod(here, submod(mul(addmod(addmod(c1, c2, m.q), st, m.q), c), mul(addmod(s1, s2, m.q), s), m.q), m.q);
        up = submod(up, addmod(mul(s1, c), mul(c1, s), m.q), m.q);
        const u64 d = addmod(mul(s2, c), mul(c2, s), m.q);
        if (parts == 3) dn = addmod(dn, d, m.q);
        else up = addmod(up, d, m.q);
        c1 = c2 = s1 = s2 = st = 0;
    }
    out[0] = here, out[poly] = up;
    if (parts == 3) out[2 * poly] = dn;
}
// p[poly][ext][n] = round(v / m2) as residues in multiplier form: v[poly][2][n] in coefficients under m1 and m2; inv: m2^-1 mod m1 in
// multiplier form
__global__ __launch_bounds__(ROT_TPB) void k_rotary_round(u64 *__restrict__ p, const u64 *__restrict__ v, const ModC *__restrict__ modc, int ma, int mb,
                                                          u64 inv, int level, int L, int ext, int n) {
    const size_t i = blockIdx.x * ROT_TPB + threadIdx.x;
    const ModC m1 = modc[ma];
    const u64 m2 = modc[mb].q, a = v[(size_t)blockIdx.y * 2 * n + i], b = v[((size_t)blockIdx.y * 2 + 1) * n + i];
    const bool above = b > m2 / 2;                         // the residue under m2 nearest to zero: b or b - m2
    const u64 r = (above ? m2 - b : b) % m1.q;
    const u64 w = redc((u128)(above ? addmod(a, r, m1.q) : submod(a, r, m1.q)) * inv, m1.q, m1.qinv);
    const bool negative = w > m1.q / 2;
    const u64 size = negative ? m1.q - w : w;
    u64 *out = p + (size_t)blockIdx.y * ext * n + i;
    for (int l = 0; l < ext; l++) {
        const ModC m = modc[l <= level ? l : L + l - level];
        const u64 x = to_mont(size, m);
        out[(size_t)l * n] = negative && x ? m.q - x : x;
    }
}
// out[z][limbs][n] = the second components of b.c[z]
struct SecondBatch {
    const u64 *c[CM_KS_BATCH];
};
__global__ __launch_bounds__(ROT_TPB) void k_second(u64 *__restrict__ out, SecondBatch b, int limbs, int n) {
    const size_t i = blockIdx.x * ROT_TPB + threadIdx.x, at = (size_t)blockIdx.y * n + i;
    out[(size_t)blockIdx.z * limbs * n + at] = b.c[blockIdx.z][(size_t)limbs * n + at];
}

// ---- weighted rotations -----------------------------------------------------------------------------------------------
// A lane has two neighbouring words of an output and runs over its items: the item's digits through the Galois map, its key's
// words, the sums reduced and multiplied by the item's plaintext.
template <bool SA>
__global__ __launch_bounds__(ROT_TPB) void k_weighted(WrBatch b, const ModC *__restrict__ modc, int beta, int ext, int level, int L, int nmod, int n,
                                                      int logn, const u64 *__restrict__ pmont, EvkA eva, const u64 *__restrict__ ubound) {
    const unsigned i2 = (blockIdx.x * ROT_TPB + threadIdx.x) * 2;
    const int r = blockIdx.y, z = blockIdx.z, mi = r <= level ? r : L + 1 + (r - level - 1);
    const ModC m = modc[mi];
    const size_t o = (size_t)r * n + i2;
    const u64 bound = ubound[mi], cg0 = ((u64)i2 + 1) * GOLD, cg1 = cg0 + GOLD, pm = r <= level ? pmont[r] : 0;
    ulonglong2 r0 = make_ulonglong2(0, 0), r1 = make_ulonglong2(0, 0);
    auto mul = [&](u64 x, u64 y) { return redc((u128)x * y, m.q, m.qinv); };
    auto pair = [](const u64 *p) { return *reinterpret_cast<const ulonglong2 *>(p); };
    if (b.extra[z]) r0 = pair(b.extra[z] + o), r1 = pair(b.extra[z] + (size_t)ext * n + o);
    if (b.here[z] && r <= level) {
        const ulonglong2 w = pair(b.here[z] + o), x = pair(b.c_here[z] + o), y = pair(b.c_here[z] + (size_t)(level + 1) * n + o);
        const u64 wx = mul(w.x, pm), wy = mul(w.y, pm);
        r0.x = addmod(r0.x, mul(x.x, wx), m.q), r0.y = addmod(r0.y, mul(x.y, wy), m.q);
        r1.x = addmod(r1.x, mul(y.x, wx), m.q), r1.y = addmod(r1.y, mul(y.y, wy), m.q);
    }
    for (int s = 0; s < b.nsum; s++) {
        const WrItem it = b.it[z * b.nsum + s];
        const unsigned src = perm_src(i2, it.g, logn), base = src & ~1u;
        const bool swap = src & 1u;
        u128 a0 = 0, a1 = 0, b0 = 0, b1 = 0;
        for (int j = 0; j < beta; j++) {
            const ulonglong2 d = pair(it.dig + ((size_t)j * ext + r) * n + base);
            const u64 dx = swap ? d.y : d.x, dy = swap ? d.x : d.y;
            const u64 *kb = it.key + ((size_t)j * nmod + mi) * n + i2;
            const u64 ex = __builtin_nontemporal_load(kb), ey = __builtin_nontemporal_load(kb + 1);
            const ulonglong2 ea = evk_a_words<SA>(it.key, eva, nmod, n, j, mi, i2, cg0, cg1, bound);
            b0 += (u128)dx * ex, b1 += (u128)dy * ey, a0 += (u128)dx * ea.x, a1 += (u128)dy * ea.y;
        }
        if (r <= level) {
            const ulonglong2 c = pair(it.c + (size_t)r * n + base);
            b0 += (u128)(swap ? c.y : c.x) * pm, b1 += (u128)(swap ? c.x : c.y) * pm;
        }
        const ulonglong2 w = pair(it.pt + o);
        r0.x = addmod(r0.x, mul(redc(b0, m.q, m.qinv), w.x), m.q), r0.y = addmod(r0.y, mul(redc(b1, m.q, m.qinv), w.y), m.q);
        r1.x = addmod(r1.x, mul(evk_a_reduce<SA>(a0, m), w.x), m.q), r1.y = addmod(r1.y, mul(evk_a_reduce<SA>(a1, m), w.y), m.q);
    }
    *reinterpret_cast<ulonglong2 *>(b.out[z] + o) = r0;
    *reinterpret_cast<ulonglong2 *>(b.out[z] + (size_t)ext * n + o) = r1;
}
void launch_weighted(cm_ctx *ctx, const WrBatch &b, int beta, int level, hipStream_t st) {
    Prof prof_(ctx, CM_K_INNER_PRODUCT, b.nz * b.nsum, st);
    const int ext = level + 1 + ctx->K;
    const dim3 grid(ctx->n / (2 * ROT_TPB), ext, b.nz);
    if (ctx->evk_stored_a)
        hipLaunchKernelGGL(k_weighted<true>, grid, dim3(ROT_TPB), 0, st, b, ctx->d_modc, beta, ext, level, ctx->L, ctx->nmod, ctx->n, ctx->logn,
                           ctx->d_pmont, evk_a_of(ctx), ctx->d_ubound);
    else
        hipLaunchKernelGGL(k_weighted<false>, grid, dim3(ROT_TPB), 0, st, b, ctx->d_modc, beta, ext, level, ctx->L, ctx->nmod, ctx->n, ctx->logn,
                           ctx->d_pmont, evk_a_of(ctx), ctx->d_ubound);
}
cm_status weighted_down(cm_ctx *ctx, u64 *us, int level, int m, u64 *const *outs, u64 *tmp, hipStream_t st) {
    if (ks_drop_fits(ctx, level, 1, m)) return ks_drop(ctx, us, level, 1, m, nullptr, 0, 0, 0, nullptr, 0, nullptr, st, false, outs);
    const size_t ublk = 2 * (size_t)(level + 1 + ctx->K) * ctx->n;
    for (int z = 0; z < m; z++) CMCHK(moddown_rescale_into(ctx, us + z * ublk, level, tmp, outs[z], st));
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
    for (int m = 0; freq && m < rot_dims / 2; m++) if (!isfinite(freq[m])) return CM_E_INVAL;
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
        get(&r->d_work, 2 * ln + r->batch * (2 * ln + dblk));
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
    const int n = ctx->n, sets = split ? ROT_SETS : 1, ext = r->level + 1 + ctx->K;
    std::vector<RotEntry> entries;
    for (int i = 0; i < r->t; i++)
        if (pos[i] >= 0)
            entries.push_back({(unsigned short)(pos[i] % r->low), (unsigned short)(pos[i] / r->low), (unsigned)galois_of_step(ctx, -i),
                               1u | (i >= split ? 2u : 4u)});
    std::sort(entries.begin(), entries.end(), [](const RotEntry &a, const RotEntry &b) { return a.high < b.high; });
    std::vector<int32_t> kept(pos, pos + r->t);
    size_t k0 = 0;
    do {
        const int m = (int)std::min<size_t>(ROT_ENTRIES, entries.size() - k0);
        RotBatch b;
        for (int k = 0; k < ROT_ENTRIES; k++) b.e[k] = k < m ? entries[k0 + k] : RotEntry{0, 0, 1, 0};
        Prof prof_(ctx, CM_K_ELEMENTWISE, sets * r->parts * 2, st);
        hipLaunchKernelGGL(k_rotary_products, dim3(n / ROT_TPB, 2, sets), dim3(ROT_TPB), 0, st, r->d_v, b, m, r->d_low, r->d_still, r->d_high, ctx->d_modc,
                           r->ma, r->mb, r->parts, n, ctx->logn, k0 > 0);
        k0 += m;
    } while (k0 < entries.size());
    launch_ntt(ctx, r->d_v, r->d_mods, sets * r->parts * 2, true, st);
    {
        Prof prof_(ctx, CM_K_ELEMENTWISE, sets * r->parts * ext, st);
        hipLaunchKernelGGL(k_rotary_round, dim3(n / ROT_TPB, sets * r->parts), dim3(ROT_TPB), 0, st, r->d_p, r->d_v, ctx->d_modc, r->ma, r->mb, r->inv, r->level,
                           ctx->L, ext, n);
    }
    launch_ntt(ctx, r->d_p, r->d_ext_mods, sets * r->parts * ext, false, st);
    r->pos.swap(kept), r->split = split, r->set = true;
    RETURN_LAUNCH_STATUS();
    CM_CATCH
}
// of up to r->batch ciphertexts, each with the plaintexts of `sets` sets from the first on: sums on the extended basis, us[z][set]
cm_status rotary_sums(cm_ctx *ctx, const cm_evk *evk, const cm_rotary *r, int m, const u64 *const *xs, int first, int sets, u64 *us, hipStream_t st) {
    const int level = r->level;
    const KsLevel &kl = ks_level(ctx, level);
    const size_t n = ctx->n, ln = (size_t)(level + 1) * n, dblk = (size_t)kl.beta * kl.ext * n, ublk = 2 * (size_t)kl.ext * n;
    u64 *second = r->d_work + 2 * ln, *ksin = second + r->batch * ln, *digits = ksin + r->batch * ln;
    const u64 *keys[2];
    unsigned g[2];
    for (int s = 0; s < r->parts - 1; s++) {
        g[s] = (unsigned)galois_of_step(ctx, s ? -r->step : r->step), keys[s] = find_key(evk, g[s]);
        if (!keys[s]) return CM_E_NOKEY;
    }
    const u64 *d = xs[0] + ln;
    if (m > 1) {
        SecondBatch b;
        for (int z = 0; z < CM_KS_BATCH; z++) b.c[z] = xs[z < m ? z : 0];
        hipLaunchKernelGGL(k_second, dim3(n / ROT_TPB, level + 1, m), dim3(ROT_TPB), 0, st, second, b, level + 1, (int)n);
        d = second;
    }
    CMCHK(ks_raise_many(ctx, r->tabs, d, ksin, digits, st, m));
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
    launch_weighted(ctx, b, kl.beta, level, st);
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
        CMCHK(rotary_sums(ctx, evk, r, m, xs, 0, 1, us, st));
        CMCHK(weighted_down(ctx, us, r->level, m, outs, r->d_work, st));
    }
    for (int i = 0; i < count; i++) y[i].level = r->level - 1, y[i].ncomp = 2, y[i].scale = x[i].scale;      // plaintext scale = the prime just removed
    RETURN_LAUNCH_STATUS();
    CM_CATCH
}
