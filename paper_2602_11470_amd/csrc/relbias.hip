// Learned relative position bias on encrypted attention scores.
//
// Scores hold the token of place c t_kv + j in row c, residue j, of every KV head; the cache is a ring of cap = E t_kv places.  A query
// at place p sees the token of a place at the distance d = (p - place) mod cap; its score takes table[head][bucket[d]].  What a
// query of row c_q adds is what one of row 0 with the same residue adds, c_q rows further on: ONE plaintext per pass and residue
// (decode) or per pass and group of residues (prompt) serves every position, through the Galois map that moves slots by whole rows --
// an exact permutation of the plaintext's values.  The mask of the rows outside the pages that a query may see (the start of a packed
// sequence, a window) is the sum of rotations of one plaintext row, formed once per number of rows.
#include <math.h>

#include <algorithm>
#include <iterator>

#include "kv.h"

typedef u64 u64x2 __attribute__((ext_vector_type(2)));

struct cm_relbias {
    cm_ctx *ctx = nullptr;
    int H, E, t_kv, G, level, passes, phases;
    bool prompt = false, masked = false;
    double scale;
    u64 *d_pts = nullptr;          // [passes][phases][level+1][n]
    u64 *d_unseen = nullptr;       // [E-1][level+1][n]: entry m - 1: the mask's value in the rows m .. E-1; null without a mask or other rows
};

// out = a + (b through the Galois map g), rows limbs
__global__ void k_add_turned(u64 *out, const u64 *a, const u64 *b, const ModC *__restrict__ modc, unsigned g, int n, int logn) {
    const unsigned i = blockIdx.x * 256 + threadIdx.x;
    const size_t row = (size_t)blockIdx.y * n;
    out[row + i] = addmod(a[row + i], b[row + perm_src(i, g, logn)], modc[blockIdx.y].q);
}

#define BIAS_BATCH 32
#define BIAS_LARGE (128 << 20)
struct BiasBatch {
    const u64 *in[BIAS_BATCH], *pt[BIAS_BATCH];
    u64 *out[BIAS_BATCH];
};
// out[z] = in[z] + (pt[z] through g, row through gr, 0).  A lane has two neighbouring words, which the Galois map leaves neighbours: 16-byte
// accesses, the plaintexts' in another order (its aligned runs of 64 stay together, so they coalesce as well).  Bound by memory: eight passes at
// level 21 (473 MB with the plaintexts) 73.5 us, 6.4 TB/s, with one word a lane 89.7; a single pass is the launch (6.3 us a call from Python, 3.9 of
// them the launch).  Stores go past the caches always (four passes at level 8 17.9 us otherwise).  LARGE: scores are read past them as well, from BIAS_LARGE
// bytes of scores on (both components, in and out).  Reads past the caches cost where the scores are still in them, as those of a few passes
// are, and pay where they are not.  Plainly and past them, each call on other scores, window masked: 75 MB (four passes at level 8) 15.4 and 17.4 us, 134 MB (eight
// at level 7) 29.3 and 27.9, 159 MB 36.5 and 32.5, 167 MB 37.1 and 33.1, 218 MB 47.6 and 42.5, 318 MB 69.6 and 60.6, 369 MB 81.1 and 73.8.  On one set of scores
// again and again 117 MB 20.8 and 22.7, 134 MB 23.5 and 26.3; on 2.5 GB of them in turn 23.8 and 22.7, 26.6 and 26.1.  In place, where a
// launch moves half of these bytes, the same line holds: four passes at level 11 (100 MB) 13.4 and 12.1 / 15.1 and 12.3, at level 15 (134 MB) 15.9 and 16.7 /
// 18.2 and 16.6, eight at level 15 (268 MB) 29.3 and 30.1 / 31.8 and 30.1.
__device__ __forceinline__ u64x2 turned(const u64 *p, unsigned src) {
    const u64x2 w = *(const u64x2 *)(p + (src & ~1u));
    return src & 1u ? u64x2{w.y, w.x} : w;
}
template <bool LARGE>
__global__ __launch_bounds__(256) void k_relbias(BiasBatch b, const u64 *row, unsigned g, unsigned gr, const ModC *__restrict__ modc, int limbs, int n,
                                                 int logn) {
    const unsigned i = 2 * (blockIdx.x * 256 + threadIdx.x);
    const int l = blockIdx.y, z = blockIdx.z;
    const size_t at = (size_t)l * n + i, cs = (size_t)limbs * n;
    const u64 q = modc[l].q;
    const u64 *in = b.in[z];
    u64 *out = b.out[z];
    auto load = [](const u64 *p) { return LARGE ? __builtin_nontemporal_load((const u64x2 *)p) : *(const u64x2 *)p; };
    auto store = [](u64x2 w, u64 *p) { __builtin_nontemporal_store(w, (u64x2 *)p); };
    const u64x2 v = load(in + at);
    u64x2 c1 = {0, 0}, r = {0, 0};
    if (out != in) c1 = load(in + at + cs);
    const u64x2 p = turned(b.pt[z] + (size_t)l * n, perm_src(i, g, logn));
    if (row) r = turned(row + (size_t)l * n, perm_src(i, gr, logn));
    const u64x2 w = {addmod(addmod(v.x, p.x, q), r.x, q), addmod(addmod(v.y, p.y, q), r.y, q)};
    store(w, out + at);
    if (out != in) store(c1, out + at + cs);
}

cm_status rows_from_on(cm_ctx *ctx, u64 *entries, const u64 *row, int B, int E, int limbs) {
    const int n = ctx->n;
    const size_t words = (size_t)limbs * n;
    // E - 1 pages visible: the row turned right by E - 1; i pages: those of i + 1 and the row turned right by i
    for (int i = E - 1; i > 0; i--) {
        const u64 g = galois_of_step(ctx, (int)(((long long)n / 2 - (long long)i * B) % (n / 2)));
        u64 *entry = entries + (i - 1) * words;
        if (i == E - 1) launch_automorphism(ctx, entry, row, limbs, g, 0);
        else hipLaunchKernelGGL(k_add_turned, dim3(n / 256, limbs), dim3(256), 0, 0, entry, entry + words, row, ctx->d_modc, (unsigned)g, n, ctx->logn);
    }
    return CM_OK;
}
extern "C" void cm_relbias_destroy(cm_relbias *rb) {
    if (!rb) return;
    hipFree(rb->d_pts), hipFree(rb->d_unseen);
    delete rb;
}
extern "C" cm_status cm_relbias_create(cm_ctx *ctx, int32_t heads, int32_t dim, int32_t group, int32_t prompt, int32_t level, double scale,
                                       int32_t nbuckets, const double *table, const int32_t *bucket, double mask, const int64_t *coeffs,
                                       cm_relbias **out) {
    return cm_relbias_create_ex(ctx, heads, dim, group, prompt, level, scale, nbuckets, table, bucket, mask, 0, coeffs, out);
}
extern "C" cm_status cm_relbias_create_ex(cm_ctx *ctx, int32_t heads, int32_t dim, int32_t group, int32_t prompt, int32_t level, double scale,
                                          int32_t nbuckets, const double *table, const int32_t *bucket, double mask, uint32_t flags,
                                          const int64_t *coeffs, cm_relbias **out) {
    (void)hipGetLastError();          // stale errors of earlier calls are not this call's
    if (!ctx || !out || heads < 1 || dim < 1 || group < 1 || nbuckets < 1 || !table || !bucket || (prompt != 0 && prompt != 1)) return CM_E_INVAL;
    if ((flags & ~(uint32_t)CM_RELBIAS_CAUSAL) || ((flags & CM_RELBIAS_CAUSAL) && mask == 0)) return CM_E_INVAL;
    if (level < 0 || level > ctx->L) return CM_E_LEVEL;
    const int S = ctx->n / 2;
    if (heads > S || dim > S) return CM_E_LAYOUT;
    const int H = 1 << ilog2(heads), real = heads;
    if (!pow2(dim) || (long long)H * dim > S || !pow2(group) || S / (H * dim) % group) return CM_E_LAYOUT;
    const int t_kv = S / (H * dim), t = t_kv / group, cap = dim * t_kv;
    if (scale == 0) scale = ctx->prm.scale;
    if (!(scale > 0) || !isfinite(scale) || !isfinite(mask)) return CM_E_INVAL;
    // a slot holds a table entry and at most one mask value: their coefficients have to fit the signed words of the encoding
    double top = fabs(mask);
    for (size_t i = 0; i < (size_t)real * group * nbuckets; i++) {
        if (!isfinite(table[i])) return CM_E_INVAL;
        top = fmax(top, fabs(table[i]));
    }
    if (top * scale >= 0x1p61) return CM_E_INVAL;
    for (int d = 0; d < cap; d++) if (bucket[d] < 0 || bucket[d] >= nbuckets) return CM_E_INVAL;
    cm_relbias *rb = new (std::nothrow) cm_relbias();
    if (!rb) return CM_E_NOMEM;
    cm_status status = CM_OK;
    u64 *row = nullptr;            // the mask's value in row 0
    try {
        rb->ctx = ctx, rb->H = H, rb->E = dim, rb->t_kv = t_kv, rb->G = group, rb->level = level, rb->prompt = prompt != 0, rb->scale = scale, rb->masked = mask != 0;
        rb->passes = prompt ? t_kv : group, rb->phases = prompt ? group : t_kv;
        const int n = ctx->n, polys = rb->passes * rb->phases;
        const size_t words = (size_t)(level + 1) * n;
        if (hipMalloc((void **)&rb->d_pts, polys * words * 8) != hipSuccess) status = CM_E_NOMEM;
        if (status == CM_OK && mask != 0 && dim > 1 &&
            (hipMalloc((void **)&rb->d_unseen, (dim - 1) * words * 8) != hipSuccess || hipMalloc((void **)&row, words * 8) != hipSuccess))
            status = CM_E_NOMEM;
        auto encode = [&](u64 *dst, const std::vector<double> &m, int i) {
            cm_pt pt;
            pt.dev = dst, pt.mont = 0;
            return coeffs ? cm_pt_from_coeffs(ctx, coeffs + (size_t)i * n, level, scale, &pt) : cm_encode(ctx, m.data(), nullptr, S, level, scale, &pt);
        };
        std::vector<double> m(S);
        for (int p = 0; p < polys && status == CM_OK; p++) {
            const int delta = p / rb->phases, phase = p % rb->phases;
            for (int x = 0; x < dim; x++)
                for (int j = 0; j < t_kv; j++) {
                    const int u = (j - delta + t_kv) % t_kv;                 // prompt: the query's residue in its page
                    const int g = prompt ? u / t : ((j / t - delta) % group + group) % group;
                    const int place = prompt ? phase * t + u % t : phase, d = ((place - j - x * t_kv) % cap + cap) % cap;
                    // the query's own page: the places behind it have the largest distances, which the oldest page of a full ring has as well
                    const double behind = (flags & CM_RELBIAS_CAUSAL) && x == 0 && j > place ? mask : 0.0;
                    for (int h = 0; h < H; h++)
                        m[(size_t)(x * H + h) * t_kv + j] = (h < real ? table[(size_t)(h * group + g) * nbuckets + bucket[d]] : 0.0) + behind;
                }
            status = encode(rb->d_pts + p * words, m, p);
        }
        if (status == CM_OK && rb->d_unseen) {
            for (int i = 0; i < S; i++) m[i] = i < H * t_kv ? mask : 0.0;
            status = encode(row, m, polys);
            if (status == CM_OK) {
                rows_from_on(ctx, rb->d_unseen, row, H * t_kv, dim, level + 1);
                if (hipDeviceSynchronize() != hipSuccess || hipGetLastError() != hipSuccess) status = CM_E_HIP;
            }
        }
    } catch (...) {
        status = CM_E_NOMEM;
    }
    hipFree(row);
    if (status != CM_OK) {
        cm_relbias_destroy(rb);
        return status;
    }
    *out = rb;
    return CM_OK;
}
// whether the words that an output is written to are another output's, or an input's other than that the pass's output is its input itself.  Arrays
// of n ciphertexts of `words` words each; by sorting where they are many.
bool relbias_outputs_shared(const cm_ct *in, const cm_ct *out, int n, size_t words) {
    const uintptr_t len = words * sizeof(u64);
    auto at = [](const cm_ct &c) { return (uintptr_t)c.dev; };
    auto meet = [len](uintptr_t a, uintptr_t b) { return (a < b ? b - a : a - b) < len; };
    if (n <= 16) {
        for (int p = 0; p < n; p++)
            for (int r = 0; r < n; r++) {
                if (r != p && meet(at(out[r]), at(out[p]))) return true;
                if (!(r == p && out[r].dev == in[p].dev) && meet(at(out[r]), at(in[p]))) return true;
            }
        return false;
    }
    std::vector<std::pair<uintptr_t, int>> o(n);
    for (int r = 0; r < n; r++) o[r] = {at(out[r]), r};
    std::sort(o.begin(), o.end());
    for (int r = 1; r < n; r++) if (meet(o[r - 1].first, o[r].first)) return true;
    for (int p = 0; p < n; p++) {
        const uintptr_t a = at(in[p]);
        // the outputs are apart: only the last one that begins in front of the input and the first one that does not can meet it
        auto next = std::lower_bound(o.begin(), o.end(), std::make_pair(a, -1));
        if (next != o.begin() && meet(std::prev(next)->first, a)) return true;
        if (next != o.end() && meet(next->first, a) && !(next->first == a && next->second == p)) return true;
    }
    return false;
}
extern "C" int32_t cm_relbias_passes(const cm_relbias *rb) { return rb ? rb->passes : 0; }
extern "C" cm_status cm_relbias_apply(cm_ctx *ctx, const cm_relbias *rb, int32_t token, int32_t first, int32_t pass0, int32_t npass, const cm_ct *in,
                                      cm_ct *out, void *stream) {
    (void)hipGetLastError();          // stale errors of earlier calls are not this call's
    if (!ctx || !rb || rb->ctx != ctx || !in || !out || npass < 1 || pass0 < 0) return CM_E_INVAL;
    const int cap = rb->E * rb->t_kv, t = rb->t_kv / rb->G;
    if (token < 0 || token >= cap || (rb->prompt && token % t) || first < -1 || first >= cap || (first > 0 && first % rb->t_kv)) return CM_E_LAYOUT;
    if (first >= 0 && !rb->masked) return CM_E_LAYOUT;
    if (npass > rb->passes - pass0) return CM_E_LAYOUT;
    for (int p = 0; p < npass; p++) {
        if (!in[p].dev || !out[p].dev || in[p].ncomp != 2) return CM_E_INVAL;
        if (in[p].level != rb->level) return CM_E_LEVEL;
        if (!(fabs(in[p].scale / rb->scale - 1) < 1e-9)) return CM_E_SCALE;
    }
    CM_TRY
    if (relbias_outputs_shared(in, out, npass, 2 * (size_t)(rb->level + 1) * ctx->n)) return CM_E_INVAL;
    hipStream_t st = (hipStream_t)stream;
    const int n = ctx->n, limbs = rb->level + 1, S = n / 2, page = token / rb->t_kv, phase = rb->prompt ? token % rb->t_kv / t : token % rb->t_kv;
    const size_t words = (size_t)limbs * n;
    auto turn = [&](int rows) { return (unsigned)galois_of_step(ctx, (int)(((long long)S - (long long)rows * rb->H * rb->t_kv) % S)); };
    const u64 *row = nullptr;
    unsigned gr = 0;
    if (first >= 0) {
        const int from = first / rb->t_kv, seen = (page - from + rb->E) % rb->E + 1;
        if (seen < rb->E) row = rb->d_unseen + (seen - 1) * words, gr = turn(from);
    }
    for (int p0 = 0; p0 < npass; p0 += BIAS_BATCH) {
        const int m = npass - p0 < BIAS_BATCH ? npass - p0 : BIAS_BATCH;
        BiasBatch b;
        for (int z = 0; z < m; z++) {
            b.in[z] = in[p0 + z].dev, b.out[z] = out[p0 + z].dev;
            b.pt[z] = rb->d_pts + ((size_t)(pass0 + p0 + z) * rb->phases + phase) * words;
        }
        Prof prof_(ctx, CM_K_ELEMENTWISE, (double)m * limbs, st);
        const bool large = (size_t)m * 4 * words * 8 >= BIAS_LARGE;
        hipLaunchKernelGGL((large ? k_relbias<true> : k_relbias<false>), dim3(n / 512, limbs, m), dim3(256), 0, st, b, row, turn(page), gr, ctx->d_modc, limbs, n, ctx->logn);
    }
    for (int p = 0; p < npass; p++) out[p].level = in[p].level, out[p].ncomp = 2, out[p].scale = in[p].scale;
    RETURN_LAUNCH_STATUS();
    CM_CATCH
}
