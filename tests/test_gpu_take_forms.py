"""Kept tokens moved into another cache (cm_kv_take) in the forms that the sizes and options choose between: both forms of the masked products and of the keys
on the large ring, key switches in more than one batch, integer limbs under the fused rescale.  Word for word against the single calls."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rings():
    """Contexts by name: ring degree, then the bits of the first and of the other primes."""
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2602_11470_amd import binding as B
    made = {}

    def get(name):
        if name not in made:
            n, first, others = (int(x) for x in name.split())
            made[name] = B.llama_ring(24, 4) if n == 65536 and first == others == 50 else B.Context(n, 8, 2, 2, first, others, 60, 2.0 ** 50)
        return made[name]
    yield get
    for c in made.values():
        c.close()


def _residues(ctx, shape, limbs, gen):
    import torch
    out = torch.empty(*shape, limbs, ctx.n, dtype=torch.int64, device="cuda")
    for i, q in enumerate(ctx.moduli()[:limbs]):
        out[..., i, :] = torch.empty(*shape, ctx.n, dtype=torch.int64, device="cuda").random_(0, int(q), generator=gen)
    return out


def _filled(ctx, heads, dim, r_i, level, index, ntok, seed):
    import torch
    from paper_2602_11470_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kv = ctx.kv_create(heads, dim, level, r_i=r_i, key_index=index)
    for w in [B.CM_QK, B.CM_SV] + ([B.CM_KV_INDEX] if index else []):
        words = kv.words(w)
        words.copy_(_residues(ctx, words.shape[:-2], level + 1, gen))
    kv.set_tokens(ntok)
    return kv


def _words(c):
    n = c.ctx.n
    return c.buf[: c.ncomp * (c.level + 1) * n].view(c.ncomp, c.level + 1, n)


def _check(ctx, heads, dim, r_i, index, level, keep, shift, add, two_step=False, stored_a=False):
    """One take against the single calls."""
    import torch
    from oracle import packing
    from paper_2602_11470_amd import binding as B
    lay = packing.KvLayout(ctx.S, heads, dim, r_i)
    which = [B.CM_QK, B.CM_SV] + ([B.CM_KV_INDEX] if index else [])
    src, dst = _filled(ctx, heads, dim, r_i, level, index, len(keep), 1), _filled(ctx, heads, dim, r_i, level - 1, index, 0, 2)
    before = {w: dst.words(w).clone() for w in which}
    scale, q = float(ctx.moduli()[level]), torch.tensor([int(m) for m in ctx.moduli()[:level]], device="cuda")[:, None]
    try:
        ctx.set_option(B.CM_OPT_TWO_STEP_MASKS, two_step)
        ctx.set_option(B.CM_OPT_EVK_STORED_A, stored_a)
        sel = ctx.kv_sel(src, keep, shift)
        keys = ctx.keygen_rotations(ctx.keygen_secret(1), sel.steps(), 2) if sel.steps() else None
        ctx.kv_take(keys, sel, src, dst, add)
        encoded = {}

        def masked(words, key, slots):
            x = B.Ct(ctx, level)
            x.buf[: words.numel()], x.d.scale = words.reshape(-1), ctx.scale
            if key not in encoded:
                encoded[key] = ctx.pt_from_coeffs(slots(), level, scale, mont=True)
            return ctx.rescale(ctx.mul_pt(x, encoded[key]))

        def compare(w, at, y):
            """y: the ciphertext or words that belong there, or None."""
            words = torch.zeros_like(before[w][at]) if y is None else y if torch.is_tensor(y) else _words(y)
            if add:
                words = words + before[w][at]
                words = torch.where(words >= q, words - q, words)
            assert torch.equal(dst.words(w)[at], words), (w, at)
        row = ctx.encode_coeffs(lay.keep_rows(keep), scale)
        pages = {c: keep[c * lay.t:(c + 1) * lay.t] for c in range(-(-len(keep) // lay.t))}
        for to in range(dim):
            p = pages.get(to - shift)
            if p is None or not p.any():
                compare(B.CM_QK, (to,), None)
            elif p.all():
                compare(B.CM_QK, (to,), src.words(B.CM_QK)[to - shift][:, :level])
            else:
                compare(B.CM_QK, (to,), masked(src.words(B.CM_QK)[to - shift], tuple(p), lambda: ctx.encode_coeffs(lay.keep_residues(keep, to - shift), scale)))
        rotations = {}
        for k in range(dim if keep.any() else 0):
            for w, place, rows in ((B.CM_SV, lay.v_place, k % r_i), (B.CM_KV_INDEX, lay.k_index_place, -(k // r_i) * r_i)):
                if w not in which:
                    continue
                at = (lambda i: (i // r_i, i % r_i)) if w == B.CM_KV_INDEX else (lambda i: (i,))
                y = masked(src.words(w)[at(k)], rows, lambda: _turned(ctx, row, rows * lay.H * lay.t))
                to, turn = place(k, shift)
                rotations[turn] = rotations.get(turn, 0) + 1
                compare(w, at(to), ctx.rotate(keys, y, turn * lay.H * lay.t) if turn else y)
        return rotations
    finally:
        ctx.set_option(B.CM_OPT_TWO_STEP_MASKS, 0)
        ctx.set_option(B.CM_OPT_EVK_STORED_A, 0)


def _turned(ctx, coeffs, step):
    """Coefficients of the plaintext whose slots are rotated left by step."""
    n = ctx.n
    e = np.arange(n) * pow(5, step % ctx.S, 2 * n) % (2 * n)
    out = np.empty(n, dtype=np.int64)
    out[e % n] = np.where(e < n, coeffs, -coeffs)
    return out


def _keep(what, ntok, t, shift):
    rng = np.random.default_rng(ntok)
    keep = rng.uniform(size=ntok) < 0.7 if what == "ragged" else np.ones(ntok, dtype=bool)
    keep[: max(0, -shift) * t] = False
    return keep


# heads, dim, r_i, index, level, tokens, what is kept, shift
@pytest.mark.parametrize("two_step,stored_a", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("case", [(32, 8, 2, True, 4, 600, "head", -3), (32, 8, 4, True, 3, 700, "ragged", 0), (64, 32, 8, True, 3, 100, "ragged", 13),
                                  (12, 16, 4, False, 9, 500, "ragged", 5)], ids=str)
def test_both_forms_of_masks_and_keys_on_the_large_ring(rings, case, add, two_step, stored_a):
    heads, dim, r_i, index, level, ntok, what, shift = case
    ctx = rings("65536 50 50")
    t = ctx.S // ((1 << (heads - 1).bit_length()) * dim)
    _check(ctx, heads, dim, r_i, index, level, _keep(what, ntok, t, shift), shift, add, two_step, stored_a)


def _batch(ctx, level):
    """Key switches that a batch takes (ks_batch_max): the arena holds the sums of 16 and the converted limbs of 8 at the top level."""
    L, K = ctx.L, ctx.K
    return min(32, 16 * (L + 1 + K) // (level + 1 + K), 8 * (L + 1) // (level + 1))


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("case", [(32, 64, 8, False, 10, 1024, -32), (32, 64, 64, True, 10, 900, -30), (64, 32, 32, True, 17, 240, 16), (64, 32, 4, True, 17, 400, -16),
                                  (16, 64, 16, False, 22, 700, 32)], ids=str)
def test_more_ciphertexts_turn_than_a_batch_of_key_switches_takes(rings, case, add):
    """From result level 6 up a batch holds fewer than 32, so the ciphertexts that turn by one amount take several."""
    heads, dim, r_i, index, level, ntok, shift = case
    ctx = rings("65536 50 50")
    assert _batch(ctx, level - 1) < 32
    t = ctx.S // (heads * dim)
    rotations = _check(ctx, heads, dim, r_i, index, level, _keep("all", ntok, t, shift), shift, add)
    assert max(m for turn, m in rotations.items() if turn) > _batch(ctx, level - 1)


@pytest.mark.parametrize("stored_a", [False, True])
def test_several_batches_of_key_switches_with_stored_keys(rings, stored_a):
    ctx = rings("65536 50 50")
    _check(ctx, 32, 64, 64, True, 10, _keep("ragged", 700, ctx.S // (32 * 64), 20), 20, True, stored_a=stored_a)


# A first prime of 60 bits over 50-bit ones, and 51-bit primes: the last limb's residues fit the others, and limbs from 2^50 on take integer butterflies.
@pytest.mark.parametrize("ring", ["4096 60 50", "4096 51 51", "65536 60 50", "65536 51 51", "4096 60 40"])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("case", [(4, 16, 4, True, 3, 300, "ragged", 0), (2, 64, 8, True, 6, 300, "ragged", 0), (4, 16, 4, True, 5, 290, "head", -3), (8, 32, 32, True, 7, 190, "ragged", 6)],
                         ids=str)
def test_integer_limbs_under_the_fused_rescale(rings, ring, case, add):
    heads, dim, r_i, index, level, ntok, what, shift = case
    ctx = rings(ring)
    last = int(ctx.moduli()[level])
    assert last < 1 << 52 and all(last < 2 * int(m) for m in ctx.moduli()[:level]) and int(ctx.moduli()[0]) >= 1 << 50
    _check(ctx, heads, dim, r_i, index, level, _keep(what, ntok, ctx.S // (heads * dim), shift), shift, add)
