"""Key switches of eight to sixteen digits under 61-bit moduli, limb for limb against the oracle, and a tree of drafts decrypted.

The sum of sixteen products of a digit with a raw draw passes 128 bits, and that of sixteen with words in multiplier form passes q 2^64, in about one word
of 40000 (uniform words; a term is below 2^125): a limb of 4096 words has one in ten limbs.  A rotation on the first ring has eighteen such limbs, on the
second eight, and every test forms at least eight rotations: some five wrong words or more if the sums were not brought down on the way, none of
which a comparison of words misses.  A word that is wrong in a special limb is divided with it and destroys the ciphertext."""
import numpy as np
import pytest

from oracle import params

pytestmark = pytest.mark.gpu
N = 4096
RINGS = {"all": (16, 2, 1, 61, 61, 61), "special": (16, 8, 1, 59, 59, 61)}


@pytest.fixture(scope="module")
def rings():
    from oracle import ckks
    from paper_2602_11470_amd import binding as B
    made = {}

    def get(name):
        if name not in made:
            n_q, n_p, alpha, _, qi, p = RINGS[name]
            qs = params.scan_primes(qi, N, n_q)
            ps = [m for m in params.scan_primes(p, N, n_p + n_q) if m not in qs][:n_p]
            prm = params.Params(n=N, q=qs, p=ps, alpha=alpha, scale=2.0 ** 55, hamming=64)
            g = B.Context(N, *RINGS[name], 2.0 ** 55, hamming=64)
            assert [int(x) for x in g.moduli()] == prm.moduli
            made[name] = (g, ckks.Context(prm))
        return made[name]
    yield get
    for g, _ in made.values():
        g.close()


def _same(octx, gctx, o, g):
    np.testing.assert_array_equal(gctx.ct_export(g), octx.canonical(o))


@pytest.mark.parametrize("stored_a", [0, 1])
@pytest.mark.parametrize("name, level", [("all", 15), ("all", 10), ("all", 7), ("special", 15)])
def test_key_switches(rings, name, level, stored_a):
    from paper_2602_11470_amd import binding as B
    gctx, octx = rings(name)
    gctx.set_option(B.CM_OPT_EVK_STORED_A, stored_a)
    try:
        osk, gsk = octx.keygen_secret(3), gctx.keygen_secret(3)
        steps = [1, -3] + [5 + i for i in range(8)]
        okeys, gkeys = octx.keygen_rotations(osk, steps, 4, with_relin=True), gctx.keygen_rotations(gsk, steps, 4, with_relin=True)
        c = octx.encode_coeffs(np.random.default_rng(level).uniform(-1, 1, octx.S), 2.0 ** 40)
        o = octx.encrypt(osk, octx.pt_from_coeffs(c, level, 2.0 ** 40), 5)
        g = gctx.encrypt(gsk, gctx.pt_from_coeffs(c, level, 2.0 ** 40), 5)
        _same(octx, gctx, octx.rotate(o, 1, okeys), gctx.rotate(gkeys, g, 1))
        h = octx.hoist(o)
        for st, got in zip(steps, gctx.rotate_hoisted(gkeys, g, steps)):
            _same(octx, gctx, octx.rotate_hoisted(o, h, st, okeys), got)
        o3, g3 = octx.mul_ct(o, o), gctx.mul_ct(g, g)
        _same(octx, gctx, octx.relinearize(o3, okeys), gctx.relinearize(gkeys, g3))
    finally:
        gctx.set_option(B.CM_OPT_EVK_STORED_A, 0)


@pytest.mark.parametrize("stored_a", [0, 1])
@pytest.mark.parametrize("level, halves", [(15, False), (15, True), (9, False)])
def test_rotary_positions(rings, level, halves, stored_a):
    from oracle import packing, vmm
    from paper_2602_11470_amd import binding as B
    gctx, octx = rings("special")
    gctx.set_option(B.CM_OPT_EVK_STORED_A, stored_a)
    try:
        tables = packing.RotaryTables(gctx.S, 8, 32, 9, rot=16, halves=halves)
        mods, slots, n = [float(m) for m in gctx.moduli()], tables.slots(), 4 * tables.low + 1
        coeffs = np.stack([gctx.encode_coeffs(v, mods[level]) for v in slots[:n]] + [gctx.encode_coeffs(v, mods[gctx.L + 2]) for v in slots[n:]])
        rotary = gctx.rotary(8, 32, level, 9, rot_dims=16, halves=halves, coeffs=coeffs)
        osk, gsk = octx.keygen_secret(3), gctx.keygen_secret(3)
        okeys, gkeys = octx.keygen_rotations(osk, rotary.steps(), 4), gctx.keygen_rotations(gsk, rotary.steps(), 4)
        rng, positions = np.random.default_rng(level), [8, -1, 3, 5, 0, 7, -1, 8]
        cs = [gctx.encode_coeffs(rng.normal(size=gctx.S), 2.0 ** 40) for _ in range(4)]
        xs = [gctx.encrypt(gsk, gctx.pt_from_coeffs(c, level, 2.0 ** 40), i) for i, c in enumerate(cs)]
        gctx.rotary_set(rotary, positions)
        pts = vmm.rotary_plaintexts(octx, tables, coeffs, positions, level)
        for i, y in enumerate(gctx.rotary_apply(gkeys, rotary, xs)):
            x = octx.encrypt(osk, octx.pt_from_coeffs(cs[i], level, 2.0 ** 40), i)
            _same(octx, gctx, vmm.rotary(octx, okeys, tables, x, pts), y)
    finally:
        gctx.set_option(B.CM_OPT_EVK_STORED_A, 0)


@pytest.mark.parametrize("index", [False, True])
def test_a_tree(rings, index):
    """Scores of eight queries, decrypted: the weighted sums of two items an output, relinearisations and giant steps of fifteen digits.  The scores' scale
    is 2^51; 32 products of values whose noise is below 2^7 units of 2^55, and some 40 key switches and rescales below 2^6 units of 2^51 a coefficient, leave
    less than 2^14 of them, times 2^6 for a slot: 2^-31."""
    from oracle import packing
    gctx, _ = rings("special")
    H, E, level = 8, 32, 14
    lay = packing.KvLayout(gctx.S, H, E, 8)
    t, rng = lay.t, np.random.default_rng(1)
    kv = gctx.kv_create(H, E, level, r_i=8, key_index=index)
    tree = gctx.tree(kv, mask=-24.0)
    sk = gctx.keygen_secret(3)
    keys = gctx.keygen_rotations(sk, kv.steps() + tree.steps(), 4, with_relin=True)
    parents, base = [-1, 0, 0, 1], 2 * t + 3
    K = 0.3 * rng.normal(size=(base + len(parents), H, E))
    enc = lambda slots, lv, seed: gctx.encrypt(sk, gctx.encode(slots, lv), seed)  # noqa: E731
    for i in range(E if index else 3):
        kv.load(4 if index else 0, i, enc(lay.pack_k_index(K, i) if index else lay.pack_k(K, i), level, 20 + i))
    kv.set_tokens(len(K))
    qs = 0.3 * rng.normal(size=(E, H, t))
    scores = gctx.tree_qk(keys, tree, kv, parents, base, enc(qs.reshape(-1), level + 1, 9))
    Kp = np.concatenate([K, np.zeros((lay.capacity - len(K), H, E))]).reshape(E, t, H, E)
    for d in range(t):
        want = np.einsum("chje,ehj->chj", Kp.transpose(0, 2, 1, 3), np.roll(qs, d, axis=2)) - 24.0 * packing.tree_hidden(lay, 1, parents, base, 0, 0, d)
        assert np.abs(gctx.decrypt(sk, scores[d]).real.reshape(E, H, t) - want).max() < 2.0 ** -31 * 2


@pytest.mark.parametrize("stored_a", [0, 1])
def test_the_full_ring(stored_a):
    """n = 65536, where other forms of the sums run (two words a lane): positions of two ciphertexts and hoisted rotations."""
    from oracle import ckks, packing, vmm
    from paper_2602_11470_amd import binding as B
    n, level = 65536, 15
    prm = params.Params(n=n, q=params.scan_primes(59, n, 16), p=params.scan_primes(61, n, 3), alpha=1, scale=2.0 ** 55, hamming=64)
    gctx, octx = B.Context(n, 16, 3, 1, 59, 59, 61, 2.0 ** 55, hamming=64), ckks.Context(prm)
    try:
        assert [int(x) for x in gctx.moduli()] == prm.moduli
        gctx.set_option(B.CM_OPT_EVK_STORED_A, stored_a)
        tables = packing.RotaryTables(gctx.S, 32, 128, 3, rot=16)
        mods, slots, low = [float(m) for m in gctx.moduli()], tables.slots(), 4 * tables.low + 1
        coeffs = np.stack([gctx.encode_coeffs(v, mods[level]) for v in slots[:low]] + [gctx.encode_coeffs(v, mods[gctx.L + 2]) for v in slots[low:]])
        rotary = gctx.rotary(32, 128, level, 3, rot_dims=16, coeffs=coeffs)
        osk, gsk = octx.keygen_secret(3), gctx.keygen_secret(3)
        steps = rotary.steps() + [5]
        okeys, gkeys = octx.keygen_rotations(osk, steps, 4), gctx.keygen_rotations(gsk, steps, 4)
        positions = [2, -1, 0, 1, 2, 2, -1, 1]
        gctx.rotary_set(rotary, positions)
        pts = vmm.rotary_plaintexts(octx, tables, coeffs, positions, level)
        c = gctx.encode_coeffs(np.random.default_rng(1).normal(size=gctx.S), 2.0 ** 40)
        o = octx.encrypt(osk, octx.pt_from_coeffs(c, level, 2.0 ** 40), 5)
        g = gctx.encrypt(gsk, gctx.pt_from_coeffs(c, level, 2.0 ** 40), 5)
        want = octx.canonical(vmm.rotary(octx, okeys, tables, o, pts))
        for y in gctx.rotary_apply(gkeys, rotary, [g, g]):
            np.testing.assert_array_equal(gctx.ct_export(y), want)
        _same(octx, gctx, octx.rotate(o, 5, okeys), gctx.rotate(gkeys, g, 5))
        h = octx.hoist(o)
        for st, got in zip(steps, gctx.rotate_hoisted(gkeys, g, steps)):
            _same(octx, gctx, octx.rotate_hoisted(o, h, st, okeys), got)
    finally:
        gctx.close()
