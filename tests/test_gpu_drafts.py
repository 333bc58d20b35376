"""Rotary positions given with the call (cm_rotary_*), appended runs (cm_kv_append_run) and attention of a tree of drafted tokens (cm_tree_*):
limb for limb against the oracle, decrypted against float64 with the library's own plaintexts, replayed from graphs, and together.

Tolerances.  Words are equal.  Decrypted at scale 2^40 on the ring of 4096: a hoisted rotation leaves 2^6 units of noise a coefficient, 5e-8 a slot; a result
here has at most 300 of them behind one another or summed: 2e-5.  At 2^50 a thousandth of that."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
TOL = 2e-5


@pytest.fixture(scope="module")
def rings():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from oracle import ckks, params
    from paper_2602_11470_amd import binding as B
    wide = params.Params(n=4096, q=params.scan_primes(58, 4096, 1) + params.scan_primes(54, 4096, 5), p=params.scan_primes(60, 4096, 2), alpha=2, scale=2.0 ** 50,
                         hamming=0, name="wide")
    # ten digits of one prime; seven special primes (no ModDown and rescale in one, no third way of raising)
    digits = lambda: params.toy(n_qi=9)  # noqa: E731
    special = lambda: params.Params(n=4096, q=params.scan_primes(50, 4096, 8), p=params.scan_primes(60, 4096, 7), alpha=4, scale=2.0 ** 50, hamming=0, name="special")  # noqa: E731
    make = {"digits": (lambda: B.Context(4096, 10, 1, 1, 50, 40, 60, 2.0 ** 40), digits), "special": (lambda: B.Context(4096, 8, 7, 4, 50, 50, 60, 2.0 ** 50), special),
            "small": (B.config1, params.config1), "wide": (lambda: B.Context(4096, 6, 2, 2, 58, 54, 60, 2.0 ** 50), lambda: wide), "big": (B.llama_ring, None)}
    made = {}

    def get(name):
        if name not in made:
            g, o = make[name]
            made[name] = (g(), ckks.Context(o()) if o else None)
        return made[name]
    yield get
    for g, _ in made.values():
        g.close()


@pytest.fixture(scope="module")
def keysets(rings):
    """Secret and rotation keys of a ring on both sides; the oracle's are made as they are asked for."""
    made = {}

    def get(name, steps, relin=True):
        gctx, octx = rings(name)
        key = (name, tuple(sorted(set(steps))), relin)
        if key not in made:
            gsk = gctx.keygen_secret(1)
            osk = octx.keygen_secret(1) if octx else None
            made[key] = (gsk, gctx.keygen_rotations(gsk, list(key[1]), 2, with_relin=relin), osk,
                         octx.keygen_rotations(osk, key[1], 2, with_relin=relin) if octx else None)
        return made[key]
    return get


def _enc(rings, keys, name, slots, level, seed, oracle=True):
    gctx, octx = rings(name)
    c = gctx.encode_coeffs(slots, gctx.scale)
    g = gctx.encrypt(keys[0], gctx.pt_from_coeffs(c, level, gctx.scale), seed)
    return g, octx.encrypt(keys[2], octx.pt_from_coeffs(c, level, gctx.scale), seed) if oracle and octx else None


def _same(rings, name, g, o):
    gctx, octx = rings(name)
    assert g.level == o.level and abs(g.scale / o.scale - 1) < 1e-12
    np.testing.assert_array_equal(gctx.ct_export(g), octx.canonical(o))


def _words(c):
    return c.buf[: 2 * (c.level + 1) * c.ctx.n].view(2, c.level + 1, c.ctx.n)


def _table(gctx, tables, level):
    """Integer coefficients of the tables, given to both sides."""
    mods = [int(m) for m in gctx.moduli()]
    q, m2 = float(mods[level]), float(mods[gctx.L + 2] if gctx.K > 1 else mods[0])
    s, n = tables.slots(), 4 * tables.low + 1
    return np.stack([gctx.encode_coeffs(v, q) for v in s[:n]] + [gctx.encode_coeffs(v, m2) for v in s[n:]])


def _status(call):
    from paper_2602_11470_amd import binding as B
    try:
        call()
        return 0
    except B.CachemirError as e:
        return e.status


# ---- rotary positions ---------------------------------------------------------------------------------------------------
# ring, heads, dim, level, rot, halves, gain, room, ciphertexts
ROTARY = [("small", 4, 16, 2, 16, True, 1.0, 60, 1), ("small", 4, 16, 4, 16, False, 1.0, 37, 3), ("small", 3, 32, 1, 8, True, 1.3, 20, 2),
          ("small", 1, 2, 2, 2, False, 1.0, 5, 1), ("small", 8, 256, 3, 64, False, 0.25, 1, 2), ("wide", 4, 64, 5, 32, True, 1.0, 50, 2),
          ("wide", 16, 16, 3, 16, True, 1.0, 9, 9), ("digits", 8, 32, 8, 32, False, 1.0, 12, 2), ("special", 8, 32, 6, 16, False, 1.0, 12, 3),
          ("special", 8, 32, 2, 32, True, 1.0, 5, 1)]


@pytest.mark.parametrize("case", ROTARY, ids=str)
def test_rotary_matches_the_oracle(rings, keysets, case):
    """All residues, some, one, none: words of the oracle, and the slots of the textbook's rotation."""
    from oracle import packing, vmm
    ring, heads, dim, level, rot, halves, gain, room, count = case
    gctx, octx = rings(ring)
    tables = packing.RotaryTables(gctx.S, heads, dim, room, rot=rot, gain=gain, halves=halves)
    lay, coeffs, rng = tables.lay, _table(gctx, tables, level), np.random.default_rng(level)
    t = lay.t
    rotary = gctx.rotary(heads, dim, level, room, rot_dims=rot, gain=gain, halves=halves, coeffs=coeffs)
    assert rotary.steps() == ([tables.step] if 2 * tables.step == gctx.S else [tables.step, -tables.step])
    keys = keysets(ring, [tables.step, -tables.step], False)
    slots = rng.normal(size=(count, gctx.S))
    xs = [_enc(rings, keys, ring, v, level, 10 + i, oracle=i in (0, count - 1)) for i, v in enumerate(slots)]
    one = [-1] * t
    one[t - 1] = room - 1
    for k, positions in enumerate(([-1] * t, one, [int(p) for p in rng.integers(-1, room, t)])):
        gctx.rotary_set(rotary, positions, split=k % t)               # a split is none of apply's business
        outs = gctx.rotary_apply(keys[1], rotary, [g for g, _ in xs])
        if t <= 64 or k < 2:
            pts = vmm.rotary_plaintexts(octx, tables, coeffs, positions, level)
            for i in {0, count - 1}:
                _same(rings, ring, outs[i], vmm.rotary(octx, keys[3], tables, xs[i][1], pts))
        for i in {0, count // 2}:
            got = gctx.decrypt(keys[0], outs[i]).real.reshape(dim, lay.H, t)
            v = slots[i].reshape(dim, lay.H, t)
            for r in range(t):
                want = tables.turn(v[:, :, r].T, positions[r]).T if positions[r] >= 0 else 0.0
                assert np.abs(got[:, :, r] - want).max() < TOL


@pytest.mark.parametrize("heads, dim, level, rot, halves, scaling, room", [(32, 128, 3, 128, False, 0, 1000), (8, 128, 22, 64, True, 3, 300), (12, 64, 7, 64, True, 1, 77), (64, 512, 2, 2, False, 2, 4)])
def test_rotary_with_its_own_tables_on_the_full_ring(rings, keysets, heads, dim, level, rot, halves, scaling, room):
    """The library encodes the tables: queries and keys of a group at their own positions, against float64."""
    from oracle import packing
    from paper_2602_11470_amd import binding as B
    gctx, _ = rings("big")
    freq = B.rotary_freqs(rot, 500000.0, scaling, [4.0, 1.0, 8.0, 256.0])
    tables = packing.RotaryTables(gctx.S, heads, dim, room, rot=rot, freq=freq, gain=1.1, halves=halves)
    t, rng = tables.lay.t, np.random.default_rng(level)
    rotary = gctx.rotary(heads, dim, level, room, rot_dims=rot, freq=freq, gain=1.1, halves=halves)
    keys = keysets("big", rotary.steps(), False)
    slots = rng.normal(size=(2, gctx.S))
    xs = [_enc(rings, keys, "big", v, level, 5 + i)[0] for i, v in enumerate(slots)]
    positions = [int(p) for p in rng.integers(-1, room, t)]
    gctx.rotary_set(rotary, positions)
    for y, v in zip(gctx.rotary_apply(keys[1], rotary, xs), slots):
        got, v = gctx.decrypt(keys[0], y).real.reshape(dim, tables.lay.H, t), v.reshape(dim, tables.lay.H, t)
        for r in range(t):
            want = tables.turn(v[:, :, r].T, positions[r]).T if positions[r] >= 0 else 0.0
            assert np.abs(got[:, :, r] - want).max() < TOL / 1000


@pytest.mark.parametrize("level, halves", [(3, False), (6, False), (12, False), (12, True), (22, False)])
def test_ciphertexts_turned_together_are_those_turned_alone(rings, keysets, level, halves):
    """On the full ring, one to six digits, odd and even counts, more than a batch: word for word."""
    import torch
    from paper_2602_11470_amd import binding as B
    gctx, _ = rings("big")
    rotary = gctx.rotary(16, 64, level, 40, halves=halves, rot_dims=32)
    keys = keysets("big", rotary.steps(), False)
    gctx.rotary_set(rotary, [(7 * i) % 40 if i % 5 else -1 for i in range(rotary.residues)])
    gen = torch.Generator(device="cuda").manual_seed(level)
    xs = []
    for i in range(11):
        x = B.Ct(gctx, level)
        x.d.scale = gctx.scale
        for l, q in enumerate(gctx.moduli()[: level + 1]):
            _words(x)[:, l] = torch.empty(2, gctx.n, dtype=torch.int64, device="cuda").random_(0, int(q), generator=gen)
        xs.append(x)
    alone = [_words(gctx.rotary_apply(keys[1], rotary, [x])[0]).clone() for x in xs]
    for count in (2, 3, 8, 11):
        for y, want in zip(gctx.rotary_apply(keys[1], rotary, xs[:count]), alone):
            assert torch.equal(_words(y), want)
    twice = gctx.rotary_apply(keys[1], rotary, [xs[1], xs[1]])
    assert all(torch.equal(_words(y), alone[1]) for y in twice)


def test_rotary_is_the_embedding_of_one_token(rings, keysets):
    """What cm_rope_* does for one position and residue, and for a group."""
    gctx, _ = rings("small")
    H, E, level, token = 4, 16, 3, 45
    rotary = gctx.rotary(H, E, level, 100)
    t = rotary.residues
    rng = np.random.default_rng(3)
    keys = keysets("small", rotary.steps(), False)
    x, _ = _enc(rings, keys, "small", rng.normal(size=gctx.S), level, 3, oracle=False)
    for tau in (0, t - 1, -1):
        rope = gctx.rope(H, E, level, token, tau=tau)
        assert sorted(rope.steps()) == sorted(rotary.steps())
        gctx.rotary_set(rotary, [token + (r if tau < 0 else 0) if tau in (-1, r) else -1 for r in range(t)])
        a, b = (gctx.decrypt(keys[0], c) for c in (gctx.rope_apply(keys[1], rope, x), gctx.rotary_apply(keys[1], rotary, [x])[0]))
        assert np.abs(a - b).max() < TOL


def test_far_positions_of_a_large_table(rings, keysets):
    """The last positions of 2^17: angles of 131071 radians keep their digits (the angle's error is 2^-53 of it, 2e-11)."""
    from oracle import packing
    gctx, _ = rings("small")
    room = 1 << 17
    rotary = gctx.rotary(4, 16, 2, room, halves=True)
    tables = packing.RotaryTables(gctx.S, 4, 16, room, halves=True)
    t, rng = tables.lay.t, np.random.default_rng(0)
    keys = keysets("small", rotary.steps(), False)
    v = rng.normal(size=gctx.S)
    x, _ = _enc(rings, keys, "small", v, 2, 3, oracle=False)
    positions = [room - 1 - 17 * r if r % 3 else r for r in range(t)]
    gctx.rotary_set(rotary, positions)
    got, v = gctx.decrypt(keys[0], gctx.rotary_apply(keys[1], rotary, [x])[0]).real.reshape(16, 4, t), v.reshape(16, 4, t)
    assert max(np.abs(got[:, :, r] - tables.turn(v[:, :, r].T, positions[r]).T).max() for r in range(t)) < TOL


def test_rotary_refusals(rings, keysets):
    from paper_2602_11470_amd import binding as B
    gctx, _ = rings("small")
    lib, h = B.lib, C.c_void_p()
    f = np.ones(8)

    def create(heads=4, dim=16, level=2, rot=16, gain=1.0, room=16, flags=0, freq=f, ctx=gctx.h):
        s = lib.cm_rotary_create(ctx, heads, dim, level, rot, freq.ctypes.data if freq is not None else None, gain, room, flags, None, C.byref(h))
        if s == 0:
            lib.cm_rotary_destroy(h)
        return s
    assert create() == 0 and create(freq=None) == 0 and create(rot=2, room=1) == 0
    assert create(heads=0) == create(dim=1) == create(rot=3) == create(rot=0) == create(gain=0.0) == create(gain=np.inf) == create(room=0) == create(flags=2) == -1
    assert create(room=(1 << 24) + 1) == create(gain=np.nan) == create(freq=np.array([np.nan] + [1.0] * 7)) == create(ctx=None) == -1
    assert create(freq=np.full(8, 2.0 ** 49)) == create(freq=np.full(8, -np.inf)) == -1 and create(freq=np.full(8, -2.0 ** 48)) == 0      # 16 positions: 2^53
    assert create(gain=float(2 ** 19)) == -1                          # 2^19 q = 2^59, half of the special modulus
    assert create(level=0) == create(level=5) == -2
    assert create(rot=18) == create(dim=48, rot=16) == create(heads=256) == create(heads=4096, dim=2, rot=2) == -5
    equal = B.Context(4096, 3, 1, 1, 60, 60, 60, 2.0 ** 50)
    try:                                                              # special moduli no larger than the ciphertext's
        assert create(ctx=equal.h) == -1
    finally:
        equal.close()
    rotary = gctx.rotary(4, 16, 2, 16)
    t = rotary.residues
    keys = keysets("small", rotary.steps(), False)
    other = keysets("small", [1], False)
    x, y = B.Ct(gctx, 2), B.Ct(gctx, 1)
    for c in (x, y):
        c.buf.zero_()
    x.d.scale = gctx.scale

    def apply(xs, ys, evk=keys[1], r=rotary, count=None):
        a, b = ((B.cm_ct * max(1, len(v)))(*[c.d for c in v]) for v in (xs, ys))
        return lib.cm_rotary_apply(gctx.h, evk.h, r.h, len(xs) if count is None else count, a, b, None)
    assert apply([x], [y]) == -5                                      # no positions yet
    pos = np.full(t, 3, dtype=np.int32)

    def put(p, split=0):
        return lib.cm_rotary_set(gctx.h, rotary.h, p.ctypes.data, split, None)
    bad = pos.copy()
    for v in (16, -2):
        bad[t - 1] = v
        assert put(bad) == -5
    assert put(pos, -1) == put(pos, t) == -5 and apply([x], [y]) == -5
    assert put(pos) == 0 and apply([x], [y]) == 0
    assert apply([x], [y], evk=other[1]) == -4 and apply([x], [y], count=0) == apply([x], [y], count=65) == -1
    low, three = B.Ct(gctx, 1), B.Ct(gctx, 2, 3)
    assert apply([low], [y]) == -2 and apply([three], [y]) == -1
    assert apply([x], [x]) == apply([x, x], [y, y]) == -1
    part = B.Ct(gctx, 1)
    part.d.dev = x.d.dev + 8 * (2 * 3 * gctx.n - 1)                   # the last word of x
    assert apply([x], [part]) == -1
    assert apply([x, x], [y, B.Ct(gctx, 1)]) == 0                     # inputs may be the same
    wide, _ = rings("wide")
    assert lib.cm_rotary_set(wide.h, rotary.h, pos.ctypes.data, 0, None) == -1


# ---- appended runs --------------------------------------------------------------------------------------------------------
# ring, heads, dim, r_i, index, level, place, ntok, rotary
RUNS = [("small", 4, 16, 16, False, 2, 77, 1, ""), ("small", 4, 16, 4, True, 2, 90, 32, ""), ("small", 8, 32, 8, False, 2, 101, 6, "pairs"),
        ("small", 8, 32, 8, True, 2, 101, 8, "halves"), ("small", 8, 32, 32, False, 3, 248, 8, "halves"), ("small", 8, 32, 1, True, 2, 251, 5, "pairs"),
        ("small", 8, 256, 16, False, 2, 9, 1, "halves"), ("small", 3, 32, 16, False, 3, 13, 4, "pairs"), ("wide", 4, 64, 8, True, 3, 63, 2, "pairs"),
        ("wide", 4, 64, 16, False, 4, 60, 8, "halves"), ("digits", 8, 32, 8, False, 7, 45, 7, "pairs"),
        ("special", 8, 32, 8, False, 4, 45, 7, "pairs"), ("special", 8, 32, 4, True, 3, 45, 7, "halves"), ("small", 1, 16, 16, False, 2, 100, 100, "halves")]


def _masks(gctx, kv, lay, level):
    ones = np.zeros((2, lay.E, lay.H, lay.t))
    ones[0, :, :, 0], ones[1, 0, :, 0] = 1, 1
    coeffs = [gctx.encode_coeffs(m.reshape(-1), float(gctx.moduli()[level + 1])) for m in ones]
    for kind, c in zip((1, 2), coeffs):
        kv.set_mask(kind, c)
    return coeffs


def _at(t, run, split=None):
    """Positions at the residues: the place itself."""
    return [next((a for a in run if a % t == r), -1) for r in range(t)]


@pytest.mark.parametrize("stored_a, two_step", [(False, False), (True, True)])
@pytest.mark.parametrize("case", RUNS, ids=str)
def test_appended_runs_match_the_oracle(rings, keysets, case, stored_a, two_step):
    """Onto a cache that holds something: every ciphertext of it, those of other pages untouched."""
    import torch
    from oracle import packing, vmm
    from oracle.ckks import Ct
    from paper_2602_11470_amd import binding as B
    ring, heads, dim, r_i, index, level, place, ntok, form = case
    gctx, octx = rings(ring)
    lay = packing.KvLayout(gctx.S, heads, dim, r_i)
    t, Bs, rng = lay.t, lay.H * lay.t, np.random.default_rng(place)
    run = list(range(place, place + ntok))
    split = max(0, place % t + ntok - t)
    lk = level + 1 + bool(index and form)
    tables = packing.RotaryTables(gctx.S, heads, dim, place + ntok, halves=form == "halves")
    steps = [tables.step, -tables.step] + [j * Bs for j in range(1, r_i)] + [-g * r_i * Bs for g in range(1, lay.r_o)]
    keys = keysets(ring, steps, False)
    gctx.set_option(B.CM_OPT_EVK_STORED_A, stored_a)
    gctx.set_option(B.CM_OPT_TWO_STEP_MASKS, two_step)
    try:
        evk = gctx.keygen_rotations(keys[0], steps, 2) if stored_a else keys[1]
        kv = gctx.kv_create(heads, dim, level, r_i=r_i, key_index=index)
        masks = [octx.pt_from_coeffs(c, level + 1, float(octx.mod[level + 1])) for c in _masks(gctx, kv, lay, level)]
        k, ok = _enc(rings, keys, ring, rng.normal(size=gctx.S), lk, 3)
        v, ov = _enc(rings, keys, ring, rng.normal(size=gctx.S), level + 1, 4)
        rotary, turned = None, None
        if form:
            coeffs = _table(gctx, tables, lk)
            rotary = gctx.rotary(heads, dim, lk, place + ntok, halves=form == "halves", coeffs=coeffs)
            gctx.rotary_set(rotary, _at(t, run), split)
            turn = lambda part: vmm.rotary(octx, keys[3], tables, ok, vmm.rotary_plaintexts(octx, tables, coeffs, _at(t, part), lk))  # noqa: E731
            if index:
                ok = turn(run)
            else:
                turned = [turn([a for a in run if a // t == p]) for p in sorted({a // t for a in run})]
        # what the cache holds already: uniform residues
        which = [B.CM_QK, B.CM_SV] + ([B.CM_KV_INDEX] if index else [])
        gen = torch.Generator(device="cuda").manual_seed(9)
        for w in which:
            for i, q in enumerate(gctx.moduli()[: level + 1]):
                kv.words(w)[..., i, :] = torch.empty(kv.words(w).shape[:-2] + (gctx.n,), dtype=torch.int64, device="cuda").random_(0, int(q), generator=gen)
        before = {w: [kv.export(w, i) for i in range(dim)] for w in which}

        def held(w):
            idx = octx.q_idx(level)
            return [Ct([octx.ntt(c, idx) for c in b], level, gctx.scale) for b in before[w]]
        k_cts, v_cts, x_cts = held(B.CM_QK), held(B.CM_SV), held(B.CM_KV_INDEX) if index else None
        vmm.kv_append_run(octx, keys[3], lay, k_cts, v_cts, place, ntok, ok, ov, *masks, turned, x_cts)
        kv.set_tokens(place)
        kv.append_run(evk, k, v, ntok, rotary=rotary)
        assert kv.tokens() == place + ntok
        for w, want in zip(which, (k_cts, v_cts, x_cts)):
            for i in range(dim):
                if w == B.CM_QK and i not in {a // t for a in run}:
                    np.testing.assert_array_equal(kv.export(w, i), before[w][i])
                else:
                    np.testing.assert_array_equal(kv.export(w, i), octx.canonical(want[i]))
    finally:
        gctx.set_option(B.CM_OPT_EVK_STORED_A, 0)
        gctx.set_option(B.CM_OPT_TWO_STEP_MASKS, 0)


@pytest.mark.parametrize("index", [False, True])
def test_a_run_of_one_is_a_single_append(rings, keysets, index):
    """Word for word, at several residues of a page; and places filled again behind cm_kv_seek."""
    import torch
    from paper_2602_11470_amd import binding as B
    gctx, _ = rings("small")
    a, b = (gctx.kv_create(8, 32, 3, r_i=8, key_index=index) for _ in range(2))
    keys = keysets("small", a.steps(), True)
    rng = np.random.default_rng(2)
    for kv in (a, b):
        kv.set_tokens(6)
    for i in range(4):
        k, v = (_enc(rings, keys, "small", rng.normal(size=gctx.S), 4, 20 + 2 * i + j, oracle=False)[0] for j in (0, 1))
        if i == 3:
            a.seek(100), b.seek(100)
        a.append(keys[1], k, v)
        b.append_run(keys[1], k, v, 1)
    assert a.tokens() == b.tokens() == 101
    for w in [B.CM_QK, B.CM_SV] + ([B.CM_KV_INDEX] if index else []):
        assert torch.equal(a.words(w), b.words(w))


def test_append_run_refusals(rings, keysets):
    from paper_2602_11470_amd import binding as B
    gctx, _ = rings("small")
    kv = gctx.kv_create(8, 32, 2, r_i=8, max_tokens=40)
    indexed = gctx.kv_create(8, 32, 2, r_i=8, key_index=True)
    t, half = 8, 16 * 8 * 8
    rotary, high = gctx.rotary(8, 32, 3, 64, halves=True), gctx.rotary(8, 32, 4, 64, halves=True)
    keys = keysets("small", kv.steps() + [half], True)
    few, no_turn = keysets("small", [half], False), keysets("small", [-g * half // 2 for g in (1, 2, 3)], False)
    cts = {}
    for level in (2, 3, 4):
        cts[level] = B.Ct(gctx, level)
        cts[level].buf.zero_()
        cts[level].d.scale = gctx.scale
    k, v = cts[3], B.Ct(gctx, 3)
    v.buf.zero_()
    v.d.scale = gctx.scale
    run = lambda ntok=3, k=k, v=v, r=None, evk=keys[1], kv=kv: _status(lambda: kv.append_run(evk, k, v, ntok, rotary=r))  # noqa: E731
    kv.set_tokens(5)
    assert run(0) == run(9) == run(-1) == -5
    assert run(k=cts[2]) == run(v=cts[2]) == run(k=cts[4]) == run(r=high) == -2
    assert run(evk=few[1]) == -4
    three = B.Ct(gctx, 3, 3)
    assert run(k=three) == -1
    other = B.Ct(gctx, 3)
    other.d.scale = 2 * gctx.scale
    assert run(v=other) == -3
    assert run(r=rotary) == -5                                        # no positions
    gctx.rotary_set(rotary, [-1] * 5 + [1, 2, 3])
    pairs = gctx.rotary(8, 32, 3, 64)
    gctx.rotary_set(pairs, [-1] * 5 + [1, 2, 3])
    assert run(r=pairs, evk=no_turn[1]) == -4
    assert run(2, r=rotary) == run(4, r=rotary) == -5                 # other residues
    narrow = gctx.rotary(8, 64, 3, 64)
    gctx.rotary_set(narrow, [0] * narrow.residues)
    assert run(r=narrow) == -5
    kv.set_tokens(6)
    gctx.rotary_set(rotary, [3, -1, -1, -1, -1, -1, 1, 2], split=0)
    assert run(r=rotary) == -5                                        # the run passes into the next page: split is 1
    gctx.rotary_set(rotary, [3, -1, -1, -1, -1, -1, 1, 2], split=2)
    assert run(r=rotary) == -5
    gctx.rotary_set(rotary, [3, -1, -1, -1, -1, -1, 1, 2], split=1)
    assert kv.tokens() == 6 and run(r=rotary) == 0 and kv.tokens() == 9
    kv.set_tokens(38)
    assert run(3) == -5 and run(2) == 0                               # room for 40
    assert run(1) == -5
    indexed.set_tokens(0)
    gctx.rotary_set(high, [0, 1, 2] + [-1] * 5)
    gctx.rotary_set(rotary, [0, 1, 2] + [-1] * 5)
    assert run(r=rotary, kv=indexed) == -2 and run(r=high, kv=indexed) == -2      # rotated keys of an index come two levels above it
    assert run(r=high, k=cts[4], kv=indexed) == 0
    top = gctx.kv_create(8, 32, 4, r_i=8)
    assert run(kv=top) == -2
    wide, _ = rings("wide")
    assert B.lib.cm_kv_append_run(wide.h, keys[1].h, kv.h, None, 1, C.byref(k.d), C.byref(v.d), None) == -1


# ---- trees -----------------------------------------------------------------------------------------------------------------
# ring, heads, dim, group, r_i, level, form, base, parents, node0, first
TREES = [("small", 8, 32, 1, 8, 3, "index", 101, [-1, 0, 0, 1, -1, 3], 0, 64), ("small", 8, 32, 2, 8, 3, "index", 101, [-1, 0, 0, 1, -1, 3], 3, 0),
         ("small", 16, 32, 4, 32, 3, "index unrolled", 16, [-1], 0, 16), ("small", 8, 128, 1, 16, 3, "index unrolled", 250, [-1, 0, 1, 2, 3, 3], 2, 128),
         ("small", 16, 128, 1, 16, 2, "index", 30, [-1, 0], 1, 0), ("small", 8, 16, 1, 4, 3, "", 13, [-1, 0, 1], 0, 0), ("small", 8, 16, 2, 16, 3, "unrolled", 16, [-1, -1, 1], 0, 0),
         ("small", 8, 32, 1, 2, 3, "index unrolled", 40, [-1, 0, 1], 0, 0), ("digits", 8, 32, 1, 8, 7, "index unrolled", 40, [-1, 0, 1], 0, 0),
         ("special", 8, 32, 2, 8, 5, "index unrolled", 40, [-1, 0, 1], 0, 0), ("special", 8, 32, 1, 16, 3, "index", 40, [-1, 0, 1], 0, 0),
         ("wide", 6, 32, 1, 8, 3, "index unrolled", 0, [-1, 0, 0, 1], 0, 0), ("wide", 4, 32, 16, 8, 2, "index", 511 - 16, [-1] * 17, 5, 0)]


@pytest.mark.parametrize("case", TREES, ids=str)
def test_tree_matches_the_oracle(rings, keysets, case):
    """Scores and values, in the cache's forms of the products; masks that leave a query nothing but itself among them."""
    from oracle import packing, vmm
    from paper_2602_11470_amd import binding as B
    ring, heads, dim, group, r_i, level, form, base, parents, node0, first = case
    gctx, octx = rings(ring)
    lay, mask = packing.KvLayout(gctx.S, heads, dim, r_i), -24.0
    t, H, rng, ntok = lay.t, lay.H, np.random.default_rng(base), base + len(parents)
    index, unrolled = "index" in form, "unrolled" in form
    kv = gctx.kv_create(heads, dim, level, r_i=r_i, key_index=index, unrolled_ladders=unrolled)
    mods = [float(m) for m in gctx.moduli()]
    scale = gctx.scale ** 2 / mods[level]
    moves = [[gctx.encode_coeffs((np.arange(gctx.S) % t >= d).astype(float), mods[lv]) for d in range(1, t)] for lv in (level + 1, level - 1)]
    one, row = np.zeros((2, dim, H, t))
    one[0, :, 0] = row[0] = mask
    one, row = (gctx.encode_coeffs(m.reshape(-1), scale) for m in (one, row))
    tree = gctx.tree(kv, group=group, mask=mask, coeffs=np.stack(moves[0] + moves[1] + [one, row]))
    assert tree.passes == t
    steps = kv.steps() + tree.steps()
    keys = keysets(ring, steps, True)
    okeys, ls = keys[3], level - (1 if index else 2)
    ops = vmm.CkksOps(octx, okeys)
    sv = (lambda x, cts: vmm.score_times_v_unrolled(octx, okeys, lay, x, cts, reduce=False)) if unrolled else \
        (lambda x, cts: vmm.score_times_v(ops, lay, x, cts, reduce=False))
    K, V = 0.3 * rng.normal(size=(2, ntok, heads, dim))
    load = lambda w, cts: [kv.load(w, i, g) for i, (g, _) in enumerate(cts)]  # noqa: E731
    v_cts = [_enc(rings, keys, ring, lay.pack_v(V, k), level, 50 + k) for k in range(dim)]
    load(B.CM_SV, v_cts)
    if index:
        cts = [_enc(rings, keys, ring, lay.pack_k_index(K, k), level, 200 + k) for k in range(dim)]
        load(B.CM_KV_INDEX, cts)
        product = lambda x: sv(x, [o for _, o in cts])  # noqa: E731
    else:
        cts = [_enc(rings, keys, ring, lay.pack_k(K, c), level, 200 + c) for c in range(-(-ntok // t))]
        load(B.CM_QK, cts)
        copy = np.zeros((dim, H, t))
        copy[0] = 1
        copy = gctx.encode_coeffs(copy.reshape(-1), mods[level - 1])
        kv.set_mask(0, copy)
        idx = octx.q_idx(level - 1)
        from oracle.ckks import Pt
        qk_masks = []
        for c in range(len(cts)):
            m = octx.automorphism(octx.ntt(octx.from_i64(copy, idx), idx), idx, octx.galois(-c * H * t))
            qk_masks.append(Pt(m, level - 1, mods[level - 1]))
        if unrolled:
            product = lambda x: vmm.qk_scores_unrolled(octx, okeys, lay, x, [o for _, o in cts], qk_masks, replicate=False)  # noqa: E731
        else:
            product = lambda x: vmm.qk_scores(ops, lay, x, [o for _, o in cts], qk_masks, replicate=False)  # noqa: E731
    kv.set_tokens(ntok)
    hidden = [packing.tree_hidden(lay, group, parents, base, node0, first, d) for d in range(t)]
    idx, page, last = octx.q_idx(ls), base // t, (ntok - 1) // t
    turned = lambda c, step: octx.automorphism(octx.ntt(octx.from_i64(c, idx), idx), idx, octx.galois(step))  # noqa: E731
    pts = []
    for d in range(t):
        m = np.zeros((ls + 1, octx.n), dtype=np.uint64)
        for c in range(dim):
            if not first // t <= c <= last:
                m = octx.add(m, turned(row, -c * H * t), idx)
            elif c >= page:
                for j in np.nonzero(hidden[d][c, 0])[0]:
                    m = octx.add(m, turned(one, -(c * H * t + int(j))), idx)
        pts.append(m)
    qs = 0.3 * rng.normal(size=gctx.S)
    q, oq = _enc(rings, keys, ring, qs, level + 1, 5)
    want = vmm.tree_qk(octx, okeys, lay, oq, moves[0], product, pts)
    got = gctx.tree_qk(keys[1], tree, kv, parents, base, q, node0=node0, first=first)
    Kp = np.concatenate([K, np.zeros((lay.capacity - ntok, heads, dim))]).reshape(dim, t, heads, dim)
    for d in range(t):
        _same(rings, ring, got[d], want[d])
        moved = np.roll(qs.reshape(dim, H, t), d, axis=2)[:, :heads]
        plain = np.einsum("chje,ehj->chj", Kp.transpose(0, 2, 1, 3), moved) + mask * hidden[d][:, :heads]
        assert np.abs(gctx.decrypt(keys[0], got[d]).real.reshape(dim, H, t)[:, :heads] - plain).max() < TOL
    s = 0.3 * rng.normal(size=(t, dim, H, t))
    scores = [_enc(rings, keys, ring, s[d].reshape(-1), level, 80 + d) for d in range(t)]
    out = gctx.tree_sv(keys[1], tree, kv, [g for g, _ in scores])
    _same(rings, ring, out, vmm.tree_sv(octx, okeys, lay, [o for _, o in scores], moves[1], lambda x: sv(x, [o for _, o in v_cts])))
    Vp = np.concatenate([V, np.zeros((lay.capacity - ntok, heads, dim))]).reshape(dim, t, heads, dim)
    plain = sum(np.roll(np.einsum("chj,cjhe->ehj", s[d][:, :heads], Vp), -d, axis=2) for d in range(t))
    assert np.abs(gctx.decrypt(keys[0], out).real.reshape(dim, H, t)[:, :heads] - plain).max() < TOL


def test_tree_refusals(rings, keysets):
    from paper_2602_11470_amd import binding as B
    gctx, _ = rings("small")
    lib, h = B.lib, C.c_void_p()
    kv = gctx.kv_create(8, 32, 3, r_i=8, key_index=True)

    def create(kv=kv, group=1, mask=-24.0, scale=0.0, ctx=gctx):
        s = lib.cm_tree_create(ctx.h, kv.h, group, mask, scale, None, C.byref(h))
        if s == 0:
            lib.cm_tree_destroy(h)
        return s
    assert create() == create(group=8) == create(mask=0.0) == 0
    assert create(group=0) == create(mask=np.nan) == create(scale=np.inf) == create(scale=-1.0) == create(mask=2.0 ** 21) == create(ctx=rings("wide")[0]) == -1
    assert create(group=3) == create(group=16) == create(kv=gctx.kv_create(1, 16, 3)) == -5        # 128 residues
    assert create(kv=gctx.kv_create(8, 32, 4, r_i=8)) == -2
    tree = gctx.tree(kv)
    t = tree.passes
    keys = keysets("small", kv.steps() + tree.steps(), True)
    part = keysets("small", kv.steps(), True)
    kv.set_tokens(50)
    q = B.Ct(gctx, 4)
    q.buf.zero_()
    q.d.scale = gctx.scale
    scores = [B.Ct(gctx, 2) for _ in range(t)]

    def qk(parents=(-1, 0, 0), base=40, node0=0, first=0, q=q, evk=keys[1], kv=kv, tree=tree, outs=scores):
        p = np.array(parents, dtype=np.int32)
        return _status(lambda: gctx.tree_qk(evk, tree, kv, p, base, q, node0=node0, first=first, outs=outs))
    assert qk() == qk(base=47) == qk(base=0) == qk(first=40) == qk(node0=2) == 0
    assert qk(base=48) == qk(base=-1) == qk(node0=3) == qk(node0=-1) == qk(first=4) == qk(first=48) == qk(first=-8) == qk(parents=[-1] * 51, base=0) == -5
    assert qk(parents=[0]) == qk(parents=[-1, 1]) == qk(parents=[-1, -2]) == -1
    assert _status(lambda: gctx.tree_qk(keys[1], tree, kv, np.zeros(0, dtype=np.int32), 40, q, outs=scores)) == -5
    low = B.Ct(gctx, 3)
    low.d.scale = gctx.scale
    assert qk(q=low) == -2 and qk(evk=part[1]) == -4 and qk(q=B.Ct(gctx, 4, 3)) == -1
    far = B.Ct(gctx, 4)
    far.d.scale = 2 * gctx.scale
    assert qk(q=far) == -3
    assert qk(outs=scores[:-1] + [scores[0]]) == -1
    same = B.Ct(gctx, 2)
    same.d.dev = q.d.dev
    assert qk(outs=scores[:-1] + [same]) == -1
    other = gctx.kv_create(8, 64, 3, r_i=8, key_index=True)
    other.set_tokens(50)
    assert qk(kv=other) == -5
    lower = gctx.kv_create(8, 32, 2, r_i=8, key_index=True)
    lower.set_tokens(50)
    assert qk(kv=lower) == -2
    at = [B.Ct(gctx, 3) for _ in range(t)]
    for c in at:
        c.buf.zero_()
        c.d.scale = gctx.scale
    out = B.Ct(gctx, 1)
    sv = lambda s, evk=keys[1], kv=kv: _status(lambda: gctx.tree_sv(evk, tree, kv, s, out=out))  # noqa: E731
    assert sv(at) == 0 and out.level == 1
    assert sv(at, evk=part[1]) == -4 and sv(at, kv=other) == -5 and sv(at, kv=lower) == -2 and sv(at[:-1] + [q]) == -2
    at[3].d.scale *= 2
    assert sv(at) == -3


@pytest.mark.parametrize("ring, heads, dim, level", [("small", 8, 32, 2), ("big", 32, 128, 3)])
def test_products_of_extreme_words(rings, keysets, ring, heads, dim, level):
    """Pass 0 of the joint products against the single one, sixteen equal terms a sum: a query without second component keeps its constant words
    under rotation.  Halves of the modulus on either side, its largest word, and factors whose product is halfway between two multiples."""
    import torch
    from paper_2602_11470_amd import binding as B
    gctx, _ = rings(ring)
    kv = gctx.kv_create(heads, dim, level, r_i=16, key_index=True, unrolled_ladders=True)
    tree = gctx.tree(kv, mask=0.0, scale=gctx.scale ** 2 / float(gctx.moduli()[level]))
    keys = keysets(ring, kv.steps() + tree.steps(), True)
    kv.set_tokens(2 * tree.passes)
    q, mods = B.Ct(gctx, level + 1), [int(m) for m in gctx.moduli()]
    q.d.scale = gctx.scale
    pairs = [lambda m: (m // 2, m // 2), lambda m: (m // 2 + 1, m // 2), lambda m: (m // 2 + 1, m // 2 + 1), lambda m: (m - 1, m - 1),
             lambda m: (m // 2 - 1, m // 2 * pow(m // 2 - 1, -1, m) % m), lambda m: (m // 3, (m // 2 + 1) * pow(m // 3, -1, m) % m)]
    index = kv.words(B.CM_KV_INDEX)
    for pair in pairs:
        _words(q).zero_()
        for l in range(level + 2):
            _words(q)[0, l] = pair(mods[l])[0]
            if l <= level:
                index[..., l, :] = pair(mods[l])[1]
        scores = gctx.tree_qk(keys[1], tree, kv, [-1], 2 * tree.passes - 1, q)
        single = gctx.vmm_kv(keys[1], kv, B.CM_QK_GROUP, gctx.level_drop(q, level))
        assert torch.equal(_words(scores[0]), _words(single))


@pytest.mark.parametrize("ring, heads, dim, r_i, level", [("small", 8, 32, 8, 2), ("big", 64, 64, 16, 2)])
def test_stored_key_halves_give_the_same_words(rings, ring, heads, dim, r_i, level):
    """Keys with both halves stored (CM_OPT_EVK_STORED_A) go through kernels of their own."""
    import torch
    from paper_2602_11470_amd import binding as B
    gctx, _ = rings(ring)
    kv = gctx.kv_create(heads, dim, level, r_i=r_i, key_index=True, unrolled_ladders=True)
    pairs, tree = [gctx.rotary(heads, dim, level + 2, 32, halves=h) for h in (False, True)], gctx.tree(kv)
    t = tree.passes
    sk = gctx.keygen_secret(1)
    steps = kv.steps() + tree.steps() + pairs[0].steps() + pairs[1].steps()
    gen = torch.Generator(device="cuda").manual_seed(3)

    def uniform(words):
        for i in range(words.shape[-2]):
            words[..., i, :] = torch.empty(words.shape[:-2] + (gctx.n,), dtype=torch.int64, device="cuda").random_(0, int(gctx.moduli()[i]), generator=gen)

    def ct(lv):
        c = B.Ct(gctx, lv)
        c.d.scale = gctx.scale
        uniform(_words(c))
        return c
    x, k, v, q, weights = [ct(level + 2) for _ in range(3)], ct(level + 2), ct(level + 1), ct(level + 1), [ct(level) for _ in range(t)]
    cache = [kv.words(w) for w in (B.CM_QK, B.CM_SV, B.CM_KV_INDEX)]
    for w in cache:
        uniform(w)
    before, found = [w.clone() for w in cache], []
    try:
        for stored in (0, 1):
            gctx.set_option(B.CM_OPT_EVK_STORED_A, stored)
            keys = gctx.keygen_rotations(sk, steps, 2, with_relin=True)
            out = []
            for w, b in zip(cache, before):
                w.copy_(b)
            kv.set_tokens(2 * t + 1)
            for r in pairs:
                gctx.rotary_set(r, [i if i % 3 else -1 for i in range(t)])
                out += gctx.rotary_apply(keys, r, x)
            gctx.rotary_set(pairs[1], [-1] + [3] * 3 + [-1] * (t - 4))
            kv.append_run(keys, k, v, 3, rotary=pairs[1])
            out += gctx.tree_qk(keys, tree, kv, [-1, 0, 0], 2 * t + 1, q) + [gctx.tree_sv(keys, tree, kv, weights)]
            found.append([_words(c).clone() for c in out] + [w.clone() for w in cache])
            del keys
    finally:
        gctx.set_option(B.CM_OPT_EVK_STORED_A, 0)
    assert all(torch.equal(a, b) for a, b in zip(*found))


def test_a_drafting_step_on_the_full_ring(rings, keysets):
    """64 heads of 64 dims: a prompt of nine tokens and five drafted ones appended with their positions, the scores and values of their queries."""
    from oracle import packing
    gctx, _ = rings("big")
    H, E, level = 64, 64, 3
    lay = packing.KvLayout(gctx.S, H, E, 16)
    tables = packing.RotaryTables(gctx.S, H, E, 32, halves=True)
    t, rng = lay.t, np.random.default_rng(1)
    kv = gctx.kv_create(H, E, level, r_i=16, key_index=True, unrolled_ladders=True)
    rotary, tree = gctx.rotary(H, E, level + 2, 32, halves=True), gctx.tree(kv)
    keys = keysets("big", kv.steps() + tree.steps() + rotary.steps(), True)
    enc = lambda slots, lv: _enc(rings, keys, "big", slots, lv, int(rng.integers(1 << 30)))[0]  # noqa: E731
    K, V = np.zeros((2, lay.capacity, H, E))
    parents, depth = [-1, 0, 0, 2, 1], [0, 1, 1, 2, 2]
    place = 0
    for positions in (range(8), [8], [9 + d for d in depth]):
        ks, vs = 0.3 * rng.normal(size=(2, E, H, t))
        at = [-1] * t
        for i, p in enumerate(positions):
            a = place + i
            at[a % t] = p
            K[a], V[a] = tables.turn(ks[:, :, a % t].T, p), vs[:, :, a % t].T
        gctx.rotary_set(rotary, at, max(0, place % t + len(positions) - t))
        kv.append_run(keys[1], enc(ks.reshape(-1), level + 2), enc(vs.reshape(-1), level + 1), len(positions), rotary=rotary)
        place += len(positions)
    assert place == 14 and kv.tokens() == 14
    qs = 0.3 * rng.normal(size=(E, H, t))
    scores = gctx.tree_qk(keys[1], tree, kv, parents, 9, enc(qs.reshape(-1), level + 1))
    Kp, Vp = K.reshape(E, t, H, E), V.reshape(E, t, H, E)
    s = 0.3 * rng.normal(size=(t, E, H, t))
    want = np.zeros((E, H, t))
    for d in range(t):
        plain = np.einsum("chje,ehj->chj", Kp.transpose(0, 2, 1, 3), np.roll(qs, d, axis=2)) - 24.0 * packing.tree_hidden(lay, 1, parents, 9, 0, 0, d)
        # scale 2^50: noise of 2^6 units a coefficient times the 64 products of a sum
        assert np.abs(gctx.decrypt(keys[0], scores[d]).real.reshape(E, H, t) - plain).max() < TOL / 100
        want += np.roll(np.einsum("chj,cjhe->ehj", s[d], Vp), -d, axis=2)
    out = gctx.tree_sv(keys[1], tree, kv, [enc(s[d].reshape(-1), level) for d in range(t)])
    assert out.level == 1 and np.abs(gctx.decrypt(keys[0], out).real.reshape(E, H, t) - want).max() < TOL / 100


# ---- replayed, on other streams, together --------------------------------------------------------------------------------
@pytest.mark.parametrize("ring, heads, dim, r_i, level", [("small", 8, 32, 8, 2), ("big", 64, 64, 16, 2)])
def test_captured_and_replayed(rings, keysets, ring, heads, dim, r_i, level):
    """A drafting step in one graph, captured on a stream of its own: positions, an appended run, scores, values; replayed with
    other inputs and the same calls made eagerly in between."""
    import torch
    from paper_2602_11470_amd import binding as B
    gctx, _ = rings(ring)
    index = True
    kv = gctx.kv_create(heads, dim, level, r_i=r_i, key_index=index, unrolled_ladders=True)
    t = gctx.S // (heads * dim)
    rotary, qrot, tree = gctx.rotary(heads, dim, level + 2, 64, halves=True), gctx.rotary(heads, dim, level + 2, 64, halves=True), gctx.tree(kv, scale=0.0)
    keys = keysets(ring, kv.steps() + tree.steps() + rotary.steps(), True)
    base, parents = 5 * t + t // 2, [-1] + [0] * (t // 2)
    n = len(parents)
    run = range(base, base + n)
    positions = [next((base + (a > base) for a in run if a % t == r), -1) for r in range(t)]
    split = max(0, base % t + n - t)

    def ct(lv):
        c = B.Ct(gctx, lv)
        c.d.scale = gctx.scale
        return c
    k, q, v, qr = ct(level + 2), ct(level + 2), ct(level + 1), ct(level + 1)
    scores, weights, out = [ct(level - 1) for _ in range(t)], [ct(level) for _ in range(t)], ct(level - 2)
    words = [_words(c) for c in [k, q, v] + weights] + [kv.words(w) for w in (B.CM_QK, B.CM_SV, B.CM_KV_INDEX)]

    def fill(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for w in words:
            for i in range(w.shape[-2]):
                w[..., i, :] = torch.empty(w.shape[:-2] + (gctx.n,), dtype=torch.int64, device="cuda").random_(0, int(gctx.moduli()[i]), generator=gen)

    def work():
        gctx.rotary_set(rotary, positions, split)
        gctx.rotary_set(qrot, positions)
        gctx.rotary_apply(keys[1], qrot, [q], outs=[qr])
        kv.seek(base)
        kv.append_run(keys[1], k, v, n, rotary=rotary)
        gctx.tree_qk(keys[1], tree, kv, parents, base, qr, outs=scores)
        gctx.tree_sv(keys[1], tree, kv, weights, out=out)

    def results():
        return [_words(c).clone() for c in scores + [out]] + [kv.words(w).clone() for w in (B.CM_QK, B.CM_SV, B.CM_KV_INDEX)]
    fill(1)
    work()
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        work()
    for seed in (2, 3, 4):
        fill(seed)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = results()
        fill(seed)
        gctx.rotary_set(rotary, [0] * t)                              # other positions in between
        work()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, results()))


@pytest.mark.parametrize("heads, dim, r_i, group", [(8, 32, 8, 1), (4, 32, 8, 2)])
def test_a_drafting_session(rings, heads, dim, r_i, group):
    """A prompt appended in runs, a tree drafted behind it, its attention (softmax in the clear in between), the rejected tokens dropped, a second
    tree: after every step the attention of every query is float64's."""
    from oracle import packing
    from paper_2602_11470_amd import binding as B
    ctx = B.Context(4096, 9, 2, 2, 50, 50, 60, 2.0 ** 50)
    try:
        lay = packing.KvLayout(ctx.S, heads, dim, r_i)
        H, t, rng, room = lay.H, lay.t, np.random.default_rng(7), 64
        tables = packing.RotaryTables(ctx.S, heads, dim, room, halves=True)
        sk = ctx.keygen_secret(1)
        caches = [ctx.kv_create(heads, dim, lv, r_i=r_i, key_index=True, unrolled_ladders=True) for lv in (6, 5)]
        trees = [ctx.tree(c, group=group) for c in caches]
        rots = {lv: ctx.rotary(heads, dim, lv, room, halves=True) for lv in (8, 7)}
        keys = ctx.keygen_rotations(sk, caches[0].steps() + trees[0].steps() + rots[8].steps(), 2, with_relin=True)
        seeds = iter(range(100, 1000))
        enc = lambda slots, lv: ctx.encrypt(sk, ctx.encode(slots, lv), next(seeds))  # noqa: E731
        K, V = np.zeros((2, 0, heads, dim))

        def append(kv, rot, place, positions):
            """Tokens at place, place + 1, ..; returns their keys and values."""
            nonlocal K, V
            n = len(positions)
            ks, vs = 0.3 * rng.normal(size=(2, dim, H, t))
            at = [-1] * t
            for i, p in enumerate(positions):
                r = (place + i) % t
                at[r] = p
                K, V = np.concatenate([K, tables.turn(ks[:, :heads, r].T, p)[None]]), np.concatenate([V, vs[:, :heads, r].T[None]])
            ctx.rotary_set(rot, at, max(0, place % t + n - t))
            kv.append_run(keys, enc(ks.reshape(-1), rot.level), enc(vs.reshape(-1), kv.level + 1), n, rotary=rot)
            assert kv.tokens() == len(K) == place + n

        def attend(kv, tree, base, parents, node0, first):
            qs = 0.3 * rng.normal(size=(dim, H, t))
            scores = ctx.tree_qk(keys, tree, kv, parents, base, enc(qs.reshape(-1), kv.level + 1), node0=node0, first=first)
            s = np.stack([ctx.decrypt(sk, c).real.reshape(dim, H, t)[:, :heads] for c in scores])
            per, ntok = t // group, base + len(parents)
            probs, want = np.zeros((t, dim, H, t)), np.zeros((dim, heads, t))
            for u in range(t):                                            # the query in slot u: its scores over the passes
                node = node0 + (u % per - base - node0) % per
                seen = set(range(first, base))
                k = node if node < len(parents) else -1
                while k >= 0:
                    seen.add(base + k)
                    k = parents[k]
                places = [(p, p // t, p % t, (p % t - u) % t) for p in range(lay.capacity)]
                row = np.stack([s[d, c, :, j] for _, c, j, d in places])
                e = np.exp(row - row.max(0))
                w = e / e.sum(0)
                hidden = [p for p, _, _, _ in places if p not in seen]
                # exp(-24 + what scores differ by, at most 8) of at most 512 places
                assert w[hidden].max() < 1e-4 if seen else True
                for p, c, j, d in places:
                    probs[d, c, :heads, j] = w[p] if p in seen else 0.0
                exact = np.array([[K[p, h] @ qs[:, h, u] for h in range(heads)] for p in sorted(seen)]) if seen else np.zeros((1, heads))
                e = np.exp(exact - exact.max(0))
                if seen:
                    want[:, :, u] = np.einsum("ph,phe->eh", e / e.sum(0), V[sorted(seen)])
            out = ctx.tree_sv(keys, tree, kv, [enc(probs[d].reshape(-1), kv.level) for d in range(t)])
            got = ctx.decrypt(sk, out).real.reshape(dim, H, t)[:, :heads]
            assert np.abs(got - want).max() < 1e-3                        # the hidden places' share of the sums of exponentials

        kv, tree = caches[0], trees[0]
        place = 0
        for n in (t, t, 3):                                               # a prompt of 2 t + 3 tokens
            append(kv, rots[8], place, range(place, place + n))
            place += n
        parents = [-1, 0, 0, 1, 2][: t]
        depth = []
        for p in parents:
            depth.append(0 if p < 0 else depth[p] + 1)
        base = place
        append(kv, rots[8], base, [base + d for d in depth])
        attend(kv, tree, base, parents, 0, 0)
        attend(kv, tree, base, parents, 1, t)
        # tokens 0, 2, 4 are accepted: the others leave (their places stay empty until the next tokens fill what follows)
        keep = np.ones(len(K), dtype=bool)
        keep[[base + 1, base + 3]] = False
        ctx.kv_take(None, ctx.kv_sel(kv, keep), kv, caches[1])
        K[~keep], V[~keep] = 0, 0
        kv, tree = caches[1], trees[1]
        base = len(K)
        append(kv, rots[7], base, [base])
        attend(kv, tree, base, [-1], 0, 0)
    finally:
        ctx.close()
