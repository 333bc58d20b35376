"""Rotary positions by tables, appended runs and attention of a tree (oracle/vmm.py): decrypted against float64; and what the library's
calls for them do without a GPU.

Tolerances.  Scale 2^40: an operation leaves at most a few 2^6 coefficients of noise (a hoisted rotation's, here multiplied by plaintexts with slots of at
most 1.2), i.e. 5e-8 a slot on the ring of 4096 and less on a smaller one; the sums here have at most 130 such terms."""
import ctypes as C

import numpy as np
import pytest

TOL = 2e-5


@pytest.fixture(scope="module")
def env():
    from oracle import ckks, params
    ctx = ckks.Context(params.toy(n=512))
    return ctx, ctx.keygen_secret(1)


def _enc(env, slots, level, seed):
    ctx, sk = env
    return ctx.encrypt(sk, ctx.pt_from_coeffs(ctx.encode_coeffs(slots, 2.0 ** 40), level, 2.0 ** 40), seed)


def _table(ctx, tables, level):
    q, m2 = float(ctx.mod[level]), float(ctx.mod[0])
    s = tables.slots()
    n = 4 * tables.low + 1
    return [ctx.encode_coeffs(v, q) for v in s[:n]] + [ctx.encode_coeffs(v, m2) for v in s[n:]]


@pytest.mark.parametrize("heads, dim, rot, halves, gain, room", [(4, 8, 8, False, 1.0, 40), (4, 8, 8, True, 1.0, 7), (3, 16, 4, True, 1.2, 100), (2, 4, 2, False, 1.0, 1),
                                                                 (1, 2, 2, False, 1.0, 9), (8, 32, 16, False, 0.5, 33)])
def test_rotary_positions_by_tables(env, heads, dim, rot, halves, gain, room):
    from oracle import packing, vmm
    ctx, sk = env
    tables = packing.RotaryTables(ctx.S, heads, dim, room, rot=rot, gain=gain, halves=halves)
    lay, level, rng = tables.lay, 3, np.random.default_rng(room)
    coeffs = _table(ctx, tables, level)
    keys = ctx.keygen_rotations(sk, [tables.step, -tables.step], 2)
    slots = rng.normal(size=ctx.S)
    x = _enc((ctx, sk), slots, level, 5)
    v = slots.reshape(dim, lay.H, lay.t)
    for positions in ([room - 1] * lay.t, [-1] * lay.t, [int(p) for p in rng.integers(-1, room, lay.t)]):
        y = vmm.rotary(ctx, keys, tables, x, vmm.rotary_plaintexts(ctx, tables, coeffs, positions, level))
        got = ctx.decrypt(sk, y).real.reshape(dim, lay.H, lay.t)
        for r, p in enumerate(positions):
            want = tables.turn(v[:, :, r].T, p).T if p >= 0 else 0.0
            assert np.abs(got[:, :, r] - want).max() < TOL


@pytest.mark.parametrize("place, ntok, index, rotate", [(0, 1, False, False), (5, 8, True, False), (14, 3, True, True), (23, 8, False, True), (16, 8, False, True), (7, 1, False, True)])
def test_appended_runs(env, place, ntok, index, rotate):
    from oracle import packing, vmm
    ctx, sk = env
    H, E, r_i = 4, 8, 4
    lay, lv = packing.KvLayout(ctx.S, H, E, r_i), 2
    tables = packing.RotaryTables(ctx.S, H, E, 64, halves=True)
    B, rng = lay.H * lay.t, np.random.default_rng(place)
    steps = [tables.step, -tables.step] + [j * B for j in range(1, r_i)] + [-g * r_i * B for g in range(1, lay.r_o)]
    keys = ctx.keygen_rotations(sk, steps, 2)
    ks, vs = rng.normal(size=(2, ctx.S))
    lk = lv + 1 + (rotate and index)
    ck, cv = _enc(env, ks, lk, 3), _enc(env, vs, lv + 1, 4)
    t = lay.t
    run = [place + i for i in range(ntok)]
    K, V = np.zeros((2, lay.capacity, H, E))
    for a in run:
        k = ks.reshape(E, H, t)[:, :, a % t].T
        K[a], V[a] = tables.turn(k, a) if rotate else k, vs.reshape(E, H, t)[:, :, a % t].T
    ones = np.zeros((2, E, H, t))
    ones[0, :, :, 0], ones[1, 0, :, 0] = 1, 1
    residue, row = (ctx.pt_from_coeffs(ctx.encode_coeffs(m.reshape(-1), float(ctx.mod[lv + 1])), lv + 1, float(ctx.mod[lv + 1])) for m in ones)
    turned = None
    if rotate:
        coeffs = _table(ctx, tables, lk)
        at = lambda keep: [next((a for a in run if a % t == r and keep(a)), -1) for r in range(t)]  # noqa: E731
        if index:
            ck = vmm.rotary(ctx, keys, tables, ck, vmm.rotary_plaintexts(ctx, tables, coeffs, at(lambda a: True), lk))
        else:
            pages = sorted({a // t for a in run})
            turned = [vmm.rotary(ctx, keys, tables, ck, vmm.rotary_plaintexts(ctx, tables, coeffs, at(lambda a, p=p: a // t == p), lk)) for p in pages]
    k_cts, v_cts, x_cts = [None] * E, [None] * E, [None] * E if index else None
    vmm.kv_append_run(ctx, keys, lay, k_cts, v_cts, place, ntok, ck, cv, residue, row, turned, x_cts)
    slots = lambda c: ctx.decrypt(sk, c).real  # noqa: E731
    for c in range(E):
        assert (k_cts[c] is None) == (c not in {a // t for a in run})
        if k_cts[c] is not None:
            assert np.abs(slots(k_cts[c]) - lay.pack_k(K, c)).max() < TOL
        assert np.abs(slots(v_cts[c]) - lay.pack_v(V, c)).max() < TOL
        if index:
            assert np.abs(slots(x_cts[c]) - lay.pack_k_index(K, c)).max() < TOL


@pytest.mark.parametrize("group, base, parents, node0, first", [(1, 13, [-1, 0, 0, 1, -1, 3], 0, 0), (2, 16, [-1, 0, 1, 2, 2], 2, 8), (8, 21, [-1], 0, 16), (1, 0, [-1, 0, 1], 0, 0)])
def test_tree_scores_and_values(env, group, base, parents, node0, first):
    from oracle import packing, vmm
    ctx, sk = env
    H, E, r_i = 4, 8, 4
    lay, lv, mask = packing.KvLayout(ctx.S, H, E, r_i), 3, -24.0
    t, rng, ntok = lay.t, np.random.default_rng(base), base + len(parents)
    B = lay.H * t
    steps = vmm.sv_unrolled_steps(lay) + [s for d in range(1, t) for s in (-d, t - d)]
    keys = ctx.keygen_rotations(sk, steps, 2, with_relin=True)
    K, V = 0.3 * rng.normal(size=(2, ntok, H, E))
    moves = [[ctx.encode_coeffs((np.arange(ctx.S) % t >= d).astype(float), float(ctx.mod[level])) for d in range(1, t)] for level in (lv + 1, lv - 1)]
    qs = 0.3 * rng.normal(size=ctx.S)
    scale = 2.0 ** 80 / float(ctx.mod[lv])
    pts = [ctx.encode(mask * packing.tree_hidden(lay, group, parents, base, node0, first, d).reshape(-1), lv - 1, scale).m for d in range(t)]
    sv = lambda cts: lambda x: vmm.score_times_v_unrolled(ctx, keys, lay, x, cts, reduce=False)  # noqa: E731
    x_cts = [_enc(env, lay.pack_k_index(K, k), lv, 10 + k) for k in range(E)]
    got = vmm.tree_qk(ctx, keys, lay, _enc(env, qs, lv + 1, 5), moves[0], sv(x_cts), pts)
    q = qs.reshape(E, H, t)
    Kp = np.concatenate([K, np.zeros((lay.capacity - ntok, H, E))]).reshape(E, t, H, E)
    for d in range(t):
        moved = np.roll(q, d, axis=2)
        want = np.einsum("chje,ehj->chj", Kp.transpose(0, 2, 1, 3), moved) + mask * packing.tree_hidden(lay, group, parents, base, node0, first, d)
        assert np.abs(ctx.decrypt(sk, got[d]).real.reshape(E, H, t) - want).max() < TOL
    v_cts = [_enc(env, lay.pack_v(V, k), lv, 50 + k) for k in range(E)]
    s = 0.3 * rng.normal(size=(t, E, H, t))
    out = vmm.tree_sv(ctx, keys, lay, [_enc(env, s[d].reshape(-1), lv, 80 + d) for d in range(t)], moves[1], sv(v_cts))
    Vp = np.concatenate([V, np.zeros((lay.capacity - ntok, H, E))]).reshape(E, t, H, E)
    want = sum(np.roll(np.einsum("chj,cjhe->ehj", s[d], Vp), -d, axis=2) for d in range(t))
    assert np.abs(ctx.decrypt(sk, out).real.reshape(E, H, t) - want).max() < TOL


def test_hidden_places_by_hand():
    """Two tokens a page, one head: base 3, tokens 0 <- 1, 0 <- 2 at places 3, 4, 5; queries of the first two (residues 1 and 0)."""
    from oracle import packing
    lay = packing.KvLayout(8, 1, 4)
    h = [packing.tree_hidden(lay, 1, [-1, 0, 0], 3, 0, 2, d)[:, 0] for d in range(2)]
    # pass 0 pairs equal residues: residue 0 is token 1's query (place 4), residue 1 token 0's (place 3)
    assert h[0].tolist() == [[1, 1], [0, 0], [0, 1], [1, 1]]
    # pass 1: residue 0 holds token 0's query against places 0, 2, 4, 6; residue 1 token 1's against 1, 3, 5, 7
    assert h[1].tolist() == [[1, 1], [0, 0], [1, 1], [1, 1]]


def test_frequencies():
    from paper_2602_11470_amd import binding as B
    plain = 10000.0 ** (-np.arange(0, 64, 2) / 64)
    np.testing.assert_allclose(B.rotary_freqs(64), plain, rtol=1e-14)
    np.testing.assert_allclose(B.rotary_freqs(64, 500000.0), 500000.0 ** (-np.arange(0, 64, 2) / 64), rtol=1e-14)
    np.testing.assert_allclose(B.rotary_freqs(64, scaling=B.CM_ROTARY_LINEAR, par=[8.0]), plain / 8, rtol=1e-14)
    np.testing.assert_allclose(B.rotary_freqs(64, scaling=B.CM_ROTARY_BASE, par=[4.0]), (10000.0 * 4 ** (64 / 62)) ** (-np.arange(0, 64, 2) / 64), rtol=1e-13)
    turns = 8192 * plain / (2 * np.pi)
    got = B.rotary_freqs(64, scaling=B.CM_ROTARY_BANDS, par=[8.0, 1.0, 4.0, 8192.0])
    # two powers of the same numbers, each within one unit of the last place (2^-52): they differ by at most two, and by three after the division
    np.testing.assert_allclose(got[turns >= 4], plain[turns >= 4], rtol=2 * 2.0 ** -52, atol=0)
    assert np.allclose(got[turns <= 1], plain[turns <= 1] / 8, rtol=1e-14)
    between = (turns > 1) & (turns < 4)
    keep = (turns[between] - 1) / 3
    assert between.any() and np.allclose(got[between], keep * plain[between] + (1 - keep) * plain[between] / 8, rtol=1e-13)
    assert B.rotary_freqs(2, scaling=B.CM_ROTARY_BASE, par=[4.0])[0] == 1.0


def test_refusals_without_a_context():
    from paper_2602_11470_amd import binding as B
    lib, out = B.lib, np.empty(64)
    p = np.array([4.0, 1.0, 8.0, 256.0])

    def freqs(rot, base, scaling, par=p):
        return lib.cm_rotary_freqs(rot, base, scaling, par.ctypes.data if par is not None else None, out.ctypes.data)
    assert freqs(64, 1e4, B.CM_ROTARY_BANDS) == 0 and freqs(64, 1e4, B.CM_ROTARY_PLAIN, None) == 0
    assert freqs(63, 1e4, 0) == freqs(0, 1e4, 0) == freqs(64, 1.0, 0) == freqs(64, np.nan, 0) == freqs(64, 1e4, 4) == freqs(64, 1e4, -1) == -1
    assert freqs(64, 1e4, B.CM_ROTARY_LINEAR, None) == freqs(64, 1e4, B.CM_ROTARY_LINEAR, np.zeros(4)) == -1
    assert freqs(64, 1e4, B.CM_ROTARY_BANDS, np.array([4.0, 8.0, 8.0, 256.0])) == freqs(64, 1e4, B.CM_ROTARY_BANDS, np.array([4.0, 1.0, 8.0, 0.0])) == -1
    assert freqs(64, 1e4, B.CM_ROTARY_BANDS, np.array([4.0, np.nan, 8.0, 256.0])) == -1
    assert lib.cm_rotary_freqs(64, 1e4, 0, None, None) == -1
    # low parts, high parts: 1 and 1, 2 and 1, 2 and 2, 32 and 32, 64 and 17
    assert [lib.cm_rotary_polys(r) for r in (1, 2, 3, 1024, 1025)] == [4 + 1 + 2, 8 + 1 + 2, 8 + 1 + 4, 128 + 1 + 64, 256 + 1 + 34]
    assert lib.cm_rotary_polys(0) == lib.cm_rotary_polys(-1) == lib.cm_rotary_polys((1 << 24) + 1) == 0
    h = C.c_void_p()
    assert lib.cm_rotary_create(None, 4, 16, 2, 16, None, 1.0, 64, 0, None, C.byref(h)) == -1
    assert lib.cm_rotary_set(None, None, out.ctypes.data, 0, None) == lib.cm_rotary_apply(None, None, None, 1, None, None, None) == -1
    d = B.cm_ct()
    assert lib.cm_kv_append_run(None, None, None, None, 1, C.byref(d), C.byref(d), None) == -1
    assert lib.cm_tree_create(None, None, 1, -24.0, 0.0, None, C.byref(h)) == -1
    assert lib.cm_tree_qk(None, None, None, None, out.ctypes.data, 1, 0, 0, 0, C.byref(d), None, None) == -1
    assert lib.cm_tree_sv(None, None, None, None, None, C.byref(d), None) == -1
    assert lib.cm_rotary_steps(None, None, 0) == lib.cm_tree_steps(None, None, 0) == lib.cm_tree_passes(None) == 0
    lib.cm_rotary_destroy(None), lib.cm_tree_destroy(None)
