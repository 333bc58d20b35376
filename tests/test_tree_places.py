"""Places of a cache without a token (dropped by cm_kv_take between kept ones): no query of a tree sees them (cm_tree_set_empty)."""
import ctypes as C

import numpy as np
import pytest

MASK = -24.0


def test_hidden_places_by_hand():
    """Two tokens a page, one head; places 0, 1, 3 and 4 were kept, 2 was dropped, 5 and 6 are drafted, 6 behind 5."""
    from oracle import packing
    lay = packing.KvLayout(8, 1, 4)
    seen = [packing.tree_hidden(lay, 1, [-1, 0], 5, 0, 0, d)[:, 0].tolist() for d in range(2)]
    # pass 0: residue 0 is the query of place 6, residue 1 that of place 5; without being told, both see place 2
    assert seen[0] == [[0, 0], [0, 0], [0, 0], [0, 1]] and seen[1] == [[0, 0], [0, 0], [0, 0], [1, 1]]
    told = [packing.tree_hidden(lay, 1, [-1, 0], 5, 0, 0, d, empty=[2])[:, 0].tolist() for d in range(2)]
    assert told[0] == [[0, 0], [1, 0], [0, 0], [0, 1]] and told[1] == [[0, 0], [1, 0], [0, 0], [1, 1]]


def test_refused_without_an_object():
    from paper_2602_11470_amd import binding as B
    p = np.zeros(1, dtype=np.int32)
    assert B.lib.cm_tree_set_empty(None, p.ctypes.data, 1) == B.lib.cm_tree_set_empty(None, None, 0) == -1


@pytest.fixture(scope="module")
def small():
    from oracle import ckks, params
    from paper_2602_11470_amd import binding as B
    gctx = B.config1()
    yield gctx, ckks.Context(params.config1())
    gctx.close()


# heads, dim, group, index, base, parents, node0, first, empty
CASES = [(8, 32, 1, True, 21, [-1, 0, 0], 0, 0, [3, 17, 20]), (8, 32, 2, True, 50, [-1, 0, 0, 1], 1, 16, [2, 9, 16, 17, 23, 33, 41, 41, 49, 200]),
         (8, 32, 1, False, 24, [-1, -1], 0, 8, [0, 8, 15, 23]), (16, 128, 1, True, 6, [-1, 0], 0, 0, [1, 4]), (8, 32, 8, True, 80, [-1], 0, 0, list(range(0, 80, 9)))]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=str)
def test_empty_places_take_the_mask(small, case):
    """Word for word: what the scores are without, and the mask's value at the empty places that nothing else hides, once; none where none is set."""
    from oracle import packing
    from paper_2602_11470_amd import binding as B
    heads, dim, group, index, base, parents, node0, first, empty = case
    gctx, octx = small
    level, lay = 3, packing.KvLayout(gctx.S, heads, dim, 8)
    t, H, rng = lay.t, lay.H, np.random.default_rng(base)
    kv = gctx.kv_create(heads, dim, level, r_i=8, key_index=index)
    scale = gctx.scale ** 2 / float(gctx.moduli()[level])
    one, row = np.zeros((2, dim, H, t))
    one[0, :, 0] = row[0] = MASK
    moves = [[gctx.encode_coeffs((np.arange(gctx.S) % t >= d).astype(float), float(gctx.moduli()[lv])) for d in range(1, t)] for lv in (level + 1, level - 1)]
    one, row = (gctx.encode_coeffs(m.reshape(-1), scale) for m in (one, row))
    tree = gctx.tree(kv, group=group, mask=MASK, coeffs=np.stack(moves[0] + moves[1] + [one, row]))
    sk = gctx.keygen_secret(1)
    keys = gctx.keygen_rotations(sk, kv.steps() + tree.steps(), 2, with_relin=True)
    K = 0.3 * rng.normal(size=(base + len(parents), heads, dim))
    K[[p for p in empty if p < base]] = 0
    enc = lambda slots, lv, seed: gctx.encrypt(sk, gctx.encode(slots, lv), seed)  # noqa: E731
    for i in range(dim if index else -(-len(K) // t)):
        kv.load(B.CM_KV_INDEX if index else B.CM_QK, i, enc(lay.pack_k_index(K, i) if index else lay.pack_k(K, i), level, 20 + i))
    kv.set_tokens(len(K))
    q = enc(0.3 * rng.normal(size=gctx.S), level + 1, 9)
    export = lambda: [gctx.ct_export(s) for s in gctx.tree_qk(keys, tree, kv, parents, base, q, node0=node0, first=first)]  # noqa: E731
    plain = export()
    tree.set_empty(empty)
    got = export()
    idx = octx.q_idx(level - 1 if index else level - 2)
    for d in range(t):
        more = packing.tree_hidden(lay, group, parents, base, node0, first, d, empty) - packing.tree_hidden(lay, group, parents, base, node0, first, d)
        want = octx.ntt(plain[d][0], idx)
        for c, j in np.argwhere(more[:, 0]):
            want = octx.add(want, octx.automorphism(octx.ntt(octx.from_i64(one, idx), idx), idx, octx.galois(-(int(c) * H * t + int(j)))), idx)
        np.testing.assert_array_equal(got[d][0], octx.intt(want, idx))
        np.testing.assert_array_equal(got[d][1], plain[d][1])
    tree.set_empty([])
    assert all(np.array_equal(a, b) for a, b in zip(export(), plain))


@pytest.mark.gpu
def test_refusals(small):
    from paper_2602_11470_amd import binding as B
    gctx, _ = small
    tree = gctx.tree(gctx.kv_create(8, 32, 3, r_i=8, key_index=True))

    def put(places, count=None):
        p = np.array(places, dtype=np.int32)
        return B.lib.cm_tree_set_empty(tree.h, p.ctypes.data, p.size if count is None else count)
    assert put([0, 255]) == 0 and put([255, 255, 3]) == 0
    assert put([256]) == put([-1]) == put([3, -5]) == -5 and put([3], -1) == -1
    assert B.lib.cm_tree_set_empty(tree.h, None, 1) == -1 and B.lib.cm_tree_set_empty(tree.h, None, 0) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("heads, dim, r_i, group", [(8, 32, 8, 1), (4, 32, 8, 2)])
def test_a_session_that_attends_to_kept_tokens_alone(heads, dim, r_i, group):
    """A prompt, a tree drafted behind it, its rejected tokens dropped between accepted ones, a second tree: its queries' attention (softmax in the clear) is that
    over the kept tokens.  What the empty places get of a softmax's sum is at most exp(-24 + what scores differ by, at most 8) each, 512 of them 6e-5."""
    from oracle import packing
    from paper_2602_11470_amd import binding as B
    ctx = B.Context(4096, 9, 2, 2, 50, 50, 60, 2.0 ** 50)
    try:
        lay = packing.KvLayout(ctx.S, heads, dim, r_i)
        H, t, per, rng = lay.H, lay.t, lay.t // group, np.random.default_rng(11)
        sk = ctx.keygen_secret(1)
        caches = [ctx.kv_create(heads, dim, lv, r_i=r_i, key_index=True, unrolled_ladders=True) for lv in (6, 5)]
        tables = packing.RotaryTables(ctx.S, heads, dim, 64, halves=True)
        rots = [ctx.rotary(heads, dim, lv, 64, halves=True) for lv in (8, 7)]
        tree = ctx.tree(caches[1], group=group)
        keys = ctx.keygen_rotations(sk, caches[0].steps() + tree.steps() + rots[0].steps(), 2, with_relin=True)
        seeds = iter(range(100, 1000))
        enc = lambda slots, lv: ctx.encrypt(sk, ctx.encode(slots, lv), next(seeds))  # noqa: E731
        K, V = np.zeros((2, 0, heads, dim))

        def append(kv, rot, positions):
            nonlocal K, V
            place, n = len(K), len(positions)
            ks, vs = 0.3 * rng.normal(size=(2, dim, H, t))
            at = [-1] * t
            for i, p in enumerate(positions):
                r = (place + i) % t
                at[r] = p
                K, V = np.concatenate([K, tables.turn(ks[:, :heads, r].T, p)[None]]), np.concatenate([V, vs[:, :heads, r].T[None]])
            ctx.rotary_set(rot, at, max(0, place % t + n - t))
            kv.append_run(keys, enc(ks.reshape(-1), rot.level), enc(vs.reshape(-1), kv.level + 1), n, rotary=rot)
        for n in (t, t, 3):
            append(caches[0], rots[0], range(len(K), len(K) + n))
        base = len(K)
        append(caches[0], rots[0], [base, base + 1, base + 1, base + 2, base + 2])
        keep = np.ones(len(K), dtype=bool)
        keep[[base + 1, base + 3]] = False                            # 0, 2 and 4 are accepted
        ctx.kv_take(None, ctx.kv_sel(caches[0], keep), caches[0], caches[1])
        base, parents = len(K), [-1, 0, 0]
        append(caches[1], rots[1], [base - 2, base - 1, base - 1])
        tree.set_empty(np.nonzero(~keep)[0])
        qs = 0.3 * rng.normal(size=(dim, H, t))
        scores = ctx.tree_qk(keys, tree, caches[1], parents, base, enc(qs.reshape(-1), 6))
        s = np.stack([ctx.decrypt(sk, c).real.reshape(dim, H, t)[:, :heads] for c in scores])
        probs, want = np.zeros((t, dim, H, t)), np.zeros((dim, heads, t))
        for u in range(t):
            node = (u % per - base) % per
            seen = [p for p in range(base) if keep[p]]
            k = node if node < len(parents) else -1
            while k >= 0:
                seen.append(base + k)
                k = parents[k]
            row = np.stack([s[(p % t - u) % t, p // t, :, p % t] for p in range(lay.capacity)])
            e = np.exp(row - row.max(0))
            for p, w in enumerate(e / e.sum(0)):                          # the softmax over every place of the cache
                probs[(p % t - u) % t, p // t, :heads, p % t] = w
            e = np.exp(np.array([[K[p, h] @ qs[:, h, u] for h in range(heads)] for p in seen]))
            want[:, :, u] = np.einsum("ph,phe->eh", e / e.sum(0), V[seen])
        out = ctx.tree_sv(keys, tree, caches[1], [enc(probs[d].reshape(-1), 5) for d in range(t)])
        got = ctx.decrypt(sk, out).real.reshape(dim, H, t)[:, :heads]
        # 6e-5 of a sum, twice (the hidden places' shares, and what the others lose), times values of at most 2
        assert np.abs(got - want).max() < 3e-4
    finally:
        ctx.close()
