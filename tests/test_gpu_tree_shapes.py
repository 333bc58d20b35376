"""Trees of drafts in shapes beside those of one page of eight on the full ring: query groups, pages of 32 residues, caches without the key index and with
more giant steps than are taken together; and caches whose baby steps are not those of the cache that the object was made from."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
# scale 2^50: what an operation leaves, 2^6 units a coefficient and 2^8 times that a slot, is 2^-36; at most 300 of them are summed
TOL = 300 * 2.0 ** -36


@pytest.fixture(scope="module")
def big():
    from paper_2602_11470_amd import binding as B
    ctx = B.llama_ring()
    yield ctx
    ctx.close()


# heads, dim, group, r_i, level, form, base, parents, node0, first
CASES = [(8, 128, 4, 16, 3, "index unrolled", 70, [-1, 0, 0, 1, -1, 3, 5], 2, 32), (8, 128, 1, 16, 2, "index", 60, [-1, 0, 1, 1, 2], 0, 0),
         (64, 64, 1, 16, 3, "unrolled", 13, [-1, 0, 0, 2], 1, 8), (64, 64, 2, 4, 3, "index unrolled", 20, [-1, 0], 0, 0)]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_decrypted_on_the_full_ring(big, case):
    from oracle import packing
    from paper_2602_11470_amd import binding as B
    heads, dim, group, r_i, level, form, base, parents, node0, first = case
    lay, rng, ntok, index = packing.KvLayout(big.S, heads, dim, r_i), np.random.default_rng(base), base + len(parents), "index" in form
    t, H = lay.t, lay.H
    kv = big.kv_create(heads, dim, level, r_i=r_i, key_index=index, unrolled_ladders="unrolled" in form)
    tree = big.tree(kv, group=group)
    sk = big.keygen_secret(1)
    keys = big.keygen_rotations(sk, kv.steps() + tree.steps(), 2, with_relin=True)
    seeds = iter(range(100, 10000))
    enc = lambda slots, lv: big.encrypt(sk, big.encode(slots, lv), next(seeds))  # noqa: E731
    K, V = 0.3 * rng.normal(size=(2, ntok, heads, dim))
    for k in range(dim):
        kv.load(B.CM_SV, k, enc(lay.pack_v(V, k), level))
        if index:
            kv.load(B.CM_KV_INDEX, k, enc(lay.pack_k_index(K, k), level))
    for c in range(0 if index else -(-ntok // t)):
        kv.load(B.CM_QK, c, enc(lay.pack_k(K, c), level))
    kv.set_tokens(ntok)
    qs = 0.3 * rng.normal(size=(dim, H, t))
    scores = big.tree_qk(keys, tree, kv, parents, base, enc(qs.reshape(-1), level + 1), node0=node0, first=first)
    Kp, Vp = (np.concatenate([a, np.zeros((lay.capacity - ntok, heads, dim))]).reshape(dim, t, heads, dim) for a in (K, V))
    for d in range(t):
        want = np.einsum("chje,ehj->chj", Kp.transpose(0, 2, 1, 3), np.roll(qs, d, axis=2)) - 24.0 * packing.tree_hidden(lay, group, parents, base, node0, first, d)
        assert np.abs(big.decrypt(sk, scores[d]).real.reshape(dim, H, t) - want).max() < TOL
    s = 0.3 * rng.normal(size=(t, dim, H, t))
    out = big.tree_sv(keys, tree, kv, [enc(s[d].reshape(-1), level) for d in range(t)])
    want = sum(np.roll(np.einsum("chj,cjhe->ehj", s[d], Vp), -d, axis=2) for d in range(t))
    assert np.abs(big.decrypt(sk, out).real.reshape(dim, H, t) - want).max() < TOL


@pytest.mark.parametrize("made, used", [(8, 16), (8, 4), (16, 8), (2, 32)])
def test_caches_of_other_baby_steps(made, used):
    """An object made from one cache and used on another: the words of an object made for that one (32 dims: r_i 2 has sixteen giant steps, taken alone)."""
    import torch
    from paper_2602_11470_amd import binding as B
    ctx = B.config1()
    try:
        caches = {r: ctx.kv_create(8, 32, 3, r_i=r, key_index=True, unrolled_ladders=True) for r in (made, used)}
        kv, gen = caches[used], torch.Generator(device="cuda").manual_seed(used)
        trees = [ctx.tree(caches[made]), ctx.tree(kv)]
        sk = ctx.keygen_secret(1)
        keys = ctx.keygen_rotations(sk, kv.steps() + trees[0].steps(), 2, with_relin=True)

        def uniform(words):
            for i in range(words.shape[-2]):
                words[..., i, :] = torch.empty(words.shape[:-2] + (ctx.n,), dtype=torch.int64, device="cuda").random_(0, int(ctx.moduli()[i]), generator=gen)

        def ct(level):
            c = B.Ct(ctx, level)
            c.d.scale = ctx.scale
            uniform(c.buf[: 2 * (level + 1) * ctx.n].view(2, level + 1, ctx.n))
            return c
        for w in (B.CM_SV, B.CM_KV_INDEX):
            uniform(kv.words(w))
        kv.set_tokens(44)
        q, weights = ct(4), [ct(3) for _ in range(8)]
        found = []
        for tree in trees:
            outs = ctx.tree_qk(keys, tree, kv, [-1, 0, 0, 1], 40, q) + [ctx.tree_sv(keys, tree, kv, weights)]
            found.append([ctx.ct_export(c) for c in outs])
        assert all(np.array_equal(a, b) for a, b in zip(*found))
    finally:
        ctx.close()
