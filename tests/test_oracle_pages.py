"""Taking tokens out of a cache and moving its pages, and the relative position bias, on plain slot vectors: the oracle's
steps give the layouts of the kept, moved token matrices, and scores plus bias are the textbook's."""
import numpy as np
import pytest

from oracle import packing, vmm


def _moved(M, keep, shift, t):
    """The token matrix with dropped tokens zero, `shift` pages on."""
    out = np.zeros((M.shape[0] + max(0, shift) * t,) + M.shape[1:])
    for n in np.flatnonzero(keep):
        out[n + shift * t] = M[n]
    return out


@pytest.mark.parametrize("S,H,E,r_i", [(64, 2, 8, 4), (64, 2, 8, 8), (64, 2, 8, 1), (128, 3, 16, 4), (64, 1, 32, 8)])
@pytest.mark.parametrize("shift", [0, 1, 3, 4, -1, -2, -4])
def test_taking_gives_the_layouts_of_the_kept_tokens(S, H, E, r_i, shift):
    lay = packing.KvLayout(S, H, E, r_i)
    rng = np.random.default_rng(E + shift)
    pages = E - 4
    ntok = pages * lay.t - lay.t // 2
    K, V = rng.normal(size=(2, ntok, H, E))
    keep = rng.uniform(size=ntok) < 0.6
    keep[:max(0, -shift) * lay.t] = False
    keep[2 * lay.t:3 * lay.t] = shift > -3                      # a page kept whole, or dropped whole
    nk = -(-ntok // lay.t)
    masks = {r: np.roll(lay.keep_rows(keep), -r * lay.H * lay.t) for r in range(E)}
    k, v, x = vmm.kv_take(vmm.SlotOps(), lay, [lay.pack_k(K, c) for c in range(nk)], [lay.pack_v(V, c) for c in range(E)], keep, shift, masks,
                          {c: lay.keep_residues(keep, c) for c in lay.partial_pages(keep)}, [lay.pack_k_index(K, c) for c in range(E)])
    K2, V2 = _moved(K, keep, shift, lay.t), _moved(V, keep, shift, lay.t)
    for c in range(E):
        assert np.array_equal(k.get(c, np.zeros(S)), lay.pack_k(K2, c)), c
        assert np.array_equal(v[c], lay.pack_v(V2, c)), c
        assert np.array_equal(x[c], lay.pack_k_index(K2, c)), c
    if shift == 0:
        assert lay.take_steps(shift, True) == []
    if shift % r_i == 0:
        assert all(lay.k_index_place(c, shift)[1] == 0 for c in range(E))
    if r_i == E:
        assert all(lay.v_place(c, shift)[1] == 0 for c in range(E))


@pytest.mark.parametrize("token,first", [(0, None), (37, None), (63, 16), (20, 48), (63, 0), (9, 8)])
@pytest.mark.parametrize("group,prompt", [(1, False), (2, False), (4, False), (1, True), (2, True), (4, True)])
def test_bias_is_the_tables_entry_of_every_pair(token, first, group, prompt):
    """Every slot against loops over heads, queries and keys; and the plaintext of a page is that of page 0, whole rows on."""
    S, Hkv, E = 128, 2, 16
    lay = packing.KvLayout(S, Hkv, E)
    t_kv, cap = lay.t, E * lay.t
    t = t_kv // group
    token -= token % t if prompt else 0
    rng = np.random.default_rng(1)
    table, bucket = rng.normal(size=(Hkv * group, 7)), rng.integers(0, 7, cap)
    passes = t_kv if prompt else group
    got = [lay.bias_slots(table, bucket, token, first, -9.0, group, d, prompt) for d in range(passes)]
    seen = set()
    for hk in range(Hkv):
        for g in range(group):
            for tau in range(t if prompt else 1):
                for key in range(cap):
                    c, j = key // t_kv, key % t_kv
                    # decode: the pass whose run of residue j holds query head g; prompt: the one that moved the query to j
                    delta = (j - (g * t + tau)) % t_kv if prompt else (j // t - g) % group
                    want = table[hk * group + g][bucket[(token + tau - key) % cap]]
                    if first is not None:
                        pages = [(first // t_kv + i) % E for i in range((token // t_kv - first // t_kv) % E + 1)]
                        want += 0.0 if c in pages else -9.0
                    assert got[delta][lay.slot(c, hk, j)] == want
                    seen.add((delta, lay.slot(c, hk, j)))
    assert len(seen) == passes * S
    page, rest = token // t_kv, token % t_kv
    for d in range(passes):
        assert np.array_equal(lay.bias_slots(table, bucket, token, None, 0.0, group, d, prompt),
                              np.roll(lay.bias_slots(table, bucket, rest, None, 0.0, group, d, prompt), page * lay.H * t_kv))


def test_biased_scores_of_packed_prompts_are_causal():
    """Two sequences packed page by page in one cache: scores of a prompt group in all its passes, plus a causal bias and the pages
    of the other sequence hidden, against the dense matrix."""
    S, H, E = 64, 2, 8
    lay = packing.KvLayout(S, H, E)
    rng = np.random.default_rng(4)
    cap, t = E * lay.t, lay.t
    lengths = [11, 9]                                           # 3 pages of 4 tokens, then 3
    starts = [0, -(-lengths[0] // t) * t]
    K = np.zeros((starts[1] + lengths[1], H, E))
    for s, n in zip(starts, lengths):
        K[s:s + n] = rng.normal(size=(n, H, E))
    bucket = np.where(np.arange(cap) > cap - t, 2, np.minimum(np.arange(cap) // 3, 1))
    table = np.concatenate([rng.normal(size=(H, 2)), np.full((H, 1), -50.0)], 1)
    masks = [lay.qk_mask(c) for c in range(E)]
    kc = [lay.pack_k(K, c) for c in range(-(-len(K) // t))]
    for p0, first in [(0, 0), (8, 0), (12, 12), (16, 12)]:
        Q = rng.normal(size=(t, H, E))
        q = sum(lay.pack_vec(Q[r], r) for r in range(t))
        for delta in range(t):
            y = vmm.inner_rotate(vmm.SlotOps(), lay, q, delta, lay.inner_rotation_plaintexts(delta)) if delta else q
            s = vmm.qk_scores(vmm.SlotOps(), lay, y, kc, masks, replicate=False)
            s = s + lay.bias_slots(table, bucket, p0, first, -50.0, 1, delta, True)
            for j in range(t):
                tau = (j - delta) % t
                for c in range(E):
                    key, mine = c * t + j, first // t <= c <= p0 // t
                    for h in range(H):
                        got, dot = s[lay.slot(c, h, j)], (Q[tau, h] @ K[key, h] if key < len(K) else 0.0)
                        if mine and key <= p0 + tau:
                            assert abs(got - dot - table[h][bucket[p0 + tau - key]]) < 1e-12
                        else:
                            assert got - dot < -40.0
