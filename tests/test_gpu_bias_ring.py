"""Causal bias (CM_RELBIAS_CAUSAL) on scores of a ring whose pages are all in use: the library's plaintexts against the oracle's slots, together with q K^T,
and its refusals."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2602_11470_amd import binding as B
    c = B.Context(4096, 6, 2, 2, 58, 54, 60, 2.0 ** 50)
    yield c
    c.close()


@pytest.mark.parametrize("heads,dim,group,prompt,token,first", [
    (4, 16, 1, False, 333, -1), (4, 16, 1, False, 511, 0), (3, 64, 4, False, 102, 104), (4, 128, 2, True, 250, 252), (4, 64, 1, True, 64, 72), (4, 64, 2, True, 508, 16),
    (1, 1, 1, False, 1000, 0), (8, 256, 1, False, 17, -1)])
def test_own_plaintexts_are_the_oracles_slots(ctx, heads, dim, group, prompt, token, first):
    """Decrypted scores differ by the oracle's slots.  The sum of up to `dim` encodings is off by half a unit of the scale each in every
    coefficient, at most dim * n / 2 / scale in a slot, next to the noise of one encryption."""
    from oracle import packing
    sk = ctx.keygen_secret(1)
    lay = packing.KvLayout(ctx.S, heads, dim)
    rng = np.random.default_rng(dim)
    cap, level = dim * lay.t, 3
    table, bucket = rng.normal(size=(heads * group, 9)), rng.integers(0, 9, cap)
    bias = ctx.relbias(heads, dim, table, bucket, level, group=group, prompt=prompt, mask=-30.0, causal=True)
    z = [rng.normal(size=ctx.S) for _ in range(bias.passes)]
    scores = [ctx.encrypt(sk, ctx.encode(v, level), 50 + i) for i, v in enumerate(z)]
    outs = ctx.relbias_apply(bias, token, scores, first=first)
    for d in sorted({0, 1 % bias.passes, bias.passes - 1}):
        want = z[d] + lay.bias_slots(table, bucket, token, first if first >= 0 else None, -30.0, group, d, prompt, causal=True)
        noise = np.abs(ctx.decrypt(sk, scores[d]) - z[d]).max()
        assert np.abs(ctx.decrypt(sk, outs[d]) - want).max() <= noise + dim * ctx.n / 2 / ctx.scale + 1e-12 * 64


def test_with_the_scores_of_a_full_ring(ctx):
    """q K^T of a grouped decode step and of a prompt group against a ring that has gone round: every page holds tokens, the query's own page up to the
    query.  The oldest tokens keep their scores at every residue of the query."""
    from oracle import packing
    from paper_2602_11470_amd import binding as B
    sk = ctx.keygen_secret(1)
    Hkv, E, G = 8, 32, 4
    lay = packing.KvLayout(ctx.S, Hkv, E, 8)
    t_kv, cap = lay.t, E * lay.t
    t, rng = t_kv // G, np.random.default_rng(2)
    K = rng.normal(size=(cap, Hkv, E)) * 0.2
    token, page = 5 * t_kv + 2 * t, 5
    keys, made = None, {}
    for prompt, last in ((False, token), (True, token + t - 1)):
        K1 = K.copy()
        K1[last + 1: (page + 1) * t_kv] = 0                                   # places behind the query: not filled yet
        kv = made[prompt] = ctx.kv_create(Hkv, E, 4, r_i=8, key_index=True, unrolled_ladders=True)
        for k in range(E):
            kv.load(B.CM_KV_INDEX, k, ctx.encrypt(sk, ctx.encode(lay.pack_k_index(K1, k), 4), 100 + k))
        kv.set_tokens(cap)
        gqa = ctx.gqa(kv, t_kv if prompt else G)
        if keys is None:
            keys = ctx.keygen_rotations(sk, sorted(set(kv.steps() + gqa.steps() + ctx.gqa(kv, t_kv).steps())), 2, with_relin=True)
        q = rng.normal(size=(t if prompt else 1, Hkv, G, E)) * 0.2
        slots = np.zeros(ctx.S)
        for e in range(E):
            for hk in range(Hkv):
                for g in range(G):
                    for tau in range(len(q)):
                        slots[lay.slot(e, hk, g * t + tau)] = q[tau, hk, g, e]
        plain = ctx.gqa_qk(keys, gqa, ctx.encrypt(sk, ctx.encode(slots, 5), 9))
        bucket, table = np.minimum(np.arange(cap) // 16, 7), rng.normal(size=(Hkv * G, 8))
        bias = ctx.relbias(Hkv, E, table, bucket, plain[0].level, plain[0].scale, group=G, prompt=prompt, mask=-40.0, causal=True)
        for first in (-1, (page + 1) % E * t_kv):
            vecs = [ctx.decrypt(sk, s).real for s in ctx.relbias_apply(bias, token, plain, first=first)]
            for hk in range(Hkv):
                for g in range(G):
                    for tau in range(len(q)):
                        for key in range(cap):
                            c, j = key // t_kv, key % t_kv
                            delta = (j - (g * t + tau)) % t_kv if prompt else (j // t - g) % G
                            got, dot = vecs[delta][lay.slot(c, hk, j)], q[tau, hk, g] @ K1[key, hk]
                            if token + tau < key < (page + 1) * t_kv:
                                assert got - dot < -30.0
                            else:
                                assert abs(got - dot - table[hk * G + g][bucket[(token + tau - key) % cap]]) < 1e-4


def test_refusals(ctx):
    from paper_2602_11470_amd import binding as B
    table, bucket, h = np.zeros((8, 3)), np.zeros(512, dtype=np.int32), C.c_void_p()

    def create(flags, mask):
        return B.lib.cm_relbias_create_ex(ctx.h, 4, 16, 2, 0, 2, 0.0, 3, table.ctypes.data, bucket.ctypes.data, mask, flags, None, C.byref(h))
    assert create(2, -9.0) == -1 and create(1 << 31, -9.0) == -1 and create(3, -9.0) == -1
    assert create(B.CM_RELBIAS_CAUSAL, 0.0) == -1                            # nothing to put behind the query
    assert create(B.CM_RELBIAS_CAUSAL, float("nan")) == -1 and create(B.CM_RELBIAS_CAUSAL, -(2.0 ** 11)) == -1      # 2^11 * 2^50 does not fit
    assert h.value is None
    for flags, mask in ((B.CM_RELBIAS_CAUSAL, -9.0), (0, 0.0), (0, -9.0)):
        assert create(flags, mask) == 0
        B.lib.cm_relbias_destroy(h)


def test_memory_of_an_object_with_a_mask():
    """group * t_kv plaintexts, and one for every number of visible pages with hidden ones: less than one more is taken."""
    import torch
    from paper_2602_11470_amd import binding as B
    ctx = B.llama_ring(24, 4)
    try:
        heads, dim, level = 32, 64, 21
        cap = ctx.S // heads
        make = lambda: ctx.relbias(heads, dim, np.ones((heads, 2)), np.zeros(cap, dtype=np.int32), level, mask=-9.0)  # noqa: E731
        first = make()                                                       # what the context makes on the way
        torch.cuda.synchronize()
        before = torch.cuda.mem_get_info()[0]
        second = make()
        used = before - torch.cuda.mem_get_info()[0]
        pt = (level + 1) * ctx.n * 8
        assert 0 < used < (cap // dim + dim) * pt                           # memory that the runtime holds from the first counts as used before
        del first, second
    finally:
        ctx.close()
