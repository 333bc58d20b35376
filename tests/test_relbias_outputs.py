"""Which arrays of scores a bias refuses: an output whose words are another output's or, unless it is the pass's own input, an input's.  The rule is
called in the library; no GPU is needed."""
import ctypes as C

import numpy as np
import pytest

WORDS = 96


def _shared(ins, outs):
    """ins, outs: the first words of the ciphertexts, as numbers of words."""
    from paper_2602_11470_amd import binding as B
    f = B.lib._Z22relbias_outputs_sharedPK5cm_ctS1_im
    f.restype = C.c_bool
    a, b = ((B.cm_ct * len(x))(*[B.cm_ct((1 << 20) + 8 * w, 2, 2, 1.0) for w in x]) for x in (ins, outs))
    return f(a, b, len(ins), C.c_size_t(WORDS))


@pytest.mark.parametrize("n", [1, 2, 5, 16, 17, 40])
def test_in_place_out_of_place_and_touching(n):
    at = [i * WORDS for i in range(n)]
    assert not _shared(at, at)                                                # every pass in place
    assert not _shared(at, [(n + i) * WORDS for i in range(n)])               # the outputs right behind the inputs
    assert not _shared([(n + i) * WORDS for i in range(n)], at)
    assert not _shared([0] * n, [(1 + i) * WORDS for i in range(n)])          # one input in every pass
    assert not _shared([i for i in range(n)], [2 * n * WORDS + i * WORDS for i in range(n)])   # inputs that overlap one another
    assert not _shared(at, at[: n // 2] + [(n + i) * WORDS for i in range(n // 2, n)])


@pytest.mark.parametrize("n", [1, 2, 5, 16, 17, 40])
@pytest.mark.parametrize("off", [1, 32, WORDS - 1, -1, -32, -(WORDS - 1)])
def test_shifted_against_an_input_or_an_output(n, off):
    rng = np.random.default_rng(n)
    ins = (rng.permutation(n) * 4 * WORDS).tolist()
    outs = (rng.permutation(n) * 4 * WORDS + 2 * WORDS).tolist()
    assert not _shared(ins, outs)
    for p in {0, n // 2, n - 1}:
        for q in {0, n // 2, n - 1}:
            assert _shared(ins, [ins[q] + off if r == p else o for r, o in enumerate(outs)])          # over its own input (p == q), or another's
            if p != q:
                assert _shared(ins, [outs[q] + off if r == p else o for r, o in enumerate(outs)])
                assert _shared(ins, [outs[q] if r == p else o for r, o in enumerate(outs)])
                assert _shared(ins, [ins[q] if r == p else o for r, o in enumerate(outs)])
        assert not _shared(ins, [ins[p] if r == p else o for r, o in enumerate(outs)])


def test_against_every_pair():
    """Random places: the sorted rule for many passes and the pairwise one for few say what the definition says."""
    rng = np.random.default_rng(3)
    answers = []
    for n in (3, 16, 17, 30):
        for _ in range(300):
            span = int(rng.integers(2, 200)) * n
            ins, outs = rng.integers(0, span * WORDS // 8, size=(2, n)).tolist()
            if rng.uniform() < 0.7:
                outs = [WORDS * 2 * i + int(rng.integers(0, WORDS)) for i in rng.permutation(n).tolist()]
            if rng.uniform() < 0.5:
                ins = [o if rng.uniform() < 0.9 else w for o, w in zip(outs, ins)]
            cover = [(np.arange(WORDS) + o).tolist() for o in outs]
            want = any(set(cover[r]) & set(cover[p]) for r in range(n) for p in range(r))
            want |= any(abs(outs[r] - ins[p]) < WORDS and not (r == p and outs[r] == ins[p]) for r in range(n) for p in range(n))
            assert _shared(ins, outs) == want
            answers.append(want)
    assert 0.1 < np.mean(answers) < 0.9
