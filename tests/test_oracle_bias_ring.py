"""Causal bias where every page of the ring is in use, on plain slot vectors: a query at any residue of its page sees all live tokens, the first ones of
the oldest page among them, and none of the places behind it."""
import numpy as np
import pytest

from oracle import packing


@pytest.mark.parametrize("group,prompt", [(1, False), (2, False), (4, False), (1, True), (2, True), (4, True)])
@pytest.mark.parametrize("token", [0, 7, 20, 37, 63])
@pytest.mark.parametrize("hidden_pages", [None, 0, 1, 9])
def test_every_live_token_is_seen(token, group, prompt, hidden_pages):
    S, Hkv, E = 128, 3, 8                                        # three heads of a padded four, pages of four tokens
    lay = packing.KvLayout(S, Hkv, E)
    t_kv, cap = lay.t, E * lay.t
    token %= cap
    t = t_kv // group
    token -= token % t if prompt else 0
    page = token // t_kv
    # the window's first page: None and 0 hidden pages are the full ring, whose oldest page lies behind the query's
    first = None if hidden_pages is None else (page + 1 + hidden_pages) % E * t_kv
    pages = E if hidden_pages is None else (page - first // t_kv) % E + 1
    rng = np.random.default_rng(token)
    table, bucket = rng.normal(size=(Hkv * group, 7)), rng.integers(0, 7, cap)
    got = [lay.bias_slots(table, bucket, token, first, -9.0, group, d, prompt, causal=True) for d in range(t_kv if prompt else group)]
    for hk in range(Hkv):
        for g in range(group):
            for tau in range(t if prompt else 1):
                query = token + tau
                # the live tokens in their order: the window's pages, oldest first, up to the query
                live = [(page - pages + 1 + i) % E * t_kv + j for i in range(pages) for j in range(t_kv)]
                live = live[: live.index(query) + 1]
                assert len(live) == (pages - 1) * t_kv + query % t_kv + 1
                for age, key in enumerate(reversed(live)):
                    assert age == (query - key) % cap
                for key in range(cap):
                    c, j = key // t_kv, key % t_kv
                    delta = (j - (g * t + tau)) % t_kv if prompt else (j // t - g) % group
                    want = table[hk * group + g][bucket[(query - key) % cap]] + (0.0 if key in live else -9.0)
                    assert got[delta][lay.slot(c, hk, j)] == want


def test_a_bucket_of_the_largest_distances_hides_live_tokens():
    """Why the places behind the query are told by their place: in a full ring the oldest page has the same distances."""
    lay = packing.KvLayout(16, 1, 4)                             # four pages of four tokens
    bucket = (np.arange(16) > 16 - 4).astype(int)
    table = np.array([[0.0, -9.0]])
    slots = lay.bias_slots(table, bucket, 6)                     # page 1, residue 2
    assert np.flatnonzero(slots).tolist() == [7, 8, 9]           # place 7 lies behind the query; 8 and 9 are tokens of 14 and 13 steps ago
    slots = lay.bias_slots(np.zeros((1, 1)), np.zeros(16, dtype=int), 6, mask=-9.0, causal=True)
    assert np.flatnonzero(slots).tolist() == [7]


def test_a_page_on_is_the_same_plaintext_whole_rows_on():
    lay = packing.KvLayout(128, 2, 16)
    rng = np.random.default_rng(2)
    table, bucket = rng.normal(size=(8, 5)), rng.integers(0, 5, 64)
    for prompt, rest in ((False, 3), (False, 1), (True, 2)):
        for group in (1, 2, 4):
            if prompt and rest % (lay.t // group):
                continue
            for d in range(lay.t if prompt else group):
                at = lambda token: lay.bias_slots(table, bucket, token, None, -9.0, group, d, prompt, causal=True)  # noqa: E731
                assert np.array_equal(at(11 * lay.t + rest), np.roll(at(rest), 11 * lay.H * lay.t))
