"""The cases of the cache and score operators (perf/operators.py): what the library's side keeps between them."""
import gc
import types
import weakref


def test_key_sets_held_are_bounded(monkeypatch):
    """One key of the large ring is 88 MB: sets of other steps push the oldest out, equal ones are the same set."""
    from perf import operators

    class Keys:
        pass
    made = []

    def keygen(sk, steps, seed):
        keys = Keys()
        made.append(weakref.ref(keys))
        return keys
    monkeypatch.setattr(operators, "_context", lambda ring: types.SimpleNamespace(keygen_secret=lambda seed: None, keygen_rotations=keygen))
    try:
        for i in range(10):
            assert operators._own_keys(operators.SMALL, (i, i + 1)) is operators._own_keys(operators.SMALL, (i, i + 1))
        gc.collect()
        assert len(made) == 10 and sum(r() is not None for r in made) <= operators._keys.cache_info().maxsize == 4
    finally:
        operators._own_keys.cache_clear()
