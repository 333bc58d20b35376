"""Attention of drafted tokens on an encrypted cache, as cases for timing and comparison.

What a program that serves encrypted attention calls around its products, from the projections of one or several new tokens to
their scores and values:

  rotary    rotary positions of queries and keys at places that are given with the call: pairs of neighbouring dims or of the two
            halves of a head, a part of the head, frequencies scaled for long contexts, a position of its own for every token of a
            group (cm_rotary_set, cm_rotary_apply)
  append    a run of tokens, of any length up to a page and from any place on, put into the cache, the keys with their positions
            applied on the way (cm_kv_append_run)
  tree_qk   the scores of a group of drafted tokens against the cache, every token seeing what was committed, itself and the
            drafted tokens that it follows (cm_tree_qk)
  tree_sv   such scores times the values, summed over the passes (cm_tree_sv)

Inputs: a ciphertext's limbs are uniform residues under their moduli (what an encryption looks like without the secret key).
Positions and trees are data of the call.  Masks and tables of positions are plaintexts that a program keeps: their integer
coefficients are made here and given to both sides.  Keys are made from fixed seeds by the scheme's own counter-based generator.

The plain form writes the scheme out in 64-bit integer tensors: residues, the negacyclic transform stage by stage, the Galois
permutation, base conversion, key switch, rescale.  Every output is whole words, which have to be equal.

Layout (all heads padded to a power of two H; E dims; t = S / (H E) token residues; S = n / 2 slots; B = H t slots a row):
slot (e, h, r) = (e H + h) t + r.  Page c = the t tokens c t .. c t + t - 1, the token of place a at residue a mod t.  K ciphertext c
holds page c, V ciphertext k = g r_i + j page c in row c - j (mod E), as element c - j - g r_i, index ciphertext k page c in row
c + g r_i, as dim c + g r_i + j.  Scores hold page c in row c.
"""
import functools
import math
import random
from decimal import Decimal, getcontext

import numpy as np
import torch

own = False

DEVICE = "cuda" if torch.cuda.is_available() else "cpu"
# ring degree, bits of the first prime, of the other ciphertext primes, of the special primes; their counts; primes per
# key-switch digit, Hamming weight of the secret (0: uniform ternary), log2 of the scale
RINGS = {"4096: 5+1": (4096, 50, 40, 60, 5, 1, 1, 0, 40), "65536: 24+4": (65536, 50, 50, 60, 24, 4, 4, 192, 50)}
SMALL, BIG = RINGS
MASK = -24.0                # what hides a place from a query: added to its score


# ---- cases ------------------------------------------------------------------------------------------------------
def _rotary(name, ring, heads, dim, level, rot, halves, scaling, room, position, live, count):
    """room: positions the tables hold.  live: the residues that hold a token and how their positions follow from `position`."""
    return dict(name=name, op="rotary", ring=ring, heads=heads, dim=dim, level=level, rot=rot, halves=halves, scaling=scaling, room=room,
                position=position, live=live, count=count)


def _append(name, ring, heads, dim, r_i, index, level, tokens, run, rotary, room):
    """tokens: in the cache before; run: appended.  rotary: "" (keys as they are), "pairs" or "halves"."""
    return dict(name=name, op="append", ring=ring, heads=heads, dim=dim, r_i=r_i, index=index, level=level, tokens=tokens, run=run,
                rotary=rotary, room=room)


def _tree(name, op, ring, heads, dim, group, r_i, level, base, nodes, first, tree):
    """base: committed tokens; nodes: drafted ones behind them; tree: the seed of their shape; first: the first token that is seen."""
    return dict(name=name, op=op, ring=ring, heads=heads, dim=dim, group=group, r_i=r_i, level=level, base=base, nodes=nodes, first=first,
                tree=tree)


def listed():
    return [
        # the smallest call: the query of one token, pairs of halves, small ring
        _rotary("rotary_small", SMALL, 4, 16, 2, 16, True, "", 512, 300, "one 5", 1),
        # query and key of a decode step's token, 32 heads of 128 dims, neighbouring pairs, at the level the paper works at
        _rotary("rotary_decode", BIG, 32, 128, 3, 128, False, "", 1024, 777, "one 1", 2),
        # a group of prompt tokens in the middle of the chain, the first half of each head turned, scaled for a context four times as long
        _rotary("rotary_group_partial", BIG, 32, 128, 12, 64, True, "bands 4 1 8 256", 1024, 640, "group", 2),
        # drafted tokens of a tree at the top level: 8 heads, 21 of a page's 32 residues, each at its depth behind the context
        _rotary("rotary_tree", BIG, 8, 128, 22, 128, True, "", 4096, 4000, "tree 27 21 5", 2),
        # one token into a small cache
        _append("append_small", SMALL, 4, 16, 16, False, 2, 77, 1, "pairs", 512),
        # five drafted tokens that begin in one page and end in the next
        _append("append_draft", BIG, 32, 128, 16, False, 4, 126, 5, "halves", 1024),
        # the same number into a cache with the key index
        _append("append_index", BIG, 32, 128, 16, True, 4, 121, 5, "halves", 1024),
        # the ragged end of a prompt in the middle of the chain, keys without positions
        _append("append_ragged", BIG, 8, 128, 16, False, 9, 96, 21, "", 0),
        # a tree of six on the small ring
        _tree("tree_qk_small", "tree_qk", SMALL, 8, 32, 1, 8, 3, 101, 6, 0, 1),
        _tree("tree_sv_small", "tree_sv", SMALL, 8, 32, 2, 8, 3, 101, 6, 0, 1),
        # eight drafted tokens behind a context that ends inside a page, its oldest pages out of sight
        _tree("tree_qk_draft", "tree_qk", BIG, 32, 128, 1, 16, 4, 900, 8, 256, 2),
        _tree("tree_sv_draft", "tree_sv", BIG, 32, 128, 1, 16, 3, 900, 8, 256, 2),
    ]


def draw(rng):
    def logpick(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotary", "rotary", "rotary", "append", "append", "append", "tree_qk", "tree_sv"])
    small = rng.random() < (0.4 if op in ("rotary", "append") else 0.8)
    ring = SMALL if small else BIG
    if op.startswith("tree"):
        heads, dim = rng.choice([(8, 32), (4, 64), (16, 16), (4, 128), (16, 32), (6, 32)] if small else [(64, 64), (32, 128), (64, 128), (40, 64)])
        t = _residues_of(ring, heads, dim)
        base = logpick(1, dim * t - t)
        first = rng.choice([0, 0, base // t // 2 * t])
        return _without_name(_tree("", op, ring, heads, dim, rng.choice([g for g in (1, 1, 2, 4) if g <= t]), rng.choice([r for r in (8, 16) if r <= dim]),
                                   rng.randint(2, 3) if small else 3, base, rng.randint(1, t), first, rng.randrange(99)))
    heads, dim = rng.choice([(4, 16), (2, 64), (8, 32), (3, 32), (4, 128), (1, 128)] if small else [(32, 128), (32, 64), (12, 64), (8, 128), (64, 64)])
    t = _residues_of(ring, heads, dim)
    if op == "rotary":
        room = logpick(64, 1024)
        run = rng.randint(1, t)
        live = rng.choice(["one %d" % rng.randrange(t), "group", "tree %d %d %d" % (rng.randrange(t), run, rng.randrange(99)), "gaps %d" % rng.randrange(99)])
        return _without_name(_rotary("", ring, heads, dim, rng.randint(1, 4) if small else logpick(1, 20), rng.choice([dim, dim, dim // 2, dim // 4]),
                                     rng.random() < 0.5, rng.choice(["", "linear 4", "bands 4 1 8 256", "base 8"]), max(room, 2 * t),
                                     rng.randrange(max(room, 2 * t) - t), live, rng.choice([1, 1, 2, 3])))
    r_i = rng.choice([r for r in (dim, dim // 8, 16, 4) if 1 <= r <= dim])
    index = rng.random() < 0.4
    level = 2 if small else logpick(2, 8)
    run = rng.randint(1, t)
    tokens = rng.randrange(min(512, dim * t) - run + 1)
    return _without_name(_append("", ring, heads, dim, r_i, index, level, tokens, run, rng.choice(["", "pairs", "halves"]), 512))


def _without_name(case):
    del case["name"]
    return case


def _residues_of(ring, heads, dim):
    return RINGS[ring][0] // 2 // ((1 << (heads - 1).bit_length()) * dim)


def _shape(case):
    """(H padded, E, t, r_i, r_o) of a cache."""
    hp, dim = 1 << (case["heads"] - 1).bit_length(), case["dim"]
    r_i = case.get("r_i", dim)
    return hp, dim, RINGS[case["ring"]][0] // 2 // (hp * dim), r_i, dim // r_i


def _parents(nodes, seed):
    """A tree: of every drafted token the one that it follows (-1: the last committed token), earlier ones more often."""
    rng = random.Random(seed)
    return [-1 if i == 0 else max(-1, min(i - 1, int(rng.random() ** 2 * (i + 1)) - 1)) for i in range(nodes)]


def _positions(case):
    """Position of the token at every residue, -1 where there is none."""
    _, _, t, _, _ = _shape(case)
    if case["op"] == "append":
        start, run = case["tokens"], case["run"]
        return [next((a for a in range(start, start + run) if a % t == r), -1) for r in range(t)]
    what, *args = case["live"].split()
    args = [int(a) for a in args]
    if what == "one":
        return [case["position"] if r == args[0] else -1 for r in range(t)]
    if what == "group":
        return [case["position"] + r for r in range(t)]
    out = [-1] * t
    if what == "tree":
        depth = []
        for i, p in enumerate(_parents(args[1], args[2])):
            depth.append(0 if p < 0 else depth[p] + 1)
            out[(args[0] + i) % t] = case["position"] + depth[i]
        return out
    rng = random.Random(args[0])
    return [rng.randrange(case["room"]) if rng.random() < 0.6 else -1 for _ in range(t)]


# ---- the scheme's constants ---------------------------------------------------------------------------------------
def _is_prime(m):
    if any(m % p == 0 for p in (2, 3, 5, 7, 11, 13)):
        return False
    d = m - 1
    r = (d & -d).bit_length() - 1
    return all(x in (1, m - 1) or any(pow(x, 1 << i, m) == m - 1 for i in range(1, r)) for x in (pow(a, d >> r, m) for a in (2, 3, 5, 7, 11, 13, 17, 19, 23, 29, 31, 37)))


def _primes(bits, n, count):
    found = (c for c in ((1 << bits) + 1 - k * 2 * n for k in range(1, 1 << 20)) if _is_prime(c))
    return [next(found) for _ in range(count)]


@functools.lru_cache(None)
def _moduli(ring):
    n, b0, bq, bp, nq, np_, _, _, _ = RINGS[ring]
    q = _primes(bq, n, nq) if b0 == bq else _primes(b0, n, 1) + _primes(bq, n, nq - 1)
    return q + _primes(bp, n, np_)


def _psi(q, n):
    """The smallest-base primitive 2n-th root of unity."""
    return next(w for w in (pow(x, (q - 1) // (2 * n), q) for x in range(2, 1000)) if pow(w, n, q) == q - 1)


def _ints(values):
    return torch.tensor([int(v) for v in values], dtype=torch.int64, device=DEVICE)


@functools.lru_cache(None)
def _places(n):
    """Bit-reversed indices."""
    i, r = torch.arange(n, device=DEVICE), torch.zeros(n, dtype=torch.int64, device=DEVICE)
    for b in range(n.bit_length() - 1):
        r |= ((i >> b) & 1) << (n.bit_length() - 2 - b)
    return r


@functools.lru_cache(None)
def _twiddles(ring, limbs, inverse):
    """psi^brev(k) of the moduli, or their inverses, [limbs][n]."""
    n, mods = RINGS[ring][0], [_moduli(ring)[i] for i in limbs]
    base = [pow(_psi(m, n), -1 if inverse else 1, m) for m in mods]
    out = torch.ones(len(mods), 1, dtype=torch.int64, device=DEVICE)
    while out.shape[1] < n:                                                  # psi^0 .. psi^(2^b - 1), then the next half
        out = torch.cat([out, _mul(out, _ints(pow(w, out.shape[1], m) for w, m in zip(base, mods))[:, None], *_q(ring, limbs))], 1)
    return out[:, _places(n)].contiguous()


# ---- residues -----------------------------------------------------------------------------------------------------
def _mul30(a, s, q):
    """a s mod q for a below q < 2^61 and s below 2^30: the quotient is below 2^30, so a double has it up to one."""
    r = a * s - (a.double() * s.double() / q.double()).long() * q
    return torch.where(r < 0, r + q, torch.where(r >= q, r - q, r))


def _mul(a, b, q, wide):
    """a b mod q, whole words.  Below 2^50 the quotient fits a double; larger moduli (wide) take b in two halves."""
    if not wide:
        r = a * b - (a.double() * b.double() / q.double()).long() * q
        return torch.where(r < 0, r + q, torch.where(r >= q, r - q, r))
    hi = _mul30(_mul30(a, b >> 30, q), torch.full_like(q, 1 << 30), q)
    return _add(hi, _mul30(a, b & ((1 << 30) - 1), q), q)


def _add(a, b, q):
    s = a + b
    return torch.where(s >= q, s - q, s)


def _sub(a, b, q):
    s = a - b
    return torch.where(s < 0, s + q, s)


@functools.lru_cache(None)
def _q(ring, limbs):
    """Moduli of limbs, [limbs][1], and whether they need wide products."""
    mods = [_moduli(ring)[i] for i in limbs]
    return _ints(mods)[:, None], max(mods) >= 1 << 50


@functools.lru_cache(None)
def _inverses(ring, limbs, value):
    """value^-1 mod q_i of limbs, [limbs][1]."""
    return _ints(pow(value, -1, _moduli(ring)[i]) for i in limbs)[:, None]


def _span(level):
    return tuple(range(level + 1))


def _ntt(x, ring, limbs):
    """Negacyclic transform of x[..., limb, n]: place i holds the value at psi^(2 brev(i) + 1)."""
    n, tw, (q, wide), m = x.shape[-1], _twiddles(ring, limbs, False), _q(ring, limbs), 1
    q = q[:, None]
    while m < n:
        a = x.reshape(*x.shape[:-1], m, 2, n // (2 * m))
        hi = _mul(a[..., 1, :], tw[:, m: 2 * m, None], q, wide)
        x = torch.stack([_add(a[..., 0, :], hi, q), _sub(a[..., 0, :], hi, q)], -2).reshape(x.shape)
        m *= 2
    return x


def _intt(x, ring, limbs):
    n, tw, (q, wide), m = x.shape[-1], _twiddles(ring, limbs, True), _q(ring, limbs), x.shape[-1] // 2
    q = q[:, None]
    while m:
        a = x.reshape(*x.shape[:-1], m, 2, n // (2 * m))
        lo, hi = _add(a[..., 0, :], a[..., 1, :], q), _mul(_sub(a[..., 0, :], a[..., 1, :], q), tw[:, m: 2 * m, None], q, wide)
        x = torch.stack([lo, hi], -2).reshape(x.shape)
        m //= 2
    return _mul(x, _inverses(ring, limbs, n), *_q(ring, limbs))


def _galois(ring, step):
    """Galois element of a left rotation by `step` slots."""
    n = RINGS[ring][0]
    return pow(5, step % (n // 2), 2 * n)


@functools.lru_cache(256)
def _perm(g, n):
    """out[i] = in[_perm(g)[i]] maps X to X^g: place i of exponent e = 2 brev(i) + 1 takes the value at exponent e g."""
    brev = _places(n)
    return brev[(((2 * brev + 1) * g) % (2 * n) - 1) // 2]


def _rescale(c, ring):
    """c[..., l + 1, n] divided by its last modulus, floor."""
    l = c.shape[-2] - 1
    limbs, (q, wide) = _span(l - 1), _q(ring, _span(l - 1))
    last = _intt(c[..., l:, :], ring, (l,)) % q
    return _mul(_sub(c[..., :l, :], _ntt(last, ring, limbs), q), _inverses(ring, limbs, _moduli(ring)[l]), q, wide)


@functools.lru_cache(None)
def _conversion(ring, src, dst):
    """Of a base conversion: the inverses of B / q_m under the sources, and B / q_m under the targets."""
    mods = _moduli(ring)
    big = math.prod(mods[i] for i in src)
    return _ints(pow(big // mods[i], -1, mods[i]) for i in src)[:, None], [_ints(big // mods[i] % mods[j] for j in dst)[:, None] for i in src]


def _convert(x, ring, src, dst):
    """Fast base conversion of x[..., len(src), n], coefficients, to the moduli dst."""
    inv, weights = _conversion(ring, src, dst)
    r, wide = _q(ring, dst)
    y = _mul(x, inv, *_q(ring, src))
    return functools.reduce(lambda a, b: _add(a, b, r), (_mul(y[..., k: k + 1, :] % r, w, r, wide) for k, w in enumerate(weights)))


def _moddown(u, ring, level):
    mods, nq = _moduli(ring), RINGS[ring][4]
    limbs, special, (q, wide) = _span(level), tuple(range(nq, len(mods))), _q(ring, _span(level))
    conv = _ntt(_convert(_intt(u[..., level + 1:, :], ring, special), ring, special, limbs), ring, limbs)
    return _mul(_sub(u[..., : level + 1, :], conv, q), _inverses(ring, limbs, math.prod(mods[nq:])), q, wide)


def _extended(ring, level):
    """Limbs of the extended basis: the ciphertext's and the special ones."""
    return _span(level) + tuple(range(RINGS[ring][4], len(_moduli(ring))))


def _raise(d, ring):
    """Digits of d[..., l + 1, n] on the extended basis, [..., digit, ext, n]."""
    level, alpha = d.shape[-2] - 1, RINGS[ring][6]
    ext, coeff, out = _extended(ring, level), _intt(d, ring, _span(level)), []
    for lo in range(0, level + 1, alpha):
        hi = min(lo + alpha, level + 1)
        others = tuple(i for i in ext if not lo <= i < hi)
        raised = _ntt(_convert(coeff[..., lo:hi, :], ring, tuple(range(lo, hi)), others), ring, others)
        out.append(torch.cat([raised[..., :lo, :], d[..., lo:hi, :], raised[..., lo:, :]], -2))
    return torch.stack(out, -3)


def _switch(digits, ring, g, key, level):
    """sum_j of the digits [..., digit, ext, n] through the Galois map times key[digit][2][ext][n]: [..., 2, ext, n]."""
    q, wide = _q(ring, _extended(ring, level))
    digits = digits[..., _perm(g, digits.shape[-1])] if g else digits
    return functools.reduce(lambda a, b: _add(a, b, q), (_mul(digits[..., j, None, :, :], k, q, wide) for j, k in enumerate(key)))


def _times_p(c, ring):
    """c[..., l + 1, n] times the product of the special moduli, on the extended basis (nothing on the special limbs)."""
    level, mods = c.shape[-2] - 1, _moduli(ring)
    p = math.prod(mods[RINGS[ring][4]:])
    out = _mul(c, _ints(p % mods[i] for i in _span(level))[:, None], *_q(ring, _span(level)))
    return torch.cat([out, out.new_zeros(*c.shape[:-2], len(mods) - RINGS[ring][4], c.shape[-1])], -2)


def _turn_raised(raised, digits, ring, g, key):
    """A rotation that stays on the extended basis: of the ciphertexts whose first component times P is raised [..., ext, n]."""
    level = raised.shape[-2] - 1 - RINGS[ring][5]
    one = _switch(digits, ring, g, key, level)
    one[..., 0, :, :] = _add(one[..., 0, :, :], raised[..., _perm(g, raised.shape[-1])], _q(ring, _extended(ring, level))[0])
    return one


def _weighted(c, ring, terms, here=None, digits=None):
    """here c + the rotations of c times plaintexts, on the extended basis: c[..., 2, l + 1, n], terms (Galois element, key,
    plaintext[ext][n]), here a plaintext[ext][n].  The rotations share their digits."""
    level = c.shape[-2] - 1
    q, wide = _q(ring, _extended(ring, level))
    raised, digits = _times_p(c, ring), _raise(c[..., 1, :, :], ring) if digits is None else digits
    parts = [_mul(raised, here, q, wide)] if here is not None else []
    parts += [_mul(_turn_raised(raised[..., 0, :, :], digits, ring, g, key), plain, q, wide) for g, key, plain in terms]
    return functools.reduce(lambda a, b: _add(a, b, q), parts)


def _rotations(c, ring, steps, keys):
    """The ciphertexts c[..., 2, l + 1, n] and their left rotations by steps, which share their digits, [1 + steps, ..., 2, l + 1, n]."""
    level = c.shape[-2] - 1
    if not steps:
        return c[None]
    digits, galois = _raise(c[..., 1, :, :], ring), [_galois(ring, step) for step in steps]
    out = _moddown(torch.stack([_switch(digits, ring, g, keys[g], level) for g in galois]), ring, level)
    turned = torch.stack([c[..., 0, :, :][..., _perm(g, c.shape[-1])] for g in galois])
    out[..., 0, :, :] = _add(out[..., 0, :, :], turned, _q(ring, _span(level))[0])
    return torch.cat([c[None], out])


# ---- keys: the scheme's counter-based generator, in tensors of 64-bit words ------------------------------------------
GOLD, M64 = 0x9E3779B97F4A7C15, (1 << 64) - 1


def _signed(v):
    v &= M64
    return v - (1 << 64) if v >> 63 else v


def _shr(z, s):
    return (z >> s) & ((1 << (64 - s)) - 1)


def _mix(z):
    """The finaliser of SplitMix64, on an integer or on a tensor of words."""
    if isinstance(z, int):
        z &= M64
        z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9 & M64
        z = (z ^ (z >> 27)) * 0x94D049BB133111EB & M64
        return z ^ (z >> 31)
    z = (z ^ _shr(z, 30)) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ _shr(z, 27)) * _signed(0x94D049BB133111EB)
    return z ^ _shr(z, 31)


def _stream(seed, purpose, ident=0, digit=0, limb=0):
    return _mix(_mix(seed) ^ (purpose << 56 | ident << 16 | digit << 8 | limb))


def _draw_words(key, n, attempt=0):
    ctr = torch.arange(n, device=DEVICE) + (attempt << 32) + 1
    return _mix(ctr * _signed(GOLD) + _signed(key))


def _uniform(key, q, n):
    """Residues under q: the first of an element's draws below q floor(2^64 / q), mod q."""
    v, attempt, bound = _draw_words(key, n), 0, _signed(q * ((1 << 64) // q)) ^ -(1 << 63)
    while bool((bad := (v ^ -(1 << 63)) >= bound).any()):
        attempt += 1
        v = torch.where(bad, _draw_words(key, n, attempt), v)
    qt = _ints([q])
    return _add(_mul(_shr(v, 32) % qt, _ints([(1 << 32) % q]), qt, True), (v & 0xFFFFFFFF) % qt, qt)


@functools.lru_cache(None)
def _gauss_table():
    """2^63 times the cumulative probabilities of the magnitudes of the error, a Gaussian of sigma 3.2 cut at 19."""
    getcontext().prec = 80
    w = [(-(Decimal(k) ** 2) / (2 * Decimal("3.2") ** 2)).exp() * (1 if k == 0 else 2) for k in range(20)]
    z = sum(w)
    return [int(sum(w[: k + 1]) / z * (1 << 63)) for k in range(19)]


@functools.lru_cache(None)
def _secret(ring, seed):
    """Ternary secret, int64[n]."""
    n, h, key = RINGS[ring][0], RINGS[ring][7], _stream(seed, 1)
    one = lambda ctr: _mix(key + (ctr + 1) * GOLD)  # noqa: E731
    if h == 0:
        return _ints((0, 1, -1)[one(i) % 3] for i in range(n))
    s, perm = [0] * n, list(range(n))
    for i in range(h):
        j = i + one(i) % (n - i)
        perm[i], perm[j] = perm[j], perm[i]
        s[perm[i]] = -1 if one(n + i) & 1 else 1
    return _ints(s)


def _key(ring, g, level, secret_seed=1, seed=2):
    """Evaluation key of the Galois element g (0: of the secret's square) as far as a level uses it, [digit][2][ext][n]: b = -a s + e +
    [P on the digit's own limbs] s(X^g), and a."""
    n, mods, nq, alpha = RINGS[ring][0], _moduli(ring), RINGS[ring][4], RINGS[ring][6]
    limbs, p = _extended(ring, level), math.prod(mods[nq:])
    q, wide = _q(ring, limbs)
    s = _ntt(_secret(ring, secret_seed)[None] % q, ring, limbs)
    target = s[:, _perm(g, n)] if g else _mul(s, s, q, wide)
    noise, digits = _mix(_mix(secret_seed) ^ 6 << 56), []
    table = _ints(_gauss_table())
    for j, lo in enumerate(range(0, level + 1, alpha)):
        a = torch.stack([_uniform(_stream(seed, 2, g, j, i), mods[i], n) for i in limbs])
        v = _draw_words(_stream(seed ^ noise, 3, g, j), n)
        e = (_shr(v, 1)[:, None] >= table).sum(1)
        e = _ntt(torch.where(v & 1 == 1, -e, e)[None] % q, ring, limbs)
        factor = _ints(p % mods[i] if lo <= i < min(lo + alpha, nq) else 0 for i in limbs)[:, None]
        digits.append(torch.stack([_add(_sub(e, _mul(a, s, q, wide), q), _mul(target, factor, q, wide), q), a]))
    return torch.stack(digits)


@functools.lru_cache(4)
def _keys(ring, galois, level):
    return {g: _key(ring, g, level) for g in galois}


# ---- plaintexts -----------------------------------------------------------------------------------------------------
@functools.lru_cache(None)
def _slot_places(n):
    g, out = 1, np.empty(n // 2, dtype=np.int64)
    for j in range(n // 2):
        out[j] = (g - 1) // 2
        g = g * 5 % (2 * n)
    return out


def _coefficients(slots, n, scale):
    """round(scale m_k) of the real polynomials whose slot values are slots[..., S]."""
    v = np.zeros(slots.shape[:-1] + (n,), dtype=np.complex128)
    v[..., _slot_places(n)] = slots
    v[..., n - 1 - _slot_places(n)] = slots
    return np.rint((np.fft.fft(v) * np.exp(-1j * np.pi * np.arange(n) / n) / n).real * scale).astype(np.int64)


def _plaintext(coeffs, ring, limbs):
    coeffs = torch.from_numpy(coeffs).to(DEVICE) if isinstance(coeffs, np.ndarray) else coeffs
    return _ntt(coeffs[..., None, :] % _q(ring, limbs)[0], ring, limbs)


def _key_of(case):
    """What a case's plaintexts depend on, as a key of the caches below."""
    return tuple(sorted((k, v) for k, v in case.items() if k in ("op", "ring", "heads", "dim", "level", "rot", "halves", "scaling", "room", "rotary", "index")))


def _rotation(case):
    """Of a case with rotary positions: (dims turned, whether the pairs are halves, scaling, level of the keys)."""
    if case["op"] == "rotary":
        return case["rot"], case["halves"], case["scaling"], case["level"]
    return case["dim"], case["rotary"] == "halves", "", case["level"] + (2 if case["index"] else 1)


def _frequencies(rot, scaling):
    """Angles a position of the pairs, and the factor of cosines and sines."""
    what, *args = scaling.split() or [""]
    args = [float(a) for a in args]
    freq = 10000.0 ** (-2.0 * np.arange(rot // 2) / rot)
    if what == "linear":
        return freq / args[0], 1.0
    if what == "base":
        return (10000.0 * args[0] ** (rot / (rot - 2))) ** (-2.0 * np.arange(rot // 2) / rot) if rot > 2 else freq, 1.0
    if what == "bands":                     # turns within the original context: many kept, few slowed down, a ramp between
        factor, low, high, context = args
        keep = np.clip((context * freq / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        return keep * freq + (1 - keep) * freq / factor, 1.0 + 0.1 * math.log(factor)
    return freq, 1.0


def _table_sizes(room):
    """Positions are R high + low: (R, number of high parts)."""
    r = 1 << (max(room - 1, 0).bit_length() + 1) // 2
    return r, -(-room // r)


def _pair_modulus(ring):
    """Indices of the two moduli that the tables are multiplied under: the first special one, and the one whose value is the scale of the
    high parts."""
    nq, n_p = RINGS[ring][4], RINGS[ring][5]
    return nq, nq + 1 if n_p > 1 else 0


@functools.lru_cache(4)
def _table(key):
    """Coefficients of the tables of positions: for every low part cosines in the first and in the second rows of the pairs, then sines
    likewise, all at residue 0; ones in the rows that are not turned, residue 0; for every high part cosines (one in rows not
    turned) and sines in all slots."""
    case = dict(key)
    rot, halves, scaling, level = _rotation(case)
    (hp, dim, t, _, _), ring = _shape(case), case["ring"]
    n, room = RINGS[ring][0], case["room"]
    (freq, gain), (r, high), e = _frequencies(rot, scaling), _table_sizes(room), np.arange(dim)
    first = (e < rot // 2) if halves else (e < rot) & (e % 2 == 0)
    second = (e < rot) & ~first
    theta = np.where(e < rot, freq[np.minimum(e % (rot // 2) if halves else e // 2, rot // 2 - 1)], 0.0)
    rows = []
    for i in range(r):
        rows += [gain * np.cos(i * theta) * first, gain * np.cos(i * theta) * second, gain * np.sin(i * theta) * first, gain * np.sin(i * theta) * second]
    rows.append((e >= rot).astype(float))
    low = np.zeros((len(rows), dim, hp, t))
    low[..., 0] = np.array(rows)[:, :, None]
    high_rows = np.stack([f(h * r * theta) for h in range(high) for f in (np.cos, np.sin)])
    full = np.broadcast_to(high_rows[:, :, None, None], (2 * high, dim, hp, t))
    mods, (_, second_mod) = _moduli(ring), _pair_modulus(ring)
    return np.concatenate([_coefficients(part.reshape(-1, dim * hp * t), n, float(mods[m])) for x, m in ((low, level), (full, second_mod))
                           for part in np.array_split(x, max(1, len(x) // 32))])


@functools.lru_cache(8)
def _run_masks(key):
    """Coefficients of the masks of an append: the slots of residue 0, and those of row 0 at residue 0."""
    case = dict(key)
    hp, dim, t, _, _ = _shape(case)
    m = np.zeros((2, dim, hp, t))
    m[0, :, :, 0] = 1
    m[1, 0, :, 0] = 1
    return _coefficients(m.reshape(2, -1), RINGS[case["ring"]][0], float(_moduli(case["ring"])[case["level"] + 1]))


def _score_scale(case):
    """Of the scores of a query at the context's scale against keys at it."""
    return 2.0 ** (2 * RINGS[case["ring"]][8]) / _moduli(case["ring"])[case["level"]]


@functools.lru_cache(8)
def _tree_coefficients(key):
    """Coefficients of the masks of a tree's passes: of the residues from 1, 2, .. t - 1 on, for the queries and for the results, then
    MASK at row 0, residue 0, and in all of row 0."""
    case = dict(key)
    (hp, dim, t, _, _), ring, mods = _shape(case), case["ring"], _moduli(case["ring"])
    from_on = (np.arange(t) >= np.arange(1, t)[:, None]).astype(float)
    slots = np.broadcast_to(from_on[:, None, :], (t - 1, dim * hp, t)).reshape(t - 1, dim * hp * t)
    rows = np.zeros((2, dim, hp, t))
    rows[0, 0, :, 0] = rows[1, 0] = MASK
    n = RINGS[ring][0]
    parts = [_coefficients(slots, n, float(mods[case["level"] + 1])), _coefficients(slots, n, float(mods[case["level"] - 1]))] if t > 1 else []
    return np.concatenate(parts + [_coefficients(rows.reshape(2, -1), n, _score_scale(case))])


def _hidden(case):
    """Of every pass, the (row behind the first drafted token's page, residue) of the places that its queries may not see among those
    from that page's on to the last drafted token's: pass delta holds at residue j the scores of the query of slot (j - delta) mod t."""
    _, _, t, _, _ = _shape(case)
    base, nodes, per = case["base"], case["nodes"], t // case["group"]
    follows, start = [], base % t
    for i, p in enumerate(_parents(nodes, case["tree"])):
        follows.append({i} | (follows[p] if p >= 0 else set()))
    out = []
    for delta in range(t):
        hidden = []
        for place in range(t * -(-(start + nodes) // t)):
            u = (place - delta) % t % per                             # the query's residue among those of its head
            node, at = (u - base) % per, place - start
            if at >= 0 and not (node < nodes and at in follows[node]):
                hidden.append((place // t, place % t))
        out.append(hidden)
    return out


# ---- states ---------------------------------------------------------------------------------------------------------
def _residues(ring, shape, limbs, gen):
    """Uniform residues [*shape][limbs][n]."""
    n, mods = RINGS[ring][0], _moduli(ring)
    out = torch.empty(*shape, limbs, n, dtype=torch.int64, device=DEVICE)
    for i in range(limbs):
        out[..., i, :] = torch.empty(*shape, n, dtype=torch.int64, device=DEVICE).random_(0, mods[i], generator=gen)
    return out


def _pages(case):
    """Pages of K ciphertexts that the case's cache has."""
    _, _, t, _, _ = _shape(case)
    return -(-(case["tokens"] + case["run"] if case["op"] == "append" else case["base"] + case["nodes"]) // t)


def _step_of_pairs(case):
    rot, halves, _, _ = _rotation(case)
    hp, _, t, _, _ = _shape(case)
    return (rot // 2 if halves else 1) * hp * t


def _steps(case):
    """Rotation steps of a case (left)."""
    hp, dim, t, r_i, r_o = _shape(case)
    b, steps = hp * t, []
    if case["op"] == "rotary" or case.get("rotary"):
        steps += [_step_of_pairs(case), -_step_of_pairs(case)]
    if case["op"] == "append":
        steps += [-g * r_i * b for g in range(1, r_o)] + ([j * b for j in range(1, r_i)] if case["index"] else [])
    if case["op"].startswith("tree"):
        steps += [j * b for j in range(1, r_i)] + [g * r_i * b for g in range(1, r_o)]
        steps += [s for d in range(1, t) for s in (-d, t - d)]
    return steps


def prepare(case, seed):
    gen, ring = torch.Generator(device=DEVICE).manual_seed(int(seed)), case["ring"]
    _, dim, t, r_i, r_o = _shape(case)
    level, op, s = case["level"], case["op"], dict(case=case)
    if op == "rotary":
        words = dict(x=_residues(ring, (case["count"], 2), level + 1, gen))
    elif op == "append":
        words = dict(k=_residues(ring, (2,), _rotation(case)[3] + 1 if case["rotary"] else level + 2, gen), v=_residues(ring, (2,), level + 2, gen))
        sizes = {"K": (_pages(case),), "V": (dim,)} | ({"X": (r_o, r_i)} if case["index"] else {})
        words |= {w: _residues(ring, (*z, 2), level + 1, gen) for w, z in sizes.items()}
    elif op == "tree_qk":
        words = dict(q=_residues(ring, (2,), level + 2, gen), X=_residues(ring, (r_o, r_i, 2), level + 1, gen))
    else:
        words = dict(scores=_residues(ring, (t, 2), level + 1, gen), V=_residues(ring, (r_o * r_i, 2), level + 1, gen))
    if own:
        return _own_state(s, words)
    s |= words
    lk = level + 1 if op in ("append", "tree_qk") else level
    galois = tuple(sorted({_galois(ring, x) for x in _steps(case)} | ({0} if op.startswith("tree") else set())))
    s["keys"] = {g: _keys(ring, galois, _rotation(case)[3] if case.get("rotary") or op == "rotary" else lk)[g] for g in galois}
    if op == "rotary" or case.get("rotary"):
        s["low"], s["high"] = _plain_tables(case)
        if op == "append":                               # the positions are set once for all layers
            parts = [lambda r: True] if case["index"] else _page_parts(case)
            s["turns"] = [_turns(s, [p if keep(r) else -1 for r, p in enumerate(_positions(case))]) for keep in parts]
    if op == "append":
        s["masks"] = _plaintext(_run_masks(_key_of(case)), ring, _span(level + 1))
    elif op.startswith("tree"):
        coeffs = torch.from_numpy(_tree_coefficients(_key_of(case))).to(DEVICE)
        qk = op == "tree_qk"
        at = level + 1 if qk else level - 1
        scale = int(_moduli(ring)[at])
        masks = coeffs[: t - 1] if qk else coeffs[t - 1: 2 * t - 2]
        rest = -masks
        rest[:, 0] += scale                              # the scale everywhere, less the mask
        s["from"], s["below"] = (_plaintext(m, ring, _extended(ring, at)) for m in (masks, rest))
        s["one"], s["row"] = _plaintext(coeffs[-2:], ring, _span(level - 1))
    return s


def _plain_tables(case):
    """The entries of the tables that the case's positions use, under both moduli: {low part: [4][2][n]}, {high part: [2][2][n]}."""
    coeffs, (r, _), mods = _table(_key_of(case)), _table_sizes(case["room"]), _pair_modulus(case["ring"])
    used = [p for p in _positions(case) if p >= 0]
    low = {i: _plaintext(coeffs[4 * i: 4 * i + 4], case["ring"], mods) for i in {p % r for p in used}}
    low[None] = _plaintext(coeffs[4 * r], case["ring"], mods)
    at = 4 * r + 1
    return low, {h: _plaintext(coeffs[at + 2 * h: at + 2 * h + 2], case["ring"], mods) for h in {p // r for p in used}}


# ---- the plain form -------------------------------------------------------------------------------------------------
def _turns(s, positions):
    """Plaintexts of the rotary positions on the extended basis: of what stays in its row, and of the rotations up and down (one where
    they are the same).  Of angles that are sums the cosines and sines are products of the tables', under two moduli; division
    by the second rounds to the nearest."""
    case = s["case"]
    ring, level = case["ring"], _rotation(case)[3]
    hp, dim, t, _, _ = _shape(case)
    n, (r, _), two = RINGS[ring][0], _table_sizes(case["room"]), _pair_modulus(ring)
    q, wide = _q(ring, two)
    mul, add, sub = (lambda a, b: _mul(a, b, q, wide)), (lambda a, b: _add(a, b, q)), (lambda a, b: _sub(a, b, q))
    here = up = down = torch.zeros(2, n, dtype=torch.int64, device=DEVICE)
    for high in sorted({p // r for p in positions if p >= 0}):
        c1 = c2 = s1 = s2 = torch.zeros_like(here)
        for residue, p in enumerate(positions):
            if p >= 0 and p // r == high:
                turn = _perm(_galois(ring, -residue), n)
                low = s["low"][p % r][..., turn]
                c1, c2, s1, s2 = add(c1, low[0]), add(c2, low[1]), add(s1, low[2]), add(s2, low[3])
                here = add(here, mul(s["low"][None][:, turn], s["high"][high][0]))
        c, w = s["high"][high]
        here = add(here, sub(mul(add(c1, c2), c), mul(add(s1, s2), w)))
        up = sub(up, add(mul(s1, c), mul(c1, w)))
        down = add(down, add(mul(s2, c), mul(c2, w)))
    parts = torch.stack([here, add(up, down)] if 2 * _step_of_pairs(case) == n // 2 else [here, up, down])
    m1, m2 = (_moduli(ring)[i] for i in two)
    v = _intt(parts, ring, two)
    low = torch.where(v[:, 1] > m2 // 2, v[:, 1] - m2, v[:, 1])
    w = _mul((v[:, 0] - low) % m1, _ints([pow(m2, -1, m1)]), _ints([m1]), True)
    return _plaintext(torch.where(w > m1 // 2, w - m1, w), ring, _extended(ring, level))


def _turned(x, turns, s):
    """Ciphertexts with their positions, one level below."""
    case, ring, step = s["case"], s["case"]["ring"], _step_of_pairs(s["case"])
    terms = [(g, s["keys"][g], p) for g, p in zip((_galois(ring, step), _galois(ring, -step)), turns[1:])]
    return _rescale(_moddown(_weighted(x, ring, terms, turns[0]), ring, x.shape[-2] - 1), ring)


def _page_parts(case):
    """Which residues of a run lie in the page that it begins in, and in the next one."""
    _, _, t, _, _ = _shape(case)
    begin, end = case["tokens"] % t, case["tokens"] % t + case["run"]
    return [lambda r: begin <= r < end] + ([lambda r: r + t < end] if end > t else [])


def _masked(x, mask, galois, ring):
    """Ciphertexts x[m] times the mask through their Galois maps, rescaled."""
    mask = torch.stack([mask[:, _perm(g, x.shape[-1])] for g in galois])
    return _rescale(_mul(x, mask[:, None], *_q(ring, _span(x.shape[-2] - 1))), ring)


def _append_run(s):
    case, ring = s["case"], s["case"]["ring"]
    hp, dim, t, r_i, r_o = _shape(case)
    n, b, level, page = RINGS[ring][0], hp * t, case["level"], case["tokens"] // t
    (q, _), (q1, _) = _q(ring, _span(level)), _q(ring, _span(level + 1))
    k, keys, total = s["k"], _low_keys(s["keys"], ring, level + 1), lambda terms: functools.reduce(lambda x, y: _add(x, y, q1), terms)
    parts = [[r for r in range(t) if keep(r)] for keep in _page_parts(case)]
    if case["rotary"] and case["index"]:
        k = _turned(k, s["turns"][0], s)
    for i, residues in enumerate(parts):
        if case["rotary"] and not case["index"]:
            new = _turned(k, s["turns"][i], s)
        else:
            new = _masked(k[None], total(s["masks"][0][:, _perm(_galois(ring, -r), n)] for r in residues), [1], ring)[0]
        s["K"][page + i] = _add(s["K"][page + i], new, q)
    rows = total(s["masks"][1][:, _perm(_galois(ring, -(i * b + r)), n)] for i, part in enumerate(parts) for r in part)
    shifted = _rotations(s["v"], ring, [-g * r_i * b for g in range(1, r_o)], keys)
    at = [_galois(ring, -((page - i) % dim + i // r_i * r_i) * b) for i in range(dim)]
    s["V"][:] = _add(s["V"], _masked(shifted.repeat_interleave(r_i, 0), rows, at, ring), q)
    if case["index"]:
        babies = _rotations(k, ring, [j * b for j in range(1, r_i)], keys)
        at = [_galois(ring, -((page + g * r_i) % dim) * b) for g in range(r_o) for _ in range(r_i)]
        s["X"][:] = _add(s["X"], _masked(babies.repeat(r_o, 1, 1, 1), rows, at, ring).unflatten(0, (r_o, r_i)), q)
    return {w: s[w] for w in ("K", "V", "X") if w in s}


def _product(s, x, array):
    """A pass for each of the ciphertexts x[m]: their rotations by rows times those of the cache, summed, relinearised, turned and
    rescaled; array [r_o][r_i][2][l + 1][n]."""
    case, ring, keys = s["case"], s["case"]["ring"], s["keys"]
    hp, _, t, r_i, r_o = _shape(case)
    level, b = case["level"], hp * t
    (q, wide), (qe, _) = _q(ring, _span(level)), _q(ring, _extended(ring, level))
    babies = _rotations(x, ring, [j * b for j in range(1, r_i)], keys)
    a0, a1, sums = babies[:, :, 0], babies[:, :, 1], []
    for g in range(r_o):                                     # sums of at most 128 words below 2^50
        b0, b1 = array[g, :, None, 0], array[g, :, None, 1]
        sums.append(torch.stack([v.sum(0) % q for v in (_mul(a0, b0, q, wide), _mul(a0, b1, q, wide) + _mul(a1, b0, q, wide), _mul(a1, b1, q, wide))], 1))
    sums = torch.stack(sums)                                 # [g][m][3]
    inner = _moddown(_switch(_raise(sums[:, :, 2], ring), ring, 0, keys[0], level), ring, level)
    inner = _add(inner, sums[:, :, :2], q)
    raised, acc = _times_p(inner[:, :, 0], ring), _times_p(inner[0], ring)
    for g in range(1, r_o):
        e = _galois(ring, g * r_i * b)
        acc = _add(acc, _turn_raised(raised[g], _raise(inner[g, :, 1], ring), ring, e, keys[e]), qe)
    return _rescale(_moddown(acc, ring, level), ring)


def _inner(s, x, delta, digits=None):
    """Residue r of every block moved to (r + delta) mod t, on the extended basis."""
    ring, (_, _, t, _, _) = s["case"]["ring"], _shape(s["case"])
    g = [_galois(ring, -delta), _galois(ring, t - delta)]
    return _weighted(x, ring, [(g[0], s["keys"][g[0]], s["from"][delta - 1]), (g[1], s["keys"][g[1]], s["below"][delta - 1])], digits=digits)


def _low_keys(keys, ring, level):
    """Keys as a lower level uses them."""
    if not keys or level == next(iter(keys.values())).shape[2] - RINGS[ring][5] - 1:
        return keys
    digits = -(-(level + 1) // RINGS[ring][6])
    return {g: torch.cat([k[:digits, :, : level + 1], k[:digits, :, -RINGS[ring][5]:]], 2) for g, k in keys.items()}


def _tree_qk(s):
    case, ring = s["case"], s["case"]["ring"]
    hp, dim, t, _, _ = _shape(case)
    level, n, b, q = case["level"], RINGS[ring][0], hp * t, s["q"]
    low, digits = dict(s, keys=_low_keys(s["keys"], ring, level)), _raise(q[1], ring)
    page, hidden, qs = case["base"] // t, _hidden(case), _q(ring, _span(level - 1))[0]
    last = (case["base"] + case["nodes"] - 1) // t
    x = q[None, :, : level + 1]
    if t > 1:
        moved = torch.stack([_inner(s, q, delta, digits) for delta in range(1, t)])
        x = torch.cat([x, _rescale(_moddown(moved, ring, level + 1), ring)])
    out = _product(low, x, s["X"])
    unseen = [c for c in range(dim) if not case["first"] // t <= c <= last]
    rows = functools.reduce(lambda v, m: _add(v, m, qs), (s["row"][:, _perm(_galois(ring, -c * b), n)] for c in unseen), torch.zeros_like(s["row"]))
    out[:, 0] = _add(out[:, 0], rows, qs)
    for delta in range(t):
        hide = (s["one"][:, _perm(_galois(ring, -((page + c) * b + j)), n)] for c, j in hidden[delta])
        out[delta, 0] = functools.reduce(lambda v, m: _add(v, m, qs), hide, out[delta, 0])
    return out


def _tree_sv(s):
    case, ring = s["case"], s["case"]["ring"]
    _, _, t, r_i, r_o = _shape(case)
    level, array = case["level"], s["V"].unflatten(0, (r_o, r_i))
    low, parts = dict(s, keys=_low_keys(s["keys"], ring, level - 1)), _product(s, s["scores"], array)
    out, q = parts[0, :, : level - 1], _q(ring, _extended(ring, level - 1))[0]
    if t == 1:
        return out
    moved = functools.reduce(lambda u, v: _add(u, v, q), (_inner(low, parts[delta], t - delta) for delta in range(1, t)))
    return _add(out, _rescale(_moddown(moved, ring, level - 1), ring), _q(ring, _span(level - 2))[0])


def run(s):
    case = s["case"]
    if own:
        return _own_run(s)
    if case["op"] == "rotary":
        turns = _turns(s, _positions(case))
        return list(_turned(s["x"], turns, s))
    return {"append": _append_run, "tree_qk": _tree_qk, "tree_sv": _tree_sv}[case["op"]](s)


# ---- the framework's calls --------------------------------------------------------------------------------------------
_contexts = {}


def _context(ring):
    from paper_2602_11470_amd import binding
    if ring not in _contexts:
        _contexts[ring] = binding.config1() if ring == SMALL else binding.llama_ring()
    return _contexts[ring]


@functools.lru_cache(4)
def _own_keys(ring, steps, relin):
    """The library's key set, as few of them held as of the plain form's (_keys)."""
    ctx = _context(ring)
    return ctx.keygen_rotations(ctx.keygen_secret(1), steps, 2, with_relin=relin)


@functools.lru_cache(4)
def _own_rotary(key, positions, split):
    """Tables of positions, and the positions of an append's step, which are set once for all layers."""
    case = dict(key)
    ctx = _context(case["ring"])
    rot, halves, scaling, level = _rotation(case)
    freq, gain = _frequencies(rot, scaling)
    rotary = ctx.rotary(case["heads"], case["dim"], level, case["room"], rot_dims=rot, freq=freq, gain=gain, halves=halves,
                        coeffs=_table(_key_of(case)))
    if positions:
        ctx.rotary_set(rotary, positions, split)
    return rotary


@functools.lru_cache(4)
def _own_tree(key):
    case = dict(key)
    ctx = _context(case["ring"])
    kv = ctx.kv_create(case["heads"], case["dim"], case["level"], r_i=case["r_i"], max_tokens=1, unrolled_ladders=True)
    return ctx.tree(kv, group=case["group"], mask=MASK, scale=_score_scale(case), coeffs=_tree_coefficients(_key_of(case)))


def _ct(ctx, level, words=None):
    from paper_2602_11470_amd import binding
    c = binding.Ct(ctx, level)
    c.d.scale = ctx.scale
    if words is not None:
        _words(c).copy_(words)
    return c


def _words(c):
    return c.buf[: 2 * (c.level + 1) * c.ctx.n].view(2, c.level + 1, c.ctx.n)


def _own_state(s, words):
    from paper_2602_11470_amd import binding
    case, op = s["case"], s["case"]["op"]
    level, ring = case["level"], case["ring"]
    ctx = s["ctx"] = _context(ring)
    s["keys"] = _own_keys(ring, tuple(sorted(set(_steps(case)))), op.startswith("tree"))
    rotating = op == "rotary" or bool(case.get("rotary"))
    everything = tuple(sorted(case.items()))
    if rotating:
        _, _, t, _, _ = _shape(case)
        end = case["tokens"] % t + case["run"] if op == "append" else 0
        s["rotary"] = _own_rotary(everything, tuple(_positions(case)) if op == "append" else (), max(0, end - t) if op == "append" else 0)
    if op == "rotary":
        s["positions"] = np.array(_positions(case), dtype=np.int32)
        s["in"], s["out"] = [_ct(ctx, level, w) for w in words["x"]], [_ct(ctx, level - 1) for _ in words["x"]]
        return s
    if op == "append":
        s["kv"] = ctx.kv_create(case["heads"], case["dim"], level, r_i=case["r_i"], max_tokens=case["tokens"] + case["run"], key_index=case["index"])
        for kind, c in zip((1, 2), _run_masks(_key_of(case))):
            s["kv"].set_mask(kind, c)
        which = {"K": binding.CM_QK, "V": binding.CM_SV, "X": binding.CM_KV_INDEX}
        s["cache"] = {w: s["kv"].words(which[w]) for w in which if w in words}
        for w, x in s["cache"].items():
            x.copy_(words[w])
        s["k"], s["v"] = (_ct(ctx, words[w].shape[-2] - 1, words[w]) for w in "kv")
        s["kv"].set_tokens(case["tokens"])
        return s
    total = case["base"] + case["nodes"]
    s["kv"] = ctx.kv_create(case["heads"], case["dim"], level, r_i=case["r_i"], max_tokens=total, unrolled_ladders=True, key_index=op == "tree_qk")
    s["kv"].words(binding.CM_KV_INDEX if op == "tree_qk" else binding.CM_SV).copy_(words["X" if op == "tree_qk" else "V"])
    s["kv"].set_tokens(total)
    s["tree"] = _own_tree(everything)
    s["parents"] = np.array(_parents(case["nodes"], case["tree"]), dtype=np.int32)
    if op == "tree_qk":
        t = _shape(case)[2]
        s["q"] = _ct(ctx, level + 1, words["q"])
        s["buffer"] = torch.empty(t, 2, level, ctx.n, dtype=torch.int64, device=DEVICE)
        s["out"] = [_ct(ctx, level - 1) for _ in range(t)]
        for c, buf in zip(s["out"], s["buffer"]):
            c.buf, c.d.dev = buf.view(-1), buf.data_ptr()
    else:
        s["scores"], s["out"] = [_ct(ctx, level, w) for w in words["scores"]], _ct(ctx, level - 2)
    return s


def _own_run(s):
    case, ctx = s["case"], s["ctx"]
    if case["op"] == "rotary":
        ctx.rotary_set(s["rotary"], s["positions"])
        return [_words(c) for c in ctx.rotary_apply(s["keys"], s["rotary"], s["in"], outs=s["out"])]
    if case["op"] == "append":
        s["kv"].seek(case["tokens"])
        s["kv"].append_run(s["keys"], s["k"], s["v"], case["run"], rotary=s.get("rotary"))
        return s["cache"]
    if case["op"] == "tree_qk":
        ctx.tree_qk(s["keys"], s["tree"], s["kv"], s["parents"], case["base"], s["q"], first=case["first"], outs=s["out"])
        return s["buffer"]
    return _words(ctx.tree_sv(s["keys"], s["tree"], s["kv"], s["scores"], out=s["out"]))


# ---- what a pass cannot do without --------------------------------------------------------------------------------------
def work(case):
    n, _, _, _, _, n_p, alpha, _, _ = RINGS[case["ring"]]
    hp, dim, t, r_i, r_o = _shape(case)
    limb, level, op = 8 * n, case["level"], case["op"]
    butterfly = 4 * n // 2 * (n.bit_length() - 1)             # of a transform: a product (two operations), a sum, a difference each

    def switch(at, raises, rotations, downs):
        """(operations, bytes of different keys a rotation) of key switches at a level."""
        digits, ext = -(-(at + 1) // alpha), at + 1 + n_p
        return (raises * (at + 1 + digits * ext) + downs * 2 * ext) * butterfly + rotations * 4 * digits * ext * n, digits * ext * limb

    def masked(at):
        return 2 * ((at + 1) * butterfly + 4 * (at + 1) * n)
    steps = len({_galois(case["ring"], x) for x in _steps(case)})
    turned = 2 if op == "rotary" or case.get("rotary") else 0
    if op == "rotary":
        live = [p for p in _positions(case) if p >= 0]
        r, _ = _table_sizes(case["room"])
        flops, key = switch(level, case["count"], 2 * case["count"], case["count"])
        tables = (4 * len({p % r for p in live}) + 1 + 2 * len({p // r for p in live})) * 2 * limb
        flops += 3 * (level + 3 + n_p) * butterfly + 6 * 4 * (level + 1 + n_p) * n * case["count"]
        return {"bytes": case["count"] * 2 * (2 * level + 1) * limb + steps * key + tables, "flops": flops}
    if op == "append":
        arrays, pages = 2 if case["index"] else 1, len(_page_parts(case))
        at = _rotation(case)[3] if turned else level + 1
        flops, key = switch(level + 1, 1 + arrays, steps, steps)
        # cache words are read and written, the new ciphertexts read once
        bytes_ = (pages + arrays * dim) * 2 * 2 * (level + 1) * limb + 2 * (at + 1) * limb + 2 * (level + 2) * limb + steps * key
        bytes_ += (2 + 3 * pages * bool(turned)) * (level + 2) * limb
        return {"bytes": bytes_, "flops": flops + (pages + arrays * dim) * masked(level + 1)}
    products = r_o * r_i * 4 * 2 * (level + 1) * n * t
    flops, key = switch(level, t * (1 + 2 * r_o - 1), t * (r_i + 2 * r_o - 2), t * (r_i - 1 + r_o + 1))
    inner, inner_key = switch(level + 1 if op == "tree_qk" else level - 1, 1 if op == "tree_qk" else t - 1, 2 * (t - 1), t - 1 if op == "tree_qk" else 1)
    bytes_ = r_o * r_i * 2 * (level + 1) * limb + (r_i + r_o - 1) * key + 2 * (t - 1) * inner_key
    bytes_ += (2 * (level + 2) + t * 2 * level) * limb if op == "tree_qk" else (t * 2 * (level + 1) + 2 * (level - 1)) * limb
    return {"bytes": bytes_, "flops": flops + inner + products}


# ---- from the definition, apart from the above ---------------------------------------------------------------------------
@functools.lru_cache(None)
def _powers(w, q, count, step):
    out, x = [w % q if step == 2 else 1], w * w % q if step == 2 else w % q
    for _ in range(count - 1):
        out.append(out[-1] * x % q)
    return np.array(out, dtype=object)


def _at_odd(c, w, q):
    """Values of a polynomial at w^(2 k + 1), k = 0 .. len - 1, w^len = -1, by halving, in Python's integers."""
    if len(c) == 1:
        return c
    even, odd = _at_odd(c[::2], w * w % q, q), _at_odd(c[1::2], w * w % q, q)
    turn = _powers(w, q, len(even), 2) * odd % q
    return np.concatenate([even + turn, even - turn]) % q


def _at_all(c, w, q):
    """Values at w^k, w^len = 1."""
    if len(c) == 1:
        return c
    even, odd = _at_all(c[::2], w * w % q, q), _at_all(c[1::2], w * w % q, q)
    turn = _powers(w, q, len(even), 1) * odd % q
    return np.concatenate([even + turn, even - turn]) % q


def _from_odd(v, w, q):
    """The polynomial that has these values."""
    n, inverse = len(v), pow(w, -1, q)
    return _at_all(v, inverse * inverse % q, q) * pow(n, -1, q) * _powers(inverse, q, n, 1) % q


def _exact_turns(case, positions):
    """Integer coefficients of the plaintexts of rotary positions: here, up, down (one for both where the rotations are the same)."""
    ring, (_, _, t, _, _) = case["ring"], _shape(case)
    n, (r, _), two, table = RINGS[ring][0], _table_sizes(case["room"]), _pair_modulus(ring), _table(_key_of(case))

    def moved(c, slots):                                    # X -> X^g in coefficients
        g, out = pow(5, slots % (n // 2), 2 * n), np.zeros(n, dtype=object)
        at = np.arange(n) * g % (2 * n)
        out[at % n] = np.where(at < n, c, -c)
        return out
    sums = []
    for i in two:
        q = _moduli(ring)[i]
        w = _psi(q, n)
        here = up = down = np.zeros(n, dtype=object)
        for residue, p in enumerate(positions):
            if p >= 0:
                c1, c2, s1, s2, still = (_at_odd(moved(table[row].astype(object), -residue) % q, w, q)
                                         for row in (*range(4 * (p % r), 4 * (p % r) + 4), 4 * r))
                cos, sin = (_at_odd(table[4 * r + 1 + 2 * (p // r) + k].astype(object) % q, w, q) for k in (0, 1))
                here, up, down = here + (c1 + c2 + still) * cos - (s1 + s2) * sin, up - s1 * cos - c1 * sin, down + s2 * cos + c2 * sin
        sums.append([_from_odd(v % q, w, q) for v in ([here, up + down] if 2 * _step_of_pairs(case) == n // 2 else [here, up, down])])
    (m1, m2), out = (_moduli(ring)[i] for i in two), []
    for a, b in zip(*sums):                                  # the integer below m1 m2 / 2 in size that both say, over m2, to the nearest
        value = (b + m2 * ((a - b) * pow(m2, -1, m1) % m1)) % (m1 * m2)
        value = np.where(2 * value > m1 * m2, value - m1 * m2, value)
        out.append((2 * value + m2) // (2 * m2))
    return out


def exact(case, seed):
    """The turned ciphertexts of the small ring from Python's integers; the outputs of every other case are too many for that.  All
    outputs are whole words, which are compared for equality."""
    if case["op"] != "rotary" or case["ring"] != SMALL or sum(p >= 0 for p in _positions(case)) > 40:
        return None
    ring, level, brev = SMALL, case["level"], _places(RINGS[SMALL][0]).cpu().numpy()
    n, mods, nq = RINGS[ring][0], _moduli(ring), RINGS[ring][4]
    words = _residues(ring, (case["count"], 2), level + 1, torch.Generator(device=DEVICE).manual_seed(int(seed))).cpu().numpy().astype(object)
    ext, p, step, out = [*range(level + 1), nq], mods[nq], _step_of_pairs(case), []
    root = {i: _psi(mods[i], n) for i in ext}
    plain = [[_at_odd(c % mods[i], root[i], mods[i]) for i in ext] for c in _exact_turns(case, _positions(case))]
    galois = [pow(5, x % (n // 2), 2 * n) for x in (step, -step)][: len(plain) - 1]
    keys = [_key(ring, g, level).cpu().numpy().astype(object)[..., brev] for g in galois]
    for x in words[..., brev]:                               # place k: the value at the 2 k + 1-th power
        digits = [_from_odd(x[1, j], root[j], mods[j]) for j in range(level + 1)]
        digits = [[_at_odd(d % mods[i], root[i], mods[i]) for i in ext] for d in digits]
        u = [[plain[0][e] * x[c, e] * p % mods[i] if e <= level else 0 * plain[0][e] for e, i in enumerate(ext)] for c in (0, 1)]
        for g, key, w in zip(galois, keys, plain[1:]):
            at = ((2 * np.arange(n) + 1) * g % (2 * n) - 1) // 2
            for c in (0, 1):
                for e, i in enumerate(ext):
                    one = sum(digits[j][e][at] * key[j][c][e] for j in range(level + 1)) + (x[0, e][at] * p if c == 0 and e <= level else 0)
                    u[c][e] = (u[c][e] + one * w[e]) % mods[i]
        y = np.empty((2, level, n), dtype=object)
        for c in (0, 1):
            special = _from_odd(u[c][-1], root[nq], p)
            down = [(u[c][e] - _at_odd(special % mods[e], root[e], mods[e])) * pow(p, -1, mods[e]) % mods[e] for e in range(level + 1)]
            last = _from_odd(down[level], root[level], mods[level])
            for e in range(level):
                y[c, e] = (down[e] - _at_odd(last % mods[e], root[e], mods[e])) * pow(mods[level], -1, mods[e]) % mods[e]
        out.append(torch.from_numpy(y[..., brev].astype(np.int64)))
    return out
