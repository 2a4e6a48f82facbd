"""How a pick of blocks cuts a range of scores, step by step in whole numbers as the kernels do, at the ends of that range."""
import random
import struct

import pytest

from paper_2505_23219_amd import binding as B

INF = 0xff800000                # the key of a block that holds an infinity or NaN
RANKED = 64                     # keys that a wavefront ranks


def _key(score):
    """The order of scores as that of unsigned numbers."""
    b = struct.unpack("I", struct.pack("f", score + 0.0))[0]
    return b ^ (0xffffffff if b >> 31 else 0x80000000)


def _pick(keys, need):
    """The places of the `need` best, the lowest first on ties."""
    lib = B.lib()
    end = lambda *a: lib.ghd_debug_pick_step_end(*a) & 0xffffffff
    low, high, taken = min(keys), max(keys), []
    shift = lib.ghd_debug_pick_shift(low, high)
    while True:
        steps = [0] * 256
        for k in keys:
            if low <= k <= high:
                steps[k - low >> shift] += 1
        step, above = 255, 0
        while above + steps[step] < need:
            above += steps[step]
            step -= 1
        first = low + (step << shift)
        last = end(first, high, shift)
        assert first <= last <= high and first < 1 << 32
        taken += [b for b, k in enumerate(keys) if last < k <= high]
        low, high, need, inside = first, last, need - above, steps[step]
        assert inside == sum(low <= k <= high for k in keys) >= need
        if inside == need or inside <= RANKED or shift == 0:
            break
        shift = max(0, shift - 8)
    rest = sorted((b for b, k in enumerate(keys) if low <= k <= high), key=lambda b: (-keys[b], b))
    return sorted(taken + rest[:need])


def _check(keys, need):
    want = sorted(sorted(range(len(keys)), key=lambda b: (-keys[b], b))[:need])
    assert _pick(keys, need) == want


@pytest.mark.parametrize("scores", [[-20.0, -0.5, 3.0, None, 7.0, 2.0], [-1.5, 2.0, None, 3.0, 1.0, 0.5], [-1.5, None, None, 3.0, None],
                                    [-3.0, None, -4.0, -5.0], [-2.0, None], [0.0, None, None], [-0.0, 0.0, None]])
def test_a_few_blocks(scores):
    keys = [INF if s is None else _key(s) for s in scores]
    for need in range(1, len(keys) + 1):
        _check(keys, need)


@pytest.mark.parametrize("exponent", range(-30, 31, 3))
def test_lowest_scores_of_any_size(exponent):
    r = random.Random(exponent)
    for parity in (0, 1):
        for infinite in (0, 1, 3, 70):
            low = [-2.0 ** (exponent + parity) * r.uniform(1, 2) for _ in range(1)]
            keys = [_key(x) for x in low + [2.0 ** exponent * r.uniform(-0.9, 3) for _ in range(120)]] + [INF] * infinite
            r.shuffle(keys)
            for need in {1, 2, max(infinite, 1), infinite + 1, infinite + 70, len(keys)}:
                _check(keys, need)


def test_the_ends_of_the_range():
    """Keys of the lowest and highest finite score, of minus infinity, of infinity; ranges of every width."""
    ends = [0x007fffff, _key(-3.4028234e38), _key(-1e-45), _key(0.0), _key(1e-45), _key(3.4028234e38), INF]
    r = random.Random(1)
    for low in ends:
        for high in ends:
            if low > high:
                continue
            keys = [low, high] + [r.randint(low, high) for _ in range(200)] + [high] * r.choice((0, 90))
            for need in (1, 2, 90, 91, 150, len(keys)):
                _check(keys, min(need, len(keys)))
    for bits in range(33):
        low = (1 << 32) - (1 << bits) if bits < 32 else 0
        keys = [low, 0xffffffff] + [r.randint(low, 0xffffffff) for _ in range(150)]
        for need in (1, 3, 100):
            _check(keys, need)
