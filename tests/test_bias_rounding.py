"""The table's gradient in 16 bits: sums in fp64, rounded once.  A bucket has two distances with one fp32 value each, whose sum is
exact in fp64; what it rounds to is computed in whole numbers."""
import math
from fractions import Fraction

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

# bits of the mantissa, least exponent (of a mantissa in [1, 2)), largest value
KINDS = {"bfloat16": (8, -126, (2 - 2.0 ** -7) * 2.0 ** 127), "float16": (11, -14, 65504.0)}


def _rounded(x, kind):
    """x (a Fraction) to the nearest value, ties to even."""
    bits, least, most = KINDS[kind]
    if x == 0:
        return 0.0
    e = max(math.frexp(float(abs(x)))[1] - 1, least)
    unit = Fraction(2) ** (e - bits + 1)
    y = round(x / unit) * unit                                 # Python's round: halves to even
    return math.copysign(math.inf, x) if abs(y) > most else float(y)


def _sums(kind):
    rng = np.random.default_rng(1)
    bits = KINDS[kind][0]
    half, pairs = 2.0 ** -bits, []
    for sign in (1.0, -1.0):
        for odd in (1, 3, 5, 255):                             # halfway between two values, and a little beside it
            for little in (0.0, 2.0 ** -25, 2.0 ** -30, 2.0 ** -40, 2.0 ** -44):
                for way in (1.0, -1.0):
                    pairs.append((sign * (1 + odd * half), way * little))
    for big in (65504.0, 65519.0, 65520.0, 3.3895e38, 3.4e38):
        pairs += [(big, 2.0 ** -12 * big), (big, -(2.0 ** -24) * big), (-big, 2.0 ** -12 * big), (big, 2.0 ** -24 * big)]
    for small in (2.0 ** -24, 2.0 ** -25, 3 * 2.0 ** -25, 2.0 ** -14, 5 * 2.0 ** -26, 2.0 ** -126, 2.0 ** -133):
        pairs += [(small, 0.0), (small, small * 2.0 ** -13), (small, -small * 2.0 ** -13), (-small, small * 2.0 ** -13)]
    for _ in range(800):
        a = float(np.float32(rng.standard_normal()))
        few = float(np.float16(rng.standard_normal()))         # eleven bits: the sum has at most 53
        pairs.append((a, math.ldexp(few, math.frexp(a)[1] - int(rng.integers(0, 20)))))
    return np.array(pairs, dtype=np.float32)


@pytest.mark.parametrize("kind", list(KINDS))
def test_rounded_once(kind):
    import torch
    import paper_2206_10581_amd as tt
    pairs = _sums(kind)
    n = len(pairs)
    exact = [Fraction(float(a)) + Fraction(float(b)) for a, b in pairs]
    assert all(Fraction(float(x)) == x for x in exact)        # in fp64
    of = torch.zeros(4 * n + 1, dtype=torch.int32)
    of[2 * n:4 * n] = torch.arange(2 * n) // 2
    of[4 * n] = of[4 * n - 1]
    grad = torch.from_numpy(pairs.reshape(1, 1, 1, 2 * n)).cuda()
    bias = tt.PositionBias(torch.zeros((n, 1), dtype=getattr(torch, kind), device="cuda"), of.cuda(), fill=0.0)
    want = [_rounded(x, kind) for x in exact]
    got = bias.backward(grad).flatten().double().tolist()
    assert [(x, y, z) for x, y, z in zip(pairs.tolist(), got, want) if y != z] == []
    # added to a value: 1 + what lies halfway, or a little beside it
    room = torch.ones((n, 1), dtype=getattr(torch, kind), device="cuda")
    got = bias.backward(grad, out=room, add=True).flatten().double().tolist()
    total = [x + 1 for x in exact]
    want = [_rounded(x, kind) if Fraction(float(x)) == x else y for x, y in zip(total, got)]   # where fp64 holds the sum
    assert sum(Fraction(float(x)) == x for x in total) > n // 2
    assert [(x, y, z) for x, y, z in zip(pairs.tolist(), got, want) if y != z] == []


def test_what_is_no_number():
    import torch
    import paper_2206_10581_amd as tt
    for kind in KINDS:
        grad = torch.tensor([math.nan, math.inf, -math.inf, 3.0], device="cuda").view(1, 1, 1, 4)
        of = torch.tensor([0, 0, 0, 0, 0, 1, 2, 3, 3], dtype=torch.int32, device="cuda")
        bias = tt.PositionBias(torch.zeros((4, 1), dtype=getattr(torch, kind), device="cuda"), of)
        got = bias.backward(grad).flatten().tolist()
        assert math.isnan(got[0]) and got[1:] == [math.inf, -math.inf, 3.0]
