"""The closed form of treekv_tree_verify's refusals, P_k = max(P - c_k Q, 0) / W_k with c_1 = 1 and c_k+1 = c_k + W_k, in double
against the rule carried out step by step in exact arithmetic: what is left is good to the rounding of c_k Q over what is left."""
import random
from fractions import Fraction

import pytest


def exact(P, Q, refusals):
    """P after each refusal: max(P - Q, 0) over its sum, P where that is 0.  And the part of the first P that is left."""
    P, Q, left, got = [Fraction(x) for x in P], [Fraction(x) for x in Q], Fraction(1), []
    for _ in range(refusals):
        R = [max(p - q, Fraction(0)) for p, q in zip(P, Q)]
        W = sum(R)
        if W > 0:
            P, left = [r / W for r in R], left * W
        got.append((P, left))
    return got


def closed(P, Q, refusals):
    """(max(P - c Q, 0), W, c) after each, as the kernel has them."""
    c, W, asked, got = 0.0, 1.0, None, []
    R = list(P)
    for _ in range(refusals):
        asked = c + W
        new = [max(p - asked * q, 0.0) for p, q in zip(P, Q)]
        if sum(new) > 0.0:
            c, W, R = asked, sum(new), new
        got.append((R, W, c))
    return got


def fp32(x):
    import struct

    return struct.unpack("f", struct.pack("f", x))[0]


@pytest.mark.parametrize("seed", range(40))
def test_refusals_in_double(seed):
    rng = random.Random(seed)
    V = rng.choice([2, 3, 8, 40])
    P, Q = ([fp32(rng.random() ** rng.choice([1, 4])) for _ in range(V)] for _ in "pq")
    # (the kernel takes rows as they are; sums of one are what makes W a part)
    P, Q = ([fp32(x / sum(y)) for x in y] for y in (P, Q))
    steps = 0
    for k, ((want, left), (R, W, c)) in enumerate(zip(exact(P, Q, 60), closed(P, Q, 60)), 1):
        # c_k+1 = c_k + W(c_k), and W falls where c rises, so an error of c does not grow; a step adds the roundings of c, of the products
        # and differences (c Q and 1 in sum) and of the sum (V terms).  Over W, twice, for W's own
        room = 2 * (k + 2) * (2 * c + 2 + V) * 2.0 ** -53 / float(left)
        if room > 2.0 ** -8:
            break                                    # no longer defined by the rule, in double
        steps = k
        assert abs(W - float(left)) <= room * float(left)
        for r, w in zip(R, want):
            assert abs(r / W - float(w)) <= room, (k, r / W, float(w), room)
    assert steps >= 4


def test_refusals_until_nothing_is_left():
    """Each refusal halves what is left: after 52 of them that is the rounding of c Q, and at last 0, where P stays as it was: the
    token that the rule leaves keeps all of it."""
    P, Q = [fp32(0.9), fp32(0.1)], [0.5, 0.5]
    for R, W, c in closed(P, Q, 200)[1:]:
        assert R[1] == 0.0 and R[0] == W > 0.0
