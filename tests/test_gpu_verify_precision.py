"""The token behind a rejected draft is decided by the weights' sums in 64 bits: two weights that make the threshold lie between their neighbours, closer than 32-bit
remainders of the differences could tell."""
import math

import numpy as np
import pytest
import torch

from paper_2609_07306_b200.verify import verify_drafts


def lane(rng):
    """Eight pairs p > q of about one size, q below the last bit of p: a difference takes some 50 bits, which 64-bit numbers hold."""
    p = rng.uniform(0.06, 0.12, 8).astype(np.float32)
    return p, (p * rng.uniform(0.2, 0.9, 8) * 2.0 ** -24).astype(np.float32)


def pair_for(value):
    """(x, y) with x - y next to value: 48 bits."""
    x = np.float32(value)
    if float(x) < value:
        x = np.nextafter(x, np.float32(4.0))
    return x, np.float32(float(x) - value)


def cases():
    """(p, q, the token): one lane's eight weights, sum s, against a weight w behind them, with the threshold at half of all: the last of the eight where s > w, else
    the one behind.  w / s is off 1 by more than 1.2e-15.  In 64 bits the differences are exact, a sum of eight is off by at most 5 roundings on its longest way (three of
    four terms, two joins), the total and its half by one more: 6 x 2^-53 = 6.7e-16."""
    rng, out = np.random.default_rng(1), []
    for i in range(400):
        p, q = lane(rng)
        s = math.fsum(float(a) - float(b) for a, b in zip(p, q))
        x, y = pair_for(s * (1 + (-2e-15 if i % 2 else 2e-15)))
        w = float(x) - float(y)
        if not 1.2e-15 < abs(w / s - 1) < 2.5e-15:
            continue
        P, Q = np.zeros(300, np.float32), np.zeros(300, np.float32)
        P[5:256:32], Q[5:256:32] = p, q                    # the entries of one lane of a block
        P[290], Q[290] = x, y                              # and one of the next block
        out.append((P, Q, 290 if w > s else 229))
    return out


def test_the_pairs():
    assert len(cases()) > 100
    for P, Q, token in cases():
        w = [float(a) - float(b) for a, b in zip(P, Q)]
        upto = math.fsum(w[:256])
        assert (upto > 0.5 * math.fsum(w)) == (token == 229) and w[290] > 0 and w[229] > 0


@pytest.mark.gpu
def test_thresholds_between_neighbours():
    data = cases()
    n = len(data)
    target, draft = np.zeros((2 * n, 300), np.float32), np.zeros((2 * n, 300), np.float32)
    for i, (P, Q, _) in enumerate(data):
        target[2 * i], draft[2 * i] = P, Q
    u = torch.full((2 * n,), 0.5, device="cuda")
    u[::2] = 1.0                                           # the draft, which the target has nothing for, is rejected
    tokens = torch.zeros(2 * n, dtype=torch.int32, device="cuda")
    cu = torch.arange(0, 2 * n + 1, 2, device="cuda").int()
    got, accepted = verify_drafts(torch.from_numpy(target).cuda(), tokens, cu, draft=torch.from_numpy(draft).cuda(), uniform=u)
    assert (accepted == 0).all() and got[::2].tolist() == [t for _, _, t in data]
