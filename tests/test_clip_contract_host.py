"""What the header promises about opening the gradients' squared norm, and that it is so, on the oracle.  No GPU is used."""
import os

import numpy as np

from oracle import ring_oracle as ro
from paper_2104_10949_amd import workloads as wl

MOD = 1 << 64
KEYS = [bytes([17 * k + 3] * 16) for k in range(3)]


def header():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    return " ".join(open(os.path.join(root, "include", "cg.h")).read().replace(" * ", " ").split())


def test_an_unblinded_share_of_the_norm_tells_the_missing_word():
    """P_2 holds s_2 and s_0.  z_0 = s_0 (s_0 + 2 s_1) of one element, sent as it is, gives it s_1 but for the top bit; with the zero
    share it does not, and the norm is the same."""
    s = [int(v) | 1 for v in wl.draw_ring((3,), 700)]
    z = [ro.sq_norm([(np.array([s[i]], np.uint64), np.array([s[(i + 1) % 3]], np.uint64))]) for i in range(3)]

    def told(z0):
        return (z0 - s[0] * s[0]) * pow(s[0], -1, MOD) % MOD // 2
    assert told(z[0]) == s[1] % (1 << 63)
    blind = [int(ro.reshare(np.array([v], np.uint64), KEYS[i], KEYS[(i - 1) % 3], 9, 0)[0]) for i, v in enumerate(z)]
    assert told(blind[0]) != s[1] % (1 << 63) and all(a != b for a, b in zip(z, blind))
    assert sum(blind) % MOD == sum(z) % MOD == sum(s) ** 2 % MOD


def test_the_header_says_that_shares_are_blinded_before_they_are_sent():
    text = header()
    assert "blinds it with a zero share (cg_reshare) before it sends it" in text
    assert "s0, s1, s2: the three parties' blinded words" in text
