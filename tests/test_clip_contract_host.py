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


def norm_of(x):
    """The opened sum of squares of plain words, by way of three parties' shares."""
    s = ro.share(x, wl.draw_ring(x.shape, 710), wl.draw_ring(x.shape, 711))
    return sum(ro.sq_norm([(s[i], s[(i + 1) % 3])]) for i in range(3)) % MOD


def test_the_norm_is_right_below_2_to_the_32_and_wraps_from_there():
    """At 16 fractional bits: a norm of 65536 - 2^-16 is clipped, one of 65536 is taken for zero; no bound of 2^32 or more clips."""
    largest = np.array([(1 << 32) - 1], np.uint64)
    assert norm_of(largest) == ((1 << 32) - 1) ** 2
    assert ro.clip_factor(norm_of(largest), 1 << 16, 16) == 1
    beyond = np.array([1 << 32], np.uint64)
    assert norm_of(beyond) == 0 and ro.clip_factor(norm_of(beyond), 1 << 16, 16) == 1 << 16
    several = np.array([1 << 31] * 4 + [-(1 << 31) % MOD] * 3 + [3], np.uint64)      # 7/4 of 2^64, and 9
    assert norm_of(several) == (7 * (1 << 62) + 9) % MOD
    assert ro.clip_factor(MOD - 1, 1 << 32, 16) == 1 << 16


def test_the_header_states_the_range():
    text = header()
    assert "S is the squared norm only while that is below 2^64, that is, N below 2^32: a real norm below 2^(32-f) at f fractional bits" in text
    assert "A max_norm of 2^32 or more is never exceeded" in text
    assert "which it is only while that sum is below 2^64" in text
