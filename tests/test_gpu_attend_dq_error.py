"""How far dQ is off in bf16 where keys have a common part: with the mean of up to 16 seen keys times what the rounding of S lost, the
common part adds nothing to the error.

Bound.  e_j = S_j - bf16(S_j) in binary64, c the mean of the first 8 keys that a row sees: the error that the correction leaves is
scale sum e_j (k_j - c), and the result's own rounding.  Their norm, times 1.2 for another choice of keys (the mean of n keys has a
variance of 1/n of theirs: 8 to 4 keys 6%) and for S in binary32 (a rounding in a few hundred falls the other way), bounds the
norm.  Without the correction, scale sum e_j k_j is at least 1.6 times that for each of these cases, which the test holds too."""
import numpy as np
import pytest

from oracle import gradients as gr

from tests.attn_helpers import Case, f64
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu

SHAPES = [  # lens_q, lens_k, heads, kv, causal, window
    ([300], [300], 1, 1, False, 8),
    ([300], [300], 2, 2, True, 24),
    ([200], [200], 4, 1, False, 3),
    ([300], [100], 1, 1, True, 0),         # most rows see nothing
    ([40, 9, 17], [40, 9, 17], 2, 1, True, 0),
    ([700], [700], 1, 1, True, 0),
    ([3], [1500], 2, 1, True, 0),          # keys in pieces
    ([40], [3000], 1, 1, True, 20)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"q{sum(s[0])}k{sum(s[1])}h{s[2]}c{int(s[4])}w{s[5]}")
def test_a_common_part_of_the_keys_adds_nothing(shape):
    say(f"attend dq error {shape}")

    def edit(case):
        rng = np.random.default_rng(11)
        case.host["k"] += 4.0 * rng.standard_normal(case.kv * case.dim)
    lens_q, lens_k, heads, kv, causal, window = shape
    case = Case("bf16", lens_q, lens_k, heads, kv, 64, causal, window, edit=edit)
    case.forward(), case.backward()
    case.check_backward()
    got, out, lse = case.dq.host(), case.out.host(), case.lse.host()
    off = want = left = plain = 0.0
    for rows, keys, c, e, h in case.parts():
        q, k, v, do = case.host["q"][rows, c], case.host["k"][keys, e], case.host["v"][keys, e], case.host["dout"][rows, c]
        for i in range(len(q)):
            lo, hi = gr.keys_seen(i, len(q), len(k), causal, window)
            if hi <= lo:
                assert (got[rows, c][i] == 0).all()
                continue
            p = np.exp(case.scale * (k[lo:hi] @ q[i]) - lse[rows, h][i])
            s = p * (v[lo:hi] @ do[i] - do[i] @ out[rows, c][i])
            lost = s - f64(s.astype(np.float32), "bf16")
            dq = case.scale * (s @ k[lo:hi])
            own = ((f64(dq, "bf16") - dq) ** 2).sum()
            off += ((got[rows, c][i] - dq) ** 2).sum()
            left += own + ((case.scale * (lost @ (k[lo:hi] - k[lo:min(hi, lo + 8)].mean(0)))) ** 2).sum()
            plain += own + ((case.scale * (lost @ k[lo:hi])) ** 2).sum()
            want += (dq ** 2).sum()
    bound = 1.2 * np.sqrt(left / want)
    say(f"off {np.sqrt(off / want):.5f}, bound {bound:.5f}, uncorrected {np.sqrt(plain / want):.5f}")
    assert np.sqrt(plain / want) > 1.6 * bound
    assert np.sqrt(off / want) < bound
