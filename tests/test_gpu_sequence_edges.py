"""GPU: recurrences and group normalisation at the edges of what their layouts, plans and part sizes allow."""
import numpy as np
import pytest

import sequence_plain as plain
from test_gpu_sequence import BITS, limit, refused

pytestmark = pytest.mark.gpu
ARG = -1


# --- shared gates and part-filled ciphertexts ---

@pytest.mark.parametrize("c_inner,gates,channels", [(4, 3, 6), (3, 2, 4), (3, 5, 10), (4, 7, 14)])
def test_shared_gates_have_to_fill_their_ciphertexts(c_inner, gates, channels):
    """Ciphertexts and channels divide alike, but slot group c_inner - 1 of the last gate ciphertext holds no gate."""
    from paper_1810_00845_amd import hisa
    g = hisa.Context(12, [50] + [BITS] * 5, 2, 50, 5)
    g.keygen()
    layout = dict(c_inner=c_inner, c_stride=16)
    a, x = (g.tensor_encrypt(np.zeros((1, n, 1, 3)), 2.0 ** BITS, 6, **layout) for n in (gates, channels))
    g.gen_rot_mul_keys(g.recurrence_rot_steps(x) + g.recurrence_rot_steps(x, False, True))
    refused(ARG, g.recurrence, a, x)
    refused(ARG, g.recurrence_step, a, x, x)
    refused(ARG, g.recurrence_grad, a, x, x)
    g.close()


@pytest.mark.parametrize("c_inner,gates,channels", [(4, 3, 3), (4, 6, 6), (3, 3, 9)])
def test_part_filled_and_shared_values(c_inner, gates, channels):
    """As many gates as channels in a part-filled last ciphertext, and full ciphertexts of gates shared by three."""
    from paper_1810_00845_amd import hisa
    rng = np.random.default_rng(channels)
    shape = (2, channels, 2, 5)
    x, gr, st = (rng.uniform(-1, 1, shape) for _ in range(3))
    a = rng.uniform(0.2, 0.9, (2, gates, 2, 5))
    g = hisa.Context(13, [50] + [BITS] * 8, 3, 50, 7)
    g.keygen()
    ta, tx, tg, ts = (g.tensor_encrypt(v, 2.0 ** BITS, 9, c_inner=c_inner, c_stride=32) for v in (a, x, gr, st))
    g.gen_rot_mul_keys(g.recurrence_rot_steps(tx) + g.recurrence_rot_steps(tx, False, True))
    one = g.tensor_decrypt(g.recurrence_step(ta, ts, tx))
    assert np.abs(one - (x + plain.shared_gates(a, channels, c_inner) * st)).max() <= limit(13, g.K, 2, 2.0)
    ta = g.recurrence_gates(ta)
    want = plain.recurrence(a, x, False, c_inner)
    # an error in a gate or a token counts up to 1 / (1 - 0.9) times, a state is at most ten; three levels and the mask's
    tol = limit(13, g.K, 4, 100.0)
    h = g.recurrence(ta, tx)
    assert np.abs(g.tensor_decrypt(h) - want).max() <= tol
    dx, dg = g.recurrence_grad(ta, h, tg)
    wx, wa = plain.recurrence_grad(a, want, gr, False, c_inner)
    assert np.abs(g.tensor_decrypt(dx) - wx).max() <= tol
    # products of states and gradients below ten each, summed over the sharers
    assert np.abs(g.tensor_decrypt(g.recurrence_gates(dg)) - wa).max() <= tol * 20 * (channels // gates)
    g.close()
