"""GPU: recurrences and group normalisation at the edges of what their layouts, plans and part sizes allow."""
from dataclasses import replace

import numpy as np
import pytest

import sequence_plain as plain
from test_gpu_sequence import BITS, limit, pair, random_tensors, refused, same

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


# --- a group that ends in a part-filled ciphertext ---

def test_one_group_in_a_part_filled_ciphertext_bits():
    from oracle import sequence as seq
    from paper_1810_00845_amd import synth
    g, o = pair(12, 7, 3)
    gt, ot = random_tensors(g, o, 4, 7, 2.0 ** BITS, 3, batch=2, channels=7, height=2, width=3, c_inner=4, c_stride=16)
    steps = g.group_norm_rot_steps(gt)
    g.gen_rot_keys(steps); o.gen_rot_keys(steps)
    gamma, beta = (np.stack([synth.plaintext_coeffs(k + i, g.N, bits) for i in range(2)]) for k, bits in ((7, 30), (70, 40)))
    args = (1, 1e-3, 0.05, 2.0, 1)
    plan = g.group_norm_prepare_fixed(gt, gamma, 2.0 ** 35, beta, *args, act_ratio=0.5)
    same(g, o, g.group_norm_apply(gt, plan), seq.group_norm_fixed(o, ot, gamma, 2.0 ** 35, beta, *args, 0.5))
    g.group_norm_plan_free(plan)
    g.close()


@pytest.mark.parametrize("shape,layout", [((2, 5, 3, 4), dict(c_inner=4, c_stride=1, w_stride=4)), ((1, 3, 3, 3), dict(c_inner=8, c_stride=16))])
def test_one_group_in_a_part_filled_ciphertext_values(shape, layout):
    from paper_1810_00845_amd import hisa
    rng = np.random.default_rng(shape[1])
    x = rng.normal(0.3, 0.8, shape)
    gamma, beta = rng.uniform(0.5, 1.5, shape[1]), rng.uniform(-1, 1, shape[1])
    var = x.reshape(shape[0], -1).var(-1)
    lo, hi = var.min() / 2, var.max() * 2
    g = hisa.Context(13, [50] + [BITS] * 12, 3, 50, 7)
    g.keygen()
    t = g.tensor_encrypt(x, 2.0 ** BITS, 13, **layout)
    g.gen_rot_keys(g.group_norm_rot_steps(t))
    # as test_group_norm_values: the cubics' error, and noise at 1 / 64 of the scale over twelve divisions
    tol = np.abs(x).max() / np.sqrt(lo) * 1.5 * plain.cubic_error(lo, hi, 4) + limit(13, g.K, 64 * 12, np.abs(x).max() / np.sqrt(lo) * 1.5 / lo)
    for ga, be in ((gamma, beta), (None, None)):
        plan = g.group_norm_prepare(t, ga, be, 1, 1e-3, lo, hi, 4)
        y = g.group_norm_apply(t, plan)
        want = plain.group_norm(x, *((np.ones(shape[1]), np.zeros(shape[1])) if ga is None else (ga, be)), 1, 1e-3)
        assert y.clean and np.abs(g.tensor_decrypt(y) - want).max() <= tol
        # the slots of the missing channels hold zeros
        assert np.abs(g.tensor_decrypt(y.shaped_like(channels=len(y.cts) // shape[0] * layout["c_inner"]))[:, shape[1]:]).max() <= tol
        g.group_norm_plan_free(plan)
    g.close()


# --- plans and layouts ---

@pytest.mark.parametrize("shape,other", [((1, 2, 3, 4), dict(c_stride=7)), ((1, 2, 1, 4), dict(h_stride=9)), ((1, 2, 3, 1), dict(w_stride=5)),
                                         ((1, 2, 1, 1), dict(h_stride=9, w_stride=5, c_stride=3))])
def test_a_plan_does_not_ask_for_strides_of_single_elements(shape, other):
    """Strides of an extent of one place nothing: the same slots, the same plan, the same bits."""
    from paper_1810_00845_amd import hisa
    g = hisa.Context(12, [50] + [BITS] * 6, 2, 50, 5)
    g.keygen()
    t = g.tensor_encrypt(np.random.default_rng(1).normal(size=shape), 2.0 ** BITS, 7)
    g.gen_rot_keys(g.group_norm_rot_steps(t) or [0])
    plan = g.group_norm_prepare(t, None, None, 1, 1e-3, 0.1, 4.0, 1)
    want = g.group_norm_apply(t, plan)
    moved = t.shaped_like(**other)
    assert g.group_norm_rot_steps(moved) == g.group_norm_rot_steps(t)
    for a, b in zip(want.cts, g.group_norm_apply(moved, plan).cts):
        assert np.array_equal(g.ct_export(a), g.ct_export(b))
    for wrong in (dict(offset=1), dict(height=shape[2] + 1), dict(width=shape[3] + 1)):
        refused(ARG, g.group_norm_apply, t.shaped_like(**wrong), plan)
    if shape[2] > 1 and shape[3] > 1:
        refused(ARG, g.group_norm_apply, t.shaped_like(h_stride=t.h_stride + 1), plan)
        refused(ARG, g.group_norm_apply, t.shaped_like(w_stride=2, h_stride=8), plan)
    g.group_norm_plan_free(plan)
    g.close()


def test_more_elements_than_slots_are_refused():
    from paper_1810_00845_amd import hisa
    g = hisa.Context(12, [50] + [BITS] * 6, 2, 50, 5)
    t = g.tensor_encrypt(np.zeros((1, 2, 2, 3)), 2.0 ** BITS, 7)
    g.keygen()
    g.gen_rot_mul_keys(g.recurrence_rot_steps(t) + g.recurrence_rot_steps(t, False, True))
    norm = (None, None, 1, 1e-3, 0.1, 4.0, 1)
    plan = g.group_norm_prepare(t, *norm)
    for many in (dict(h_stride=0, height=683), dict(h_stride=0, height=0xffffffff), dict(w_stride=0, h_stride=0, height=0xffffffff, width=0xffffffff),
                 dict(w_stride=0, width=1025), dict(c_inner=0x80000000, c_stride=1, channels=0xffffffff)):
        bad = t.shaped_like(**many)
        refused(ARG, g.recurrence, bad, bad)
        refused(ARG, g.recurrence_step, bad, bad, bad)
        refused(ARG, g.recurrence_grad, bad, bad, bad)
        refused(ARG, g.recurrence_gates, bad)
        refused(ARG, g.group_norm_prepare_fixed, t.shaped_like(h_stride=0, height=683), np.zeros((2, g.N)), 2.0 ** 30, np.zeros((2, g.N)), *norm[2:])
        refused(ARG, g.group_norm_apply, bad, plan)
        if "channels" not in many:
            refused(ARG, g.group_norm_prepare, bad, *norm)
    crowd = t.shaped_like(cts=t.cts[:1] * 16385, channels=16385)
    refused(ARG, g.recurrence, crowd, crowd)
    refused(ARG, g.recurrence_step, crowd, crowd, crowd)
    refused(ARG, g.recurrence_grad, crowd, crowd, crowd)
    refused(ARG, g.group_norm_prepare, crowd, *norm)
    full = t.shaped_like(h_stride=3, height=682)       # 2046 of 2048 slots
    assert g.recurrence_gates(full).cts[0].limbs == 6
    g.group_norm_plan_free(plan)
    g.close()


# --- work in parts ---

def launches(g, f):
    """What f returned, and how often each kernel ran."""
    g.profile_enable(True)
    out = f()
    counts = {k: n for k, (n, _ms) in g.profile_read().items()}
    g.profile_enable(False)
    return out, counts


def row(g, cts, width):
    from paper_1810_00845_amd import hisa
    return hisa.CipherTensor(g, cts, 1, len(cts), 1, width, width, 1, 0, 1)


def test_gates_of_a_gradient_are_moved_in_parts():
    """130 gates, each with three digits of 22 limbs at N = 2^15: 17 MB, so 62 to a part of 1 GB."""
    from paper_1810_00845_amd import hisa
    g = hisa.Context(15, [50] + [BITS] * 15, 3, 50, 5)
    n = 130
    a, h, gr = (row(g, g.ct_random_batch(n, 16, 2.0 ** BITS, k), 2) for k in (1000, 2000, 3000))
    g.gen_rot_mul_keys(g.recurrence_rot_steps(a, False, True))
    (dx, dg), counts = launches(g, lambda: g.recurrence_grad(a, h, gr))
    # the rows behind the columns of one polynomial's key switch: of the rotation alone
    assert counts["ntt_fp_kernel<5, 6, false>"] == 3, counts
    for i in (0, 43, 44, 86, 87, n - 1):      # around the parts' ends
        few = g.recurrence_grad(*(row(g, t.cts[i:i + 1], 2) for t in (a, h, gr)))
        for t, whole in zip(few, (dx, dg)):
            assert np.array_equal(g.ct_export(t.cts[0]), g.ct_export(whole.cts[i]))
    g.close()


PARTS = (15, [50] + [BITS] * 15, 3, 50, 5)      # an entry of a key switch at 16 limbs is 17 MB of digits, of a rotated product 35: 62 and 31 to a part


def equal(g, one, many):
    assert len(one) == len(many)
    for a, b in zip(one, many):
        assert np.array_equal(g.ct_export(a), g.ct_export(b))


def test_scan_and_gradient_in_parts():
    """141 ciphertexts, three to a gate: parts that begin inside a shared gate, hold the last tokens and the first gates, or gates alone; sums of
    three products in parts.  Against every gate and its sharers alone, where a call is one part."""
    from paper_1810_00845_amd import hisa
    g = hisa.Context(*PARTS)
    shared, n = 3, 141
    a, x, h = (row(g, g.ct_random_batch(k, 16, 2.0 ** BITS, c), 3) for k, c in ((n // shared, 1000), (n, 2000), (n, 4000)))
    g.gen_rot_mul_keys(g.recurrence_rot_steps(x) + g.recurrence_rot_steps(x, False, True))
    out, counts = launches(g, lambda: g.recurrence(a, x))
    # 188 entries at 16 limbs, 141 at 15 (32 to a part)
    assert counts["product_rows_kernel<true>"] == 7 + 5, counts
    (dx, dg), counts = launches(g, lambda: g.recurrence_grad(a, h, x))
    assert counts["product_rows_kernel<true>"] == 7 + 5 + 2, counts         # 47 sums at 14 limbs, 34 to a part
    for i in (0, 8, 9, 10, 23, 24, 36, n // shared - 1):
        own = slice(i * shared, (i + 1) * shared)
        ai, xi, hi = row(g, a.cts[i:i + 1], 3), row(g, x.cts[own], 3), row(g, h.cts[own], 3)
        equal(g, g.recurrence(ai, xi).cts, out.cts[own])
        one = g.recurrence_grad(ai, hi, xi)
        equal(g, one[0].cts, dx.cts[own])
        equal(g, one[1].cts, dg.cts[i:i + 1])
    # as many gates as inputs: the second of two parts begins with the first gate
    a, x = row(g, x.cts[:31], 3), row(g, x.cts[31:62], 3)
    out, counts = launches(g, lambda: g.recurrence(a, x))
    assert counts["product_rows_kernel<true>"] == 2 + 1, counts
    for i in range(0, 31, 6):
        equal(g, g.recurrence(row(g, a.cts[i:i + 1], 3), row(g, x.cts[i:i + 1], 3)).cts, out.cts[i:i + 1])
    g.close()


def test_single_tokens_in_parts():
    from paper_1810_00845_amd import hisa
    g = hisa.Context(*PARTS)
    g.keygen()
    shared, n = 3, 141
    a, s, x = (row(g, g.ct_random_batch(k, 16, 2.0 ** BITS, c), 2) for k, c in ((n // shared, 1000), (n, 2000), (n, 4000)))
    out, counts = launches(g, lambda: g.recurrence_step(a, s, x))
    assert counts["product_rows_kernel<false>"] == 3, counts        # 47 each: the second begins with the last sharer of a gate
    for i in (0, 15, 16, 31, 32, n // shared - 1):
        own = slice(i * shared, (i + 1) * shared)
        equal(g, g.recurrence_step(row(g, a.cts[i:i + 1], 2), row(g, s.cts[own], 2), row(g, x.cts[own], 2)).cts, out.cts[own])
    g.close()


@pytest.mark.parametrize("groups,products", [(9, 1 + 1 + 1 + 2 + 2), (45, 3 + 4 + 2 + 2 + 2)])
def test_normalisation_in_parts(groups, products):
    """Three images of 45 channels: groups of five, whose products with one 1 / sqrt are in two parts that begin inside a group and an image,
    and of one, where relinearisations, sums of rotations and the products of the variances are in parts too.  Against every group alone."""
    from paper_1810_00845_amd import hisa
    g = hisa.Context(*PARTS)
    g.keygen()
    batch, channels = 3, 45
    per = channels // groups
    cts = g.ct_random_batch(batch * channels, 16, 2.0 ** BITS, 1000)
    t = hisa.CipherTensor(g, cts, batch, channels, 1, 3, 3 * 512, 512, 0, 1)       # five doublings: two sums
    g.gen_rot_keys(g.group_norm_rot_steps(t))
    rng = np.random.default_rng(groups)
    gamma, beta = rng.uniform(0.5, 1.5, channels), rng.uniform(-1, 1, channels)
    args = (1e-3, 0.1, 1.0, 1)
    plan = g.group_norm_prepare(t, gamma, beta, groups, *args, act_ratio=0.5)
    y, counts = launches(g, lambda: g.group_norm_apply(t, plan))
    # the variances at 16 limbs, an iteration's pair at 14 and product at 13, the normalised values at 12, their activation at 11.  A digit has
    # limbs + 6 limbs of 256 KB, three digits down to 13 limbs, then two: 62, 68, 71, 113 and 120 entries to a part of 1 GB
    assert counts["product_rows_kernel<false>"] == products, counts
    g.group_norm_plan_free(plan)
    for e in (0, 67, 68, 90, 134):
        b, first = e // channels, e % channels // per * per
        own = slice(b * channels + first, b * channels + first + per)
        one = hisa.CipherTensor(g, cts[own], 1, per, 1, 3, 3 * 512, 512, 0, 1)
        plan = g.group_norm_prepare(one, gamma[first:first + per], beta[first:first + per], 1, *args, act_ratio=0.5)
        equal(g, g.group_norm_apply(one, plan).cts, y.cts[own])
        g.group_norm_plan_free(plan)
    g.close()


# --- kernels that only larger calls and other parameters reach ---

def test_chains_of_sums_by_rows_of_one_wave():
    """Sixteen groups at 9 limbs, N = 2^12: the rows between two sums are 2304, more than four waves a row serve.  Bits against the oracle and
    against a group alone."""
    from oracle import sequence as seq
    from paper_1810_00845_amd import synth
    g, o = pair(12, 9, 3)
    gt, ot = random_tensors(g, o, 16, 9, 2.0 ** BITS, 3, batch=16, height=1, width=3, w_stride=64)
    steps = g.group_norm_rot_steps(gt)
    g.gen_rot_keys(steps); o.gen_rot_keys(steps)
    gamma, beta = (np.stack([synth.plaintext_coeffs(k, g.N, bits)]) for k, bits in ((7, 30), (70, 40)))
    args = (1, 1e-3, 0.05, 2.0, 1)
    plan = g.group_norm_prepare_fixed(gt, gamma, 2.0 ** 35, beta, *args)
    y, counts = launches(g, lambda: g.group_norm_apply(gt, plan))
    assert counts["final_inverse_rows_kernel"] == 1 and "final_inverse_wide_kernel" not in counts, counts
    for i in range(16):
        one, counts = launches(g, lambda: g.group_norm_apply(gt.shaped_like(cts=gt.cts[i:i + 1], batch=1), plan))
        assert counts["final_inverse_wide_kernel"] == 1
        equal(g, one.cts, y.cts[i:i + 1])
    for i in (0, 15):
        want = seq.group_norm_fixed(o, replace(ot, cts=ot.cts[i:i + 1], batch=1), gamma, 2.0 ** 35, beta, *args)
        assert np.array_equal(g.ct_export(y.cts[i]), o.export(want.cts[0]))
    g.group_norm_plan_free(plan)
    g.close()


@pytest.mark.parametrize("limbs,dnum,gates,x", [(9, 8, 2, 6), (8, 8, 5, 5), (10, 5, 1, 4)])
def test_pairs_of_more_than_four_digits(limbs, dnum, gates, x):
    """Inner products of four pairs at a time, the last ones part filled."""
    from oracle import sequence as seq
    g, o = pair(12, limbs, dnum)
    ga, oa = random_tensors(g, o, gates, limbs, 2.0 ** BITS, 1, width=3)
    gx, ox = random_tensors(g, o, x, limbs, 2.0 ** BITS, 2, width=3)
    steps = g.recurrence_rot_steps(gx)
    g.gen_rot_mul_keys(steps); seq.gen_rot_mul_keys(o, steps)
    out, counts = launches(g, lambda: g.recurrence(ga, gx))
    assert counts["pair_inner_kernel"] >= 1, counts
    same(g, o, out, seq.recurrence(o, oa, ox))
    g.close()


def test_dry_run_of_a_gradient():
    from paper_1810_00845_amd import hisa
    g = hisa.Context(12, [50] + [BITS] * 7, 2, 50, 5)
    like = g.tensor_encrypt(np.zeros((1, 4, 1, 6)), 2.0 ** BITS, 8)
    g.analysis_begin()
    x, h = (g.tensor_encrypt(np.zeros((1, 4, 1, 6)), 2.0 ** BITS, 8) for _ in range(2))
    a = g.tensor_encrypt(np.zeros((1, 2, 1, 6)), 2.0 ** BITS, 8)
    dx, dg = g.recurrence_grad(a, h, x, True)
    counts, steps = g.analysis_end()
    assert sorted(steps) == sorted(g.recurrence_rot_steps(like, True, True))
    assert (len(dx.cts), dx.cts[0].limbs, len(dg.cts), dg.cts[0].limbs) == (4, 5, 2, 4) and counts["min_limbs"] == 4
    # the gates moved, three rounds on four ciphertexts and (but for the last) two gates, two sums of products
    assert counts["rot_left"] == 2 + 3 * 4 + 2 * 2 + 2 and counts["relinearize"] == counts["mul"] == 3 * 4 + 2 * 2 + 2
    g.close()
