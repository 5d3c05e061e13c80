"""GPU: recurrences and group normalisation through the C ABI, bit for bit against the oracle, decrypted against plain fp64 arrays,
and what they refuse."""
import ctypes as C

import numpy as np
import pytest

import sequence_plain as plain

pytestmark = pytest.mark.gpu

BITS = 40


def pair(log_n, limbs, dnum, bits=BITS, seed=5):
    from oracle import Oracle
    from paper_1810_00845_amd import hisa
    q = [50] + [bits] * (limbs - 1)
    g, o = hisa.Context(log_n, q, dnum, 50, seed), Oracle(log_n, q, dnum, 50, seed)
    g.keygen(); o.keygen()
    return g, o


def random_tensors(g, o, cts, limbs, scale, seed, batch=1, channels=None, height=1, width=1, h_stride=0, w_stride=1, offset=0, c_inner=1, c_stride=0, clean=1):
    """Uniform residues on both sides (what encryptions look like): bits only, nothing to decrypt."""
    from oracle import layers
    from paper_1810_00845_amd import hisa, synth
    res = synth.uniform_residues(seed, (cts, 2, limbs, g.N), g.primes[:limbs])
    channels = channels or cts // batch * c_inner
    meta = (batch, channels, height, width, h_stride or width * w_stride, w_stride, offset, clean, c_inner, c_stride)
    return (hisa.CipherTensor(g, g.ct_import_batch(res, scale), *meta), layers.OTensor([o.import_ct(r, scale) for r in res], *meta))


def same(g, o, gt, ot):
    assert len(gt.cts) == len(ot.cts)
    assert (gt.channels, gt.height, gt.width, gt.clean, gt.c_inner) == (ot.channels, ot.height, ot.width, ot.clean, ot.c_inner)
    for a, b in zip(gt.cts, ot.cts):
        assert abs(a.scale - b.scale) <= 1e-9 * b.scale
        assert np.array_equal(g.ct_export(a), o.export(b))


def limit(log_n, special, levels, size=1.0, bits=BITS):
    # as on the CPU, with the largest of 10^5 slots within 12 standard deviations
    return 12 * plain.noise(log_n, special, 2.0 ** bits) * levels * max(1.0, size)


# --- bits ---

@pytest.mark.parametrize("limbs,dnum,gate_level,x_level,batch,gates,x,width,height,w_stride,reverse", [
    (4, 2, 4, 4, 1, 1, 1, 2, 1, 1, False),      # one level
    (6, 3, 6, 6, 1, 1, 2, 5, 2, 3, True),       # a gate for two, last digit whole
    (7, 2, 6, 7, 2, 1, 3, 9, 1, 1, False),      # a level higher than its gates, down to one limb of two digits
    (5, 1, 5, 4, 1, 2, 2, 3, 1, 2, False),      # one digit
    (6, 5, 6, 6, 1, 1, 1, 8, 1, 1, True),       # digits of two, five asked for
    (9, 8, 9, 9, 1, 1, 1, 3, 1, 1, False),      # more than four digits
])
def test_recurrence_bits(limbs, dnum, gate_level, x_level, batch, gates, x, width, height, w_stride, reverse):
    from oracle import sequence as seq
    g, o = pair(12, limbs, dnum)
    layout = dict(batch=batch, width=width, height=height, w_stride=w_stride)
    ga, oa = random_tensors(g, o, batch * gates, gate_level, 2.0 ** BITS, 1, **layout)
    gx, ox = random_tensors(g, o, batch * x, x_level, 2.0 ** BITS, 2, **layout)
    steps = g.recurrence_rot_steps(gx, reverse)
    assert steps == seq.recurrence_steps(o, ox, reverse)
    g.gen_rot_mul_keys(steps); seq.gen_rot_mul_keys(o, steps)
    same(g, o, g.recurrence(ga, gx, reverse), seq.recurrence(o, oa, ox, reverse))
    g.close()


def test_recurrence_of_one_token_is_its_input():
    g, o = pair(12, 4, 2)
    ga, _ = random_tensors(g, o, 1, 4, 2.0 ** BITS, 1)
    gx, ox = random_tensors(g, o, 2, 3, 2.0 ** BITS, 2)
    assert g.recurrence_rot_steps(gx) == []
    same(g, o, g.recurrence(ga, gx), ox)
    g.close()


@pytest.mark.parametrize("limbs,dnum,levels,gates,x", [(4, 2, (4, 4, 4), 1, 1), (6, 3, (6, 4, 5), 1, 3), (3, 3, (2, 3, 3), 2, 2)])
def test_step_bits(limbs, dnum, levels, gates, x):
    from oracle import sequence as seq
    g, o = pair(12, limbs, dnum)
    scales = (2.0 ** BITS, 2.0 ** BITS * 1.25, 2.0 ** (BITS - 1))
    (ga, oa), (gs, os_), (gx, ox) = (random_tensors(g, o, n, l, s, k) for k, (n, l, s) in enumerate(zip((gates, x, x), levels, scales)))
    same(g, o, g.recurrence_step(ga, gs, gx), seq.recurrence_step(o, oa, os_, ox))
    g.close()


@pytest.mark.parametrize("limbs,dnum,level_h,gates,x,width,reverse", [(5, 2, 5, 1, 1, 2, False), (7, 3, 4, 1, 3, 5, True), (6, 2, 6, 2, 2, 4, False),
                                                                    (5, 2, 4, 1, 9, 3, False)])
def test_gradient_bits(limbs, dnum, level_h, gates, x, width, reverse):
    from oracle import sequence as seq
    g, o = pair(12, limbs, dnum)
    ga, oa = random_tensors(g, o, gates, limbs, 2.0 ** BITS, 1, width=width)
    gg, og = random_tensors(g, o, x, limbs, 2.0 ** BITS, 2, width=width)
    gh, oh = random_tensors(g, o, x, level_h, 2.0 ** BITS, 3, width=width)
    steps = g.recurrence_rot_steps(gg, reverse, True)
    assert steps == seq.recurrence_steps(o, og, reverse, True)
    g.gen_rot_mul_keys(steps); seq.gen_rot_mul_keys(o, steps)
    for got, want in zip(g.recurrence_grad(ga, gh, gg, reverse), seq.recurrence_grad(o, oa, oh, og, reverse)):
        same(g, o, got, want)
    g.close()


@pytest.mark.parametrize("reverse", [False, True])
def test_gates_bits(reverse):
    from oracle import sequence as seq
    g, o = pair(12, 3, 3)
    ga, oa = random_tensors(g, o, 4, 3, 2.0 ** BITS, 1, batch=2, height=2, width=3, w_stride=2, c_inner=2, c_stride=40, channels=3, clean=0)
    mask, scale = seq.gates_mask(o, oa, reverse)
    same(g, o, g.recurrence_gates_fixed(ga, mask, scale), seq.gates_fixed(o, oa, mask, scale))
    g.close()


@pytest.mark.parametrize("limbs,dnum,cts,groups,batch,iterations,act,layout", [
    (6, 2, 1, 1, 1, 1, None, dict(height=3, width=3)),
    (9, 3, 6, 2, 1, 2, 0.5, dict(height=2, width=4, w_stride=2, h_stride=8, offset=5)),
    (8, 3, 4, 1, 2, 1, 0.0, dict(height=4, width=2, c_inner=4, c_stride=1, w_stride=4)),
    (6, 5, 7, 1, 1, 1, None, dict(height=1, width=1)),     # no sums over slots; seven ciphertexts to a group
])
def test_group_norm_bits(limbs, dnum, cts, groups, batch, iterations, act, layout):
    from oracle import sequence as seq
    from paper_1810_00845_amd import synth
    g, o = pair(12, limbs, dnum)
    gt, ot = random_tensors(g, o, cts, limbs, 2.0 ** BITS, 3, batch=batch, **layout)
    steps = g.group_norm_rot_steps(gt)
    assert steps == sorted({s for sums in seq.norm_sums(o, ot) for s in sums})
    g.gen_rot_keys(steps) if steps else None
    o.gen_rot_keys(steps)
    gamma = np.stack([synth.plaintext_coeffs(7 + i, g.N, 30) for i in range(cts // batch)])
    beta = np.stack([synth.plaintext_coeffs(70 + i, g.N, 40) for i in range(cts // batch)])
    args = (groups, 1e-3, 0.05, 2.0, iterations)
    plan = g.group_norm_prepare_fixed(gt, gamma, 2.0 ** 35, beta, *args, act_ratio=act)
    want = seq.group_norm_fixed(o, ot, gamma, 2.0 ** 35, beta, *args, act)
    for _ in range(2):
        same(g, o, g.group_norm_apply(gt, plan), want)
    g.group_norm_plan_free(plan)
    g.close()


def test_keys_bits_and_import():
    from oracle import sequence as seq
    from paper_1810_00845_amd import hisa
    g, o = pair(12, 4, 2)
    g.gen_rot_mul_keys([3, 0, -2]); seq.gen_rot_mul_keys(o, [3, -2])
    ids = [0] + [f(g.galois_elt(s)) for s in (3, -2) for f in (int, seq.product_key_id)]
    other = hisa.Context(12, [50] + [BITS] * 3, 2, 50, 99)
    for k in ids:
        key = g.key_export(k)
        assert np.array_equal(key, o.keys[k])
        other.key_import(k, key)
        other.key_import(k, key)
        assert np.array_equal(other.key_export(k), key)
    key[1, 0, 2, 7] = g.primes[2]
    for bad in (2, 1, 1 << 32, (2 << 32) | 5, 2 * g.N + 1, (1 << 32) | 4):
        with pytest.raises(hisa.HisaError) as e:
            other.key_import(bad, o.keys[0])
        assert e.value.code == -1
    with pytest.raises(hisa.HisaError) as e:
        other.key_import(0, key)
    assert e.value.code == -1
    assert np.array_equal(other.key_export(0), o.keys[0])
    g.close(); other.close()


def test_many_ciphertexts_are_those_of_few():
    """More entries than one part of the work holds, gates shared by a number that divides no part."""
    from paper_1810_00845_amd import hisa
    g = hisa.Context(12, [50] + [BITS] * 3, 2, 50, 5)
    g.keygen()
    shared, n = 7, 1505

    def tensor(cts):
        return hisa.CipherTensor(g, cts, 1, len(cts), 1, 3, 3, 1, 0, 1)
    a, x = g.ct_random_batch(n // shared, 4, 2.0 ** BITS, 11), g.ct_random_batch(n, 4, 2.0 ** BITS, 22)
    g.gen_rot_mul_keys(g.recurrence_rot_steps(tensor(x)))
    out = g.recurrence(tensor(a), tensor(x)).cts
    for i in (0, 3, 90, n // shared - 1):
        few = g.recurrence(tensor(a[i:i + 1]), tensor(x[i * shared:(i + 1) * shared])).cts
        for k in (0, shared - 1):
            assert np.array_equal(g.ct_export(few[k]), g.ct_export(out[i * shared + k]))
    for t in (tensor(a), tensor(x)):
        t.free()
    # the normalisation's products of 1500 ciphertexts with one 1 / sqrt, in parts that begin inside the group
    g.close()
    g = hisa.Context(12, [50] + [BITS] * 7, 2, 50, 5)
    g.keygen()
    x = g.ct_random_batch(1500, 8, 2.0 ** BITS, 33)
    whole = tensor(x)
    g.gen_rot_keys(g.group_norm_rot_steps(whole))
    plan = g.group_norm_prepare(whole, None, None, 1, 1e-3, 0.1, 1.0, 1)
    out = g.group_norm_apply(whole, plan).cts
    two = g.group_norm_apply(whole.shaped_like(cts=[g.copy(c) for c in x]), plan).cts       # an allocation each
    for i in (0, 749, 750, 1499):
        assert np.array_equal(g.ct_export(out[i]), g.ct_export(two[i]))
    g.group_norm_plan_free(plan)
    # and against the product that the last part should hold: the same ciphertext twice in a group normalises to the same
    same_ct = whole.shaped_like(cts=x[:750] + x[:750])
    plan = g.group_norm_prepare(whole, np.ones(1500), np.zeros(1500), 1, 1e-3, 0.1, 1.0, 1)
    out = g.group_norm_apply(same_ct, plan).cts
    for i in (0, 200, 749):
        assert np.array_equal(g.ct_export(out[i]), g.ct_export(out[750 + i]))
    g.group_norm_plan_free(plan)
    g.close()


# --- values ---

@pytest.mark.parametrize("log_n,limbs,dnum,shape,gates,layout,reverse", [
    (13, 8, 2, (1, 2, 3, 5), 1, dict(offset=3), False),
    (14, 12, 3, (2, 4, 2, 100), 2, dict(c_inner=2, c_stride=512), False),
    (13, 9, 4, (1, 4, 1, 9), 4, dict(c_inner=4, c_stride=1, w_stride=4), True),
    (15, 18, 3, (1, 1, 1, 16384), 1, {}, True),             # every slot a token
])
def test_recurrence_and_gradient_values(log_n, limbs, dnum, shape, gates, layout, reverse):
    from paper_1810_00845_amd import hisa
    rng = np.random.default_rng(log_n + shape[3])
    x, a, gr = rng.uniform(-1, 1, shape), rng.uniform(0.2, 0.9, (shape[0], gates) + shape[2:]), rng.uniform(-1, 1, shape)
    ci = layout.get("c_inner", 1)
    g = hisa.Context(log_n, [50] + [BITS] * (limbs - 1), dnum, 50, 7)
    g.keygen()
    ta, tx, tg = (g.tensor_encrypt(v, 2.0 ** BITS, limbs, **layout) for v in (a, x, gr))
    g.gen_rot_mul_keys(sorted(set(g.recurrence_rot_steps(tx, reverse) + g.recurrence_rot_steps(tx, reverse, True))))
    ta = g.recurrence_gates(ta, reverse)
    h = g.recurrence(ta, tx, reverse)
    want = plain.recurrence(a, x, reverse, ci)
    levels = (shape[3] - 1).bit_length()
    # an error in a gate or a token counts up to 1 / (1 - 0.9) times, a state is at most ten
    tol = limit(log_n, g.K, levels + 1, 100.0)
    assert h.cts[0].limbs == limbs - 1 - levels
    assert np.abs(g.tensor_decrypt(h) - want).max() <= tol
    dx, dg = g.recurrence_grad(ta, h, tg, reverse)
    wx, wa = plain.recurrence_grad(a, want, gr, reverse, ci)
    assert np.abs(g.tensor_decrypt(dx) - wx).max() <= tol
    dg = g.tensor_decrypt(g.recurrence_gates(dg, reverse))
    assert np.abs(dg - wa).max() <= tol * 20 * shape[1] // gates + tol * 20 * (shape[1] // gates)
    g.close()


def test_state_in_front_of_a_scan():
    """Two halves of a sequence, the second continued from the state the first ended in, are the whole."""
    from paper_1810_00845_amd import hisa
    rng = np.random.default_rng(4)
    x, a = rng.uniform(-1, 1, (1, 1, 1, 8)), rng.uniform(0.3, 0.9, (1, 1, 1, 8))
    g = hisa.Context(13, [50] + [BITS] * 8, 3, 50, 7)
    g.keygen()
    put = lambda v: g.tensor_encrypt(v, 2.0 ** BITS, 9)  # noqa: E731
    first = plain.recurrence(a[..., :4], x[..., :4])
    state = np.zeros((1, 1, 1, 4))
    state[..., 0] = first[..., 3]
    ta, tx = put(a[..., 4:]), put(x[..., 4:])
    g.gen_rot_mul_keys(g.recurrence_rot_steps(tx))
    h = g.recurrence(g.recurrence_gates(ta), g.recurrence_step(ta, put(state), tx))
    assert np.abs(g.tensor_decrypt(h) - plain.recurrence(a, x)[..., 4:]).max() <= limit(13, g.K, 4, 100.0)
    g.close()


@pytest.mark.parametrize("log_n,limbs,dnum,shape,groups,iterations,act,layout", [
    (13, 9, 2, (1, 1, 5, 5), 1, 2, None, {}),
    (13, 13, 3, (2, 6, 9, 7), 3, 4, None, dict(h_stride=16, w_stride=2, offset=1)),
    (14, 14, 3, (1, 32, 6, 6), 2, 4, 0.5, dict(c_inner=16, c_stride=1, w_stride=16)),     # channels last
])
def test_group_norm_values(log_n, limbs, dnum, shape, groups, iterations, act, layout):
    from paper_1810_00845_amd import hisa
    rng = np.random.default_rng(shape[1])
    x = rng.normal(0.3, 0.8, shape)
    gamma, beta = rng.uniform(0.5, 1.5, shape[1]), rng.uniform(-1, 1, shape[1])
    var = x.reshape(shape[0], groups, -1).var(-1)
    lo, hi = var.min() / 2, var.max() * 2
    g = hisa.Context(log_n, [50] + [BITS] * (limbs - 1), dnum, 50, 7)
    g.keygen()
    t = g.tensor_encrypt(x, 2.0 ** BITS, limbs, **layout)
    g.gen_rot_keys(g.group_norm_rot_steps(t))
    plan = g.group_norm_prepare(t, gamma, beta, groups, 1e-3, lo, hi, iterations, act_ratio=act)
    got = g.tensor_decrypt(g.group_norm_apply(t, plan))
    base, want = plain.group_norm(x, gamma, beta, groups, 1e-3), plain.group_norm(x, gamma, beta, groups, 1e-3, act)
    top = np.abs(x).max() / np.sqrt(lo) * 1.5
    # 1 / sqrt within its cubics' error; noise of v at 1 / 64 of the scale, of the sums at n of it (averaged: one), twelve divisions of either
    tol = top * plain.cubic_error(lo, hi, iterations) + limit(log_n, g.K, 64 * 12, top / lo)
    if act is not None:
        tol *= 2 * np.abs(base).max() + abs(act) + tol
    assert np.abs(got - want).max() <= tol
    g.group_norm_plan_free(plan)
    default = g.group_norm_prepare(t, None, None, groups, 1e-3, lo, hi, iterations, act_ratio=act)
    ones = plain.group_norm(x, np.ones(shape[1]), np.zeros(shape[1]), groups, 1e-3, act)
    assert np.abs(g.tensor_decrypt(g.group_norm_apply(t, default)) - ones).max() <= tol
    g.group_norm_plan_free(default)
    g.close()


def test_a_block_of_both():
    """Scan, normalisation by heads with its activation, and a fully connected layer on what comes out, in one run; on a stream of its own."""
    import torch
    from paper_1810_00845_amd import hisa
    rng = np.random.default_rng(8)
    x, a, w = rng.uniform(-1, 1, (1, 4, 1, 8)), rng.uniform(0.2, 0.9, (1, 2, 1, 8)), rng.normal(0, 0.2, (3, 4, 1, 8))
    stream = torch.cuda.Stream()
    g = hisa.Context(13, [50] + [BITS] * 15, 3, 50, 7, stream=stream.cuda_stream)
    g.keygen()
    ta, tx = (g.tensor_encrypt(v, 2.0 ** BITS, 16) for v in (a, x))
    h0 = plain.recurrence(a, x)
    var = h0.reshape(1, 2, -1).var(-1)
    lo, hi = var.min() / 2, var.max() * 2
    g.gen_rot_mul_keys(g.recurrence_rot_steps(tx))
    g.gen_rot_keys(g.group_norm_rot_steps(tx) + g.fc_rot_steps(tx))
    h = g.recurrence(g.recurrence_gates(ta), tx)
    plan = g.group_norm_prepare(h, None, None, 2, 1e-3, lo, hi, 3, act_ratio=1.0)
    y = g.group_norm_apply(h, plan)
    out = g.fc(y, w)
    want = plain.group_norm(h0, np.ones(4), np.zeros(4), 2, 1e-3, 1.0)
    got = g.tensor_decrypt(out)[0, :, 0, 0]
    top = np.abs(h0).max() / np.sqrt(lo) * 1.5
    tol = (top * plain.cubic_error(lo, hi, 3) + limit(13, g.K, 64 * 12, 100 * top / lo)) * (2 * top + 2)
    assert np.abs(g.tensor_decrypt(y) - want).max() <= tol
    assert np.abs(got - (w * want).sum((1, 2, 3))).max() <= tol * np.abs(w).sum((1, 2, 3)).max() + 1e-4
    g.group_norm_plan_free(plan)
    g.close()


@pytest.mark.parametrize("limbs,dnum", [(12, 3), (12, 1), (11, 2)])
def test_rotation_sums_of_a_ragged_number(limbs, dnum):
    """Sums of rotations of three and more ciphertexts, the last group of outputs part filled, against one at a time."""
    from paper_1810_00845_amd import hisa
    g = hisa.Context(15, [50] + [BITS] * (limbs - 1), dnum, 50, 5)
    steps = [0, 1, 2, 3, 4, 5, 6, 7]
    g.gen_rot_keys(steps[1:])
    cts = g.ct_random_batch(7, limbs, 2.0 ** BITS, 3)
    one = [g.ct_export(g.rot_left_sum_batch([[c]] * 8, steps)[0]) for c in cts]
    for n in (3, 5, 6, 7):
        some = [g.copy(c) for c in cts[7 - n:]] if n == 5 else cts[7 - n:]      # an allocation each, views of one
        for got, want in zip(g.rot_left_sum_batch([some] * 8, steps), one[7 - n:]):
            assert np.array_equal(g.ct_export(got), want)
    g.close()


def test_two_contexts_at_once():
    """Two contexts of one key and seed on streams of their own, their layers queued in turn: what one of them alone leaves."""
    import torch
    from paper_1810_00845_amd import hisa
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = []
    for st in streams:
        g = hisa.Context(13, [50] + [BITS] * 8, 3, 50, 5, stream=st.cuda_stream)
        g.keygen()
        cts = g.ct_random_batch(8, 9, 2.0 ** BITS, 21)
        x, a = (hisa.CipherTensor(g, c, 1, len(c), 1, 7, 7, 1, 0, 1) for c in (cts[:6], cts[6:]))
        g.gen_rot_mul_keys(g.recurrence_rot_steps(x) + g.recurrence_rot_steps(x, False, True))
        g.gen_rot_keys(g.group_norm_rot_steps(x))
        both.append((g, x, a, g.group_norm_prepare(x, None, None, 2, 1e-3, 0.1, 1.0, 2)))

    def layers(g, x, a, plan):
        h = g.recurrence(a, x)
        return [h, *g.recurrence_grad(a, h, x), g.group_norm_apply(x, plan)]
    want = [[both[0][0].ct_export(c) for c in t.cts] for t in layers(*both[0])]
    torch.cuda.synchronize()
    queued = [layers(*both[i % 2]) for i in range(6)]
    for i, run in enumerate(queued):
        for t, w in zip(run, want):
            for c, v in zip(t.cts, w):
                assert np.array_equal(both[i % 2][0].ct_export(c), v)
    for g, _x, _a, plan in both:
        g.group_norm_plan_free(plan)
        g.close()


# --- dry runs and refusals ---

def test_dry_run_names_keys_and_levels():
    from paper_1810_00845_amd import hisa
    g = hisa.Context(12, [50] + [BITS] * 7, 2, 50, 5)
    g.analysis_begin()
    x = g.tensor_encrypt(np.zeros((1, 2, 1, 6)), 2.0 ** BITS, 8)
    a = g.tensor_encrypt(np.zeros((1, 1, 1, 6)), 2.0 ** BITS, 8)
    h = g.recurrence(g.recurrence_gates(a), x)
    counts, steps = g.analysis_end()
    assert steps == g.recurrence_rot_steps(x)
    assert counts["min_limbs"] == 4 and h.cts[0].limbs == 4
    assert counts["rot_left"] == 3 + 3 + 2 and counts["relinearize"] == counts["mul"] == 8
    g.close()


def test_dry_run_of_a_normalisation():
    from paper_1810_00845_amd import hisa
    g = hisa.Context(12, [50] + [BITS] * 8, 2, 50, 5)
    like = g.tensor_encrypt(np.zeros((2, 4, 2, 3)), 2.0 ** BITS, 9)
    plan = g.group_norm_prepare(like, None, None, 2, 1e-3, 0.1, 1.0, 2, act_ratio=0.5)
    g.analysis_begin()
    x = g.tensor_encrypt(np.zeros((2, 4, 2, 3)), 2.0 ** BITS, 9)
    y = g.group_norm_apply(x, plan)
    counts, steps = g.analysis_end()
    assert sorted(steps) == sorted(set(g.group_norm_rot_steps(like)))
    assert y.cts[0].limbs == counts["min_limbs"] == 9 - 8
    # x x and its sums' product a group, three products an iteration and group, the normalised values' two; rotations of both sums
    assert counts["relinearize"] == 4 + 4 + 2 * 3 * 4 + 2 * 8
    assert counts["rot_left"] == 8 * len(g.group_norm_rot_steps(like))
    g.group_norm_plan_free(plan)
    g.close()


def refused(code, f, *args, **kw):
    from paper_1810_00845_amd import hisa
    with pytest.raises(hisa.HisaError) as e:
        f(*args, **kw)
    assert e.value.code == code, e.value


def test_refusals():
    from paper_1810_00845_amd import hisa
    g = hisa.Context(12, [50] + [BITS] * 5, 2, 50, 5)
    ARG, LEVEL, SCALE, KEY, DEPTH = -1, -2, -3, -4, -6

    def tensor(limbs=6, channels=2, width=4, scale=2.0 ** BITS, **kw):
        kw.setdefault("w_stride", 1)
        t = g.tensor_encrypt(np.zeros((1, channels, kw.pop("height", 1), width)), scale, limbs, **kw)
        return t
    a, x = tensor(), tensor()
    refused(KEY, g.recurrence, a, x)
    refused(KEY, g.recurrence_grad, a, x, x)
    refused(KEY, g.recurrence_step, a, x, x)
    g.gen_rot_keys(g.recurrence_rot_steps(x))
    refused(KEY, g.recurrence, a, x)             # the rotations' keys alone are not enough
    g.keygen()
    g.gen_rot_mul_keys(g.recurrence_rot_steps(x) + g.recurrence_rot_steps(x, False, True))
    assert g.recurrence(a, x).cts[0].limbs == 4
    refused(DEPTH, g.recurrence, tensor(limbs=2), x)
    refused(DEPTH, g.recurrence_grad, tensor(limbs=3), x, x)
    refused(DEPTH, g.recurrence_step, tensor(limbs=1), x, x)
    for other in (tensor(width=5), tensor(channels=3), tensor(w_stride=2), tensor(offset=1), tensor(channels=4)):
        refused(ARG, g.recurrence, other, x)
        refused(ARG, g.recurrence_step, a, other, x)
    refused(ARG, g.recurrence, a.shaped_like(clean=0), x)
    refused(ARG, g.recurrence, a, x.shaped_like(clean=0))
    refused(ARG, g.recurrence, a, x.shaped_like(w_stride=0, h_stride=0))
    one = tensor(width=1)
    refused(ARG, g.recurrence_grad, one, one, one)
    both = x.shaped_like()      # one output for two gradients
    (st, _arr), (xs, _brr) = both._struct(), x._struct()
    assert hisa.load().hisa_recurrence_grad(g._vp, C.byref(xs), C.byref(xs), C.byref(xs), C.c_uint32(0), C.byref(st), C.byref(st)) == ARG
    refused(SCALE, g.recurrence, tensor(scale=2.0 ** 9.5), x)
    refused(SCALE, g.recurrence_step, tensor(scale=2.0 ** 3), tensor(scale=2.0 ** 3), x)
    mixed = x.shaped_like(cts=[x.cts[0], tensor(scale=2.0 ** 39).cts[0]])
    refused(SCALE, g.recurrence, a, mixed)
    refused(DEPTH, g.recurrence_gates, tensor(limbs=1))
    # normalisation
    n = hisa.Context(12, [50] + [BITS] * 7, 2, 50, 5)
    t = n.tensor_encrypt(np.zeros((1, 4, 3, 3)), 2.0 ** BITS, 8)
    good = dict(groups=2, eps=1e-3, var_lo=0.1, var_hi=1.0, iterations=2)
    plan = n.group_norm_prepare(t, None, None, **good)
    refused(KEY, n.group_norm_apply, t, plan)
    n.keygen()
    refused(KEY, n.group_norm_apply, t, plan)
    for bad in (dict(groups=3), dict(groups=0), dict(iterations=0), dict(iterations=17), dict(eps=-1.0), dict(eps=2.0), dict(var_lo=0.0),
                dict(var_hi=0.1), dict(var_hi=float("inf")), dict(var_lo=float("nan"))):
        refused(ARG, n.group_norm_prepare, t, None, None, **dict(good, **bad))
    refused(DEPTH, n.group_norm_prepare, t, None, None, **dict(good, iterations=3))
    refused(DEPTH, n.group_norm_prepare, t, None, None, **dict(good, act_ratio=0.5, iterations=3))
    refused(SCALE, n.group_norm_prepare, t, None, None, **dict(good, var_lo=1e9, var_hi=1e12))
    refused(SCALE, n.group_norm_prepare, t, None, None, **dict(good, eps=0.0, var_lo=1e-31, var_hi=1e-30))
    refused(ARG, n.group_norm_prepare, t, np.full(4, 1e12), None, **good)
    refused(ARG, n.group_norm_prepare, t.shaped_like(clean=0), None, None, **good)
    chw = n.tensor_encrypt(np.zeros((1, 4, 3, 3)), 2.0 ** BITS, 8, c_inner=4, c_stride=16)
    refused(ARG, n.group_norm_prepare, chw, None, None, **good)       # two groups in a ciphertext
    refused(ARG, n.group_norm_apply, chw, plan)
    refused(LEVEL, n.group_norm_apply, n.tensor_encrypt(np.zeros((1, 4, 3, 3)), 2.0 ** BITS, 7), plan)
    refused(SCALE, n.group_norm_apply, n.tensor_encrypt(np.zeros((1, 4, 3, 3)), 2.0 ** 39, 8), plan)
    n.group_norm_plan_free(plan)
    # parameters without the fused key switch
    wide = hisa.Context(12, [58, 58, 58], 3, 60, 5)
    w = wide.tensor_encrypt(np.zeros((1, 1, 1, 4)), 2.0 ** 50, 3)
    refused(ARG, wide.gen_rot_mul_keys, [1])
    refused(ARG, wide.recurrence, w, w)
    refused(ARG, wide.recurrence_step, w, w, w)
    refused(ARG, wide.group_norm_prepare, w, None, None, 1, 0.0, 0.1, 1.0, 1)
    for c in (g, n, wide):
        c.close()
