"""CPU: the oracle's recurrences and normalisation against plain fp64 arrays, the plain backward pass against differences, and what of
the library's side needs no GPU (exported symbols' argument checks, structure layout)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import sequence_plain as plain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LOG_N, BITS, SPECIAL = 7, 40, 50


def oracle(limbs, dnum=2, seed=5):
    from oracle import Oracle
    o = Oracle(LOG_N, [50] + [BITS] * (limbs - 1), dnum, SPECIAL, seed)
    o.keygen()
    return o


def encrypted(o, x, limbs, **layout):
    from oracle import layers
    if layout.get("c_inner", 1) > 1:
        return layers.tensor_encrypt_chw(o, x, 2.0 ** BITS, limbs, **layout)
    layout.pop("c_inner", None), layout.pop("c_stride", None)
    return layers.tensor_encrypt(o, x, 2.0 ** BITS, limbs, **layout)


def decrypted(o, t):
    from oracle import layers
    return layers.tensor_decrypt(o, t)


def limit(o, levels, size=1.0):
    # 64 slots, a handful of noises a level, each multiplied by what follows at most `size` times: 12 standard deviations
    return 12 * plain.noise(LOG_N, o.K, 2.0 ** BITS) * levels * max(1.0, size)


@pytest.mark.parametrize("shape,gates,layout,reverse", [
    ((1, 1, 1, 2), 1, {}, False), ((2, 2, 3, 5), 2, dict(w_stride=2), True), ((1, 4, 2, 7), 2, dict(h_stride=11, offset=3), False),
    ((1, 4, 2, 5), 2, dict(c_inner=2, c_stride=20), False), ((1, 3, 1, 64), 1, {}, False)])
def test_scan_and_its_gradient(shape, gates, layout, reverse):
    from oracle import sequence as seq
    rng = np.random.default_rng(sum(shape))
    x, a, g = rng.uniform(-1, 1, shape), rng.uniform(0.3, 1.0, (shape[0], gates) + shape[2:]), rng.uniform(-1, 1, shape)
    ci = layout.get("c_inner", 1)
    limbs = 4 + (shape[3] - 1).bit_length()
    o = oracle(limbs)
    ta, tx, tg = (encrypted(o, v, limbs, **dict(layout)) for v in (a, x, g))
    seq.gen_rot_mul_keys(o, seq.recurrence_steps(o, tx, reverse) + seq.recurrence_steps(o, tx, reverse, True))
    ta = seq.gates_fixed(o, ta, *seq.gates_mask(o, ta, reverse))
    h = seq.recurrence(o, ta, tx, reverse)
    want = plain.recurrence(a, x, reverse, ci)
    tol = limit(o, limbs, shape[3] * np.abs(want).max())
    assert np.abs(decrypted(o, h) - want).max() <= tol
    dx, dg = seq.recurrence_grad(o, ta, h, tg, reverse)
    wx, wa = plain.recurrence_grad(a, want, g, reverse, ci)
    assert np.abs(decrypted(o, dx) - wx).max() <= tol
    dg = seq.gates_fixed(o, dg, *seq.gates_mask(o, dg, reverse))
    assert np.abs(decrypted(o, dg) - wa).max() <= tol * max(1.0, np.abs(wx).max()) * shape[1]


def test_plain_gradient_against_differences():
    rng = np.random.default_rng(3)
    for reverse in (False, True):
        a, x, g = rng.uniform(0.3, 1, (1, 2, 1, 6)), rng.uniform(-1, 1, (1, 4, 1, 6)), rng.uniform(-1, 1, (1, 4, 1, 6))
        dx, da = plain.recurrence_grad(a, plain.recurrence(a, x, reverse), g, reverse)
        f = lambda a_, x_: (plain.recurrence(a_, x_, reverse) * g).sum()  # noqa: E731
        for v, d, other in ((x, dx, lambda p: f(a, p)), (a, da, lambda p: f(p, x))):
            for i in np.ndindex(v.shape):
                step = np.zeros_like(v)
                step[i] = 1e-5
                # polynomials of degree at most six with values of order one: central differences err by 1e-10 and roundings of 1e-10
                assert abs((other(v + step) - other(v - step)) / 2e-5 - d[i]) < 1e-8


def test_steps_one_by_one_are_the_scan():
    from oracle import sequence as seq
    rng = np.random.default_rng(9)
    o = oracle(6)
    x, a = rng.uniform(-1, 1, (1, 2, 2, 4)), rng.uniform(0.3, 1, (1, 1, 2, 4))
    one = lambda v, t: encrypted(o, v[..., t:t + 1], 6)  # noqa: E731
    state = one(x, 0)
    want = plain.recurrence(a, x)
    for t in range(1, 4):
        state = seq.recurrence_step(o, one(a, t), state, one(x, t))
        assert np.abs(decrypted(o, state) - want[..., t:t + 1]).max() <= limit(o, t, 2.0)
    assert state.cts[0].limbs == 3


@pytest.mark.parametrize("shape,groups,iterations,act,layout", [
    ((1, 1, 3, 3), 1, 3, None, {}), ((2, 4, 2, 3), 2, 4, 0.5, dict(offset=2, h_stride=4)),
    ((1, 4, 3, 3), 2, 3, 0.0, dict(c_inner=2, c_stride=1, w_stride=2, h_stride=6))])
def test_normalisation(shape, groups, iterations, act, layout):
    from oracle import sequence as seq
    rng = np.random.default_rng(shape[1])
    x = rng.uniform(-1, 1, shape) * np.sqrt(3) + 0.3
    v = x.reshape(shape[0], groups, -1).var(-1)
    lo, hi = v.min() / 1.5, v.max() * 1.5
    limbs = 5 + 2 * iterations + (act is not None)
    o = oracle(limbs, dnum=3)
    t = encrypted(o, x, limbs, **dict(layout))
    o.gen_rot_keys([s for sums in seq.norm_sums(o, t) for s in sums])
    n = shape[1] // groups * shape[2] * shape[3]
    gamma, beta = rng.uniform(0.5, 1.5, shape[1]), rng.uniform(-1, 1, shape[1])
    ci = t.c_inner
    level = limbs - 2 - 2 * iterations
    gamma_scale = float(o.primes[level]) / n

    def coeffs(values, scale):
        rows = []
        for j in range(shape[1] // ci):
            z = np.zeros(o.slots)
            for c in range(ci):
                for yy in range(shape[2]):
                    for xx in range(shape[3]):
                        z[t.offset + c * t.c_stride + yy * t.h_stride + xx * t.w_stride] = values[j * ci + c]
            rows.append(o.encode_coeffs(z, scale))
        return np.stack(rows)
    zero = seq.group_norm_fixed(o, t, coeffs(gamma, gamma_scale), gamma_scale, coeffs(0 * beta, 1.0), groups, 1e-3, lo, hi, iterations)
    y = seq.group_norm_fixed(o, t, coeffs(gamma, gamma_scale), gamma_scale, coeffs(beta, zero.cts[0].scale), groups, 1e-3, lo, hi, iterations, act)
    want = plain.group_norm(x, gamma, beta, groups, 1e-3, act)
    err = plain.cubic_error(lo, hi, iterations)
    base = plain.group_norm(x, gamma, beta, groups, 1e-3)
    # the relative error of 1 / sqrt on what is normalised; noise at most n / var_lo of the level's (n x^2 - sums of n values), at 1 / 64 of the scale
    tol = np.abs(base - beta[:, None, None]).max() * err + limit(o, 64 * limbs, n * n / lo)
    if act is not None:
        tol *= 2 * np.abs(base).max() + abs(act) + tol
    assert np.abs(decrypted(o, y) - want).max() <= tol, (np.abs(decrypted(o, y) - want).max(), tol)
    assert y.cts[0].limbs == limbs - 3 - 2 * iterations - (act is not None)


def test_entry_points_refuse_missing_contexts():
    from paper_1810_00845_amd import hisa
    lib = hisa.load()
    n = ctypes.c_size_t()
    assert lib.hisa_recurrence(None, None, None, 0, None) == -1
    assert lib.hisa_recurrence_step(None, None, None, None, None) == -1
    assert lib.hisa_recurrence_grad(None, None, None, None, 0, None, None) == -1
    assert lib.hisa_recurrence_gates(None, None, 0, None) == -1
    assert lib.hisa_recurrence_rot_steps(None, None, 0, 0, None, ctypes.c_size_t(0), ctypes.byref(n)) == -1
    assert lib.hisa_gen_rot_mul_keys(None, None, ctypes.c_size_t(0)) == -1
    assert lib.hisa_key_import(None, ctypes.c_uint64(0), None) == -1
    assert lib.hisa_group_norm_prepare(None, None, None, None, None, None) == -1
    assert lib.hisa_group_norm_apply(None, None, None, None) == -1
    assert lib.hisa_group_norm_plan_free(None, None) == -1


def test_geometry_has_the_layout_of_the_header(tmp_path):
    from paper_1810_00845_amd import hisa
    src, exe = tmp_path / "g.c", tmp_path / "g"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hisa.h"\nint main(void) {\n'
                   '    printf("%zu %zu\\n", sizeof(hisa_norm_geom), offsetof(hisa_norm_geom, act));\n    return 0;\n}\n')
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    assert subprocess.check_output([str(exe)]).split() == [b"%d" % ctypes.sizeof(hisa.NormGeom), b"%d" % hisa.NormGeom.act.offset]


def test_whole_numbers_as_residues(tmp_path):
    """fp_whole of csrc/fparith.hpp, compiled for the host, against Python integers: doubles that are whole numbers up to 2^120."""
    import random
    src, lib = tmp_path / "w.cpp", tmp_path / "w.so"
    src.write_text('#include "fparith.hpp"\nextern "C" double whole(double v, double p) { return fp_whole(v, p, 1.0 / p); }\n')
    inc = os.path.join(ROOT, "paper_1810_00845_amd", "csrc")
    base = ["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-shared", "-fPIC", "-I", inc, str(src), "-o", str(lib)]
    if subprocess.run(base[:4] + ["-mfma"] + base[4:], capture_output=True).returncode != 0:
        subprocess.run(base, check=True)
    f = ctypes.CDLL(str(lib)).whole
    f.restype, f.argtypes = ctypes.c_double, [ctypes.c_double] * 2
    rng = random.Random(1)
    for p in ((1 << 50) - 27, (1 << 40) - 87, (1 << 30) - 35, 16411):
        values = [0.0, 1.0, -1.0, 2.0 ** 52, 2.0 ** 53 - 1, -2.0 ** 53, 2.0 ** 53 + 2, 2.0 ** 119, -(2.0 ** 119) * 1.9999]
        values += [float(int(rng.uniform(-1, 1) * 2.0 ** rng.uniform(0, 120))) for _ in range(2000)]
        for v in values:
            r = f(v, float(p))
            assert r == int(r) and abs(r) <= 0.51 * p and (int(r) - int(v)) % p == 0, (p, v, r)
