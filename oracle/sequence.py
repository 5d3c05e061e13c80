"""Oracle side of the layers of sequence models (TEST INFRASTRUCTURE, not product code): the gated linear recurrence and
group normalisation, as plain loops over ciphertexts on the oracle's primitives."""
from __future__ import annotations

import math
from dataclasses import replace

import numpy as np

from .ckks import Ct, Oracle, OracleError, lib, round_half_away
from .layers import OTensor, cts_per_image, divide_by_p_and_last


def product_key_id(g):
    return (1 << 32) | g


def gen_rot_mul_keys(o: Oracle, steps):
    """Beside the rotation keys, per Galois element g the key from s * sigma_g(s)."""
    from .ckks import _p
    o.gen_rot_keys(steps)
    primes = list(range(o.L + o.K))
    for r in steps:
        if r % o.slots == 0:
            continue
        g = o.galois_elt(r)
        if product_key_id(g) in o.keys:
            continue
        s, moved, target = (np.zeros((len(primes), o.N), dtype=np.uint64) for _ in range(3))
        lib().orc_secret_automorph(o._h, 1, _p(s))
        lib().orc_secret_automorph(o._h, g, _p(moved))
        o.fma_plain(target, s, moved, primes)
        key = np.zeros((o.dnum, 2, len(primes), o.N), dtype=np.uint64)
        lib().orc_gen_switch_key(o._h, product_key_id(g), _p(target), _p(key))
        o.keys[product_key_id(g)] = key


def _low(ct: Ct, l):
    return Ct(np.ascontiguousarray(ct.data[:, :l]), ct.scale)


def _products(o, a, b, l):
    """The four products a_i b_j on l limbs, as (00, 10, 01, 11)."""
    out = []
    for i, j in ((0, 0), (1, 0), (0, 1), (1, 1)):
        v = np.zeros((l, o.N), dtype=np.uint64)
        o.fma_plain(v, a[i], b[j], list(range(l)))
        out.append(v)
    return out


def whole_factor(v):
    r = round_half_away(v)
    if not math.isfinite(v) or r == 0 or abs(r - v) > 2.0 ** -16 * abs(v):
        raise OracleError("scale mismatch")
    return r


def rotated_product(o: Oracle, pairs, steps, add=None, factor=0):
    """sum over (a, b) of a rot(b, steps), + factor add, divided by q_{l-1} P at once."""
    l = min(min(a.limbs, b.limbs) for a, b in pairs)
    qs = list(range(l))
    g = o.galois_elt(steps)
    e = [np.zeros((l, o.N), dtype=np.uint64) for _ in range(4)]
    for a, b in pairs:
        moved = o.automorph_ntt(_low(b, l).data.reshape(2, l, o.N)[0], g), o.automorph_ntt(_low(b, l).data[1], g)
        for acc, v in zip(e, _products(o, _low(a, l).data, moved, l)):
            o.fma_const(acc, v, 1, qs)
    if add is not None:
        for u in (0, 1):
            o.fma_const(e[u], _low(add, l).data[u], factor, qs)
    acc = [np.zeros((l + o.K, o.N), dtype=np.uint64) for _ in range(2)]
    for d, key in ((e[2], g), (e[3], product_key_id(g))):
        for total, part in zip(acc, o.key_switch_acc(d, key)):
            o.fma_const(total, part, 1, o.ext_primes(l))
    return divide_by_p_and_last(o, acc[0], acc[1], e[:2], l, pairs[0][0].scale * pairs[0][1].scale)


def product(o: Oracle, a, b, factor_ab=1, add=None, factor=0, scale=None):
    """factor_ab a b + factor add, relinearised and divided by q_{l-1} P at once."""
    l = min(a.limbs, b.limbs)
    qs = list(range(l))
    e = _products(o, _low(a, l).data, _low(b, l).data, l)
    o.fma_const(e[1], e[2], 1, qs)
    z = []
    for v in (e[0], e[1], e[3]):
        scaled = np.zeros_like(v)
        o.fma_const(scaled, v, factor_ab, qs)
        z.append(scaled)
    if add is not None:
        for u in (0, 1):
            o.fma_const(z[u], _low(add, l).data[u], factor, qs)
    e_b, e_a = o.key_switch_acc(z[2], 0)
    return divide_by_p_and_last(o, e_b, e_a, z[:2], l, a.scale * b.scale if scale is None else scale)


def scan_steps(t: OTensor, reverse):
    return [(1 if reverse else -1) * (t.w_stride << i) for i in range((t.width - 1).bit_length())]


def recurrence_steps(o, t: OTensor, reverse=False, backward=False):
    steps = scan_steps(t, reverse != backward)
    return sorted({s % o.slots for s in steps + ([-steps[0]] if backward and steps else [])})


def _scan(o, gates, x, steps, shared):
    l = min(gates[0].limbs, x[0].limbs)
    gates = [_low(c, l) for c in gates]
    for step in steps:
        f = whole_factor(gates[0].scale)
        x = [rotated_product(o, [(gates[i // shared], c)], step, c, f) for i, c in enumerate(x)]
        gates = [rotated_product(o, [(c, c)], step) for c in gates]
    return x


def recurrence(o: Oracle, gates: OTensor, x: OTensor, reverse=False) -> OTensor:
    shared = cts_per_image(x) // cts_per_image(gates)
    return replace(x, cts=_scan(o, gates.cts, x.cts, scan_steps(x, reverse), shared), clean=1)


def recurrence_step(o: Oracle, gates: OTensor, state: OTensor, x: OTensor) -> OTensor:
    shared = cts_per_image(x) // cts_per_image(gates)
    l = min(t.cts[0].limbs for t in (gates, state, x))
    out = []
    for i, (s, c) in enumerate(zip(state.cts, x.cts)):
        a = gates.cts[i // shared]
        out.append(product(o, _low(a, l), _low(s, l), 1, c, whole_factor(a.scale * s.scale / c.scale)))
    return replace(x, cts=out, clean=int(x.clean and (gates.clean or state.clean)))


def recurrence_grad(o: Oracle, gates: OTensor, h: OTensor, grad: OTensor, reverse=False):
    shared = cts_per_image(grad) // cts_per_image(gates)
    steps = scan_steps(grad, not reverse)
    dx = _scan(o, [o.rot_left(c, steps[0]) for c in gates.cts], grad.cts, steps, shared)
    pairs = list(zip(dx, h.cts))
    dg = [rotated_product(o, pairs[i:i + shared], -steps[0]) for i in range(0, len(pairs), shared)]
    return replace(grad, cts=dx, clean=1), replace(gates, cts=dg, clean=0)


def gates_mask(o: Oracle, t: OTensor, reverse=False):
    """(coefficients [ciphertexts of an image][N], scale) of the mask that hisa_recurrence_gates multiplies by."""
    scale = float(o.primes[t.cts[0].limbs - 1])
    out = []
    for j in range(cts_per_image(t)):
        z = np.zeros(o.slots)
        for c in range(min(t.c_inner, t.channels - j * t.c_inner)):
            for y in range(t.height):
                for x in range(t.width):
                    z[t.offset + c * t.c_stride + y * t.h_stride + x * t.w_stride] = x != (t.width - 1 if reverse else 0)
        out.append(o.encode_coeffs(z, scale))
    return np.stack(out), scale


def gates_fixed(o: Oracle, t: OTensor, coeffs, scale) -> OTensor:
    per = cts_per_image(t)
    return replace(t, cts=[o.rescale(o.mul_plain(c, o.pt_from_coeffs(coeffs[i % per], scale, c.limbs))) for i, c in enumerate(t.cts)], clean=1)


def norm_sums(o: Oracle, t: OTensor):
    unit = o.slots
    for count, stride in ((t.height, t.h_stride), (t.width, t.w_stride), (t.c_inner, t.c_stride)):
        while count > 1 and stride % unit:
            unit //= 2
    sums = []
    while unit < o.slots:
        few = min(3, (o.slots // unit).bit_length() - 1)
        sums.append([k * unit for k in range(1, 1 << few)])
        unit <<= few
    return sums


def odd_cubic(a, b):
    s = a * a + a * b + b * b
    top, low = math.sqrt(s / 3.0), a * b * (a + b)
    c3 = 2.0 / (2.0 / 3.0 * s * top + low)
    return c3 * s, c3, c3 * low, 2.0 - c3 * low


def _shift(o, ct: Ct, v):
    c = np.array([int(v) % o.primes[i] for i in range(ct.limbs)], dtype=np.uint64)
    out = ct.data.copy()
    for i in range(ct.limbs):
        out[0, i] = (out[0, i] + c[i]) % np.uint64(o.primes[i])
    return Ct(out, ct.scale)


def _times(o, ct: Ct, v, scale):
    out = np.zeros_like(ct.data)
    for u in range(ct.polys):
        o.fma_const(out[u], ct.data[u], int(v), list(range(ct.limbs)))
    return Ct(out, scale)


def group_norm_fixed(o: Oracle, t: OTensor, gamma, gamma_scale, beta, groups, eps, lo, hi, iterations, act_ratio=None) -> OTensor:
    """gamma, beta: coefficients [ciphertexts of an image][N], beta's at the scale of what they are added to."""
    per_image = cts_per_image(t)
    per = per_image // groups
    n = t.channels // groups * t.height * t.width
    s = t.cts[0].scale
    outs = []
    for at in range(0, len(t.cts), per):
        group, l = t.cts[at:at + per], t.cts[0].limbs
        qs = list(range(l))
        first = Ct(np.zeros((2, l, o.N), dtype=np.uint64), s)
        second = np.zeros((3, l, o.N), dtype=np.uint64)
        for c in group:
            sq = o.mul_no_relin(c, c)
            for u in range(2):
                o.fma_const(first.data[u], c.data[u], 1, qs)
            for u in range(3):
                o.fma_const(second[u], sq.data[u], 1, qs)
        both = [first, o.relinearize(Ct(second, s * s))]
        for amounts in norm_sums(o, t):
            moved = []
            for c in both:
                acc = [np.zeros((l + o.K, o.N), dtype=np.uint64) for _ in range(2)]
                z = c.data.copy()
                for r in amounts:
                    g = o.galois_elt(r)
                    o.fma_const(z[0], o.automorph_ntt(c.data[0], g), 1, qs)
                    for total, part in zip(acc, o.key_switch_acc(o.automorph_ntt(c.data[1], g), g)):
                        o.fma_const(total, part, 1, o.ext_primes(l))
                down = Ct(np.stack([o.mod_down(v, l) for v in acc]), c.scale)
                moved.append(o.add(Ct(z, c.scale), down))
            both = moved
        mean, squares = both
        v = product(o, mean, mean, -1, squares, n)
        sv = s * s / o.primes[l - 1] * n * n * hi
        c1, c3, a, b = odd_cubic(math.sqrt(lo / hi), 1.0)
        q = o.primes[l - 2]
        kw, ky = max(1, round_half_away(s * (1.0 / 64.0) * q / sv)), max(1, round_half_away(s * c3 * q / sv))
        w, y = o.rescale(_times(o, v, kw, sv * kw)), o.rescale(_times(o, v, -ky, sv * ky))
        sw, sy = sv * kw / q, sv * ky / q / c3
        w = _shift(o, w, round_half_away(eps / hi * sw))
        y = _shift(o, y, round_half_away((c1 - c3 * (eps / hi)) * sy))
        l -= 2
        for _ in range(iterations):
            c1, c3, a, b = odd_cubic(a, b)
            s1, s2 = sw * sy / o.primes[l - 1] / c3, sy * sy / o.primes[l - 1]
            wy, yy = product(o, w, y), product(o, y, y)
            s3 = s1 * s2
            m = max(1, round_half_away(s * o.primes[l - 2] / s3))
            s3 *= m
            y = product(o, wy, yy, -m, y, whole_factor(c1 * s3 / sy))
            sy = s3 / o.primes[l - 2]
            l -= 2
        sy *= math.sqrt(hi)
        scale = s * n * gamma_scale / o.primes[l] * sy / o.primes[l - 1]
        for i, c in enumerate(group):
            j = (at + i) % per_image
            d = o.sub(_times(o, _low(c, l + 1), n, 1.0), Ct(_low(mean, l + 1).data, 1.0))
            u = o.rescale(o.mul_plain(d, o.pt_from_coeffs(gamma[j], gamma_scale, l + 1)))
            out = product(o, y, u)
            out = o.add_plain(Ct(out.data, scale), o.pt_from_coeffs(beta[j], scale, l - 1))
            if act_ratio is not None:
                out = product(o, out, out, 1, out if act_ratio else None, round_half_away(act_ratio * scale))
            outs.append(out)
    return replace(t, cts=outs, clean=1)
