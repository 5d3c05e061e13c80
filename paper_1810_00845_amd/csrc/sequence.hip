// Layers of sequence models on CipherTensors: the gated linear recurrence h[t] = x[t] + a[t] h[t - 1] (a scan over the tokens of
// a row, one token at a time, and the backward pass) and group normalisation.  Only products and sums of ciphertexts: what
// softmax attention needs comparisons for, a recurrence does without, and its scan takes log2 T levels for T tokens.
#include <math.h>

#include <algorithm>
#include <memory>

#include "fp_device.hpp"

#define NT 256

// ---------------------------------------------------------------------------
// the inner products of a pair with its two keys
// ---------------------------------------------------------------------------
// A thread owns a coefficient of a limb and up to PAIR_CH pairs, for which the values of both keys serve once loaded.
// Bound by memory: eight pairs at N = 2^15, 21 limbs, seven digits 252 us for the 1.07 GB it cannot do without (4.2 TB/s).
#define PAIR_CH 4
__global__ __launch_bounds__(NT) void pair_inner_kernel(const FpPrime* fprimes, const double* ext, int digits, int l, int K, int L, int alpha,
                                                        const u64* key, const u64* key2, int total, const u64* pairs, const u64* plain,
                                                        const u64* pmod, u64* acc, u64 n_pairs, int log_n) {
    const u64 n = (u64)1 << log_n;
    const uint32_t j = blockIdx.x * NT + threadIdx.x;
    const int x = blockIdx.z, ext_limbs = l + K, prime = x < l ? x : L + (x - l), own = x < l ? x / alpha : -1;
    const double p = as_const(&fprimes[prime].p)[0], pinv = as_const(&fprimes[prime].p)[1];
    const u64 b0 = (u64)blockIdx.y * PAIR_CH;
    const int live = (int)(n_pairs - b0 < PAIR_CH ? n_pairs - b0 : PAIR_CH);
    double sb[PAIR_CH] = {}, sa[PAIR_CH] = {};
    for (int half = 0; half < 2; half++) {
        const double* k = (const double*)(half ? key2 : key) + (u64)prime * n + j;
        for (int d = 0; d < digits; d++) {
            const double kb = k[(u64)(2 * d) * total * n], ka = k[(u64)(2 * d + 1) * total * n];
#pragma unroll
            for (int u = 0; u < PAIR_CH; u++) {
                if (u >= live) break;
                const u64 e = (b0 + u) * 2 + half;
                const double v = d == own ? fp_from_u64(pairs[(e * l + x) * n + j]) : ext[((e * digits + d) * ext_limbs + x) * n + j];
                // at most four products within 0.875 p on a normalised value
                sb[u] += fp_mulmod(v, kb, p, pinv);
                sa[u] += fp_mulmod(v, ka, p, pinv);
                if ((d & 3) == 3 || d + 1 == digits) {
                    sb[u] = fp_norm(sb[u], p, pinv);
                    sa[u] = fp_norm(sa[u], p, pinv);
                }
            }
        }
    }
#pragma unroll
    for (int u = 0; u < PAIR_CH; u++) {
        if (u >= live) break;
        const u64 b = b0 + u;
        if (x < l) {
            const double pm = fp_from_u64(pmod[prime]);
            sb[u] += fp_mulmod(fp_from_u64(plain[((b * 2) * l + x) * n + j]), pm, p, pinv);
            sa[u] += fp_mulmod(fp_from_u64(plain[((b * 2 + 1) * l + x) * n + j]), pm, p, pinv);
        }
        acc[((b * 2) * ext_limbs + x) * n + j] = fp_canonical(sb[u], p, pinv);
        acc[((b * 2 + 1) * ext_limbs + x) * n + j] = fp_canonical(sa[u], p, pinv);
    }
}

hipError_t launch_pair_inner_fp(const FpPrime* fprimes, const double* ext, int digits, int l, int K, int L, int alpha, const u64* key,
                                const u64* key2, int total, const u64* pairs, const u64* plain, const u64* pmod, u64* acc, u64 n_pairs,
                                int log_n, hipStream_t st) {
    DRY_RUN_RETURN();
    if (!fprimes || !ext || !key || !key2 || !pairs || !plain || !pmod || !acc || digits < 1 || l < 1 || K < 1 || alpha < 1 ||
        digits != (l + alpha - 1) / alpha || n_pairs == 0 || (n_pairs + PAIR_CH - 1) / PAIR_CH > 65535)
        return hipErrorInvalidValue;
    const dim3 grid((1u << log_n) / NT, (unsigned)((n_pairs + PAIR_CH - 1) / PAIR_CH), l + K);
    ProfScope prof__("pair_inner_kernel", st);
    hipLaunchKernelGGL(pair_inner_kernel, grid, dim3(NT), 0, st, fprimes, ext, digits, l, K, L, alpha, key, key2, total, pairs, plain, pmod,
                       acc, n_pairs, log_n);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// shared by the layers
// ---------------------------------------------------------------------------
static int need_fused(hisa_ctx* ctx, const char* what) {
    if (!fused_key_switch_available(ctx)) return fail(ctx, HISA_ERR_ARG, "%s needs " FUSED_PATH, what);
    return HISA_OK;
}

// A tensor that a layer takes: one scale, and no more elements to a ciphertext than it has slots (a stride of zero passes every
// other check, whatever the extent, and masks and plans are encoded from host arrays of an entry an element).
static int check_operand(hisa_ctx* ctx, const hisa_tensor* t) {
    TRY(check_tensor(ctx, t));
    if ((double)t_ci(t) * t->height * t->width > (double)(ctx->N / 2))
        return fail(ctx, HISA_ERR_ARG, "%u x %u x %u elements do not fit %u slots", t_ci(t), t->height, t->width, ctx->N / 2);
    const double s = t->cts[0]->scale;
    if (!(s > 0.0) || !isfinite(s)) return fail(ctx, HISA_ERR_SCALE_MISMATCH, "a scale that is not a positive number");
    for (size_t i = 1; i < t_ncts(t); i++)
        if (t->cts[i]->scale != s) return fail(ctx, HISA_ERR_SCALE_MISMATCH, "ciphertexts of one tensor at different scales");
    return HISA_OK;
}

// whether the elements of a ciphertext lie in the same slots: the stride of an extent of one says nothing
static bool same_slots(const hisa_tensor& a, const hisa_tensor& b) {
    return a.height == b.height && a.width == b.width && a.offset == b.offset && t_ci(&a) == t_ci(&b) &&
           (a.height == 1 || a.h_stride == b.h_stride) && (a.width == 1 || a.w_stride == b.w_stride) && (t_ci(&a) == 1 || a.c_stride == b.c_stride);
}

// round(v), ties away from zero, as the whole number that stands for a factor.  Scales as small as the primes of a
// parameter set leave such factors 25 bits and more; one that is off by more than 2^-16 says that the scales do not fit the primes.
static int whole_factor(hisa_ctx* ctx, double v, double* out) {
    const double r = fabs(v) >= 4503599627370496.0 ? v : (v >= 0 ? floor(v + 0.5) : -floor(-v + 0.5));
    if (!isfinite(v) || fabs(v) >= 0x1p120 || r == 0.0 || fabs(r - v) > ldexp(fabs(v), -16))
        return fail(ctx, HISA_ERR_SCALE_MISMATCH, "the scales leave a factor of %g, which no whole number is near enough to", v);
    *out = r;
    return HISA_OK;
}

// a batch of ciphertexts somewhere in device memory
struct Cts {
    const u64* base;
    u64 bs;
    int limbs;         // of every polynomial
};
static Cts cts_of(const BatchIn& b, int limbs) { return {b.base, b.stride, limbs}; }
static void operand_a(ProductSide& s, const Cts& c, u64 n, unsigned div) { s.a = c.base; s.a_bs = c.bs; s.a_ps = (u64)c.limbs * n; s.a_div = div; }
static void operand_b(ProductSide& s, const Cts& c, u64 n) { s.b = c.base; s.b_bs = c.bs; s.b_ps = (u64)c.limbs * n; }
static void operand_add(ProductSide& s, const Cts& c, u64 n) { s.add = c.base; s.add_bs = c.bs; s.add_ps = (u64)c.limbs * n; }

struct Gathered {      // a tensor's ciphertexts as one strided array for the duration of a call
    hisa_ctx* ctx;
    BatchIn b;
    explicit Gathered(hisa_ctx* c) : ctx(c) {}
    ~Gathered() { dev_release(ctx, b.tmp); }
    int take(const hisa_tensor* t) { return gather_batch(ctx, (const hisa_ct* const*)t->cts, t_ncts(t), &b); }
    Gathered(const Gathered&) = delete;
};

// Calls go in parts whose extended digits stay below PART_BYTES: more entries at a time would only ask for more memory.  (Parts that fit the
// last-level cache are slower, their launches being smaller: 38 tokens at N = 2^15, 16 limbs in one part 1.02 ms, in parts of 250 MB 1.40.)
#define PART_BYTES ((size_t)1 << 30)
static size_t entries_at_once(const hisa_ctx* ctx, int l, int polys) {
    const size_t digits = ((size_t)l + ctx->alpha - 1) / ctx->alpha, one = polys * digits * (l + ctx->K) * ctx->N * sizeof(u64);
    return std::max<size_t>(1, PART_BYTES / one);
}
// fn(first, count) over parts of about equal size
template <class F>
static int in_parts(size_t entries, size_t most, F fn) {
    const size_t parts = (entries + most - 1) / most;
    for (size_t i = 0, e0 = 0; i < parts; i++) {
        const size_t cnt = (entries - e0 + (parts - i) - 1) / (parts - i);
        TRY(fn(e0, cnt));
        e0 += cnt;
    }
    return HISA_OK;
}
static ProductArgs product_base(const hisa_ctx* ctx, int l) {
    ProductArgs g = {};
    g.fprimes = ctx->d_fprimes;
    g.limbs = l; g.terms = 1;
    return g;
}
// the part [e0, e0 + cnt) of the entries of g
static ProductArgs product_part(const ProductArgs& g, size_t e0, size_t cnt) {
    ProductArgs r = g;
    auto skip = [&](ProductSide& s, size_t by, size_t terms) {
        if (terms > 1) s.a += (u64)by * terms * s.a_bs;
        else s.a_skip += (unsigned)by;
        s.b += (u64)by * terms * s.b_bs;
        if (s.add && !g.plain_period) s.add += (u64)by * s.add_bs;
    };
    if (e0 < g.n_first) {
        skip(r.s[0], e0, g.terms);
        r.n_first = (unsigned)std::min<size_t>(cnt, g.n_first - e0);
    } else {
        skip(r.s[1], e0 - g.n_first, 1);
        r.n_first = 0;
    }
    return r;
}
// products of rotated ciphertexts, or relinearised ones, with their key switches and the rescale: out [entries][2][l - 1][N]
static int rotated_products(hisa_ctx* ctx, const ProductArgs& g, size_t entries, int32_t step, u64* out) {
    return in_parts(entries, entries_at_once(ctx, g.limbs, 2), [&](size_t e0, size_t cnt) {
        return rotated_products_fp(ctx, product_part(g, e0, cnt), cnt, step, out + e0 * 2 * (g.limbs - 1) * ctx->N);
    });
}
static int relinearised_products(hisa_ctx* ctx, const ProductArgs& g, size_t entries, u64* out) {
    return in_parts(entries, entries_at_once(ctx, g.limbs, 1), [&](size_t e0, size_t cnt) {
        return products_rescale_fp(ctx, product_part(g, e0, cnt), cnt, out + e0 * 2 * (g.limbs - 1) * ctx->N);
    });
}

// ---------------------------------------------------------------------------
// gated linear recurrence
// ---------------------------------------------------------------------------
// how many ciphertexts of x share a gate; both tensors have one layout
static int check_gates(hisa_ctx* ctx, const hisa_tensor* gates, const hisa_tensor* x, unsigned* shared) {
    TRY(check_operand(ctx, gates));
    TRY(check_operand(ctx, x));
    if (gates->batch != x->batch || !same_slots(*gates, *x)) return fail(ctx, HISA_ERR_ARG, "gates and inputs have different layouts");
    if (x->channels % gates->channels || t_per(x) % t_per(gates) || x->channels / gates->channels != t_per(x) / t_per(gates))
        return fail(ctx, HISA_ERR_ARG, "%u channels do not share the gates of %u", x->channels, gates->channels);
    *shared = (unsigned)(t_per(x) / t_per(gates));
    // x's channels beside the missing ones of a part-filled gate ciphertext would have no gate
    if (*shared > 1 && gates->channels % t_ci(gates))
        return fail(ctx, HISA_ERR_ARG, "shared gates have to fill their ciphertexts: %u channels, %u to a ciphertext", gates->channels, t_ci(gates));
    if (t_ncts(x) > 16384) return fail(ctx, HISA_ERR_ARG, "%zu ciphertexts in one call", t_ncts(x));
    return HISA_OK;
}
static int check_clean(hisa_ctx* ctx, const hisa_tensor* t, const char* what) {
    if (!t->clean) return fail(ctx, HISA_ERR_ARG, "%s: slots beside the elements have to hold zeros (hisa_tensor_mask)", what);
    return HISA_OK;
}
// left rotation amounts of a scan, one per level: token t of a row meets token t - 2^i, reverse: t + 2^i
static int scan_steps(hisa_ctx* ctx, const hisa_tensor* t, bool reverse, std::vector<int32_t>& steps) {
    for (u64 s = 1; s < t->width; s <<= 1) {
        const i64 by = (i64)(s * t->w_stride);
        const int32_t step = norm_step(ctx, reverse ? by : -by);
        if (step == 0) return fail(ctx, HISA_ERR_ARG, "tokens of a row %u slots apart", t->w_stride);
        steps.push_back(step);
    }
    return HISA_OK;
}

// h = scan of x with the gates: log2 T rounds of B <- B s(A) + A rot(B), A <- A rot(A), round i over 2^i tokens.  A gate of zero at
// the first token of every row makes A zero wherever a product would reach beyond the row, so that rows, channels and the rest of
// the slots stay apart without a mask.  Both products share the rotation's keys and one set of launches.
// out: n ciphertexts [2][l - rounds][N] at *scale
static int scan_run(hisa_ctx* ctx, Cts gates, double gate_scale, Cts x, size_t n_x, unsigned shared, const std::vector<int32_t>& steps,
                    int l, u64* out) {
    const size_t n = ctx->N, n_g = n_x / shared;
    std::unique_ptr<Temp> now;
    for (size_t i = 0; i < steps.size(); i++) {
        const bool last = i + 1 == steps.size();
        const size_t entries = n_x + (last ? 0 : n_g);
        ProductArgs g = product_base(ctx, l);
        double factor;
        TRY(whole_factor(ctx, gate_scale, &factor));
        g.factor = factor;
        g.n_first = (unsigned)n_x;
        operand_a(g.s[0], gates, n, shared); operand_b(g.s[0], x, n); operand_add(g.s[0], x, n);
        operand_a(g.s[1], gates, n, 1); operand_b(g.s[1], gates, n);
        const size_t words = (size_t)2 * (l - 1) * n;
        std::unique_ptr<Temp> next(last ? nullptr : new Temp(ctx, entries * words * sizeof(u64)));
        if (next && !next->ok()) return HISA_ERR_OOM;
        u64* dst = last ? out : next->u();
        TRY(rotated_products(ctx, g, entries, steps[i], dst));
        gate_scale = gate_scale * gate_scale / (double)ctx->mod[l - 1];
        l -= 1;
        x = {dst, words, l};
        gates = {dst + n_x * words, words, l};
        now = std::move(next);
    }
    return HISA_OK;
}
// the scale of a scan's result
static double scan_scale(const hisa_ctx* ctx, double gate_scale, double x_scale, int l, size_t rounds) {
    for (size_t i = 0; i < rounds; i++, l--) {
        x_scale = gate_scale * x_scale / (double)ctx->mod[l - 1];
        gate_scale = gate_scale * gate_scale / (double)ctx->mod[l - 1];
    }
    return x_scale;
}

// handles of a result whose first use is by this call: released again unless the call succeeds
struct Outputs {
    hisa_ctx* ctx;
    std::vector<hisa_ct*> v;
    explicit Outputs(hisa_ctx* c) : ctx(c) {}
    ~Outputs() { free_handles(ctx, v); }
    int make(size_t count, int limbs, double scale) {
        v.assign(count, nullptr);
        const int rc = alloc_ct_batch(ctx, count, 2, (uint32_t)limbs, scale, v.data());
        if (rc != HISA_OK) v.clear();
        return rc;
    }
    u64* data() const { return v[0]->data; }
    void give(hisa_tensor* out, const hisa_tensor* like, uint32_t channels, uint32_t clean) {
        for (size_t i = 0; i < v.size(); i++) out->cts[i] = v[i];
        v.clear();
        fill_out_meta(out, like->batch, channels, like->height, like->width, like->h_stride, like->w_stride, like->offset, clean, t_ci(like),
                      like->c_stride);
    }
};

// the first `limbs` limbs of ciphertexts, side by side
static int copy_limbs(hisa_ctx* ctx, const Cts& c, size_t count, int limbs, u64* out) {
    if (t_analysis) return HISA_OK;
    const size_t n = ctx->N, row = (size_t)limbs * n * sizeof(u64);
    for (size_t i = 0; i < count; i++)
        HIP_TRY(ctx, hipMemcpy2DAsync(out + i * 2 * limbs * n, row, c.base + i * c.bs, (size_t)c.limbs * n * sizeof(u64), row, 2,
                                      hipMemcpyDeviceToDevice, ctx->stream));
    return HISA_OK;
}

static int recurrence(hisa_ctx* ctx, const hisa_tensor* gates, const hisa_tensor* x, bool reverse, hisa_tensor* out) {
    unsigned shared;
    TRY(check_gates(ctx, gates, x, &shared));
    if (!out || !out->cts) return fail(ctx, HISA_ERR_ARG, "bad output tensor");
    TRY(need_fused(ctx, "a recurrence"));
    TRY(check_clean(ctx, gates, "gates of a recurrence"));
    TRY(check_clean(ctx, x, "inputs of a recurrence"));
    std::vector<int32_t> steps;
    TRY(scan_steps(ctx, x, reverse, steps));
    const int lg = (int)gates->cts[0]->limbs, lx = (int)x->cts[0]->limbs, l = std::min(lg, lx), rounds = (int)steps.size();
    if (rounds && l - rounds < 1)
        return fail(ctx, HISA_ERR_DEPTH_EXHAUSTED, "a scan of %u tokens takes %d levels of %d", x->width, rounds, l - 1);
    for (int32_t s : steps) TRY(product_keys_present(ctx, s));
    const size_t n_x = t_ncts(x);
    const double sg = gates->cts[0]->scale, sx = x->cts[0]->scale;
    Gathered gg(ctx), gx(ctx);
    TRY(gg.take(gates));
    TRY(gx.take(x));
    Outputs o(ctx);
    if (!rounds) {          // one token: what comes in
        TRY(o.make(n_x, lx, sx));
        TRY(copy_limbs(ctx, cts_of(gx.b, lx), n_x, lx, o.data()));
    } else {
        TRY(o.make(n_x, l - rounds, scan_scale(ctx, sg, sx, l, rounds)));
        TRY(scan_run(ctx, cts_of(gg.b, lg), sg, cts_of(gx.b, lx), n_x, shared, steps, l, o.data()));
    }
    o.give(out, x, x->channels, 1);
    return HISA_OK;
}

extern "C" int hisa_recurrence(hisa_ctx* ctx, const hisa_tensor* gates, const hisa_tensor* x, uint32_t reverse, hisa_tensor* out) {
    return guarded(ctx, [&] { return recurrence(ctx, gates, x, reverse != 0, out); });
}

static int recurrence_step(hisa_ctx* ctx, const hisa_tensor* gates, const hisa_tensor* state, const hisa_tensor* x, hisa_tensor* out) {
    unsigned shared, same;
    TRY(check_gates(ctx, gates, x, &shared));
    TRY(check_gates(ctx, x, state, &same));
    if (same != 1) return fail(ctx, HISA_ERR_ARG, "state and inputs have different channels");
    if (!out || !out->cts) return fail(ctx, HISA_ERR_ARG, "bad output tensor");
    TRY(need_fused(ctx, "a recurrence"));
    const int lg = (int)gates->cts[0]->limbs, ls = (int)state->cts[0]->limbs, lx = (int)x->cts[0]->limbs, l = std::min(lg, std::min(ls, lx));
    if (l < 2) return fail(ctx, HISA_ERR_DEPTH_EXHAUSTED, "a token takes a level");
    if (!t_analysis && ctx->keys.find(0) == ctx->keys.end()) return fail(ctx, HISA_ERR_NO_KEY, "no relinearisation key: call hisa_keygen");
    const double sg = gates->cts[0]->scale, ss = state->cts[0]->scale, sx = x->cts[0]->scale;
    double factor;
    TRY(whole_factor(ctx, sg * ss / sx, &factor));
    const size_t n_x = t_ncts(x), n = ctx->N;
    Gathered gg(ctx), gs(ctx), gx(ctx);
    TRY(gg.take(gates));
    TRY(gs.take(state));
    TRY(gx.take(x));
    Outputs o(ctx);
    TRY(o.make(n_x, l - 1, sg * ss / (double)ctx->mod[l - 1]));
    ProductArgs g = product_base(ctx, l);
    g.n_first = (unsigned)n_x;
    g.factor = factor;
    operand_a(g.s[0], cts_of(gg.b, lg), n, shared);
    operand_b(g.s[0], cts_of(gs.b, ls), n);
    operand_add(g.s[0], cts_of(gx.b, lx), n);
    TRY(relinearised_products(ctx, g, n_x, o.data()));
    o.give(out, x, x->channels, x->clean && (gates->clean || state->clean));
    return HISA_OK;
}

extern "C" int hisa_recurrence_step(hisa_ctx* ctx, const hisa_tensor* gates, const hisa_tensor* state, const hisa_tensor* x, hisa_tensor* out) {
    return guarded(ctx, [&] { return recurrence_step(ctx, gates, state, x, out); });
}

// h[t] = x[t] + a[t] h[t - 1]:  dx[t] = g[t] + a[t + 1] dx[t + 1], a scan the other way with the gates one token on (the zero at
// the first token comes to stand behind the last one of the row before), and da[t] = dx[t] h[t - 1], summed over the ciphertexts
// that share a gate before the key switch.
static int recurrence_grad(hisa_ctx* ctx, const hisa_tensor* gates, const hisa_tensor* h, const hisa_tensor* grad, bool reverse, hisa_tensor* dx,
                           hisa_tensor* dgates) {
    unsigned shared, same;
    TRY(check_gates(ctx, gates, grad, &shared));
    TRY(check_gates(ctx, h, grad, &same));
    if (same != 1) return fail(ctx, HISA_ERR_ARG, "states and gradients have different channels");
    if (!dx || !dx->cts || !dgates || !dgates->cts || dx->cts == dgates->cts)
        return fail(ctx, HISA_ERR_ARG, "bad output tensor");
    TRY(need_fused(ctx, "a recurrence"));
    TRY(check_clean(ctx, gates, "gates of a recurrence"));
    TRY(check_clean(ctx, grad, "gradients of a recurrence"));
    if (grad->width < 2) return fail(ctx, HISA_ERR_ARG, "rows of one token have no gates to differentiate: their gradient is that of the inputs");
    std::vector<int32_t> steps;
    TRY(scan_steps(ctx, grad, !reverse, steps));
    const int32_t on = steps[0], back = norm_step(ctx, -(i64)on);       // towards the next token of the recurrence, and back
    const int lg = (int)gates->cts[0]->limbs, lh = (int)h->cts[0]->limbs, lx = (int)grad->cts[0]->limbs, l = std::min(lg, lx);
    const int rounds = (int)steps.size(), ld = l - rounds, la = std::min(ld, lh);
    if (la < 2) return fail(ctx, HISA_ERR_DEPTH_EXHAUSTED, "the backward pass over %u tokens takes %d levels of %d", grad->width, rounds + 1, l - 1);
    for (int32_t s : steps) TRY(product_keys_present(ctx, s));
    TRY(product_keys_present(ctx, back));
    const size_t n_x = t_ncts(grad), n_g = n_x / shared, n = ctx->N;
    const double sg = gates->cts[0]->scale, sx = grad->cts[0]->scale, sd = scan_scale(ctx, sg, sx, l, rounds);
    Gathered gg(ctx), gh(ctx), gx(ctx);
    TRY(gg.take(gates));
    TRY(gh.take(h));
    TRY(gx.take(grad));
    const size_t words = ct_words(ctx, 2, (uint32_t)lg);
    Temp moved(ctx, n_g * words * sizeof(u64));
    if (!moved.ok()) return HISA_ERR_OOM;
    TRY(in_parts(n_g, entries_at_once(ctx, lg, 1), [&](size_t e0, size_t cnt) {
        return rotate_fp(ctx, gg.b.base + e0 * gg.b.stride, gg.b.stride, cnt, lg, on, moved.u() + e0 * words);
    }));
    Outputs o(ctx), og(ctx);
    TRY(o.make(n_x, ld, sd));
    TRY(scan_run(ctx, {moved.u(), words, lg}, sg, cts_of(gx.b, lx), n_x, shared, steps, l, o.data()));
    TRY(og.make(n_g, la - 1, sd * h->cts[0]->scale / (double)ctx->mod[la - 1]));
    ProductArgs g = product_base(ctx, la);
    g.n_first = (unsigned)n_g; g.terms = shared;
    operand_a(g.s[0], {o.data(), ct_words(ctx, 2, (uint32_t)ld), ld}, n, 1);
    operand_b(g.s[0], cts_of(gh.b, lh), n);
    TRY(rotated_products(ctx, g, n_g, back, og.data()));
    o.give(dx, grad, grad->channels, 1);
    og.give(dgates, grad, gates->channels, 0);
    return HISA_OK;
}

extern "C" int hisa_recurrence_grad(hisa_ctx* ctx, const hisa_tensor* gates, const hisa_tensor* h, const hisa_tensor* grad, uint32_t reverse,
                                    hisa_tensor* dx, hisa_tensor* dgates) {
    return guarded(ctx, [&] { return recurrence_grad(ctx, gates, h, grad, reverse != 0, dx, dgates); });
}

extern "C" int hisa_recurrence_rot_steps(hisa_ctx* ctx, const hisa_tensor* like, uint32_t reverse, uint32_t backward, int32_t* steps, size_t cap,
                                         size_t* n) {
    if (!ctx || !like || !n) return HISA_ERR_ARG;
    return guarded(ctx, [&] {
        std::vector<int32_t> all;
        TRY(scan_steps(ctx, like, (reverse != 0) != (backward != 0), all));
        if (backward && !all.empty()) all.push_back(norm_step(ctx, -(i64)all[0]));
        return write_steps(all, steps, cap, n);
    });
}

// The gates of a row with zero at the token that has no predecessor: the masking multiply with that element left out
static int recurrence_gates(hisa_ctx* ctx, const hisa_tensor* gates, bool reverse, const int64_t* coeffs, double scale, bool fixed, hisa_tensor* out) {
    TRY(check_operand(ctx, gates));
    if (!out || !out->cts || (fixed && (!coeffs || !(scale > 0.0)))) return fail(ctx, HISA_ERR_ARG, "bad argument");
    const uint32_t l = gates->cts[0]->limbs, ci = t_ci(gates), per = (uint32_t)t_per(gates), w = gates->width;
    if (l < 2) return fail(ctx, HISA_ERR_DEPTH_EXHAUSTED, "the masking multiply needs a level to rescale into");
    Temp masks(ctx, (size_t)per * l * ctx->N * sizeof(u64));
    if (!masks.ok()) return HISA_ERR_OOM;
    if (fixed) {
        if (!t_analysis) TRY(coeffs_to_plain_batch(ctx, coeffs, per, (int)l, masks.u()));
    } else {
        scale = (double)ctx->mod[l - 1];
        const size_t hw = (size_t)gates->height * w;
        std::vector<double> ones((size_t)per * ci * hw, 0.0);
        for (uint32_t j = 0; j < per; j++)
            for (uint32_t c = 0; c < std::min(ci, gates->channels - j * ci); c++)
                for (size_t k = 0; k < hw; k++) ones[((size_t)j * ci + c) * hw + k] = k % w == (reverse ? w - 1 : 0) ? 0.0 : 1.0;
        if (!t_analysis) TRY(encode_sparse_batch(ctx, tensor_slots(gates), ones.data(), per, scale, (int)l, masks.u()));
    }
    Outputs o(ctx);
    TRY(mask_run(ctx, gates, masks.u(), scale, o.v));
    TRY(mask_finish(ctx, gates, o.v, out));
    o.v.clear();
    return HISA_OK;
}

extern "C" int hisa_recurrence_gates(hisa_ctx* ctx, const hisa_tensor* gates, uint32_t reverse, hisa_tensor* out) {
    return guarded(ctx, [&] { return recurrence_gates(ctx, gates, reverse != 0, nullptr, 0.0, false, out); });
}

extern "C" int hisa_recurrence_gates_fixed(hisa_ctx* ctx, const hisa_tensor* gates, const int64_t* mask_coeffs, double mask_scale, hisa_tensor* out) {
    return guarded(ctx, [&] { return recurrence_gates(ctx, gates, false, mask_coeffs, mask_scale, true, out); });
}

// ---------------------------------------------------------------------------
// group normalisation
// ---------------------------------------------------------------------------
// Sums over the ciphertexts of a group: out2 [groups][2][l][N] = sum x, out3 [groups][3][l][N] = sum x x before key switching.
__global__ __launch_bounds__(NT) void group_moments_kernel(const FpPrime* fprimes, const u64* x, u64 x_bs, int limbs, unsigned per, u64* out2, u64* out3,
                                                           int log_n) {
    const u64 n = (u64)1 << log_n, lw = (u64)limbs * n;
    const int limb = blockIdx.y;
    const u64 group = blockIdx.z, at = (u64)limb * n + (u64)blockIdx.x * NT + threadIdx.x;
    const double p = as_const(&fprimes[limb].p)[0], pinv = as_const(&fprimes[limb].p)[1], half = as_const(&fprimes[limb].p)[2];
    double m0 = 0.0, m1 = 0.0, s00 = 0.0, s01 = 0.0, s11 = 0.0;
    for (unsigned i = 0; i < per; i++) {
        const u64* c = x + (group * per + i) * x_bs + at;
        const double c0 = fp_centred_from_u64(c[0], p, half), c1 = fp_centred_from_u64(c[lw], p, half);
        // six of at most 0.875 p on a normalised value stay below 2^53
        m0 += c0;
        m1 += c1;
        s00 += fp_mulmod(c0, c0, p, pinv);
        s01 += fp_mulmod(c0, c1, p, pinv);
        s11 += fp_mulmod(c1, c1, p, pinv);
        if (i % 6 == 5) {
            m0 = fp_norm(m0, p, pinv); m1 = fp_norm(m1, p, pinv);
            s00 = fp_norm(s00, p, pinv); s01 = fp_norm(s01, p, pinv); s11 = fp_norm(s11, p, pinv);
        }
    }
    s01 = fp_norm(s01, p, pinv);
    out2[group * 2 * lw + at] = fp_canonical(m0, p, pinv);
    out2[group * 2 * lw + lw + at] = fp_canonical(m1, p, pinv);
    out3[group * 3 * lw + at] = fp_canonical(s00, p, pinv);
    out3[group * 3 * lw + lw + at] = fp_canonical(s01 + s01, p, pinv);
    out3[group * 3 * lw + 2 * lw + at] = fp_canonical(s11, p, pinv);
}

// k_w x + c_w q and -k_y x + c_y q side by side: the variances, polynomials [2 groups][limbs][N], on their way to two scales, with constants
// (at every evaluation point the same, of first polynomials) that the division by q leaves as c_w and c_y
__global__ __launch_bounds__(NT) void norm_times_kernel(const FpPrime* fprimes, const u64* x, u64* out, int limbs, double kw, double ky, double cw, double cy,
                                                        double last, int log_n) {
    const int limb = blockIdx.y;
    const u64 at = (((u64)blockIdx.z * limbs + limb) << log_n) + (u64)blockIdx.x * NT + threadIdx.x;
    const double p = as_const(&fprimes[limb].p)[0], pinv = as_const(&fprimes[limb].p)[1], half = as_const(&fprimes[limb].p)[2];
    const double v = fp_centred_from_u64(x[at], p, half);
    const double q = blockIdx.z & 1 ? 0.0 : fp_whole(last, p, pinv);
    const double w = fp_mulmod(v, fp_whole(kw, p, pinv), p, pinv) + fp_mulmod(q, fp_whole(cw, p, pinv), p, pinv);
    const double y = fp_mulmod(v, fp_whole(ky, p, pinv), p, pinv) + fp_mulmod(q, fp_whole(cy, p, pinv), p, pinv);
    out[at] = fp_canonical(w, p, pinv);
    out[at + (((u64)gridDim.z * limbs) << log_n)] = fp_canonical(y, p, pinv);
}

static dim3 norm_grid(const hisa_ctx* ctx, int limbs, size_t entries) { return dim3(ctx->N / NT, limbs, (unsigned)entries); }

#define HISA_MAGIC_NORMPLAN 0x4e4f524du
struct hisa_norm_plan {
    uint32_t magic;
    hisa_tensor like;            // its layout, without handles
    uint32_t limbs;
    double scale;
    hisa_norm_geom geom;
    double gamma_scale;
    DevBlock *gamma, *beta;      // [ciphertexts of an image][limbs][N]
};

// c1 z - c3 z^3 that stays nearest to one for z in [a, b] (equal and largest deviations at a, at its top and at b), and [a, b]'s image
static void odd_cubic(double& a, double& b, double* c1, double* c3) {
    const double s = a * a + a * b + b * b, top = sqrt(s / 3.0), low = a * b * (a + b);
    *c3 = 2.0 / (2.0 / 3.0 * s * top + low);
    *c1 = *c3 * s;
    a = *c3 * low;
    b = 2.0 - *c3 * low;
}

// Every whole number and scale of a normalisation, from the level and scale of its inputs.
// y ~ 1 / sqrt(v), v = (variance + eps) / hi in [lo / hi, 1]: z = y sqrt(v) starts as the odd cubic in sqrt(v), y = c1 - c3 v, and
// each iteration applies the one for its interval: y <- c1 y - c3 v y^3 as c1 y - ((c3 v) y) (y y).  c3, 1 / hi, 1 / n and sqrt(hi) are
// taken up by scales (the same residues at scale s c stand for 1 / c of what they stand for at s) and cost nothing.  Left to itself
// the scale of y would go with its third power from one iteration to the next: v is kept at a 64th of the inputs' scale, so that a
// whole factor on the product, 64 and more, brings y back to that scale within its rounding.
#define NORM_SHARE (1.0 / 64.0)
struct NormSchedule {
    double count;                // elements of a group
    double kw, ky, cw, cy;       // w = kw V / q + cw, y = cy - ky V / q
    struct Step { double y, product; };
    std::vector<Step> steps;     // an iteration: y <- (y's factor) y - (the product's) (w y) (y y)
    int level_y;                 // of 1 / sqrt
    double scale_y;
    int out_level;
    double norm_scale, act, out_scale;
};
static int norm_schedule(hisa_ctx* ctx, const hisa_norm_geom& geom, double n, int level, double s, double gamma_scale, NormSchedule* r) {
    auto q = [&](int l) { return (double)ctx->mod[l - 1]; };
    const int need = 3 + 2 * (int)geom.iterations + (geom.act ? 1 : 0);
    if (level - need < 1)
        return fail(ctx, HISA_ERR_DEPTH_EXHAUSTED, "a normalisation with %u iterations takes %d levels of %d", geom.iterations, need, level - 1);
    r->count = n;
    const double sv = s * s / q(level) * n * n * geom.var_hi;
    level -= 1;
    auto whole = [](double v) { return fabs(v) >= 4503599627370496.0 ? v : floor(v + 0.5); };
    double a = sqrt(geom.var_lo / geom.var_hi), b = 1.0, c1, c3;
    odd_cubic(a, b, &c1, &c3);
    r->kw = fmax(1.0, whole(s * NORM_SHARE * q(level) / sv));
    r->ky = fmax(1.0, whole(s * c3 * q(level) / sv));
    if (!(r->kw < 0x1p120) || !(r->ky < 0x1p120)) return fail(ctx, HISA_ERR_SCALE_MISMATCH, "a variance of %g is too small for the scale", geom.var_hi);
    const double sw = sv * r->kw / q(level);
    double sy = sv * r->ky / q(level) / c3;
    level -= 1;
    r->cw = whole(geom.eps / geom.var_hi * sw);
    r->cy = whole((c1 - c3 * (geom.eps / geom.var_hi)) * sy);
    for (uint32_t i = 0; i < geom.iterations; i++) {
        odd_cubic(a, b, &c1, &c3);
        const double s1 = sw * sy / q(level) / c3, s2 = sy * sy / q(level);
        level -= 1;
        const double s3 = s1 * s2, m = fmax(1.0, whole(s * q(level) / s3));
        // v at the inputs' scale or beyond: n^2 var_hi is too large for these primes, and y leaves their scale
        if (!(s3 * m < 2.0 * s * q(level))) return fail(ctx, HISA_ERR_SCALE_MISMATCH, "%g elements and a variance of %g are too many for the primes", n, geom.var_hi);
        double f;
        TRY(whole_factor(ctx, c1 * (s3 * m) / sy, &f));
        r->steps.push_back({f, m});
        sy = s3 * m / q(level);
        level -= 1;
    }
    sy *= sqrt(geom.var_hi);
    r->level_y = level;
    r->scale_y = sy;
    r->norm_scale = s * n * gamma_scale / q(level + 1) * sy / q(level);
    level -= 1;
    r->act = 0.0;
    r->out_scale = r->norm_scale;
    if (geom.act) {
        const double f = geom.act_ratio * r->norm_scale;
        if (geom.act_ratio != 0.0) TRY(whole_factor(ctx, f, &r->act));
        r->out_scale = r->norm_scale * r->norm_scale / q(level);
        level -= 1;
    }
    r->out_level = level;
    return HISA_OK;
}

// The sum over a ciphertext's elements in every slot that could hold one: x <- sum of rotations by u, 2u, .. over all slots, u the power of
// two that divides every stride in use (slots of other residues modulo u stay apart, and hold nothing).  Over all slots, not the window of
// the elements alone: no slot is left with part of a sum, whose variance could lie outside [lo, hi] by any amount and end beyond
// the modulus.  Up to three doublings are one sum of seven rotations of one ciphertext.
static std::vector<std::vector<int32_t>> norm_sums(const hisa_ctx* ctx, const hisa_tensor* t) {
    const u64 slots = ctx->N / 2;
    u64 unit = slots;
    const uint32_t counts[3] = {t->height, t->width, t_ci(t)}, strides[3] = {t->h_stride, t->w_stride, t->c_stride};
    for (int i = 0; i < 3; i++)
        while (counts[i] > 1 && strides[i] % unit) unit /= 2;
    std::vector<std::vector<int32_t>> sums;
    while (unit < slots) {
        int few = 1;
        while (few < 3 && (unit << (few + 1)) <= slots) few++;
        std::vector<int32_t> steps;
        for (int k = 1; k < 1 << few; k++) steps.push_back((int32_t)(k * unit));
        sums.push_back(steps);
        unit <<= few;
    }
    return sums;
}

static int check_norm(hisa_ctx* ctx, const hisa_tensor* t, const hisa_norm_geom* g) {
    TRY(check_operand(ctx, t));
    TRY(need_fused(ctx, "a normalisation"));
    TRY(check_clean(ctx, t, "inputs of a normalisation"));
    if (!g || g->groups == 0 || t->channels % g->groups || (g->groups > 1 && (t->channels / g->groups) % t_ci(t)))
        return fail(ctx, HISA_ERR_ARG, "%u channels, %u to a ciphertext: no ciphertext may hold channels of two groups", t->channels, t_ci(t));
    if (g->iterations < 1 || g->iterations > 16 || g->act > 1) return fail(ctx, HISA_ERR_ARG, "iterations 1 to 16, act 0 or 1");
    if (!(g->eps >= 0.0) || !(g->var_lo > 0.0) || !(g->var_hi > g->var_lo) || !isfinite(g->var_hi) || !(g->eps <= g->var_hi) || (g->act && !isfinite(g->act_ratio)))
        return fail(ctx, HISA_ERR_ARG, "0 <= eps, 0 < var_lo < var_hi");
    if (t_ncts(t) > 16384) return fail(ctx, HISA_ERR_ARG, "%zu ciphertexts in one call", t_ncts(t));
    return HISA_OK;
}
static double group_count(const hisa_tensor* t, const hisa_norm_geom& g) {
    return (double)(t->channels / g.groups) * (double)t->height * (double)t->width;
}

static int norm_plan_free(hisa_ctx* ctx, hisa_norm_plan* p) {
    dev_release(ctx, p->gamma);
    dev_release(ctx, p->beta);
    p->magic = 0;
    delete p;
    return HISA_OK;
}

// gamma, beta: per channel (null: one, zero), or as coefficients [ciphertexts of an image][N] (fixed)
static int norm_prepare(hisa_ctx* ctx, const hisa_tensor* like, const double* gamma, const double* beta, const int64_t* gamma_coeffs,
                        double gamma_scale, const int64_t* beta_coeffs, const hisa_norm_geom* geom, hisa_norm_plan** out) {
    if (!ctx || !out) return fail(ctx, HISA_ERR_ARG, "bad argument");
    if (t_analysis) return fail(ctx, HISA_ERR_ARG, "plans cannot be prepared during an analysis (no kernel runs)");
    TRY(check_norm(ctx, like, geom));
    const int level = (int)like->cts[0]->limbs;
    const double s = like->cts[0]->scale, n = group_count(like, *geom);
    const int level_y = level - 2 - 2 * (int)geom->iterations;
    if (level_y < 2) return fail(ctx, HISA_ERR_DEPTH_EXHAUSTED, "a normalisation with %u iterations at %d limbs", geom->iterations, level);
    // the sums are n times the scale of x: gamma at the 1 / n of the modulus that is divided by brings the scale back
    if (!gamma_coeffs) gamma_scale = (double)ctx->mod[level_y] / n;
    if (!(gamma_scale >= 1024.0) || !isfinite(gamma_scale)) return fail(ctx, HISA_ERR_SCALE_MISMATCH, "%g elements leave gamma no precision", n);
    NormSchedule full;
    TRY(norm_schedule(ctx, *geom, n, level, s, gamma_scale, &full));
    const uint32_t ci = t_ci(like), per = (uint32_t)t_per(like);
    const size_t hw = (size_t)like->height * like->width, lg = (size_t)full.level_y + 1, lb = (size_t)full.level_y;
    auto free_plan = [&](hisa_norm_plan* q) { norm_plan_free(ctx, q); };       // also where the host has no memory to encode from
    std::unique_ptr<hisa_norm_plan, decltype(free_plan)> p(
        new hisa_norm_plan{HISA_MAGIC_NORMPLAN, *like, (uint32_t)level, s, *geom, gamma_scale, nullptr, nullptr}, free_plan);
    p->like.cts = nullptr;
    auto encode = [&](const double* values, double missing, double scale, size_t limbs, u64* dst) {
        std::vector<double> v((size_t)per * ci * hw);
        for (size_t c = 0; c < (size_t)per * ci; c++) {
            const double x = c >= like->channels ? 0.0 : values ? values[c] : missing;      // beside a part-filled last ciphertext's
            if (!(fabs(x) * scale < 4.6e18)) return fail(ctx, HISA_ERR_ARG, "a factor or bias times its scale does not fit 63 bits");
            std::fill(v.begin() + c * hw, v.begin() + (c + 1) * hw, x);
        }
        return encode_sparse_batch(ctx, tensor_slots(like), v.data(), per, scale, (int)limbs, dst);
    };
    p->gamma = dev_alloc(ctx, (size_t)per * lg * ctx->N * sizeof(u64));
    p->beta = p->gamma ? dev_alloc(ctx, (size_t)per * lb * ctx->N * sizeof(u64)) : nullptr;
    if (!p->beta) return HISA_ERR_OOM;
    u64 *g = (u64*)p->gamma->ptr, *b = (u64*)p->beta->ptr;
    TRY(gamma_coeffs ? coeffs_to_plain_batch(ctx, gamma_coeffs, per, (int)lg, g) : encode(gamma, 1.0, gamma_scale, lg, g));
    TRY(beta_coeffs ? coeffs_to_plain_batch(ctx, beta_coeffs, per, (int)lb, b) : encode(beta, 0.0, full.norm_scale, lb, b));
    *out = p.release();
    return HISA_OK;
}

extern "C" int hisa_group_norm_prepare(hisa_ctx* ctx, const hisa_tensor* like, const double* gamma, const double* beta, const hisa_norm_geom* geom,
                                       hisa_norm_plan** plan) {
    return guarded(ctx, [&] { return norm_prepare(ctx, like, gamma, beta, nullptr, 0.0, nullptr, geom, plan); });
}
extern "C" int hisa_group_norm_prepare_fixed(hisa_ctx* ctx, const hisa_tensor* like, const int64_t* gamma_coeffs, double gamma_scale,
                                             const int64_t* beta_coeffs, const hisa_norm_geom* geom, hisa_norm_plan** plan) {
    if (!gamma_coeffs || !beta_coeffs) return fail(ctx, HISA_ERR_ARG, "bad argument");
    return guarded(ctx, [&] { return norm_prepare(ctx, like, nullptr, nullptr, gamma_coeffs, gamma_scale, beta_coeffs, geom, plan); });
}
extern "C" int hisa_group_norm_plan_free(hisa_ctx* ctx, hisa_norm_plan* plan) {
    if (!ctx || !plan || plan->magic != HISA_MAGIC_NORMPLAN) return fail(ctx, HISA_ERR_ARG, "not a normalisation plan");
    return norm_plan_free(ctx, plan);
}

extern "C" int hisa_group_norm_rot_steps(hisa_ctx* ctx, const hisa_tensor* in, int32_t* steps, size_t cap, size_t* n) {
    if (!ctx || !in || !n) return HISA_ERR_ARG;
    return guarded(ctx, [&] {
        std::vector<int32_t> all;
        for (const auto& s : norm_sums(ctx, in)) all.insert(all.end(), s.begin(), s.end());
        return write_steps(all, steps, cap, n);
    });
}

static int norm_apply(hisa_ctx* ctx, const hisa_tensor* in, const hisa_norm_plan* p, hisa_tensor* out) {
    if (!ctx) return HISA_ERR_ARG;
    if (!p || p->magic != HISA_MAGIC_NORMPLAN || !out || !out->cts) return fail(ctx, HISA_ERR_ARG, "bad argument");
    TRY(check_norm(ctx, in, &p->geom));
    if (in->channels != p->like.channels || !same_slots(*in, p->like))
        return fail(ctx, HISA_ERR_ARG, "the plan was prepared for another layout");
    if (in->cts[0]->limbs != p->limbs) return fail(ctx, HISA_ERR_LEVEL_MISMATCH, "the plan was prepared for %u limbs", p->limbs);
    if (fabs(in->cts[0]->scale - p->scale) > ldexp(p->scale, -30)) return fail(ctx, HISA_ERR_SCALE_MISMATCH, "the plan was prepared for scale %g", p->scale);
    const auto sums = norm_sums(ctx, in);
    if (!t_analysis) {      // every key before any work is queued
        if (ctx->keys.find(0) == ctx->keys.end()) return fail(ctx, HISA_ERR_NO_KEY, "no relinearisation key: call hisa_keygen");
        for (const auto& s : sums)
            for (int32_t a : s)
                if (ctx->keys.find(galois_of(ctx, a)) == ctx->keys.end()) return fail(ctx, HISA_ERR_NO_KEY, "no rotation key for %d slots", a);
    }
    NormSchedule r;
    TRY(norm_schedule(ctx, p->geom, group_count(in, p->geom), (int)p->limbs, p->scale, p->gamma_scale, &r));
    hipStream_t st = ctx->stream;
    const size_t n = ctx->N, cts = t_ncts(in), groups = (size_t)in->batch * p->geom.groups, images = t_per(in);
    const unsigned per = (unsigned)(cts / groups);
    const int log_n = (int)ctx->log_n;
    int l = (int)p->limbs;
    auto words = [&](int polys, int limbs) { return (size_t)polys * limbs * n; };
    Gathered gx(ctx);
    TRY(gx.take(in));
    const Cts x = cts_of(gx.b, l);
    // sums of x and of x x: over the ciphertexts, then over the slots, both at once
    Temp sum_a(ctx, 2 * groups * words(2, l) * 8), sum_b(ctx, 2 * groups * words(2, l) * 8);
    if (!sum_a.ok() || !sum_b.ok()) return HISA_ERR_OOM;
    {
        Temp squares(ctx, groups * words(3, l) * 8);
        if (!squares.ok()) return HISA_ERR_OOM;
        if (t_analysis) TALLY(mul, HISA_OP_MUL, cts, l);
        if (!t_analysis) {
            ProfScope prof__("group_moments_kernel", st);
            hipLaunchKernelGGL(group_moments_kernel, norm_grid(ctx, l, groups), dim3(NT), 0, st, ctx->d_fprimes, x.base, x.bs, l, per, sum_a.u(),
                               squares.u(), log_n);
            HIP_TRY(ctx, hipGetLastError());
        }
        TRY(in_parts(groups, entries_at_once(ctx, l, 1), [&](size_t e0, size_t cnt) {
            return relinearize_fp(ctx, squares.u() + e0 * words(3, l), cnt, l, sum_a.u() + (groups + e0) * words(2, l));
        }));
    }
    u64* from = nullptr;      // where the last sums are: in the same of the two for every part
    TRY(in_parts(2 * groups, entries_at_once(ctx, l, 1), [&](size_t e0, size_t cnt) {
        u64* part = nullptr;
        TRY(rotate_sum_chain_fp(ctx, sum_a.u() + e0 * words(2, l), sum_b.u() + e0 * words(2, l), cnt, l, sums, &part));
        if (e0 == 0) from = part;
        return HISA_OK;
    }));
    const Cts total = {from, words(2, l), l}, total2 = {from + groups * words(2, l), words(2, l), l};
    // V = n sum x^2 - (sum x)^2
    Temp v(ctx, groups * words(2, l - 1) * 8), scaled(ctx, 2 * groups * words(2, l - 1) * 8), wy(ctx, 2 * groups * words(2, l - 2) * 8);
    if (!v.ok() || !scaled.ok() || !wy.ok()) return HISA_ERR_OOM;
    {
        ProductArgs g = product_base(ctx, l);
        g.n_first = (unsigned)groups; g.scaled = 1;
        g.factor_ab = -1.0;
        g.factor = r.count;
        operand_a(g.s[0], total, n, 1); operand_b(g.s[0], total, n); operand_add(g.s[0], total2, n);
        TRY(relinearised_products(ctx, g, groups, v.u()));
        l -= 1;
    }
    if (t_analysis) TALLY(mul_scalar, HISA_OP_MUL_SCALAR, 2 * groups, l);
    if (!t_analysis) {
        ProfScope prof__("norm_times_kernel", st);
        hipLaunchKernelGGL(norm_times_kernel, norm_grid(ctx, l, 2 * groups), dim3(NT), 0, st, ctx->d_fprimes, v.u(), scaled.u(), l, r.kw, -r.ky, r.cw, r.cy,
                           (double)ctx->mod[l - 1], log_n);
        HIP_TRY(ctx, hipGetLastError());
    }
    TRY(rescale_fp(ctx, scaled.u(), 4 * groups, l, wy.u()));
    l -= 1;
    const int lw = l;
    const u64* w = wy.u();
    Temp pair(ctx, 2 * groups * words(2, l) * 8), y1(ctx, groups * words(2, l) * 8), y2(ctx, groups * words(2, l) * 8);
    if (!pair.ok() || !y1.ok() || !y2.ok()) return HISA_ERR_OOM;
    u64 *y = wy.u() + groups * words(2, lw), *y_next = y1.u(), *y_free = y2.u();
    for (const NormSchedule::Step& step : r.steps) {
        const Cts cy = {y, words(2, l), l};
        ProductArgs g = product_base(ctx, l);
        g.n_first = (unsigned)groups;
        operand_a(g.s[0], {w, words(2, lw), lw}, n, 1); operand_b(g.s[0], cy, n);
        operand_a(g.s[1], cy, n, 1); operand_b(g.s[1], cy, n);
        TRY(relinearised_products(ctx, g, 2 * groups, pair.u()));
        l -= 1;
        ProductArgs h = product_base(ctx, l);
        h.n_first = (unsigned)groups; h.scaled = 1;
        h.factor = step.y;
        h.factor_ab = -step.product;
        operand_a(h.s[0], {pair.u(), words(2, l), l}, n, 1);
        operand_b(h.s[0], {pair.u() + groups * words(2, l), words(2, l), l}, n);
        operand_add(h.s[0], cy, n);
        TRY(relinearised_products(ctx, h, groups, y_next));
        l -= 1;
        y = y_next;
        std::swap(y_next, y_free);
    }
    // (x - mean) gamma, one level above 1 / sqrt
    Temp u(ctx, cts * words(2, l) * 8);
    if (!u.ok()) return HISA_ERR_OOM;
    const CentreArgs centre = {ctx->d_fprimes, x.base, total.base, (const u64*)p->gamma->ptr, x.bs, (u64)x.limbs * n, total.bs, (u64)total.limbs * n,
                               per, (unsigned)images, l + 1, r.count};
    TRY(centred_rescale_fp(ctx, centre, cts, u.u()));
    Outputs o(ctx), mid(ctx);
    Outputs& first = p->geom.act ? mid : o;
    TRY(first.make(cts, l - 1, r.norm_scale));
    {
        ProductArgs g = product_base(ctx, l);
        g.n_first = (unsigned)cts;
        operand_a(g.s[0], {y, words(2, l), l}, n, per); operand_b(g.s[0], {u.u(), words(2, l), l}, n);
        // beta q, which the division by q leaves as beta
        g.plain_period = (unsigned)images;
        g.s[0].add = (const u64*)p->beta->ptr; g.s[0].add_bs = words(1, l);
        g.factor = (double)ctx->mod[l - 1];
        TRY(relinearised_products(ctx, g, cts, first.data()));
        l -= 1;
    }
    if (p->geom.act) {
        TRY(o.make(cts, l - 1, r.out_scale));
        const Cts c = {mid.data(), words(2, l), l};
        ProductArgs g = product_base(ctx, l);
        g.n_first = (unsigned)cts;
        operand_a(g.s[0], c, n, 1); operand_b(g.s[0], c, n);
        if (r.act != 0.0) {
            operand_add(g.s[0], c, n);
            g.factor = r.act;
        }
        TRY(relinearised_products(ctx, g, cts, o.data()));
    }
    o.give(out, in, in->channels, 1);
    return HISA_OK;
}

extern "C" int hisa_group_norm_apply(hisa_ctx* ctx, const hisa_tensor* in, const hisa_norm_plan* plan, hisa_tensor* out) {
    return guarded(ctx, [&] { return norm_apply(ctx, in, plan, out); });
}
