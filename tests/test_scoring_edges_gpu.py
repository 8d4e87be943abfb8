"""The label-scoring operators where digits, infinities, autograd's bookkeeping
and sizes at their limits decide: sums that cancel, disallowed labels, states
written in place, large batches."""
import numpy as np
import pytest

import scoringref as R
from test_scoring_gpu import S, gen, labels_of, near, normal  # noqa: F401 (S: the fixture)

pytestmark = pytest.mark.gpu

U64 = 2.0 ** -53


@pytest.mark.parametrize("P,T,V,dtype", [(16, 500, 65, "bfloat16"), (7, 511, 1000, "float32"),
                                         (3, 2001, 40, "float16"), (5, 1, 9, "float32")])
def test_preference_margins_of_near_references(S, P, T, V, dtype):
    """Sequence sums of thousands, references within a few units of them: of the
    log-probabilities (32 bits each) everything is formed in 64 bits and rounded once."""
    import torch
    g = gen(P * T)
    x = normal(g, 2 * P, T, V, dtype=dtype, scale=2.0)
    t = labels_of(g, (2 * P, T), V)
    lp = R.f64(S.label_logprob(x, t))
    L = lp.sum(1)
    ref = (torch.from_numpy(L).cuda() + 5 * normal(g, 2 * P).double()).float()
    loss, seq, margin = S.preference_loss(x, t, ref, beta=0.1)
    off = (T + 8) * U64 * np.abs(lp).sum(1)  # of a sum in 64 bits
    near(seq, L, R.U32 * np.abs(L) * 1.01 + off, "sequences")
    gain, b = L - R.f64(ref), float(np.float32(0.1))
    z = b * (gain[:P] - gain[P:])
    zoff = b * (off[:P] + off[P:]) * 1.01
    near(margin, z, R.U32 * np.abs(z) * 1.01 + zoff, "margin")
    each = np.logaddexp(0, -z)
    near(loss, np.array(each.mean()), R.U32 * each.mean() * 1.01 + zoff.max() + 16 * U64 * each.mean(),
         "loss")


@pytest.mark.parametrize("eps", [0.0, 0.1])
@pytest.mark.parametrize("beta", [0.5, 0.0])
def test_preference_of_disallowed_labels(S, eps, beta):
    """Sequences of log-probability -inf.  Pairs: fine; the preferred one
    disallowed; the other; both; the other, by the reference too; the other by the reference alone;
    fine.  A margin without a value (infinities that cancel) is NaN, and its pair has no loss and
    no weight; what the rest gives is what it gives alone."""
    import torch
    g = gen(60)
    P, T, V, inf = 7, 4, 30, np.inf
    x = normal(g, 2 * P, T, V, scale=2.0)
    t = labels_of(g, (2 * P, T), V, pad=0.0)
    ref = -10 * torch.rand(2 * P, generator=g, device="cuda")

    def disallow(s):
        x[s, 1, int(t[s, 1])] = -inf

    disallow(1)
    disallow(P + 2)
    disallow(3), disallow(P + 3)
    disallow(P + 4)
    ref[P + 4] = -inf
    ref[P + 5] = -inf
    x.requires_grad_()
    loss, seq, z = S.preference_loss(x, t, ref, beta=beta, label_smoothing=eps)
    d, = torch.autograd.grad(loss, x)
    b, e = float(np.float32(beta)), float(np.float32(eps))
    lp, p, _ = R.logprob(R.f64(x), t.cpu().numpy())
    L = lp.sum(1)
    assert np.isneginf(L[[1, 3, P + 2, P + 3, P + 4]]).all()
    near(seq, L, 1e-5 * np.where(np.isfinite(L), np.abs(L), 1), "sequences")
    fine = np.array([0, 6])
    with np.errstate(invalid="ignore"):
        gain = L - R.f64(ref)
    want = np.zeros(P)
    want[fine] = b * (gain[fine] - gain[P + fine])
    want[[1, 2, 5]] = [-inf, inf, -inf] if beta else 0.0
    want[[3, 4]] = np.nan
    near(z, want, 1e-4, "margin")
    each = np.zeros(P)
    some = ~np.isnan(want)
    each[some] = (1 - e) * np.logaddexp(0, -want[some])
    if eps:
        each[some] += e * np.logaddexp(0, want[some])
    near(loss.detach(), np.array(each.mean()), 1e-4, "loss")
    with np.errstate(over="ignore"):
        dz = np.where(some, (e - 1 / (1 + np.exp(np.where(some, want, 0)))) * b / P, 0.0)
    w = np.repeat(np.concatenate([dz, -dz]), T).reshape(2 * P, T)
    near(d, R.logprob_grad(R.f64(x), t.cpu().numpy(), w), 1e-5, "gradient")
    # without the pairs of an infinite loss
    some = torch.tensor([0, 2, 3, 4, 6], device="cuda")
    both = torch.cat([some, P + some])
    loss, _, _ = S.preference_loss(x.detach()[both], t[both], ref[both], beta=beta, label_smoothing=eps)
    near(loss, np.array(each[some.cpu().numpy()].mean()), 1e-4, "loss of some")
    # the pairs that always have a value, alone: their rows of the gradient
    keep = torch.tensor([0, 6, P, P + 6], device="cuda")
    y = x.detach()[keep].requires_grad_()
    alone, = torch.autograd.grad(S.preference_loss(y, t[keep], ref[keep], beta=beta,
                                                   label_smoothing=eps)[0], y)
    near(d[keep], R.f64(alone) * 2 / P, 1e-6, "rows of the other pairs")


def test_a_margin_of_nan_logits_is_seen(S):
    """A pair without a value is left out only where infinities cancel: NaN stays NaN."""
    import torch
    x = torch.zeros(4, 2, 5, device="cuda")
    x[1, 0, 3] = float("nan")
    t = torch.ones(4, 2, dtype=torch.int32, device="cuda")
    loss, seq, z = S.preference_loss(x, t, torch.zeros(4, device="cuda"))
    assert torch.isnan(loss) and torch.isnan(seq[1]) and torch.isnan(z[1]) and torch.isfinite(z[0])
    ref = torch.tensor([0.0, float("nan"), 0.0, 0.0], device="cuda")
    loss, _, z = S.preference_loss(torch.zeros_like(x), t, ref)
    assert torch.isnan(loss) and torch.isnan(z[1])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_logprob_is_rounded_once(S, dtype):
    """Rows whose sum of exponentials is exact: V - 1 equal logits, the label's so far below
    that its own adds nothing.  The rest, difference and logarithm, is rounded once."""
    import torch
    g = gen(61)
    for V in (2, 3, 10, 77, 1000, 4095, 50_001):
        n = 600
        top = normal(g, n, 1, dtype=dtype)
        x = top.expand(n, V).clone()
        x[:, -1] = (top[:, 0].float() - 120 - 40 * torch.rand(n, generator=g, device="cuda")).to(x.dtype)
        t = torch.full((n,), V - 1, dtype=torch.int32, device="cuda")
        X = R.f64(x)
        want = (X[:, -1] - X[:, 0]) - np.log(V - 1)
        near(S.label_logprob(x, t), want, R.U32 * np.abs(want) * (1 + 2.0 ** -20), f"{V} labels")


def test_float32_softmax_far_below_the_maximum(S):
    """Probabilities of float32 logits 12 to 85 below the row's maximum, each to its own
    digits.  The row's sum is 1 + at most 64 exp(-12): nine additions (four of a thread's elements,
    one of its vectors, four of lanes) and its inverse, one unit of 2^-24 each, what the exponentials
    below add is off by less than another; an exponential three, the product one."""
    import torch
    g = gen(62)
    n, V = 700, 64
    x = -12 - 73 * torch.rand(n, V, generator=g, device="cuda")
    at = torch.randint(0, V, (n,), generator=g, device="cuda")
    shift = normal(g, n, scale=3.0)
    x[torch.arange(n), at] = 0
    # (differences from the maximum without a rounding)
    x = torch.round((x + shift[:, None]) * 2.0 ** 16) / 2.0 ** 16
    x.requires_grad_()
    d, = torch.autograd.grad(S.label_logprob(x, at), x, torch.ones(n, device="cuda"))
    X = R.f64(x)
    want = -R.logprob(X, at.cpu().numpy())[1]
    others = np.ones((n, V), bool)
    others[np.arange(n), at.cpu().numpy()] = False
    off = np.abs(R.f64(d) / want - 1)[others]
    assert off.max() <= 15 * R.U32, f"{off.max() / R.U32:.1f} units"


def test_step_in_place_is_seen_by_autograd(S):
    """A state that a step writes while a backward pass still needs it: the pass raises, as
    after any in-place operation."""
    import torch
    g = gen(63)
    q, k, v = (normal(g, 2, 5, 2, 8).requires_grad_() for _ in range(3))
    one = [normal(g, 2, 2, 8) for _ in range(3)]
    ld = -torch.rand(2, generator=g, device="cuda")
    pool = normal(g, 4, 2, 8, 8)
    parents = torch.tensor([3, 2], dtype=torch.int32, device="cuda")
    for args, out_state in ((dict(state=pool[:2]), pool[:2]),
                            (dict(state=pool[2:].clone(), parents=parents - 2), pool[:2])):
        out, _ = S.linear_attention(q, k, v, ld, initial_state=pool[:2])
        torch.autograd.grad(out.sum(), q, retain_graph=True)
        S.linear_attention_step(*one, ld, out_state=out_state, **args)
        with pytest.raises(RuntimeError, match="inplace operation"):
            torch.autograd.grad(out.sum(), q)
    # written by a step without the caller's buffer: nothing changes under the pass
    out, _ = S.linear_attention(q, k, v, ld, initial_state=pool[:2])
    S.linear_attention_step(*one, ld, pool[:2])
    torch.autograd.grad(out.sum(), q)
    with torch.inference_mode():
        state = torch.ones(2, 2, 8, 8, device="cuda")
        o, new = S.linear_attention_step(*one, ld, state, out_state=state)
        assert new is state and torch.isfinite(o).all()


def test_step_into_a_state_that_wants_a_gradient(S):
    import torch
    from paper_1805_06383_amd.fstc import FstcError
    g = gen(64)
    one = [normal(g, 2, 2, 8) for _ in range(3)]
    ld = torch.zeros(2, device="cuda")
    state = normal(g, 2, 2, 8, 8)
    leaf = torch.zeros_like(state).requires_grad_()
    with pytest.raises(FstcError, match="gradient"):
        S.linear_attention_step(*one, ld, state, out_state=leaf)
    assert not leaf.any()
    with torch.no_grad():
        S.linear_attention_step(*one, ld, state, out_state=leaf)
    assert leaf.any()


def calls_of(S):
    """(name, function of its floating inputs, the inputs) of each operator."""
    import torch
    g = gen(65)
    t = torch.tensor([[1, 2], [3, 0]], dtype=torch.int32, device="cuda")
    ld = -torch.rand(2, generator=g, device="cuda")
    q = [normal(g, 2, 3, 2, 4) for _ in range(3)]
    one = [normal(g, 2, 2, 4) for _ in range(3)]
    s0 = normal(g, 2, 2, 4, 4)
    x = normal(g, 2, 2, 5)
    ref = normal(g, 2)
    return [("embed", lambda w: S.embed(w, t), [normal(g, 5, 4)]),
            ("linear_attention", lambda *a: S.linear_attention(*a[:4], initial_state=a[4]), [*q, ld, s0]),
            ("linear_attention_step", lambda *a: S.linear_attention_step(*a), [*one, ld, s0]),
            ("label_logprob", lambda y: S.label_logprob(y, t), [x]),
            ("preference_loss", lambda y, r: S.preference_loss(y, t, r), [x, ref])]


def test_forward_mode_derivatives_are_refused(S):
    import torch
    import torch.autograd.forward_ad as fwd
    from paper_1805_06383_amd.fstc import FstcError
    for name, f, inputs in calls_of(S):
        for i in range(len(inputs)):
            with fwd.dual_level():
                f(*inputs)  # (no tangents: as ever)
                dual = list(inputs)
                dual[i] = fwd.make_dual(inputs[i], torch.ones_like(inputs[i]))
                with pytest.raises(FstcError, match="forward-mode"):
                    f(*dual)
            if name == "linear_attention_step":
                continue
            # the tangent of what a backward pass starts from
            y = f(inputs[0].clone().requires_grad_(), *inputs[1:])
            y = y if isinstance(y, torch.Tensor) else y[0]
            with fwd.dual_level(), pytest.raises(FstcError, match="forward-mode"):
                y.backward(fwd.make_dual(torch.ones_like(y), torch.ones_like(y)))


def test_tracing_is_refused(S):
    import torch
    from paper_1805_06383_amd.fstc import FstcError
    for name, f, inputs in calls_of(S):
        with pytest.raises(FstcError, match="trace"):
            torch.jit.trace(f, tuple(inputs), check_trace=False)
        f(*inputs)


def test_tracing_by_fx_is_refused(S):
    from torch.fx.experimental.proxy_tensor import make_fx
    from paper_1805_06383_amd.fstc import FstcError
    for name, f, inputs in calls_of(S):
        with pytest.raises(FstcError, match="trace"):
            make_fx(f)(*inputs)
        f(*inputs)


def test_a_reference_that_wants_a_gradient_is_refused(S):
    import torch
    from paper_1805_06383_amd.fstc import FstcError
    x = torch.zeros(2, 3, 5, device="cuda", requires_grad=True)
    t = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    ref = torch.zeros(2, device="cuda", requires_grad=True)
    for y in (x, x.detach()):
        with pytest.raises(FstcError, match="ref_logprob"):
            S.preference_loss(y, t, ref)
    S.preference_loss(x, t, ref.detach())[0].backward()
    with torch.no_grad():
        S.preference_loss(x, t, ref)


def test_preference_loss_refuses_before_it_enqueues(S, monkeypatch):
    import torch
    from paper_1805_06383_amd.fstc import FstcError
    x = torch.zeros(2, 3, 5, device="cuda")
    t = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    ref = torch.zeros(2, device="cuda")
    called, call = [], S._call
    monkeypatch.setattr(S, "_call", lambda name, *a: (called.append(name), call(name, *a))[1])
    for eps in (0.5, -0.1, float("nan")):
        for y in (x, x.clone().requires_grad_()):
            with pytest.raises(FstcError, match="label_smoothing"):
                S.preference_loss(y, t, ref, label_smoothing=eps)
    assert not called
    S.preference_loss(x, t, ref, label_smoothing=0.49)
    assert called


def test_embed_refuses_what_its_gradient_would(S):
    """A table of 2^28 rows has a lookup but no gradient: asked for one, the lookup refuses."""
    import torch
    from paper_1805_06383_amd.fstc import FSTC_ERR_RANGE, FstcError
    w = torch.zeros(1 << 28, 1, dtype=torch.bfloat16, device="cuda")
    t = torch.tensor([0, (1 << 28) - 1], dtype=torch.int64, device="cuda")
    w[-1] = 3.0
    assert S.embed(w, t).tolist() == [[0.0], [3.0]]
    w.requires_grad_()
    with pytest.raises(FstcError, match="2\\^28") as e:
        S.embed(w, t)
    assert e.value.code == FSTC_ERR_RANGE
    with torch.no_grad():
        S.embed(w, t)


def test_step_from_no_states(S):
    """Hypotheses that all start anew, and a pool of no states."""
    import torch
    g = gen(66)
    one = [normal(g, 3, 2, 8) for _ in range(3)]
    ld = -torch.rand(2, generator=g, device="cuda")
    fresh = torch.full((3,), -1, dtype=torch.int32, device="cuda")
    out, new = S.linear_attention_step(*one, ld, torch.empty(0, 2, 8, 8, device="cuda"), parents=fresh)
    want, state = S.linear_attention_step(*one, ld, torch.ones(1, 2, 8, 8, device="cuda"), parents=fresh)
    assert torch.equal(out, want) and torch.equal(new, state)


def test_attention_of_many_short_rows(S):
    """65,536 states, padded to 256 x 256: their join, a thread an element, would be more threads
    than one launch holds.  Every batch row repeats one of four, by bits."""
    import torch
    g = gen(67)
    B, H, T, dk, dv, few = 4096, 16, 2, 130, 132, 4
    q, k = (normal(g, few, T, H, dk, dtype="bfloat16") for _ in range(2))
    v = normal(g, few, T, H, dv, dtype="bfloat16")
    ld = -torch.rand(H, generator=g, device="cuda")
    s0 = normal(g, few, H, dk, dv)
    many = [x.repeat(B // few, *[1] * (x.ndim - 1)) for x in (q, k, v)]
    s1 = s0.repeat(B // few, 1, 1, 1)
    out, final = S.linear_attention(q, k, v, ld, initial_state=s0)
    o, f = S.linear_attention(*many, ld, initial_state=s1)
    assert torch.equal(o.view(-1, *out.shape), out.expand(B // few, *out.shape))
    assert torch.equal(f.view(-1, *final.shape), final.expand(B // few, *final.shape))


HALF16 = ["bfloat16", "float16"]


@pytest.mark.parametrize("dtype", HALF16)
@pytest.mark.parametrize("B,T,dk,dv", [(1, 2, 8, 8), (3, 40, 64, 64), (1, 70, 48, 80), (2, 9, 128, 128),
                                       (600, 2, 64, 64), (2, 3, 200, 40)])
def test_attention_scores_that_cancel(S, B, T, dk, dv, dtype):
    """Scores of more than 16 digits whose values cancel: whole numbers, exact in 32-bit sums."""
    import torch
    g = gen(70 + dk)
    few = 8  # elements that are not zero: every sum stays below 2^24
    big, small = (255, 127) if dtype == "bfloat16" else (2047, 500)
    q, k = (torch.zeros(B, T, 1, dk, device="cuda") for _ in range(2))
    at = torch.randperm(dk, generator=g, device="cuda")[:few]
    q[..., at] = torch.randint(1, small, (B, T, 1, few), generator=g, device="cuda").float()
    k[..., at] = torch.randint(big // 2, big, (B, T, 1, few), generator=g, device="cuda").float()
    # position 1's key is position 0's but for one, and its value the negative
    k[:, 1] = k[:, 0]
    k[:, 1, :, at[3]] += 1
    v = torch.zeros(B, T, 1, dv, device="cuda")
    v[:, 0], v[:, 1] = 1.0, -1.0
    dt = getattr(torch, dtype)
    for x in (q, k, v):
        assert torch.equal(x, x.to(dt).float())
    out, _ = S.linear_attention(*(x.to(dt) for x in (q, k, v)), torch.zeros(1, device="cuda"))
    want = -(q[:, 1:, :, at[3]])
    assert torch.equal(want, want.to(dt).float())
    assert torch.equal(out[:, 1:].float(), want[..., None].expand(B, T - 1, 1, dv))


@pytest.mark.parametrize("dtype", HALF16)
@pytest.mark.parametrize("B,T,dk,dv", [(1, 1, 8, 8), (3, 70, 64, 64), (2, 9, 128, 128), (1, 131, 48, 80),
                                       (600, 2, 64, 64), (2, 3, 200, 40)])
def test_attention_states_that_cancel(S, B, T, dk, dv, dtype):
    """Whole numbers of 23 digits in the entering state, of which the outputs see the
    difference of two."""
    import torch
    g = gen(71 + dk)
    s0 = torch.randint(1 << 22, (1 << 23) - 256, (B, 1, dk, dv), generator=g, device="cuda").float()
    d = torch.randint(-120, 120, (B, 1, dv), generator=g, device="cuda").float()
    s0[:, :, 1] = s0[:, :, dk - 1] + d
    q = torch.zeros(B, T, 1, dk, device="cuda")
    q[..., 1], q[..., dk - 1] = 1.0, -1.0
    z = torch.zeros(B, T, 1, max(dk, dv), device="cuda")
    dt = getattr(torch, dtype)
    out, final = S.linear_attention(q.to(dt), z[..., :dk].to(dt), z[..., :dv].to(dt),
                                    torch.zeros(1, device="cuda"), initial_state=s0)
    assert torch.equal(final, s0)
    assert torch.equal(out.float(), d[:, None].expand(B, T, 1, dv))


@pytest.mark.parametrize("dtype", HALF16)
@pytest.mark.parametrize("d", [48, 64])
@pytest.mark.parametrize("T", [130, 4000])
def test_attention_decayed_values_that_cancel(S, d, T, dtype):
    """Two positions whose decayed values cancel to a thousandth, seen 69 positions and a
    chunk later.  What is rounded on the way: the decays' powers, a value's weight, the state (twice), its
    factor in the output: 16 units of 2^-24 of the terms at most."""
    import torch
    g = gen(72 + d)
    H = 48
    dt = getattr(torch, dtype)
    a = (1 + torch.rand(H, generator=g, device="cuda")).to(dt)
    b = (a.float() * 0.985).to(dt)
    ld = (torch.log(b.double() / a.double()) + 1e-3).float()
    q, k, v = (torch.zeros(1, T, H, d, device="cuda", dtype=dt) for _ in range(3))
    k[:, :2, :, 5] = 1
    q[..., 5] = 1
    v[:, 0] = a[None, :, None]
    v[:, 1] = -b[None, :, None]
    out, _ = S.linear_attention(q, k, v, ld)
    A, Bv, L = (R.f64(x) for x in (a, b, ld))
    for t in (66, 70, 127, 129):
        want = np.exp(L * t) * A - np.exp(L * (t - 1)) * Bv
        mag = np.exp(L * t) * A + np.exp(L * (t - 1)) * Bv
        bound = R.HALF[dtype] * 1.01 * np.abs(want) + 16 * R.U32 * mag + R.TINY[dtype]
        near(out[0, t], np.repeat(want[:, None], d, 1), bound[:, None], f"position {t}")


def dense(q, k, v, ld, scale, s0, n):
    """out and final state from the whole masked, decayed score matrix."""
    import torch
    T = q.shape[1]
    q, k, v = (x.transpose(1, 2) for x in (q, k, v))
    at = torch.arange(T, dtype=torch.float64, device=q.device)
    n = torch.full((q.shape[0],), T, device=q.device) if n is None else n
    n = n.double().view(-1, 1, 1, 1)
    live = (at.view(1, 1, T, 1) < n).double()
    k, v = k * live, v * live
    g = ld.view(1, -1, 1, 1)
    gap = at[:, None] - at[None, :]
    scores = q @ k.transpose(2, 3).contiguous() * (torch.exp(g * gap.clamp(min=0)) * (gap >= 0))
    reach = torch.exp(g * (at.view(1, 1, T, 1) + 1))
    out = scale * live * (scores @ v + reach * (q @ s0))
    left = torch.exp(g * (n - 1 - at.view(1, 1, T, 1)).clamp(min=0))
    return out.transpose(1, 2), (k * left).transpose(2, 3).contiguous() @ v + torch.exp(g * n) * s0


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("B,T,H,dk,dv", [(48, 70, 16, 64, 64), (48, 70, 16, 64, 128), (48, 70, 16, 48, 80),
                                         (48, 67, 16, 33, 65), (48, 70, 16, 128, 128),
                                         (40, 70, 13, 128, 64), (9, 70, 5, 200, 32), (9, 70, 5, 32, 200),
                                         (40, 70, 16, 256, 200), (9, 70, 5, 201, 33),
                                         (33, 70, 16, 100, 33), (3, 70, 5, 255, 129)])
def test_attention_of_many_rows(S, B, T, H, dk, dv, dtype):
    """More rows and heads than compute units, of every width, against the whole score matrix in 64
    bits; gradients against that form's own."""
    import torch
    g = gen(80 + dk + dv)
    q, k, v = (normal(g, B, T, H, d, dtype=dtype).requires_grad_() for d in (dk, dk, dv))
    ld = -torch.exp(torch.empty(H, device="cuda").uniform_(-7, 0, generator=g))
    s0 = normal(g, B, H, dk, dv).requires_grad_()
    n = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    n[0], n[1] = T, 0
    scale = float(np.float32(dk ** -0.5))
    out, final = S.linear_attention(q, k, v, ld, scale=scale, initial_state=s0, lengths=n)
    do, ds = normal(g, *out.shape, dtype=dtype), normal(g, *final.shape)
    got = [out, final, *torch.autograd.grad((out, final), (q, k, v, s0), (do, ds))]
    found = []
    for magnitude in (False, True):
        x = [y.detach().double() for y in (q, k, v, s0, do, ds)]
        if magnitude:
            x = [y.abs() for y in x]
        for y in x[:4]:
            y.requires_grad_()
        o, f = dense(*x[:3], ld.double(), scale, x[3], n)
        found.append([o.detach(), f.detach(), *torch.autograd.grad((o, f), x[:4], x[4:])])
    terms = (dk + dv + 2 * T + 64) * R.U32
    for name, a, w, m in zip(("out", "final", "dq", "dk", "dv", "dinit"), got, *found):
        t = str(a.dtype).replace("torch.", "")
        assert a.shape == w.shape and torch.isfinite(a).all(), name
        off = (a.double() - w).abs() - (R.HALF[t] * 1.01 * w.abs() + terms * m + R.TINY[t])
        assert off.max() <= 0, f"{name}: {float(off.max()):.3g} beyond what is allowed"


def test_calls_from_several_threads(S):
    """Calls of four threads, each on a stream of its own, give what they give alone."""
    import threading
    import torch
    g = gen(90)
    w = normal(g, 300, 64)
    ld = -torch.rand(2, generator=g, device="cuda")
    work = []
    for i in range(4):
        t = labels_of(g, (2000 + i,), 300)
        x = normal(g, 40, 1000 + i, dtype="bfloat16")
        q = normal(g, 2, 200 + i, 2, 64, dtype="bfloat16")
        go = normal(g, 2000 + i, 64)
        work.append((t, x, q, go))

    def run(t, x, q, go):
        a = w.detach().requires_grad_()
        e = S.embed(a, t)
        o, s = S.linear_attention(q, q, q, ld)
        return [e.detach(), *torch.autograd.grad(e, a, go), o, s,
                S.label_logprob(x, t[:40] % 1000), S.linear_attention_step(q[:, 0], q[:, 1], q[:, 2], ld, s)[0]]

    want = [run(*a) for a in work]
    torch.cuda.synchronize()
    found, failed = [None] * 4, []

    def body(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(10):
                    found[i] = run(*work[i])
                    with pytest.raises(Exception, match=f"\\({i + 7},"):
                        S.label_logprob(work[i][1][:, :3], torch.zeros(i + 7, dtype=torch.int32, device="cuda"))
                s.synchronize()
        except BaseException as e:  # noqa: B036 (told by the thread that waits)
            failed.append((i, repr(e)))

    threads = [threading.Thread(target=body, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    for a, b in zip(want, found):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_saved_tensors_in_another_layout(S):
    """What a backward pass has kept may come back laid out otherwise (moved to the host and back, or
    as a hook left it): the gradients are the same, by bits."""
    import contextlib
    import torch
    g = gen(68)
    wide = normal(g, 4, 3, 2000, dtype="bfloat16")
    t = labels_of(g, (4, 3), 900)
    ref = normal(g, 4)
    qkv = normal(g, 2, 70, 3, 2, 64, dtype="bfloat16")
    s0 = normal(g, 2, 2, 64, 64)
    ld = -torch.rand(2, generator=g, device="cuda")
    n = torch.tensor([70, 33], dtype=torch.int32, device="cuda")
    w = normal(g, 900, 20)

    def turned(x):
        if x.ndim >= 2:
            return x.transpose(0, -1).contiguous().transpose(0, -1)
        return torch.stack([x, x], -1)[..., 0] if x.ndim else x

    def grads():
        x = wide[:, :, 7:907].detach().requires_grad_()
        q, k, v = (y.detach().requires_grad_() for y in qkv.unbind(2))
        i = s0.detach().requires_grad_()
        a = w.detach().requires_grad_()
        o, f = S.linear_attention(q, k, v, ld, initial_state=i, lengths=n)
        return [lambda: torch.autograd.grad(S.label_logprob(x, t).sum(), x),
                lambda: torch.autograd.grad(S.preference_loss(x, t, ref)[0], x),
                lambda: torch.autograd.grad(o.float().sum() + f.sum(), (q, k, v, i)),
                lambda: torch.autograd.grad(S.embed(a, t).square().sum(), a)]

    found = []
    for hooks in (contextlib.nullcontext(), torch.autograd.graph.save_on_cpu(),
                  torch.autograd.graph.saved_tensors_hooks(lambda x: x, turned)):
        with hooks:
            found.append([y for f in grads() for y in f()])
    for other in found[1:]:
        for a, b in zip(found[0], other):
            assert torch.equal(a, b)
