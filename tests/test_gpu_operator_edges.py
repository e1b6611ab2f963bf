"""The feed-forward and update operators where inputs are at the edge of what they promise: updates that are zero,
momentum past its type's range, views with long pitches, tensors of other streams, autograd.

References are the formulas in 64 bits on the CPU; a tolerance that is not a type's own rounding is derived
where it stands.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
NS = (3.4445, -4.7750, 2.0315)
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def gs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1710_09854_amd as m

    m.lib()
    return m


def steps64(g, steps=5, coef=NS, eps=1e-7):
    x = g.detach().cpu().double()
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.transpose(-1, -2)
    for _ in range(steps):
        a = x @ x.transpose(-1, -2)
        x = coef[0] * x + (coef[1] * a + coef[2] * a @ a) @ x
    return x.transpose(-1, -2) if tall else x


def off(got, want):
    got, want = got.detach().cpu().double(), want.detach().cpu().double()
    assert got.shape == want.shape and bool(torch.isfinite(got).all())
    return float((got - want).norm() / want.norm().clamp_min(1e-300))


def normal(shape, seed, dtype=F32, k=1.0):
    return torch.from_numpy(k * np.random.default_rng(seed).standard_normal(shape)).to(dtype).cuda()


# Every way through the update: tiles read and written by vectors, along and across, and through the last pass; panels
# that read the caller's rows themselves, several and one; and those that go through the first pass, tall and not.
PATHS = [(3, 300, 264), (3, 304, 264), (3, 300, 261), (3, 261, 301), (3, 64, 576), (3, 100, 120), (3, 50, 70), (3, 50, 300), (3, 576, 64),
         (3, 120, 100)]


@pytest.mark.parametrize("eps", [0.0, 5e-324, 1e-7])
@pytest.mark.parametrize("shape", PATHS, ids=str)
def test_zero_update_stays_zero(gs, shape, eps):
    """A zero matrix has a zero result whatever is added to its norm (nothing, or a number whose reciprocal is infinite,
    included), and a step with it only decays the weights."""
    for dtype in (F32, BF16):
        g = normal(shape, 1, dtype)
        g[0], g[2] = 0, 0
        out = gs.orthogonalize(g, eps=eps)
        assert out.flags.tolist() == [gs.FLAG_ALLZERO, 0, gs.FLAG_ALLZERO]
        assert not out.o[0].any() and not out.o[2].any()
        assert off(out.o[1], steps64(g[1], eps=eps)) <= {F32: 2e-5, BF16: 5e-3}[dtype]
        w, mom = normal(shape, 2, dtype), torch.zeros(shape, device="cuda")
        copy = torch.full(shape, 7.0, dtype=F16, device="cuda")
        decayed = (w.float() * np.float32(0.95)).to(dtype)  # one product in 32 bits, rounded to the type
        flags = gs.muon_step(w, mom, g, 0.1, weight_decay=0.5, eps=eps, w_copy=copy)
        assert flags.tolist() == [gs.FLAG_ALLZERO, 0, gs.FLAG_ALLZERO]
        for k in (0, 2):
            assert torch.equal(w[k], decayed[k]) and not mom[k].any() and bool(torch.isfinite(copy[k]).all())
        assert bool(torch.isfinite(w[1]).all()) and not torch.equal(w[1], decayed[1])


@pytest.mark.parametrize("kind", ["normal", "low"])
@pytest.mark.parametrize("shape", [(64, 576), (128, 1024), (1024, 128), (100, 120), (300, 520), (777, 333), (512, 2048), (260, 4001)], ids=str)
def test_float16_results_are_rounded_once(gs, shape, kind):
    """A float16 result is off by its own rounding. Tolerance, on 2-norms: what rounding the formula's result costs, which
    over 12,000 elements and more is the same for a result within 2e-5 of it to a few per cent (a tenth is
    allowed), and the 2e-5 to which 32-bit results of rank 32 and more are held."""
    g = normal(shape, 3)
    if kind == "low":
        r = min(shape) // 8
        g = normal((shape[0], r), 4) @ normal((r, shape[1]), 5) / math.sqrt(r) + 0.1 * g
    for t in (F16, F32):
        x = g.to(t)
        want = steps64(x)
        most = 1.1 * off(want.half(), want) + 2e-5
        assert off(gs.orthogonalize(x, out_dtype=F16).o, want) <= most
    # the same for weights, where all of them is the update
    w, mom = torch.zeros(shape, dtype=F16, device="cuda"), torch.zeros(shape, device="cuda")
    gs.muon_step(w, mom, g, 1.0, beta=0.5, nesterov=False)
    want = -steps64(g)
    assert off(w, want) <= 1.1 * off(want.half(), want) + 2e-5


@pytest.mark.parametrize("shape", [(200, 300), (304, 200), (264, 520), (260, 261)], ids=str)
def test_coefficients_of_the_other_sign(gs, shape):
    """With all coefficients negated a step gives -X in place of X, through the same roundings: what is kept in fewer bits
    goes by a coefficient's size. Seen in the 32-bit copy of bfloat16 weights, whose products take the upper parts.

    Tolerance: the matrix cores' 32-bit sums may differ in their last bits when one side is negated (2 in 1000 do). Were all
    off by 2^-23, one of 2^13 roundings to 11 bits would turn by a whole place, 2^-10: 2^-10 * 2^-6.5 = 1.1e-5 of A, of B
    and of the upper parts in each of three steps, 3.3e-5 in all. A last X without its lower parts shows as 8e-5 or more
    with the first set."""
    for coef in ((4.5, -8.0, 3.0), NS):
        g, got = normal(shape, 6), []
        for sign in (1, -1):
            w, copy = torch.zeros(shape, dtype=BF16, device="cuda"), torch.zeros(shape, device="cuda")
            gs.muon_step(w, torch.zeros(shape, device="cuda"), g, sign, nesterov=False, steps=3,
                         coefficients=tuple(sign * c for c in coef), w_copy=copy)
            got.append(copy)
        assert off(got[1], got[0]) <= 4e-5, coef


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape", PATHS, ids=str)
def test_momentum_past_its_range(gs, shape, nesterov):
    """A new momentum that its type cannot hold skips the matrix's step like any overflow, and a later one that it can
    hold takes it."""
    # float16: 0.95 * 6e4 + 1e4 = 67,000, past 65,504. bfloat16: its largest number is 255/256 * 2^128, to which 1e36
    # adds more than half of the last place, 2^119 = 6.6e35.
    for mt, beta, m0, g0 in ((F16, 0.95, 6e4, 1e4), (BF16, 1.0, float(torch.finfo(BF16).max), 1e36)):
        if mt == BF16 and nesterov:
            continue  # U itself is past 32 bits then
        w, mom, g = normal(shape, 7), normal(shape, 8, mt), normal(shape, 9)
        mom[1, 3, 5], g[1, 3, 5] = m0, g0
        w0, mom0 = w.clone(), mom.clone()
        copy = torch.full(shape, 3.0, dtype=BF16, device="cuda")
        flags = gs.muon_step(w, mom, g, 0.1, beta=beta, nesterov=nesterov, w_copy=copy)
        assert flags.tolist() == [0, gs.FLAG_NONFINITE, 0]
        assert torch.equal(w[1], w0[1]) and torch.equal(mom[1], mom0[1]) and bool((copy[1] == 3.0).all())
        for k in (0, 2):
            assert not torch.equal(w[k], w0[k]) and not torch.equal(mom[k], mom0[k])
        g[1, 3, 5] = 0.0
        assert not gs.muon_step(w, mom, g, 0.1, beta=beta, nesterov=nesterov, w_copy=copy).any()
        assert bool(torch.isfinite(mom).all()) and not torch.equal(w[1], w0[1]) and torch.equal(copy, w.bfloat16())


def test_long_pitches(gs):
    """Rows on 16-byte boundaries further apart than a tile's reads of them reach: a workspace of its own is large enough
    for the copies that such operands take."""
    T, d, f, far = 33, 64, 40, 4_000_008
    x, wg, wu, dh = normal((T, d), 10, BF16), normal((f, d), 11, BF16, 0.125), normal((f, d), 12, BF16, 0.125), normal((T, f), 13, BF16)
    want = gs.gated_ff(x, wg, wu, save=True)
    ref = gs.gated_ff_backward(dh, x, wg, wu, want.saved)

    def spread(t):
        big = torch.zeros(((t.shape[0] - 1) * far + t.shape[1],), dtype=t.dtype, device="cuda")
        view = big.as_strided(t.shape, (far, 1))
        view.copy_(t)
        return view

    for a, b in ((spread(x), wg), (x, spread(wg))):
        y = gs.gated_ff(a, b, wu, save=True, workspace=gs.Workspace())
        assert torch.equal(y.h, want.h) and torch.equal(y.saved, want.saved)
        got = gs.gated_ff_backward(dh, a, b, wu, y.saved, workspace=gs.Workspace())
        assert all(torch.equal(p, q) for p, q in zip((got.dx, got.dw_gate, got.dw_up), (ref.dx, ref.dw_gate, ref.dw_up)))
