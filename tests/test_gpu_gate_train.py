"""The calls that train a gate, through the C ABI, against oracle/gate_train_oracle.py (64 bits).

Tolerances follow from the arithmetic the header promises: fp32 tables and sums, u = 2^-24 the half step of fp32.
  probabilities   exp of a rounded difference of size r is off by r u + 2 u, the sum over E <= 256 experts of positive
                  terms by at most 16 u (4 in a row, then pairs) and the quotient by u: (r + 24) u, relative, r = the
                  spread of a row's scores
  sums over T     of positive terms: T / 512 + 64 additions in a row at most
  gradients       p (g - sum p g): each factor by the above and the inner sum once more, on the sum of sizes
  matrix sums     n terms: (n + 8) * 2 u of the sum of sizes (matrix instructions add in no documented order; a factor
                  of 2 covers additions that cut instead of rounding)
"""
import numpy as np
import pytest

import synth_inputs as si
from oracle import gate_train_oracle as go
from oracle import moe_oracle as orc

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

from paper_2603_06350_amd import binding as B  # noqa: E402
from paper_2603_06350_amd import layer  # noqa: E402

U = 2.0 ** -24
TINY = 1e-37          # below it fp32 results may be flushed
PAD = 64              # guard elements around outputs


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load()


class Guarded:
    """An output between guard elements: what the call must not touch."""

    def __init__(self, shape, dtype=torch.float32, fill=-77.0):
        n = int(np.prod(shape))
        self.all = torch.full((n + 2 * PAD,), fill, dtype=dtype, device="cuda")
        self.t = self.all[PAD:PAD + n].view(shape)
        self.fill = fill

    def np(self):
        torch.cuda.synchronize()
        a = self.all.float().cpu().numpy() if self.all.dtype == torch.bfloat16 else self.all.cpu().numpy()
        n = self.t.numel()
        assert (a[:PAD] == self.fill).all() and (a[PAD + n:] == self.fill).all(), "written outside the output"
        return a[PAD:PAD + n].reshape(tuple(self.t.shape)).astype(np.float64)


def mask_of(kind, T, seed):
    if kind == "none":
        return None
    m = np.zeros(T, dtype=np.uint8)
    if kind == "some":
        m[:] = np.random.default_rng([seed, 9]).random(T) < 0.6
    elif kind == "one":
        m[T // 2] = 1
    elif kind == "odd_bytes":                       # any byte but 0 counts
        m[::2] = 200
    return m                                        # "nothing": all zero


def poison(a, mask, value=np.nan):
    if mask is None:
        return a
    a = a.copy()
    a[mask == 0] = value
    return a


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def workspace(sh):
    nb = B.moe_train_workspace_bytes(sh)
    return torch.full((nb,), 0x5A, dtype=torch.uint8, device="cuda"), nb


def shape_of(T, E, k, renorm=0, d=8, dtype=B.MOE_BF16):
    return B.make_shape(T, d, E, k, 8, dtype, renorm)


def tables(T, E, k, seed, mask=None, spread=1.0):
    rng = np.random.default_rng([seed, T, E, k])
    scores = (spread * rng.standard_normal((T, E))).astype(np.float32)
    idx = orc.topk_select(scores, k) if T else np.zeros((0, k), dtype=np.int32)
    return rng, scores, idx


def spread_of(*tables_):
    return max([float(np.abs(t[np.isfinite(t)]).max()) * 2 if np.isfinite(t).any() else 0.0 for t in tables_])


def p_tol(scores, E):
    return (spread_of(scores) + 24) * U


SIZES = [(1, 1, 1), (1, 8, 2), (2, 3, 3), (5, 2, 1), (63, 7, 3), (64, 8, 2), (65, 12, 3), (100, 16, 2), (257, 17, 5),
         (300, 40, 6), (501, 64, 6), (333, 65, 2), (250, 100, 7), (129, 128, 8), (130, 129, 64), (77, 200, 3), (200, 255, 8),
         (1000, 256, 64), (4999, 24, 1), (9001, 8, 2), (20011, 12, 3), (5003, 256, 8)]


def check_balance(T, E, k, mask, scores, idx, sh=None, stream=None):
    sh = sh or shape_of(T, E, k)
    ws, nb = workspace(sh)
    counts, prob_sum, loss = Guarded((E,), torch.int32, -77), Guarded((E,)), Guarded((1,))
    B.moe_balance_loss(sh, dev(poison(scores, mask)), dev(poison(idx, mask, -5)), dev(mask), counts.t, prob_sum.t, loss.t, ws, nb, stream)
    rc, rp, rl = go.balance_loss(scores, idx, mask)
    got_c, got_p, got_l = counts.np(), prob_sum.np(), loss.np()[0]
    assert np.array_equal(got_c, rc)
    tol = p_tol(scores, E) + (T / 512 + 64) * U
    assert (np.abs(got_p - rp) <= tol * rp + TINY).all(), np.abs(got_p - rp).max()
    assert abs(got_l - rl) <= (tol + 2 * U) * abs(rl)


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("mask", ["none", "some"])
def test_balance_loss(T, E, k, mask):
    _, scores, idx = tables(T, E, k, 1)
    check_balance(T, E, k, mask_of(mask, T, 1), scores, idx)


@pytest.mark.parametrize("mask", ["nothing", "one", "odd_bytes"])
def test_balance_loss_of_masks_that_leave_little(mask):
    _, scores, idx = tables(301, 24, 3, 2)
    check_balance(301, 24, 3, mask_of(mask, 301, 2), scores, idx)


def route_bound(scores, idx, dw, counts, coef, renorm, mask, k):
    """Sum of the sizes of what a gradient element adds up, times the relative error of its parts."""
    T, E = scores.shape
    p = go.softmax(scores)
    size = np.zeros((T, E))
    g = np.zeros((T, E))
    if counts is not None and counts.sum() > 0:
        g += abs(coef) * E * k * counts[None, :] / float(counts.sum()) ** 2
    if dw is not None:
        w = go.routing_weights(scores, idx, renorm)
        for j in range(idx.shape[1]):
            ok = np.flatnonzero((idx[:, j] >= 0) & (idx[:, j] < E))
            if renorm:
                size[ok, idx[ok, j]] += (w[:, j] * (np.abs(dw[:, j]) + (w * np.abs(dw)).sum(axis=1)))[ok]
            else:
                g[ok, idx[ok, j]] += np.abs(dw[ok, j])
    size += p * (g + (p * g).sum(axis=1, keepdims=True))
    tol = (2 * (spread_of(scores) + 24) + 24 + k) * U * size + TINY
    if mask is not None:
        tol[mask == 0] = 0.0
    return tol


def check_route_backward(T, E, k, renorm, mask, scores, idx, dw, counts, coef, accumulate):
    sh = shape_of(T, E, k, renorm)
    out = Guarded((T, E))
    before = np.zeros((T, E))
    if accumulate:
        before = np.random.default_rng(3).standard_normal((T, E)).astype(np.float32)
        out.t.copy_(torch.from_numpy(before))
        before = before.astype(np.float64)
    B.moe_route_backward(sh, dev(poison(scores, mask)), dev(poison(idx, mask, 2 ** 30)) if dw is not None else None,
                         None if dw is None else dev(poison(dw, mask)), None if counts is None else dev(counts.astype(np.int32)),
                         coef, dev(mask), out.t, accumulate)
    ref = go.route_backward(scores, idx, dw, counts, coef, renorm, mask, k)
    tol = route_bound(scores, idx, dw, None if counts is None else counts.astype(np.float64), coef, renorm, mask, k)
    tol = tol + (U * np.abs(before + ref) if accumulate else 0.0)
    got = out.np()
    assert (np.abs(got - (before + ref)) <= tol).all(), np.abs(got - before - ref).max()


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("renorm", [0, 1])
def test_route_backward(T, E, k, renorm):
    rng, scores, idx = tables(T, E, k, 4)
    dw = rng.standard_normal((T, k)).astype(np.float32)
    counts = go.balance_loss(scores, idx)[0]
    check_route_backward(T, E, k, renorm, None, scores, idx, dw, counts, 0.5 * T, 0)
    mask = mask_of("some", T, 4)
    check_route_backward(T, E, k, renorm, mask, scores, idx, dw, None, 0.0, 1)
    check_route_backward(T, E, k, renorm, mask, scores, idx, None, counts, 0.5 * T, 0)


def test_route_backward_of_odd_choices():
    """The same expert twice, indices that name no expert, experts that are not the best, no load, nothing masked in."""
    rng, scores, _ = tables(97, 16, 4, 5)
    dw = rng.standard_normal((97, 4)).astype(np.float32)
    idx = rng.integers(0, 16, (97, 4)).astype(np.int32)
    idx[::3, 1] = idx[::3, 0]
    idx[5] = [-1, 16, 2 ** 31 - 1, -2 ** 31]
    idx[6, 2] = -1
    for renorm in (0, 1):
        check_route_backward(97, 16, 4, renorm, None, scores, idx, dw, None, 0.0, 0)
        check_route_backward(97, 16, 4, renorm, mask_of("nothing", 97, 0), scores, idx, dw, None, 0.0, 0)
        check_route_backward(97, 16, 4, renorm, mask_of("one", 97, 0), scores, idx, dw, np.zeros(16, dtype=np.int64), 1.0, 1)
    check_balance(97, 16, 4, None, scores, idx)
    # counts of a whole job: sums far above this GPU's own
    check_route_backward(97, 16, 4, 0, None, scores, idx, None, np.arange(16, dtype=np.int64) * 100000000, 1e9, 0)


@pytest.mark.parametrize("E", [1, 8, 60, 256])
def test_even_loads_have_no_balance_gradient(E):
    _, scores, _ = tables(300, E, 1, 7, spread=3.0)
    out = Guarded((300, E))
    B.moe_route_backward(shape_of(300, E, 1), dev(scores), None, None, torch.full((E,), 12345, dtype=torch.int32, device="cuda"), 1e4, None, out.t)
    assert not out.np().any()


@pytest.mark.parametrize("E,k,renorm", [(1, 1, 0), (1, 1, 1), (8, 1, 1), (64, 1, 1), (250, 1, 1)])
def test_weights_that_are_always_one_have_no_gradient(E, k, renorm):
    rng, scores, idx = tables(500, E, k, 8, spread=5.0)
    out = Guarded((500, E))
    dw = dev(rng.standard_normal((500, k)).astype(np.float32))
    B.moe_route_backward(shape_of(500, E, k, renorm), dev(scores), dev(idx), dw, None, 0.0, None, out.t)
    assert not out.np().any()


@pytest.mark.parametrize("E", [1, 7, 64, 256])
def test_one_expert_left_is_no_loss(E):
    """Every token has one expert that is not switched off, the same in both gates: probabilities of exactly 1."""
    rng = np.random.default_rng([9, E])
    only = rng.integers(0, E, 400)
    scores, target = (np.full((400, E), -np.inf, dtype=np.float32) for _ in range(2))
    scores[np.arange(400), only] = 7 * rng.standard_normal(400)
    target[np.arange(400), only] = 7 * rng.standard_normal(400)
    sh = shape_of(400, E, 1)
    ws, nb = workspace(sh)
    loss, out = Guarded((1,)), Guarded((400, E))
    B.moe_gate_distill(sh, dev(scores), dev(target), None, 1.0, loss.t, out.t, 0, ws, nb)
    assert loss.np()[0] == 0.0 and not out.np().any()


@pytest.mark.parametrize("E,k", [(9, 3), (13, 4), (16, 4), (36, 9), (50, 16), (100, 7), (250, 64)])
@pytest.mark.parametrize("renorm", [0, 1])
def test_route_backward_of_a_few_odd_choices(E, k, renorm):
    """Tokens that list an expert twice or three times among tokens that do not, and indices just behind the last expert."""
    T = 700
    rng, scores, idx = tables(T, E, k, 6)
    dw = rng.standard_normal((T, k)).astype(np.float32)
    idx[100, 1] = idx[100, 0]
    idx[300:303, :3] = idx[300:303, :1]
    idx[500] = idx[500, 0]
    idx[200, 0], idx[201, k - 1], idx[202] = E, E + 1, E
    check_route_backward(T, E, k, renorm, None, scores, idx, dw, go.balance_loss(scores, idx)[0], 0.5 * T, 0)
    check_route_backward(T, E, k, renorm, mask_of("some", T, 5), scores, idx, dw, None, 0.0, 1)
    dw[200, 0] = dw[201, k - 1] = dw[202, 0] = np.nan  # the weights of nobody
    out = Guarded((T, E))
    B.moe_route_backward(shape_of(T, E, k, renorm), dev(scores), dev(idx), dev(dw), None, 0.0, None, out.t)
    assert np.isfinite(out.np()).all()


def check_distill(T, E, mask, scores, target, coef, accumulate, with_grad=True):
    sh = shape_of(T, E, 1)
    ws, nb = workspace(sh)
    out, loss = Guarded((T, E)), Guarded((1,))
    before = np.zeros((T, E))
    if accumulate:
        before = np.random.default_rng(6).standard_normal((T, E)).astype(np.float32)
        out.t.copy_(torch.from_numpy(before))
        before = before.astype(np.float64)
    B.moe_gate_distill(sh, dev(poison(scores, mask)), dev(poison(target, mask, np.inf)), dev(mask), coef, loss.t,
                       out.t if with_grad else None, accumulate, ws, nb)
    rl, rg = go.gate_distill(scores, target, coef, mask)
    rows = np.arange(T) if mask is None else np.flatnonzero(mask)
    n = max(1, rows.size)
    p, q = go.softmax(scores), go.softmax(target)
    r = spread_of(scores, target)
    got = out.np()
    if with_grad:
        tol = (r + 28) * U * abs(coef) / n * (p + q) + TINY
        if mask is not None:
            tol[mask == 0] = 0.0
        tol = tol + (U * np.abs(before + rg) if accumulate else 0.0)
        assert (np.abs(got - (before + rg)) <= tol).all(), np.abs(got - before - rg).max()
    else:
        assert (got == -77.0).all()
    # a row: terms q (log q - log p) of sizes q (|log q| + |log p|), each log and the sum off by (r + 24) u
    fin = np.isfinite(scores) & np.isfinite(target)
    size = (q * (2 * r + 32) * np.where(fin, 1.0, 0.0)).sum(axis=1)[rows].sum() / n * (r + 32) * U
    if np.isinf(rl):
        assert np.isinf(loss.np()[0])
    else:
        assert abs(loss.np()[0] - rl) <= size + 2 * U * abs(rl), (loss.np()[0], rl)


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("mask", ["none", "some"])
def test_gate_distill(T, E, k, mask):
    rng, scores, _ = tables(T, E, k, 7)
    target = (scores + 0.5 * rng.standard_normal((T, E))).astype(np.float32)
    check_distill(T, E, mask_of(mask, T, 7), scores, target, 1.0, 0)
    check_distill(T, E, mask_of(mask, T, 7), scores, target, -3.0 * T, 1)


@pytest.mark.parametrize("mask", ["nothing", "one", "odd_bytes"])
def test_gate_distill_of_masks_that_leave_little(mask):
    rng, scores, _ = tables(301, 24, 3, 8)
    target = rng.standard_normal((301, 24)).astype(np.float32)
    check_distill(301, 24, mask_of(mask, 301, 8), scores, target, 2.0, 0)
    check_distill(301, 24, mask_of(mask, 301, 8), scores, target, 2.0, 0, with_grad=False)


@pytest.mark.parametrize("E", [5, 16, 64, 100, 256])
def test_switched_off_experts_and_empty_rows(E):
    """Scores of -inf and of the type's lowest value; rows in which nothing is left; a target that switches off more."""
    T, k = 75, 2
    rng, scores, _ = tables(T, E, k, 9)
    off = rng.random((T, E)) < 0.4
    off[:, 0] = False
    scores[off] = -np.inf
    idx = np.zeros((T, k), dtype=np.int32)
    idx[:, 1] = 1 % E
    target = scores.copy()
    target[:, 1:][rng.random((T, E - 1)) < 0.3] = -np.inf
    scores[7] = -np.inf
    target[9] = -np.inf
    scores[11, ~off[11]] = -np.finfo(np.float32).max          # all alike: 1 / n each
    target[11, ~off[11]] = -np.finfo(np.float32).max
    dw = rng.standard_normal((T, k)).astype(np.float32)
    with np.errstate(invalid="ignore"):
        low = np.where(np.abs(scores) > 1e30, 0.0, scores).astype(np.float32)      # for the spread in the bounds
    ws, nb = workspace(shape_of(T, E, k))
    counts, prob_sum, loss = Guarded((E,), torch.int32, -77), Guarded((E,)), Guarded((1,))
    B.moe_balance_loss(shape_of(T, E, k), dev(scores), dev(idx), None, counts.t, prob_sum.t, loss.t, ws, nb)
    rc, rp, rl = go.balance_loss(scores, idx)
    tol = p_tol(low, E) + 72 * U
    assert np.array_equal(counts.np(), rc) and (np.abs(prob_sum.np() - rp) <= tol * rp + TINY).all()
    for renorm in (0, 1):
        out = Guarded((T, E))
        B.moe_route_backward(shape_of(T, E, k, renorm), dev(scores), dev(idx), dev(dw), dev(rc.astype(np.int32)), 1.0, None, out.t, 0)
        ref = go.route_backward(scores, idx, dw, rc, 1.0, renorm)
        assert np.isfinite(out.np()).all() and not out.np()[7].any()
        assert np.abs(out.np() - ref).max() <= 200 * U * (np.abs(dw).max() + E * k * rc.max() / rc.sum() ** 2)
    out, loss = Guarded((T, E)), Guarded((1,))
    B.moe_gate_distill(shape_of(T, E, k), dev(scores), dev(target), None, 1.0, loss.t, out.t, 0, ws, nb)
    rl, rg = go.gate_distill(scores, target)
    assert not out.np()[7].any() and not out.np()[9].any()
    assert np.abs(out.np() - rg).max() <= 100 * U / T
    assert abs(loss.np()[0] - rl) <= (2 * spread_of(low) + 32) ** 2 * U
    # the other way round a target wants what the scores cannot give
    if E > 1 and (np.isfinite(scores) & ~np.isfinite(target)).any():
        B.moe_gate_distill(shape_of(T, E, k), dev(target), dev(scores), None, 1.0, loss.t, None, 0, ws, nb)
        assert np.isinf(loss.np()[0])


@pytest.mark.parametrize("E", [8, 64, 200])
def test_scores_far_apart(E):
    """Probabilities from 1 down to below the smallest fp32 number."""
    T, k = 130, min(E, 4)
    rng, scores, idx = tables(T, E, k, 10, spread=40.0)
    check_balance(T, E, k, None, scores, idx)
    dw = rng.standard_normal((T, k)).astype(np.float32)
    for renorm in (0, 1):
        check_route_backward(T, E, k, renorm, None, scores, idx, dw, None, 0.0, 0)
    target = (40.0 * rng.standard_normal((T, E))).astype(np.float32)
    check_distill(T, E, None, scores, target, 1.0, 0)


# ------------------------------------------------------------------------------------------------ the gate product
def store(a, dtype):
    return a.astype(np.float32) if dtype == B.MOE_F32 else si.f32_to_bf16_bits(a.astype(np.float32))


def check_gate(T, d, E, dtype, mask, seed, accumulate=0, parts="wbx", stream=None, scale=1.0, tokens=None):
    """tokens: the only ones with a gradient; the sums over tokens then have that many terms, whatever T is."""
    rng = np.random.default_rng([seed, T, d, E])
    x, w = store(rng.standard_normal((T, d)), dtype), store(rng.standard_normal((E, d)) / np.sqrt(d), dtype)
    ds = (scale * rng.standard_normal((T, E)) * 10.0 ** rng.integers(-3, 1, (T, 1))).astype(np.float32)
    if tokens is not None:
        keep = np.zeros(T, dtype=bool)
        keep[tokens] = True
        ds[~keep] = 0.0
    nan = np.float32(np.nan) if dtype == B.MOE_F32 else np.uint16(0x7FC0)
    sh = shape_of(T, E, 1, 0, d, dtype)
    ws, nb = workspace(sh)
    xt = torch.float32 if dtype == B.MOE_F32 else torch.bfloat16
    dw, db, dx = Guarded((E, d)), Guarded((E,)), Guarded((T, d), xt, -77.0)
    old = [np.full(o.t.shape, 0.0) for o in (dw, db, dx)]
    for i, (o, flag, part) in enumerate(((dw, 1, "w"), (db, 1, "b"), (dx, 2, "x"))):
        if accumulate & flag and part in parts:
            o.t.copy_(torch.from_numpy(rng.standard_normal(tuple(o.t.shape)).astype(np.float32)))
            old[i] = o.t.double().cpu().numpy()
    B.moe_gate_backward(sh, layer.to_device(poison(x, mask, nan)) if "w" in parts else None,
                        layer.to_device(w) if "x" in parts else None, dev(poison(ds, mask)), dev(mask),
                        dw.t if "w" in parts else None, db.t if "b" in parts else None, dx.t if "x" in parts else None,
                        accumulate, ws, nb, stream)
    x64, w64 = orc.to_f64(x), orc.to_f64(w)
    rw, rb, rx = go.gate_backward(x64, w64, ds, mask)
    rw_size, rb_size, rx_size = go.gate_backward(np.abs(x64), np.abs(w64), np.abs(ds), mask)
    n = T if mask is None else int((mask != 0).sum())
    n = n if tokens is None else len(tokens)
    where = f"T={T} d={d} E={E} dtype={dtype} accumulate={accumulate}"
    if "w" in parts:
        err, tol = np.abs(dw.np() - old[0] - rw), (n + 8) * 2 * U * rw_size + 2 * U * np.abs(old[0] + rw)
        assert (err <= tol).all(), f"{where}: d_w_gate {err.max():.3e}, {(err - tol).max():.3e} over"
    else:
        assert (dw.np() == -77.0).all()
    if "b" in parts:
        err, tol = np.abs(db.np() - old[1] - rb), (n + 8) * 2 * U * rb_size + 2 * U * np.abs(old[1] + rb)
        assert (err <= tol).all(), f"{where}: d_gate_bias {err.max():.3e}"
    else:
        assert (db.np() == -77.0).all()
    if "x" in parts:
        # one rounding to storage; bf16 layers may multiply d_scores in two bf16 pieces (16 bits of it)
        half = U if dtype == B.MOE_F32 else 2.0 ** -8
        piece = 0.0 if dtype == B.MOE_F32 else 2.0 ** -16
        err = np.abs(dx.np() - old[2] - rx)
        tol = half * np.abs(old[2] + rx) + (1 + half) * ((E + 8) * 2 * U + piece) * rx_size + 2 * U * np.abs(old[2])
        assert (err <= tol).all(), f"{where}: d_x {err.max():.3e}, {(err - tol).max():.3e} over"
    else:
        assert (dx.np() == -77.0).all()


GATES = [(1, 8, 1), (1, 64, 8), (2, 16, 3), (3, 136, 16), (15, 120, 7), (16, 128, 8), (17, 8, 256), (31, 264, 17), (33, 72, 31),
         (64, 128, 8), (65, 1048, 12), (100, 520, 33), (127, 256, 64), (129, 512, 65), (200, 2048, 64), (255, 384, 100),
         (257, 1024, 128), (300, 200, 129), (500, 4096, 8), (511, 640, 255), (513, 1000, 256), (1000, 5120, 16), (2049, 1048, 24),
         (5000, 64, 40), (8191, 136, 12)]


@pytest.mark.parametrize("T,d,E", GATES)
@pytest.mark.parametrize("dtype", [B.MOE_BF16, B.MOE_F32])
def test_gate_backward(T, d, E, dtype):
    check_gate(T, d, E, dtype, None, 11)
    check_gate(T, d, E, dtype, mask_of("some", T, 11), 12, accumulate=3)


@pytest.mark.parametrize("T,d,E,dtype", [(70001, 520, 8, 0), (70001, 264, 24, 1), (70001, 1048, 50, 1), (40001, 520, 64, 0), (33001, 1048, 65, 1),
                                         (8200, 1048, 200, 1), (8201, 1048, 130, 0), (9001, 4096, 128, 1)])
def test_gate_backward_of_large_batches(T, d, E, dtype):
    """Blocks of 64 experts, several steps of a block, several parts; 60 tokens with a gradient, ends and edges among them."""
    rng = np.random.default_rng([T, E])
    tokens = np.unique(np.concatenate([[0, 1, 31, 32, 63, 64, 127, 128, T - 1, T - 2, T - 33, T - 64], rng.integers(0, T, 48)]))
    check_gate(T, d, E, dtype, None, 16, tokens=tokens)
    check_gate(T, d, E, dtype, mask_of("some", T, 16), 17, accumulate=3, tokens=tokens)


@pytest.mark.parametrize("T,E", [(0, 8), (7, 8), (40, 24), (700, 64), (70, 256)])
@pytest.mark.parametrize("dtype", [B.MOE_BF16, B.MOE_F32])
def test_gate_backward_parts_and_masks(T, E, dtype):
    d = 4 * 33 if dtype == B.MOE_F32 else 8 * 33      # rows that are odd multiples of 16 bytes
    for mask in ("nothing", "one", "odd_bytes"):
        m = mask_of(mask, T, 13) if T else None
        check_gate(T, d, E, dtype, m, 13)
        check_gate(T, d, E, dtype, m, 13, accumulate=1)
    for parts in ("w", "b", "x", "wb", "bx", "wx"):
        check_gate(T, d, E, dtype, None, 14, parts=parts, accumulate=2)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e25])
@pytest.mark.parametrize("dtype", [B.MOE_BF16, B.MOE_F32])
def test_gate_backward_of_gradients_of_any_size(scale, dtype):
    check_gate(77, 136, 20, dtype, None, 15, scale=scale)


# ------------------------------------------------------------------------------------------------ norm and clipping
@pytest.mark.parametrize("E", [2, 24, 40])
def test_gate_backward_of_the_longest_rows(E):
    """Rows of 16 MiB; columns at both ends and in between against 64 bits, tolerances as in check_gate."""
    T, d, n = 130, 2 ** 23, 512
    gen = torch.Generator(device="cuda").manual_seed(E)
    x = torch.empty((T, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    w = torch.empty((E, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    ds = torch.empty((T, E), device="cuda").normal_(generator=gen)
    dw, db = torch.full((E, d), -77.0, device="cuda"), torch.full((E,), -77.0, device="cuda")
    dx = torch.full((T, d), -77.0, dtype=torch.bfloat16, device="cuda")
    sh = shape_of(T, E, 1, 0, d)
    ws, nb = workspace(sh)
    B.moe_gate_backward(sh, x, w, ds, None, dw, db, dx, 0, ws, nb)
    at = torch.cat([torch.arange(n), torch.randint(0, d, (n,), generator=torch.Generator().manual_seed(1)), torch.arange(d - n, d)]).cuda()
    x64, w64, ds64 = (t.double().cpu().numpy() for t in (x[:, at], w[:, at], ds))
    rw, rb, rx = go.gate_backward(x64, w64, ds64)
    rw_size, rb_size, rx_size = go.gate_backward(np.abs(x64), np.abs(w64), np.abs(ds64))
    assert (np.abs(dw[:, at].double().cpu().numpy() - rw) <= (T + 8) * 2 * U * rw_size + 2 * U * np.abs(rw)).all()
    assert (np.abs(db.double().cpu().numpy() - rb) <= (T + 8) * 2 * U * rb_size + 2 * U * np.abs(rb)).all()
    half = 2.0 ** -8
    tol = half * np.abs(rx) + (1 + half) * ((E + 8) * 2 * U + 2.0 ** -16) * rx_size
    assert (np.abs(dx[:, at].double().cpu().numpy() - rx) <= tol).all()


def make_grads(sizes, seed, kinds="fb", offset=0):
    """Tensors of the given sizes, alternately fp32 and bf16, each starting `offset` elements into its allocation."""
    rng = np.random.default_rng([seed, len(sizes)])
    out = []
    for i, n in enumerate(sizes):
        dt = torch.float32 if kinds[i % len(kinds)] == "f" else torch.bfloat16
        base = torch.zeros(n + offset + 8, dtype=dt, device="cuda")
        t = base[offset:offset + n]
        t.copy_(torch.from_numpy((rng.standard_normal(n) * 10.0 ** -(i % 5)).astype(np.float32)))
        out.append(t)
    return out


def check_clip(grads, share, in_place=False, out_offset=0):
    before = [g.double().cpu().numpy() for g in grads]
    norm_ref = go.clip_grads(before, 1.0)[0]
    max_norm = float(np.float32(share * norm_ref)) if norm_ref else 1.0
    norm_ref, ref = go.clip_grads(before, max_norm)
    holders = None if in_place else [torch.full((g.numel() + 2 * PAD + out_offset,), -77.0, dtype=g.dtype, device="cuda") for g in grads]
    outs = None if in_place else [h[PAD + out_offset:PAD + out_offset + g.numel()] for h, g in zip(holders, grads)]
    lst = B.GradList(grads, outs)
    nb = B.moe_grad_workspace_bytes(lst)
    ws = torch.full((nb,), 0x5A, dtype=torch.uint8, device="cuda")
    norm = Guarded((1,))
    B.moe_grad_norm(lst, norm.t, ws, nb)
    assert abs(norm.np()[0] - norm_ref) <= 2 * U * norm_ref
    norm.t.fill_(-1)
    B.moe_clip_grads(lst, max_norm, norm.t, ws, nb)
    assert abs(norm.np()[0] - norm_ref) <= 2 * U * norm_ref
    for i, (r, o) in enumerate(zip(ref, grads if in_place else outs)):
        half = U if o.dtype == torch.float32 else 2.0 ** -8
        err = np.abs(o.double().cpu().numpy() - r)
        assert (err <= half * np.abs(r) + 3 * U * np.abs(r) + TINY).all(), (i, err.max())
        if share >= 1.0:
            assert np.array_equal(o.double().cpu().numpy(), before[i])
    if not in_place:
        for g, b in zip(grads, before):
            assert np.array_equal(g.double().cpu().numpy(), b)
        for h, o in zip(holders, outs):
            keep = torch.ones(h.numel(), dtype=torch.bool, device="cuda")
            keep[PAD + out_offset:PAD + out_offset + o.numel()] = False
            assert (h[keep] == -77.0).all()


@pytest.mark.parametrize("sizes", [[], [1], [0, 5, 0], [3, 4, 5], [4095, 4096, 4097], [7] * 127, [33] * 128, [65, 1] * 65,
                                   [1000003], [2048 * 64] * 5 + [17, 0, 9000001], [1] * 300], ids=lambda s: f"{len(s)}x{max(s + [0])}")
@pytest.mark.parametrize("share", [0.25, 1.5])
def test_clip_grads(sizes, share):
    check_clip(make_grads(sizes, 16), share)
    check_clip(make_grads(sizes, 16, "b"), share, in_place=True)
    check_clip(make_grads(sizes, 16, "f"), share, in_place=True)


@pytest.mark.parametrize("offset,out_offset", [(1, 0), (0, 1), (3, 3), (5, 2), (7, 6)])
def test_clip_grads_at_any_alignment(offset, out_offset):
    check_clip(make_grads([1, 2, 7, 8, 9, 100, 4097, 70001], 17, offset=offset), 0.5, out_offset=out_offset)
    check_clip(make_grads([1, 2, 7, 8, 9, 100, 4097, 70001], 17, offset=offset), 0.5, in_place=True)


def test_clip_grads_outside_the_range_of_squares():
    for scale in (1e-30, 1e-25, 1e25, 1e37):
        g = [torch.full((1000,), scale, dtype=torch.float32, device="cuda"), torch.full((77,), scale, dtype=torch.bfloat16, device="cuda")]
        check_clip(g, 0.5)
    # no elements but zeros: the norm is 0 and nothing is divided
    lst = B.GradList([torch.zeros(100, device="cuda")], [torch.ones(100, device="cuda")])
    nb = B.moe_grad_workspace_bytes(lst)
    ws, norm = torch.empty(nb, dtype=torch.uint8, device="cuda"), torch.full((1,), -1.0, device="cuda")
    for max_norm in (0.0, 1.0, float("inf")):
        B.moe_clip_grads(lst, max_norm, norm, ws, nb)
        assert float(norm) == 0.0 and not lst.out[0].any()


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_gradients_that_are_not_finite_are_left_and_reported(bad):
    g = make_grads([5000, 300], 18)
    g[1][7] = bad
    out = [torch.empty_like(t) for t in g]
    lst = B.GradList(g, out)
    nb = B.moe_grad_workspace_bytes(lst)
    ws, norm = torch.empty(nb, dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda")
    B.moe_clip_grads(lst, 1e-3, norm, ws, nb)
    assert not np.isfinite(float(norm))
    for a, b in zip(g, out):
        assert torch.equal(torch.nan_to_num(a.float(), 5.0), torch.nan_to_num(b.float(), 5.0))


def test_a_norm_beyond_fp32_leaves_the_gradients():
    g = [torch.full((4,), 3e38, device="cuda"), torch.ones(9, device="cuda")]
    lst = B.GradList(g, [torch.zeros_like(t) for t in g])
    nb = B.moe_grad_workspace_bytes(lst)
    ws, norm = torch.empty(nb, dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda")
    B.moe_clip_grads(lst, 1.0, norm, ws, nb)
    assert np.isinf(float(norm)) and all(torch.equal(a, b) for a, b in zip(g, lst.out))


# ------------------------------------------------------------------------------------------------ as they are used
def chain(sh, ws, nb, x, w, target, mask, bufs, stream):
    B.moe_route(sh, x, w, None, bufs["idx"], bufs["topk_w"], bufs["scores"], stream)
    B.moe_gate_distill(sh, bufs["scores"], target, mask, 1.0, bufs["loss"], bufs["d_scores"], 0, ws, nb, stream)
    B.moe_balance_loss(sh, bufs["scores"], bufs["idx"], mask, bufs["counts"], bufs["prob_sum"], bufs["balance"], ws, nb, stream)
    B.moe_route_backward(sh, bufs["scores"], bufs["idx"], None, bufs["counts"], 0.1, mask, bufs["d_scores"], 1, stream)
    B.moe_gate_backward(sh, x, w, bufs["d_scores"], mask, bufs["d_w"], bufs["d_b"], bufs["d_x"], 0, ws, nb, stream)
    B.moe_clip_grads(bufs["list"], bufs["max_norm"], bufs["norm"], bufs["gws"], bufs["gnb"], stream)


def chain_setup(T, d, E, k, seed):
    cfg = si.small_config(T=T, d=d, E=E, k=k, F=64, seed=seed)
    L = si.make_layer(cfg, parts=("x", "w_gate"))
    sh = B.make_shape(T, d, E, k, 64, cfg.dtype, cfg.renorm)
    ws, nb = workspace(sh)
    kw = dict(device="cuda")
    b = dict(idx=torch.empty((T, k), dtype=torch.int32, **kw), topk_w=torch.empty((T, k), **kw), scores=torch.empty((T, E), **kw),
             loss=torch.empty(1, **kw), balance=torch.empty(1, **kw), counts=torch.empty(E, dtype=torch.int32, **kw),
             prob_sum=torch.empty(E, **kw), d_scores=torch.empty((T, E), **kw), d_w=torch.empty((E, d), **kw),
             d_b=torch.empty(E, **kw), d_x=torch.empty((T, d), dtype=torch.bfloat16, **kw), norm=torch.empty(1, **kw))
    b["clipped"] = [torch.empty_like(b["d_w"]), torch.empty_like(b["d_b"])]
    b["list"] = B.GradList([b["d_w"], b["d_b"]], b["clipped"])
    b["max_norm"] = 1e-3
    b["gnb"] = B.moe_grad_workspace_bytes(b["list"])
    b["gws"] = torch.empty(b["gnb"], dtype=torch.uint8, **kw)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    target = torch.randn((T, E), generator=gen, **kw)
    mask = torch.rand(T, generator=gen, **kw) < 0.8
    return sh, ws, nb, L, layer.to_device(L["x"]), layer.to_device(L["w_gate"]), target, mask, b


OUTPUTS = ("loss", "balance", "counts", "prob_sum", "d_scores", "d_w", "d_b", "d_x", "norm")


def snapshot(b):
    torch.cuda.synchronize()
    return {n: b[n].clone() for n in OUTPUTS} | {f"clipped{i}": t.clone() for i, t in enumerate(b["clipped"])}


def test_a_training_step_against_the_oracle_in_a_stream_and_in_a_graph():
    T, d, E, k = 700, 264, 24, 3
    sh, ws, nb, L, x, w, target, mask, b = chain_setup(T, d, E, k, 21)
    chain(sh, ws, nb, x, w, target, mask, b, None)
    first = snapshot(b)
    m = mask.cpu().numpy().astype(np.uint8)
    scores, idx = b["scores"].cpu().numpy(), b["idx"].cpu().numpy()
    loss, g = go.gate_distill(scores, target.cpu().numpy(), 1.0, m)
    counts, prob_sum, balance = go.balance_loss(scores, idx, m)
    g = g + go.route_backward(scores, idx, None, counts, 0.1, sh.renorm, m, k)
    dw, db, _ = go.gate_backward(orc.to_f64(L["x"]), orc.to_f64(L["w_gate"]), g, m)
    norm, clipped = go.clip_grads([dw, db], 1e-3)
    assert float(first["loss"]) == pytest.approx(loss, rel=1e-5) and float(first["balance"]) == pytest.approx(balance, rel=1e-5)
    assert np.array_equal(first["counts"].cpu().numpy(), counts)
    assert np.abs(first["d_w"].cpu().numpy() - dw).max() <= 1e-5 * np.abs(dw).max()
    assert float(first["norm"]) == pytest.approx(norm, rel=1e-5)
    assert np.abs(first["clipped0"].cpu().numpy() - clipped[0]).max() <= 1e-5 * np.abs(clipped[0]).max()
    # another stream than the current one
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for n in OUTPUTS:
        b[n].zero_()
    side.wait_stream(torch.cuda.current_stream())
    chain(sh, ws, nb, x, w, target, mask, b, side)
    second = snapshot(b)
    assert all(torch.equal(first[n], second[n]) for n in first)
    # a captured step, replayed with other inputs and eager work in between
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(sh, ws, nb, x, w, target, mask, b, torch.cuda.current_stream())
    for i in range(4):
        x.copy_(torch.roll(x, 1, 0))
        target.mul_(-1.1)
        for n in OUTPUTS:
            b[n].fill_(3)
        graph.replay()
        replayed = snapshot(b)
        chain(sh, ws, nb, x, w, target, mask, b, None)
        eager = snapshot(b)
        for n in eager:
            assert torch.equal(eager[n], replayed[n]), f"replay {i}: {n}"


def test_two_steps_at_once_on_two_streams():
    a = chain_setup(900, 136, 16, 2, 22)
    c = chain_setup(650, 520, 64, 6, 23)
    alone = []
    for sh, ws, nb, _, x, w, target, mask, b in (a, c):
        chain(sh, ws, nb, x, w, target, mask, b, None)
        alone.append(snapshot(b))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for (sh, ws, nb, _, x, w, target, mask, b), s in zip((a, c), streams):
            chain(sh, ws, nb, x, w, target, mask, b, s)
    for ref, (*_, b) in zip(alone, (a, c)):
        got = snapshot(b)
        assert all(torch.equal(ref[n], got[n]) for n in ref)


@pytest.mark.parametrize("dtype,balance_coef", [(B.MOE_BF16, 0.0), (B.MOE_BF16, 0.05), (B.MOE_F32, 0.05)])
def test_gate_trainer_against_the_oracle(dtype, balance_coef):
    """Two gates, one of them in two micro-batches, a padded batch, d_x, and the clipped gradients of both."""
    T, d, E, k, n = 130, 72, 20, 3, 2
    rng = np.random.default_rng(31)
    tr = layer.GateTrainer(T, d, E, k, n, dtype, 1, max_norm=0.05, balance_coef=balance_coef)
    mask = mask_of("some", T, 31)
    sums, norms = [], 0.0
    for i in range(n):
        dw_sum, db_sum = np.zeros((E, d)), np.zeros(E)
        for micro in range(1 + i):
            x, w = store(rng.standard_normal((T, d)), dtype), store(rng.standard_normal((E, d)) / np.sqrt(d), dtype)
            target = rng.standard_normal((T, E)).astype(np.float32)
            d_x = torch.zeros((T, d), dtype=torch.float32 if dtype == B.MOE_F32 else torch.bfloat16, device="cuda")
            tr.enqueue(i, layer.to_device(x), layer.to_device(w), dev(target), token_mask=dev(mask), accumulate=micro > 0, d_x=d_x)
            scores, idx = tr.scores.cpu().numpy(), tr.topk_idx.cpu().numpy()
            assert np.abs(scores - orc.gate_scores(x, w)).max() <= 1e-4
            loss, g = go.gate_distill(scores, target, 1.0, mask)
            counts, _, balance = go.balance_loss(scores, idx, mask)
            if balance_coef:
                g = g + go.route_backward(scores, idx, None, counts, balance_coef, 1, mask, k)
            dw, db, dx = go.gate_backward(orc.to_f64(x), orc.to_f64(w), g, mask)
            dw_sum, db_sum = dw_sum + dw, db_sum + db
            assert float(tr.loss[i]) == pytest.approx(loss, rel=1e-5) and float(tr.balance[i]) == pytest.approx(balance, rel=1e-5)
            assert np.array_equal(tr.counts[i].cpu().numpy(), counts)
            half = 2.0 ** -8 if dtype == B.MOE_BF16 else 1e-5
            assert np.abs(d_x.double().cpu().numpy() - dx).max() <= half * np.abs(dx).max() + 1e-5 * np.abs(dx).max()
        assert np.abs(tr.d_w_gate[i].cpu().numpy() - dw_sum).max() <= 1e-5 * np.abs(dw_sum).max()
        assert np.abs(tr.d_gate_bias[i].cpu().numpy() - db_sum).max() <= 1e-5 * np.abs(dw_sum).max()
        sums.append((dw_sum, db_sum))
    norm, clipped = go.clip_grads([t for pair in sums for t in pair], 0.05)
    assert float(tr.clip()) == pytest.approx(norm, rel=1e-5)
    for i in range(n):
        assert np.abs(tr.d_w_gate[i].cpu().numpy() - clipped[2 * i]).max() <= 1e-5 * np.abs(clipped[2 * i]).max()


def test_finetuning_runs():
    T, d, E, k = 300, 64, 8, 2
    cfg = si.small_config(T=T, d=d, E=E, k=k, F=64, seed=33)
    L = si.make_layer(cfg, parts=("x", "w_gate"))
    x, w = layer.to_device(L["x"]), layer.to_device(L["w_gate"])
    tr = layer.GateTrainer(T, d, E, k, 1, cfg.dtype, cfg.renorm)
    target = torch.empty((T, E), device="cuda")
    tr.score(torch.roll(x, 1, 1).contiguous(), w, target)
    new, losses = layer.finetune_predictor(tr, x, target, w, 3, 1e-3)
    assert new.shape == w.shape and new.dtype == w.dtype and len(losses) == 3 and np.isfinite(losses).all()
    test = layer.LoadPredictor(T, d, E, k, cfg.dtype, cfg.renorm, E)
    pred, true, kept = layer.predicted_vs_actual_loads(test, x, x, new, w_later=w)
    assert pred.sum() == true.sum() == T * k and 0.0 <= kept <= 1.0
    assert layer.predicted_vs_actual_loads(test, x, x, w)[2] == 1.0


@pytest.mark.parametrize("T,E", [(301, 6), (2049, 40), (40001, 8)])
@pytest.mark.parametrize("start", [1, 7])
def test_masks_at_any_address(T, E, start):
    """A mask that begins inside a buffer gives the same bits as an aligned copy of it, whatever lies around it."""
    k, d = 2, 64
    rng, scores, idx = tables(T, E, k, 41)
    mask = mask_of("some", T, 41)
    around = torch.full((T + 64,), 255, dtype=torch.uint8, device="cuda")
    inside = around[start:start + T]
    inside.copy_(dev(mask))
    s, t, i = dev(scores), dev(rng.standard_normal((T, E)).astype(np.float32)), dev(idx)
    x, w = torch.from_numpy(rng.standard_normal((T, d))).cuda().bfloat16(), torch.from_numpy(rng.standard_normal((E, d))).cuda().bfloat16()
    sh = shape_of(T, E, k, 0, d)
    ws, nb = workspace(sh)
    results = []
    for m in (dev(mask), inside):
        f = lambda *n, dtype=torch.float32: torch.full(n, -7, dtype=dtype, device="cuda")          # noqa: E731
        out = [f(E, dtype=torch.int32), f(E), f(1), f(1), f(T, E), f(T, E), f(E, d), f(E), f(T, d, dtype=torch.bfloat16)]
        B.moe_balance_loss(sh, s, i, m, *out[:3], ws, nb)
        B.moe_gate_distill(sh, s, t, m, 1.0, out[3], out[4], 0, ws, nb)
        B.moe_route_backward(sh, s, i, s.view(-1)[:T * k], out[0], 0.5, m, out[5], 0)
        B.moe_gate_backward(sh, x, w, out[4], m, *out[6:], 0, ws, nb)
        results.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert int(results[0][0].sum()) == int((mask != 0).sum()) * k


def test_trainer_takes_nothing_that_does_not_fit():
    T, d, E = 32, 64, 8
    tr = layer.GateTrainer(T, d, E, 2, 1, B.MOE_BF16, 1)
    f = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")          # noqa: E731
    x, w, target = f(T, d), f(E, d), f(T, E, dtype=torch.float32)
    for args, kw in (((0, x[:T - 1], w, target), {}), ((0, x, w.float(), target), {}), ((0, x, f(d, E).t(), target), {}),
                     ((0, x, w, target[:, :E - 1]), {}), ((1, x, w, target), {}), ((0, x, w, target), dict(gate_bias=f(E))),
                     ((0, x, w, target), dict(token_mask=f(T - 1, dtype=torch.bool))), ((0, x, w, target), dict(d_x=f(T, d + 8)))):
        with pytest.raises(ValueError):
            tr.enqueue(*args, **kw)
    with pytest.raises(B.MoeError):
        tr.enqueue(0, x, w, target, d_x=x)
    # a gate that is part of a model: its own gradient is not touched
    model = w.clone().requires_grad_(True)
    new, _ = layer.finetune_predictor(tr, x, target, model, 1, 1e-3)
    assert not new.requires_grad and model.grad is None
    with pytest.raises(ValueError):
        layer.finetune_predictor(layer.GateTrainer(T, d, E, 2, 2, B.MOE_BF16, 1), x, target, w, 1, 1e-3)


def test_an_empty_batch_gives_zeros_or_leaves_what_is_there():
    for E in (1, 8, 200):
        sh = shape_of(0, E, 1, 0, 64)
        ws, nb = workspace(sh)
        counts, prob_sum, loss = Guarded((E,), torch.int32, -77), Guarded((E,)), Guarded((1,))
        B.moe_balance_loss(sh, None, None, None, counts.t, prob_sum.t, loss.t, ws, nb)
        assert not counts.np().any() and not prob_sum.np().any() and loss.np()[0] == 0.0
        B.moe_gate_distill(sh, None, None, None, 1.0, loss.t.fill_(5), None, 0, ws, nb)
        assert loss.np()[0] == 0.0
        B.moe_route_backward(sh, None, None, None, counts.t, 1.0, None, None, 0)
        dw, db = Guarded((E, 64)), Guarded((E,))
        B.moe_gate_backward(sh, None, None, None, None, dw.t, db.t, None, 1, ws, nb)
        assert (dw.np() == -77).all() and (db.np() == -77).all()
        B.moe_gate_backward(sh, None, None, None, None, dw.t, db.t, None, 0, ws, nb)
        assert not dw.np().any() and not db.np().any()


def test_tensors_that_do_not_fit_are_refused():
    T, E, k, d = 10, 8, 2, 64
    sh = shape_of(T, E, k, 0, d)
    ws, nb = workspace(sh)
    f = lambda *s: torch.zeros(s, device="cuda")          # noqa: E731
    scores, idx, counts, loss = f(T, E), torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros(E, dtype=torch.int32, device="cuda"), f(1)
    bad = [
        lambda: B.moe_balance_loss(sh, f(T, E - 1), idx, None, counts, f(E), loss, ws, nb),
        lambda: B.moe_balance_loss(sh, scores, idx.long(), None, counts, f(E), loss, ws, nb),
        lambda: B.moe_balance_loss(sh, f(E, T).t(), idx, None, counts, f(E), loss, ws, nb),
        lambda: B.moe_balance_loss(sh, scores, idx, torch.ones(T - 1, dtype=torch.bool, device="cuda"), counts, f(E), loss, ws, nb),
        lambda: B.moe_balance_loss(sh, scores, idx, f(T), counts, f(E), loss, ws, nb),
        lambda: B.moe_balance_loss(sh, scores.cpu(), idx, None, counts, f(E), loss, ws, nb),
        lambda: B.moe_balance_loss(sh, scores, idx, None, counts, f(E), loss, ws[:nb // 2], nb),
        lambda: B.moe_route_backward(sh, scores, idx, f(T, k + 1), None, 0.0, None, f(T, E)),
        lambda: B.moe_gate_distill(sh, scores, scores.double(), None, 1.0, loss, f(T, E), 0, ws, nb),
        lambda: B.moe_gate_backward(sh, f(T, d), None, scores, None, f(E, d), None, None, 0, ws, nb),      # fp32 x of a bf16 shape
        lambda: B.moe_gate_backward(sh, None, torch.zeros((E, d), dtype=torch.bfloat16, device="cuda"), scores, None, None, None, f(T, d), 0, ws, nb),
        lambda: B.GradList([f(4).double()]),
        lambda: B.GradList([f(4, 4).t()[1:]]),
        lambda: B.GradList([f(4)], [f(5)]),
        lambda: B.GradList([f(4)], [f(4).bfloat16()]),
        lambda: B.GradList([scores, scores]),
        lambda: B.GradList([scores[:5], f(40)], [f(5, E), scores.view(-1)[20:60]]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(f"case {i} was taken")
    with pytest.raises(B.MoeError) as err:
        B.moe_gate_distill(sh, scores, scores, None, 1.0, loss, f(T, E), 0, ws[:nb // 2].clone(), 16)
    assert err.value.code == -3
    # the same gradient may be read twice
    lst = B.GradList([scores, scores], [f(T, E), f(T, E)])
    assert len(lst) == 2


# ------------------------------------------------------------------------------------------------ products of few terms
@pytest.mark.parametrize("T,d,E", [(257, 136, 8), (300, 264, 24), (3000, 520, 64), (129, 512, 100), (65, 1048, 200)])
@pytest.mark.parametrize("dtype", [B.MOE_BF16, B.MOE_F32])
def test_d_x_of_terms_that_cancel(T, d, E, dtype):
    """Two experts of a token with nearly opposite gradients, and gate rows with a common part: what is left is small
    beside its two terms, whose 24 bits have to be in it: (2 + 8) 2u of the terms' sizes, and one rounding to storage."""
    rng = np.random.default_rng([55, T, E])
    w = store(1.0 + 0.03 * rng.standard_normal((E, d)), dtype)
    ds = np.zeros((T, E), dtype=np.float32)
    pick = np.stack([rng.permutation(E)[:2] for _ in range(T)])
    a = (rng.random(T) + 0.5).astype(np.float32)
    ds[np.arange(T), pick[:, 0]] = a
    ds[np.arange(T), pick[:, 1]] = -a * (1 + 0.03 * rng.standard_normal(T)).astype(np.float32)
    sh = shape_of(T, E, 1, 0, d, dtype)
    dx = Guarded((T, d), torch.float32 if dtype == B.MOE_F32 else torch.bfloat16)
    B.moe_gate_backward(sh, None, layer.to_device(w), dev(ds), None, None, None, dx.t, 0, None, 0)
    w64 = orc.to_f64(w)
    ref, size = ds.astype(np.float64) @ w64, np.abs(ds.astype(np.float64)) @ np.abs(w64)
    half = U if dtype == B.MOE_F32 else 2.0 ** -8
    err, tol = np.abs(dx.np() - ref), half * np.abs(ref) + (1 + half) * 20 * U * size
    assert (err <= tol).all(), f"{(err > tol).mean():.4f} of the elements, {(err / size).max() / U:.1f} u of the terms"


# ------------------------------------------------------------------------------------------------ scores of any size
def shifted(scores):
    """Rows less their maximum, cut at -104, below which e^s is no fp32 number: the same probabilities to within 1e-45."""
    s = np.asarray(scores, dtype=np.float64)
    m = s.max(axis=1, keepdims=True)
    return np.maximum(s - np.where(np.isneginf(m), 0.0, m), -104.0)


def check_losses_of_large_scores(scores, target, idx, mask=None):
    """The three calls on a table whose rows' maxima may have any size.  Tolerances as above, with the spread of what is not
    zero in fp32; a term q (log q - log p) of the loss is off by 32 u of its parts' sizes, and its sum over E by 16 u."""
    T, E = scores.shape
    k = idx.shape[1]
    rows = np.arange(T) if mask is None else np.flatnonzero(mask)
    low = shifted(scores)
    rng = np.random.default_rng([T, E])
    dw = rng.standard_normal((T, k)).astype(np.float32)
    sh = shape_of(T, E, k)
    ws, nb = workspace(sh)
    m = dev(mask)
    counts, prob_sum, loss = Guarded((E,), torch.int32, -77), Guarded((E,)), Guarded((1,))
    B.moe_balance_loss(sh, dev(scores), dev(idx), m, counts.t, prob_sum.t, loss.t, ws, nb)
    rc, rp, rl = go.balance_loss(scores, idx, mask)
    tol = (2 * 104 + 24 + T / 512 + 64) * U
    assert np.array_equal(counts.np(), rc)
    assert (np.abs(prob_sum.np() - rp) <= tol * rp + TINY).all(), (prob_sum.np(), rp)
    assert abs(loss.np()[0] - rl) <= (tol + 2 * U) * abs(rl)
    for renorm in (0, 1):
        out = Guarded((T, E))
        B.moe_route_backward(shape_of(T, E, k, renorm), dev(scores), dev(idx), dev(dw), dev(rc.astype(np.int32)), 0.5 * T, m, out.t)
        ref = go.route_backward(scores, idx, dw, rc, 0.5 * T, renorm, mask)
        # (the chosen experts have a maximum of their own: what they are is not what is left of `low`)
        size = route_bound(low, idx, dw, rc.astype(np.float64), 0.5 * T, 0, mask, k)
        for j in range(k if renorm else 0):
            size[rows, idx[rows, j]] += (2 * (208 + 24) + 24 + k) * U * 2 * np.abs(dw[rows]).max(axis=1)
        err = np.abs(out.np() - ref)
        assert (err <= size).all(), (renorm, np.argwhere(~(err <= size))[:4], err.max())
    out, loss = Guarded((T, E)), Guarded((1,))
    B.moe_gate_distill(sh, dev(scores), dev(target), m, 2.0, loss.t, out.t, 0, ws, nb)
    rl, rg = go.gate_distill(scores, target, 2.0, mask)
    p, q = go.softmax(scores), go.softmax(target)
    err = np.abs(out.np() - rg)
    assert (err <= (208 + 28) * U * 2.0 / rows.size * (p + q) + TINY).all(), err.max()
    s64, t64 = scores.astype(np.float64), target.astype(np.float64)
    log_p = s64 - s64.max(axis=1, keepdims=True) - np.log(np.exp(s64 - s64.max(axis=1, keepdims=True)).sum(axis=1, keepdims=True))
    log_q = t64 - t64.max(axis=1, keepdims=True) - np.log(np.exp(t64 - t64.max(axis=1, keepdims=True)).sum(axis=1, keepdims=True))
    size = np.where(q > 0, q * (np.abs(log_p) + np.abs(log_q) + 24), 0.0)[rows].sum() / rows.size
    assert np.isfinite(rl) and abs(loss.np()[0] - rl) <= 48 * U * size + 2 * U * abs(rl), (loss.np()[0], rl)


LARGE = [7e4, 1e6, -1e6, 1e8, -1e8, 1.6e9, 3e9, 5e9, -5e9, 1e10, -1e10, 1e12, 1e20, -1e20, 1e29, -1e29, -1e30, 2e30, -3e38]


@pytest.mark.parametrize("E", [4, 7, 64, 200])
def test_chosen_experts_with_a_switch_off_value(E):
    """Finite switch-off values: of all chosen experts, of all but one, of all experts."""
    rng = np.random.default_rng([52, E])
    for off in (-1e9, -1e10, -1e20, -1e30, -np.finfo(np.float32).max):
        scores = rng.standard_normal((90, E)).astype(np.float32)
        idx = np.stack([rng.permutation(E)[:2] for _ in range(90)]).astype(np.int32)
        scores[np.arange(30), idx[:30, 0]] = off
        scores[np.arange(30), idx[:30, 1]] = off
        scores[30:60] = np.where(np.arange(E) == idx[30:60, :1], scores[30:60], off)
        scores[60:70] = off
        check_losses_of_large_scores(scores, scores, idx)


@pytest.mark.parametrize("E", [1, 6, 8, 64, 250])
def test_rows_of_large_scores(E):
    """A batch of ordinary tokens and of tokens whose scores are all alike, or a few steps of fp32 apart, at any size."""
    rng = np.random.default_rng([51, E])
    k = min(E, 3)
    T = 3 * len(LARGE) + 40
    scores = rng.standard_normal((T, E)).astype(np.float32)
    for i, v in enumerate(LARGE):
        scores[3 * i] = v
        steps = rng.integers(-3, 4, E)
        scores[3 * i + 1] = np.float32(v) + steps * np.spacing(np.float32(abs(v)))
        scores[3 * i + 2, rng.random(E) < 0.5] = v
    target = scores.copy()
    target[:, 0] += np.float32(0.5)
    target[::3] = rng.standard_normal((len(target[::3]), E))
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    check_losses_of_large_scores(scores, np.where(np.arange(T)[:, None] % 3 == 0, target, scores), idx)
    check_losses_of_large_scores(target, target, idx, mask_of("some", T, 51))


@pytest.mark.parametrize("E", [2, 5, 64, 130])
def test_a_target_that_wants_finite_scores_far_below(E):
    """The loss is finite as long as the scores are: q times a difference that passes the largest fp32 number itself, too."""
    rng = np.random.default_rng([53, E])
    T = 40
    for top, low in ((0.3, -3.4e38), (1.0, -1e38), (2e38, -2e38), (3e38, -3.4e38), (1e20, -1e30)):
        scores = rng.standard_normal((T, E)).astype(np.float32)
        target = rng.standard_normal((T, E)).astype(np.float32)
        scores[5, 0], scores[5, 1] = top, low
        scores[9] = low
        scores[9, 1] = top
        target[[5, 9]] = rng.standard_normal((2, E))
        target[5, 1] = -2.0
        check_losses_of_large_scores(scores, target, np.zeros((T, 1), dtype=np.int32))


@pytest.mark.parametrize("E", [1, 6, 64, 129])
@pytest.mark.parametrize("where", ["all scores", "one score", "scores beside -inf", "one target", "all targets"])
def test_nan_scores_of_a_token_that_counts_are_seen(E, where):
    """A NaN makes the loss and the token's own gradient NaN; it is not taken for a token with no expert left."""
    rng = np.random.default_rng([54, E])
    T = 70
    scores, target = (rng.standard_normal((T, E)).astype(np.float32) for _ in range(2))
    table = scores if "score" in where else target
    if where.startswith("all"):
        table[11] = np.nan
    else:
        if "beside" in where:
            table[11] = -np.inf
        table[11, E // 2] = np.nan
    sh = shape_of(T, E, 1)
    ws, nb = workspace(sh)
    loss, out = Guarded((1,)), Guarded((T, E))
    B.moe_gate_distill(sh, dev(scores), dev(target), None, 1.0, loss.t, out.t, 0, ws, nb)
    got = out.np()
    assert np.isnan(loss.np()[0]) and np.isnan(got[11]).all()
    assert np.isfinite(np.delete(got, 11, axis=0)).all()
    mask = np.ones(T, dtype=np.uint8)
    mask[11] = 0
    check_distill(T, E, mask, np.where(np.isnan(scores), 0, scores), np.where(np.isnan(target), 0, target), 1.0, 0)


def test_clip_grads_by_factors_below_the_normal_numbers():
    """max_norm / norm is a number of few bits in fp32, or none, where the scaled gradients are ordinary numbers."""
    for value, share in ((1e35, 1e-39), (1e35, 3e-44), (1e36, 1e-45), (7e36, 7e-47)):
        g = [torch.full((1000,), value, dtype=torch.float32, device="cuda"), torch.full((77,), -value, dtype=torch.bfloat16, device="cuda")]
        check_clip([t.clone() for t in g], share)
        check_clip([t.clone() for t in g], share, in_place=True)
        check_clip([t.clone() for t in g], share, out_offset=1)


# (the last four: blocks of 64 experts)
ALONE = [(1, 264, 24), (40, 264, 20), (64, 128, 8), (300, 520, 33), (129, 512, 65), (200, 264, 129), (257, 1024, 200),
         (33001, 1048, 50), (40001, 1048, 64), (8200, 1048, 200), (16500, 1048, 128)]


@pytest.mark.parametrize("T,d,E", ALONE)
@pytest.mark.parametrize("dtype", [B.MOE_BF16, B.MOE_F32])
def test_products_that_are_alone_in_their_sums(T, d, E, dtype):
    """Gradients, at most one to a token and one to an expert: every row of d_w_gate and d_x is one product.  fp32 layers: eight
    of nine piece products (the ninth is below 2^-31 of the whole), seven of them, 2^-6 of it, cut at 24 bits each, and a rounded
    addition: 1.25 u.  d_w_gate of bf16 layers: three piece products whose sum is cut: 2.1 u.  d_x of bf16 layers: its storage."""
    rng = np.random.default_rng([56, T, E])
    n = min(T, E)
    x, w = store(rng.standard_normal((T, d)), dtype), store(rng.standard_normal((E, d)), dtype)
    t = rng.permutation(T)[:n]
    t[:min(n, 2)] = [T - 1, 0][:min(n, 2)]
    t = np.unique(t)
    e = rng.permutation(E)[:t.size]
    ds = np.zeros((T, E), dtype=np.float32)
    ds[t, e] = rng.standard_normal(t.size) * 10.0 ** rng.integers(-6, 3, t.size)
    sh = shape_of(T, E, 1, 0, d, dtype)
    ws, nb = workspace(sh)
    dw, db, dx = Guarded((E, d)), Guarded((E,)), Guarded((T, d), torch.float32 if dtype == B.MOE_F32 else torch.bfloat16)
    B.moe_gate_backward(sh, layer.to_device(x), layer.to_device(w), dev(ds), None, dw.t, db.t, dx.t, 0, ws, nb)
    rw, rb, rx = go.gate_backward(orc.to_f64(x), orc.to_f64(w), ds)
    of_w, of_x = (1.25 * U, 1.25 * U) if dtype == B.MOE_F32 else (2.1 * U, 2.0 ** -8)
    err = np.abs(dw.np() - rw)
    assert (err <= of_w * np.abs(rw)).all(), f"d_w_gate: {(err[rw != 0] / np.abs(rw[rw != 0])).max() / U:.3f} u"
    err = np.abs(dx.np() - rx)
    assert (err <= of_x * np.abs(rx)).all(), f"d_x: {(err[rx != 0] / np.abs(rx[rx != 0])).max() / U:.3f} u"
    assert np.array_equal(db.np(), rb)


@pytest.mark.parametrize("T,d,E", [(300, 64, 8), (70001, 64, 8), (30000, 72, 24), (5000, 64, 40), (33001, 1048, 64), (8200, 1048, 200)])
@pytest.mark.parametrize("dtype", [B.MOE_BF16, B.MOE_F32])
def test_bias_gradients_of_one_large_and_many_small_terms(T, d, E, dtype):
    """Small terms below half a step of the large one: eight terms of a lane are added in 32 bits (three roundings), the rest
    in 64, a part's sum and the whole are rounded once: 5 u of the sizes."""
    ds = np.full((T, E), 2.0 ** -25, dtype=np.float32)
    ds[T // 3] = 1.0
    x = torch.zeros((T, d), dtype=torch.float32 if dtype == B.MOE_F32 else torch.bfloat16, device="cuda")
    sh = shape_of(T, E, 1, 0, d, dtype)
    ws, nb = workspace(sh)
    for with_w in (True, False):
        dw, db = Guarded((E, d)), Guarded((E,))
        B.moe_gate_backward(sh, x, None, dev(ds), None, dw.t if with_w else None, db.t, None, 0, ws, nb)
        ref = 1.0 + (T - 1) * 2.0 ** -25
        assert (np.abs(db.np() - ref) <= 5 * U * ref).all(), (db.np() - ref) / U


@pytest.mark.parametrize("max_norm", [float("inf"), 1e-3])
def test_finetuning_clips_by_what_it_trains(max_norm):
    """Without a trained bias the norm is that of the weights' gradient, and the bias' gradient stays unscaled."""
    T, d, E = 200, 64, 16
    rng = np.random.default_rng(57)
    x, w = store(rng.standard_normal((T, d)), B.MOE_BF16), store(rng.standard_normal((E, d)) / 8, B.MOE_BF16)
    target = (rng.standard_normal((T, E)) + 3.0 * np.arange(E) / E).astype(np.float32)      # a bias that the gate lacks
    tr = layer.GateTrainer(T, d, E, 2, 1, B.MOE_BF16, 1, max_norm=max_norm)
    layer.finetune_predictor(tr, layer.to_device(x), dev(target), layer.to_device(w), 1, 0.0)
    _, g = go.gate_distill(orc.gate_scores(x, w), target)
    dw, db, _ = go.gate_backward(orc.to_f64(x), orc.to_f64(w), g)
    norm, (clipped,) = go.clip_grads([dw], max_norm)
    assert float(tr.norm) == pytest.approx(norm, rel=1e-5)
    assert np.abs(tr.d_w_gate[0].cpu().numpy() - clipped).max() <= 1e-5 * np.abs(clipped).max()
    assert np.abs(tr.d_gate_bias[0].cpu().numpy() - db).max() <= 1e-5 * np.abs(db).max()
    both = go.clip_grads([dw, db], max_norm)[0]
    assert float(tr.clip()) == pytest.approx(np.hypot(min(norm, max_norm), np.linalg.norm(db)), rel=1e-5) and both > 1.01 * norm


@pytest.mark.parametrize("dtype", [B.MOE_BF16, B.MOE_F32])
def test_finetuning_of_a_gate_with_a_bias(dtype):
    """One step: scores and losses with the bias, a norm of both gradients, and both moved by Adam's first step, lr against
    the gradient's sign; the bias that was given, and the later gate's, are left."""
    T, d, E, k, lr = 200, 64, 16, 2, 1e-2
    rng = np.random.default_rng(58)
    x, w = store(rng.standard_normal((T, d)), dtype), store(rng.standard_normal((E, d)) / 8, dtype)
    bias = np.linspace(-1.5, 1.5, E).astype(np.float32)
    target = rng.standard_normal((T, E)).astype(np.float32)
    tr = layer.GateTrainer(T, d, E, k, 1, dtype, 1, max_norm=float("inf"))
    xd, wd, bd = layer.to_device(x), layer.to_device(w), dev(bias)
    new, losses, new_bias = layer.finetune_predictor(tr, xd, dev(target), wd, 1, lr, gate_bias=bd)
    loss, g = go.gate_distill(orc.gate_scores(x, w, bias), target)
    dw, db, _ = go.gate_backward(orc.to_f64(x), orc.to_f64(w), g)
    assert losses == [pytest.approx(loss, rel=1e-5)] and np.array_equal(bd.cpu().numpy(), bias)
    assert float(tr.norm) == pytest.approx(go.clip_grads([dw, db], 1.0)[0], rel=1e-5)
    moved = new_bias.double().cpu().numpy() - bias
    assert (np.abs(moved + lr * np.sign(db))[np.abs(db) > 1e-4] <= 1e-3 * lr).all() and (np.abs(db) > 1e-4).sum() > E // 2
    if dtype == B.MOE_F32:
        moved, large = new.double().cpu().numpy() - orc.to_f64(w), np.abs(dw) > 1e-4
        assert (np.abs(moved + lr * np.sign(dw))[large] <= 1e-3 * lr).all()
    assert not new_bias.requires_grad and not new.requires_grad and new.dtype == wd.dtype
    # the accuracy study with a bias of either gate
    pred = layer.LoadPredictor(T, d, E, k, dtype, 1, E)
    a = layer.predicted_vs_actual_loads(pred, xd, xd, new, new_bias, w_later=wd, bias_later=bd)
    idx = orc.topk_select(orc.gate_scores(x, w, bias), k)
    assert np.array_equal(a[1], np.bincount(idx.ravel(), minlength=E))
    assert layer.predicted_vs_actual_loads(pred, xd, xd, wd, bd)[2] == 1.0


@pytest.mark.parametrize("where", ["x", "target"])
def test_finetuning_on_what_is_not_finite_is_refused(where):
    T, d, E = 100, 64, 8
    gen = torch.Generator(device="cuda").manual_seed(59)
    x, w = (torch.randn(s, generator=gen, device="cuda").bfloat16() for s in ((T, d), (E, d)))
    target = torch.randn((T, E), generator=gen, device="cuda")
    tr = layer.GateTrainer(T, d, E, 2, 1, B.MOE_BF16, 1)
    mask = torch.ones(T, dtype=torch.bool, device="cuda")
    mask[7] = False
    if where == "x":
        x[7, 3] = float("inf")
    else:
        target[7, 3] = float("nan")
    with pytest.raises(ValueError, match="step 0"):
        layer.finetune_predictor(tr, x, target, w, 3, 1e-3)
    new, losses = layer.finetune_predictor(tr, x, target, w, 3, 1e-3, token_mask=mask)      # a padded token's
    assert torch.isfinite(new.float()).all() and np.isfinite(losses).all()


def test_micro_batches_add_up_to_the_mean_over_all_tokens():
    T, d, E, k = 96, 64, 12, 2
    rng = np.random.default_rng(60)
    w = store(rng.standard_normal((E, d)) / 8, B.MOE_BF16)
    tr = layer.GateTrainer(T, d, E, k, 1, B.MOE_BF16, 1, balance_coef=0.05)
    masks = [mask_of("some", T, 61), mask_of("odd_bytes", T, 0), mask_of("one", T, 0)]
    n = [int((m != 0).sum()) for m in masks]
    pieces = []
    for i, m in enumerate(masks):
        x, target = store(rng.standard_normal((T, d)), B.MOE_BF16), rng.standard_normal((T, E)).astype(np.float32)
        tr.enqueue(0, layer.to_device(x), layer.to_device(w), dev(target), token_mask=dev(m), accumulate=i > 0, coef=n[i] / sum(n))
        scores, idx = orc.gate_scores(x, w), tr.topk_idx.cpu().numpy()
        loss, _ = go.gate_distill(scores, target, 1.0, m)
        assert float(tr.loss[0]) == pytest.approx(loss, rel=1e-5)
        pieces.append((x, scores, target, idx, m))
    x, scores, target, idx, m = (np.concatenate(p) for p in zip(*pieces))
    _, g = go.gate_distill(scores, target, 1.0, m)
    # the balance loss is each micro-batch's own, in its share
    g = g + np.concatenate([n[i] / sum(n) * go.route_backward(s, e, None, go.balance_loss(s, e, v)[0], 0.05, 1, v, k)
                            for i, (_, s, _, e, v) in enumerate(pieces)])
    dw, db, _ = go.gate_backward(orc.to_f64(x), orc.to_f64(w), g, m)
    assert np.abs(tr.d_w_gate[0].cpu().numpy() - dw).max() <= 1e-5 * np.abs(dw).max()
    assert np.abs(tr.d_gate_bias[0].cpu().numpy() - db).max() <= 1e-5 * np.abs(dw).max()


@pytest.mark.parametrize("T", [32767, 32768, 32769, 40001, 65536])
@pytest.mark.parametrize("mask", ["some", "nothing", "one", "odd_bytes", "last"])
def test_gate_distill_of_masks_that_a_launch_counts(T, mask):
    """From 32768 tokens on the mask is counted before the gradients are made; all of its parts have tokens."""
    E = 8
    rng, scores, _ = tables(T, E, 1, 62)
    target = (scores + 0.5 * rng.standard_normal((T, E))).astype(np.float32)
    m = mask_of(mask if mask != "last" else "nothing", T, 62)
    if mask == "last":
        m[[0, T // 64 - 1, T // 64, T - 1]] = 1
    check_distill(T, E, m, scores, target, 1.0, 0)
    check_distill(T, E, m, scores, target, -0.1 * T, 1)


@pytest.mark.parametrize("T,d,E", [(33001, 1048, 64), (8200, 1048, 200)])
def test_a_training_step_of_large_blocks_in_a_graph_and_on_two_streams(T, d, E):
    """The kernels of large batches, of more than 32 experts: replayed with other inputs, and two batches at once."""
    sh, ws, nb, _, x, w, target, mask, b = chain_setup(T, d, E, 3, 63)
    chain(sh, ws, nb, x, w, target, mask, b, None)
    first = snapshot(b)
    other = chain_setup(T - 1000, d, E, 3, 64)
    chain(*other[:3], *other[4:], None)
    alone = snapshot(other[-1])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        chain(sh, ws, nb, x, w, target, mask, b, streams[0])
        chain(*other[:3], *other[4:], streams[1])
    got, got_other = snapshot(b), snapshot(other[-1])
    assert all(torch.equal(first[n], got[n]) for n in first) and all(torch.equal(alone[n], got_other[n]) for n in alone)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(sh, ws, nb, x, w, target, mask, b, torch.cuda.current_stream())
    for i in range(3):
        x.copy_(torch.roll(x, 1, 0))
        target.mul_(-1.1)
        for n in OUTPUTS:
            b[n].fill_(3)
        graph.replay()
        replayed = snapshot(b)
        chain(sh, ws, nb, x, w, target, mask, b, None)
        eager = snapshot(b)
        for n in eager:
            assert torch.equal(eager[n], replayed[n]), f"replay {i}: {n}"
