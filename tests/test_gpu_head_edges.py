"""Losses of the output head where their references, weights and 16-bit exponents are under strain: every output finite and within bounds that follow the roundings one by one."""
import numpy as np
import pytest
import torch

import paper_2509_22418_amd as pp
from test_gpu_head import TYPES, call, check, make

pytestmark = pytest.mark.gpu


def strict(got, *a, **k):
    """check(), and no output is NaN or infinite (its bounds on dx and dw are comparisons, which NaN passes)."""
    for name, v in got.items():
        assert np.isfinite(v).all(), (name, int((~np.isfinite(v)).sum()), np.argwhere(~np.isfinite(v))[:3].tolist())
    return check(got, *a, **k)


# n, vocab, entries, absent ones in front: bf16, a group of entries per wave is 4 (40 and 900 rows) or 16 (600); 900 x 8200: losses alone go by the reference too
@pytest.mark.parametrize("n,vocab,top,gone,dtype", [(40, 600, 24, 6, "bf16"), (600, 5000, 40, 16, "bf16"), (600, 5000, 40, 35, "bf16"), (900, 8200, 6, 4, "bf16"), (40, 600, 24, 6, "f32"),
                                                    (12, 600, 24, 6, "bf16"), (3, 600, 128, 70, "f32")])
@pytest.mark.parametrize("tau,share", [(1.0, 1.0), (0.25, 1.0), (2.0, 0.5), (0.25, 0.5), (1.0, 0.5)])
@pytest.mark.parametrize("by", ["id", "logit"])
def test_rows_whose_first_entries_are_absent(n, vocab, top, gone, dtype, tau, share, by):
    """The first entries of a row are none, it has no target, and all its logits lie far below 0 (or above): the softmax has the same weights wherever the entries stand in the list."""
    print(f"case head late entries {n}x{vocab} top={top} gone={gone} by={by} {dtype} tau={tau} share={share}", flush=True)
    x, w, y, ids, u = make(n, vocab, 64, TYPES[dtype], top=top, ragged=False, seed=7)
    if by == "id":
        ids[:, :gone:2], ids[:, 1:gone:2], u[:, :gone] = -1, vocab, torch.nan
    else:
        u[:, :gone] = -torch.inf
    y[::2] = -1
    w[:, 0] = 1.0
    low = -100.0 * min(1.0, tau)
    x[:, 0] = torch.tensor([low, 0.0, low / 3, low, -low, 3 * low], device="cuda").repeat(n)[:n]
    a = dict(ids=ids, u=u, tau=tau, share=share)
    strict(call(x, w, y, dw=(0, vocab), **a), x, w, y, dw=(0, vocab), **a)
    strict(call(x, w, y, dx=False, **a), x, w, y, **a)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [9, 333])
@pytest.mark.parametrize("top,tau,share", [(0, 1.0, 1.0), (4, 1.0, 0.5), (4, 2.0, 1.0), (4, 3.0, 0.4)])
def test_weights_down_to_the_smallest_floats(top, tau, share, n, dtype):
    """Weights that fade along a sequence, down to numbers below the smallest normal float, and up to 1e20: rows of them have their part of the gradients or none, and spoil nothing."""
    print(f"case head fading weights n={n} top={top} tau={tau} share={share} {dtype}", flush=True)
    x, w, y, ids, u = make(n, 900, 64, TYPES[dtype], top=top, seed=8, ignored=0.1, ragged=False)
    weight = 10.0 ** torch.linspace(0.0, -44.0, n, dtype=torch.float64, device="cuda")
    weight[::3] *= -1
    weight = weight.float()
    # some rows' largest logit 39 above the target's
    w[:, 0] = 0.0
    w[7, 0], w[11, 0] = 1.0, -1.0
    x[:, 0] = 0.0
    x[3::5, 0], y[3::5] = 19.5, 11
    if top:
        ids[3::5, 0] = 11
    a = dict(ids=ids, u=u, tau=tau, share=share) if top else {}
    for scale in (1.0, 1e20):
        wt = (weight * scale).contiguous()
        strict(call(x, w, y, weight=wt, dw=(0, 900), dw_type=torch.float32, **a), x, w, y, weight=wt, dw=(0, 900), **a)
    # nothing but small weights, a power of two: the gradients are those of weights of 1 times it, bit for bit
    small = 2.0 ** -40
    got, one = (call(x, w, y, weight=torch.full((n,), v, device="cuda"), dw=(0, 900), dw_type=torch.float32, **a) for v in (small, 1.0))
    for name in ("dx", "dw"):
        assert np.array_equal(got[name], small * one[name]), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [7, 200])
def test_operands_side_by_side_in_one_buffer(n, dtype):
    """X and dX, W and dW as column ranges of one buffer each: they share no element, and the call is as with buffers of their own."""
    x, w, y, _, _ = make(n, 500, 72, TYPES[dtype])
    one, two = torch.zeros((n, 144), dtype=x.dtype, device="cuda"), torch.zeros((500, 200), dtype=x.dtype, device="cuda")
    one[:, :72], two[:, 100:172] = x, w
    out = dict(loss=torch.empty(1, device="cuda"), row_loss=torch.empty(n, device="cuda"), row_lse=torch.empty(n, device="cuda"), dx=one[:, 72:], dw=two[20:420, :72])
    h = pp.make_head(one[:, :72], two[:, 100:172], dw_lo=5, dw_hi=405, **out)
    ws = torch.empty(pp.pp_op_head_bytes(h), dtype=torch.uint8, device="cuda")
    pp.pp_op_head_ce(torch.cuda.current_stream().cuda_stream, h, y.data_ptr(), ws.data_ptr(), ws.numel())
    strict({k: v.double().cpu().numpy() for k, v in out.items()}, x, w, y, dw=(5, 405))
    assert torch.equal(one[:, :72], x) and torch.equal(two[:, 100:172], w) and not two[420:, :72].any() and not two[:20, :72].any()


def tight(got, x, w, y, ids, u, tau, share, dw):
    """strict(), and dX and dW of a call with more than 16 rows in bf16 within the sum of the roundings that the code makes, whatever the temperature.

    An element of dz is a sum of the two softmaxes' parts and of what is taken off at the target and the entries.  Its roundings: an exponential's argument and sum in fp32 (`rel` each); the stored
    sum of both parts to bf16 (half a step, 2^-8) and the row's scale, which moves by as much (2^-8).  Two softmaxes are formed from a stored exponent y of the sharper one, in powers of two: half
    a step of it is 2^-9 from -64 on and 2^-5 below (of its largest logit, which no reference exceeds, so no y is larger than assumed here), hence 2^-9 ln 2 or 2^-5 ln 2 of the sharper part and
    those over the ratio of the temperatures of the softer one; below -2096 both are taken as 0.  Then half a step for the scaled rows of X (dW), fp32 sums, and half a step of the results."""
    ref = strict(got, x, w, y, ids, u, tau=tau, share=share, dw=dw)
    X, W, Y, I = x.double().cpu().numpy(), w.double().cpu().numpy(), y.long().cpu().numpy(), ids.long().cpu().numpy()
    n, vocab, d = X.shape[0], W.shape[0], X.shape[1]
    live, eps, half, z = ref["live"], 2.0 ** -24, 2.0 ** -8, ref["z"]
    X0 = np.where(live[:, None], X, 0.0)
    g = np.where(live, 1.0 / max(1, live.sum()), 0.0)
    it = max(1.0, 1.0 / tau)
    there = (I >= 0) & (I < vocab) & (u.cpu().numpy() != -np.inf) & live[:, None]
    c1 = g * (1 - share) * ((Y >= 0) & (Y < vocab))
    ct = g * share * tau * there.any(1)
    soft = lambda v: np.exp(v - v.max(1, keepdims=True)) / np.exp(v - v.max(1, keepdims=True)).sum(1, keepdims=True)  # noqa: E731
    one, two = c1[:, None] * soft(z), ct[:, None] * soft(z / tau)
    rel = ((d + 2) * eps * it * (np.abs(X0) @ np.abs(W).T)).max(1) + (2 * np.abs(z).max(1) * it + vocab / 64 + 80) * eps
    off = np.zeros_like(z)
    rows = np.broadcast_to(np.arange(n)[:, None], I.shape)
    np.add.at(off, (rows[there], I[there]), (ct * np.ones(I.shape).T).T[there])
    hard = np.nonzero(c1)[0]
    off[hard, Y[hard]] += c1[hard]
    err = np.abs(ref["dz"]) * (2 * rel[:, None] + 2 * half + 8 * eps) + off * (4 * rel[:, None] + 16 * eps)
    if tau != 1.0 and 0.0 < share < 1.0:
        ratio = max(tau, 1.0 / tau)
        exponent = (z - z.max(1, keepdims=True)) * it / np.log(2.0)
        step = np.where(exponent < -64, 2.0 ** -5, 2.0 ** -9) * np.log(2.0) * 1.02          # 2^s - 1 <= 1.02 s ln 2 for these s
        sharper, softer = (one, two) if tau > 1.0 else (two, one)
        lost = exponent < -2096
        plain = off == 0          # places are formed in fp32
        err += np.where(plain, sharper * np.where(lost, 1.0, step) + softer * np.where(lost, 1.0, step / ratio), 0.0)
    part, absW, lo, hi = np.abs(ref["dz"]), np.abs(W), *dw
    tol = err @ absW + (vocab + 64) * eps * (part @ absW) + half * np.abs(ref["dx"]) + 1e-36
    worst = np.abs(got["dx"] - ref["dx"]) / tol
    assert worst.max() <= 1, ("dx", float(worst.max()), np.argwhere(worst > 1)[:3].tolist())
    tol = (err + part * half)[:, lo:hi].T @ np.abs(X0) + (n + 64) * eps * (part[:, lo:hi].T @ np.abs(X0)) + half * np.abs(ref["dw"][lo:hi]) + 1e-36
    worst = np.abs(got["dw"] - ref["dw"][lo:hi]) / tol
    assert worst.max() <= 1, ("dw", float(worst.max()), np.argwhere(worst > 1)[:3].tolist())


@pytest.mark.parametrize("n,vocab", [(40, 600), (700, 3000), (2100, 4100)])
@pytest.mark.parametrize("tau,std", [(64.0, 30.0), (16.0, 30.0), (3.0, 8.0), (2.0, 0.5), (1.5, 30.0), (0.7, 8.0), (0.7, 40.0), (0.5, 8.0), (0.25, 2.0), (0.125, 0.5), (0.125, 8.0), (1.0 / 64, 0.05), (1.0 / 64, 1.0),
                                     (1.0 / 64, 5.0)])
def test_two_softmaxes_within_their_roundings(tau, std, n, vocab):
    print(f"case head two softmaxes {n}x{vocab} tau={tau} std={std}", flush=True)
    x, w, y, ids, u = make(n, vocab, 64, torch.bfloat16, top=6, std=std, seed=4)
    dw = (3, vocab - 2)
    tight(call(x, w, y, ids, u, tau=tau, share=0.6, dw=dw), x, w, y, ids, u, tau, 0.6, dw)


@pytest.mark.parametrize("tau,share", [(1.0, 1.0), (1.0, 0.4), (4.0, 1.0), (0.125, 1.0), (1.0 / 64, 1.0), (2.0, 0.0)])
def test_one_softmax_within_its_roundings(tau, share):
    x, w, y, ids, u = make(700, 3000, 64, torch.bfloat16, top=6, std=0.5, seed=4)
    dw = (3, 2998)
    tight(call(x, w, y, ids, u, tau=tau, share=share, dw=dw), x, w, y, ids, u, 1.0 if share == 0.0 else tau, share, dw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [5, 90])
@pytest.mark.parametrize("tau,share", [(1.0, 1.0), (0.5, 1.0), (2.0, 0.5)])
def test_lists_that_repeat_ids(tau, share, n, dtype):
    """Rows of few words listed up to twelve times, their target among them: each entry keeps its own logarithm in the loss, and the gradients are those of the sums."""
    x, w, y, ids, u = make(n, 400, 64, TYPES[dtype], top=20, ragged=False, seed=14)
    ids = (ids % 5).int()
    ids[::3, :12] = 7
    y = torch.where(y >= 0, y % 8, y).int()
    a = dict(ids=ids, u=u, tau=tau, share=share)
    strict(call(x, w, y, dw=(0, 400), **a), x, w, y, dw=(0, 400), **a)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [4, 16, 70])
@pytest.mark.parametrize("top", [1, 3, 70, 128])
def test_rows_of_nothing_but_minus_infinity(top, n, dtype):
    """Valid ids whose logits are all -inf are no entries: such a row has no KL term, and is left out where it has no target either."""
    x, w, y, ids, u = make(n, 300, 64, TYPES[dtype], top=top, ragged=False, seed=15, ignored=0.5)
    u[::2] = -torch.inf
    y[0], y[1] = -1, 5
    x[0] = torch.nan
    for tau, share in ((1.0, 1.0), (2.0, 0.5), (0.5, 0.25)):
        a = dict(ids=ids, u=u, tau=tau, share=share)
        got = call(x, w, y, dw=(0, 300), **a)
        assert got["row_loss"][0] == 0 and not got["dx"][0].any()
        strict(got, x, w, y, dw=(0, 300), **a)
