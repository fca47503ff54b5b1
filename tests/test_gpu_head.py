"""Losses of the output head and their gradients on the GPU against the 64-bit oracle: sizes from one row and one word of vocabulary up, odd ones, rows and entries left out,
strides, pieces, logits far from the target's, graphs and streams."""
import numpy as np
import pytest
import torch

import paper_2509_22418_amd as pp
from oracle import pp_oracle as O

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
NONE = dict(top=0, tau=1.0, share=1.0)


def make(n, vocab, d, dtype, seed=0, std=0.5, top=0, ignored=0.2, ragged=True):
    """Inputs on the GPU; x has unit variance, logits a deviation of std * sqrt(d / 16)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    x, w = r(n, d).to(dtype), (r(vocab, d) * std / 4).to(dtype)
    y = torch.randint(0, vocab, (n,), device="cuda", generator=g, dtype=torch.int32)
    y = torch.where(torch.rand(n, device="cuda", generator=g) < ignored, -1, y.long()).int()
    ids = u = None
    if top:
        ids = torch.randint(0, vocab, (n, top), device="cuda", generator=g, dtype=torch.int32)
        u = 2 * r(n, top)
        if ragged:
            absent = torch.rand((n, top), device="cuda", generator=g) < 0.3
            ids = torch.where(absent, torch.where(torch.rand((n, top), device="cuda", generator=g) < 0.5, -1, vocab), ids.long()).int()
            u = torch.where(absent, torch.nan, u)
            ids[::5] = -1
    return x, w, y, ids, u


def call(x, w, y, ids=None, u=None, tau=1.0, share=1.0, weight=None, dx=True, dw=None, dw_type=None, dw_add=False, piece=0, pad=0, stream=None, ws=None):
    """One call with outputs of its own between guard values; returns them in 64 bits."""
    n, d = x.shape
    dev = x.device
    guard = 7.0
    new = lambda *s, t=torch.float32: torch.full(s, guard, dtype=t, device=dev)  # noqa: E731
    out = dict(loss=new(1), row_loss=new(n), row_lse=new(n))
    full = {}
    if dx:
        full["dx"] = new(n, d + pad, t=x.dtype)
    if dw:
        full["dw"] = new(dw[1] - dw[0], d + pad, t=dw_type or w.dtype)
    views = {k: v[:, :d] for k, v in full.items()}
    h = pp.make_head(x, w, row_weight=weight, dw_lo=dw[0] if dw else 0, dw_add=dw_add, piece=piece, **out, **views)
    top = ids.shape[1] if ids is not None else 0
    if ws is None:
        ws = torch.full((pp.pp_op_head_bytes(h, top),), 0xFF, dtype=torch.uint8, device=dev)          # NaN in every type: nothing of it may be used
    st = (stream or torch.cuda.current_stream()).cuda_stream
    if ids is None:
        pp.pp_op_head_ce(st, h, y.data_ptr(), ws.data_ptr(), ws.numel())
    else:
        pp.pp_op_head_distill(st, h, ids.data_ptr(), u.data_ptr(), top, tau, share, None if y is None else y.data_ptr(), ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    for v in full.values():
        assert bool((v[:, d:] == guard).all())          # nothing past a row's end
    return {k: v.double().cpu().numpy() for k, v in {**out, **views}.items()}


def check(got, x, w, y, ids=None, u=None, tau=1.0, share=1.0, weight=None, dw=None, base=0.0, pieces=1):
    """Every output within bounds summed from the roundings on its way:
    z: fp32 sums of d products; an exponential of an argument of size A: A + 8 roundings; a row's sum: at most vocab / 64 + 64 additions one after the other; bf16: the
    exponentials (half a step, 2^-8) and the scaled rows of X (2^-8) that enter the gradients' products, the outputs' own rounding (2^-8), and a row's scale, which is chosen for its
    largest place to come out exact: a relative change of at most half a step (2^-8) of everything else in the row, so 2 * 2^-8 before the products."""
    np64 = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    ints = lambda t: None if t is None else t.long().cpu().numpy()  # noqa: E731
    X, W, wt = np64(x), np64(w), np64(weight)
    ref = O.head_loss(X, W, ints(y), wt, ints(ids), np64(u), tau, share)
    if ids is None:
        tau, share = 1.0, 0.0
    n, vocab, d = X.shape[0], W.shape[0], X.shape[1]
    live = ref["live"]
    X0 = np.where(live[:, None], X, 0.0)
    half = 2.0 ** -8 if x.dtype == torch.bfloat16 else EPS
    it = max(1.0, 1.0 / tau)
    ez = (d + 2) * EPS * (np.abs(X0) @ np.abs(W).T) * it                 # [n, vocab]
    size = np.abs(ref["z"]).max(axis=1) * it                             # [n]
    rel = ez.max(axis=1) + (2 * size + vocab / 64 + 80) * EPS             # of an exponential over its row's sum
    k = max(1.0, tau) ** 2
    tol_row = 4 * k * (rel + EPS * (size + 20))
    assert np.all(np.abs(got["row_lse"] - ref["row_lse"]) <= tol_row), "row_lse"
    assert np.all(np.abs(got["row_loss"] - ref["row_loss"]) <= tol_row), "row_loss"
    assert np.all(got["row_lse"][~live] == 0) and np.all(got["row_loss"][~live] == 0)
    g = wt if wt is not None else np.full(n, 1.0 / max(1, live.sum()))
    g = np.where(live, g, 0.0)
    assert abs(got["loss"][0] - ref["loss"]) <= np.sum(np.abs(g) * (tol_row + (n / 256 + 40) * EPS * np.abs(ref["row_loss"]))) + 1e-30, "loss"
    # |dz| before its parts cancel: the softmaxes (vocabulary) and what is taken off at the target and the entries
    part = np.abs(ref["dz"])
    ez_rel = 2 * rel[:, None] + 2 * half + (8 * EPS)
    off = np.zeros_like(part)          # absolute error where p and the taken-off part cancel: fp32 roundings of parts of size g
    if share < 1.0:
        Y = ints(y)
        for t in np.nonzero(live)[0]:
            if 0 <= Y[t] < vocab:
                off[t, Y[t]] += abs(g[t]) * (1 - share)
    if ids is not None:
        I = ints(ids)
        rows = np.broadcast_to(np.arange(n)[:, None], I.shape)
        there = (I >= 0) & (I < vocab) & live[:, None]
        off[rows[there], I[there]] = np.abs(g[rows[there]]) * (1 + share * tau)
    # with both softmaxes at different temperatures one is a power of the other's rounded value
    both = 1.0 if tau == 1.0 or share in (0.0, 1.0) else 1.0 + it
    err = part * (ez_rel * both) + off * (4 * rel[:, None] + 16 * EPS)
    if "dx" in got:
        tol = err @ np.abs(W) + (vocab + 64) * EPS * (part @ np.abs(W)) + half * np.abs(ref["dx"]) + 1e-36
        bad = np.abs(got["dx"] - ref["dx"]) > tol
        assert not bad.any(), ("dx", int(bad.sum()), np.argwhere(bad)[:3].tolist(), float((np.abs(got["dx"] - ref["dx"]) / tol).max()))
        assert np.all(got["dx"][~live] == 0)
    if "dw" in got:
        lo, hi = dw
        tol = (err + part * half)[:, lo:hi].T @ np.abs(X0) + (n + 64) * EPS * (part[:, lo:hi].T @ np.abs(X0)) + half * (np.abs(ref["dw"][lo:hi]) + abs(base)) + 1e-36
        # every piece's product is added to dw by one fp32 addition, whose result is no larger than base and the parts together: half a step (EPS) of that each
        tol += pieces * EPS * (abs(base) + part[:, lo:hi].T @ np.abs(X0))
        bad = np.abs(got["dw"] - base - ref["dw"][lo:hi]) > tol
        assert not bad.any(), ("dw", int(bad.sum()), np.argwhere(bad)[:3].tolist(), float((np.abs(got["dw"] - base - ref["dw"][lo:hi]) / tol).max()))
    return ref


SIZES = [(16, 777, 2100), (17, 300, 64), (5, 40000, 96), (1, 1, 1), (1, 8, 8), (1, 257, 64), (2, 2, 3), (3, 1000, 65), (64, 256, 64), (65, 511, 128), (130, 1003, 200), (257, 640, 72), (300, 2049, 320)]
KINDS = {"ce": NONE, "kd": dict(top=5, tau=1.0, share=1.0), "kd_hard": dict(top=9, tau=1.0, share=0.5), "kd_tau": dict(top=3, tau=2.0, share=1.0), "kd_sharp": dict(top=128, tau=0.5, share=1.0),
         "mixed": dict(top=7, tau=2.0, share=0.3), "mixed_sharp": dict(top=2, tau=0.7, share=0.8), "hard_only": dict(top=2, tau=2.0, share=0.0)}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab,d", SIZES)
def test_cross_entropy(n, vocab, d, dtype):
    print(f"case head ce {n}x{vocab}x{d} {dtype}", flush=True)
    x, w, y, _, _ = make(n, vocab, d, TYPES[dtype], ignored=0.2 if n > 3 else 0.0)
    check(call(x, w, y, dw=(0, vocab)), x, w, y, dw=(0, vocab))
    check(call(x, w, y, dx=False), x, w, y)
    check(call(x, w, y), x, w, y)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", [k for k in KINDS if k != "ce"])
@pytest.mark.parametrize("n,vocab,d", [(1, 17, 8), (4, 1500, 40), (16, 333, 130), (70, 515, 136), (260, 1024, 64)])
def test_distillation(n, vocab, d, kind, dtype):
    print(f"case head {kind} {n}x{vocab}x{d} {dtype}", flush=True)
    k = dict(KINDS[kind])
    x, w, y, ids, u = make(n, vocab, d, TYPES[dtype], top=k.pop("top"), seed=3)
    if n == 1:
        ids[0, 0], u[0, 0] = 3, 0.5
    a = dict(ids=ids, u=u, **k)
    check(call(x, w, y, dw=(0, vocab), **a), x, w, y, dw=(0, vocab), **a)
    check(call(x, w, y, dx=False, **a), x, w, y, **a)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["ce", "kd_hard", "mixed"])
def test_pieces_strides_slices_and_weights(kind, dtype):
    """Many pieces (some without a row that counts), rows of X, W and the gradients further apart than d, bases off their alignment, a slice of W, row weights with zeros
    and negative ones, NaN and infinities in everything that is left out."""
    k = dict(KINDS[kind])
    top = k.pop("top")
    for n, vocab, d, piece, lo, hi in ((300, 700, 96, 64, 13, 400), (333, 129, 40, 128, 128, 129), (200, 1001, 192, 64, 0, 1001), (11, 600, 70, 0, 5, 590)):
        print(f"case head pieces {kind} {n}x{vocab}x{d} piece={piece} {dtype}", flush=True)
        x0, w0, y, ids, u = make(n, vocab, d, TYPES[dtype], top=top, seed=5)
        y[64:200] = -1
        if top:
            ids[64:200] = -1
            u[64:150] = torch.nan
        x = torch.full((n, d + 5), torch.nan, dtype=x0.dtype, device="cuda")[:, 1:d + 1]
        w = torch.full((vocab, d + 3), torch.nan, dtype=x0.dtype, device="cuda")[:, 2:d + 2]
        x.copy_(x0)
        w.copy_(w0)
        weight = torch.rand(n, device="cuda") - 0.2
        weight[3:min(20, n - 4)] = 0.0
        weight = weight / n
        x[3:min(20, n - 4)] = torch.nan
        x[70:100] = torch.inf
        a = dict(ids=ids, u=u, **k) if top else {}
        check(call(x, w, y, weight=weight, dw=(lo, hi), piece=piece, pad=3, **a), x, w, y, weight=weight, dw=(lo, hi), **a)
        f = call(x, w, y, weight=weight, dw=(lo, hi), piece=piece, pad=2, dw_type=torch.float32, **a)
        check(f, x, w, y, weight=weight, dw=(lo, hi), **a)
        check(call(x, w, y, weight=weight, dx=False, dw=(lo, hi), piece=piece, dw_type=torch.float32, dw_add=True, pad=1, **a), x, w, y, weight=weight, dw=(lo, hi), base=7.0, pieces=-(-n // piece) if piece else 1, **a)


@pytest.mark.parametrize("n,vocab,d,top,piece", [(3000, 5000, 256, 128, 0), (2801, 6001, 200, 120, 0), (5000, 3001, 128, 128, 2944)])
@pytest.mark.parametrize("tau,share", [(1.0, 0.5), (2.0, 1.0), (2.0, 0.6)])
def test_entries_picked_from_the_product(n, vocab, d, top, piece, tau, share):
    """Enough entries for their logits to be picked from the first product: lists of all lengths (none for whole blocks of rows), a quarter of all entries on one column, equal ids within
    rows, the last tiles ragged."""
    print(f"case head picked {n}x{vocab}x{d} top={top} tau={tau} share={share} piece={piece}", flush=True)
    x, w, y, ids, u = make(n, vocab, d, torch.bfloat16, top=top, seed=13)
    there = (ids >= 0) & (ids < vocab)          # absent entries hold NaN and stay absent
    ids[::4] = torch.where(there[::4], vocab - 1, ids[::4].long()).int()
    ids[7] = torch.where(there[7], 5, ids[7].long()).int()
    ids[512:768] = -1
    y[600:700] = -1
    a = dict(ids=ids, u=u, tau=tau, share=share)
    check(call(x, w, y, dw=(0, vocab), piece=piece, **a), x, w, y, dw=(0, vocab), **a)


@pytest.mark.parametrize("dtype", TYPES)
def test_nothing_counts(dtype):
    """All rows left out, and no rows at all: loss 0, gradients of zeros, a float dw that is added to unchanged."""
    x, w, y, ids, u = make(70, 300, 64, TYPES[dtype], top=4)
    x[:] = torch.nan
    y[:], ids[:] = -1, 300
    for a in ({}, dict(ids=ids, u=u, share=0.5)):
        got = call(x, w, y, dw=(0, 300), **a)
        assert all(np.all(v == 0) for v in got.values())
        assert np.all(call(x, w, y, dw=(0, 300), dw_type=torch.float32, dw_add=True, **a)["dw"] == 7.0)
    none = dict(x=x[:0], w=w, y=y[:0])
    got = call(**none, dw=(5, 300))
    assert np.all(got["loss"] == 0) and np.all(got["dw"] == 0)
    assert np.all(call(**none, dw=(5, 300), dw_type=torch.float32)["dw"] == 0)
    assert np.all(call(**none, dw=(5, 300), dw_type=torch.float32, dw_add=True)["dw"] == 7.0)
    assert np.all(call(**none, ids=ids[:0], u=u[:0])["loss"] == 0)


def test_entries_of_minus_infinity_equal_ids_and_rows_of_one_word():
    """A logit of -inf is no entry, equal ids add up (the target among them), a vocabulary of one word has no loss."""
    x, w, y, ids, u = make(66, 40, 64, torch.bfloat16, top=6, ragged=False)
    u[:, 2] = -torch.inf
    ids[:, 4], ids[:, 5] = ids[:, 0], ids[:, 0]
    y = ids[:, 0].contiguous()
    u[7] = -torch.inf
    for k in (dict(tau=1.0, share=0.5), dict(tau=2.0, share=1.0), dict(tau=2.0, share=0.5)):
        check(call(x, w, y, ids, u, dw=(0, 40), **k), x, w, y, ids, u, dw=(0, 40), **k)
    one = call(x, w[:1], torch.zeros_like(y), dw=(0, 1))
    assert np.all(np.abs(one["row_loss"]) <= 1e-5) and np.all(np.abs(one["dx"]) <= 1e-5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["ce", "kd_tau", "mixed"])
def test_logits_far_from_the_target(kind, dtype):
    """Rows whose largest logit is tens to hundreds above the target's or the first entry's, or as far below, next to ordinary ones: the softmax needs no luck with its reference."""
    for n in (600, 16):
        far(n, kind, dtype)


def far(n, kind, dtype):
    vocab, d = 900, 64
    k = dict(KINDS[kind])
    x, w, y, ids, u = make(n, vocab, d, TYPES[dtype], top=k.pop("top"), ignored=0.0, ragged=False, seed=9)
    w[:, 0] = 0.0
    w[7, 0], w[11, 0] = 1.0, -1.0
    x[:, 0] = 0.0
    for t, v in ((0, 39.0), (1, 45.0), (2, 80.0), (3, 100.0), (4, 250.0), (5, -60.0), (6, -300.0), (300, 120.0), (301, 500.0), (599, 90.0)):
        if t < n:
            x[t, 0] = v
    y[:] = 11
    y[4:7] = 7
    y[301:302] = 500
    if ids is not None:
        ids[:, 0] = y
    a = dict(ids=ids, u=u, **k) if ids is not None else {}
    check(call(x, w, y, dw=(0, vocab), **a), x, w, y, dw=(0, vocab), **a)
    check(call(x, w, y, dx=False, **a), x, w, y, **a)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab", [(40, 600), (2100, 4100)])
@pytest.mark.parametrize("tau,std", [(64.0, 30.0), (16.0, 30.0), (3.0, 8.0), (0.125, 8.0), (1.0 / 64, 1.0)])
def test_two_softmaxes_of_logits_far_apart(tau, std, n, vocab, dtype):
    """Hard targets and a teacher at a temperature far from 1: where one softmax has nothing left of a logit (hundreds below the largest), the other still has."""
    x, w, y, ids, u = make(n, vocab, 64, TYPES[dtype], top=6, std=std, seed=4)
    a = dict(ids=ids, u=u, tau=tau, share=0.6)
    dw = (3, vocab // 2)
    check(call(x, w, y, dw=dw, **a), x, w, y, dw=dw, **a)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [5, 40])
def test_rows_far_apart_in_memory(n, dtype):
    """Rows of W and X so long that the offsets of 64 of them pass 31 bits."""
    ld, d, vocab = (1 << 24) + 8, 64, 70
    x, w, y, _, _ = make(n, vocab, d, TYPES[dtype])
    far_w, far_x = torch.empty((vocab, ld), dtype=w.dtype, device="cuda")[:, :d], torch.empty((n, ld), dtype=x.dtype, device="cuda")[:, :d]
    far_w.copy_(w)
    far_x.copy_(x)
    check(call(far_x, far_w, y, dw=(1, 69)), x, w, y, dw=(1, 69))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["ce", "mixed"])
def test_rows_wider_than_a_workgroup_holds(kind, dtype):
    """Vocabularies beyond 32768: fp32 rows of logits that do not fit a workgroup's registers; their largest logits first, last and in the middle."""
    n, vocab, d = 40, 50001, 64
    k = dict(KINDS[kind])
    x, w, y, ids, u = make(n, vocab, d, TYPES[dtype], top=k.pop("top"), std=2.0)
    w[0], w[vocab - 1], w[30000] = 3 * w[0], 4 * w[vocab - 1], 5 * w[30000]
    a = dict(ids=ids, u=u, **k) if ids is not None else {}
    check(call(x, w, y, dw=(49000, vocab), **a), x, w, y, dw=(49000, vocab), **a)
    x[3] = torch.nan
    bad = call(x, w, y.clamp(min=0), **a)
    assert np.isnan(bad["row_loss"][3]) and np.isnan(bad["dx"][3]).all() and not np.isnan(bad["dx"][[2, 4]]).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [12, 70])
@pytest.mark.parametrize("tau,share", [(0.25, 1.0), (0.25, 0.5), (2.0, 0.5)])
def test_entries_of_the_lowest_finite_value(tau, share, n, dtype):
    """The lowest finite float is an entry like any other: alone in a row it has the whole probability, at any temperature."""
    x, w, y, ids, u = make(n, 300, 64, TYPES[dtype], top=5, ragged=False)
    low = torch.finfo(torch.float32).min
    u[0] = low
    u[1, 1:] = low
    u[2, :4] = low
    ids[3, 1:], u[3] = -1, low
    a = dict(ids=ids, u=u, tau=tau, share=share)
    check(call(x, w, y, dw=(0, 300), **a), x, w, y, dw=(0, 300), **a)


def test_non_finite_rows_that_count_stay_in_their_rows():
    """NaN in a row that counts: its loss and its dX row are NaN, the other rows' are as without it."""
    x, w, y, _, _ = make(300, 500, 64, torch.bfloat16, ignored=0.0)
    clean = call(x, w, y)
    x2 = x.clone()
    x2[17, 3] = torch.nan
    got = call(x2, w, y)
    keep = np.arange(300) != 17
    assert np.isnan(got["row_loss"][17]) and np.isnan(got["dx"][17]).all() and np.isnan(got["loss"][0])
    assert np.array_equal(got["row_loss"][keep], clean["row_loss"][keep]) and np.array_equal(got["dx"][keep], clean["dx"][keep])


def test_results_do_not_depend_on_the_run_or_the_workspace():
    for n in (500, 12):
        x, w, y, ids, u = make(n, 3001, 256, torch.bfloat16, top=12, seed=2)
        k = dict(ids=ids, u=u, tau=2.0, share=0.5, dw=(0, 3001))
        first, second = call(x, w, y, **k), call(x, w, y, ws=torch.zeros(1 << 28, dtype=torch.uint8, device="cuda"), **k)
        assert all(np.array_equal(first[v], second[v]) for v in first)


def test_two_streams_at_once():
    """Calls on two streams with a workspace each."""
    jobs = []
    for seed, n in ((1, 400), (2, 700)):
        x, w, y, ids, u = make(n, 2000, 128, torch.bfloat16, top=8, seed=seed)
        jobs.append((x, w, y, ids, u, call(x, w, y, ids, u, share=0.5)))
    outs = []
    for x, w, y, ids, u, _ in jobs:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        o = dict(loss=torch.empty(1, device="cuda"), row_loss=torch.empty(len(y), device="cuda"), row_lse=torch.empty(len(y), device="cuda"), dx=torch.empty_like(x))
        h = pp.make_head(x, w, **o)
        ws = torch.empty(pp.pp_op_head_bytes(h, 8), dtype=torch.uint8, device="cuda")
        outs.append((s, o, h, ws, ids, u, y))
    torch.cuda.synchronize()
    for _ in range(4):
        for s, o, h, ws, ids, u, y in outs:
            pp.pp_op_head_distill(s.cuda_stream, h, ids.data_ptr(), u.data_ptr(), 8, 1.0, 0.5, y.data_ptr(), ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    for (s, o, *_), (*_, ref) in zip(outs, jobs):
        for name, v in o.items():
            assert np.array_equal(v.double().cpu().numpy(), ref[name])


@pytest.mark.parametrize("kind", ["ce", "mixed"])
def test_captured_and_replayed(kind):
    """One call captured into a graph and replayed on changed inputs, with eager work between the replays; every replay equals the eager call."""
    k = dict(KINDS[kind])
    top = k.pop("top")
    x, w, y, ids, u = make(333, 1500, 128, torch.bfloat16, top=top, ragged=False)
    o = dict(loss=torch.empty(1, device="cuda"), row_loss=torch.empty(333, device="cuda"), row_lse=torch.empty(333, device="cuda"), dx=torch.empty_like(x), dw=torch.empty((1500, 128), dtype=x.dtype, device="cuda"))
    h = pp.make_head(x, w, piece=128, **o)
    ws = torch.empty(pp.pp_op_head_bytes(h, top), dtype=torch.uint8, device="cuda")

    def go():
        st = torch.cuda.current_stream().cuda_stream
        if top:
            pp.pp_op_head_distill(st, h, ids.data_ptr(), u.data_ptr(), top, k["tau"], k["share"], y.data_ptr(), ws.data_ptr(), ws.numel())
        else:
            pp.pp_op_head_ce(st, h, y.data_ptr(), ws.data_ptr(), ws.numel())
    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for seed in range(4):
        x2, w2, y2, ids2, u2 = make(333, 1500, 128, torch.bfloat16, top=top, ragged=True, seed=20 + seed, ignored=0.3 * seed)
        x.copy_(x2)
        w.copy_(w2)
        y.copy_(y2)
        if top:
            ids.copy_(ids2)
            u.copy_(u2)
        graph.replay()
        torch.cuda.synchronize()
        a = dict(ids=ids, u=u, **k) if top else {}
        ref = call(x, w, y, dw=(0, 1500), piece=128, **a)
        for name, v in o.items():
            assert np.array_equal(v.double().cpu().numpy(), ref[name]), (seed, name)


@pytest.mark.parametrize("n,vocab,d,top,dtype,grads", [(3, 500, 72, 5, "bf16", True), (9, 500, 72, 0, "f32", False), (100, 300, 40, 4, "f32", True), (200, 700, 64, 6, "bf16", False), (2500, 3000, 128, 100, "bf16", True)])
def test_two_captured_calls_share_a_workspace(n, vocab, d, top, dtype, grads):
    """Few rows, fp32, losses alone and picked entries: two graphs over one workspace, replayed one after the other with eager calls in between."""
    ins = [make(n, vocab, d, TYPES[dtype], top=top, seed=30 + i) for i in range(2)]
    outs = [dict(loss=torch.empty(1, device="cuda"), row_loss=torch.empty(n, device="cuda"), row_lse=torch.empty(n, device="cuda"),
                 **(dict(dx=torch.empty_like(i[0]), dw=torch.empty((vocab, d), device="cuda")) if grads else {})) for i in ins]
    heads = [pp.make_head(i[0], i[1], **o) for i, o in zip(ins, outs)]
    ws = torch.empty(max(pp.pp_op_head_bytes(h, top) for h in heads), dtype=torch.uint8, device="cuda")

    def go(h, x, w, y, ids, u):
        st = torch.cuda.current_stream().cuda_stream
        if top:
            pp.pp_op_head_distill(st, h, ids.data_ptr(), u.data_ptr(), top, 2.0, 0.5, y.data_ptr(), ws.data_ptr(), ws.numel())
        else:
            pp.pp_op_head_ce(st, h, y.data_ptr(), ws.data_ptr(), ws.numel())
    graphs = []
    for h, i in zip(heads, ins):
        go(h, *i)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            go(h, *i)
    for turn in range(3):
        for g, i, o in zip(graphs, ins, outs):
            g.replay()
            torch.cuda.synchronize()
            a = dict(ids=i[3], u=i[4], tau=2.0, share=0.5) if top else {}
            ref = call(*i[:3], dx=grads, dw=(0, vocab) if grads else None, dw_type=torch.float32 if grads else None, **a)
            for name, v in o.items():
                assert np.array_equal(v.double().cpu().numpy(), ref[name]), (turn, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["ce", "mixed"])
@pytest.mark.parametrize("n,vocab,d", [(18, 1 << 20, 8), (3, 1 << 20, 8), (20, 100, 1 << 14), (3, 100, 1 << 14), (270001, 9, 8)])
def test_largest_sizes(n, vocab, d, kind, dtype):
    k = dict(KINDS[kind])
    x, w, y, ids, u = make(n, vocab, d, TYPES[dtype], top=k.pop("top"), std=0.5 if d < 64 else 0.02)
    a = dict(ids=ids, u=u, **k) if ids is not None else {}
    dw = (vocab - 7, vocab)
    check(call(x, w, y, dw=dw, **a), x, w, y, dw=dw, pieces=2, **a)


def test_refusals_name_what_is_wrong():
    x, w, y, _, _ = make(8, 100, 64, torch.bfloat16)
    h = pp.make_head(x, w, loss=torch.empty(1, device="cuda"))
    ws = torch.empty(pp.pp_op_head_bytes(h), dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    with pytest.raises(pp.PPError, match="needs"):
        pp.pp_op_head_ce(st, h, y.data_ptr(), ws.data_ptr(), ws.numel() - 256)
    with pytest.raises(pp.PPError, match="targets"):
        pp.pp_op_head_ce(st, h, None, ws.data_ptr(), ws.numel())
    with pytest.raises(pp.PPError, match="make_head"):
        pp.make_head(x, w.cpu())
