"""Losses of the output head without a GPU: the oracle against library autograd and differences, and every refusal of the entry points."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2509_22418_amd as pp
from oracle import pp_oracle as O


def problem(n=7, vocab=23, d=5, top=4, seed=0):
    r = np.random.default_rng(seed)
    x, w = r.normal(size=(n, d)), r.normal(size=(vocab, d))
    y = r.integers(-1, vocab, n)
    ids, u = r.integers(-1, vocab, (n, top)), 2 * r.normal(size=(n, top))
    ids[0] = -1                                  # a row without entries
    ids[1] = (3, 3, 5, vocab)                    # equal ids, one outside
    u[2, 0] = -np.inf
    y[3] = -1
    return x, w, y, ids, u


@pytest.mark.parametrize("tau,share,weighted", [(None, 0.0, False), (1.0, 1.0, False), (2.0, 1.0, True), (0.5, 0.3, False), (3.0, 0.0, True)])
def test_oracle_matches_library_autograd_and_differences(tau, share, weighted):
    x, w, y, ids, u = problem()
    wt = np.linspace(0.1, 0.7, len(y)) if weighted else None
    if weighted:
        wt[4] = 0.0
    ref = O.head_loss(x, w, y, wt, None if tau is None else ids, u, tau or 1.0, share)

    def loss(xt, wm):
        z = xt @ wm.T
        hard = torch.tensor((y >= 0) & (share < 1))
        row = torch.zeros(len(y), dtype=torch.float64)
        live = hard.clone()
        row = row + (1 - share) * torch.nn.functional.cross_entropy(z, torch.tensor(np.where(hard, y, -100)), ignore_index=-100, reduction="none")
        if tau is not None and share > 0:
            full = torch.full_like(z, -np.inf).detach()          # the teacher's logits as a row of the vocabulary; equal ids: log of the sum
            for t in range(len(y)):
                for i, v in zip(ids[t], u[t]):
                    if 0 <= i < z.shape[1]:
                        full[t, i] = torch.logaddexp(full[t, i], torch.tensor(v / tau))
            soft = torch.isfinite(full).any(1)
            q = torch.softmax(torch.where(soft[:, None], full, torch.zeros(())), 1) * soft[:, None]
            logp = torch.log_softmax(z / tau, 1)
            # entropies of equal ids differ (they are two entries of the list, one place of the vocabulary): only what depends on z is compared
            row = row + share * tau ** 2 * (-(q * logp).sum(1))
            live = live | soft
        g = torch.tensor(wt) if weighted else torch.full((len(y),), 1.0 / int(live.sum()), dtype=torch.float64)
        return (g * live * row).sum(), live

    xt, wm = torch.tensor(x, requires_grad=True), torch.tensor(w, requires_grad=True)
    out, live = loss(xt, wm)
    out.backward()
    if weighted:
        live[4] = False
    assert np.array_equal(live.numpy(), ref["live"])
    np.testing.assert_allclose(xt.grad.numpy(), ref["dx"], rtol=1e-11, atol=1e-13)
    np.testing.assert_allclose(wm.grad.numpy(), ref["dw"], rtol=1e-11, atol=1e-13)
    # differences of the loss itself (the entropies do not depend on x)
    for t, c in ((1, 0), (2, 3), (5, 1)):
        h, v = 1e-6, []
        for s in (h, -h):
            xs = x.copy()
            xs[t, c] += s
            v.append(O.head_loss(xs, w, y, wt, None if tau is None else ids, u, tau or 1.0, share)["loss"])
        assert (v[0] - v[1]) / (2 * h) == pytest.approx(ref["dx"][t, c], rel=1e-6, abs=1e-9)


def test_distillation_from_every_logit_is_the_divergence_of_two_softmaxes():
    """With the whole vocabulary listed the loss is the library's KL divergence, and 0 where teacher and student agree."""
    x, w, y, _, _ = problem()
    ids = np.tile(np.arange(23), (7, 1))
    u = np.random.default_rng(1).normal(size=(7, 23))
    ref = O.head_loss(x, w, None, None, ids, u, 2.0, 1.0)
    z = torch.tensor(x @ w.T)
    want = 4.0 * torch.nn.functional.kl_div(torch.log_softmax(z / 2, 1), torch.softmax(torch.tensor(u) / 2, 1), reduction="none").sum(1)
    np.testing.assert_allclose(ref["row_loss"], want.numpy(), rtol=1e-12)
    same = O.head_loss(x, w, None, None, ids, x @ w.T, 2.0, 1.0)
    assert abs(same["loss"]) < 1e-13 and np.abs(same["dx"]).max() < 1e-13


# ------------------------------------------------------------------------------------------------ refusals (all made on the host, before anything is launched)
def head(**over):
    x = 0x1000          # never read: the calls below are refused
    f = dict(x=x, w=x, row_weight=None, loss=x, row_loss=None, row_lse=None, dx=x, dw=x, ldx=64, ldw=64, lddx=64, lddw=64, dtype=pp.PP_BF16, n=10, vocab=100, d=64, dw_lo=0, dw_hi=100,
             dw_f32=0, piece=0)
    f.update(over)
    return pp.PPHead(*[f[k] for k, _ in pp.PPHead._fields_])


@pytest.mark.parametrize("over,text", [
    (dict(dtype=2), "dtype"), (dict(n=-1), "n outside"), (dict(n=(1 << 24) + 1), "n outside"), (dict(vocab=0), "vocab"), (dict(vocab=(1 << 20) + 1), "vocab"), (dict(d=0), "d outside"),
    (dict(d=(1 << 14) + 1, ldx=1 << 15, ldw=1 << 15, lddx=1 << 15, lddw=1 << 15), "d outside"), (dict(dw_lo=-1), "dw rows"), (dict(dw_lo=5, dw_hi=4), "dw rows"), (dict(dw_hi=101), "dw rows"),
    (dict(dw_f32=3), "dw_f32"), (dict(piece=-1), "piece"), (dict(ldx=63), "leading"), (dict(ldw=63), "leading"), (dict(lddx=63), "leading"), (dict(lddw=63), "leading"),
    (dict(x=None), "NULL"), (dict(w=None), "NULL"), (dict(dw=None), "NULL"), (dict(x=0x1001), "aligned"), (dict(w=0x1001), "aligned"), (dict(dx=0x1003), "aligned"),
    (dict(dtype=pp.PP_F32, x=0x1002), "aligned"), (dict(dw=0x1002, dw_f32=1), "aligned")])
def test_bad_heads_are_refused(over, text):
    lib = pp.load_library()
    h = head(**over)
    assert lib.pp_op_head_bytes(ctypes.byref(h), 0) == 0 and text in pp.pp_last_error()
    for call in (lambda: pp.pp_op_head_ce(None, h, 0x1000, 0x1000, 1 << 40), lambda: pp.pp_op_head_distill(None, h, 0x1000, 0x1000, 4, 1.0, 0.5, 0x1000, 0x1000, 1 << 40)):
        with pytest.raises(pp.PPError, match=text):
            call()


def test_bad_calls_are_refused():
    lib = pp.load_library()
    h = head()
    need = pp.pp_op_head_bytes(h)
    assert lib.pp_op_head_bytes(None, 0) == 0
    for top in (-1, pp.PP_HEAD_TOP_MAX + 1):
        with pytest.raises(pp.PPError, match="top"):
            pp.pp_op_head_bytes(h, top)
    with pytest.raises(pp.PPError, match="targets"):
        pp.pp_op_head_ce(None, h, None, 0x1000, need)
    with pytest.raises(pp.PPError, match="needs %d" % need):
        pp.pp_op_head_ce(None, h, 0x1000, 0x1000, need - 1)
    for ws in (None, 0x1080):
        with pytest.raises(pp.PPError, match="256-byte"):
            pp.pp_op_head_ce(None, h, 0x1000, ws, need)
    good = dict(ids=0x1000, logits=0x1000, top=4, tau=1.0, share=0.5, targets=0x1000)

    def distill(**over):
        a = dict(good, **over)
        pp.pp_op_head_distill(None, h, a["ids"], a["logits"], a["top"], a["tau"], a["share"], a["targets"], 0x1000, 1 << 40)
    for over, text in ((dict(top=0), "top"), (dict(top=129), "top"), (dict(tau=0.0), "temperature"), (dict(tau=-1.0), "temperature"), (dict(tau=float("nan")), "temperature"),
                       (dict(tau=65.0), "temperature"), (dict(share=-0.1), "share"), (dict(share=1.1), "share"), (dict(share=float("nan")), "share"), (dict(ids=None), "NULL"),
                       (dict(logits=None), "NULL"), (dict(targets=None), "NULL")):
        with pytest.raises(pp.PPError, match=text):
            distill(**over)


def test_workspace_is_bounded_and_follows_the_options():
    """The piece buffers do not grow with n; no gradient buffers where no gradient is asked for."""
    big = lambda **o: pp.pp_op_head_bytes(head(**dict(dict(n=1 << 20, vocab=128000, d=4096, ldx=4096, ldw=4096, lddx=4096, lddw=4096, dw_lo=0, dw_hi=0, dw=None), **o)))  # noqa: E731
    rows = lambda n: n * (4096 * 2 + 64)  # noqa: E731  -- the copy of X and a few words per row
    assert big(dx=None) <= rows(1 << 20) + (1100 << 20)          # the logits would be 537 GB in fp32
    assert big() - big(n=1 << 19) <= rows(1 << 19)
    assert big(piece=64) < big()
    assert big(dx=None) < big()
    assert pp.pp_op_head_bytes(head(), 64) >= pp.pp_op_head_bytes(head())


def test_make_head_checks_its_tensors():
    bf, f32 = torch.bfloat16, torch.float32
    x, w = torch.zeros((6, 8), dtype=bf), torch.zeros((20, 8), dtype=bf)
    h = pp.make_head(x, w, dw=torch.zeros((5, 8), dtype=f32), dw_lo=3, dw_add=True)
    assert (h.n, h.vocab, h.d, h.dw_lo, h.dw_hi, h.dw_f32, h.ldx) == (6, 20, 8, 3, 8, 2, 8)
    assert pp.make_head(torch.zeros((6, 24), dtype=bf)[:, 8:16], w).ldx == 24
    for bad in (dict(x=x.float()), dict(x=x.half(), w=w.half()), dict(x=torch.zeros((8, 6), dtype=bf).t()), dict(dx=torch.zeros((6, 9), dtype=bf)), dict(dx=torch.zeros((6, 8))),
                dict(dw=torch.zeros((5, 8), dtype=bf), dw_add=True), dict(loss=torch.zeros(2)), dict(row_weight=torch.zeros(6, dtype=torch.float64)), dict(row_loss=torch.zeros(12)[::2]),
                dict(dw=torch.zeros((5, 8), dtype=bf), dw_lo=0, dw_hi=6)):
        args = dict(dict(x=x, w=w), **bad)
        with pytest.raises(pp.PPError, match="make_head"):
            pp.make_head(args.pop("x"), args.pop("w"), **args)


def test_model_without_kept_logits_plans_less_and_takes_larger_vocabularies():
    import pp_inputs as gen
    from paper_2509_22418_amd import binding as b
    cfg = gen.make_config("1p3b")
    ask = lambda c, which=b.PP_BYTES_WORKSPACE: b.pp_query_bytes(b.make_config(c), b.make_mask(gen.ffn_slice_mask(cfg, 0, 32)), which)  # noqa: E731
    kept, pieces = ask(cfg), ask(dict(cfg, head_pieces=1))
    logits = 8 * 2048 * 32000 * 2
    assert kept - pieces >= logits // 4
    assert ask(dict(cfg, head_pieces=1, recompute=1)) < ask(dict(cfg, recompute=1))
    assert ask(dict(cfg, head_pieces=1), b.PP_BYTES_SHADOW) == ask(cfg, b.PP_BYTES_SHADOW)
    for c in (dict(cfg, vocab=128000), dict(gen.make_config("tiny"), vocab=20000)):
        with pytest.raises(pp.PPError, match="vocab"):
            ask(c)
        assert ask(dict(c, head_pieces=1)) > 0
    with pytest.raises(pp.PPError, match="vocab"):
        ask(dict(cfg, vocab=(1 << 20) + 8, head_pieces=1))
    lib = b.load_library()
    for bad in (2, 3, 6, 8, -1):
        c = b.make_config(dict(cfg, recompute=bad))
        assert lib.pp_query_bytes(ctypes.byref(c), None, 0) == 0 and "recompute" in b.pp_last_error()


def test_workspace_is_bounded_for_any_piece():
    """A piece asked for in rows is cut to 2 GiB of logits; smaller ones are as large as asked."""
    size = lambda piece: pp.pp_op_head_bytes(head(n=1 << 18, vocab=1 << 20, d=64, ldx=64, ldw=64, lddx=64, dw_lo=0, dw_hi=0, dw=None, piece=piece), 0)  # noqa: E731
    assert size(1 << 24) == size(1024) > size(960)
    assert size(1 << 24) <= (2 << 30) + (1 << 30)


@pytest.mark.parametrize("over", [dict(dx=0x1000), dict(dx=0x2000), dict(dw=0x1000), dict(dw=0x2000), dict(dw=0x3000)])
def test_gradients_in_the_place_of_operands_are_refused(over):
    h = head(**dict(dict(x=0x1000, w=0x2000, dx=0x3000, dw=0x4000), **over))
    for call in (lambda: pp.pp_op_head_ce(None, h, 0x1000, 0x1000, 1 << 40), lambda: pp.pp_op_head_distill(None, h, 0x1000, 0x1000, 4, 1.0, 0.5, 0x1000, 0x1000, 1 << 40)):
        with pytest.raises(pp.PPError, match="place of another"):
            call()
