"""The step of a model whose logits are not kept (PP_HEAD_PIECES), with cross entropy and distilled from a teacher's top logits, against the CPU oracle."""
import ctypes

import numpy as np
import pytest
import torch

import pp_inputs as gen
import paper_2509_22418_amd as pp
from oracle import pp_oracle as O
from harness import HP, cosine, segment_slices, make_gpu_model, frozen_bytes_equal, expand_mask

pytestmark = pytest.mark.gpu

MASKS = {
    "ffn_quarter": lambda c: gen.ffn_slice_mask(c, node=1, n_slices=4),
    "all": lambda c: dict(all=1),
    "paper_mlp_heads": lambda c: gen.paper_mlp_mask(c, node=1, n_slices=2, slice_heads=True),
    "lm_head_only": lambda c: dict(gen.ffn_slice_mask(c, 0, 4), ffn_lo=0, ffn_hi=0, train_lm_head=1),
}
SMALL = dict(n_layers=2, d_model=128, n_heads=2, d_ff=256, vocab=512, batch=2, seq=96, dtype="bf16")


def teacher(cfg, tok, tgt, top, seed):
    """The top logits of a model with other weights at every position, as a teacher's files hold them; lists of all lengths."""
    _, cache = O.forward(cfg, O.to_f64(gen.make_weights(cfg, seed=seed, std=0.05)), tok, tgt)
    z = cache["z"] if "z" in cache else cache["nf"] @ O.to_f64(gen.make_weights(cfg, seed=seed, std=0.05))["lm_head"].T
    ids = np.argsort(-z, axis=1, kind="stable")[:, :top].astype(np.int32)
    u = np.take_along_axis(z, ids.astype(np.int64), 1).astype(np.float32)
    r = np.random.default_rng(seed)
    absent = np.arange(top)[None] >= r.integers(0, top + 1, (len(z), 1))
    ids[absent], u[absent] = -1, np.nan
    return ids.reshape(*tok.shape, top), u.reshape(*tok.shape, top)


def compare(cfg, omask, loss, g, loss_ref, g_ref):
    bf16 = cfg["dtype"] == "bf16"
    assert abs(loss - loss_ref) <= (1e-2 if bf16 else 1e-5) * abs(loss_ref), (loss, loss_ref)          # the tolerances of the steps that keep their logits
    for name, off, n in segment_slices(cfg, omask):
        a, b = g[off:off + n], g_ref[off:off + n]
        if not b.any():
            # A sequence of one token: its only score's softmax is 1 and the gradients of q and k are 0 by dS = P (dP - D), dP and D sums of the same dh products with roundings of
            # half a step each (bf16: of O, 2^-8) of size |dO| |v|, the size that dV and with it the value rows' gradient have: far below these shares of the largest gradient.
            assert np.max(np.abs(a)) <= (2.0 ** -6 if bf16 else 1e-4) * np.max(np.abs(g_ref)), name
            continue
        assert cosine(a, b) >= 0.999, (name, cosine(a, b))
        if not bf16:
            assert np.max(np.abs(a - b)) <= 1e-4 * np.max(np.abs(b)) + 1e-9, name


@pytest.mark.parametrize("over", [dict(), SMALL], ids=["f32", "bf16"])
@pytest.mark.parametrize("mname", list(MASKS))
def test_step_without_logits_matches_oracle(mname, over):
    cfg = gen.make_config("tiny", **over)
    weights = gen.make_weights(cfg, seed=1)
    tok, tgt = gen.make_tokens(cfg, seed=1)
    mask = MASKS[mname](cfg)
    omask = expand_mask(cfg, mask)
    print(f"case head step {mname} {cfg['dtype']}", flush=True)
    runs = []
    for extra in (dict(head_pieces=1), dict(head_pieces=1, recompute=1)):
        m = make_gpu_model(dict(cfg, **extra), weights, mask)
        td, gd = m.upload_tokens(tok, tgt)
        loss = float(m.step(td, gd, HP).item())
        runs.append((loss, m.get_state("g"), m.get_state("p")))
        cnt = m.counters()
        assert frozen_bytes_equal(cfg, m, weights, mask) == []
        if cfg["dtype"] == "bf16":
            assert m.launch_counts()["plain_calls"] == 0
        with pytest.raises(pp.PPError, match="not kept"):
            m.get_raw("dbg.logits", (tok.size, cfg["vocab"]), np.uint16 if cfg["dtype"] == "bf16" else np.float32)
        m.close()
    for a, b in zip(*runs):
        assert np.array_equal(a, b)          # with activations recomputed: the same bits
    loss_ref, g_ref = O.LocalTrainer(cfg, weights, omask).step(tok, tgt, HP)
    compare(cfg, omask, runs[0][0], runs[0][1].astype(np.float64), loss_ref, g_ref)
    _, cache = O.forward(cfg, O.to_f64(weights), tok, tgt)
    _, info = O.backward_restricted(cfg, O.to_f64(weights), cache, omask)
    assert cnt["flops_fwd"] == O.flops_forward(cfg, *tok.shape) and cnt["flops_bwd"] == info["flops_bwd"]


@pytest.mark.parametrize("over", [dict(), SMALL], ids=["f32", "bf16"])
@pytest.mark.parametrize("tau,share", [(1.0, 1.0), (1.0, 0.5), (2.0, 0.7)])
def test_distilled_step_matches_oracle(over, tau, share):
    cfg = gen.make_config("tiny", **over)
    weights = gen.make_weights(cfg, seed=4)
    tok, tgt = gen.make_tokens(cfg, seed=4)
    ids, u = teacher(cfg, tok, tgt, 12, seed=9)
    print(f"case distilled step tau={tau} share={share} {cfg['dtype']}", flush=True)
    for mname in ("ffn_quarter", "all"):
        mask = MASKS[mname](cfg)
        omask = expand_mask(cfg, mask)
        m = make_gpu_model(dict(cfg, head_pieces=1), weights, mask)
        td, gd = m.upload_tokens(tok, tgt)
        i_d, u_d = torch.from_numpy(ids).cuda(), torch.from_numpy(u).cuda()
        loss = float(m.step_distill(td, None if share == 1.0 else gd, i_d, u_d, tau, share, None).item())
        loss_ref, g_ref = O.distilled(cfg, O.to_f64(weights), tok, tgt, omask, ids, u, tau, share)
        compare(cfg, omask, loss, m.get_state("g").astype(np.float64), loss_ref, g_ref)
        m.close()


def test_a_run_of_distilled_and_ordinary_steps():
    """Distilled steps, an ordinary one and the scoring of the result on one handle, as a program uses them: three updates track the oracle's."""
    cfg = gen.make_config("tiny")
    weights = gen.make_weights(cfg, seed=5)
    tok, tgt = gen.make_tokens(cfg, seed=5)
    ids, u = teacher(cfg, tok, tgt, 8, seed=11)
    mask = MASKS["all"](cfg)
    omask = expand_mask(cfg, mask)
    m = make_gpu_model(dict(cfg, head_pieces=1), weights, mask)
    td, gd = m.upload_tokens(tok, tgt)
    i_d, u_d = torch.from_numpy(ids).cuda(), torch.from_numpy(u).cuda()
    tr = O.LocalTrainer(cfg, weights, omask)
    for step, kd in enumerate((True, False, True)):
        if kd:
            loss = float(m.step_distill(td, gd, i_d, u_d, 2.0, 0.5, HP).item())
            loss_ref, g = O.distilled(cfg, tr.params, tok, tgt, omask, ids, u, 2.0, 0.5)
            tr.t += 1
            tr.master, tr.m, tr.v = O.adamw_update(tr.master, tr.m, tr.v, g, tr.t, HP["lr"], HP["beta1"], HP["beta2"], HP["eps"], HP["weight_decay"], tr.decay)
            O.unpack_into(tr.params, tr.segs, tr.master)
        else:
            loss = float(m.step(td, gd, HP).item())
            loss_ref, _ = tr.step(tok, tgt, HP)
        assert abs(loss - loss_ref) <= 1e-4 * abs(loss_ref), (step, loss, loss_ref)
    # the trained head scores given hidden states
    w = torch.from_numpy(m.get_weight("lm_head", (cfg["vocab"], cfg["d_model"]))).cuda()
    x = torch.randn((tok.size, cfg["d_model"]), device="cuda")
    rows = torch.empty(tok.size, device="cuda")
    h = pp.make_head(x, w, row_loss=rows)
    ws = torch.empty(pp.pp_op_head_bytes(h), dtype=torch.uint8, device="cuda")
    pp.pp_op_head_ce(torch.cuda.current_stream().cuda_stream, h, gd.data_ptr(), ws.data_ptr(), ws.numel())
    want = O.head_loss(x.cpu().numpy(), w.cpu().numpy(), tgt.reshape(-1))["row_loss"]
    assert np.max(np.abs(rows.cpu().numpy() - want)) <= 1e-4
    m.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_batches_smaller_than_planned(dtype):
    """One handle, batches from one token to its whole size (the kernels of few rows among them): each equals a handle of its own size, and the workspace suffices for all."""
    cfg = gen.make_config("tiny", **dict(SMALL, dtype=dtype))
    weights = gen.make_weights(cfg, seed=6)
    tok, tgt = gen.make_tokens(cfg, seed=6)
    mask = MASKS["all"](cfg)
    m = make_gpu_model(dict(cfg, head_pieces=1), weights, mask)
    m.ws[:] = 0xFF
    m.h = pp.pp_init_model(m.ccfg, m.params.data_ptr(), m.bytes_params, m.ws.data_ptr(), m.bytes_ws, m.stream.cuda_stream)
    m.set_mask()
    for b, s in ((1, 1), (1, 16), (2, 33), (2, 96)):
        print(f"case head step batch {b}x{s} {dtype}", flush=True)
        t, g = tok[:b, :s].copy(), tgt[:b, :s].copy()
        td, gd = m.upload_tokens(t, g)
        loss = float(m.step(td, gd, None).item())
        loss_ref, g_ref = O.LocalTrainer(cfg, weights, expand_mask(cfg, mask)).step(t, g, HP)
        compare(cfg, expand_mask(cfg, mask), loss, m.get_state("g").astype(np.float64), loss_ref, g_ref)
    m.close()


def test_vocabulary_beyond_the_kept_logits():
    """Vocabularies that the kernels of kept logits refuse."""
    for dtype, vocab in (("bf16", 70000), ("f32", 20000)):
        cfg = gen.make_config("tiny", n_layers=1, d_model=64, n_heads=1, d_ff=64, vocab=vocab, batch=1, seq=40, dtype=dtype)
        with pytest.raises(pp.PPError, match="vocab"):
            pp.LocalStepModel(cfg, dict(ffn_lo=0, ffn_hi=32))
        weights = gen.make_weights(cfg, seed=2)
        tok, tgt = gen.make_tokens(cfg, seed=2)
        mask = dict(gen.ffn_slice_mask(cfg, 0, 2), train_lm_head=1)
        m = make_gpu_model(dict(cfg, head_pieces=1), weights, mask)
        td, gd = m.upload_tokens(tok, tgt)
        loss = float(m.step(td, gd, None).item())
        loss_ref, g_ref = O.LocalTrainer(cfg, weights, mask).step(tok, tgt, HP)
        compare(cfg, mask, loss, m.get_state("g").astype(np.float64), loss_ref, g_ref)
        m.close()


def test_refusals():
    cfg = gen.make_config("tiny")
    lib = pp.load_library()
    for pieces, text in ((0, "PP_HEAD_PIECES"), (1, None)):
        m = make_gpu_model(dict(cfg, head_pieces=pieces), gen.make_weights(cfg, 1), MASKS["all"](cfg))
        tok, tgt = gen.make_tokens(cfg, 1)
        td, gd = m.upload_tokens(tok, tgt)
        i_d = torch.zeros((*tok.shape, 4), dtype=torch.int32, device="cuda")
        u_d = torch.zeros((*tok.shape, 4), device="cuda")
        if text:
            with pytest.raises(pp.PPError, match=text):
                m.step_distill(td, gd, i_d, u_d, 1.0, 0.5, None)
            m.close()
            continue
        for tau, share, word in ((0.0, 0.5, "temperature"), (1.0, 1.5, "share"), (float("nan"), 0.5, "temperature")):
            with pytest.raises(pp.PPError, match=word):
                m.step_distill(td, gd, i_d, u_d, tau, share, None)
        with pytest.raises(pp.PPError, match="NULL"):
            m.step_distill(td, None, i_d, u_d, 1.0, 0.5, None)
        with pytest.raises(pp.PPError, match="step_distill"):
            m.step_distill(td, gd, i_d.long(), u_d, 1.0, 0.5, None)
        assert lib.pp_local_step_distill(m.h, td.data_ptr(), gd.data_ptr(), *tok.shape, i_d.data_ptr(), u_d.data_ptr(), 129, 1.0, 0.5, None, m.loss.data_ptr()) == -1
        assert lib.pp_local_step_distill(None, td.data_ptr(), gd.data_ptr(), *tok.shape, i_d.data_ptr(), u_d.data_ptr(), 4, 1.0, 0.5, None, m.loss.data_ptr()) == -1
        assert lib.pp_local_step_distill(m.h, td.data_ptr(), gd.data_ptr(), 5, 32, i_d.data_ptr(), u_d.data_ptr(), 4, 1.0, 0.5, None, m.loss.data_ptr()) == -1
        opt = pp.PPAdamW(1e-3, 1.5, 0.95, 1e-8, 0.1)
        assert lib.pp_local_step_distill(m.h, td.data_ptr(), gd.data_ptr(), *tok.shape, i_d.data_ptr(), u_d.data_ptr(), 4, 1.0, 0.5, ctypes.byref(opt), m.loss.data_ptr()) == -1
        m.close()
