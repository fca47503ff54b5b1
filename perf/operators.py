"""Cases of the output head's losses: softmax cross entropy and distillation from a teacher's top logits, both over the product of hidden states and
head weights with its gradients, without the logits being kept.

With z = X W^T, X [n x d] the final hidden states and W [vocab x d] the head:
  ce       l_t = lse(z_t) - z_t[y_t];  rows with a target outside [0, vocab) are left out
  distill  l_t = (1 - share) CE_t + share tau^2 KL(q_t || softmax(z_t / tau)),  q_t = softmax(u_t / tau) over the teacher's listed entries (an index outside
           [0, vocab) is no entry, equal indices add up); a row without entries has no KL, one without a target no CE, one without both is left out
loss = sum_t w_t l_t, w_t the row weights or 1 / (rows that are not left out); gradients of that loss for X and for the rows [dw_lo, dw_hi) of W.
Outputs: loss, row_loss (l_t, 0 where left out), row_lse (log-sum-exp of z_t / tau, tau = 1 for ce, 0 where left out), and dx, dw where the case asks for them.

A case is a dict of plain values: n, vocab, d, dtype, dx (truth value), dw_lo, dw_hi (equal: no weight gradient), ignored (share of rows without target), weights (row
weights given), top (entries per row, 0: ce), tau, share, ragged (lists of all lengths from none to top).
"""
import math

import torch

own = False


# ------------------------------------------------------------------------------------------------ the cases
def _case(name, n, vocab, d, dtype, dx=True, dw=(0, 0), ignored=0.0, weights=False, top=0, tau=1.0, share=1.0, ragged=False):
    c = dict(n=n, vocab=vocab, d=d, dtype=dtype, dx=dx, dw_lo=dw[0], dw_hi=dw[1], ignored=ignored, weights=weights, top=top, tau=tau, share=share, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest training call: the 2 x 64 model's batch of 4 x 32 tokens in fp32, head trainable
        _case("ce_tiny_f32", 128, 256, 64, "f32", dw=(0, 256)),
        # scoring one token (its log-probability): no gradients
        _case("ce_one_token", 1, 32000, 2048, "bf16", dx=False),
        # evaluation of one odd-sized text over an odd vocabulary: losses alone
        _case("ce_eval_odd", 611, 50257, 768, "bf16", dx=False),
        # the 125M-shape step's head with every weight trainable
        _case("ce_125m_all", 8192, 32000, 768, "bf16", dw=(0, 32000)),
        # the headline's head: 8 x 2048 tokens, 1.3B width, head frozen, one position per sequence without target
        _case("ce_1p3b_frozen", 16384, 32000, 2048, "bf16", ignored=1.0 / 2048),
        # instruction tuning: most positions are prompt or padding and have no target, weights per token, a slice of the head trainable
        _case("ce_masked_slice", 8192, 32000, 2048, "bf16", dw=(4000, 8000), ignored=0.6, weights=True),
        # a vocabulary of the size that made this operator: the logits would be 2 GB in fp32
        _case("ce_large_vocab", 4096, 128000, 4096, "bf16", dw=(0, 128000)),
        # a reference run in fp32 storage and arithmetic
        _case("ce_small_f32", 1024, 8000, 512, "f32", dw=(0, 8000), ignored=0.1),
        # distillation at temperature 2 in fp32, a short odd batch, lists of all lengths
        _case("distill_small_f32", 500, 8000, 512, "f32", dw=(0, 8000), top=16, tau=2.0, ragged=True),
        # the 1.3B head distilled from 64 logits per token, half the loss from the hard targets, head frozen
        _case("distill_1p3b", 8192, 32000, 2048, "bf16", ignored=1.0 / 2048, top=64, share=0.5),
        # the 125M shape, temperature 2 beside hard targets (two softmaxes of the same logits), ragged batch and lists, head trainable
        _case("distill_mixed_tau", 3055, 32000, 768, "bf16", dw=(0, 32000), ignored=0.2, top=32, tau=2.0, share=0.7, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: both losses in equal parts, sizes spread over their logarithm, odd ones among them."""
    while True:
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        n, vocab, d = _log(rng, 1, 16384), _log(rng, 200, 128000), _log(rng, 48, 4096)
        if rng.random() < 0.6:
            d = max(64, d // 64 * 64)
        if rng.random() < 0.5:
            vocab = max(8, vocab // 8 * 8)
        lo = rng.randint(0, vocab - 1)
        dw = rng.choice([(0, 0), (0, vocab), (lo, rng.randint(lo + 1, vocab))])
        top = rng.choice([0, _log(rng, 1, 128)])
        c = _case(None, n, vocab, d, dtype, dx=rng.random() < 0.75, dw=dw, ignored=rng.choice([0.0, 0.1, 0.5]), weights=rng.random() < 0.3, top=top,
                  tau=rng.choice([1.0, round(rng.uniform(0.5, 4.0), 2)]) if top else 1.0, share=rng.choice([1.0, round(rng.uniform(0.1, 0.9), 2)]) if top else 1.0,
                  ragged=rng.random() < 0.5 and top > 0)
        flops = work(c)["flops"]
        if flops > (3e11 if dtype == "f32" else 4e12):
            continue
        return c


def work(case):
    """x and w read once, gradients and row outputs written once; one product for the losses, one for dx, the slice's part of one for dw, over the rows that count."""
    c, es = case, 4 if case["dtype"] == "f32" else 2
    n, vocab, d, rows = c["n"], c["vocab"], c["d"], c["dw_hi"] - c["dw_lo"]
    live = n if c["top"] else max(1, round(n * (1.0 - c["ignored"])))
    grads = (vocab if c["dx"] else 0) + rows
    return dict(bytes=es * (live * d + vocab * d + (n * d if c["dx"] else 0) + rows * d) + 12 * n + 8 * n * c["top"], flops=2 * live * d * (vocab + grads))


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed(1000003 * (seed + 1) + stream)


def _zipf(vocab, shape, seed, stream):
    p = torch.arange(1, vocab + 1, dtype=torch.float64, device="cuda").pow_(-1.1)
    cdf = torch.cumsum(p, 0)
    u = torch.rand(shape, dtype=torch.float64, device="cuda", generator=_gen(seed, stream)) * cdf[-1]
    return torch.searchsorted(cdf, u).clamp_(max=vocab - 1).to(torch.int32)


def _inputs(c, seed):
    """Hidden states of unit variance that lean towards their target's weights by a random amount (a model somewhere in its training), weights N(0, 0.02), Zipf(1.1)
    targets, the teacher's logits in falling order with the target first in most rows; absent entries hold NaN."""
    n, vocab, d, dt = c["n"], c["vocab"], c["d"], torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    w = torch.empty((vocab, d), device="cuda").normal_(0.0, 0.02, generator=_gen(seed, 1)).to(dt)
    y = _zipf(vocab, (n,), seed, 2)
    wt = w[y.long()].float()
    lean = torch.rand((n, 1), device="cuda", generator=_gen(seed, 3)) * min(10.0, 0.08 * d)
    x = (torch.randn((n, d), device="cuda", generator=_gen(seed, 4)) + lean * wt / wt.square().sum(1, keepdim=True)).to(dt)
    s = dict(case=c, x=x, w=w)
    if c["top"]:
        ids = _zipf(vocab, (n, c["top"]), seed, 5)
        ids[:, 0] = torch.where(torch.rand(n, device="cuda", generator=_gen(seed, 6)) < 0.7, y, ids[:, 0])
        u = torch.sort(2.5 * torch.randn((n, c["top"]), device="cuda", generator=_gen(seed, 7)), dim=1, descending=True).values
        if c["ragged"]:
            length = torch.randint(0, c["top"] + 1, (n, 1), device="cuda", generator=_gen(seed, 8))
            absent = torch.arange(c["top"], device="cuda")[None] >= length
            ids, u = ids.masked_fill(absent, -1), u.masked_fill(absent, math.nan)
        s["ids"], s["u"] = ids.contiguous(), u.contiguous()
    out = torch.rand(n, device="cuda", generator=_gen(seed, 9)) < c["ignored"]
    s["targets"] = torch.where(out, torch.full_like(y, -1), y)
    s["weights"] = torch.rand(n, device="cuda", generator=_gen(seed, 10)) / n if c["weights"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:          # the output buffers and the workspace that a program keeps from call to call
        import paper_2509_22418_amd as pp
        c, dev, dt = case, "cuda", s["x"].dtype
        out = dict(loss=torch.empty(1, device=dev), row_loss=torch.empty(c["n"], device=dev), row_lse=torch.empty(c["n"], device=dev))
        if c["dx"]:
            out["dx"] = torch.empty((c["n"], c["d"]), dtype=dt, device=dev)
        if c["dw_hi"] > c["dw_lo"]:
            out["dw"] = torch.empty((c["dw_hi"] - c["dw_lo"], c["d"]), dtype=dt, device=dev)
        s["head"] = pp.make_head(s["x"], s["w"], row_weight=s["weights"], dw_lo=c["dw_lo"], dw_hi=c["dw_hi"], **out)
        s["ws"] = torch.empty(pp.pp_op_head_bytes(s["head"], c["top"]), dtype=torch.uint8, device=dev)
        s["out"], s["stream"] = out, torch.cuda.current_stream().cuda_stream
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2509_22418_amd as pp
        if c["top"]:
            pp.pp_op_head_distill(s["stream"], s["head"], s["ids"].data_ptr(), s["u"].data_ptr(), c["top"], c["tau"], c["share"], s["targets"].data_ptr() if c["share"] < 1.0 else None,
                                  s["ws"].data_ptr(), s["ws"].numel())
        else:
            pp.pp_op_head_ce(s["stream"], s["head"], s["targets"].data_ptr(), s["ws"].data_ptr(), s["ws"].numel())
        return s["out"]
    return _plain(s, c)


def _softmax(z):
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    t = e.sum(1, keepdim=True)
    return e / t, (m + torch.log(t))[:, 0]


def _plain(s, c):
    x, w, y = s["x"].float(), s["w"].float(), s["targets"].long()
    tau, share = (c["tau"], c["share"]) if c["top"] else (1.0, 0.0)
    hard = (y >= 0) if share < 1.0 else torch.zeros_like(y, dtype=torch.bool)
    at = y.clamp(min=0)[:, None]
    z = x @ w.T
    p, lse = _softmax(z / tau)
    row, lse_out, grads = torch.zeros_like(lse), lse, c["dx"] or c["dw_hi"] > c["dw_lo"]
    dz = torch.zeros_like(z) if grads else None
    live = hard
    if c["top"]:
        there = s["ids"] >= 0
        ids = s["ids"].long().clamp(min=0)
        soft = there.any(1)
        u = torch.where(there, s["u"] / tau, -math.inf)
        q = torch.where(there, torch.exp(u - torch.where(soft, u.amax(1), 0.0)[:, None]), 0.0)
        q = q / torch.where(soft, q.sum(1), 1.0)[:, None]
        kl = torch.where(q > 0, q * (torch.log(q) - z.gather(1, ids) / tau + lse[:, None]), 0.0).sum(1)
        row += share * tau * tau * torch.where(soft, kl, 0.0)
        if grads:
            dz += torch.where(soft, share * tau, 0.0)[:, None] * p
            dz.scatter_add_(1, ids, -share * tau * q)
        live = live | soft
        if share < 1.0 and tau != 1.0:
            p, lse = _softmax(z)
    if share < 1.0:
        row += torch.where(hard, (1.0 - share) * (lse - z.gather(1, at)[:, 0]), 0.0)
        if grads:
            dz += torch.where(hard, 1.0 - share, 0.0)[:, None] * p
            dz.scatter_add_(1, at, torch.where(hard, share - 1.0, 0.0)[:, None])
    g = s["weights"] if s["weights"] is not None else 1.0 / live.sum().clamp(min=1).float()
    g = torch.where(live, g, 0.0)
    out = dict(loss=(g * row).sum()[None], row_loss=row, row_lse=torch.where(live, lse_out, 0.0))
    if grads:
        dz *= g[:, None]
    if c["dx"]:
        out["dx"] = (dz @ w).to(s["x"].dtype)
    if c["dw_hi"] > c["dw_lo"]:
        out["dw"] = (dz[:, c["dw_lo"]:c["dw_hi"]].T @ x).to(s["w"].dtype)
    return out


# ------------------------------------------------------------------------------------------------ 64-bit values
def exact(case, seed):
    """The loss as its definition has it, differentiated by torch in 64 bits, some rows at a time."""
    c, s = case, _inputs(case, seed)
    n, w = c["n"], s["w"].double().requires_grad_(c["dw_hi"] > c["dw_lo"])
    hard_share = 1.0 - c["share"] if c["top"] else 1.0
    none = torch.zeros(n, dtype=torch.bool, device="cuda")
    hard = s["targets"] >= 0 if hard_share > 0 else none
    soft = (s["ids"] >= 0).any(1) if c["top"] else none
    live = hard | soft
    g = (s["weights"].double() if s["weights"] is not None else torch.full((n,), 1.0 / max(1, int(live.sum())), dtype=torch.float64, device="cuda")) * live
    loss, rows, lses, dxs = 0.0, [], [], []
    for a in range(0, n, 2048):
        b = min(n, a + 2048)
        x = s["x"][a:b].double().requires_grad_(c["dx"])
        z = torch.matmul(x, w.T)
        lse = torch.logsumexp(z / c["tau"], 1)
        row = torch.zeros(b - a, dtype=torch.float64, device="cuda")
        if hard_share > 0:
            nll = torch.nn.functional.cross_entropy(z, s["targets"][a:b].long(), ignore_index=-1, reduction="none")
            row = row + hard_share * nll
        if c["top"]:
            ids, there = s["ids"][a:b].long(), s["ids"][a:b] >= 0
            u = torch.where(there, s["u"][a:b].double(), torch.full((), -1e300, dtype=torch.float64, device="cuda"))
            logq = torch.log_softmax(u / c["tau"], 1)
            logp = z.gather(1, ids.clamp(min=0)) / c["tau"] - lse[:, None]
            row = row + c["share"] * c["tau"] ** 2 * torch.where(there, logq.exp() * (logq - logp), 0.0).sum(1)
        part = (g[a:b] * row).sum()
        if c["dx"] or w.requires_grad:
            part.backward()
        loss += float(part.detach())
        rows.append(row.detach())
        lses.append(torch.where(live[a:b], lse.detach(), 0.0))
        dxs.append(x.grad)
    out = dict(loss=torch.tensor([loss], dtype=torch.float64), row_loss=torch.cat(rows), row_lse=torch.cat(lses))
    if c["dx"]:
        out["dx"] = torch.cat(dxs)
    if c["dw_hi"] > c["dw_lo"]:
        out["dw"] = w.grad[c["dw_lo"]:c["dw_hi"]]
    return out
