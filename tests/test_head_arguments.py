"""Arguments of the output head's losses that the binding and the library refuse, and calls next to those that they take.  No GPU: nothing is launched."""
import ctypes
import random
import types

import pytest
import torch

import paper_2509_22418_amd as pp


def holder():
    """A LocalStepModel without a handle: what its checks let through ends in the library's refusal of the NULL handle."""
    m = pp.LocalStepModel.__new__(pp.LocalStepModel)
    m.torch, m.h, m.dev, m.loss = torch, None, torch.device("cpu"), torch.zeros(1)
    return m


def distill_args(**over):
    i32 = torch.int32
    return dict(dict(tokens_dev=torch.zeros((2, 5), dtype=i32), targets_dev=torch.zeros((2, 5), dtype=i32), ids_dev=torch.zeros((2, 5, 3), dtype=i32), logits_dev=torch.zeros((2, 5, 3)),
                     temperature=1.0, share=0.5, hp=None), **over)


@pytest.mark.parametrize("over", [dict(), dict(targets_dev=None, share=1.0), dict(targets_dev=torch.zeros(3), share=1.0)])
def test_distilled_step_passes_its_tensors_on(over):
    with pytest.raises(pp.PPError, match="pp_local_step_distill: NULL pointer"):
        holder().step_distill(**distill_args(**over))


@pytest.mark.parametrize("name,bad", [
    ("tokens", torch.zeros((2, 5), dtype=torch.int64)), ("tokens", torch.zeros((2, 4), dtype=torch.int32)), ("tokens", torch.zeros((5, 2), dtype=torch.int32).t()),
    ("targets", torch.zeros((2, 5), dtype=torch.int64)), ("targets", torch.zeros((10,), dtype=torch.int32)), ("targets", torch.zeros((5, 2), dtype=torch.int32).t()),
    ("ids", torch.zeros((2, 5, 3), dtype=torch.int64)), ("ids", torch.zeros((10, 3), dtype=torch.int32)), ("ids", torch.zeros((2, 5, 6), dtype=torch.int32)[:, :, ::2]),
    ("logits", torch.zeros((2, 5, 3), dtype=torch.float64)), ("logits", torch.zeros((2, 5, 4))), ("logits", torch.zeros((2, 3, 5)).transpose(1, 2))])
def test_distilled_step_refuses_other_tensors(name, bad):
    with pytest.raises(pp.PPError, match=f"step_distill: {name}"):
        holder().step_distill(**distill_args(**{name + "_dev": bad}))


@pytest.mark.parametrize("name", ["tokens", "targets", "ids", "logits"])
def test_distilled_step_refuses_tensors_of_another_device(name):
    a = distill_args()
    a[name + "_dev"] = a[name + "_dev"].to("meta")
    with pytest.raises(pp.PPError, match=f"step_distill: {name}"):
        holder().step_distill(**a)


# ------------------------------------------------------------------------------------------------ operands in each other's place
def rows_overlap(*a):
    f = pp.load_library()["_ZN2pp12rows_overlapEPKvmmmS1_mmm"]
    f.restype, f.argtypes = ctypes.c_bool, 2 * [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_size_t]
    return f(*a)


def test_overlap_of_rows_is_exact():
    """Against sets of bytes: rows of all pitches, equal ones (column ranges of one buffer) among them, none and one row."""
    r = random.Random(0)
    seen = [0, 0]
    for k in range(6000):
        a, b = ([r.randint(1, 80), r.randint(0, 6), 0, r.randint(0, 7)] for _ in range(2))
        for v in (a, b):
            v[2] = v[1] + r.randint(0, 9)
        if k % 2:          # one buffer
            a[2] = b[2] = max(a[2], b[2])
        p, q = ({v[0] + i * v[2] + c for i in range(v[3]) for c in range(v[1])} for v in (a, b))
        assert rows_overlap(*a, *b) == bool(p & q), (a, b)
        seen[bool(p & q)] += 1
    assert min(seen) > 1000
    big = 1 << 40          # 2^24 rows of 2^31 elements
    assert not rows_overlap(big, 64, 1 << 33, 1 << 24, big + 64, 64, 1 << 33, 1 << 24)
    assert rows_overlap(big, 65, 1 << 33, 1 << 24, big + 64, 64, 1 << 33, 1 << 24)


M = 1 << 20
PLACES = dict(x=1 * M, w=2 * M, row_weight=3 * M, loss=4 * M, row_loss=5 * M, row_lse=6 * M, dx=7 * M, dw=8 * M)
SIZES = dict(x=10 * 128, w=100 * 128, row_weight=40, loss=4, row_loss=40, row_lse=40, dx=10 * 128, dw=100 * 128)
CALL = dict(targets=9 * M, ids=10 * M, logits=11 * M)
ROWS = [("dx", "x"), ("dx", "w"), ("dx", "row_weight"), ("dx", "targets"), ("dx", "ids"), ("dx", "logits"), ("dx", "dw"), ("dx", "row_loss"), ("dx", "row_lse"), ("dx", "loss"), ("dw", "x"), ("dw", "w"),
        ("dw", "row_weight"), ("dw", "targets"), ("dw", "logits"), ("dw", "row_lse"), ("row_loss", "row_weight"), ("row_loss", "targets"), ("row_lse", "logits"), ("row_lse", "x"), ("loss", "ids"),
        ("loss", "row_weight")] + [("workspace", k) for k in ("x", "w", "row_weight", "loss", "row_loss", "row_lse", "dx", "dw", "targets", "ids", "logits")]


@pytest.mark.parametrize("first,second", ROWS)
def test_operands_that_share_bytes_are_refused(first, second):
    """The first operand's last four bytes on the second's first ones, and the other way around."""
    for swap in (False, True):
        at = dict(PLACES, **CALL, workspace=16 * M)
        size = dict(SIZES, targets=40, ids=160, logits=160)
        if first == "workspace":          # aligned: it begins 256 bytes behind the beginning of a large operand, or it holds the other
            at[second] = at["workspace"] - (256 if swap and size[second] > 256 else -512)
        elif swap:
            at[first] = at[second] + size[second] - 4
        else:
            at[first] = at[second] - size[first] + 4
        h = pp.PPHead(*[at[k] for k in ("x", "w", "row_weight", "loss", "row_loss", "row_lse", "dx", "dw")], 64, 64, 64, 64, pp.PP_BF16, 10, 100, 64, 0, 100, 0, 0)
        with pytest.raises(pp.PPError, match="place of another operand") as e:
            pp.pp_op_head_distill(None, h, at["ids"], at["logits"], 4, 1.0, 0.5, at["targets"], at["workspace"], 1 << 40)
        assert first in str(e.value) and second in str(e.value)


@pytest.mark.parametrize("over", [dict(dx=M + 128), dict(dx=M + 64 * 128 // 2 + 1200), dict(dw=2 * M - 128), dict(dw=2 * M + 128 * 50)])
def test_gradients_that_begin_inside_an_operand_are_refused(over):
    at = dict(PLACES, **over)
    h = pp.PPHead(*[at[k] for k in ("x", "w", "row_weight", "loss", "row_loss", "row_lse", "dx", "dw")], 128, 64, 64, 64, pp.PP_BF16, 40, 100, 64, 0, 100, 0, 0)
    with pytest.raises(pp.PPError, match="place of another operand"):
        pp.pp_op_head_ce(None, h, 9 * M, 16 * M, 1 << 40)


# ------------------------------------------------------------------------------------------------ the step's workspace
def test_no_batch_needs_more_workspace_than_the_largest():
    """A model plans its head's workspace once, for max_batch x max_seq tokens and the longest lists: every smaller batch, list and set of gradients has to fit."""
    f = pp.load_library()["_ZN2pp15step_head_bytesERK9pp_configbbii"]
    f.restype, f.argtypes = ctypes.c_size_t, [ctypes.c_void_p, ctypes.c_bool, ctypes.c_bool, ctypes.c_int, ctypes.c_int]
    r = random.Random(1)
    for dtype in (pp.PP_F32, pp.PP_BF16):
        for vocab, d, most in [(8, 8, 40000), (512, 128, 1 << 18), (8000, 512, 9000), (20000, 64, 5000), (32000, 768, 16384), (32000, 2048, 16384), (50264, 776, 5000), (128000, 4096, 8192), (1 << 20, 1 << 14, 4096),
                               (1 << 20, 64, 1 << 15)] + [(8 * r.randint(1, 20000), 8 * r.randint(1, 512), r.randint(1, 20000)) for _ in range(30)]:
            c = pp.PPConfig(1, d, 1, 8, vocab, 1, most, dtype, 1e-5, 1e4, pp.PP_HEAD_PIECES)
            for trained in (False, True):
                planned = f(ctypes.byref(c), trained, True, most, pp.PP_HEAD_TOP_MAX)
                sizes = {1, 16, 17, 64, 65, 256, 257, most, most - 1, *(int(most ** r.random()) for _ in range(20)), *(r.randint(1, most) for _ in range(20))}
                for n in sizes:
                    for dw, dx, top in ((trained, True, 0), (trained, False, 128), (trained, True, r.randint(1, 128)), (False, False, 0), (False, True, r.choice((1, 2, 8, 64, 128)))):
                        if 0 < n <= most:
                            assert f(ctypes.byref(c), dw, dx, n, top) <= planned, (dtype, vocab, d, most, trained, n, dw, dx, top)


def stated(dtype, vocab, d, tokens, trained):
    """What include/pp.h says PP_HEAD_PIECES holds, in bytes."""
    up = lambda v, m: -(-v // m) * m  # noqa: E731
    bf, es = dtype == pp.PP_BF16, 2 if dtype == pp.PP_BF16 else 4
    rows = min(up(tokens, 64), max(256, (256 << 20) // (vocab * es) // 256 * 256))
    logits = rows * up(vocab, 64 if bf else 128) * es
    wide = up(d, 64 if bf else 4)
    total = logits + (64 << 20) + up(tokens, 64) * wide * es
    if bf:
        return total + logits // 5 + 1100 * up(tokens, 64) + (rows * wide * es if trained else 0) + (vocab * wide * es if d % 64 else 0)
    total += d * up(vocab, 128) * es if vocab % 128 else 0
    return total + (max(0, vocab * d * es - (64 << 20)) if trained and rows < tokens else 0)


@pytest.mark.parametrize("dtype", [pp.PP_F32, pp.PP_BF16])
def test_the_head_takes_what_the_header_says(dtype):
    f = pp.load_library()["_ZN2pp15step_head_bytesERK9pp_configbbii"]
    f.restype, f.argtypes = ctypes.c_size_t, [ctypes.c_void_p, ctypes.c_bool, ctypes.c_bool, ctypes.c_int, ctypes.c_int]
    for vocab, d, tokens in [(512, 128, 192), (8000, 512, 9000), (20000, 64, 5000), (32000, 768, 16384), (32000, 2048, 16384), (50264, 776, 5000), (128000, 4096, 8192), (1 << 20, 64, 1 << 15),
                             (1 << 20, 1 << 14, 4096), (1 << 20, 4096, 200), (40000, 1000, 1 << 17)]:
        c = pp.PPConfig(1, d, 1, 8, vocab, 1, tokens, dtype, 1e-5, 1e4, pp.PP_HEAD_PIECES)
        for trained in (False, True):
            size, said = f(ctypes.byref(c), trained, True, tokens, pp.PP_HEAD_TOP_MAX), stated(dtype, vocab, d, tokens, trained)
            assert said * 0.9 <= size <= said * 1.005 + (2 << 20), (vocab, d, tokens, trained, size >> 20, said >> 20)


# ------------------------------------------------------------------------------------------------ make_head
def meta(rows, cols, pitch=None):
    return torch.empty_strided((rows, cols), (pitch or cols, 1), dtype=torch.bfloat16, device="meta")


@pytest.mark.parametrize("x,w,over,text", [
    (meta((1 << 32) + 5, 8), meta(20, 8), {}, "rows of x"), (meta(6, 8), meta((1 << 32) + 20, 8), {}, "rows of w"), (meta(6, 8, (1 << 32) + 8), meta(20, 8), {}, "stride of x"),
    (meta(6, 8), meta(20, 8, 1 << 31), {}, "stride of w"), (meta(6, 8), meta(20, 8), dict(dx=meta(6, 8, 1 << 33)), "stride of dx"), (meta(6, 8), meta(20, 8), dict(dw=meta(20, 8, 1 << 33)), "stride of dw"),
    (meta(6, 8), meta(20, 8), dict(piece=1 << 32), "piece"), (meta(6, 8), meta(20, 8), dict(dw_lo=1 << 32, dw_hi=(1 << 32) + 3, dw=meta(3, 8)), "dw_lo")])
def test_sizes_beyond_32_bits_are_refused_and_not_cut(x, w, over, text):
    with pytest.raises(pp.PPError, match=f"make_head: {text}"):
        pp.make_head(x, w, **over)


def test_largest_strides_are_taken():
    h = pp.make_head(meta(6, 8, (1 << 31) - 1), meta(20, 8, (1 << 31) - 1))
    assert (h.ldx, h.ldw) == ((1 << 31) - 1, (1 << 31) - 1)


def test_single_columns_have_no_stride():
    """The stride of a dimension of one element says nothing: a column of a wider tensor, one row weight, the column that a transposed row is."""
    bf = torch.bfloat16
    h = pp.make_head(torch.zeros((6, 8), dtype=bf)[:, 3:4], torch.zeros((1, 20), dtype=bf).t(), row_weight=torch.zeros(6))
    assert (h.n, h.vocab, h.d, h.ldx, h.ldw) == (6, 20, 1, 8, 1)
    h = pp.make_head(torch.zeros((1, 8), dtype=bf), torch.zeros((20, 8), dtype=bf), row_weight=torch.zeros(12)[::12], loss=torch.zeros(5)[::5])
    assert (h.n, h.ldx) == (1, 8)


def test_tensors_of_another_device_than_the_current_one_are_refused(monkeypatch):
    """With the default stream the library cannot tell: its kernels would run on the current device."""
    h = pp.make_head(torch.zeros((6, 8)), torch.zeros((20, 8)))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    calls = (lambda: pp.pp_op_head_ce(None, h, 0x1000, None, 0), lambda: pp.pp_op_head_distill(None, h, 0x1000, 0x1000, 4, 1.0, 0.5, 0x1000, None, 0))
    for index, text in ((1, "current device"), (0, "256-byte")):          # on the current one the call reaches the library, which refuses its missing workspace
        h.tensors = (types.SimpleNamespace(is_cuda=True, device=torch.device("cuda", index)),)
        for call in calls:
            with pytest.raises(pp.PPError, match=text):
                call()
