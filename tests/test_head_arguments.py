"""Arguments of the output head's losses that the binding and the library refuse, and calls next to those that they take.  No GPU: nothing is launched."""
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
