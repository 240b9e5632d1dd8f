"""What an AdamW was made with is not replaced without effect."""
import pytest
import torch

import paper_2103_03936_amd as pf


def test_assignments_that_no_step_would_read_raise():
    opt = pf.AdamW.__new__(pf.AdamW)
    opt.lr = opt.steps = opt.betas = opt.params = None  # while it is made
    opt._args = ()
    for name in ("lr", "steps", "betas", "params", "_args"):
        with pytest.raises(AttributeError, match=name):
            setattr(opt, name, 1e-4)
    opt.note = 1  # one's own
    assert opt.note == 1 and opt.lr is None


@pytest.mark.gpu
def test_lr_is_written_into():
    p, g = torch.ones(100, device="cuda"), torch.ones(100, device="cuda")
    opt = pf.AdamW([p], [g], lr=0.1, weight_decay=0.0)
    with pytest.raises(AttributeError):
        opt.lr = 0.5
    opt.lr.fill_(0.5)
    opt.step()
    assert (p - 0.5).abs().max() <= 2.0 ** -20  # the first step has the gradient's sign times lr, less eps
