"""Sums, norms and gathered sums lie apart from the tensors of a clipping plan: what one of its calls writes is nothing that it
or the next one reads."""
import pytest
import torch

import paper_2109_08751_b200 as sp
from test_train_clip import Case
from test_train_host import refused

pytestmark = pytest.mark.gpu


def test_sums_and_norms_in_tensors_are_refused():
    c = Case([70000, 3, 20000], ["bf16", "f32", "f32"], [1, 0, 1], 2)
    x, y = c.grads[2], c.out[2]
    before = [t.clone() for t in c.grads]
    refused(sp.ERR_ALIAS, c.plan.sums, x.data_ptr())
    refused(sp.ERR_ALIAS, c.plan.sums, x.data_ptr() + 4 * 20000 - 8)
    refused(sp.ERR_ALIAS, c.plan.sums, c.grads[0].data_ptr() - 8)
    scale = lambda gathered, norms: c.plan.scale(gathered, 2, 1.0, norms)  # noqa: E731
    refused(sp.ERR_ALIAS, scale, c.gathered, x.data_ptr())
    refused(sp.ERR_ALIAS, scale, c.gathered, y.data_ptr() + 4 * 20000 - 4)
    refused(sp.ERR_ALIAS, scale, y.data_ptr(), c.norms)
    refused(sp.ERR_ALIAS, scale, y.data_ptr() - 24, c.norms)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, c.grads))
    # between the tensors, and where gathered sums are only read beside what is only read, they may lie
    c.plan.sums(c.grads[0].data_ptr() - 16)
    c.plan.set_tensors(c.grads)
    refused(sp.ERR_ALIAS, c.plan.sums, x.data_ptr())
    refused(sp.ERR_ALIAS, scale, c.gathered, x.data_ptr())
    c.plan.scale(c.gathered, 2, 1.0, y.data_ptr())
