"""Plans of different sizes on host threads of their own: a plan belongs to one thread at a time, and what one thread's plan
needs (f32: as much shared memory as its sizes take) is nothing to another's."""
import threading

import pytest
import torch

import paper_2109_08751_b200 as sp
from paper_2109_08751_b200.binding import lib
from test_train_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes", [[(128, 128), (65, 16), (128, 100), (16, 65)], [(64, 64), (8, 8), (33, 17), (1, 1)]])
def test_linear_attention_plans_of_other_sizes_on_other_threads(sizes):
    cases = [Case([2], 1, kd, vd, "f32", seed=i) for i, (kd, vd) in enumerate(sizes)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    start, errors = threading.Barrier(len(cases)), []

    def work(c, stream):
        # the library's own call, with nothing around it: threads meet inside it as often as they can
        args = (c.plan._h, c.q.data_ptr(), c.kd, c.k.data_ptr(), c.kd, c.v.data_ptr(), c.vd, c.log_decay.data_ptr(),
                c.first.data_ptr(), c.inner("o").data_ptr(), c.vd, c.summary.data_ptr(), stream.cuda_stream)
        call = lib.sparbit_linear_attention_forward
        start.wait()
        errors.extend(code for code in [call(*args) for _ in range(5000)] if code != sp.OK)

    threads = [threading.Thread(target=work, args=x) for x in zip(cases, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, (len(errors), errors[:8])
    for c, stream in zip(cases, streams):
        c.run(stream=stream)
        c.check()
