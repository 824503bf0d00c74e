"""The status word of a worker's own operators: a report is returned once, whichever stream it comes from."""
import threading

import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_every_report_is_returned_once():
    """One stream reports while four threads read the word on streams of their own: neither lost nor returned twice."""
    z, out = torch.zeros(8, 4, device=DEV), torch.empty(8, 4, device=DEV)
    expert, dw = torch.full((8, 1), 9, dtype=torch.int32, device=DEV), torch.ones(8, 1, device=DEV)      # an expert that does not exist
    dgs.route_experts_grad(z, expert, dw, out=out)
    assert dgs.operator_status(DEV) == dgs.DGS_EINVAL and dgs.operator_status(DEV) == 0
    rounds, readers = 300, 4
    gate = threading.Barrier(readers + 1)
    seen = [[] for _ in range(readers)]

    def read(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(rounds):
                gate.wait()
                seen[i].append([dgs.operator_status(DEV) for _ in range(5)])
                gate.wait()

    threads = [threading.Thread(target=read, args=(i,)) for i in range(readers)]
    for t in threads:
        t.start()
    rest = []
    with torch.cuda.stream(torch.cuda.Stream()):
        for _ in range(rounds):
            gate.wait()
            dgs.route_experts_grad(z, expert, dw, out=out)
            gate.wait()                                  # all have read
            rest.append(dgs.operator_status(DEV))
    for t in threads:
        t.join()
    for n in range(rounds):
        values = [v for s in seen for v in s[n]] + [rest[n]]
        assert sorted(values) == [dgs.DGS_EINVAL] + [0] * (5 * readers), n
