"""A training loop asks for the loss and its gradient in turn: each finds its plan of the step before.  No GPU needed."""
import ctypes as C
import time

import paper_1910_10929_b200 as dgs

P = 1 << 36


def test_a_loss_and_its_gradient_in_turn_cost_what_both_cost_alone():
    L, out = dgs.lib(), C.c_uint64(0)
    h, w = (dgs.dgs_matrix(P * i, rows, 512, 512, dgs.DGS_TYPE_BF16) for i, rows in ((1, 2000), (2, 8000)))     # a plan of 12 us, looked up in a fraction of one
    calls = [lambda: L.dgs_vocabulary_loss_bytes(h, w, C.byref(out)), lambda: L.dgs_vocabulary_loss_grad_bytes(h, w, C.byref(out))]

    def best(*turn):
        times = []
        for _ in range(30):
            at = time.perf_counter()
            for _ in range(20):
                for call in turn:
                    call()
            times.append(time.perf_counter() - at)
        return min(times)

    assert best(*calls) < 1.5 * (best(calls[0]) + best(calls[1]))
    # and each has its own answer, in whatever order they are asked for
    sizes = []
    for _ in range(3):
        for call in calls:
            assert call() == dgs.DGS_OK
            sizes.append(out.value)
    assert len(set(sizes[0::2])) == len(set(sizes[1::2])) == 1 and sizes[0] != sizes[1]
    # a question that is refused leaves nothing behind
    none = dgs.dgs_matrix(P, 2000, 512, (1 << 24) + 8, dgs.DGS_TYPE_BF16)
    assert L.dgs_vocabulary_loss_grad_bytes(none, none, C.byref(out)) != dgs.DGS_OK
    assert calls[1]() == dgs.DGS_OK and out.value == sizes[1]
