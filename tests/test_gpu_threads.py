"""Host threads with a plan each: aggregation and partial gradients, whose kernels need different amounts of shared memory."""
import sys
import threading

import numpy as np
import pytest

from paper_1902_01981_b200 import binding as B
from paper_1902_01981_b200 import build as cr_build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

THREADS = 8


@pytest.fixture(scope="module", autouse=True)
def built():
    cr_build.build()
    assert torch.cuda.is_available()


class Calls:
    """C calls with their arguments ready, so that the threads spend their time inside them."""

    def __init__(self):
        self.keep = []

    def new(self, shape, value, dtype=torch.float32):
        self.keep.append(torch.full(shape, value, dtype=dtype, device="cuda"))
        return self.keep[-1].data_ptr()

    def aggregate(self, batch):
        def make(plan, d, stream):
            N, m = B.cr_plan_num_nodes(plan), B.cr_plan_load(plan)
            masks = np.zeros((batch, B.cr_plan_num_groups(plan)), dtype=np.uint32)
            self.keep.append(masks)
            need = B.lib().cr_aggregate_workspace_bytes(plan, batch, B.CR_AGG_FUSED)
            args = (self.new((N, m, d), 1.0), masks.ctypes.data, batch, self.new((batch, d), 0.0), B.CR_AGG_FUSED,
                    self.new((max(need, 16),), 0, torch.uint8), need, stream)
            return lambda: B.lib().cr_aggregate(plan, *args)
        return make

    def gradients(self, plan, d, stream):
        N, m, rows = B.cr_plan_num_nodes(plan), B.cr_plan_load(plan), 8
        need = B.lib().cr_partial_gradients_workspace_bytes(plan, rows)
        parts = int(B.slot_partitions(plan).max()) + 1
        args = (self.new((parts, rows, d), 1.0), self.new((parts, rows), 1.0), rows, self.new((d,), 0.5), self.new((N, m, d), 0.0),
                self.new((max(need, 16),), 0, torch.uint8), need, stream)
        return lambda: B.lib().cr_partial_gradients(plan, *args)


# (partitions, length of the gradient) of the two kinds of plan: nodes of 8 and of 16 rows; gradients of one instance of the kernel
CASES = [("aggregate", (48, 1024), (96, 1024)), ("batch", (48, 1024), (96, 1024)), ("gradients", (24, 2100), (24, 4096))]


@pytest.mark.parametrize("kind,small,large", CASES)
def test_no_call_takes_shared_memory_from_another(kind, small, large):
    calls = Calls()
    make = {"aggregate": calls.aggregate(1), "batch": calls.aggregate(4), "gradients": calls.gradients}[kind]
    plans, run, kernels = [], [], []
    interval = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        streams = [torch.cuda.Stream() for _ in range(THREADS)]
        for i in range(THREADS):
            P, d = (small, large)[i % 2]
            plans.append(B.cr_plan_create(4, 2, 1, P, d, device=0))
            run.append(make(plans[i], d, streams[i].cuda_stream))
            torch.cuda.synchronize()
            assert run[i]() == B.CR_OK
            kernels.append(B.cr_plan_last_kernel(plans[i]))
        torch.cuda.synchronize()
        failed, begin = [0] * THREADS, threading.Barrier(THREADS)

        def work(i):
            begin.wait()
            for _ in range(4000):
                failed[i] += run[i]() != B.CR_OK

        threads = [threading.Thread(target=work, args=(i,)) for i in range(THREADS)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        torch.cuda.synchronize()
        assert not any(failed), (kind, failed)
        assert len(set(kernels)) == 1, kernels
    finally:
        sys.setswitchinterval(interval)
        torch.cuda.synchronize()
        for p in plans:
            B.cr_plan_destroy(p)
