"""Two gloo ranks whose workers get one tensor's gradient apart from the flat vector (`rows`): the same iterations as with the
whole gradient in the vector.  The device side is the oracle's stand-in, whose "row gradient" is a part and what to add to it."""
import os

import numpy as np
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from paper_2307_03500_b200 import deft
from paper_2307_03500_b200 import workloads as W
from tests.test_distributed_cpu import STEPS, OracleOps, _free_port, _single_process_reference, _worker_grad

PART = (4096 + 64, 4096 + 64 + 16384)      # the third tensor


class PartOps(OracleOps):
    def layer_norms(self, e, g, rows=()):
        g = g.clone()
        for a, b, delta in rows:
            assert torch.isnan(g[a:b]).all()
            g[a:b] = delta
        return super().layer_norms(e, g)


def _rank_main(rank, world, port, result_dir):
    from paper_2307_03500_b200.distributed import DistributedWorker
    dist.init_process_group("gloo", init_method="tcp://127.0.0.1:%d" % port, rank=rank, world_size=world)
    try:
        w = W.tiny()
        worker = DistributedWorker(w.sizes, w.density, "deft", ops=PartOps(w.sizes, world, w.density))
        ref = _single_process_reference("deft", w, world)
        for t in range(STEPS):
            grad = torch.from_numpy(_worker_grad(w, t, rank))
            rows = []
            if rank == 0 or t != 1:                          # a worker may come without rows in a step
                a, b = PART
                rows = [(a, b, grad[a:b].clone())]
                grad[a:b] = float("nan")                     # not read there
            rep = worker.step(grad, rows)
            union, mean, dens, err, max_k, e_ref = ref[t]
            assert np.array_equal(rep.union.numpy(), union) and rep.mean.numpy().tobytes() == mean.tobytes()
            assert rep.density == dens and rep.max_rank_k == max_k and abs(rep.error - err) <= 1e-12 * err
            assert worker.e.numpy().tobytes() == e_ref[rank].tobytes()
        open(os.path.join(result_dir, "ok.%d" % rank), "w").write("ok")
    finally:
        dist.destroy_process_group()


def test_two_gloo_ranks_with_a_part_by_rows(tmp_path):
    deft.lib()
    mp.spawn(_rank_main, args=(2, _free_port(), str(tmp_path)), nprocs=2, join=True)
    assert all(os.path.exists(os.path.join(str(tmp_path), "ok.%d" % r)) for r in range(2))
