"""Sorts of different numbers of experts from several host threads at once, each on its own stream, through the C ABI
(whose calls, unlike those of the Python module, hold no lock): every one is accepted and right."""
import threading

import numpy as np
import pytest

from oracle import f8

pytestmark = pytest.mark.gpu


def test_sorts_of_different_sizes_from_several_threads():
    import torch
    from paper_2009_06488_b200 import binding as q4
    work = []
    for i, (E, n) in enumerate([(1024, 600), (256, 5000), (512, 9000), (64, 600)]):
        ids = np.random.default_rng(E).integers(-1, E, n).astype(np.int32)
        rows = f8.sort_rows(n, E, 16)
        i32 = lambda k: torch.full((k,), 77, dtype=torch.int32, device="cuda")
        out = (i32(E + 1), i32(rows), i32(n))
        ws = torch.empty(max(16, q4.q4_expert_sort_workspace_bytes(n, E)), dtype=torch.uint8, device="cuda")
        work.append((torch.from_numpy(ids).cuda(), E, out, ws, torch.cuda.Stream(), f8.sort(ids, E, 16, rows)))
    torch.cuda.synchronize()
    codes = []
    gate = threading.Barrier(len(work))

    def sort(ids, E, out, ws, stream, want):
        torch.cuda.set_device(0)
        p = [t.data_ptr() for t in (ids, *out, ws)]
        gate.wait()
        codes.extend({q4._lib.q4_expert_sort(p[0], ids.numel(), E, 16, p[1], p[2], out[1].numel(), p[3], p[4], ws.numel(),
                                             stream.cuda_stream) for _ in range(2000)})
    threads = [threading.Thread(target=sort, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert set(codes) == {q4.Q4_OK}
    for ids, E, out, ws, stream, want in work:
        for g, w in zip(out, want):
            assert (g.cpu().numpy() == w).all()
