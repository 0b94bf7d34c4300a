"""Evictions of different sizes from two host threads, each with a stream and workspace of its own."""
import threading

import pytest
import torch

from paper_2609_00097_b200 import ffd
from tests.chunk_cases import Chunk
from tests.test_gpu_weigh_evict import Evict, lengths

pytestmark = pytest.mark.gpu


def test_two_threads():
    # a CTA for each of 160 sequences, with room for 320 pages' weights (80 KB), against eight pages'
    jobs = [Evict(Chunk(lengths(20480, *[70] * 159), 1, 1, seed=1, room=0), 200, 3, 30), Evict(Chunk(lengths(500), 2, 1, seed=2, room=0), 200, 3, 30)]
    torch.cuda.synchronize()
    failed, go = [], threading.Barrier(2)

    def work(job):
        with torch.cuda.stream(torch.cuda.Stream()):
            go.wait()
            for _ in range(400):
                try:
                    job.run()
                except ffd.FfdError as e:
                    failed.append(e)
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(j,)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, (len(failed), str(failed[0]))
    for job in jobs:
        job.check()
