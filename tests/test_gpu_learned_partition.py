"""The example that runs the partition head's operators together: it learns, and it serves what it learned."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_a_learned_partition_is_more_even_than_k_means():
    import learned_partition as example
    import paper_2604_01000_b200 as ep
    import synth
    work = synth.scaled(synth.WORKLOADS["cfg1"], 6000)
    x = synth.embeddings(work, device="cuda:0")
    rowptr, colidx = synth.graph(work, device="cuda:0")
    before = ep.default_context().launch_count()
    head, km, history = example.train(x, 8, 150)
    assert ep.default_context().launch_count() - before > 150 * 15
    ids = head.forward(x, 1)[1].ids.view(-1)
    assert int(ids.min()) >= 0 and int(ids.max()) < 8
    assert history[-1][1] < history[0][1]
    cut_km, even_km = example.quality(rowptr, colidx, km.assign, 8)
    cut, even = example.quality(rowptr, colidx, ids, 8)
    assert even < even_km and 0.0 < cut < 1.0
    # 8-bit weights and rows (each within 2^-4 of itself) may move a vertex that lies between two parts, no more
    answer = head.serving()
    one_by_one = torch.cat([answer(x[i:i + 1]).view(-1) for i in range(0, 6000, 60)])
    assert float((one_by_one == ids[::60]).float().mean()) >= 0.9
    assert float((answer(x[:500]).view(-1) == ids[:500]).float().mean()) >= 0.9
    ep.default_context().check()
