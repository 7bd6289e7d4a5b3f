"""build_step_tables in a captured graph that moves the free list on by itself: the call keeps no
place in the list, so every replay takes pages from its start."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_16824_amd as cwlib

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seqs", [6, 5000])
def test_replays_take_the_next_pages_of_a_list_moved_on_the_gpu(seqs):
    print(f"\n[case] captured step tables of {seqs} sequences with a moving free list", flush=True)
    page, steps, tokens, stride = 16, 5, 40 * seqs, 16
    rng = np.random.default_rng(seqs)
    n_free = 12 * seqs
    pages = rng.permutation(n_free).astype(np.int32)
    i32 = dict(dtype=torch.int32, device="cuda")
    lens, new = torch.zeros(seqs, **i32), torch.ones(seqs, **i32)
    free, at = torch.from_numpy(pages).cuda(), torch.arange(n_free, device="cuda")
    table = torch.full((seqs, stride), -7, **i32)
    bufs = dict(cu_rows=torch.empty(seqs + 1, **i32), seq_ids=torch.empty(tokens, **i32), positions=torch.empty(tokens, **i32),
                slots=torch.empty(tokens, dtype=torch.int64, device="cuda"),
                info=torch.empty(3, dtype=torch.int64, device="cuda"))
    ws = torch.empty(max(16, cwlib.step_tables_workspace_bytes(seqs)), dtype=torch.uint8, device="cuda")

    def step():
        cwlib.build_step_tables(lens, new, free, table, page, tokens, workspace=ws, **bufs)
        lens.add_(new)
        free.copy_(free[(at + bufs["info"][0]).clamp(max=n_free - 1)])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    lens.zero_(), table.fill_(-7), free.copy_(torch.from_numpy(pages))
    host, want, left = np.zeros(seqs, dtype=np.int64), np.full((seqs, stride), -7), pages
    for k in range(steps):
        ls = rng.integers(0, 40, size=seqs)
        ls[rng.random(seqs) < 0.5] = 1
        new.copy_(torch.from_numpy(ls.astype(np.int32)))
        g.replay()
        other = torch.randn(1000, device="cuda").sum()  # the program's own work between the replays
        want, cu, seq, pos, slots, info = oracle.step_tables(host, ls, left, want, page, tokens)
        torch.cuda.synchronize()
        assert bool(other.isfinite()) and np.array_equal(table.cpu().numpy(), want), k
        for name, ref in (("cu_rows", cu), ("seq_ids", seq), ("positions", pos), ("slots", slots), ("info", info)):
            assert np.array_equal(bufs[name].cpu().numpy(), ref), (k, name)
        host, left = host + ls, left[int(info[0]):]
    taken = want[want >= 0]
    assert len(taken) > seqs and len(np.unique(taken)) == len(taken)  # no page twice
