"""build_step_tables against the oracle: every integer equal."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_16824_amd as cwlib

pytestmark = pytest.mark.gpu
KEEP = 1 << 29  # entries that no call may touch


def _case(lp, ls, page, stride=None, num_free=None, max_tokens=None, seed=0, more_rows=2):
    lp, ls = np.asarray(lp, dtype=np.int32), np.asarray(ls, dtype=np.int32)
    p, s = np.maximum(lp, 0).astype(np.int64), np.maximum(ls, 0).astype(np.int64)
    held, need = -(-p // page), -(-(p + s) // page)
    stride = int(max(need.max(initial=1), 1)) + 1 if stride is None else stride
    rng = np.random.default_rng(seed)
    table = np.full((len(lp) + more_rows, stride), KEEP, dtype=np.int32)
    for b in range(len(lp)):
        n = min(int(held[b]), stride)
        table[b, :n] = rng.integers(0, 1 << 20, size=n)
    want_pages = int((np.minimum(need, stride) - np.minimum(held, stride)).sum())
    free = rng.permutation((want_pages if num_free is None else num_free) + (3 if num_free is None else 0)).astype(np.int32)
    return lp, ls, free, table, (int(s.sum()) if max_tokens is None else max_tokens)


def _check(lp, ls, free, table, max_tokens, page, stream=None):
    dev = lambda a: torch.from_numpy(a).cuda()
    args = (dev(lp), dev(ls), dev(free), dev(table))
    torch.cuda.synchronize()
    with torch.cuda.stream(stream or torch.cuda.current_stream()):
        r = cwlib.build_step_tables(*args, page, max_tokens)
    torch.cuda.synchronize()
    want = oracle.step_tables(lp, ls, free, table[:len(lp)], page, max_tokens)
    got_table = args[3].cpu().numpy()
    assert np.array_equal(got_table[:len(lp)], want[0])
    assert np.array_equal(got_table[len(lp):], table[len(lp):])
    for name, got, ref in zip(r._fields, r, want[1:]):
        assert np.array_equal(got.cpu().numpy(), ref), name
    return r


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("lp,ls", [
    ([0], [1]), ([16], [1]), ([15], [1]), ([0], [0]), ([0, 0, 0], [0, 0, 0]), ([5, 64, 0, 63], [0, 1, 130, 2]),
    ([1000, 0, 17, 31, 64], [1, 1, 1, 1, 1]), ([0, 200, 3], [0, 65, 0]), ([40000], [2500]),
])
def test_small(lp, ls, page):
    print(f"\n[case] tables {lp} {ls} {page}", flush=True)
    _check(*_case(lp, ls, page), page)


@pytest.mark.parametrize("n,page", [(63, 16), (64, 64), (257, 16), (1000, 64), (4095, 16), (4096, 64), (4097, 16), (9001, 64)])
def test_many_sequences(n, page):
    print(f"\n[case] tables of {n} sequences, pages of {page}", flush=True)
    rng = np.random.default_rng(n)
    ls = rng.integers(0, 40, size=n)
    ls[rng.random(n) < 0.6] = 1
    ls[rng.random(n) < 0.2] = 0
    _check(*_case(rng.integers(0, 300, size=n), ls, page, seed=n), page)


@pytest.mark.parametrize("n", [7, 5000])
def test_what_does_not_fit_is_left_out(n):
    """A free list that runs out, rows too short, token arrays too short and too long."""
    print(f"\n[case] tables of {n} sequences that do not fit", flush=True)
    rng = np.random.default_rng(n)
    lp, ls = rng.integers(0, 120, size=n), rng.integers(0, 50, size=n)
    for kw in (dict(num_free=n // 2), dict(num_free=0), dict(stride=4), dict(stride=1, num_free=3), dict(max_tokens=n),
               dict(max_tokens=0), dict(max_tokens=int(ls.sum()) + 777)):
        _check(*_case(lp, ls, 16, **kw), 16)


def test_negative_and_huge_lengths():
    print("\n[case] tables of negative and huge lengths", flush=True)
    big = (1 << 31) - 1
    lp, ls, free, table, _ = _case([-5, 3, 0, 8], [4, -2, 2, 1], 16)
    _check(lp, ls, free, table, 20, 16)
    # 6 x 2^31 new tokens: the sums pass 32 bits, the arrays hold the first ones
    lens = np.array([3] + [big] * 6, dtype=np.int32)
    t = dict(dtype=torch.int32, device="cuda")
    table = torch.full((7, 2), 77, **t)
    r = cwlib.build_step_tables(torch.zeros(7, **t), torch.from_numpy(lens).cuda(), torch.arange(5, **t), table, 16, 40)
    assert r.info.tolist() == [13, 3 + 6 * big, 6]
    assert r.cu_rows.tolist() == [0, 3] + [big] * 6
    assert table.tolist() == [[0, 77], [1, 2], [3, 4], [-1, -1], [-1, -1], [-1, -1], [-1, -1]]
    assert r.seq_ids.tolist() == [0] * 3 + [1] * 37
    assert r.slots.tolist() == [0, 1, 2] + list(range(16, 48)) + [-1] * 5
    # a position past INT32_MAX is clipped, its slot is none
    r = cwlib.build_step_tables(torch.full((1,), big, **t), torch.full((1,), 3, **t), torch.arange(5, **t), table[:1], 16, 3)
    assert r.positions.tolist() == [big] * 3 and r.slots.tolist() == [-1] * 3 and r.info.tolist() == [0, 3, 1]


def test_optional_outputs_and_no_sequences():
    print("\n[case] tables without outputs, without sequences", flush=True)
    t = dict(dtype=torch.int32, device="cuda")
    r = cwlib.build_step_tables(torch.empty(0, **t), torch.empty(0, **t), torch.empty(0, **t), torch.empty(0, 1, **t), 16, 5)
    assert r.cu_rows.tolist() == [0] and r.slots.tolist() == [-1] * 5 and r.info.tolist() == [0, 0, 0]
    lp, ls, free, table, tokens = _case([20, 0], [5, 33], 16)
    d = [torch.from_numpy(a).cuda() for a in (lp, ls, free, table)]
    lib = cwlib.library()
    assert lib.cw_build_step_tables(d[0].data_ptr(), d[1].data_ptr(), 2, d[2].data_ptr(), len(free), 16, d[3].data_ptr(),
                                    table.shape[1], tokens, None, None, None, None, None, None, 0,
                                    torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert np.array_equal(d[3].cpu().numpy()[:2], oracle.step_tables(lp, ls, free, table[:2], 16, tokens)[0])


def test_other_stream_and_repeats():
    print("\n[case] tables on another stream, twice", flush=True)
    case = _case([100, 0, 31], [20, 16, 2], 16)
    s = torch.cuda.Stream()
    a, b = _check(*case, 16, stream=s), _check(*case, 16)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
