"""Calls of the dense operators beside and behind one another: inputs and
workspaces that are written again right before a call, host threads, sizes
that an int32 does not hold. Values are small integers where sums are
compared, so that these are exact and equal whatever their order."""

import threading

import pytest
import torch
from torch.autograd import forward_ad

from paper_2603_18599_gb300 import dense, sjd

pytestmark = pytest.mark.gpu

DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def whole(g, most, *shape):
    """Whole numbers of magnitudes up to `most`, in fp32."""
    return torch.randint(-most, most + 1, shape, device=DEV, generator=g).float()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,v,d", [(1500, 3000, 512), (1500, 3000, 130), (4000, 300, 257)])
def test_a_tables_gradient_reads_what_was_written_right_before(t, v, d, dtype):
    """Ids and rows that other kernels write into the same memory before every
    call, and a workspace that is the same memory too: the rows of ids that have few
    are added up beside those of ids that have many, with the index of this call."""
    g = gen(t + d)
    sets = []
    for _ in range(3):
        ids = (v * torch.rand(t, device=DEV, generator=g) ** 3).long().clamp(max=v - 1).int()
        ids[torch.rand(t, device=DEV, generator=g) < 0.05] = -1
        rows = whole(g, 8, t, d)
        inside = ids >= 0
        want = torch.zeros(v, d, dtype=torch.float64, device=DEV).index_add_(0, ids[inside].long(), rows[inside].double())
        sets.append((ids, rows.to(dtype), want.float()))
    ids, rows = torch.empty_like(sets[0][0]), torch.empty_like(sets[0][1])

    def turns(n):
        out = []
        for i in range(n):
            ids.copy_(sets[i % 3][0])
            rows.copy_(sets[i % 3][1])
            out.append(dense.embed_gradient(rows, ids, v))
        return out

    out = turns(60)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = turns(6)
    for _ in range(5):
        graph.replay()
        out += [x.clone() for x in captured]
    for i, x in enumerate(out):
        assert torch.equal(x, sets[i % 3][2]), i


def test_host_threads_at_once():
    """Host threads whose calls of many rows take kernels of one kind with
    different amounts of shared memory, each on a stream of its own: every call
    is taken, and gives what it gives alone."""
    L, rows, turns = dense.load(), 400, 4000
    g = gen(11)

    def calls(d):
        """Calls at the C boundary, and their outputs: a loop over them is as dense as a host thread's can be."""
        x, y, dx = normal(g, rows, d).bfloat16(), torch.empty(rows, d, dtype=BF16, device=DEV), torch.empty(rows, d, dtype=BF16, device=DEV)
        codes, scale, dgain = torch.empty(rows, d, dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV), torch.empty(d, device=DEV)
        size = L.sjd_norm_gradient_workspace_size(rows, d, sjd.SJD_BF16)
        room = torch.empty(size, dtype=torch.uint8, device=DEV)
        at = [dense._pack(t) for t in (x, y, dx)]
        some = [(L.sjd_norm_gradient, at[0], at[0], None, 1e-6, 0, None, rows, d, sjd.SJD_BF16, at[2], dgain.data_ptr(), None, room.data_ptr(), size)]
        if d <= 8192:
            some += [(L.sjd_norm, at[0], None, None, None, 1e-6, 0, rows, d, sjd.SJD_BF16, None, at[1], None, None),
                     (L.sjd_quantise, at[0], rows, d, sjd.SJD_BF16, codes.data_ptr(), scale.data_ptr())]
        return some, (x, room), (y, dx, codes, scale, dgain) if d <= 8192 else (dx, dgain)

    jobs = [calls(d) for d in (8192, 4096, 16384, 9000)]
    want = []
    for some, _, out in jobs:
        for call, *args in some:
            assert call(*args, None) == sjd.SJD_OK
        torch.cuda.synchronize()
        want.append([t.clone() for t in out])
        for t in out:
            t.zero_()
    begin, refused = threading.Barrier(len(jobs)), [0] * len(jobs)
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()

    def work(i):
        raw = streams[i].cuda_stream
        begin.wait(60)
        for _ in range(turns):
            for call, *args in jobs[i][0]:
                refused[i] += call(*args, raw) != sjd.SJD_OK

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not any(refused), refused
    for (_, _, out), alone in zip(jobs, want):
        assert all(torch.equal(a, b) for a, b in zip(out, alone))


def test_sizes_that_an_int32_does_not_hold_are_refused():
    """2^32 + 5 of anything would arrive as 5."""
    n = 2 ** 32 + 5
    row, code, vector = torch.ones(1, 1, device=DEV), torch.ones(1, 1, dtype=torch.int8, device=DEV), torch.ones(1, device=DEV)
    weight, few = dense.Weight(code, vector), torch.zeros(3, dtype=torch.int32, device=DEV)
    many, ids = row.expand(n, 1), torch.empty(n, dtype=torch.int32, device=DEV)
    scale = ids.view(F32)
    calls = {
        "quantise": lambda: dense.quantise(many), "norm": lambda: dense.norm(many), "norm_codes": lambda: dense.norm_codes(many),
        "norm_gradient": lambda: dense.norm_gradient(many, many), "product": lambda: dense.product(code.expand(n, 1), scale, weight),
        "channels": lambda: dense.Weight(code.expand(n, 1), scale), "features": lambda: dense.Weight(torch.empty(1, n, dtype=torch.int8, device=DEV), vector),
        "table": lambda: dense.embed(many, few), "tokens": lambda: dense.embed(row, ids), "rows": lambda: dense.embed_gradient(many, ids, 3),
        "vocabulary": lambda: dense.embed_gradient(row.expand(3, 1), few, n),
    }
    taken = []
    for name, call in calls.items():
        try:
            call()
            taken.append(name)
        except ValueError:
            pass
    assert not taken


def test_the_largest_numbers_of_rows_and_ids():
    n = 2 ** 31 - 1
    x = torch.full((1, 1), -3.0, device=DEV)
    codes, scale = dense.quantise(x.expand(n, 1))
    assert codes.shape == (n, 1) and bool((codes.view(-1)[::4097] == -127).all()) and bool((scale[::4097] == scale[0]).all())
    assert codes[-1] == -127 and scale[-1] == scale[0]
    del codes, scale
    # ids at both ends, some of them in many rows
    ids = torch.tensor([0, n - 1, n - 2, 1] * 10 + [n - 1] * 60 + [-1, n], dtype=torch.int32, device=DEV)
    rows = torch.arange(ids.numel(), device=DEV, dtype=F32)[:, None].contiguous()
    grad = dense.embed_gradient(rows, ids, n)
    for v in (0, 1, n - 2, n - 1):
        assert grad[v] == rows[ids == v].sum(), v
    assert torch.count_nonzero(grad) == 4


def test_tangents_of_forward_mode_are_refused():
    x, w = torch.ones(4, 64, device=DEV), torch.ones(64, device=DEV)
    ids, codes = torch.zeros(4, dtype=torch.int32, device=DEV), torch.ones(4, 64, dtype=torch.int8, device=DEV)
    weight = dense.Weight(codes, w[:4].contiguous())
    with forward_ad.dual_level():
        d, dw, ds = (forward_ad.make_dual(t, torch.ones_like(t)) for t in (x, w, w[:4].contiguous()))
        for call in (lambda: dense.quantise(d), lambda: dense.norm(d), lambda: dense.norm(x, dw), lambda: dense.norm(x, w, dw), lambda: dense.norm(x, residual=d),
                     lambda: dense.norm_codes(d[None]), lambda: dense.norm_gradient(d, x), lambda: dense.norm_gradient(x, d), lambda: dense.norm_gradient(x, x, dh=d),
                     lambda: dense.embed(d, ids), lambda: dense.embed_gradient(d, ids, 3), lambda: dense.product(codes, ds, weight),
                     lambda: dense.product(codes, w[:4], weight, bias=ds), lambda: dense.product(codes, w[:4], weight, residual=d[:, :4], dtype=F32),
                     lambda: dense.Weight(codes, ds), lambda: dense.Weight.quantise(d)):
            with pytest.raises(ValueError, match="tangent"):
                call()
        assert torch.equal(dense.norm(d.detach(), w), dense.norm(x, w))
    assert torch.equal(dense.norm(x, w), dense.norm(x))
