"""Calls of the dense operators beside and behind one another: inputs and
workspaces that are written again right before a call, host threads, sizes
that an int32 does not hold. Values are small integers where sums are
compared, so that these are exact and equal whatever their order."""

import pytest
import torch

from paper_2603_18599_gb300 import dense

pytestmark = pytest.mark.gpu

DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


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
