"""Which `out` tensors a list of gradients takes: those that lie in memory as the
gradients do, however their strides are written."""
import pytest
import torch

import paper_2105_14713_amd as onexn

CL = torch.channels_last


def test_layouts():
    same = onexn._same_layout
    w = torch.empty(6, 4, 1, 1)
    assert w.stride() != w.to(memory_format=CL).stride() and same(w, w.to(memory_format=CL))
    assert same(torch.empty(1, 5), torch.empty(3, 7)[:1, :5]) and same(torch.empty(()), torch.empty(()))
    assert same(torch.empty(0, 3).t(), torch.empty(3, 0))
    k = torch.empty(6, 4, 3, 3)
    assert same(k, torch.empty(6, 4, 3, 3)) and not same(k, k.to(memory_format=CL))
    assert not same(torch.empty(5, 5), torch.empty(5, 5).t())


@pytest.mark.gpu
def test_out_in_the_other_memory_format():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gen = torch.Generator().manual_seed(1)
    # Gradients of +-1 and 0, clipped to a quarter of their norm: +-1/4 up to a step of fp32.
    g = [torch.ones(32, 8, 1, 1).cuda(), torch.ones(16, 16, 3, 3)[:, :, :1, :1].contiguous().cuda()]
    g = [torch.where(torch.rand(t.shape, generator=gen).cuda() < 0.5, t, -t) for t in g]
    g.append(torch.zeros(8, 4, 3, 3, device="cuda"))
    norm = float(sum(t.numel() for t in g[:2])) ** 0.5
    for formats in ((CL, torch.contiguous_format), (torch.contiguous_format, CL)):
        grads = [t.contiguous(memory_format=formats[0]) for t in g[:2]] + [g[2]]
        out = [torch.full_like(t, 3.0).contiguous(memory_format=formats[1]) for t in g[:2]] + [torch.empty_like(g[2])]
        got = onexn.clip_grads(grads, norm / 4, out=out)
        assert float(got) == float(torch.tensor(norm))
        assert all(torch.allclose(o, t / 4, rtol=2 ** -23, atol=0) for o, t in zip(out, g))
        onexn.BoundGrads(grads, out)
    with pytest.raises(ValueError, match="out 0"):
        onexn.clip_grads([g[2]], 1.0, out=[torch.empty_like(g[2]).contiguous(memory_format=CL)])
