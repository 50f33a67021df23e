"""A GradList whose tensors were given other memory: it goes on with the memory it was made with, and that is still there."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_list_keeps_the_memory_it_was_made_with():
    import gc

    import torch
    from paper_2609_05255_b200 import api
    ctx = api.Context(0)
    n = 3_000_000                                          # a block of its own, which a free gives back to the allocator
    g, more, out = (torch.ones((n,), device="cuda") for _ in range(3))
    where = [t.data_ptr() for t in (g, more, out)]
    grads = api.GradList([api.GradTensor(g, more_grads=[more], out=out)])
    clip, ws = torch.empty((2,), device="cuda"), torch.empty((api.gs_grad_workspace_bytes(),), device="cuda", dtype=torch.uint8)
    for t in (g, more, out):
        t.data = torch.zeros((1,), device="cuda")
    gc.collect()
    taken = [torch.full((n,), 100.0, device="cuda") for _ in range(6)]
    assert not {t.data_ptr() for t in taken} & set(where), "the list's memory went to another tensor"
    api.gs_clip_grads(ctx, grads, 1e9, clip, ws)
    assert abs(float(clip[0]) - 2 * n ** 0.5) <= 2 * n ** 0.5 * 2.0 ** -20      # (the norm's sums: tests of the norm itself)
    assert all(bool(torch.all(t == 100)) for t in taken)
    del grads
    gc.collect()
    again = [torch.empty((n,), device="cuda").data_ptr() for _ in range(1)]
    assert again[0] in where                               # given back with the list
    ctx.close()
