"""What the table and clipping calls write, torch knows to have been written: a value that autograd keeps for its backward pass and that a call then changes is
noticed there, as it is after torch's own operations in place."""
import pytest

pytestmark = pytest.mark.gpu


def _calls():
    import torch
    import paper_2506_02023_amd as M
    ids = torch.tensor([0, 1, 1, -1], device="cuda")
    t, g = torch.ones((2, 3), device="cuda"), torch.ones((4, 3), device="cuda")
    big = torch.ones((300_000,), device="cuda")
    return {"lookup": lambda x: M.mlip_embed(t, ids, out=x), "gradient": lambda x: M.mlip_embed_grad(x.new_ones((4, 3)), ids, 4, out=x),
            "gradient, added": lambda x: M.mlip_embed_grad(g, ids, 4, out=x, accumulate=True),
            "clip in place": lambda x: M.mlip_clip_grads([x], 0.5), "clip in place, of several": lambda x: M.mlip_clip_grads([big, x], 0.5),
            "clip into": lambda x: M.mlip_clip_grads([g * 2], 0.5, out=[x]), "clip into, in a generator": lambda x: M.mlip_clip_grads(iter([g]), 0.5, out=iter([x]))}


@pytest.mark.parametrize("call", ["lookup", "gradient", "gradient, added", "clip in place", "clip in place, of several", "clip into", "clip into, in a generator"])
def test_a_changed_value_is_noticed_in_the_backward_pass(call):
    import torch
    x = torch.ones((4, 3), device="cuda")
    leaf = torch.ones((4, 3), device="cuda", requires_grad=True)
    y = (leaf * x).sum()        # keeps x
    before = x._version
    _calls()[call](x)
    assert x._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_what_is_only_read_keeps_its_version():
    import torch
    import paper_2506_02023_amd as M
    ids = torch.tensor([0, 1, 1, -1], device="cuda")
    t, g = torch.ones((2, 3), device="cuda"), torch.ones((4, 3), device="cuda")
    M.mlip_embed(t, ids, out=torch.empty((4, 3), device="cuda"))
    M.mlip_embed_grad(g, ids, 2, out=torch.empty((2, 3), device="cuda"))
    M.mlip_grad_norm([t, g])
    M.mlip_clip_grads([t, g], 0.5, out=[torch.empty_like(t), torch.empty_like(g)])
    assert t._version == g._version == ids._version == 0
