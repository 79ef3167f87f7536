"""Adam and kept lists on tensors that are given other memory after they were handed over."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2410_05911_amd as P
    P.lib()
    return P


@pytest.mark.parametrize("how", ["data", "round trip", "copies too"])
def test_adam_updates_parameters_where_they_are(P, how):
    """Two updates with the memory exchanged between them, against the same updates without: bit for bit, and what the
    parameter's first memory holds now stays as it is."""
    gen = torch.Generator("cuda").manual_seed(1)
    p0, g = ([torch.randn(s, device="cuda", generator=gen) for s in ((1000,), (7, 11))] for _ in range(2))
    twin_p, p = [t.clone() for t in p0], [t.clone() for t in p0]
    twin_c, c = ([torch.zeros_like(t, dtype=torch.bfloat16) for t in p0] for _ in range(2))
    twin = P.Adam(twin_p, lr=1e-2, max_norm=1.0, copies=twin_c)
    opt = P.Adam(p, lr=1e-2, max_norm=1.0, copies=c)
    twin.step(g)
    opt.step(g)
    first = [t.data for t in p + c]        # the memory as it was, held here
    if how == "round trip":
        for t in p:
            t.data = t.data.cpu()
        with pytest.raises(ValueError):
            opt.step(g)
        for t in p:
            t.data = t.data.cuda()
    else:
        for t in p:
            t.data = t.data.clone()
    if how == "copies too":
        for t in c:
            t.data = t.data.clone()
    before = [t.clone() for t in first]
    twin.step(g)
    opt.step(g)
    assert all(torch.equal(a, b) for a, b in zip(p + c, twin_p + twin_c))
    assert all(torch.equal(a, b) for a, b in zip(opt.m.tensors + opt.v.tensors, twin.m.tensors + twin.v.tensors))
    moved = len(p) if how != "copies too" else len(p + c)
    assert all(torch.equal(a, b) for a, b in zip(first[:moved], before[:moved]))
    assert opt.step_count.item() == 2


def test_kept_lists_hold_their_memory(P):
    t = torch.ones(1 << 20, device="cuda")
    address = t.data_ptr()
    kept = P.TensorList([t])
    t.data = torch.zeros(3, device="cuda")
    others = [torch.full((1 << 20,), 5.0, device="cuda") for _ in range(4)]
    assert address not in [o.data_ptr() for o in others]
    assert P.grad_norm(kept).item() == 1024.0
    P.grad_clip(kept, 1.0)
    assert all((o == 5).all() for o in others) and (t == 0).all()
