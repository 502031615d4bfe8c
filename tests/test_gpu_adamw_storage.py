"""AdamW on tensors whose storage is replaced between two steps: the step goes where the tensors are, or is refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_1312_5766_b200 import binding
    return binding


def tensors(dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(0)
    new = lambda n: torch.randn(n, generator=gen, device="cuda").to(dtype)
    return [new(n) for n in (1000, 3, 700)], [new(n) for n in (1000, 3, 700)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("how", ["data", "set_", "resize_"])
def test_parameters_that_moved(b, how, bits):
    p, g = tensors()
    q = [t.clone() for t in p]
    one, two = b.AdamW(p, bits=bits), b.AdamW(q, bits=bits)
    one.step(g, step=1)
    two.step(g, step=1)
    old = p[0].view(-1)                                  # keeps the first storage
    before, new = old.clone(), old.clone()
    if how == "data":
        p[0].data = new
    elif how == "set_":
        p[0].set_(new)
    else:                                                # grown and cut to size again: elsewhere
        p[2].resize_(1 << 20).resize_(700).copy_(q[2])
    for t in (2, 3):
        one.step(g, step=t)
        two.step(g, step=t)
    assert all(torch.equal(x, y) for x, y in zip(p, q))
    if how != "resize_":
        assert torch.equal(old, before) and p[0].data_ptr() == new.data_ptr()


def test_masters_that_moved_and_moments_that_stay(b):
    """Masters are followed; moments are the object's own memory, whatever happens to the tensors that they came as."""
    p, g = tensors(torch.bfloat16)
    q = [t.clone() for t in p]
    masters, others = [t.float() for t in p], [t.float() for t in q]
    moments = [[torch.zeros_like(t) for t in masters] for _ in range(2)]
    one, two = b.AdamW(p, masters=masters, moments=moments), b.AdamW(q, masters=others)
    for t in range(1, 5):
        one.step(g, step=t)
        two.step(g, step=t)
        assert t > 2 or all(torch.equal(x, y) for x, y in zip(moments[0], two.moments()[0]))      # kept up to date
        if t == 1:
            masters[1].data = masters[1].clone()
        if t == 2:
            moments[0][2].data = torch.ones_like(moments[0][2])
            one.state[1][0].data = torch.ones_like(moments[1][0])
            del moments[1][:]
    assert all(torch.equal(x, y) for x, y in zip(p + masters, q + others))
    for x, y in zip(one.moments(), two.moments()):
        assert all(torch.equal(s, t) for s, t in zip(x, y))


@pytest.mark.parametrize("bits", [32, 8])
def test_the_state_can_be_written_in_place(b, bits):
    p, g = tensors()
    q = [t.clone() for t in p]
    one, two = b.AdamW(p, bits=bits), b.AdamW(q, bits=bits)
    one.step(g, step=1)
    for mine, other in zip(two.state, one.state):
        for x, y in zip(mine, other):
            x.copy_(y)
    for x, y in zip(q, p):
        x.copy_(y)
    one.step(g, step=2)
    two.step(g, step=2)
    assert all(torch.equal(x, y) for x, y in zip(p, q))


def test_what_no_longer_fits_is_refused(b):
    for new, error in ((lambda t: t[:999].clone(), ValueError), (lambda t: t.half(), TypeError), (lambda t: t.repeat(2)[::2], ValueError)):
        p, g = tensors()
        opt = b.AdamW(p)
        opt.step(g, step=1)
        keep = [t.clone() for t in p]
        p[0].data = new(p[0])
        for _ in range(2):                               # until it fits again
            with pytest.raises(error):
                opt.step(g, step=2)
        assert all(torch.equal(x, y) for x, y in zip(p[1:], keep[1:]))
    p, g = tensors()
    opt = b.AdamW(p)
    p[2].data = p[0].data[:700]                          # in another parameter's memory
    with pytest.raises(ValueError):
        opt.step(g, step=1)
