"""AdamW over many tensors at once, moments in 32 and in 8 bits.

The step is a fixed sequence of correctly rounded binary32 operations, so it is compared bit for bit with the same sequence in
numpy (whose float32 sums, products, quotients and square roots are correctly rounded too), and with the formula in 64 bits.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BLOCK = 256
F = np.float32
SIZES = [1, 5, 255, 256, 257, 0, 2047, 2048, 2049, 5000, 31]
LR, B1, B2, EPS = 3e-3, 0.9, 0.995, 1e-8


@pytest.fixture(scope="module")
def b():
    from paper_1312_5766_b200 import binding
    return binding


def encode(mag, finite, largest, least_one):
    """Codes of magnitudes (float32) in blocks of 256, and the scales: the square of the code times the scale is the magnitude."""
    n = len(mag)
    rows = np.zeros((-(-n // BLOCK), BLOCK), F)
    rows.reshape(-1)[:n] = np.where(finite, mag, F(0))
    top = rows.max(1) if n else np.zeros(0, F)
    s = np.where(top >= F(2.0 ** -100), top * (F(1) / F(largest)), F(0)).astype(F)
    with np.errstate(divide="ignore"):
        r = np.where(s > 0, F(1) / s, F(0)).astype(F)
    q = np.rint(np.sqrt(rows * r[:, None])).astype(np.int32)
    if least_one:
        q = np.where(rows > 0, np.maximum(q, 1), q)
    return q.reshape(-1)[:n], s


def decode(q, s):
    return (q * q).astype(F) * np.repeat(s, BLOCK)[: len(q)]


def scalars(t, decay, l1, scale):
    return dict(move=F(LR / (1 - B1 ** t)), unbias=F(1 / np.sqrt(1 - B2 ** t)), keep=F(1 - LR * decay), thr=F(LR * l1), scale=F(scale))


def step32(p, g, m, v, c):
    """The step in float32, operation by operation; also the root of the new second moment."""
    with np.errstate(all="ignore"):
        g = g * c["scale"]
        m = m * F(B1) + g * F(1 - B1)
        v = v * F(B2) + (g * g) * F(1 - B2)
        root = np.sqrt(v)
        inv = F(1) / (root * c["unbias"] + F(EPS))
        p = p * c["keep"] - (m * c["move"]) * inv
        if c["thr"] > 0:
            size = np.abs(p) - c["thr"] * inv
            p = np.where(size < 0, F(0), np.copysign(size, p))
    return p.astype(F), m, v, root


def step64(p, g, m, v, t, decay, l1, scale):
    p, g, m, v = (x.astype(np.float64) for x in (p, g, m, v))
    g = g * scale
    m = B1 * m + (1 - B1) * g
    v = B2 * v + (1 - B2) * g * g
    d = np.sqrt(v / (1 - B2 ** t)) + EPS
    q = p * (1 - LR * decay) - LR * m / (1 - B1 ** t) / d
    size = np.abs(p) + LR * (np.abs(m - (1 - B1) * g) + (1 - B1) * np.abs(g)) / (1 - B1 ** t) / d + LR * l1 / d
    return np.sign(q) * np.maximum(np.abs(q) - LR * l1 / d, 0), m, v, size


def make(sizes, ptype, gtype, masters, offset, seed=0):
    """Tensors as views of flat buffers (offset elements apart from a 16-byte boundary), with guards between them."""
    gen = torch.Generator().manual_seed(seed)
    starts, at = [], 16
    for n in sizes:
        starts.append(at + offset)
        at += (n + offset + 8 + 15) // 16 * 16
    flat = {}
    size = torch.exp(torch.rand(at, generator=gen) * -8)
    flat["p32"] = torch.randn(at, generator=gen) * 0.1
    flat["grad"] = (torch.randn(at, generator=gen) * size).to(gtype)
    flat["param"] = flat["p32"].to(ptype)
    flat["m"] = torch.randn(at, generator=gen) * size * 0.3
    flat["v"] = (torch.rand(at, generator=gen) * size * size) * (torch.rand(at, generator=gen) < 0.9)
    return {k: v.cuda() for k, v in flat.items()}, lambda t: [t[a:a + n] for a, n in zip(starts, sizes)]


def bits_equal(a, w):
    a, w = np.asarray(a), np.asarray(w)
    nan = np.isnan(w)
    return np.array_equal(np.isnan(a), nan) and np.array_equal(a[~nan], w[~nan])


CASES = [(torch.float32, torch.float32, False), (torch.bfloat16, torch.bfloat16, False), (torch.bfloat16, torch.float32, True),
         (torch.bfloat16, torch.bfloat16, True), (torch.bfloat16, torch.float32, False), (torch.float16, torch.float16, True),
         (torch.float16, torch.float32, False), (torch.float16, torch.float32, True), (torch.float16, torch.float16, False)]


@pytest.mark.parametrize("offset", [0, 3])
@pytest.mark.parametrize("ptype,gtype,masters", CASES)
def test_32_bit_moments(b, ptype, gtype, masters, offset):
    flat, cut = make(SIZES, ptype, gtype, masters, offset)
    before = {k: v.clone() for k, v in flat.items()}
    opt = b.AdamW(cut(flat["param"]), masters=cut(flat["p32"]) if masters else None, moments=(cut(flat["m"]), cut(flat["v"])),
                  betas=(B1, B2), eps=EPS, weight_decay=0.1, l1=0.02)
    host = {k: [x.float().cpu().numpy() for x in cut(v)] for k, v in flat.items()}
    for t in (7, 8, 100_000):
        opt.step(cut(flat["grad"]), lr=LR, step=t, grad_scale=0.5)
        c = scalars(t, 0.1, 0.02, 0.5)
        for i in range(len(SIZES)):
            p = host["p32"][i] if masters else host["param"][i]
            want, m, v, _ = step32(p, host["grad"][i], host["m"][i], host["v"][i], c)
            exact, m64, v64, size = step64(p, host["grad"][i], host["m"][i], host["v"][i], t, 0.1, 0.02, 0.5)
            # roundings of half a step, 2^-24 each, the scalars' among them: a moment's terms have three (m) and five (v); the root
            # half of v's and one, the metric two more and the sum with eps, its inverse one: seven; with the moment's, the
            # scalar's and the products' that is fourteen for the move, and two for the sums behind it
            assert np.all(np.abs(want - exact) <= 16 * 2.0 ** -24 * size)
            assert np.all(np.abs(m - m64) <= 4 * 2.0 ** -24 * (np.abs(host["m"][i]) + np.abs(host["grad"][i])))
            assert np.all(np.abs(v - v64) <= 6 * 2.0 ** -24 * v64 + 1e-44)
            host["m"][i], host["v"][i] = m, v
            rounded = torch.from_numpy(want).to(ptype).float().numpy()
            host["param"][i] = rounded
            if masters:
                host["p32"][i] = want
        for key in ("m", "v", "param", "p32"):
            for got, w in zip(cut(flat[key]), host[key]):
                assert bits_equal(got.float().cpu().numpy(), w), (key, t)
    # what lies between the tensors is as it was
    for key in flat:
        inside = torch.zeros_like(flat[key], dtype=torch.bool)
        for view in cut(inside):
            view.fill_(True)
        assert torch.equal(flat[key][~inside], before[key][~inside])
    assert torch.equal(flat["grad"], before["grad"])


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("ptype,gtype,masters", CASES)
def test_8_bit_moments(b, ptype, gtype, masters, offset):
    flat, cut = make(SIZES, ptype, gtype, masters, offset, seed=1)
    total = flat["m"].numel()
    code1, code2 = torch.zeros(total, dtype=torch.int8, device="cuda"), torch.zeros(total, dtype=torch.uint8, device="cuda")
    blocks = [-(-n // BLOCK) for n in SIZES]
    scale1, scale2 = torch.zeros(sum(blocks), device="cuda"), torch.zeros(sum(blocks), device="cuda")
    opt = b.AdamW(cut(flat["param"]), bits=8, masters=cut(flat["p32"]) if masters else None,
                  moments=(cut(code1), scale1.split(blocks), cut(code2), scale2.split(blocks)), betas=(B1, B2), eps=EPS, weight_decay=0.1)
    host = {k: [x.float().cpu().numpy() for x in cut(v)] for k, v in flat.items()}
    m = [np.zeros(n, F) for n in SIZES]
    root = [np.zeros(n, F) for n in SIZES]
    for t in (1, 2, 3, 4):
        flat["grad"].mul_(-0.75 if t % 2 else 1.5)
        g = [x.float().cpu().numpy() for x in cut(flat["grad"])]
        opt.step(cut(flat["grad"]), lr=LR, step=t)
        first, second = opt.moments()
        c = scalars(t, 0.1, 0.0, 1.0)
        for i, n in enumerate(SIZES):
            p = host["p32"][i] if masters else host["param"][i]
            want, mi, _, ri = step32(p, g[i], m[i], root[i] * root[i], c)
            q1, s1 = encode(np.abs(mi), np.isfinite(mi), 16129, False)
            q2, s2 = encode(ri, np.isfinite(ri), 64516, True)
            q1 = np.where(mi < 0, -q1, q1)
            assert np.array_equal(cut(code1)[i].cpu().numpy(), q1) and np.array_equal(cut(code2)[i].cpu().numpy(), q2)
            assert np.array_equal(scale1.split(blocks)[i].cpu().numpy(), s1) and np.array_equal(scale2.split(blocks)[i].cpu().numpy(), s2)
            m[i], root[i] = np.sign(q1).astype(F) * decode(q1, s1), decode(q2, s2)
            # half a step of the code either way: the square of the code lies within (q + 1/2)^2
            assert np.all(np.abs(m[i] - mi) <= (np.abs(q1) + 0.2501) * np.repeat(s1, BLOCK)[:n])
            rounded = torch.from_numpy(want).to(ptype).float().numpy()
            host["param"][i], host["p32"][i] = rounded, want
            assert bits_equal(first[i].cpu().numpy(), m[i]) and bits_equal(second[i].cpu().numpy(), root[i] * root[i])
            assert bits_equal(cut(flat["param"])[i].float().cpu().numpy(), rounded)
            if masters:
                assert bits_equal(cut(flat["p32"])[i].cpu().numpy(), want)


def test_moments_allocated_by_the_class_and_values_into_given_tensors(b):
    p = [torch.randn(n, device="cuda") for n in SIZES]
    q = [x.clone() for x in p]
    g = [torch.randn(n, device="cuda") for n in SIZES]
    one, two = b.AdamW(p, bits=8), b.AdamW(q)
    one.step(g, lr=LR, step=1)
    two.step(g, lr=LR, step=1)
    for x, y in zip(p, q):                               # from nothing, the first step is the same whatever holds the moments
        assert torch.equal(x, y)
    out = [[torch.full((n,), 7.0, device="cuda") for n in SIZES] for _ in range(2)]
    first, second = one.moments(out=out)
    assert all(x is y for x, y in zip(first, out[0]))
    # a code q stands for what lies within (q +- 1/2)^2, so it is off by at most q + 1/4 in units of the scale: of the block's largest
    # at most 127.25 / 127^2 = 0.00789 for m (the largest code is 127), and 254.25 / 254^2 = 0.00394 for the root of v, twice that and
    # its square, 0.00790, for v
    for x, y in zip(first, two.moments()[0]):
        assert x.numel() == 0 or (x - y).abs().max() <= 0.0080 * y.abs().max()
    for x, y in zip(second, two.moments()[1]):
        assert x.numel() == 0 or (x - y).abs().max() <= 0.0080 * y.abs().max()


@pytest.mark.parametrize("count", [1, 16, 17, 440, 441, 1000])
@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(b, count, bits):
    """Lists that fill a launch's table, and that need several launches: the same as tensor by tensor."""
    sizes = [1 + (i * 37) % 700 for i in range(count)]
    gen = torch.Generator(device="cuda").manual_seed(count)
    p = [torch.randn(n, generator=gen, device="cuda") for n in sizes]
    g = [torch.randn(n, generator=gen, device="cuda") for n in sizes]
    q = [x.clone() for x in p]
    perm = torch.randperm(count, generator=torch.Generator().manual_seed(0)).tolist()
    many = b.AdamW([p[i] for i in perm], bits=bits)
    for t in (1, 2):
        many.step([g[i] for i in perm], lr=LR, step=t)
    for x, y, h in zip(p, q, g):
        one = b.AdamW([y], bits=bits)
        for t in (1, 2):
            one.step([h], lr=LR, step=t)
    assert all(torch.equal(x, y) for x, y in zip(p, q))


def test_gradients_that_are_not_finite_stay_with_their_element(b):
    n = 700
    for bits in (32, 8):
        p = torch.linspace(-1, 1, n, device="cuda")
        g = torch.linspace(-1, 1, n, device="cuda") + 0.01
        clean_p = p.clone()
        b.AdamW([clean_p], bits=bits).step([g], lr=LR, step=1)
        bad = g.clone()
        bad[3], bad[300], bad[699] = float("nan"), float("inf"), float("-inf")
        opt = b.AdamW([p], bits=bits)
        opt.step([bad], lr=LR, step=1)
        hit = torch.zeros(n, dtype=torch.bool, device="cuda")
        hit[[3, 300, 699]] = True
        assert torch.equal(p[~hit], clean_p[~hit])
        assert torch.isnan(p[hit]).all()
        first, second = opt.moments()
        assert torch.isfinite(first[0][~hit]).all() and torch.isfinite(second[0][~hit]).all()
        assert not torch.isfinite(first[0][hit]).any() and not torch.isfinite(second[0][hit]).any()
        opt.step([g], lr=LR, step=2)                     # and do not recover, nor spread
        assert torch.isnan(p[hit]).all() and torch.isfinite(p[~hit]).all()


def test_small_and_zero_blocks(b):
    """Blocks of noughts, of magnitudes below 2^-100, and a small second moment beside a large one."""
    g = torch.zeros(1024, device="cuda")
    g[256:512] = 1e-30                                   # first moment 1e-31 < 2^-100: stored as noughts; g^2 is 0 in binary32
    g[512:768] = 1e-12
    g[512] = 1e6
    p = torch.ones(1024, device="cuda")
    opt = b.AdamW([p], bits=8, betas=(B1, B2), eps=EPS)
    opt.step([g], lr=LR, step=1)
    first, second = (x[0] for x in opt.moments())
    assert not first[:512].any() and not second[:512].any()
    assert torch.equal(opt.state[0][0][:512], torch.zeros(512, dtype=torch.int8, device="cuda"))
    assert (second[513:768] > 0).all()                   # never stored as 0
    assert torch.isfinite(p).all() and torch.equal(p[:256], torch.ones(256, device="cuda"))


@pytest.mark.parametrize("bits", [32, 8])
def test_scalars_on_the_device_in_a_captured_step(b, bits):
    sizes = [1000, 3, 4097]
    gen = torch.Generator(device="cuda").manual_seed(5)
    p = [torch.randn(n, generator=gen, device="cuda") for n in sizes]
    q = [x.clone() for x in p]
    g = [torch.randn(n, generator=gen, device="cuda") for n in sizes]
    lr, step = torch.tensor([1e-3], device="cuda"), torch.tensor([0], dtype=torch.int64, device="cuda")
    scale, skip = torch.tensor([1.0], device="cuda"), torch.tensor([0], dtype=torch.int32, device="cuda")
    a, w = b.AdamW(p, bits=bits, weight_decay=0.01, l1=0.01), b.AdamW(q, bits=bits, weight_decay=0.01, l1=0.01)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        a.step(g, lr=lr, step=step, grad_scale=scale, skip=skip)
    assert torch.equal(p[0], q[0])                       # captured, not run
    for t in range(1, 6):
        lr.fill_(1e-3 / t)
        scale.fill_(0.5 * t)
        g[0].mul_(-0.9)
        skip.fill_(1 if t == 3 else 0)
        graph.replay()
        if t != 3:
            w.step(g, lr=float(lr), step=t, grad_scale=0.5 * t)
        for x, y in zip(p + a.moments()[0] + a.moments()[1], q + w.moments()[0] + w.moments()[1]):
            assert torch.equal(x, y), t


def test_a_solution_of_the_lasso_is_where_the_step_rests(b):
    """Eq. 1's optimality conditions: the gradient is -lambda sign(beta_j) where beta_j is not 0, within lambda elsewhere.  With the moments
    at rest there (m = g, v = g^2) a step moves beta_j by lr lambda / d and its threshold takes that back: what is left are the roundings
    of the three terms, at most 16 of half a step each."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    n, lam = 5000, 0.3
    beta = torch.randn(n, generator=gen, device="cuda") * (torch.rand(n, generator=gen, device="cuda") < 0.3)
    g = torch.where(beta != 0, -lam * beta.sign(), lam * 0.99 * (2 * torch.rand(n, generator=gen, device="cuda") - 1))
    p = beta.clone()
    opt = b.AdamW([p], moments=([g.clone()], [g * g]), l1=lam, betas=(B1, B2), eps=EPS)
    opt.step([g], lr=LR, step=10_000_000)                # (so far on that no moment is corrected)
    assert ((p == 0) == (beta == 0)).all()
    assert ((p - beta).abs() <= 16 * 2.0 ** -24 * (beta.abs() + 2 * LR)).all()


def test_on_another_stream(b):
    s = torch.cuda.Stream()
    p, g = torch.randn(1_000_000, device="cuda"), torch.randn(1_000_000, device="cuda")
    q = p.clone()
    one, two = b.AdamW([p]), b.AdamW([q])
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for t in range(1, 20):
            one.step([g], step=t)
    for t in range(1, 20):
        two.step([g], step=t)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(p, q)


@pytest.mark.parametrize("bits", [32, 8])
def test_more_than_two_to_the_31_elements(b, bits):
    if torch.cuda.mem_get_info()[0] < 60e9:
        pytest.skip("needs 60 GB")
    n = (1 << 31) + 1000
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    at = [0, 5, (1 << 31) - 1, 1 << 31, (1 << 31) + 257, n - 1]
    g[at] = 1.0
    opt = b.AdamW([p], bits=bits)
    opt.step([g], lr=0.5, step=1)
    want = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    want[at] = -0.5                                      # the first step's length is lr, to 1e-8
    assert torch.equal(p, want)


def test_the_class_refuses(b):
    p = torch.randn(100, device="cuda")
    g = torch.randn(100, device="cuda")
    with pytest.raises(ValueError):
        b.AdamW([p, p])                                  # the same parameters twice
    with pytest.raises(ValueError):
        b.AdamW([p[:60], p[50:]])
    with pytest.raises(ValueError):
        b.AdamW([p], moments=([p], [torch.zeros(100, device="cuda")]))      # a moment in the parameters' memory
    with pytest.raises(ValueError):
        b.AdamW([torch.randn(10, 10, device="cuda").t()])
    with pytest.raises(ValueError):
        b.AdamW([p], moments=([torch.zeros(99, device="cuda")], [torch.zeros(100, device="cuda")]))
    with pytest.raises(TypeError):
        b.AdamW([p], bits=8, moments=([torch.zeros(100, device="cuda")], [torch.zeros(1, device="cuda")]) * 2)
    opt = b.AdamW([p])
    for bad in ([g[:50]], [g, g], [g.cpu()]):
        with pytest.raises(ValueError):
            opt.step(bad)
    with pytest.raises(TypeError):
        opt.step([g.half()])
    for kw in (dict(step=0), dict(lr=-1.0), dict(lr=float("nan"))):
        with pytest.raises(b.StradsError):
            opt.step([g], **kw)
    for kw in (dict(lr=torch.tensor([1.0])), dict(step=torch.tensor([1], device="cuda", dtype=torch.int32)),
               dict(skip=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            opt.step([g], **kw)
