"""GPU: the AdamW step over lists of tensors, states in 32 and in 8 bits, through the C ABI, against the fp64
definition.

Tolerances, U = 2^-24.  m = b1 m + (1 - b1) g: the two factors, the scaled gradient, two products and the sum are
rounded: 5 U (|b1 m| + |(1 - b1) g|).  v likewise with one product more, all terms positive: 6 U v.  The update
m / (sqrt(v) c + eps) lr': half of v's error, the root, c, the fused sum, the quotient (two units), lr' and the product:
16 U of itself, and m's error passed on.  p: its decay and the difference are rounded, 3 U (|p| + |update|), then to its
type.  States in 8 bits: scales bit for bit; codes too, but where m or the root is nearer to the border between two
codes than its error, 5 U (|b1 m| + |(1 - b1) g|) and 8 U root (half of v's, the root's two units, one rounding), plus
2^-29 of the scale where 2^-6 has been added to a small number; there it may be the neighbour."""
import numpy as np
import pytest
import torch

from oracle import ops_oracle as oo
from paper_2602_01469_b200 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
BF16, F32 = torch.bfloat16, torch.float32
F8 = torch.float8_e4m3fn
HOW = dict(lr=3e-3, beta1=0.9, beta2=0.98, eps=1e-7)


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def f64(t):
    return t.detach().double().cpu().numpy()


def make(gen, n, dtype, gdtype, bits, master, decay, offset=0):
    """One tensor of n elements in the middle of longer buffers (``offset`` elements in), with what follows it."""
    def put(x):
        buf = torch.full((n + offset + 40,), 1.0, dtype=torch.float32).to(x.dtype).to(DEV)
        buf[offset:offset + n] = x.to(DEV)
        return buf[offset:offset + n]

    w = torch.randn(n, generator=gen)
    # gradients over several decades, a stretch of zeros, exact zeros among the states
    g = torch.randn(n, generator=gen) * torch.exp(3 * torch.randn(n, generator=gen)) * 1e-3
    g[n // 3: n // 3 + n // 7] = 0
    m, root = 0.5 * torch.randn(n, generator=gen) * g.abs(), g.abs() * (0.5 + torch.rand(n, generator=gen))
    item = {"grad": put(g.to(gdtype)), "weight_decay": decay, "master": put(w) if master else None, "param": put(w.to(dtype))}
    if bits == 32:
        item.update(m=put(m), v=put(root ** 2))
    else:
        blocks = -(-n // 256)
        ms = torch.tensor(oo.block_scale(m.double().numpy()), dtype=F32)
        vs = torch.tensor(oo.block_scale(root.double().numpy()), dtype=F32)
        per = lambda s: s.repeat_interleave(256)[:n]
        item.update(m=put((m / per(ms)).to(F8).view(torch.uint8)).view(F8), v=put((root / per(vs)).to(F8).view(torch.uint8)).view(F8),
                    m_scale=ms.to(DEV), v_scale=vs.to(DEV))
        assert ms.shape[0] == blocks
    return item


def snapshot(item):
    return {k: (t.clone() if isinstance(t, torch.Tensor) else t) for k, t in item.items()}


def outside(got, want, bound):
    bad = ~((np.abs(got - want) <= bound) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])


def check(before, after, place, step, seed, how=HOW, factor=1.0):
    n = before["param"].numel()
    p = f64(before["master"] if before["master"] is not None else before["param"]).ravel()
    g = f64((before["grad"].float().cpu() * np.float32(factor))).ravel()
    b1, b2 = how["beta1"], how["beta2"]
    if "m_scale" in before:
        code = lambda t: t.view(torch.uint8).cpu().numpy().ravel()
        m, root, mc, vc, off_m, off_v, ms, vs = oo.adamw_states8(g, code(before["m"]), code(before["v"]),
                                                                 f64(before["m_scale"]), f64(before["v_scale"]), b1, b2,
                                                                 seed, step, place)
        assert np.array_equal(f64(after["m_scale"]), ms) and np.array_equal(f64(after["v_scale"]), vs)
        per = lambda s: np.repeat(s, 256)[:n]
        m0 = oo.e4m3_values()[code(before["m"])] * per(f64(before["m_scale"]))
        em = 5 * U * (np.abs(b1 * m0) + np.abs((1 - b1) * g))
        m, root = m.astype(np.float64), root.astype(np.float64)
        for got, want, off, err in ((after["m"], mc, off_m, em + 2.0 ** -29 * per(ms)),
                                    (after["v"], vc, off_v, 8 * U * root + 2.0 ** -29 * per(vs))):
            got = code(got)
            a, b = oo.e4m3_values()[got], oo.e4m3_values()[want]
            near = (np.abs((got & 127).astype(int) - (want & 127)) == 1) & (off <= err)
            other = ~((a == b) | (np.isnan(a) & np.isnan(b)))
            assert not (other & ~near).any(), (int((other & ~near).sum()), np.argwhere(other & ~near)[:4].tolist())
        v = root ** 2
    else:
        m0, v0 = f64(before["m"]).ravel(), f64(before["v"]).ravel()
        _, m, v = oo.adamw(p, g, m0, v0, how["lr"], b1, b2, how["eps"], 0.0, step)
        em = 5 * U * (np.abs(b1 * m0) + np.abs((1 - b1) * g))
        outside(f64(after["m"]).ravel(), m, em + 2.0 ** -126)
        outside(f64(after["v"]).ravel(), v, 6 * U * v + 2.0 ** -126)
    lr = how["lr"] / (1 - b1 ** step)
    below = np.sqrt(v / (1 - b2 ** step)) + how["eps"]
    update = lr * m / below
    want = p - how["lr"] * float(np.float32(before["weight_decay"])) * p - update
    err = 16 * U * np.abs(update) + lr * em / below + 3 * U * (np.abs(p) + np.abs(update))
    if before["master"] is not None:
        outside(f64(after["master"]).ravel(), want, err)
        assert torch.equal(after["param"], after["master"].to(BF16))
    else:
        dt = after["param"].dtype
        outside(f64(after["param"]).ravel(), want, HALF[dt] * np.abs(want) + err)
    assert n == after["param"].numel()


KINDS = [  # param, grad, bits, master
    (F32, F32, 32, False), (BF16, BF16, 32, True), (BF16, F32, 32, True), (BF16, BF16, 32, False), (F32, BF16, 32, False),
    (F32, F32, 8, False), (BF16, BF16, 8, True), (BF16, BF16, 8, False), (BF16, F32, 8, True),
]
SIZES = [1, 7, 255, 256, 257, 1000, 2048, 4096 + 8, 20011]


@pytest.mark.parametrize("dtype,gdtype,bits,master", KINDS)
def test_lists_of_tensors(ctx, dtype, gdtype, bits, master):
    gen = torch.Generator().manual_seed(bits + int(master))
    items = [make(gen, n, dtype, gdtype, bits, master, 0.1 * (i % 3), offset=i % 4) for i, n in enumerate(SIZES)]
    items.insert(3, make(gen, 0, dtype, gdtype, bits, master, 0.0))
    items.append(make(gen, 0, dtype, gdtype, bits, master, 0.0))
    tensors = binding.AdamWTensors(items)
    for step in (1, 2, 50):
        before = [snapshot(i) for i in items]
        behind = [i["param"]._base[-30:].clone() if i["param"]._base is not None else None for i in items]
        binding.peagle_adamw_step(ctx, tensors, step=step, seed=77, **HOW)
        torch.cuda.synchronize()
        for k, (b, a) in enumerate(zip(before, items)):
            check(b, a, k, step, 77)
            if behind[k] is not None:
                assert torch.equal(a["param"]._base[-30:], behind[k])
    assert binding.peagle_poll_status(ctx) == 0


def test_mixed_kinds_and_more_tensors_than_a_launch_takes(ctx):
    gen = torch.Generator().manual_seed(5)
    items = [make(gen, 1 + (i * 37) % 600, *KINDS[i % len(KINDS)], 0.01, offset=i % 3) for i in range(900)]
    before = [snapshot(i) for i in items]
    n = binding.peagle_launch_count(ctx)
    binding.peagle_adamw_step(ctx, binding.AdamWTensors(items), step=3, seed=1, **HOW)
    torch.cuda.synchronize()
    assert binding.peagle_launch_count(ctx) - n == 3             # 384 tensors each
    for k, (b, a) in enumerate(zip(before, items)):
        check(b, a, k, 3, 1)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_large_tensor(ctx, bits):
    gen = torch.Generator().manual_seed(6)
    item = make(gen, 3_000_001, BF16, BF16, bits, True, 0.1)
    before = snapshot(item)
    binding.peagle_adamw_step(ctx, binding.AdamWTensors([item]), step=4, seed=9, **HOW)
    torch.cuda.synchronize()
    check(before, item, 0, 4, 9)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_code_is_the_defined_one(ctx, dtype):
    """m and v as from fp64, rounded to fp32 once: also where a number lies next to the border of its code, and a step
    later, when a code on the other side would have moved its block's scale."""
    gen = torch.Generator().manual_seed(12)
    item = make(gen, 1_500_003, dtype, dtype, 8, False, 0.1)
    tensors = binding.AdamWTensors([item])
    code = lambda t: t.view(torch.uint8).cpu().numpy().ravel()
    for step in (3, 4):
        b = snapshot(item)
        binding.peagle_adamw_step(ctx, tensors, step=step, seed=5, **HOW)
        torch.cuda.synchronize()
        _, _, mc, vc, _, _, ms, vs = oo.adamw_states8(f64(b["grad"]).ravel(), code(b["m"]), code(b["v"]), f64(b["m_scale"]),
                                                      f64(b["v_scale"]), HOW["beta1"], HOW["beta2"], 5, step, 0)
        assert np.array_equal(f64(item["m_scale"]), ms) and np.array_equal(f64(item["v_scale"]), vs)
        values = oo.e4m3_values()
        for name, want in (("m", mc), ("v", vc)):
            assert np.array_equal(values[code(item[name])], values[want], equal_nan=True), name


@pytest.mark.parametrize("bits", [8, 32])
def test_untouched_elements_stay_with_the_smallest_eps(ctx, bits):
    """m = v = g = 0, a row of an embedding that no token has met: the step is 0 / eps = 0, the decay remains."""
    gen = torch.Generator().manual_seed(13)
    item = make(gen, 3000, F32, F32, bits, False, 0.1, offset=1)
    for name in ("m", "v"):
        item[name].view(torch.uint8 if bits == 8 else F32).zero_()
    item["grad"].zero_()
    how = dict(lr=3e-3, beta1=0.9, beta2=0.98, eps=2.0 ** -126)
    before = snapshot(item)
    binding.peagle_adamw_step(ctx, binding.AdamWTensors([item]), step=1, seed=2, **how)
    torch.cuda.synchronize()
    check(before, item, 0, 1, 2, how)


@pytest.mark.parametrize("beta1", [0.9, 0.95, 0.5, 0.0])
def test_blocks_whose_average_cancels(ctx, beta1):
    """m = beta1 m + (1 - beta1) g of nearly nothing in all elements of a block: codes and scales are those of fp64."""
    rng = np.random.default_rng(31)
    values = oo.e4m3_values()
    items = []
    for k in range(400):
        n = 1 if k < 300 else 1 + k % 256
        # one code for a block, mostly: what cancels in one element cancels in all of them
        c = rng.integers(0x50, 0x78, n if k % 3 == 0 else 1).astype(np.uint8) | (128 * rng.integers(0, 2, 1)).astype(np.uint8)
        c = np.broadcast_to(c, n).copy()
        scale = 2.0 ** rng.integers(-20, 5)
        g = -(beta1 / (1 - beta1)) * values[c] * scale
        g = g * (1 + (0.0, 2.0 ** -22, -2.0 ** -18, 2.0 ** -12, 2.0 ** -6)[k % 5]) if beta1 else values[c] * scale * 2.0 ** -(k % 30)
        item = {"param": torch.zeros(n, device=DEV), "grad": torch.tensor(g, dtype=F32, device=DEV), "weight_decay": 0.0,
                "master": None, "m": torch.tensor(c, device=DEV).view(F8), "m_scale": torch.full((1,), scale, device=DEV),
                "v": torch.tensor(c & 127, device=DEV).view(F8), "v_scale": torch.full((1,), scale, device=DEV)}
        items.append(item)
    before = [snapshot(i) for i in items]
    how = dict(lr=1e-3, beta1=beta1, beta2=0.98, eps=1e-8)
    binding.peagle_adamw_step(ctx, binding.AdamWTensors(items), step=3, seed=6, **how)
    torch.cuda.synchronize()
    code = lambda t: t.view(torch.uint8).cpu().numpy().ravel()
    for k, (b, a) in enumerate(zip(before, items)):
        _, _, mc, vc, _, _, ms, vs = oo.adamw_states8(f64(b["grad"]), code(b["m"]), code(b["v"]), f64(b["m_scale"]),
                                                      f64(b["v_scale"]), beta1, how["beta2"], 6, 3, k)
        assert np.array_equal(f64(a["m_scale"]), ms) and np.array_equal(f64(a["v_scale"]), vs), (k, f64(a["m_scale"]), ms)
        assert np.array_equal(values[code(a["m"])], values[mc]) and np.array_equal(values[code(a["v"])], values[vc]), k


@pytest.mark.parametrize("power", [-100, -99, -98, -60, 0])
def test_scales_next_to_a_power_of_two(ctx, power):
    """Blocks whose m is the power of two, or a few units in the last place to either side; 2^-99 is the first that moves
    the scale."""
    for beta1 in (0.9, 0.85, 0.8, 0.7, 0.6):
        at = int(np.float32(2.0 ** power / (1 - beta1)).view(np.int32))
        g = np.arange(at - 20, at + 20, dtype=np.int32).view(np.float32)
        zero = lambda dtype: torch.zeros(1, dtype=torch.uint8, device=DEV).view(F8) if dtype == F8 else torch.zeros(1, device=DEV)
        items = [{"param": zero(F32), "grad": torch.tensor([x], device=DEV), "m": zero(F8), "v": zero(F8), "m_scale": zero(F32),
                  "v_scale": zero(F32)} for x in g]
        binding.peagle_adamw_step(ctx, binding.AdamWTensors(items), step=1, lr=1e-3, beta1=beta1, beta2=0.98, eps=1e-8)
        want = oo.block_scale(((1 - beta1) * g.astype(np.float64)).astype(np.float32).astype(np.float64), 1)
        assert np.array_equal(torch.cat([i["m_scale"] for i in items]).double().cpu().numpy(), want), beta1


def tiny_gradients(gen, n):
    """From where v leaves fp32's normal numbers (1e-18) to where it is zero (1e-23), beside larger ones, zeros, and in
    blocks of their own."""
    tiny = torch.randn(n, generator=gen).sign() * 10 ** (-24 + 8 * torch.rand(n, generator=gen, dtype=torch.float64))
    some = torch.rand(n, generator=gen) < 0.3
    some[n // 2:] = True
    # and blocks in between, some larger
    rise = (10 ** (10 * torch.rand(n // 256 + 1, generator=gen))).repeat_interleave(256)[:n]
    tiny[3 * n // 4:] *= rise[3 * n // 4:]
    g = torch.where(some, tiny.float(), torch.randn(n, generator=gen) * 1e-3)
    g[torch.rand(n, generator=gen) < 0.05] = 0
    g[-600:] = 0
    return g


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("empty", [True, False])
def test_tiny_roots_are_kept_in_8_bits(ctx, dtype, empty):
    """Every code is the defined one, and no root above zero is stored as zero, where v is no normal fp32 number; the
    step divides by that root, whatever eps is."""
    gen = torch.Generator().manual_seed(21)
    n = 100_003
    item = make(gen, n, dtype, dtype, 8, False, 0.1)
    if empty:
        for name in ("m", "v"):
            item[name].view(torch.uint8).zero_()
            item[name + "_scale"].zero_()
    else:
        item["v"].view(torch.uint8)[:] = torch.where(torch.rand(n, generator=gen) < 0.4, 0, item["v"].view(torch.uint8).cpu()).to(DEV)
        item["v_scale"][::3] = 1e-22
        item["m_scale"][::3] = 1e-23
    item["grad"].copy_(tiny_gradients(gen, n))
    how = dict(lr=3e-3, beta1=0.9, beta2=0.98, eps=1e-20)
    tensors = binding.AdamWTensors([item])
    code = lambda t: t.view(torch.uint8).cpu().numpy().ravel()
    for step in (1, 2):
        b = snapshot(item)
        binding.peagle_adamw_step(ctx, tensors, step=step, seed=5, **how)
        torch.cuda.synchronize()
        _, root, mc, vc, _, _, ms, vs = oo.adamw_states8(f64(b["grad"]).ravel(), code(b["m"]), code(b["v"]), f64(b["m_scale"]),
                                                         f64(b["v_scale"]), how["beta1"], how["beta2"], 5, step, 0)
        assert np.array_equal(f64(item["m_scale"]), ms) and np.array_equal(f64(item["v_scale"]), vs)
        values = oo.e4m3_values()
        assert (values[code(item["v"])][root > 0] > 0).all()
        for name, want in (("m", mc), ("v", vc)):
            assert np.array_equal(values[code(item[name])], values[want], equal_nan=True), name
        check(b, item, 0, step, 5, how)


@pytest.mark.parametrize("count", [20, 60])
@pytest.mark.parametrize("eps", [1e-20, 1e-12])
def test_tiny_roots_among_tensors_of_all_kinds(ctx, count, eps):
    """Short and long lists, states in 8 bits alone and beside others, an eps below what fp32 settles and one above."""
    gen = torch.Generator().manual_seed(23)
    how = dict(lr=3e-3, beta1=0.9, beta2=0.98, eps=eps)
    kinds8 = [k for k in KINDS if k[2] == 8]
    for kinds in (kinds8, kinds8 + [(F32, F32, 32, False)]):
        items = [make(gen, 1 + (i * 97) % 1500, *kinds[i % len(kinds)], 0.1, offset=i % 5) for i in range(count)]
        for i in items:
            if i["m"].dtype == F8:
                i["grad"].copy_(tiny_gradients(gen, i["grad"].numel()))
                i["v"].view(torch.uint8)[::3] = 0
                i["m"].view(torch.uint8)[::3] = 0
        tensors = binding.AdamWTensors(items)
        for step in (1, 2):
            before = [snapshot(i) for i in items]
            binding.peagle_adamw_step(ctx, tensors, step=step, seed=8, **how)
            torch.cuda.synchronize()
            for k, (b, a) in enumerate(zip(before, items)):
                check(b, a, k, step, 8, how)


@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-30, 1e-20, 1e-8])
def test_tiny_roots_divide_the_step_in_32_bits(ctx, eps):
    """The step from the m and v that are stored, which are fp32's, some of them no normal numbers."""
    gen = torch.Generator().manual_seed(22)
    n = 20_003
    item = make(gen, n, F32, F32, 32, False, 0.0)
    item["grad"].copy_(tiny_gradients(gen, n))
    item["m"].zero_()
    item["v"].zero_()
    b = snapshot(item)
    beta1, beta2, lr = 0.9, 0.98, 1e-3
    binding.peagle_adamw_step(ctx, binding.AdamWTensors([item]), step=1, lr=lr, beta1=beta1, beta2=beta2, eps=eps)
    torch.cuda.synchronize()
    m, v, g, p = f64(item["m"]), f64(item["v"]), f64(b["grad"]), f64(b["param"])
    # fp32's smallest number is 2^-149; each of v's products and its sum is off by half of it at most
    outside(m, (1 - beta1) * g, 5 * U * np.abs((1 - beta1) * g) + 2.0 ** -148)
    outside(v, (1 - beta2) * g * g, 6 * U * (1 - beta2) * g * g + 2.0 ** -148)
    assert (v[(np.abs(g) > 1e-21)] > 0).all()
    update = lr * m / (1 - beta1) / (np.sqrt(v / (1 - beta2)) + eps)
    want = p - update
    outside(f64(item["param"]), want, 16 * U * np.abs(update) + 3 * U * (np.abs(p) + np.abs(update)) + U * np.abs(want))


def test_states_that_begin_at_zero(ctx):
    gen = torch.Generator().manual_seed(7)
    item = make(gen, 700, F32, F32, 8, False, 0.0)
    for name in ("m", "v"):
        item[name].view(torch.uint8).zero_()
        item[name + "_scale"].zero_()
    before = snapshot(item)
    tensors = binding.AdamWTensors([item])
    binding.peagle_adamw_step(ctx, tensors, step=1, seed=2, **HOW)
    torch.cuda.synchronize()
    check(before, item, 0, 1, 2)
    item["grad"].zero_()
    for step in range(2, 5):
        before = snapshot(item)
        binding.peagle_adamw_step(ctx, tensors, step=step, seed=2, **HOW)
        check(before, item, 0, step, 2)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_bad_gradient_stays_in_its_element(ctx, bits):
    gen = torch.Generator().manual_seed(8)
    item = make(gen, 600, F32, F32, bits, False, 0.1)
    clean = snapshot(item)
    tensors = binding.AdamWTensors([item])
    for at, bad in ((10, float("nan")), (300, float("inf")), (301, -float("inf"))):
        item["grad"][at] = bad
        clean["grad"][at] = 0
    binding.peagle_adamw_step(ctx, tensors, step=2, seed=3, **HOW)
    binding.peagle_adamw_step(ctx, binding.AdamWTensors([clean]), step=2, seed=3, **HOW)
    torch.cuda.synchronize()
    keep = torch.ones(600, dtype=torch.bool, device=DEV)
    keep[[10, 300, 301]] = False
    assert torch.equal(item["param"][keep], clean["param"][keep])
    assert torch.isnan(item["param"][~keep]).all()
    if bits == 8:
        assert torch.isnan(item["m"].float()[~keep]).all() and torch.isnan(item["v"].float()[~keep]).all()
        assert torch.equal(item["m"].view(torch.uint8)[keep], clean["m"].view(torch.uint8)[keep])
        assert torch.equal(item["v_scale"], clean["v_scale"])


def test_steps_in_a_captured_graph(ctx):
    """The step's number, the rate and the gradients' factor on the device: replays equal eager steps bit for bit."""
    gen = torch.Generator().manual_seed(9)
    items = [make(gen, 5000, BF16, BF16, b, True, 0.1) for b in (8, 32)]
    other = [snapshot(i) for i in items]
    tensors, eager = binding.AdamWTensors(items), binding.AdamWTensors(other)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    lr, factor = torch.tensor([1e-3], device=DEV), torch.tensor([0.5], device=DEV)
    betas = dict(beta1=0.9, beta2=0.98, eps=1e-7)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step.add_(1)
        binding.peagle_adamw_step(ctx, tensors, 0.0, step=0, seed=4, lr_dev=lr, step_dev=step, grad_scale=factor, **betas)
    for k in range(1, 5):
        rate = 1e-3 * k
        lr.fill_(rate)
        before = snapshot(other[1])
        g.replay()
        binding.peagle_adamw_step(ctx, eager, float(np.float32(rate)), step=k, seed=4, grad_scale=factor, **betas)
        torch.cuda.synchronize()
        check(before, other[1], 1, k, 4, dict(lr=float(np.float32(rate)), **betas), 0.5)
        for a, b in zip(items, other):
            for name in ("param", "master", "m", "v"):
                assert torch.equal(a[name].view(torch.uint8), b[name].view(torch.uint8)), name


def test_an_average_held_in_8_bits_moves(ctx):
    """beta2 = 0.999 moves v by a thousandth a step, a code is 6 to 12 % away: the average still finds the mean
    square of the gradients, from above.  (The root is rounded without bias, so its square is a few per cent high.)"""
    n = 1 << 14
    gen = torch.Generator(device=DEV).manual_seed(10)
    item = {"param": torch.zeros(n, device=DEV), "grad": torch.zeros(n, device=DEV), "m": torch.zeros(n, device=DEV).to(F8),
            "v": torch.full((n,), 128.0, device=DEV).to(F8), "m_scale": torch.ones(n // 256, device=DEV),
            "v_scale": torch.full((n // 256,), 4.0 / 128, device=DEV)}
    tensors = binding.AdamWTensors([item])
    for step in range(1, 4001):
        item["grad"].normal_(generator=gen)
        binding.peagle_adamw_step(ctx, tensors, 0.0, 0.9, 0.999, 1e-8, step=step, seed=step)
    root = item["v"].float().view(-1, 256) * item["v_scale"][:, None]
    # from 16 towards 1: 16 * 0.999^4000 = 0.29 is left of the start
    assert 1.0 < float(root.square().mean()) < 1.6


def test_set_grads_and_refusals(ctx):
    gen = torch.Generator().manual_seed(11)
    item = make(gen, 300, BF16, BF16, 32, False, 0.0)
    tensors = binding.AdamWTensors([item])
    fresh = torch.randn(300, generator=gen).to(DEV)
    tensors.set_grads([fresh])
    before = snapshot(tensors.items[0])
    binding.peagle_adamw_step(ctx, tensors, step=1, **HOW)
    torch.cuda.synchronize()
    check(before, item, 0, 1, 0)
    binding.peagle_adamw_step(ctx, binding.AdamWTensors([]), step=1, **HOW)     # nothing to do

    def refused(status, f, *args, **kw):
        with pytest.raises(binding.PeagleError) as e:
            f(*args, **kw)
        assert e.value.status == binding.STATUS[status]

    for change in ({"m": item["m"].half()}, {"m": item["m"][:200]}, {"param": item["param"].half()}, {"v": None},
                   {"master": item["m"].to(BF16)}, {"m_scale": torch.ones(2, device=DEV)}, {"grad": item["grad"][:10]},
                   {"grad": item["grad"].cpu()}, {"m": item["m"].cpu()}):
        refused("BAD_SHAPE", binding.AdamWTensors, [{**item, **change}])
    refused("BAD_RANGE", binding.AdamWTensors, [item, item])                    # the same tensor twice
    refused("BAD_RANGE", binding.AdamWTensors, [{**item, "v": item["m"]}])
    refused("BAD_SHAPE", tensors.set_grads, [])
    refused("BAD_SHAPE", binding.peagle_adamw_step, ctx, tensors, 1e-3, 0.9, 0.99, 1e-8, step=0)
    refused("BAD_SHAPE", binding.peagle_adamw_step, ctx, tensors, 1e-3, 0.9, 0.99, 1e-8, step_dev=torch.ones(1, device=DEV))


def test_refused_gradients_leave_the_old_ones(ctx):
    """A list that is refused half way changes nothing: the next step takes all gradients from the list before."""
    gen = torch.Generator().manual_seed(14)
    items = [make(gen, n, BF16, BF16, 32, False, 0.0) for n in (300, 40, 7)]
    tensors = binding.AdamWTensors(items)
    old = [i["grad"] for i in tensors.items]
    pointers = [(c.grad, c.grad_dtype) for c in tensors.c]
    fresh = [torch.randn(n, generator=gen).to(DEV) for n in (300, 40, 7)]
    for bad in (fresh[2][:6], fresh[2].half(), fresh[2].cpu()):
        with pytest.raises(binding.PeagleError) as e:
            tensors.set_grads([fresh[0], fresh[1], bad])
        assert e.value.status == binding.STATUS["BAD_SHAPE"]
        assert [(c.grad, c.grad_dtype) for c in tensors.c] == pointers
        assert all(i["grad"] is g for i, g in zip(tensors.items, old))
    tensors.set_grads(fresh)
    assert [c.grad for c in tensors.c] == [g.data_ptr() for g in fresh]
    before = [snapshot(i) for i in tensors.items]
    binding.peagle_adamw_step(ctx, tensors, step=1, **HOW)
    torch.cuda.synchronize()
    for k, (b, a) in enumerate(zip(before, tensors.items)):
        check(b, a, k, 1, 0)


def test_gradients_in_the_memory_of_what_is_written_are_refused(ctx):
    """The step reads a gradient more than once, and what it writes in between must not be in its place."""
    item = {"param": torch.zeros(300, device=DEV), "m": torch.zeros(300, device=DEV), "v": torch.zeros(300, device=DEV)}
    around = torch.zeros(1000, device=DEV)
    item["param"] = around[300:600]
    fine = [around[:300], around[600:900], torch.zeros(300, device=DEV)]
    for g in fine:
        tensors = binding.AdamWTensors([{**item, "grad": g}])
    for g in (item["param"], item["m"], item["v"], around[1:301], around[599:899], around[450:750],
              around[400:550].view(torch.uint8).view(BF16), around[599:749].view(torch.uint8).view(BF16)):
        for call in (lambda: binding.AdamWTensors([{**item, "grad": g}]), lambda: tensors.set_grads([g])):
            with pytest.raises(binding.PeagleError) as e:
                call()
            assert e.value.status == binding.STATUS["BAD_RANGE"]
    two = [{**item, "grad": fine[0]}, {"param": around[:0], "m": around[:0], "v": around[:0], "grad": item["param"][:0]}]
    binding.AdamWTensors(two)                                        # nothing of a tensor without elements is written
    other = {k: torch.zeros(300, device=DEV) for k in ("param", "m", "v")}
    binding.AdamWTensors([{**item, "grad": fine[2]}, {**other, "grad": fine[2]}])   # read twice
