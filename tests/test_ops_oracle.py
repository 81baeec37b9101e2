"""CPU pins of the fp64 definitions of the operators around the layer: closed forms, torch's own
operators and autograd, central differences; and the refusals that the library makes on the host."""
import numpy as np
import pytest
import torch

from oracle import ops_oracle as oo


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("affine", [True, False])
def test_norm_equals_torch_and_its_autograd(kind, affine):
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(5, 23, generator=gen, dtype=torch.float64, requires_grad=True)
    w = torch.randn(23, generator=gen, dtype=torch.float64, requires_grad=True) if affine else None
    b = torch.randn(23, generator=gen, dtype=torch.float64, requires_grad=True) if affine and kind == "layer" else None
    dy = torch.randn(5, 23, generator=gen, dtype=torch.float64)
    if kind == "layer":
        y = torch.nn.functional.layer_norm(x, (23,), w, b, 1e-3)
    else:
        y = torch.nn.functional.rms_norm(x, (23,), w, 1e-3)
    (y * dy).sum().backward()
    num = lambda t: None if t is None else t.detach().numpy()
    got, mean, rstd = oo.norm_fwd(kind, num(x), num(w), num(b), 1e-3)
    assert np.allclose(got, num(y), atol=1e-13)
    dx, dw, db = oo.norm_bwd(kind, num(x), num(w), mean, rstd, dy.numpy())
    assert np.allclose(dx, x.grad.numpy(), atol=1e-13)
    if affine:
        assert np.allclose(dw, w.grad.numpy(), atol=1e-13)
    if b is not None:
        assert np.allclose(db, b.grad.numpy(), atol=1e-13)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_norm_gradients_by_central_differences(kind):
    rng = np.random.default_rng(1)
    x, w, dy = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal((3, 7))

    def loss(x, w):
        return float((oo.norm_fwd(kind, x, w, None, 0.1)[0] * dy).sum())

    _, mean, rstd = oo.norm_fwd(kind, x, w, None, 0.1)
    dx, dw, _ = oo.norm_bwd(kind, x, w, mean, rstd, dy)
    h = 1e-5
    for i in np.ndindex(3, 7):
        up, dn = x.copy(), x.copy()
        up[i] += h
        dn[i] -= h
        assert (loss(up, w) - loss(dn, w)) / (2 * h) == pytest.approx(dx[i], rel=1e-6, abs=1e-8)
    for i in range(7):
        up, dn = w.copy(), w.copy()
        up[i] += h
        dn[i] -= h
        assert (loss(x, up) - loss(x, dn)) / (2 * h) == pytest.approx(dw[i], rel=1e-6, abs=1e-8)


def test_norm_closed_forms():
    y, mean, rstd = oo.norm_fwd("layer", [[3.0, 1.0]], [2.0, 2.0], [0.5, 0.5], 0.0)
    assert np.allclose(y, [[2.5, -1.5]]) and np.allclose(mean, [2.0]) and np.allclose(rstd, [1.0])
    y, _, rstd = oo.norm_fwd("rms", [[3.0, 4.0]], None, None, 0.0)
    assert np.allclose(rstd, [1 / np.sqrt(12.5)]) and np.allclose(y, np.array([[3.0, 4.0]]) / np.sqrt(12.5))


def test_token_logprobs_equal_torch_and_its_autograd():
    gen = torch.Generator().manual_seed(4)
    x = torch.randn(6, 19, generator=gen, dtype=torch.float64, requires_grad=True)
    tokens = torch.tensor([3, 0, 18, 7, -1, 2])
    g, h = torch.randn(6, generator=gen, dtype=torch.float64), torch.randn(6, generator=gen, dtype=torch.float64)
    logp = torch.log_softmax(x * 0.7, 1)
    lp = torch.where(tokens < 0, 0.0, logp.gather(1, tokens.clamp(min=0)[:, None])[:, 0])
    H = torch.distributions.Categorical(logits=x * 0.7).entropy()
    (lp * g + H * h).sum().backward()
    got = oo.token_logprobs(x.detach().numpy(), tokens.numpy(), 0.7, 4)
    assert np.allclose(got[0], lp.detach().numpy(), atol=1e-13) and np.allclose(got[2], H.detach().numpy(), atol=1e-13)
    assert np.allclose(got[1], torch.logsumexp(x * 0.7, 1).detach().numpy(), atol=1e-13)
    best = torch.topk(logp, 4, 1)
    assert np.allclose(got[3], best.values.detach().numpy(), atol=1e-13) and np.array_equal(got[4], best.indices.numpy())
    d = oo.token_logprobs_bwd(x.detach().numpy(), tokens.numpy(), 0.7, got[1], got[2], g.numpy(), h.numpy())
    assert np.allclose(d, x.grad.numpy(), atol=1e-13)


def test_token_logprobs_by_central_differences():
    rng = np.random.default_rng(2)
    x, tokens = rng.standard_normal((2, 9)), np.array([4, 8])
    g, h = rng.standard_normal(2), rng.standard_normal(2)

    def loss(x):
        lp, _, H, _, _ = oo.token_logprobs(x, tokens, 1.3, 0)
        return float((lp * g + H * h).sum())

    _, lse, H, _, _ = oo.token_logprobs(x, tokens, 1.3, 0)
    d = oo.token_logprobs_bwd(x, tokens, 1.3, lse, H, g, h)
    for i in np.ndindex(2, 9):
        up, dn = x.copy(), x.copy()
        up[i] += 1e-5
        dn[i] -= 1e-5
        assert (loss(up) - loss(dn)) / 2e-5 == pytest.approx(d[i], rel=1e-6, abs=1e-8)


def test_token_logprobs_of_rows_without_a_distribution():
    inf, nan = np.inf, np.nan
    x = np.array([[-inf, -inf, -inf], [0.0, nan, 1.0], [inf, 0.0, 0.0], [-inf, 2.0, -inf], [5.0, 5.0, 5.0], [0.0, -0.0, 1.0]])
    lp, lse, H, top, ids = oo.token_logprobs(x, np.array([1, 0, 2, 1, 2, 7]), 1.0, 2)
    assert lp[0] == lse[0] == -inf and H[0] == 0 and ids[0].tolist() == [0, 1] and np.isneginf(top[0]).all()
    assert np.isnan([lp[1], lse[1], H[1], lp[2], lse[2], H[2]]).all() and (ids[1:3] == -1).all()
    assert lp[3] == 0 and lse[3] == 2 and H[3] == 0 and ids[3].tolist() == [1, 0]
    assert lp[4] == pytest.approx(-np.log(3)) and H[4] == pytest.approx(np.log(3)) and ids[4].tolist() == [0, 1]
    assert np.isnan(lp[5]) and ids[5].tolist() == [2, 0]


def test_adamw_equals_torch():
    rng = np.random.default_rng(3)
    p0 = rng.standard_normal(20)
    p = torch.tensor(p0, requires_grad=True)
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.3)
    q, m, v = p0, np.zeros(20), np.zeros(20)
    for step in range(1, 6):
        g = rng.standard_normal(20)
        p.grad = torch.tensor(g)
        opt.step()
        q, m, v = oo.adamw(q, g, m, v, 0.01, 0.8, 0.95, 1e-6, 0.3, step)
    assert np.allclose(q, p.detach().numpy(), atol=1e-14)


def test_e4m3_values_equal_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(oo.e4m3_values(), codes.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)


def test_stochastic_code_is_unbiased_and_neighbouring():
    """Over all 2^16 values of the random bits, the mean is the number itself to 2^-16 of a step."""
    values = oo.e4m3_values()
    bits = np.arange(1 << 16, dtype=np.float64)
    for y in (0.0, 0.3 * 2.0 ** -9, 2.0 ** -9, 0.0137, 0.015625, 0.017, 1.03, 100.7, 255.9, 256.0, -3.3):
        got = values[oo.stochastic_code(np.full(1 << 16, y), bits, False)[0]]
        step = 2.0 ** -9 if abs(y) < 2.0 ** -6 else 2.0 ** (np.floor(np.log2(abs(y))) - 3)
        assert abs(got.mean() - y) <= step * 2.0 ** -15 and np.abs(got - y).max() < step
        if y > 0:
            assert values[oo.stochastic_code(np.full(1 << 16, y), bits, True)[0]].min() > 0


def test_block_scales():
    x = np.zeros(700)
    x[3], x[300], x[301] = -5.0, 2.0 ** -120, np.inf
    assert oo.block_scale(x).tolist() == [2.0 ** -5, 2.0 ** -107, 2.0 ** -107]
    assert oo.block_scale(np.array([1.0, np.nan])).tolist() == [2.0 ** -7]


def test_random_bits_are_spread():
    b = oo.adamw_random_bits(1, 2, 3, 1 << 16)
    for part in (b & np.uint64(0xFFFF), b >> np.uint64(16)):
        counts = np.bincount((part >> np.uint64(12)).astype(int), minlength=16)
        assert np.abs(counts - 4096).max() < 6 * 64          # six standard deviations
    assert len(np.unique(np.concatenate([b, oo.adamw_random_bits(1, 2, 4, 1 << 16)]))) > 2 * (1 << 16) - 20


# ------------------------------------------------------------------ refusals, before any device is touched
@pytest.fixture(scope="module")
def lib():
    from paper_2602_01469_b200 import binding, build
    build.build()
    return binding.lib()


@pytest.fixture(scope="module")
def zeros():
    """Stands in for a context: the calls below are refused, or have nothing to do, before they look into it."""
    import ctypes
    return ctypes.create_string_buffer(1 << 16)


def _norm_call(lib, ctx, back, **over):
    import ctypes
    a = dict(kind=1, x_dtype=1, w_dtype=1, rows=4, cols=64, X=4096, ldx=64, weight=0, bias=0, eps=1e-5, Y=8192, ldy=64,
             mean=0, rstd=12288, dY=16384, lddy=64)
    a.update(over)
    i32, i64, ptr = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
    head = [ctx, i32(a["kind"]), i32(a["x_dtype"]), i32(a["w_dtype"]), i32(a["rows"]), i32(a["cols"]), ptr(a["X"]),
            i64(a["ldx"]), ptr(a["weight"])]
    if back:
        return lib.peagle_norm_bwd(*head, ptr(a["mean"]), ptr(a["rstd"]), ptr(a["dY"]), i64(a["lddy"]), ptr(a["Y"]),
                                   i64(a["ldy"]), ptr(0), ptr(0), ptr(0))
    return lib.peagle_norm_fwd(*head, ptr(a["bias"]), ctypes.c_float(a["eps"]), ptr(a["Y"]), i64(a["ldy"]), ptr(a["mean"]),
                               ptr(a["rstd"]), ptr(0))


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("over,status", [
    ({"rows": 0}, "OK"), ({"rows": -1}, "BAD_SHAPE"), ({"cols": 0}, "BAD_SHAPE"),
    ({"cols": (1 << 30) + 1, "ldx": 1 << 31, "ldy": 1 << 31, "lddy": 1 << 31}, "TOO_LARGE"), ({"kind": 2}, "BAD_SHAPE"),
    ({"kind": -1}, "BAD_SHAPE"), ({"x_dtype": 2}, "BAD_SHAPE"), ({"w_dtype": -1}, "BAD_SHAPE"), ({"ldx": 63}, "BAD_SHAPE"),
    ({"ldy": 63}, "BAD_SHAPE"), ({"X": 0}, "NULL"), ({"Y": 0}, "NULL"), ({"X": 4097}, "ALIGN"), ({"Y": 8193}, "ALIGN"),
    ({"x_dtype": 0, "X": 4098}, "ALIGN"), ({"weight": 4097}, "ALIGN"), ({"rstd": 12290}, "ALIGN"),
])
def test_norm_refusals(lib, zeros, back, over, status):
    from paper_2602_01469_b200 import binding
    assert _norm_call(lib, zeros, back, **over) == binding.STATUS[status]


def test_norm_refusals_of_one_direction(lib, zeros):
    from paper_2602_01469_b200 import binding
    S = binding.STATUS
    for eps in (0.0, -1e-5, float("nan")):
        assert _norm_call(lib, zeros, False, eps=eps) == S["BAD_SHAPE"]
    assert _norm_call(lib, zeros, True, kind=0) == S["NULL"]          # layer norm without its mean
    assert _norm_call(lib, zeros, True, rstd=0) == S["NULL"]
    assert _norm_call(lib, zeros, True, dY=0) == S["NULL"]
    assert _norm_call(lib, zeros, True, lddy=10) == S["BAD_SHAPE"]
    assert _norm_call(lib, None, False) == _norm_call(lib, None, True) == S["NULL"]


def _logprob_call(lib, ctx, back, **over):
    import ctypes
    a = dict(dtype=1, rows=4, vocab=100, logits=4096, ld=100, tokens=8192, scale=1.0, lp=12288, lse=16384, H=0, k=0, top=0,
             ids=0, g=20480, h=0, d=24576, ldd=100)
    a.update(over)
    i32, i64, ptr = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
    head = [ctx, i32(a["dtype"]), i32(a["rows"]), i32(a["vocab"]), ptr(a["logits"]), i64(a["ld"]), ptr(a["tokens"]),
            ctypes.c_float(a["scale"])]
    if back:
        return lib.peagle_token_logprobs_bwd(*head, ptr(a["lse"]), ptr(a["H"]), ptr(a["g"]), ptr(a["h"]), ptr(a["d"]),
                                             i64(a["ldd"]), ptr(0))
    return lib.peagle_token_logprobs_fwd(*head, ptr(a["lp"]), ptr(a["lse"]), ptr(a["H"]), i32(a["k"]), ptr(a["top"]),
                                         ptr(a["ids"]), ptr(0))


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("over,status", [
    ({"rows": 0}, "OK"), ({"rows": -2}, "BAD_SHAPE"), ({"vocab": 0}, "BAD_SHAPE"), ({"ld": 99}, "BAD_SHAPE"),
    ({"dtype": 5}, "BAD_SHAPE"), ({"vocab": (1 << 30) + 1, "ld": 1 << 31, "ldd": 1 << 31}, "TOO_LARGE"), ({"scale": 0.0}, "BAD_SHAPE"), ({"scale": -1.0}, "BAD_SHAPE"),
    ({"scale": float("nan")}, "BAD_SHAPE"), ({"scale": float("inf")}, "BAD_SHAPE"), ({"scale": 1e-21}, "BAD_SHAPE"), ({"logits": 0}, "NULL"),
    ({"tokens": 0}, "NULL"), ({"logits": 4097}, "ALIGN"), ({"tokens": 8194}, "ALIGN"), ({"lse": 16386}, "ALIGN"),
])
def test_logprob_refusals(lib, zeros, back, over, status):
    from paper_2602_01469_b200 import binding
    assert _logprob_call(lib, zeros, back, **over) == binding.STATUS[status]


def test_logprob_refusals_of_one_direction(lib, zeros):
    from paper_2602_01469_b200 import binding
    S = binding.STATUS
    assert _logprob_call(lib, zeros, False, k=-1) == S["BAD_SHAPE"]
    assert _logprob_call(lib, zeros, False, k=101, top=4096, ids=4096) == S["BAD_SHAPE"]
    assert _logprob_call(lib, zeros, False, k=65, top=4096, ids=4096) == S["TOO_LARGE"]
    assert _logprob_call(lib, zeros, False, k=3, top=4096) == S["NULL"]
    assert _logprob_call(lib, zeros, False, k=3, ids=4096) == S["NULL"]
    assert _logprob_call(lib, zeros, True, lse=0) == S["NULL"]
    assert _logprob_call(lib, zeros, True, d=0) == S["NULL"]
    assert _logprob_call(lib, zeros, True, h=4096) == S["NULL"]          # the entropy's gradient without the entropy
    assert _logprob_call(lib, zeros, True, ldd=99) == S["BAD_SHAPE"]
    assert _logprob_call(lib, zeros, True, d=24577) == S["ALIGN"]
    assert _logprob_call(lib, None, False) == _logprob_call(lib, None, True) == S["NULL"]


def _adamw_call(lib, ctx, n=1, how=None, **over):
    import ctypes
    from paper_2602_01469_b200 import binding
    h = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, lr_dev=None, step_dev=None, grad_scale_dev=None, seed=0)
    h.update(how or {})
    t = dict(param=4096, grad=8192, master=None, m=12288, v=16384, m_scale=None, v_scale=None, count=10, param_dtype=1,
             grad_dtype=1, weight_decay=0.0)
    t.update(over)
    arr = (binding.peagle_adamw_tensor_t * 1)(binding.peagle_adamw_tensor_t(**t))
    return lib.peagle_adamw_step(ctx, ctypes.byref(binding.peagle_adamw_t(**h)), arr, n, ctypes.c_void_p(0))


@pytest.mark.parametrize("how,over,status", [
    ({"lr": -1.0}, {}, "BAD_SHAPE"), ({"lr": float("nan")}, {}, "BAD_SHAPE"), ({"beta1": 1.0}, {}, "BAD_SHAPE"),
    ({"beta2": -0.1}, {}, "BAD_SHAPE"), ({"eps": 0.0}, {}, "BAD_SHAPE"), ({"step": 0}, {}, "BAD_SHAPE"),
    ({"step_dev": 4}, {}, "ALIGN"), ({"lr_dev": 2}, {}, "ALIGN"), ({}, {"count": -1}, "BAD_SHAPE"),
    ({}, {"param": None}, "NULL"), ({}, {"grad": None}, "NULL"), ({}, {"m": None}, "NULL"), ({}, {"v": None}, "NULL"),
    ({}, {"param": 4097}, "ALIGN"), ({}, {"m": 12290}, "ALIGN"), ({}, {"param_dtype": 7}, "BAD_SHAPE"),
    ({}, {"weight_decay": -0.1}, "BAD_SHAPE"), ({}, {"weight_decay": float("nan")}, "BAD_SHAPE"),
    ({}, {"param_dtype": 0, "master": 4096}, "BAD_SHAPE"), ({}, {"m_scale": 4096}, "BAD_SHAPE"),
    ({}, {"m_scale": 4098, "v_scale": 4096}, "ALIGN"), ({}, {"count": 1 << 41}, "TOO_LARGE"),
])
def test_adamw_refusals(lib, zeros, how, over, status):
    from paper_2602_01469_b200 import binding
    assert _adamw_call(lib, zeros, 1, how, **over) == binding.STATUS[status]


@pytest.mark.parametrize("eps", [1e-300, 1e-46, 1e-45, 1e-39, float(np.finfo(np.float32).tiny) * (1 - 2.0 ** -52), -1e-8,
                                 float("nan"), float("inf"), 1e31])
def test_adamw_refuses_an_eps_that_is_no_normal_fp32_number(lib, zeros, eps):
    from paper_2602_01469_b200 import binding
    assert _adamw_call(lib, zeros, 1, {"eps": eps}) == binding.STATUS["BAD_SHAPE"]


def test_adamw_refuses_bad_lists(lib, zeros):
    from paper_2602_01469_b200 import binding
    import ctypes
    S = binding.STATUS
    assert _adamw_call(lib, zeros, -1) == S["BAD_SHAPE"]
    assert _adamw_call(lib, None, 1) == S["NULL"]
    assert lib.peagle_adamw_step(zeros, None, None, 0, None) == S["NULL"]
    how = binding.peagle_adamw_t(1e-3, 0.9, 0.99, 1e-8, 1)
    assert lib.peagle_adamw_step(zeros, ctypes.byref(how), None, 2, None) == S["NULL"]


# ------------------------------------------------------------------ the binding's own checks, on host tensors
class _Context:
    """Device 0 and no handle: a call that came to the library would be refused as NULL."""
    h, device = None, 0


def test_binding_refuses_host_tensors(lib):
    from paper_2602_01469_b200 import binding as b
    b._know_torch()
    x, f, i = torch.zeros(3, 8), torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    calls = [
        lambda: b.peagle_norm_fwd(_Context, 0, x, None, None, 1e-5, x),
        lambda: b.peagle_norm_fwd(_Context, 0, x[0], None, None, 1e-5, x[0]),
        lambda: b.peagle_norm_bwd(_Context, 1, x, None, None, f, x, x),
        lambda: b.peagle_token_logprobs_fwd(_Context, x, i, 1.0, f),
        lambda: b.peagle_token_logprobs_fwd(_Context, x, None, 1.0, None, None, None, x, None),
        lambda: b.peagle_token_logprobs_bwd(_Context, x, i, 1.0, f, None, f, None, x),
        lambda: b.AdamWTensors([{"param": x, "grad": x, "m": x, "v": x}]),
    ]
    for call in calls:
        with pytest.raises(b.PeagleError) as e:
            call()
        assert e.value.status == b.STATUS["BAD_SHAPE"]


@pytest.mark.parametrize("rows,cols", [(1 << 31, 1), (1 << 32, 1), ((1 << 32) + 3, 1), (1, (1 << 32) + 3), (2, 1 << 31)])
def test_binding_refuses_sizes_past_int32(lib, zeros, rows, cols):
    """A size whose lower 32 bits are an ordinary size, or none: it must not be taken for that one.  (On tensors without
    memory; a call that came to the library would find NULL, or no rows to do.)"""
    import ctypes
    from paper_2602_01469_b200 import binding as b
    b._know_torch()

    class ctx:
        h, device = ctypes.addressof(zeros), -1

    def meta(*shape, dtype=torch.bfloat16):
        return torch.empty(*shape, dtype=dtype, device="meta")

    x, f, i = meta(rows, cols), meta(rows, dtype=torch.float32), meta(rows, dtype=torch.int32)
    calls = [
        lambda: b.peagle_norm_fwd(ctx, 1, x, None, None, 1e-5, x, None, f, stream=0),
        lambda: b.peagle_norm_bwd(ctx, 1, x, None, None, f, x, x, stream=0),
        lambda: b.peagle_token_logprobs_fwd(ctx, x, i, 1.0, f, stream=0),
        lambda: b.peagle_token_logprobs_bwd(ctx, x, i, 1.0, f, None, f, None, x, stream=0),
        lambda: b.peagle_token_logprobs_fwd(ctx, meta(1, 4), i[:1], 1.0, f[:1], top_logprobs=meta(1, max(rows, cols), dtype=torch.float32),
                                            top_ids=meta(1, max(rows, cols), dtype=torch.int32), stream=0),
    ]
    for call in calls:
        with pytest.raises(b.PeagleError) as e:
            call()
        assert e.value.status == b.STATUS["TOO_LARGE"]
