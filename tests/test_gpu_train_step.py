"""GPU: one training step put together from the library's calls as a program would: norm, projection, rotary
prologue, attention, logits, log probabilities of the tokens with entropy, all of it backward, and AdamW on the
three weights.

Against the same chain in fp64 with torch's autograd (the mask from the oracle).  Tolerance of the gradients, as for
the layer: the chain rounds to bf16 at every interface (normed rows, fused rows, Q / K / V, probabilities, O, logits,
their gradient, dO, dQ / dK / dV, the fused rows' gradient), each time by at most 2^-8 relative, 1.1e-3 to 2.2e-3 rms,
independently: a dozen give 4e-3 to 8e-3, and the roundings of scores and logits pass through two softmaxes.  Bound 2e-2
in the relative 2-norm.  The weights after the step are compared with the definition applied to the gradients that the
library has found (a step divides by the root of the gradient's square: it would magnify the rest)."""
import math

import numpy as np
import pytest
import torch

from oracle import ops_oracle as oo
from oracle import peagle_oracle as orc
from paper_2602_01469_b200 import binding, inputs
from tests.gpu_common import rel_l2

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
BASE, EPS, ENT = 500000.0, 1e-5, 0.02
HQ, HKV, D, DM, VOCAB = 4, 2, 64, 200, 1000
WIDTH = (HQ + 2 * HKV) * D


def reference(x, wn, w, wv, anchor, depth, tokens, scale):
    """Loss gradients in fp64."""
    leaves = [t.double().requires_grad_(True) for t in (x, wn, w, wv)]
    x, wn, w, wv = leaves
    T = x.shape[0]
    fused = x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * wn @ w.t()
    pos = torch.tensor(anchor + depth, dtype=torch.float64)
    ang = pos[:, None] * torch.tensor([BASE ** (-2.0 * i / D) for i in range(D // 2)], dtype=torch.float64)[None]
    cos, sin = torch.cos(ang)[:, None], torch.sin(ang)[:, None]

    def rot(t):
        lo, hi = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)

    q = rot(fused[:, :HQ * D].reshape(T, HQ, D))
    k = rot(fused[:, HQ * D:(HQ + HKV) * D].reshape(T, HKV, D)).repeat_interleave(HQ // HKV, 1)
    v = fused[:, (HQ + HKV) * D:].reshape(T, HKV, D).repeat_interleave(HQ // HKV, 1)
    mask = torch.tensor(orc.mask_dense(anchor, depth).astype(bool))
    s = (torch.einsum("qhd,khd->hqk", q, k) * scale).masked_fill(~mask[None], -math.inf)
    o = torch.einsum("hqk,khd->qhd", torch.softmax(s, -1), v).reshape(T, HQ * D)
    logp = torch.log_softmax(o @ wv.t(), 1)
    given = tokens >= 0
    lp = logp.gather(1, tokens.clamp(min=0).long()[:, None])[:, 0] * given
    ent = -(logp.exp() * logp).sum(1)
    loss = -(lp.sum() / given.sum()) - ENT * ent.mean()
    loss.backward()
    return loss.item(), [t.grad.numpy() for t in leaves]


@pytest.mark.parametrize("bits", [32, 8])
def test_a_training_step(bits):
    ctx = binding.Context(0)
    try:
        w_ = inputs.Workload("train", (70,), 4, HQ, HKV, D, seed=5)
        cu, anchor, depth, parts = inputs.build_case(w_, binding.peagle_assign_segments)
        T = int(cu[-1])
        gen = torch.Generator().manual_seed(3)
        master = {"wn": 1 + 0.1 * torch.randn(DM, generator=gen), "w": torch.randn(WIDTH, DM, generator=gen) / math.sqrt(DM),
                  "wv": torch.randn(VOCAB, HQ * D, generator=gen) / math.sqrt(HQ * D)}
        x = (1.5 * torch.randn(T, DM, generator=gen)).to(BF16)
        par = {n: t.to(BF16) for n, t in master.items()}
        master = {n: t.float() for n, t in par.items()}      # both sides start from the same numbers
        tokens = torch.randint(VOCAB, (T,), generator=gen).to(torch.int32)
        tokens[::9] = -1
        loss, want = reference(x.float(), *(par[n].float() for n in ("wn", "w", "wv")), anchor, depth, tokens, w_.scale)

        e = lambda *s, dtype=BF16: torch.full(s, float("nan"), dtype=dtype, device=DEV)
        z = lambda *s: torch.zeros(*s, dtype=F32, device=DEV)
        x, tokens = x.to(DEV), tokens.to(DEV)
        wn, w, wv = (par[n].to(DEV) for n in ("wn", "w", "wv"))
        a, d = torch.from_numpy(anchor).to(DEV), torch.from_numpy(depth).to(DEV)
        prob = binding.Problem(cu, a, d, w_.K, HQ, HKV, D, w_.scale)
        part = binding.Partition(parts[0]["seq"], parts[0]["q"], parts[0]["k"])
        # forward
        xn, rstd, fused = e(T, DM), e(T, dtype=F32), e(T, WIDTH)
        binding.peagle_norm_fwd(ctx, binding.NORM["rms"], x, wn, None, EPS, xn, None, rstd)
        binding.peagle_gemm_bf16(ctx, xn, DM, 0, w, DM, 0, fused, WIDTH, 0, T, WIDTH, DM)
        Q, K, V, O, LSE = e(T, HQ, D), e(T, HKV, D), e(T, HKV, D), e(T, HQ, D), e(HQ, T, dtype=F32)
        binding.peagle_rope_qkv_fwd(ctx, fused, a, d, HQ, HKV, D, BASE, Q, K, V)
        binding.peagle_attn_fwd(ctx, prob, part, Q, K, V, O, LSE)
        logits, lp, lse, ent = e(T, VOCAB), e(T, dtype=F32), e(T, dtype=F32), e(T, dtype=F32)
        binding.peagle_gemm_bf16(ctx, O, HQ * D, 0, wv, HQ * D, 0, logits, VOCAB, 0, T, VOCAB, HQ * D)
        binding.peagle_token_logprobs_fwd(ctx, logits, tokens, 1.0, lp, lse, ent)
        given = int((tokens >= 0).sum())
        got = float(-(lp.sum() / given) - ENT * ent.mean())
        assert got == pytest.approx(loss, rel=5e-3)           # logits rounded to bf16: 2^-9 of about 4, averaged
        # backward; the logits' gradient in the logits' place
        binding.peagle_token_logprobs_bwd(ctx, logits, tokens, 1.0, lse, ent, torch.full((T,), -1.0 / given, device=DEV),
                                          torch.full((T,), -ENT / T, device=DEV), logits)
        dO, dwv = e(T, HQ, D), z(VOCAB, HQ * D)
        binding.peagle_gemm_bf16(ctx, logits, VOCAB, 0, wv, HQ * D, 1, dO, HQ * D, 0, T, HQ * D, VOCAB)
        binding.peagle_gemm_bf16(ctx, logits, VOCAB, 1, O, HQ * D, 1, dwv, HQ * D, 1, VOCAB, HQ * D, T)
        dQ, dKa, dVa, dK, dV = e(T, HQ, D), z(T, HKV, D), z(T, HKV, D), e(T, HKV, D), e(T, HKV, D)
        binding.peagle_attn_bwd(ctx, prob, part, Q, K, V, O, dO, LSE, dQ, dKa, dVa)
        binding.peagle_cast_grads(ctx, dKa, dVa, dK, dV)
        dfused, dxn, dw = e(T, WIDTH), e(T, DM), z(WIDTH, DM)
        binding.peagle_rope_qkv_bwd(ctx, dQ, dK, dV, a, d, HQ, HKV, D, BASE, dfused)
        binding.peagle_gemm_bf16(ctx, dfused, WIDTH, 0, w, DM, 1, dxn, DM, 0, T, DM, WIDTH)
        binding.peagle_gemm_bf16(ctx, dfused, WIDTH, 1, xn, DM, 1, dw, DM, 1, WIDTH, DM, T)
        dx, dwn = e(T, DM), z(DM)
        binding.peagle_norm_bwd(ctx, binding.NORM["rms"], x, wn, None, rstd, dxn, dx, dwn)
        assert binding.peagle_poll_status(ctx) == 0
        errs = [rel_l2(g.float().cpu().numpy(), t) for g, t in zip((dx, dwn, dw, dwv), want)]
        print("relative errors of dx, dwn, dw, dwv:", errs)
        assert max(errs) <= 2e-2
        # the step: fp32 masters, the summed fp32 gradients as they are
        how = dict(lr=1e-3, beta1=0.9, beta2=0.98, eps=1e-8)
        items = []
        for name, p, g in (("wn", wn, dwn), ("w", w, dw), ("wv", wv, dwv)):
            n = p.numel()
            blocks = -(-n // binding.ADAMW_BLOCK)
            states = ({"m": z(n), "v": z(n)} if bits == 32 else
                      {"m": z(n).to(torch.float8_e4m3fn), "v": z(n).to(torch.float8_e4m3fn), "m_scale": z(blocks), "v_scale": z(blocks)})
            items.append({"param": p, "grad": g, "master": master[name].to(DEV), "weight_decay": 0.1 if p.dim() > 1 else 0.0,
                          **states})
        binding.peagle_adamw_step(ctx, binding.AdamWTensors(items), step=1, seed=1, **how)
        torch.cuda.synchronize()
        for name, i in zip(("wn", "w", "wv"), items):
            p0, g = master[name].double().numpy().ravel(), i["grad"].double().cpu().numpy().ravel()
            p1, _, _ = oo.adamw(p0, g, 0.0, 0.0, how["lr"], 0.9, 0.98, 1e-8, i["weight_decay"], 1)
            # at step 1 the update is about lr: 20 roundings of it, three of p
            bound = 20 * 2.0 ** -24 * how["lr"] + 3 * 2.0 ** -24 * np.abs(p0) + 2e-11
            assert (np.abs(i["master"].double().cpu().numpy().ravel() - p1) <= bound).all(), name
            assert torch.equal(i["param"], i["master"].to(BF16))
    finally:
        ctx.close()
