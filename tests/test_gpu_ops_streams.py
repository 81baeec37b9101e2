"""GPU: the operators around the layer, called at once from two streams with a context each, eagerly and as replays of
captured graphs: every output equals, bit for bit, that of the calls one after the other."""
import pytest
import torch

from paper_2602_01469_b200 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16 = torch.bfloat16


class Program:
    """A norm with its backward, log probabilities with theirs, and a step over states in 8 and in 32 bits."""

    def __init__(self, seed, rows, cols, vocab):
        gen = torch.Generator().manual_seed(seed)
        rand = lambda *shape: torch.randn(*shape, generator=gen).to(DEV)
        self.x, self.dy, self.w = rand(rows, cols).to(BF16), rand(rows, cols).to(BF16), rand(cols).to(BF16)
        self.logits = rand(rows, vocab).to(BF16)
        self.tokens = torch.randint(-1, vocab, (rows,), generator=gen).to(torch.int32).to(DEV)
        self.grad = rand(cols * 300)
        self.out = {"y": torch.empty_like(self.x), "dx": torch.empty_like(self.x), "dlogits": torch.empty_like(self.logits),
                    "top": torch.empty(rows, 20, device=DEV), "ids": torch.empty(rows, 20, dtype=torch.int32, device=DEV)}
        for name in ("mean", "rstd", "lp", "lse", "H"):
            self.out[name] = torch.empty(rows, device=DEV)
        self.out.update(dw=torch.empty(cols, device=DEV), db=torch.empty(cols, device=DEV))
        n = self.grad.numel()
        for bits in (8, 32):
            dtype = torch.uint8 if bits == 8 else torch.float32
            self.out.update({f"{name}{bits}": torch.empty(n, dtype=dtype, device=DEV) for name in ("m", "v")})
            self.out[f"p{bits}"] = torch.empty(n, device=DEV)
        self.out.update(ms=torch.empty(-(-n // 256), device=DEV), vs=torch.empty(-(-n // 256), device=DEV))
        o = self.out
        self.tensors = binding.AdamWTensors([
            {"param": o["p32"], "grad": self.grad, "m": o["m32"], "v": o["v32"]},
            {"param": o["p8"], "grad": self.grad, "m": o["m8"].view(torch.float8_e4m3fn), "v": o["v8"].view(torch.float8_e4m3fn),
             "m_scale": o["ms"], "v_scale": o["vs"]}])

    def run(self, ctx):
        o = self.out
        for name in ("dw", "db", "m8", "v8", "m32", "v32", "p8", "p32", "ms", "vs"):
            o[name].zero_()
        binding.peagle_norm_fwd(ctx, 0, self.x, self.w, None, 1e-5, o["y"], o["mean"], o["rstd"])
        binding.peagle_norm_bwd(ctx, 0, self.x, self.w, o["mean"], o["rstd"], self.dy, o["dx"], o["dw"], o["db"])
        binding.peagle_token_logprobs_fwd(ctx, self.logits, self.tokens, 1.0, o["lp"], o["lse"], o["H"], o["top"], o["ids"])
        binding.peagle_token_logprobs_bwd(ctx, self.logits, self.tokens, 1.0, o["lse"], o["H"], o["lp"], o["H"], o["dlogits"])
        for step in (1, 2):
            binding.peagle_adamw_step(ctx, self.tensors, 1e-3, 0.9, 0.98, 1e-8, step=step, seed=3)

    def take(self):
        torch.cuda.synchronize()
        got = {k: t.clone().view(torch.uint8) for k, t in self.out.items()}
        for t in self.out.values():
            t.view(torch.uint8).fill_(77)
        torch.cuda.synchronize()
        return got


@pytest.mark.parametrize("captured", [False, True])
def test_two_contexts_at_once(captured):
    contexts = [binding.Context(0), binding.Context(0)]
    graphs = []
    try:
        programs = [Program(1, 700, 2880, 9001), Program(2, 300, 1001, 40000)]
        want = []
        for c, p in zip(contexts, programs):
            p.run(c)
            want.append(p.take())
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        if captured:
            for c, p, s in zip(contexts, programs, streams):
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=s):
                    p.run(c)
                graphs.append(g)
            torch.cuda.synchronize()
        for _ in range(3):
            for _ in range(4):
                for k, s in enumerate(streams):
                    with torch.cuda.stream(s):
                        graphs[k].replay() if captured else programs[k].run(contexts[k])
            for p, w in zip(programs, want):
                got = p.take()
                for name in w:
                    assert torch.equal(got[name], w[name]), name
        assert all(binding.peagle_poll_status(c) == 0 for c in contexts)
    finally:
        graphs.clear()
        torch.cuda.synchronize()
        for c in contexts:
            c.close()
