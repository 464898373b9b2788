"""A stack of decayed linear-attention layers served from one state pool.

Prompts of different lengths fill the requests' slots (stepq_linattn_prefill), then every
request takes one token a step (stepq_linattn_decode_step, the whole stack one CUDA graph).
Each layer is: RMS norm of the residual stream (stepq_group_norm), one projection to q, k, v
and the gate z, whose columns the calls read in place, the attention with its group norm and
gate, and a projection back. The projections are torch's.

    python -m paper_2609_38169_gb300.linear_layers --requests 64 --tokens 256

At its end the command serves every request again as one longer prompt, and prints how far
states and outputs of the two ways are apart.
"""
from __future__ import annotations

import argparse
import json

from . import api as A


class LinearLayers:
    """Random weights of `layers` layers and a pool of `slots` states."""

    def __init__(self, layers, slots, hidden=1024, hk=2, hv=8, dtype=None, device="cuda", seed=0):
        import torch
        self.torch, self.dtype = torch, dtype or torch.bfloat16
        self.cfg = A.Config(n_layers=layers, n_key_heads=hk, n_value_heads=hv)
        g = torch.Generator(device=device).manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device=device)  # noqa: E731
        cols = [hk * A.D, hk * A.D, hv * A.D, hv * A.D]
        self.cuts = [sum(cols[:i]) for i in range(5)]
        self.proj = (rand(layers, hidden, self.cuts[4]) / hidden ** 0.5).to(self.dtype)
        self.back = (rand(layers, hv * A.D, hidden) / (hv * A.D) ** 0.5).to(self.dtype)
        self.decay = rand(layers, hidden, hv) / hidden ** 0.5
        self.w_in, self.w_out = 1 + 0.1 * rand(layers, hidden), 1 + 0.1 * rand(layers, hv * A.D)
        self.pool = torch.zeros((slots, layers, hv, A.D, A.D), device=device)

    def _stack(self, x, attend):
        torch = self.torch
        for i in range(self.cfg.n_layers):
            h = torch.empty_like(x)
            A.stepq_group_norm(x, 1, h, A.Norm(weight=self.w_in[i], act=A.ACT_NONE, center=False))
            p = h @ self.proj[i]
            q, k, v, z = (p[:, a:b].unflatten(1, (-1, A.D)) for a, b in zip(self.cuts, self.cuts[1:]))
            gate = torch.sigmoid(h.float() @ self.decay[i] + 4.0)
            y = torch.empty(v.shape, dtype=self.dtype, device=x.device)
            attend(i, q, k / A.D ** 0.5, v, gate, y, A.Norm(weight=self.w_out[i], z=z, act=A.ACT_SILU))
            x = x + y.flatten(1) @ self.back[i]
        out = torch.empty_like(x)
        A.stepq_group_norm(x, 1, out, A.Norm(act=A.ACT_NONE, center=False))
        return out

    def prompts(self, x, slots, cu_seqlens, max_len, resume):
        """x [tokens][hidden] of the requests in `slots`, packed; resume uint8 [requests]."""
        return self._stack(x, lambda i, q, k, v, g, y, n: A.stepq_linattn_prefill(
            self.cfg, i, self.pool, slots, q, k, v, g, y, cu_seqlens=cu_seqlens, max_len=max_len, resume=resume, norm=n))

    def tokens(self, x, slots):
        """One token a request: x [requests][hidden]."""
        return self._stack(x, lambda i, q, k, v, g, y, n: A.stepq_linattn_decode_step(
            self.cfg, i, self.pool, slots, q, k, v, g, y, norm=n))


def serve(requests=16, tokens=64, longest=700, layers=4, hk=2, hv=8, hidden=1024, dtype=None, seed=0):
    """Prompts, then `tokens` tokens a request; the result is compared with one prompt of both."""
    import torch
    model = LinearLayers(layers, requests, hidden, hk, hv, dtype, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    lens = torch.randint(1, longest + 1, (requests,), generator=torch.Generator().manual_seed(seed)).tolist()
    slots = torch.randperm(requests, generator=g, device="cuda").to(torch.int32)
    new = torch.zeros(requests, dtype=torch.uint8, device="cuda")

    def bounds(extra):
        return torch.tensor([sum(lens[:b]) + extra * b for b in range(requests + 1)], dtype=torch.int32, device="cuda")

    def timed(f):
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        ev[0].record()
        r = f()
        ev[1].record()
        torch.cuda.synchronize()
        return r, ev[0].elapsed_time(ev[1])

    cu = bounds(0)
    x = torch.randn((sum(lens), hidden), generator=g, device="cuda").to(model.dtype)
    model.prompts(x, slots, cu, max(lens), new)                     # once before the clock
    out, prompt_ms = timed(lambda: model.prompts(x, slots, cu, max(lens), new))
    state = model.pool.clone()
    last = out[cu[1:].long() - 1].clone()
    model.tokens(last, slots)                                       # before the capture, and undone
    model.pool.copy_(state)
    step_in = last.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step_out = model.tokens(step_in, slots)
    fed, got = [], []

    def steps():
        for _ in range(tokens):
            fed.append(step_in.clone())
            graph.replay()
            got.append(step_out.clone())
            step_in.copy_(step_out)

    _, token_ms = timed(steps)
    # The same requests as prompts that hold the tokens too.
    served = model.pool.clone()
    rows = [torch.cat([x[a:a + n]] + [f[b:b + 1] for f in fed]) for b, (a, n) in enumerate(zip(cu.tolist(), lens))]
    whole = model.prompts(torch.cat(rows), slots, bounds(tokens), max(lens) + tokens, new)
    ends = bounds(tokens)[1:].long() - 1
    apart = lambda a, b: float((a.double() - b.double()).norm() / b.double().norm())  # noqa: E731
    return {"requests": requests, "prompt_tokens": sum(lens), "prompt_ms": round(prompt_ms, 3),
            "tokens": requests * tokens, "token_ms": round(token_ms, 3),
            "states_apart": apart(served, model.pool), "outputs_apart": apart(got[-1], whole[ends]) if tokens else 0.0,
            "device_error": A.stepq_device_error()}


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("requests", 16), ("tokens", 64), ("longest", 700), ("layers", 4), ("hk", 2), ("hv", 8),
                        ("hidden", 1024), ("seed", 0)):
        ap.add_argument(f"--{name}", type=int, default=value)
    ap.add_argument("--dtype", choices=["bfloat16", "float16", "float32"], default="bfloat16")
    args = vars(ap.parse_args(argv))
    import torch
    print(json.dumps(serve(**{**args, "dtype": getattr(torch, args["dtype"])})))


if __name__ == "__main__":
    main()
