"""The feed-forward side of one decode step with e4m3 weights: dense SwiGLU
layers and MoE layers in turn, for a few tokens.

    python -m paper_2606_22541_gb300.decode_step [--tokens 1,8,32] [--dense 1] [--moe 2] [--steps 20]

A dense layer is quantise, gate/up product, SwiGLU with quantise, down product;
a MoE layer is one asap_moe_layer_few call on a handle whose prompt batches go
through asap_moe_layer.  The step is enqueued once into a CUDA graph and
replayed; the program prints microseconds per step and the share of the time
that the weights it reads take at the given bandwidth.  Weights are random, of
the DeepSeek-V3 layer's shape; the dense layers have the inner width that a
token meets in a MoE layer (its experts' and the shared one's).
"""
import argparse

import torch

from . import api, inputs
from .configs import DSV3_FP8


class DenseFFN:
    """A SwiGLU layer in e4m3: x -> silu(x Wg^T) * (x Wu^T) Wd^T, with the
    buffers of calls of up to max_tokens tokens.  hidden and inter are multiples
    of 128 (the weights' scale blocks)."""

    def __init__(self, w_gate, w_up, w_down, max_tokens):
        """w_gate, w_up [inter, hidden], w_down [hidden, inter] fp32 on the GPU."""
        self.inter, self.hidden = w_gate.shape
        dev = w_gate.device
        self.gate_up, self.s_gate_up = inputs.quantize_block128_e4m3(torch.cat([w_gate, w_up]))
        self.down, self.s_down = inputs.quantize_block128_e4m3(w_down)
        e4m3 = dict(dtype=torch.float8_e4m3fn, device=dev)
        self.q = torch.empty((max_tokens, self.hidden), **e4m3)
        self.s = torch.empty((max_tokens, self.hidden // 128), device=dev)
        self.y = torch.empty((max_tokens, 2 * self.inter), dtype=torch.bfloat16, device=dev)
        self.hq = torch.empty((max_tokens, self.inter), **e4m3)
        self.hs = torch.empty((max_tokens, self.inter // 128), device=dev)

    def __call__(self, x, out, stream=None):
        """out [n, hidden] (bf16) = the layer of x [n, hidden] (bf16); enqueues only."""
        n, inter = x.shape[0], self.inter
        q, s, y, hq, hs = (t[:n] for t in (self.q, self.s, self.y, self.hq, self.hs))
        api.asap_moe_fp8_quantize(x, q, s, stream)
        api.asap_moe_fp8_matmul(q, s, self.gate_up, self.s_gate_up, y, stream)
        api.asap_moe_fp8_swiglu_quantize(y[:, :inter], y[:, inter:], hq, hs, stream)
        api.asap_moe_fp8_matmul(hq, hs, self.down, self.s_down, out, stream)

    def weight_bytes(self):
        return self.gate_up.numel() + self.down.numel()


class DecodeStep:
    """Dense layers, then the MoE layers of a handle, each added to its input."""

    def __init__(self, dense, handle, n_tokens, device="cuda"):
        self.dense, self.handle = dense, handle
        self.n_moe = api.asap_moe_n_layers(handle)
        self.ids = torch.arange(self.n_moe, dtype=torch.int32, device=device)
        self.ws = api.workspace(handle, n_tokens, device)
        self.y = torch.empty((n_tokens, handle.cfg.hidden), dtype=torch.bfloat16, device=device)

    def __call__(self, x):
        """Adds every layer's output to x [n, hidden] (bf16) in place, on the current stream."""
        y = self.y[:x.shape[0]]
        for layer in self.dense:
            layer(x, y)
            x += y
        for i in range(self.n_moe):
            api.asap_moe_layer_few(self.handle, x, y, self.ws, layer_id=self.ids[i:i + 1])
            x += y


def _dense_layer(hidden, inter, max_tokens, seed, device):
    def w(rows, cols, i):
        g = torch.Generator(device=device)
        g.manual_seed(seed * 10 + i)
        return torch.randn((rows, cols), generator=g, device=device) * cols ** -0.5

    return DenseFFN(w(inter, hidden, 1), w(inter, hidden, 2), w(hidden, inter, 3), max_tokens)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", default="1,8,32", help="tokens of a step, comma-separated (each at most 64)")
    ap.add_argument("--dense", type=int, default=1, help="dense layers")
    ap.add_argument("--moe", type=int, default=2, help="MoE layers")
    ap.add_argument("--steps", type=int, default=20, help="replays timed")
    ap.add_argument("--gbs", type=float, default=6786.0, help="bandwidth the share is taken of, GB/s")
    a = ap.parse_args(argv)
    sizes = [int(t) for t in a.tokens.split(",")]
    cfg = DSV3_FP8
    inter = cfg.inter * cfg.top_k + cfg.shared_inter * cfg.n_shared
    handle = api.asap_moe_create_layers(cfg, inputs.make_layer_weights(cfg, a.moe, "cuda"), max(sizes))
    dense = [_dense_layer(cfg.hidden, inter, max(sizes), 100 + i, "cuda") for i in range(a.dense)]
    for n in sizes:
        step = DecodeStep(dense, handle, n)
        x0 = inputs.make_tokens(cfg, n, 0, "cuda")
        x = x0.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())  # which makes the weights, the ids and x
        with torch.cuda.stream(side):
            step(x)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            x.copy_(x0)
            step(x)
        for _ in range(3):
            graph.replay()
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        torch.cuda.synchronize()
        ev[0].record()
        for _ in range(a.steps):
            graph.replay()
        ev[1].record()
        torch.cuda.synchronize()
        us = ev[0].elapsed_time(ev[1]) * 1e3 / a.steps
        # the experts that the first MoE layer's tokens chose, from the routing call of the prompt path
        z, y = x0.clone(), torch.empty_like(x0)
        for layer in dense:
            layer(z, y)
            z += y
        i32 = dict(dtype=torch.int32, device="cuda")
        idx, counts = torch.empty((n, cfg.top_k), **i32), torch.empty(cfg.n_experts, **i32)
        api.asap_moe_route(handle, z, idx, torch.empty((n, cfg.top_k), device="cuda"), counts,
                           torch.empty(cfg.n_experts + 1, **i32), step.ws)
        active = int((counts > 0).sum())
        expert = 3 * cfg.hidden * cfg.inter
        moe = active * expert + 3 * cfg.hidden * cfg.shared_inter + 2 * cfg.n_experts * cfg.hidden
        read = sum(d.weight_bytes() for d in dense) + a.moe * moe
        code, word = api.asap_moe_status(handle)
        if code:
            raise RuntimeError(f"device status word {word:#x}")
        print(f"{n:3d} tokens: {us:8.1f} us per step, about {read / 1e6:.0f} MB of weights ({active} experts in the first "
              f"MoE layer), {read / us / 1e3 / a.gbs:.2f} of {a.gbs:.0f} GB/s, status {word}", flush=True)
    handle.close()


if __name__ == "__main__":
    main()
