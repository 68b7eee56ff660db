"""The projections around a served model's MLP, with weights in 8 bits and requests that bring low-rank adapters, on this library's entry points:

  x + residual stream -> norm, in FP16 and in 8 bits -> 8-bit up projection with SiLU -> rows in 8 bits -> 8-bit down projection
                                                     -> a projection shared by the requests, each with its own adapter

    python examples/served_layer.py [--tokens 1 32 2048] [--width 4096] [--hidden 8192] [--adapters 8] [--rank 16] [--weights w4]

One HIP graph per batch size holds the layer's launches; prints the time per pass and checks a few rows against float64.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2110_15238_amd as bolt  # noqa: E402

GROUP = 128


def empty(*shape, dtype=torch.float16):
    return torch.empty(shape, dtype=dtype, device="cuda")


def in_8_bits(w):
    return bolt.bolt_quantize_rows(w, empty(*w.shape, dtype=torch.float8_e4m3fn), empty(w.shape[0], dtype=torch.float32))


class ServedLayer:
    def __init__(self, tokens, weight, up, down, shared, weights, adapters):
        (self.up, self.up_scales), (self.down, self.down_scales) = up, down
        hidden, width = self.up.shape
        n, out, rank = adapters[1].shape
        self.weight, self.shared, self.adapters = weight, shared, adapters
        self.x, self.stream, self.normed = empty(tokens, width), empty(tokens, width), empty(tokens, width)
        self.rows, self.row_scales = empty(tokens, width, dtype=torch.float8_e4m3fn), empty(tokens, dtype=torch.float32)
        self.hidden, self.y, self.projected = empty(tokens, hidden), empty(tokens, width), empty(tokens, out)
        self.hidden_rows, self.hidden_scales = empty(tokens, hidden, dtype=torch.float8_e4m3fn), empty(tokens, dtype=torch.float32)
        self.ids = empty(tokens, dtype=torch.int32)
        self.norm = bolt.rms_norm_desc(tokens, width)
        self.up_desc, self.down_desc = bolt.gemm_q8_desc(tokens, hidden, width, act="silu"), bolt.gemm_q8_desc(tokens, width, hidden)
        self.lora = bolt.gemm_lora_desc(tokens, out, width, n, rank, weights=weights, group=GROUP)
        self.workspace = empty(bolt.bolt_gemm_lora_workspace_bytes(self.lora), dtype=torch.uint8)

    def __call__(self):
        # (the residual stream is updated in place)
        bolt.bolt_rms_norm(self.norm, self.x, self.stream, self.weight, self.stream, self.normed, self.rows, self.row_scales)
        bolt.bolt_gemm_q8(self.up_desc, self.rows, self.row_scales, self.up, self.up_scales, None, self.hidden)
        bolt.bolt_quantize_rows(self.hidden, self.hidden_rows, self.hidden_scales)
        bolt.bolt_gemm_q8(self.down_desc, self.hidden_rows, self.hidden_scales, self.down, self.down_scales, None, self.y)
        down, up, scales = self.adapters
        bolt.bolt_gemm_lora(self.lora, self.normed, self.shared, None, self.ids, down, up, scales, self.projected, self.workspace)
        return self.y, self.projected


def check(layer, stream, shared, weight):
    """A few rows in float64, from the rows in 8 bits that the layer computed."""
    down, up, scales = layer.adapters
    for t in {0, layer.x.shape[0] // 2, layer.x.shape[0] - 1}:
        v = layer.x[t].double() + stream[t].double()
        n = v / (v.square().mean() + 1e-5).sqrt() * weight.double()
        want_h = layer.up.double() @ layer.rows[t].double() * layer.up_scales.double() * layer.row_scales[t].double()
        want_h = want_h * torch.sigmoid(want_h)
        want_y = layer.down.double() @ layer.hidden_rows[t].double() * layer.down_scales.double() * layer.hidden_scales[t].double()
        want_p = shared @ layer.normed[t].double()
        a = int(layer.ids[t])
        if a >= 0:
            want_p = want_p + scales[a].double() * (up[a].double() @ (down[a].double() @ layer.normed[t].double()))
        for got, want in ((layer.normed[t], n), (layer.hidden[t], want_h), (layer.y[t], want_y), (layer.projected[t], want_p)):
            err = (got.double() - want).abs().max().item()
            assert err <= 1e-2 * (1 + want.abs().max().item()), (t, err)


def main():
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--tokens", type=int, nargs="+", default=[1, 32, 2048])
    a.add_argument("--width", type=int, default=4096)
    a.add_argument("--hidden", type=int, default=8192)
    a.add_argument("--adapters", type=int, default=8)
    a.add_argument("--rank", type=int, default=16)
    a.add_argument("--weights", choices=("f16", "w4"), default="f16")
    a = a.parse_args()
    torch.manual_seed(0)
    normal = lambda *s, std: empty(*s).normal_(0, std)
    weight = normal(a.width, std=0.1) + 1
    up, down = in_8_bits(normal(a.hidden, a.width, std=1 / math.sqrt(a.width))), in_8_bits(normal(a.width, a.hidden, std=1 / math.sqrt(a.hidden)))
    adapters = (normal(a.adapters, a.rank, a.width, std=1 / math.sqrt(a.width)), normal(a.adapters, a.width, a.rank, std=0.2 / math.sqrt(a.rank)),
                torch.rand(a.adapters, device="cuda") + 0.5)
    if a.weights == "w4":
        q = torch.randint(0, 256, (a.width, a.width // 2), dtype=torch.uint8, device="cuda")
        scales = torch.full((a.width, -(-a.width // GROUP)), 0.2 / math.sqrt(a.width), device="cuda").half()
        shared = bolt.bolt_w4_pack(a.width, a.width, GROUP, q, scales, None, empty(bolt.bolt_w4_packed_bytes(a.width, a.width, GROUP), dtype=torch.uint8))
        held = (torch.stack((q & 15, q >> 4), 2).view(a.width, a.width).double() - 8) * scales[0, 0].double()
    else:
        shared = normal(a.width, a.width, std=1 / math.sqrt(a.width))
        held = shared.double()
    for tokens in a.tokens:
        layer = ServedLayer(tokens, weight, up, down, shared, a.weights, adapters)
        layer.x.normal_()
        layer.stream.normal_()
        layer.ids.copy_(torch.arange(tokens, device="cuda") * (a.adapters + 1) // tokens - 1)
        before = layer.stream.clone()
        layer()
        torch.cuda.synchronize()
        check(layer, before, held, weight)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer()
        layer.x.zero_()  # (or the stream would grow)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for _ in range(3):
            graph.replay()
        begin.record()
        for _ in range(20):
            graph.replay()
        end.record()
        torch.cuda.synchronize()
        print("%5d tokens: %8.1f us per pass (%d wide, %d hidden, %d adapters of rank %d, shared projection in %s)" %
              (tokens, begin.elapsed_time(end) * 50, a.width, a.hidden, a.adapters, a.rank, a.weights))


if __name__ == "__main__":
    main()
