"""A sparse MLP block as a language model runs it between its attention layers, on this library's entry points:

  x -> 4-bit projection -> router GEMM -> routing -> the chosen experts' products (+ the residual of the projection)

    python examples/sparse_mlp.py [--tokens 1 64 2048] [--experts 64] [--top-k 6] [--width 2048] [--hidden 1024] [--weights w4]

One HIP graph per batch size holds the block's launches; prints the time per pass and checks a few tokens against float64.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2110_15238_amd as bolt  # noqa: E402

GROUP = 128


def quantise(w):
    """[count][N][K] weights to 4 bits: for every group of a row a scale and zero point that span its values."""
    count, N, K = w.shape
    groups = -(-K // GROUP)
    v = torch.nn.functional.pad(w.float(), (0, groups * GROUP - K)).view(count, N, groups, GROUP)
    lo, hi = v.amin(3).clamp(max=0), v.amax(3).clamp(min=0)
    scales = ((hi - lo) / 15).clamp(min=1e-6).half()
    zeros = (-lo / scales.float()).round().clamp(0, 15).to(torch.uint8)
    q = (v / scales.float()[..., None] + zeros[..., None]).round().clamp(0, 15).to(torch.uint8).view(count, N, -1)[:, :, :K]
    held = scales.double().repeat_interleave(GROUP, 2)[:, :, :K] * (q.double() - zeros.double().repeat_interleave(GROUP, 2)[:, :, :K])
    packed = torch.empty(bolt.bolt_w4_packed_bytes(N, K, GROUP, count), dtype=torch.uint8, device=w.device)
    bolt.bolt_w4_pack(N, K, GROUP, (q[..., 0::2] | q[..., 1::2] << 4).contiguous(), scales, zeros, packed)
    return packed, held


class SparseMlp:
    def __init__(self, tokens, experts, top_k, width, hidden, weights, proj, router, up, down):
        empty = lambda *s, dtype=torch.float16: torch.empty(s, dtype=dtype, device="cuda")
        nbytes = lambda n: empty(n, dtype=torch.uint8)
        self.proj, self.router, self.up, self.down = proj, router, up, down
        self.x, self.p, self.logits, self.y = empty(tokens, width), empty(tokens, width), empty(tokens, experts), empty(tokens, width)
        self.proj_desc = bolt.gemm_w4_desc(tokens, width, width, GROUP)
        self.router_desc = bolt.gemm_desc(tokens, experts, width, act="none", b_layout=bolt.LAYOUT_NK)
        self.route_desc = bolt.moe_route_desc(tokens, experts, top_k)
        self.moe_desc = bolt.moe_desc(tokens, experts, top_k, width, hidden, act="silu", gated=True, weights=weights, group=GROUP)
        self.plan = (empty(tokens, top_k, dtype=torch.int32), empty(tokens, top_k, dtype=torch.float32),
                     empty(experts + 1, dtype=torch.int32), empty(tokens * top_k, dtype=torch.int32))
        self.proj_ws = nbytes(bolt.bolt_gemm_w4_workspace_bytes(self.proj_desc))
        self.route_ws = nbytes(bolt.bolt_moe_route_workspace_bytes(self.route_desc))
        self.moe_ws = nbytes(bolt.bolt_moe_workspace_bytes(self.moe_desc))

    def __call__(self):
        bolt.bolt_gemm_w4(self.proj_desc, self.x, self.proj, None, self.p, self.proj_ws)
        bolt.bolt_gemm_epilogue(self.router_desc, self.p, self.router, None, self.logits)
        bolt.bolt_moe_route(self.route_desc, self.logits, None, None, *self.plan, self.route_ws)
        bolt.bolt_moe_experts(self.moe_desc, self.p, self.up, None, self.down, None, *self.plan, self.y, self.moe_ws)
        self.y += self.p
        return self.y


def check(block, up, down, hidden):
    """A few tokens' experts in float64, from the projection and the routing that the block computed."""
    ids, w = block.plan[0], block.plan[1]
    for t in {0, block.x.shape[0] // 2, block.x.shape[0] - 1}:
        x = block.p[t].double()
        want = x.clone()
        for e, s in zip(ids[t].tolist(), w[t].double()):
            u = up[e].double() @ x
            want += s * (down[e].double() @ (u[:hidden] * torch.sigmoid(u[:hidden]) * u[hidden:]))
        err = (block.y[t].double() - want).abs().max().item()
        assert err <= 1e-2 * (1 + want.abs().max().item()), (t, err)


def main():
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--tokens", type=int, nargs="+", default=[1, 64, 2048])
    a.add_argument("--experts", type=int, default=64)
    a.add_argument("--top-k", type=int, default=6)
    a.add_argument("--width", type=int, default=2048)
    a.add_argument("--hidden", type=int, default=1024)
    a.add_argument("--weights", choices=("f16", "w4"), default="w4")
    a = a.parse_args()
    torch.manual_seed(0)
    normal = lambda *s, std: torch.empty(s, dtype=torch.float16, device="cuda").normal_(0, std)
    proj, _ = quantise(normal(1, a.width, a.width, std=1 / math.sqrt(a.width)))
    router = normal(a.experts, a.width, std=2 / math.sqrt(a.width))
    up = held_up = normal(a.experts, 2 * a.hidden, a.width, std=1 / math.sqrt(a.width))
    down = held_down = normal(a.experts, a.width, a.hidden, std=1 / math.sqrt(a.hidden))
    if a.weights == "w4":
        (up, held_up), (down, held_down) = quantise(up), quantise(down)
    for tokens in a.tokens:
        block = SparseMlp(tokens, a.experts, a.top_k, a.width, a.hidden, a.weights, proj, router, up, down)
        block.x.normal_()
        block()
        torch.cuda.synchronize()
        check(block, held_up, held_down, a.hidden)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            block()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for _ in range(3):
            graph.replay()
        begin.record()
        for _ in range(20):
            graph.replay()
        end.record()
        torch.cuda.synchronize()
        print("%5d tokens: %8.1f us per pass (%d experts, %d per token, %d x %d, %s)" %
              (tokens, begin.elapsed_time(end) * 50, a.experts, a.top_k, a.width, a.hidden, a.weights))


if __name__ == "__main__":
    main()
