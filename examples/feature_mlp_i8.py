"""The MLP of a block over a feature map with 8-bit products: tokens normalised by groups, quantised, multiplied, and added back.

    hb_conv3x3 (64 channels, NHWC)  ->  hb_group_norm with silu  ->  hb_linear (a 1x1 convolution to the width of the tokens)
    hb_group_norm  ->  hb_quantize_rows (a scale per token)  ->  hb_linear_i8 with gelu (to the hidden width)
    hb_quantize_rows  ->  hb_linear_i8 with bias and residual

Weights are 8-bit with a scale per output channel, made once by hb_quantize_rows.  Random weights; ``python examples/feature_mlp_i8.py`` runs it on the GPU and prints its time
beside that of the same MLP with fp16 products.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2512_02371_amd import hb


class FeatureMlpI8:
    """`images` feature maps of size x size pixels and 64 channels, tokens of `width` channels, `hidden` between the two products."""

    def __init__(self, images, size, width=1024, hidden=4096, groups=32, seed=1, device="cuda"):
        self.images, self.pixels, self.width, self.groups = images, size * size, width, groups
        gen = torch.Generator(device=device).manual_seed(seed)
        normal = lambda *shape, std=1.0: torch.randn(shape, generator=gen, device=device).mul_(std).half()
        self.conv = torch.randn((3, 3, 64, 64), generator=gen, device=device).div_(24.0).half()
        self.norms = {n: (normal(c, std=0.1).add_(1.0), normal(c, std=0.1)) for n, c in (("features", 64), ("tokens", width))}
        self.w = {"in": normal(width, 64, std=0.125), "up": normal(hidden, width, std=width ** -0.5), "down": normal(width, hidden, std=hidden ** -0.5)}
        self.b = {name: normal(w.shape[0], std=0.1) for name, w in self.w.items()}
        self.w8 = {}
        for name in ("up", "down"):
            w = self.w[name]
            self.w8[name] = hb.hb_quantize_rows(w, torch.empty(w.shape, dtype=torch.int8, device=device), torch.empty(w.shape[0], device=device))
        # buffers and scratch memory live as long as the weights: a pass allocates nothing
        M = images * self.pixels
        f16, i8, f32 = (lambda *s, t=t: torch.empty(s, dtype=t, device=device) for t in (torch.float16, torch.int8, torch.float32))
        self.features, self.x, self.normed, self.hidden, self.out = f16(images, size, size, 64), f16(M, width), f16(M, width), f16(M, hidden), f16(M, width)
        self.x8, self.x_scale, self.h8, self.h_scale = i8(M, width), f32(M), i8(M, hidden), f32(M)
        need = [hb.hb_group_norm_workspace_size(images, self.pixels, c, groups) for c in (64, width)]
        need += [size_of(M, *w.shape) for w in self.w.values() for size_of in (hb.hb_linear_i8_workspace_size, hb.hb_linear_workspace_size)]
        self.workspace = torch.empty(max(need), dtype=torch.uint8, device=device) if max(need) else None

    def tokens(self, pixels):
        hb.hb_conv3x3(pixels, self.conv, self.features)
        hb.hb_group_norm(self.features, self.features, self.groups, *self.norms["features"], act="silu", workspace=self.workspace)              # in place
        return hb.hb_linear(self.features.view(-1, 64), self.w["in"], self.x, self.workspace, self.b["in"])

    def _normed(self):
        shape = (self.images, self.pixels, self.width)
        return hb.hb_group_norm(self.x.view(shape), self.normed.view(shape), self.groups, *self.norms["tokens"], workspace=self.workspace).view(-1, self.width)

    def mlp(self):
        hb.hb_quantize_rows(self._normed(), self.x8, self.x_scale)
        hb.hb_linear_i8(self.x8, self.w8["up"][0], self.x_scale, self.w8["up"][1], self.hidden, self.workspace, self.b["up"], None, "gelu")
        hb.hb_quantize_rows(self.hidden, self.h8, self.h_scale)
        return hb.hb_linear_i8(self.h8, self.w8["down"][0], self.h_scale, self.w8["down"][1], self.out, self.workspace, self.b["down"], self.x)

    def mlp_in_fp16(self):
        hb.hb_linear(self._normed(), self.w["up"], self.hidden, self.workspace, self.b["up"], None, "gelu")
        return hb.hb_linear(self.hidden, self.w["down"], self.out, self.workspace, self.b["down"], self.x)

    def __call__(self, pixels):
        """pixels: images x size x size x 64.  Returns images x tokens x width."""
        self.tokens(pixels)
        return self.mlp().view(self.images, self.pixels, self.width)


def main():
    images, size = 4, 64
    block = FeatureMlpI8(images, size)
    pixels = torch.rand((images, size, size, 64), device="cuda").mul_(2).sub_(1).half()
    for name, run in (("the block", lambda: block(pixels)), ("its MLP", block.mlp), ("the MLP in fp16", block.mlp_in_fp16)):
        for _ in range(10):
            run()
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        for _ in range(100):
            run()
        end.record()
        end.synchronize()
        print(f"{images} x {size * size} tokens of {block.width} channels, {block.w['up'].shape[0]} hidden: {name} {start.elapsed_time(end) * 10:.1f} us")


if __name__ == "__main__":
    main()
