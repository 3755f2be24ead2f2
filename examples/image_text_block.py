"""Pixels that read a caption: the convolution layer's features as tokens that attend to the states of a text encoder.

    hb_conv3x3 (64 channels, NHWC)  ->  hb_linear (a 1x1 convolution to the width of the tokens)
    hb_linear -> queries, hb_rope_axes (row and column),  hb_linear -> keys and values of the caption
    hb_attention over the caption's states, of another length in each image
    hb_linear with bias and residual,  hb_linear with gelu,  hb_linear with bias and residual

Random weights; ``python examples/image_text_block.py`` runs it on the GPU and prints its time.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2512_02371_amd import hb


class ImageTextBlock:
    """`images` feature maps of size x size pixels and 64 channels, captions of up to `states` states of `text` channels."""

    def __init__(self, images, size, states, text=256, heads=8, channels=32, hidden=1024, seed=1, device="cuda"):
        self.images, self.tokens, self.states, self.heads, self.channels = images, size * size, states, heads, channels
        gen = torch.Generator(device=device).manual_seed(seed)
        width = heads * channels

        def matrix(n, k):
            return torch.randn((n, k), generator=gen, device=device).mul_(k ** -0.5).half()

        def vector(n):
            return torch.randn(n, generator=gen, device=device).mul_(0.1).half()

        self.conv = torch.randn((3, 3, 64, 64), generator=gen, device=device).div_(24.0).half()
        self.w = {"in": matrix(width, 64), "q": matrix(width, width), "kv": matrix(2 * width, text), "out": matrix(width, width),
                  "up": matrix(hidden, width), "down": matrix(width, hidden)}
        self.b = {name: vector(w.shape[0]) for name, w in self.w.items()}
        # a position per axis and token, a frequency per pair of channels: half of the pairs turn with the row, half with the column
        grid = torch.meshgrid(torch.arange(size), torch.arange(size), indexing="ij")
        self.positions = torch.stack(grid, dim=-1).reshape(1, self.tokens, 2).int().to(device).expand(images, -1, -1)
        pairs = channels // 4
        self.sections = [pairs, pairs]
        self.freq = (100.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).repeat(2).float().to(device)
        # buffers and scratch memory live as long as the weights: a pass allocates nothing
        M = images * self.tokens
        f16 = lambda *shape: torch.empty(shape, dtype=torch.float16, device=device)
        self.features, self.x, self.q, self.seen, self.hidden = f16(images, size, size, 64), f16(M, width), f16(M, width), f16(M, width), f16(M, hidden)
        self.kv = f16(images * states, 2 * width)
        need = [hb.hb_linear_workspace_size(images * states if n == "kv" else M, *w.shape) for n, w in self.w.items()]
        need.append(hb.hb_attention_workspace_size(images, self.tokens, states, heads, heads, channels))
        self.workspace = torch.empty(max(need), dtype=torch.uint8, device=device) if max(need) else None

    def _linear(self, x, name, out, residual=None, act="none"):
        return hb.hb_linear(x, self.w[name], out, self.workspace, self.b[name], residual, act)

    def __call__(self, pixels, caption, lengths):
        """pixels: images x size x size x 64, caption: images x states x text, lengths: images int32.  Returns images x tokens x width."""
        B, L, S, H, D = self.images, self.tokens, self.states, self.heads, self.channels
        hb.hb_conv3x3(pixels, self.conv, self.features)
        self._linear(self.features.view(B * L, 64), "in", self.x)
        q = self._linear(self.x, "q", self.q).view(B, L, H, D)
        hb.hb_rope_axes(q, q, self.positions, self.freq, self.sections)
        kv = self._linear(caption.reshape(B * S, -1), "kv", self.kv).view(B, S, 2, H, D)
        hb.hb_attention(q, kv[:, :, 0], kv[:, :, 1], self.seen.view(B, L, H, D), D ** -0.5, self.workspace, lengths)
        self._linear(self.seen, "out", self.x, residual=self.x)
        self._linear(self.x, "up", self.hidden, act="gelu")
        self._linear(self.hidden, "down", self.x, residual=self.x)
        return self.x.view(B, L, -1)


def main():
    images, size, states = 2, 64, 77
    block = ImageTextBlock(images, size, states)
    pixels = torch.rand((images, size, size, 64), device="cuda").mul_(2).sub_(1).half()
    caption = torch.randn((images, states, 256), device="cuda").half()
    lengths = torch.tensor([states, 12], dtype=torch.int32, device="cuda")
    for _ in range(10):
        out = block(pixels, caption, lengths)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(100):
        block(pixels, caption, lengths)
    end.record()
    end.synchronize()
    print(f"{images} x {size * size} tokens of {out.shape[2]} channels, {states} states: {start.elapsed_time(end) * 10:.1f} us a block")


if __name__ == "__main__":
    main()
