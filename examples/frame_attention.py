"""Attention of a video stream's frames over the frames before, on the outputs of streaming Skip-Conv layers.

Each frame goes through three 1 x 1 Skip-Conv layers (queries, keys, values), which recompute only the blocks that moved. Their
activation outputs are the tokens: one append writes the frame's keys and values into the paged cache, rotated by (frame, row, column), and
rotates the queries; one attention call lets every site of the frame attend to its own frame and the ``history`` frames before it.

    python examples/frame_attention.py --streams 2 --height 64 --width 64 --frames 12
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2104_11487_amd import synthetic as syn  # noqa: E402
from paper_2104_11487_amd.skipconv import SkipConv  # noqa: E402
from paper_2104_11487_amd.stream_attention import CacheBatch, PagedCache, Rotary, axis_frequencies  # noqa: E402


class FrameAttention:
    """weights: the projections' OIHW bf16 GPU tensors (c_out, c_in, 1, 1) for queries, keys and values, c_out = heads * head_dim."""

    def __init__(self, weights, *, n, h, w, head_dim, history, eps, block=8, page_size=64):
        self.n, self.h, self.w, self.head_dim, self.history = n, h, w, head_dim, history
        self.layers = [SkipConv(wt, n=n, h=h, w=w, eps=eps, block=block, act_out="identity") for wt in weights]
        self.tokens = h * w
        self.ring = history + 1
        if self.tokens % page_size:  # a frame takes whole pages: one, where the page size does not divide it
            page_size = self.tokens
        per_frame = self.tokens // page_size
        device = weights[0].device
        self.cache = PagedCache.empty(n * self.ring * per_frame, page_size, weights[1].shape[0] // head_dim, head_dim, device=device)
        self.table = torch.arange(n * self.ring * per_frame, dtype=torch.int32, device=device).view(n, self.ring, per_frame)
        starts = torch.arange(n + 1, dtype=torch.int32, device=device) * self.tokens
        self.batch = CacheBatch(self.table.view(n, -1), starts, torch.zeros(n, dtype=torch.int32, device=device), max_new=self.tokens)
        pairs = head_dim // 2
        self.rotary = Rotary(axis_frequencies((pairs - 2 * (pairs // 3), pairs // 3, pairs // 3), device=device), head_dim)
        y, x = torch.meshgrid(torch.arange(h), torch.arange(w), indexing="ij")
        frame = torch.stack([torch.zeros_like(y), y, x], -1).view(1, -1, 3).expand(n, -1, -1)
        self.pos = frame.reshape(-1, 3).to(torch.int32).to(device)
        self.t = 0

    def step(self, frame):
        """One frame, N x H x W x C_in bf16; returns N x H x W x (heads * head_dim)."""
        q, k, v = (self._tokens(layer, frame) for layer in self.layers)
        if self.t >= self.ring:  # the oldest frame's pages take the new one
            self.table.copy_(self.table.roll(-1, 1))
        self.batch.kv_len.fill_(min(self.t + 1, self.ring) * self.tokens)
        self.pos[:, 0] = self.t
        self.t += 1
        q = self.cache.append(k, v, self.batch, rotary=self.rotary, pos=self.pos, q=q)
        return self.cache.attend(q, self.batch, causal=False).view(self.n, self.h, self.w, -1)

    def _tokens(self, layer, frame):
        layer.step(frame)
        return layer.activation().view(self.n * self.tokens, -1, self.head_dim)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--streams", type=int, default=2)
    ap.add_argument("--height", type=int, default=64)
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--channels", type=int, default=64)
    ap.add_argument("--heads", type=int, default=4)
    ap.add_argument("--kv-heads", type=int, default=2)
    ap.add_argument("--head-dim", type=int, default=64)
    ap.add_argument("--history", type=int, default=3)
    ap.add_argument("--frames", type=int, default=12)
    a = ap.parse_args()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    weights = [(torch.randn(h * a.head_dim, a.channels, 1, 1, device="cuda", generator=g) * (2.0 / a.channels) ** 0.5).bfloat16()
               for h in (a.heads, a.kv_heads, a.kv_heads)]
    model = FrameAttention(weights, n=a.streams, h=a.height, w=a.width, head_dim=a.head_dim, history=a.history, eps=0.3)
    video = syn.RectVideo(a.height, a.width, a.channels, a.frames, seed=2, batch=a.streams, side_lo=8, side_hi=16)
    frames = [torch.from_numpy(f).cuda().bfloat16().contiguous() for f in video]
    for t, frame in enumerate(frames):
        torch.cuda.synchronize()
        begin = time.perf_counter()
        out = model.step(frame)
        torch.cuda.synchronize()
        print(f"frame {t}: {model.layers[0].active_count()[0]} active blocks, {(time.perf_counter() - begin) * 1e3:.3f} ms, "
              f"|out| {out.float().abs().mean().item():.4f}", flush=True)


if __name__ == "__main__":
    main()
