"""From an image to an answer: the kept visual tokens through a small language model.

    python examples/answer.py [--tokens 16] [--images 4]

Encoder outputs are reduced (Reducer.reduce), the kept tokens get their place in
the prompt and their (time, height, width) positions (kept_positions), and a stack
of attention layers with random weights reads them: the prompts of all images in
one step (Attention.append, Attention.attend), then token by token for all of them
together.  Last, one training step of a layer's head norms (Attention.rotate and
rotate_backward behind torch's autograd).  Weights and inputs are synthetic: the
answers mean nothing, the calls are those of a real model.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_13500_amd as tr
import synth

PAGE = 64


class Layer:
    """One attention layer: projections, head norms, and a paged cache of its own."""

    def __init__(self, attention, width, pages, g):
        a = self.attention = attention
        rows = (a.heads + 2 * a.kv_heads) * a.head_dim
        rand = lambda *s: torch.randn(*s, generator=g, device=a.device)
        self.qkv = (rand(rows, width) / math.sqrt(width)).to(a.dtype)
        self.out = (rand(width, a.heads * a.head_dim) / math.sqrt(a.heads * a.head_dim)).to(a.dtype)
        self.wq, self.wk = ((1 + 0.1 * rand(a.head_dim)).to(a.dtype) for _ in range(2))
        shape = (pages, PAGE, a.kv_heads, a.head_dim)
        self.cache = tr.KVCache(torch.zeros(shape, dtype=a.dtype, device=a.device), torch.zeros(shape, dtype=a.dtype, device=a.device))

    def split(self, x):
        """Queries, keys and values of [tokens, width] states, slices of one product."""
        a = self.attention
        return (x @ self.qkv.t()).view(x.shape[0], -1, a.head_dim).split([a.heads, a.kv_heads, a.kv_heads], 1)

    def attend(self, q, k, v, pos, step):
        q = self.attention.append(q, k, v, pos, self.cache, step, wq=self.wq, wk=self.wk)
        return self.attention.attend(q, self.cache, step)[0]

    def __call__(self, x, pos, step):
        y = self.attend(*self.split(x), pos, step)
        return x + y.flatten(1) @ self.out.t()


def unit(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


def prompts(kept, idx, K, grid, before, words):
    """Packed states and positions of one prompt an image: `before` words, its kept
    tokens, one more word.  Text counts on all three axes; an image takes
    max(grid) of them."""
    first = [sum(K[:b]) + b * (before + 1) for b in range(len(K))]              # of a prompt's rows
    total = sum(K) + len(K) * (before + 1)
    pos = torch.empty(3, total, dtype=torch.int32, device=kept.device)
    x = torch.empty(total, kept.shape[1], dtype=kept.dtype, device=kept.device)
    side, at = max(grid), 0
    for r, k in zip(first, K):
        pos[:, r:r + before] = torch.arange(before, device=kept.device)
        pos[:, r + before + k] = before + side
        x[r:r + before] = words[:before]
        x[r + before:r + before + k] = kept[at:at + k]
        x[r + before + k] = words[before]
        at += k
    tr.kept_positions(idx, K, [grid] * len(K), [(before,) * 3] * len(K), dst=[r + before for r in first], out=pos)
    return x, pos, [k + before + 1 for k in K]


def answer(layers, words, x, pos, lengths, tokens, room):
    """The prompts in one step, then `tokens` words of each: int64 [tokens, prompts]."""
    dev, seqs = x.device, len(lengths)
    pages = (room + PAGE - 1) // PAGE
    table = torch.arange(seqs * pages, dtype=torch.int32, device=dev).view(seqs, pages)
    kv_len = torch.tensor(lengths, dtype=torch.int32, device=dev)
    ends = kv_len.cumsum(0, dtype=torch.int32)
    step = tr.Step(torch.cat([ends.new_zeros(1), ends]), kv_len, table)
    last = ends.long() - 1
    at = pos[:, last].contiguous()
    said = []
    for i in range(tokens):
        for layer in layers:
            x = layer(x, pos, step)
        x = x[last] if i == 0 else x
        word = (unit(x) @ words.t()).float().argmax(1)
        said.append(word)
        kv_len, at = kv_len + 1, at + 1
        x, pos = words[word], at
        step = tr.Step(torch.arange(seqs + 1, dtype=torch.int32, device=dev), kv_len, table)
    return torch.stack(said)


def train_step(attention, q, k, pos, wq, wk, target, rate=0.1):
    """One step of the norms' weights towards scores [heads, tokens, tokens]; the loss before it."""
    wq, wk = (w.detach().requires_grad_(True) for w in (wq, wk))
    rq, rk = attention.rotate(q, k, pos, wq=wq, wk=wk)
    rk = rk.repeat_interleave(attention.heads // attention.kv_heads, 1)
    scores = torch.matmul(rq.float().transpose(0, 1), rk.float().permute(1, 2, 0)) / math.sqrt(attention.head_dim)
    loss = (scores - target).square().mean()
    loss.backward()
    with torch.no_grad():
        return float(loss), wq - rate * wq.grad, wk - rate * wk.grad


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--images", type=int, default=4)
    p.add_argument("--tokens", type=int, default=16)
    p.add_argument("--layers", type=int, default=2)
    a = p.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)
    w = synth.llava(device="cuda", B=a.images, N=576, D=4096, K=64)
    reducer = tr.Reducer(w.D, w.Dc, w.dtype, lam=w.lam, max_images=w.B, max_tokens=sum(w.N), max_N=576)
    kept = reducer.reduce(w.X, w.Xpre, w.Xpost, w.N, w.K)

    attention = tr.Attention(32, 8, 128, w.dtype, sections=(16, 24, 24), norm=True)
    words = torch.randn(1000, w.D, generator=g, device="cuda").to(w.dtype)
    x, pos, lengths = prompts(unit(kept.out), kept.idx, list(w.K), (1, 24, 24), 8, words)
    room = max(lengths) + a.tokens
    layers = [Layer(attention, w.D, a.images * ((room + PAGE - 1) // PAGE), g) for _ in range(a.layers)]
    said = answer(layers, words, x, pos, lengths, a.tokens, room)
    print("%d images of 576 tokens, %d kept of each, %d words said" % (a.images, w.K[0], said.numel()))

    q, k, _ = layers[0].split(x[:lengths[0]])
    target = torch.randn(32, lengths[0], lengths[0], generator=g, device="cuda")
    wq, wk, losses = layers[0].wq, layers[0].wk, []
    for _ in range(3):
        loss, wq, wk = train_step(attention, q, k, pos[:, :lengths[0]].contiguous(), wq, wk, target, rate=4.0)
        losses.append(loss)
    print("loss of the scores in training: " + ", ".join("%.4f" % v for v in losses))
    return said, losses


if __name__ == "__main__":
    main()
