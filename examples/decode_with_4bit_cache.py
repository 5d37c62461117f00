"""Decoding with packed weights and a 4-bit key-value cache: prompts of different lengths, then tokens one by one, through a few decoder layers.

    python examples/decode_with_4bit_cache.py [--layers 2] [--tokens 32]

Every linear is a packed layer (eqat_qlinear_fwd), q, k and v stacked in one; keys and values are slices of its output and go into the cache as they lie
(eqat_kv_write), attention reads the cache (eqat_kv_attention).  The decoding step is captured in a graph once and replayed: lengths, page table and tokens live on
the device.  Weights are random; --check compares the last step's attention with one over the values that the cache stands for (eqat_kv_read).
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2407_11062_amd as eq  # noqa: E402


class Linear:
    def __init__(self, gen, out_features, in_features, bits, group):
        W = torch.empty((out_features, in_features), device="cuda").normal_(0.0, 0.02, generator=gen).bfloat16()
        self.s, z = eq.eqat_init_minmax(W, bits, group)
        self.Wq, self.zq = eq.eqat_pack(W, self.s, z, bits, group)
        self.bits, self.group = bits, group

    def __call__(self, x):
        return eq.eqat_qlinear_fwd(x, self.Wq, self.s, self.zq, self.bits, self.group)


def rotated(x, pos):
    """rotary embedding: pairs (i, i + dim / 2) of every head turned by pos / 10000^(2 i / dim)"""
    half = x.shape[-1] // 2
    angle = pos[:, None, None].float() * torch.exp(torch.arange(half, device=x.device) * (-2 * math.log(10000.0) / x.shape[-1]))
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1).to(x.dtype)


def normed(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-5)).to(x.dtype)


class Layer:
    def __init__(self, gen, args, pages):
        h, d = args.hidden, args.head_dim
        self.heads, self.kv, self.d = h // d, args.kv_heads, d
        self.qkv = Linear(gen, (self.heads + 2 * self.kv) * d, h, args.bits, args.group)
        self.o = Linear(gen, h, h, args.bits, args.group)
        self.up, self.down = Linear(gen, 2 * args.inter, h, args.bits, args.group), Linear(gen, h, args.inter, args.bits, args.group)
        self.cache = eq.KvCache(self.kv, d, args.kv_group, args.page, pages)

    def __call__(self, x, batch, pos, ws):
        T, q_rows, kv_rows = x.shape[0], self.heads * self.d, self.kv * self.d
        y = self.qkv(normed(x))
        q = rotated(y[:, :q_rows].view(T, self.heads, self.d), pos)
        k = rotated(y[:, q_rows:q_rows + kv_rows].view(T, self.kv, self.d), pos)
        eq.eqat_kv_write(self.cache, batch, k, y[:, q_rows + kv_rows:].view(T, self.kv, self.d))
        self.q, self.a = q, eq.eqat_kv_attention(self.cache, batch, q, ws=ws)
        x = x + self.o(self.a.view(T, q_rows))
        gate, up = self.up(normed(x)).chunk(2, -1)
        return x + self.down((torch.nn.functional.silu(gate) * up).contiguous())


def run(args):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    B, n_new = len(args.prompts), args.tokens
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    width = -(-(max(args.prompts) + n_new) // args.page)
    table = torch.randperm(B * width, generator=torch.Generator().manual_seed(2)).int().view(B, width).cuda()           # pages in no order
    layers = [Layer(gen, args, B * width) for _ in range(args.layers)]
    embed = torch.empty((args.vocab, args.hidden), device="cuda").normal_(generator=gen).bfloat16()
    head = Linear(gen, args.vocab, args.hidden, args.bits, args.group)

    # the prompts, all sequences in one call
    starts = [sum(args.prompts[:b]) for b in range(B + 1)]
    first = eq.KvBatch(table, i32(args.prompts), i32(starts), tokens=starts[-1], max_new=max(args.prompts), max_len=max(args.prompts))
    pos = torch.cat([torch.arange(n) for n in args.prompts]).int().cuda()
    ws = eq.kv_workspace(layers[0].cache, first, layers[0].heads)
    x = embed[torch.randint(0, args.vocab, (starts[-1],), device="cuda", generator=gen)]
    for layer in layers:
        x = layer(x, first, pos, ws)
    tokens = head(normed(x)[[s - 1 for s in starts[1:]]].contiguous()).argmax(-1)

    # one token a sequence from here on
    lens = i32(args.prompts)
    batch = eq.KvBatch(table, lens, i32(list(range(B + 1))), tokens=B, max_new=1, max_len=width * args.page)
    out = torch.zeros((n_new, B), dtype=torch.long, device="cuda")

    def step():
        lens.add_(1)
        x = embed[tokens]
        for layer in layers:
            x = layer(x, batch, lens - 1, ws)
        tokens.copy_(head(normed(x)).argmax(-1))

    step()                                               # outside the capture once: first uses
    out[0] = tokens
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    t0 = time.perf_counter()
    for i in range(1, n_new):
        graph.replay()
        out[i] = tokens
    torch.cuda.synchronize()
    dt = time.perf_counter() - t0
    held = sum(layer.cache.pool.numel() for layer in layers)
    print(f"{B} sequences, {n_new - 1} steps: {dt / max(1, n_new - 1) * 1e6:.0f} us a step; cache of {held / 2**20:.1f} MiB "
          f"(bf16: {held / 2**20 * 2 * args.head_dim * 2 / (args.head_dim + 8 * args.head_dim / args.kv_group):.1f})")
    return layers, batch, table, lens, out


def check(args, layers, table, lens):
    """largest relative error (2-norm of a head) of the last step's attention against attention over the cache's values, in 64 bits"""
    now = lens.tolist()
    starts = [sum(now[:b]) for b in range(len(now) + 1)]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    whole = eq.KvBatch(table, lens, i32(starts), tokens=starts[-1], max_new=max(now), max_len=max(now))
    worst = 0.0
    for layer in layers:
        k, v = eq.eqat_kv_read(layer.cache, whole)
        R = layer.heads // layer.kv
        for b in range(len(now)):
            K, V = (t[starts[b]:starts[b + 1]].double().repeat_interleave(R, 1).transpose(0, 1) for t in (k, v))      # [heads, len, dim]
            p = torch.softmax((K @ layer.q[b].double()[:, :, None])[..., 0] / math.sqrt(layer.d), -1)
            ref = (p[:, None] @ V)[:, 0]
            worst = max(worst, float(((layer.a[b].double() - ref).norm(dim=-1) / ref.norm(dim=-1)).max()))
    return worst


def parser():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in dict(layers=2, hidden=4096, inter=11008, head_dim=128, kv_heads=8, vocab=32000, bits=2, group=64, kv_group=64, page=64, tokens=32).items():
        p.add_argument("--" + name.replace("_", "-"), type=int, default=value)
    p.add_argument("--prompts", type=int, nargs="+", default=[333, 1000, 17, 515])
    p.add_argument("--check", action="store_true")
    return p


def main(argv=None):
    args = parser().parse_args(argv)
    layers, batch, table, lens, out = run(args)
    if args.check:
        print(f"attention of the last step: {check(args, layers, table, lens):.1e} from 64 bits over the cache's values")
    return out


if __name__ == "__main__":
    main()
