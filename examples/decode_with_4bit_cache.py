"""Decoding with packed weights and a 4-bit key-value cache: prompts of different lengths, then tokens one by one, through a few decoder layers.

    python examples/decode_with_4bit_cache.py [--layers 2] [--tokens 32]

Every linear is a packed layer (eqat_qlinear_fwd), q, k and v stacked in one; queries, keys and values are slices of its output, and one call turns queries and keys by their
positions and writes keys and values into the cache (eqat_kv_rotary_write), attention reads the cache (eqat_kv_attention).  The residual's addition and the norm behind it are one
call (eqat_norm_fwd), and so are the feed-forward's two projections with their gate (eqat_gated_fwd).  The decoding step is captured in a graph once and replayed: lengths, page table and tokens live on
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


EPS = 1e-5


class Layer:
    def __init__(self, gen, args, pages):
        h, d = args.hidden, args.head_dim
        self.heads, self.kv, self.d = h // d, args.kv_heads, d
        self.qkv = Linear(gen, (self.heads + 2 * self.kv) * d, h, args.bits, args.group)
        self.o = Linear(gen, h, h, args.bits, args.group)
        self.up, self.down = Linear(gen, 2 * args.inter, h, args.bits, args.group), Linear(gen, h, args.inter, args.bits, args.group)
        self.cache = eq.KvCache(self.kv, d, args.kv_group, args.page, pages)
        self.rot = eq.Rotary(eq.rotary_frequencies(d, stretch=args.stretch).cuda(), d)
        self.w1, self.w2 = (torch.empty(h, device="cuda").normal_(1.0, 0.1, generator=gen) for _ in range(2))

    def __call__(self, x, residual, batch, ws):
        """x, what the last layer's feed-forward left, and the residual that it goes on top of -> the same for the next layer"""
        T, heads, kv = x.shape[0], self.heads, self.kv
        n = eq.eqat_norm_fwd(x, self.w1, EPS, R=residual, want=("S", "Y"))
        y = self.qkv(n["Y"]).view(T, heads + 2 * kv, self.d)
        self.q = eq.eqat_kv_rotary_write(self.cache, batch, self.rot, y[:, :heads], y[:, heads:heads + kv], y[:, heads + kv:])
        self.a = eq.eqat_kv_attention(self.cache, batch, self.q, ws=ws)
        n = eq.eqat_norm_fwd(self.o(self.a.view(T, heads * self.d)), self.w2, EPS, R=n["S"], want=("S", "Y"))
        return self.down(eq.eqat_gated_fwd(n["Y"], self.up.Wq, self.up.s, self.up.zq, self.up.bits, self.up.group)), n["S"]


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
    ws = eq.kv_workspace(layers[0].cache, first, layers[0].heads)
    w = torch.empty(args.hidden, device="cuda").normal_(1.0, 0.1, generator=gen)

    def through(tokens, batch, rows=None):
        x, residual = embed[tokens], None
        for layer in layers:
            x, residual = layer(x, residual, batch, ws)
        if rows is not None:
            x, residual = x[rows], residual[rows]
        return head(eq.eqat_norm_fwd(x, w, EPS, R=residual, want=("Y",))["Y"]).argmax(-1)

    tokens = through(torch.randint(0, args.vocab, (starts[-1],), device="cuda", generator=gen), first, [s - 1 for s in starts[1:]])

    # one token a sequence from here on
    lens = i32(args.prompts)
    batch = eq.KvBatch(table, lens, i32(list(range(B + 1))), tokens=B, max_new=1, max_len=width * args.page)
    out = torch.zeros((n_new, B), dtype=torch.long, device="cuda")

    def step():
        lens.add_(1)
        tokens.copy_(through(tokens, batch))

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
    p.add_argument("--stretch", type=float, default=1.0, help="rotary positions for contexts that many times longer")
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
