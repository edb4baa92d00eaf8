"""A decoding step of one pruned transformer layer on the library's operators.

The layer's seven weights are pruned N:M on the GPU (nmspmm_compress_device),
laid out once in bf16 (nmspmm_half_pack) and used for every step:

    x   -> norm -> q, k, v         one sparse product
        -> nmspmm_kv_append        rotary positions, new keys and values into the pages
        -> nmspmm_kv_attend        each sequence's new token over its pages
        -> output product          added to x in the epilogue
        -> norm -> up; silu(gate) * up in the gate product's epilogue
        -> down product            added to x in the epilogue

    python examples/decode_layer.py [--batch 8] [--steps 4] [--check]

--check compares every step with the same layer in fp64 (its keys and values
rounded to bf16 as the cache holds them).
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2503_01253_amd as nm  # noqa: E402


class Layer:
    """Weights, pages and workspaces of one layer for a batch of sequences."""

    def __init__(self, batch, hidden=512, heads=8, kv_heads=2, dim=64, inner=1408, positions=256, page=16,
                 pattern=(8, 32, 32), seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.pattern = heads, kv_heads, dim, pattern
        self.dense = {}     # the pruned weights as matrices, for the check

        def weight(name, k, n):
            N, M, V = pattern
            B = torch.randn(k, n, generator=gen, device=device) / math.sqrt(k * N / M)
            Bc = torch.empty(k // M * N, n, device=device)
            idx = torch.empty(k // M * N, n // V, dtype=torch.uint8, device=device)
            nm.nmspmm_compress_device(B, Bc, idx, N, M, V)
            at = torch.arange(Bc.shape[0], device=device)[:, None] // N * M + idx.long().repeat_interleave(V, dim=1)
            self.dense[name] = torch.zeros_like(B).scatter_(0, at, Bc).bfloat16()
            return nm.nmspmm_half_pack(Bc, idx, n, k, N, M, V)

        self.qkv = weight("qkv", hidden, (heads + 2 * kv_heads) * dim)
        self.out = weight("out", heads * dim, hidden)
        self.up, self.gate = weight("up", hidden, inner), weight("gate", hidden, inner)
        self.down = weight("down", inner, hidden)
        # every sequence's pages, scattered over the cache
        per = (positions + page - 1) // page
        pages = torch.randperm(batch * per, generator=gen, device=device).int().view(batch, per)
        shape = (batch * per, page, kv_heads, dim)
        self.cache = nm.nmspmm_kv_cache(*(torch.empty(shape, dtype=torch.bfloat16, device=device) for _ in range(2)),
                                        pages)
        angle = torch.arange(positions, device=device)[:, None] * 10000.0 ** (
            -torch.arange(dim // 2, device=device) / (dim // 2))
        self.cos, self.sin = angle.cos(), angle.sin()
        self.seq = torch.arange(batch, dtype=torch.int32, device=device)
        self.positions = positions
        size = max([nm.nmspmm_half_workspace_bytes(batch, w) for w in
                    (self.qkv, self.out, self.up, self.gate, self.down)]
                   + [nm.nmspmm_kv_attend_workspace_bytes(self.cache, heads, positions)])
        self.workspace = torch.empty(size, dtype=torch.uint8, device=device) if size else None

    def norm(self, x):
        x = x.float()
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).bfloat16()

    def step(self, x, pos):
        """One new token of every sequence: x (batch, hidden) bf16, at
        positions pos (int32); returns the layer's output."""
        batch, hidden = x.shape
        new = dict(dtype=torch.bfloat16, device=x.device)
        qkv = torch.empty(batch, self.qkv.n, **new)
        nm.nmspmm_half_run(self.norm(x), self.qkv, qkv, workspace=self.workspace)
        rows = qkv.view(batch, -1, self.dim)
        q, k, v = rows.split((self.heads, self.kv_heads, self.kv_heads), dim=1)
        nm.nmspmm_kv_append(self.cache, k, v, self.seq, pos, cos=self.cos, sin=self.sin, q=q)
        mixed = torch.empty(batch, self.heads, self.dim, **new)
        nm.nmspmm_kv_attend(self.cache, q, pos + 1, mixed, max_length=self.positions, workspace=self.workspace)
        y = torch.empty(batch, hidden, **new)
        nm.nmspmm_half_run(mixed.view(batch, -1), self.out, y, residual=x, workspace=self.workspace)
        z = self.norm(y)
        up = torch.empty(batch, self.up.n, **new)
        nm.nmspmm_half_run(z, self.up, up, workspace=self.workspace)
        nm.nmspmm_half_run(z, self.gate, up, act="silu", mul=up, workspace=self.workspace)    # in place
        nm.nmspmm_half_run(up, self.down, y, residual=y, workspace=self.workspace)            # in place
        return y


class Plain:
    """The same layer in fp64 on dense matrices, keys and values kept in lists."""

    def __init__(self, layer):
        self.l, self.keys, self.values = layer, None, None

    def norm(self, x):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    def turn(self, x, pos):
        c, s = self.l.cos[pos.long()].double()[:, None], self.l.sin[pos.long()].double()[:, None]
        a, b = x.chunk(2, dim=-1)
        return torch.cat((a * c - b * s, a * s + b * c), dim=-1)

    def step(self, x, pos):
        l, W = self.l, {name: w.double() for name, w in self.l.dense.items()}
        batch, x = x.shape[0], x.double()
        rows = (self.norm(x) @ W["qkv"]).view(batch, -1, l.dim)
        q, k, v = rows.split((l.heads, l.kv_heads, l.kv_heads), dim=1)
        q, k, v = self.turn(q, pos), self.turn(k, pos).bfloat16().double(), v.bfloat16().double()
        self.keys = k[:, None] if self.keys is None else torch.cat((self.keys, k[:, None]), dim=1)
        self.values = v[:, None] if self.values is None else torch.cat((self.values, v[:, None]), dim=1)
        group = l.heads // l.kv_heads
        K, V = (t.repeat_interleave(group, dim=2).permute(0, 2, 1, 3).contiguous() for t in (self.keys, self.values))
        p = torch.softmax((K @ q[..., None]).squeeze(-1) * l.dim ** -0.5, dim=-1)
        y = x + (p[:, :, None] @ V).reshape(batch, -1) @ W["out"]
        z = self.norm(y)
        gate = z @ W["gate"]
        return y + (gate * torch.sigmoid(gate) * (z @ W["up"])) @ W["down"]


def main(argv=None):
    """Runs the steps; returns the largest relative error against fp64 (0 without --check)."""
    arg = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    arg.add_argument("--batch", type=int, default=8)
    arg.add_argument("--steps", type=int, default=4)
    arg.add_argument("--check", action="store_true")
    a = arg.parse_args(argv)
    layer = Layer(a.batch)
    plain, worst = Plain(layer), 0.0
    gen = torch.Generator(device="cuda").manual_seed(1)
    for s in range(a.steps):
        x = torch.randn(a.batch, layer.qkv.k, generator=gen, device="cuda").bfloat16()
        pos = torch.full((a.batch,), s, dtype=torch.int32, device="cuda")
        y = layer.step(x, pos)
        if a.check:
            want = plain.step(x, pos)
            error = ((y.double() - want).norm() / want.norm()).item()
            worst = max(worst, error)
            print(f"step {s}: relative error against fp64 {error:.2e}", flush=True)
    torch.cuda.synchronize()
    print(f"{a.steps} steps of {a.batch} sequences; kernels: qkv "
          f"{nm.nmspmm_half_kernel_name(a.batch, layer.qkv)}, down {nm.nmspmm_half_kernel_name(a.batch, layer.down)}")
    return worst


if __name__ == "__main__":
    main()
