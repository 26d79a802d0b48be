"""The attention half of a layer served from its low-bit weights: q, k and v from
the packed INT4 backbone with its sidecar, the new keys and values appended to
the paged 8-bit cache with the rotation on the way, attention over the cache,
and the output projection, packed again.

A prompt per user goes through in one step (BF16, dense products of the decoded
weights); decode steps (float32, packed products, up to 8 users) are one CUDA
graph that is replayed: lengths live on the device.

    python examples/attention_layer.py --users 4 --prompt 1000 --steps 64
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_23144_gb300 as aw  # noqa: E402


class AttentionLayer:
    """Low-bit q, k, v, o projections and the cache between them."""

    def __init__(self, heads: int, kv_heads: int, dim: int, users: int, max_len: int, page: int, gen: torch.Generator):
        hidden = heads * dim
        self.heads, self.kv_heads, self.dim, self.users = heads, kv_heads, dim, users
        rows = [hidden, kv_heads * dim, kv_heads * dim, hidden]  # q, k, v, o
        self.shapes = [(r, hidden) for r in rows]
        ws = [(torch.randn(r, hidden, generator=gen) * hidden ** -0.5).cuda() for r in rows]
        self.prm = aw.params(C=64, P=4, b=4, S=256)
        self.backbones = aw.awsrc_rtn_quantize_batch(ws, sdq=True)
        act = torch.ones(hidden, device="cuda")
        mods = [{"W": w, "W0": b["W0"], "act": act} for w, b in zip(ws, self.backbones)]
        cands = aw.awsrc_encode_tiles(self.prm, mods)
        stream, counts, _ = aw.awsrc_select_records(self.prm, mods, cands, [0.162])
        records = int(counts.sum())
        self.sidecar = aw.awsrc_sidecar_prepare(self.prm, self.shapes, stream, records)
        self.dense = aw.awsrc_decode_apply(self.prm, mods, stream, records)  # the same weights, for prompts

        per_user = -(-max_len // page)
        self.cache = aw.awsrc_kv_cache_alloc(users * per_user, kv_heads, dim, page)
        self.workspace = aw.awsrc_attention_workspace(self.cache, heads)
        self.table = torch.randperm(users * per_user, generator=gen).view(users, per_user).to(torch.int32).cuda()
        self.kv_len = torch.zeros(users, dtype=torch.int32, device="cuda")
        self.max_len = max_len
        freq = 10000.0 ** (-torch.arange(dim // 2) * 2.0 / dim)
        angle = torch.arange(max_len)[:, None] * freq[None]
        self.cos, self.sin = angle.cos().cuda(), angle.sin().cuda()

    def batch(self, new: list) -> "aw.KvBatch":
        """The step in which user i brings new[i] tokens; kv_len holds the lengths with them when it runs."""
        start = torch.tensor([0] + new, dtype=torch.int32).cumsum(0, dtype=torch.int32).cuda()
        return aw.awsrc_kv_batch(start, self.kv_len, self.table, sum(new), max(new), self.max_len)

    def attend(self, batch, q, k, v):
        n = q.shape[0]
        q, k, v = (t.view(n, -1, self.dim) for t in (q, k, v))
        q = aw.awsrc_kv_append(self.cache, batch, q, k, v, self.cos, self.sin, self.workspace, q_out=q)
        return aw.awsrc_paged_attention(self.cache, batch, q, self.workspace).view(n, -1)

    def prompt(self, x: torch.Tensor, lengths: list) -> torch.Tensor:
        """x: the users' prompts one after the other, BF16."""
        w = [d.to(torch.bfloat16) for d in self.dense]
        self.kv_len += torch.tensor(lengths, dtype=torch.int32, device="cuda")
        out = self.attend(self.batch(lengths), *(x @ m.T for m in w[:3]))
        return out @ w[3].T

    def step(self, batch, x: torch.Tensor) -> torch.Tensor:
        """One token of every user, float32."""
        self.kv_len += 1
        q, k, v = aw.awsrc_packed_gemv_batch(self.prm, self.shapes, [(m, self.backbones[m], x) for m in range(3)],
                                             sidecar=self.sidecar)
        out = self.attend(batch, q, k, v)
        return aw.awsrc_packed_gemv(self.prm, self.shapes, 3, self.backbones[3], out, sidecar=self.sidecar)


def plain(layer: AttentionLayer, xs: list) -> list:
    """The layer's outputs for the users' whole sequences, float64, nothing held in 8 bits."""
    wq, wk, wv, wo = (d.double() for d in layer.dense)
    group, half = layer.heads // layer.kv_heads, layer.dim // 2
    outs = []
    for x in xs:
        n = x.shape[0]
        cos, sin = layer.cos[:n, None].double(), layer.sin[:n, None].double()

        def turned(y):
            a, b = y[..., :half], y[..., half:]
            return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

        x = x.double()
        q = turned((x @ wq.T).view(n, -1, layer.dim)).transpose(0, 1)
        k = turned((x @ wk.T).view(n, -1, layer.dim)).transpose(0, 1).repeat_interleave(group, 0)
        v = (x @ wv.T).view(n, -1, layer.dim).transpose(0, 1).repeat_interleave(group, 0)
        s = q @ k.transpose(1, 2) * layer.dim ** -0.5
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
        outs.append((s.softmax(-1) @ v).transpose(0, 1).reshape(n, -1) @ wo.T)
    return outs


def run(heads=16, kv_heads=2, dim=128, users=4, prompt=1000, steps=64, page=64, seed=0) -> dict:
    """Prompts of prompt, prompt - 1, .. tokens, then `steps` decode steps; relative errors against plain()."""
    gen = torch.Generator().manual_seed(seed)
    lengths = [max(1, prompt - i) for i in range(users)]
    layer = AttentionLayer(heads, kv_heads, dim, users, prompt + steps + 1, page, gen)
    hidden = heads * dim
    xs = [torch.randn(n + steps, hidden, generator=gen).to(torch.bfloat16).cuda() for n in lengths]

    first = layer.prompt(torch.cat([x[:n] for x, n in zip(xs, lengths)]), lengths)

    batch = layer.batch([1] * users)
    x = torch.zeros(users, hidden, device="cuda")
    layer.step(batch, x)  # warm-up before the capture; its token is written over by the first real step
    layer.kv_len -= 1
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.step(batch, x)
    ys = []
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for i in range(steps):
        x.copy_(torch.stack([s[n + i] for s, n in zip(xs, lengths)]))
        graph.replay()
        ys.append(y.clone())
    end.record()
    torch.cuda.synchronize()
    if aw.awsrc_workspace_status(layer.workspace):
        raise RuntimeError("the batch held an entry that cannot be right")

    want = plain(layer, xs)
    got = [torch.cat([f, torch.stack([s[i] for s in ys])]) for i, f in enumerate(first.float().split(lengths))]

    def error(a, b):
        return float((a.double() - b).norm() / b.norm())

    return {"prompt_error": max(error(g[:n], w[:n]) for g, w, n in zip(got, want, lengths)),
            "step_error": max(error(g[n:], w[n:]) for g, w, n in zip(got, want, lengths)),
            "us_per_step": 1e3 * begin.elapsed_time(end) / steps}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, default in (("heads", 16), ("kv-heads", 2), ("dim", 128), ("users", 4), ("prompt", 1000), ("steps", 64),
                          ("page", 64), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    for name, value in run(**vars(ap.parse_args())).items():
        print(f"{name} {value:.4g}")
