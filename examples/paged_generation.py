"""Sampling several continuations of several prompts with packed and paged keys and values.

A random model of the size of the repository's tiny workload: prompts of different lengths are appended (keys
and queries turned, keys and values paged), each is forked into a second sequence, and all sequences
generate tokens, one a step; as they grow, tokens that have left the full-precision window are transform-coded.
At the end one step's attention is compared with attention over all tokens in full precision.

    python examples/paged_generation.py [steps]
"""
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_14191_gb300 as aatc  # noqa: E402
from paper_2608_14191_gb300 import paged  # noqa: E402
from paper_2608_14191_gb300.paged_cache import PagedTailCache  # noqa: E402

D, N_KV, N_Q, LAYERS, D_MODEL, VOCAB = 128, 2, 8, 2, 512, 1000
PROMPTS = [150, 61, 333]


class Model:
    """Attention layers with residuals, and a vocabulary; everything random."""

    def __init__(self, seed=0):
        g = torch.Generator("cuda")
        g.manual_seed(seed)
        w = lambda *shape: (torch.randn(shape, generator=g, device="cuda") / math.sqrt(shape[-2])).to(torch.bfloat16)  # noqa: E731
        self.embed = torch.randn((VOCAB, D_MODEL), generator=g, device="cuda").to(torch.bfloat16)
        self.wqkv = [w(D_MODEL, (N_Q + 2 * N_KV) * D) for _ in range(LAYERS)]
        self.wo = [w(N_Q * D, D_MODEL) for _ in range(LAYERS)]
        self.unembed = w(D_MODEL, VOCAB)

    def qkv(self, layer, x):
        y = (x / x.float().square().mean(-1, keepdim=True).sqrt().to(x.dtype)) @ self.wqkv[layer]
        y = y.view(len(x), N_Q + 2 * N_KV, D)
        return y[:, :N_Q], y[:, N_Q:N_Q + N_KV], y[:, N_Q + N_KV:]


def prompt_attention(q, k, v, lens):
    """Causal attention within each prompt (the prompts' own pass; turned q and k)."""
    out, at = torch.empty(q.shape, device="cuda"), 0
    for n in lens:
        part = slice(at, at + n)
        kk, vv = (x[part].float().repeat_interleave(N_Q // N_KV, 1) for x in (k, v))
        s = torch.einsum("ihd,jhd->hij", q[part].float(), kk) / math.sqrt(D)
        s.masked_fill_(torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1), -math.inf)
        out[part] = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), vv)
        at += n
    return out


def plan_for(model, rope, bits=4.0):
    """A plan calibrated on the model's own turned keys, values and queries of random tokens."""
    x = model.embed[torch.randint(VOCAB, (1024,), device="cuda")]
    pos = torch.arange(1024, dtype=torch.int32, device="cuda")
    k, v, q = [], [], []
    for layer in range(LAYERS):
        ql, kl, vl = model.qkv(layer, x)
        ql, kl = paged.rotate(rope, ql, pos), paged.rotate(rope, kl, pos)
        for to, y in ((q, ql), (k, kl), (v, vl)):
            to.append(y.float().transpose(0, 1).cpu().numpy())
    dims = aatc.dims(LAYERS, N_KV, N_Q)
    p = aatc.calibrate(dims, np.stack(k), np.stack(v), np.stack(q), bits)
    return aatc.Plan(dims, p["basis"], p["bits"], p["scales"])


def generate(steps=100, seed=0):
    """Runs the loop; returns what it ended with."""
    torch.manual_seed(seed)
    model = Model(seed)
    rope = paged.Rotary(D, 10000.0, scaling=dict(kind="banded", factor=8.0, original=8192, low=1.0, high=4.0))
    plan = plan_for(model, rope)
    batch = 2 * len(PROMPTS)
    cache = PagedTailCache(plan, batch, 1024, window=64, step=16, tail_tokens=640, rope=rope)
    kept = [[] for _ in range(LAYERS)]                   # full precision, for the comparison alone

    # the prompts, in the even rows; the odd rows are forks of them
    lens = [n for p in PROMPTS for n in (p, 0)]
    x = model.embed[torch.randint(VOCAB, (sum(lens),), device="cuda")]
    cache.begin(lens)
    position = torch.cat([torch.arange(n, dtype=torch.int32, device="cuda") for n in lens])
    for layer in range(LAYERS):
        q, k, v = model.qkv(layer, x)
        q = cache.append(layer, k, v, q)
        k = paged.rotate(rope, k, position)
        at = 0
        for n in lens:
            kept[layer].append((k[at:at + n], v[at:at + n]))
            at += n
        x = x + (prompt_attention(q, k, v, lens).to(torch.bfloat16).reshape(len(x), -1) @ model.wo[layer])
    last = np.cumsum(lens) - 1
    shared = cache.seqs.free_pages
    for i in range(len(PROMPTS)):
        cache.fork(2 * i, 2 * i + 1)
        for layer in range(LAYERS):
            kept[layer][2 * i + 1] = kept[layer][2 * i]
    assert cache.seqs.free_pages == shared               # forks take no pages
    cache.end()
    h = x[torch.from_numpy(np.repeat(last[::2], 2)).to("cuda")]

    for step in range(steps):
        token = torch.multinomial(torch.softmax((h @ model.unembed).float(), -1), 1)[:, 0]
        x = model.embed[token]
        position = torch.tensor([cache.length(r) for r in range(batch)], dtype=torch.int32, device="cuda")
        cache.begin([1] * batch)
        worst = 0.0
        for layer in range(LAYERS):
            q, k, v = model.qkv(layer, x)
            q = cache.append(layer, k, v, q)
            out = cache.attend(layer, q)
            turned = paged.rotate(rope, k, position)
            for r in range(batch):
                kept[layer][r] = tuple(torch.cat([old, new[r:r + 1]]) for old, new in zip(kept[layer][r], (turned, v)))
            if step == steps - 1:
                for r in range(batch):
                    kk, vv = (y.double().repeat_interleave(N_Q // N_KV, 1) for y in kept[layer][r])
                    p = torch.softmax(torch.einsum("hd,nhd->hn", q[r].double(), kk) / math.sqrt(D), -1)
                    ref = torch.einsum("hn,nhd->hd", p, vv)
                    worst = max(worst, float((out[r] - ref).norm() / ref.norm()))
            x = x + out.to(torch.bfloat16).reshape(batch, -1) @ model.wo[layer]
        h = x
        cache.end()
    torch.cuda.synchronize()
    assert cache.pages.device_error() == 0 and plan.device_error() == 0
    return dict(cache=cache, worst=worst, lengths=[cache.length(r) for r in range(batch)])


if __name__ == "__main__":
    got = generate(int(sys.argv[1]) if len(sys.argv) > 1 else 100)
    c = got["cache"]
    print(f"lengths {got['lengths']}, {c.coded} tokens of each packed, {c.seqs.free_pages} of {c.pages.n_pages} pages free")
    print(f"last step against full precision: relative error {got['worst']:.3f}")
