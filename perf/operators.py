"""What is timed of the paged cache: the operators of a serving loop that keeps new tokens uncompressed in pages.

A case names one operator and its sizes:
  rotate   rotary positions of a tensor of heads, or the gradient of that
  append   new tokens of a batch: queries and keys rotated, keys and values written to their pages
  decode   attention of one new token per sequence over its pages
  copy     copies of pages over every layer: a fork's last pages, the moves of a compaction
  gather   a range of every sequence out of its pages, contiguous, as the encode takes it

Head counts, contexts and batches are those of the workloads of this repository (a
Llama-3.1-8B-shaped layer with 8 kv-heads and 32 query heads, a Qwen-2.5-7B-shaped one with 4 and
28) and odd ones around them; lengths are ragged, from none to long ones.  `own` chooses what
`run` computes with: elementary torch operations in 32 bits (False), or the framework's calls.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # the queries of a long prompt, one layer
        dict(name="rotate_prompt", op="rotate", seqs=1, most=32768, ragged=False, before=0, heads=32, rot=128,
             layout="half", scaling="none", dtype="bf16", backward=False),
        # training step on a batch of ragged sequences, half of each head turned, pairs side by side
        dict(name="rotate_gradient", op="rotate", seqs=5, most=1501, ragged=True, before=0, heads=28, rot=64,
             layout="interleaved", scaling="ramp", dtype="f16", backward=True),
        # one decode step of one request: latency only
        dict(name="append_step", op="append", seqs=1, most=1, ragged=False, before=4099, n_kv=8, n_q=32, rot=128,
             layout="half", scaling="banded", page=16, dtype="bf16"),
        # the prompts of several requests, ragged, rows of one projection's output
        dict(name="append_prompts", op="append", seqs=6, most=8192, ragged=True, before=77, n_kv=4, n_q=28, rot=128,
             layout="half", scaling="linear", page=32, dtype="bf16"),
        # the first tokens after a short prompt: a small cache, latency only
        dict(name="decode_short", op="decode", seqs=1, most=1001, ragged=False, n_kv=8, n_q=32, page=16, dtype="bf16",
             cap=0.0, window=0, slopes=False, prior=False),
        # one long request
        dict(name="decode_long", op="decode", seqs=1, most=131072, ragged=False, n_kv=8, n_q=32, page=16, dtype="bf16",
             cap=0.0, window=0, slopes=False, prior=False),
        # a batch of requests of one length, seven query heads to a kv-head
        dict(name="decode_batch", op="decode", seqs=16, most=8192, ragged=False, n_kv=4, n_q=28, page=64, dtype="f16",
             cap=0.0, window=0, slopes=False, prior=False),
        # a serving batch: ragged tails of sequences whose first part is packed (joined with its result), capped scores
        dict(name="decode_tails", op="decode", seqs=61, most=4001, ragged=True, n_kv=8, n_q=32, page=16, dtype="bf16",
             cap=30.0, window=0, slopes=False, prior=True),
        # copy on write: every sequence of a group that was forked gets its own last page
        dict(name="copy_fork", op="copy", layers=32, pages=96, pairs=7, n_kv=8, page=16, dtype="bf16"),
        # compaction of a pool after many sequences have ended
        dict(name="copy_compact", op="copy", layers=4, pages=4096, pairs=1203, n_kv=4, page=64, dtype="f16"),
        # the oldest tokens of every sequence's recent part, on their way to the packed cache
        dict(name="gather_flush", op="gather", seqs=16, most=139, ragged=False, first=5, tokens=16, n_kv=8, page=16,
             dtype="bf16", padded=False),
        # whole prompts of ragged lengths, padded to the longest
        dict(name="gather_prompts", op="gather", seqs=6, most=8192, ragged=True, first=0, tokens=8192, n_kv=8, page=32,
             dtype="bf16", padded=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "append", "decode", "decode", "decode", "decode", "copy", "gather"])
    n_kv, group = rng.choice([(8, 4), (8, 4), (4, 7), (2, 4), (4, 2), (8, 1), (1, 8), (3, 5), (1, 12)])
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "f16"]))
    if op in ("rotate", "append"):
        c.update(layout=rng.choice(["half", "half", "interleaved"]), rot=rng.choice([128, 128, 64, 32, 96, 16]),
                 scaling=rng.choice(["none", "linear", "ntk", "ramp", "banded"]), ragged=rng.random() < 0.5,
                 before=rng.choice([0, rng.randrange(1, 100000)]))
        heads = n_kv * group
        if op == "rotate":
            c.update(heads=heads, backward=rng.random() < 0.5)
        else:
            heads += 2 * n_kv
            c.update(n_kv=n_kv, n_q=n_kv * group, page=rng.choice([8, 16, 32, 64, 128, 256]), before=rng.randrange(0, 3000))
        c["most"] = _log_int(rng, 1, 32768 * 32 // heads // (2 if op == "append" else 1))
        c["seqs"] = max(1, min(_log_int(rng, 1, 64), 32768 * 32 // heads // c["most"] // 2))
        return c
    c["page"] = rng.choice([8, 16, 16, 32, 64, 128, 256])
    c["n_kv"] = n_kv
    if op == "copy":
        c["layers"] = rng.choice([1, 2, 4, 16, 28, 32])
        size = 512 * n_kv * c["page"] * c["layers"]              # bytes of a page in all layers
        c["pages"] = _log_int(rng, 4, max(8, min(8192, (1 << 29) // size)))
        c["pairs"] = min(c["pages"] // 2, _log_int(rng, 1, 2000))
        return c
    c["most"] = _log_int(rng, 1, 131072)
    c["seqs"] = max(1, min(_log_int(rng, 1, 200), 131072 * 8 // n_kv // c["most"] // 2, 131072 // c["most"]))
    c["ragged"] = rng.random() < 0.5
    if op == "gather":
        c["padded"] = rng.random() < 0.5
        c["tokens"] = _log_int(rng, 1, c["most"])
        c["first"] = rng.randrange(0, c["most"] - c["tokens"] + 1)
        return c
    c.update(n_q=n_kv * group, cap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=rng.random() < 0.25, prior=rng.random() < 0.3,
             window=rng.choice([0, 0, 0, 128, 1000, 4096]))
    return c


# ---------------------------------------------------------------- the sizes that a case stands for
def _lengths(case):
    """Tokens of every sequence (for append: the new ones), by the case alone."""
    c = case
    if not c["ragged"]:
        return [c["most"]] * c["seqs"]
    rng = random.Random(c["seqs"] * 1000003 + c["most"])
    got = [_log_int(rng, max(1, c["most"] // 64), c["most"]) for _ in range(c["seqs"])]
    got[0] = c["most"]
    if c["seqs"] > 4:
        got[3] = 0                                              # a slot of the batch with no sequence
    return got


def _frequencies(case):
    """Angles per position in 64 bits and the factor on the turned values.

    linear: all divided by 4.  ntk: the base grown so that the slowest is divided by 4.  ramp (4096
    original positions, 32 and 1 turns): fast ones kept, slow ones divided by 4, a linear ramp over
    the index between.  banded (8192 original positions, 1 and 4): the same by wavelength, by 8."""
    r, kind, base = case["rot"], case["scaling"], 500000.0 if case["scaling"] == "banded" else 10000.0
    if kind == "ntk":
        base *= 4.0 ** (r / (r - 2))
    w = base ** (-np.arange(0, r, 2) / r)
    if kind == "linear":
        return w / 4.0, 1.0
    if kind == "ramp":
        lo, hi = (r * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(base)) for turns in (32.0, 1.0))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), r - 1)
        t = np.clip((np.arange(r // 2) - lo) / max(hi - lo, 1e-3), 0, 1)
        return w / 4.0 * t + w * (1 - t), 0.1 * math.log(4.0) + 1
    if kind == "banded":
        share = np.clip((8192 * w / (2 * math.pi) - 1.0) / (4.0 - 1.0), 0, 1)      # 1: short waves, kept
        return w / 8.0 * (1 - share) + w * share, 1.0
    return w, 1.0


def _scaling(kind):
    return {"none": None, "linear": dict(kind="linear", factor=4.0), "ntk": dict(kind="ntk", factor=4.0),
            "ramp": dict(kind="ramp", factor=4.0, original=4096, fast=32.0, slow=1.0),
            "banded": dict(kind="banded", factor=8.0, original=8192, low=1.0, high=4.0)}[kind]


def _slopes(n_q):
    """One per query head, a geometric sequence."""
    return [2.0 ** (-8.0 * (i + 1) / n_q) for i in range(n_q)]


def _capacity(case):
    """Pages of one sequence's table."""
    return -(-(case["most"] + case.get("before", 0)) // case["page"])


# ---------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(DEV)
    g.manual_seed(int(seed))
    return g


def _normal(shape, gen, dtype, spread=None):
    x = torch.randn(shape, generator=gen, device=DEV)
    return (x if spread is None else x * spread).to(dtype)


def _pool(case, n_pages, layers, gen):
    """Pages [layers][n_pages][keys | values][n_kv][page][128]: keys with a falling spectrum and four outlier channels."""
    spread = torch.arange(1, D + 1, device=DEV) ** -0.25
    spread[::37] *= 4.0
    spread *= 3.0                                               # scores of a few units: some tokens stand out
    data = torch.empty((layers, n_pages, 2, case["n_kv"], case["page"], D), dtype=TYPES[case["dtype"]], device=DEV)
    for layer in range(layers):
        data[layer, :, 0] = _normal(data[layer, :, 0].shape, gen, data.dtype, spread)
        data[layer, :, 1] = _normal(data[layer, :, 1].shape, gen, data.dtype)
    return data


def _tokens_of(case, gen):
    """Packed tokens of an append or a rotation: their sequences and their indexes there."""
    lens = _lengths(case)
    rows = torch.tensor(np.repeat(np.arange(len(lens)), lens), dtype=torch.int32, device=DEV)
    index = np.concatenate([np.arange(case["before"], case["before"] + n) for n in lens])
    return rows, torch.tensor(index, dtype=torch.int32, device=DEV)


def _inputs(case, seed):
    """The tensors of one pass, from the seed alone."""
    c, g = case, _generator(seed)
    dtype = TYPES[c["dtype"]]
    if c["op"] == "rotate":
        rows, index = _tokens_of(c, g)
        return dict(x=_normal((len(index), c["heads"], D), g, dtype), positions=index)
    if c["op"] == "copy":
        order = torch.randperm(c["pages"], generator=g, device=DEV)[:2 * c["pairs"]].to(torch.int32)
        return dict(data=_pool(c, c["pages"], c["layers"], g), pairs=order.view(2, -1).T.contiguous())
    per_seq = _capacity(c)
    n_pages = c["seqs"] * per_seq + 3
    table = torch.randperm(n_pages, generator=g, device=DEV)[:c["seqs"] * per_seq].to(torch.int32).view(c["seqs"], -1)
    got = dict(data=_pool(c, n_pages, 1, g), table=table.contiguous())
    if c["op"] == "append":
        rows, index = _tokens_of(c, g)
        qkv = _normal((len(index), c["n_q"] + 2 * c["n_kv"], D), g, dtype)         # a fused projection's output
        return dict(got, rows=rows, index=index, q=qkv[:, :c["n_q"]], k=qkv[:, c["n_q"]:c["n_q"] + c["n_kv"]],
                    v=qkv[:, c["n_q"] + c["n_kv"]:])
    got["lens"] = torch.tensor(_lengths(c), dtype=torch.int32, device=DEV)
    if c["op"] == "decode":
        got["q"] = _normal((c["seqs"], c["n_q"], D), g, dtype)
        if c["slopes"]:
            got["slopes"] = torch.tensor(_slopes(c["n_q"]), dtype=torch.float32, device=DEV)
        if c["prior"]:
            got["prior"] = (torch.randn((c["seqs"], c["n_q"], D), generator=g, device=DEV) * 0.1,
                            torch.randn((c["seqs"], c["n_q"]), generator=g, device=DEV) + 6.0)
    return got


def prepare(case, seed):
    c = case
    state = dict(_inputs(c, seed), case=c)
    if "rot" in c:
        # the tables of a program that turns with elementary operations
        w, factor = _frequencies(c)
        angles = torch.arange(c["before"] + c["most"], dtype=torch.float64, device=DEV)[:, None] * torch.tensor(w, device=DEV)
        state.update(cos=(angles.cos() * factor).float(), sin=(angles.sin() * factor).float())
    if c["op"] == "append":
        state["q_out"] = torch.empty(state["q"].shape, dtype=state["q"].dtype, device=DEV)
    if c["op"] == "copy":
        state["moves"] = state["pairs"].cpu().numpy()            # a pool's bookkeeping is on the host
    if c["op"] == "decode":
        state["out"] = torch.empty((c["seqs"], c["n_q"], D), device=DEV)
        state["lse"] = torch.empty((c["seqs"], c["n_q"]), device=DEV)
    if own:
        from paper_2608_14191_gb300 import paged
        if "rot" in c:
            state["rope"] = paged.Rotary(c["rot"], 500000.0 if c["scaling"] == "banded" else 10000.0, layout=c["layout"],
                                         scaling=_scaling(c["scaling"]), device=DEV)
        if "data" in state:
            state["pages"] = paged.Pages.of(state["data"])
        if c["op"] == "decode":
            state["workspace"] = state["pages"].decode_workspace(c["n_q"])
    return state


# ---------------------------------------------------------------- one pass
def _turn(x, cos, sin, layout):
    """x [tokens][heads][128] turned by cos, sin [tokens][r / 2], in 32 bits, rounded once."""
    r = 2 * cos.shape[1]
    xf = x.float()
    cos, sin = cos[:, None], sin[:, None]
    a, b = (xf[..., :r // 2], xf[..., r // 2:r]) if layout == "half" else (xf[..., 0:r:2], xf[..., 1:r:2])
    lo, hi = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat([lo, hi], -1) if layout == "half" else torch.stack([lo, hi], -1).flatten(-2)
    return torch.cat([turned.to(x.dtype), x[..., r:]], -1)


def _plain_decode(s):
    c = s["case"]
    b, m = s["table"].shape
    kv = s["data"][0][s["table"].long()]                         # [b][m][2][n_kv][page][128]
    k, v = (kv[:, :, i].transpose(1, 2).reshape(b, c["n_kv"], m * c["page"], D).float() for i in (0, 1))
    q = s["q"].float().view(b, c["n_kv"], -1, D)
    score = q @ k.transpose(-1, -2) / math.sqrt(D)               # [b][n_kv][group][tokens]
    if c["cap"]:
        score = c["cap"] * torch.tanh(score / c["cap"])
    t = torch.arange(m * c["page"], device=DEV)
    lens = s["lens"][:, None].long()
    if c["slopes"]:
        score = score + s["slopes"].view(1, c["n_kv"], -1, 1) * (t - (lens - 1))[:, None, None].float()
    seen = t < lens
    if c["window"]:
        seen = seen & (t >= lens - c["window"])
    score = torch.where(seen[:, None, None], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    if c["prior"]:
        out0, lse0 = s["prior"][0].view(q.shape), s["prior"][1].view(top.shape)
        top = torch.maximum(top, lse0)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(score - top)
    total, acc = e.sum(-1, keepdim=True), e @ v
    if c["prior"]:
        e0 = torch.exp(lse0 - top)
        total, acc = total + e0, acc + e0 * out0
    out = torch.where(total > 0, acc / total, 0.0)
    return out.reshape(b, c["n_q"], D), (top + torch.log(total)).reshape(b, c["n_q"])


def _plain(s):
    c = s["case"]
    if c["op"] == "rotate":
        at = s["positions"].long()
        sin = s["sin"][at]
        return _turn(s["x"], s["cos"][at], -sin if c["backward"] else sin, c["layout"])
    if c["op"] == "append":
        at = s["index"].long()
        cos, sin = s["cos"][at], s["sin"][at]
        page = s["table"][s["rows"].long(), at // c["page"]].long()
        s["data"][0, page, 0, :, at % c["page"]] = _turn(s["k"], cos, sin, c["layout"])
        s["data"][0, page, 1, :, at % c["page"]] = s["v"]
        return dict(q=_turn(s["q"], cos, sin, c["layout"]), pages=s["data"])
    if c["op"] == "decode":
        out, lse = _plain_decode(s)
        return dict(out=out, lse=lse)
    if c["op"] == "copy":
        s["data"][:, s["pairs"][:, 1].long()] = s["data"][:, s["pairs"][:, 0].long()]
        return s["data"]
    t = torch.arange(c["first"], c["first"] + c["tokens"], device=DEV)
    page = s["table"][:, t // c["page"]].long()                  # [b][tokens]
    k, v = s["data"][0, page, 0, :, t % c["page"]], s["data"][0, page, 1, :, t % c["page"]]
    if c["padded"]:
        seen = (t < s["lens"][:, None])[:, :, None, None]
        k, v = torch.where(seen, k, 0), torch.where(seen, v, 0)
    return dict(k=k, v=v)


def run(state):
    if not own:
        return _plain(state)
    from paper_2608_14191_gb300 import paged
    s, c = state, state["case"]
    if c["op"] == "rotate":
        return paged.rotate(s["rope"], s["x"], s["positions"], backward=c["backward"])
    if c["op"] == "append":
        paged.append(s["pages"], 0, s["k"], s["v"], s["table"], s["index"], rows=s["rows"], rope=s["rope"], q=s["q"],
                     q_out=s["q_out"])
        return dict(q=s["q_out"], pages=s["data"])
    if c["op"] == "decode":
        paged.decode_attention(s["pages"], 0, s["q"], s["table"], s["lens"], out=s["out"], lse=s["lse"],
                               prior=s.get("prior"), cap=c["cap"], window=c["window"], slopes=s.get("slopes"),
                               workspace=s["workspace"])
        return dict(out=s["out"], lse=s["lse"])
    if c["op"] == "copy":
        paged.copy_pages(s["pages"], s["moves"])
        return s["data"]
    k, v = paged.gather(s["pages"], 0, s["table"], c["first"], c["tokens"], lens=s["lens"] if c["padded"] else None)
    return dict(k=k, v=v)


# ---------------------------------------------------------------- work and 64-bit results
def work(case):
    c = case
    if c["op"] == "copy":
        return dict(bytes=2.0 * c["pairs"] * c["layers"] * c["page"] * c["n_kv"] * D * 4, flops=0.0)
    if c["op"] == "gather":
        seen = [min(max(n - c["first"], 0), c["tokens"]) if c["padded"] else c["tokens"] for n in _lengths(c)]
        return dict(bytes=(sum(seen) + c["seqs"] * c["tokens"]) * c["n_kv"] * D * 4.0, flops=0.0)
    tokens = sum(_lengths(c))
    if c["op"] == "rotate":
        return dict(bytes=tokens * (c["heads"] * D * 4.0 + 4), flops=3.0 * tokens * c["heads"] * c["rot"])
    if c["op"] == "append":
        heads = c["n_q"] + c["n_kv"]
        return dict(bytes=tokens * ((heads + c["n_kv"]) * D * 4.0 + 8), flops=3.0 * tokens * heads * c["rot"])
    tokens = sum(min(n, c["window"] or n) for n in _lengths(c))
    rows = c["seqs"] * c["n_q"]
    return dict(bytes=tokens * c["n_kv"] * D * 4.0 + rows * (D * 6 + 4 + (D * 4 + 4 if c["prior"] else 0)),
                flops=4.0 * tokens * c["n_q"] * D)


def _exact_turn(case, x, positions, backward=False):
    """Every pair as a complex number times factor e^(i position w)."""
    w, factor = _frequencies(case)
    r = case["rot"]
    angle = positions.double()[:, None] * torch.tensor(w, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full_like(angle, factor), -angle if backward else angle)[:, None]
    y = x.double().clone()
    pairs = [slice(0, r // 2), slice(r // 2, r)] if case["layout"] == "half" else [slice(0, r, 2), slice(1, r, 2)]
    z = torch.complex(y[..., pairs[0]], y[..., pairs[1]]) * turn
    y[..., pairs[0]], y[..., pairs[1]] = z.real, z.imag
    return y


def exact(case, seed):
    c = case
    if c["op"] in ("copy", "gather"):
        return None                                             # moved, not computed
    got = _inputs(c, seed)
    if c["op"] == "rotate":
        return _exact_turn(c, got["x"], got["positions"], c["backward"])
    if c["op"] == "append":
        pages = got["data"].double()
        k = _exact_turn(c, got["k"], got["index"])
        flat = pages[0].permute(0, 3, 1, 2, 4)                   # [page][slot][keys | values][n_kv][128], a view
        at = got["index"].long()
        where = got["table"].long()[got["rows"].long(), torch.div(at, c["page"], rounding_mode="floor")]
        flat[where, at % c["page"]] = torch.stack([k, got["v"].double()], 1)
        return dict(q=_exact_turn(c, got["q"], got["index"]), pages=pages)
    out = torch.zeros((c["seqs"], c["n_q"], D), dtype=torch.float64, device=DEV)
    lse = torch.full((c["seqs"], c["n_q"]), -math.inf, dtype=torch.float64, device=DEV)
    group = c["n_q"] // c["n_kv"]
    slopes = torch.tensor(_slopes(c["n_q"]), dtype=torch.float32, device=DEV).double()
    for b, n in enumerate(_lengths(c)):
        lo = max(0, n - c["window"]) if c["window"] else 0
        used = got["data"][0][got["table"][b, :-(-n // c["page"])].long()]
        for h in range(c["n_kv"]):
            k, v = (used[:, i, h].reshape(-1, D)[lo:n].double() for i in (0, 1))
            heads = slice(h * group, (h + 1) * group)
            s = got["q"][b, heads].double() @ k.T / math.sqrt(D)
            if c["cap"]:
                s = torch.tanh(s / c["cap"]) * c["cap"]
            if c["slopes"]:
                s = s - slopes[heads, None] * torch.arange(n - 1 - lo, -1, -1, dtype=torch.float64, device=DEV)
            if c["prior"]:                                      # one more token: score lse0, value out0
                s = torch.cat([s, got["prior"][1][b, heads, None].double()], 1)
            if s.shape[1] == 0:
                continue
            p = torch.softmax(s, -1)
            out[b, heads] = p[:, :n - lo] @ v
            if c["prior"]:
                out[b, heads] += p[:, -1:] * got["prior"][0][b, heads].double()
            lse[b, heads] = torch.logsumexp(s, -1)
    return dict(out=out, lse=lse)
