"""The operators of a decode over paged caches, measured one at a time.

Three operators: attention of one new token per sequence over a paged key-value cache; the
pages themselves (copies between a session and pages, forks that share pages until they are
written, compaction); penalties, biases and allowed-token masks on logits with the reductions a
greedy step reads.  With ``own`` false ``run`` computes them in elementary torch operations in 32
bits, with ``own`` true it makes the calls of the public binding.

Shapes are this repository's own (the fp32 tiny model, the small bf16 model of the session tests,
the 8B and 32B shapes) and two odd head layouts.  Cells and queries are normal, logits N(0, 2)
like those of its gate tests, tokens of a history uniform with a repeated share.

A page holds the cells of every layer: [layer][K, V][kv heads * page cells * head_dim], K as
[kv head][cell][dim] and V transposed as [kv head][dim][cell].  A session's buffer holds, per
layer, K as [kv head][capacity][dim] and V as [kv head][dim][capacity], the capacity rounded up to
64 cells.
"""
import math

import numpy as np
import torch

own = False

# query heads, kv heads, head_dim, element type of the cells
HEADS = {
    "tiny-f32": (4, 4, 64, "f32"),
    "small": (4, 2, 64, "bf16"),
    "8b": (32, 8, 128, "bf16"),
    "32b": (64, 8, 128, "bf16"),
    "thirds": (6, 2, 64, "f32"),
    "one-kv": (20, 1, 128, "bf16"),
}
DEV = "cuda"


def listed():
    return [
        # one sequence of the fp32 model of the smoke tests: launches and latency
        {"name": "attn_tiny_f32", "op": "attention", "heads": "tiny-f32", "n": 1, "cells": 512,
         "page": 16, "ragged": False, "holes": 0.0},
        # a decode step after a fall-through: one continuation of a streaming session
        {"name": "attn_8b_one", "op": "attention", "heads": "8b", "n": 1, "cells": 8192, "page": 64,
         "ragged": False, "holes": 0.0},
        # 64 sequences of unequal lengths, as in the batched workload
        {"name": "attn_8b_ragged64", "op": "attention", "heads": "8b", "n": 64, "cells": 8192,
         "page": 64, "ragged": True, "holes": 0.0},
        # a few continuations of a long history, the 32B heads
        {"name": "attn_32b_long", "op": "attention", "heads": "32b", "n": 3, "cells": 32749,
         "page": 128, "ragged": False, "holes": 0.0},
        # small pages, short and empty sequences, pages dropped from the middle
        {"name": "attn_small_holes", "op": "attention", "heads": "small", "n": 37, "cells": 700,
         "page": 16, "ragged": True, "holes": 0.2},
        # a handful of candidate answers of the small model, half of them kept
        {"name": "fork_small", "op": "fork", "heads": "small", "layers": 2, "cells": 100, "n": 5,
         "page": 16},
        # 64 candidate answers of an 8B state, half of them kept
        {"name": "fork_8b", "op": "fork", "heads": "8b", "layers": 8, "cells": 1000, "n": 64,
         "page": 64},
        # a session's cells into pages and into another session
        {"name": "import_8b", "op": "import", "heads": "8b", "layers": 4, "cells": 8100, "page": 64},
        # one row of the tiny model's vocabulary
        {"name": "logits_tiny", "op": "logits", "vocab": 4096, "n": 1, "history": 200, "biases": 0,
         "allowed": 1.0},
        # one decode step: penalties over a conversation, a grammar that allows few tokens
        {"name": "logits_one", "op": "logits", "vocab": 128256, "n": 1, "history": 6000, "biases": 50,
         "allowed": 0.02},
        # a step of 64 sequences, penalties and biases, nothing masked
        {"name": "logits_64", "op": "logits", "vocab": 128256, "n": 64, "history": 2000, "biases": 100,
         "allowed": 1.0},
        # an odd vocabulary, half of it allowed
        {"name": "logits_odd", "op": "logits", "vocab": 152063, "n": 17, "history": 700, "biases": 9,
         "allowed": 0.5},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attention", "attention", "fork", "import", "logits", "logits"))
    if op == "logits":
        return {"op": op, "vocab": _log(rng, 2000, 160000), "n": _log(rng, 1, 52),
                "history": rng.choice((0, _log(rng, 1, 8000))), "biases": rng.choice((0, _log(rng, 1, 300))),
                "allowed": rng.choice((1.0, rng.uniform(0.001, 0.9)))}
    page = rng.choice((16, 32, 64, 128))
    if op == "attention":
        heads = rng.choice(sorted(HEADS))
        n = _log(rng, 1, 64)
        return {"op": op, "heads": heads, "n": n,
                "cells": min(_log(rng, 1, 32768), 262144 // n), "page": page,
                "ragged": rng.random() < 0.6, "holes": rng.choice((0.0, 0.0, rng.uniform(0.0, 0.5)))}
    heads = rng.choice(("tiny-f32", "small", "8b", "8b"))
    if op == "import":
        return {"op": op, "heads": heads, "layers": rng.randint(1, 4), "cells": _log(rng, 1, 8192),
                "page": page}
    # a length inside a page: what a fork has to copy
    cells = _log(rng, 1, 2000)
    return {"op": op, "heads": heads, "layers": rng.randint(1, 4),
            "cells": cells if cells % page else cells + 1, "n": _log(rng, 2, 64), "page": page}


# ---- inputs -------------------------------------------------------------------------------


def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * seed + stream)
    return g


def _dtype(case):
    return torch.float32 if HEADS[case["heads"]][3] == "f32" else torch.bfloat16


def _normal(shape, dtype, g, sigma=1.0):
    """Normal values; a large tensor is a block of 2^22 + 1 of them over and over, which is
    quick and lines up with no row."""
    n = math.prod(shape)
    block = torch.empty(min(n, (1 << 22) + 1), dtype=dtype, device=DEV).normal_(0.0, sigma, generator=g)
    if block.numel() == n:
        return block.view(shape)
    return block.repeat(-(-n // block.numel()))[:n].view(shape)


def _lengths(case):
    """Cells of each sequence: from the case alone, so that its work is known."""
    n, cells = case["n"], case["cells"]
    if not case["ragged"]:
        return np.full(n, cells)
    r = np.random.RandomState(cells + 31 * n + case["page"])  # down to an eighth; one in 16 is empty
    lengths = r.randint(max(1, cells // 8), cells + 1, n)
    lengths[r.rand(n) < 1 / 16] = 0
    return lengths


def _attention_inputs(case, seed):
    nq, nkv, dh, _ = HEADS[case["heads"]]
    n, cells, page, dt = case["n"], case["cells"], case["page"], _dtype(case)
    g = _gen(seed, 1)
    lengths = _lengths(case)
    width = -(-cells // page)
    pages = n * width + 3
    # the pages of a sequence lie anywhere, as they do after hours of serving
    table = torch.randperm(pages, generator=g, device=DEV)[:n * width].view(n, width).to(torch.int32)
    if case["holes"]:
        table[torch.rand(n, width, generator=g, device=DEV) < case["holes"]] = -1
    return {"pages": _normal((pages, 1, 2, nkv * page * dh), dt, g), "table": table,
            "lengths": torch.from_numpy(lengths).to(DEV, torch.int32),
            "q": _normal((n, nq, dh), dt, g, 1.5)}


def _fork_inputs(case, seed):
    _, nkv, dh, _ = HEADS[case["heads"]]
    base = -(-case["cells"] // case["page"])
    return {"pages": _normal((base + case["n"], case["layers"], 2, nkv * case["page"] * dh),
                             _dtype(case), _gen(seed, 2)), "base": base}


def _import_inputs(case, seed):
    _, nkv, dh, _ = HEADS[case["heads"]]
    dt, g = _dtype(case), _gen(seed, 3)
    cap = -(-case["cells"] // 64) * 64
    elems = nkv * cap * dh
    return {"kv": _normal((case["layers"], 2, elems), dt, g),
            "other": _normal((case["layers"], 2, elems), dt, g),
            "pages": _normal((-(-case["cells"] // case["page"]), case["layers"], 2,
                              nkv * case["page"] * dh), dt, g)}


REPETITION, FREQUENCY, PRESENCE = 1.2, 0.3, 0.1


def _logits_inputs(case, seed):
    n, V, T = case["n"], case["vocab"], case["history"]
    g = _gen(seed, 4)
    # histories of unequal lengths; half of each is a prompt, and a third of its tokens come from
    # a few hundred (a text repeats itself)
    r = np.random.RandomState(V + 31 * n + T)
    lens = r.randint(T // 2, T + 1, n)
    tokens = torch.randint(0, V, (n, T), device=DEV, generator=g)
    few = torch.rand(n, T, device=DEV, generator=g) < 0.33
    tokens = torch.where(few, tokens % 300, tokens).to(torch.int32)
    bias_tokens = torch.rand(n, V, device=DEV, generator=g).topk(case["biases"], dim=1).indices.to(torch.int32)
    words = -(-V // 32)
    allowed = None
    if case["allowed"] < 1.0:
        bits = torch.rand(n, words, 32, device=DEV, generator=g) < case["allowed"]
        bits[:, (V // 3) >> 5, (V // 3) & 31] = True  # a grammar always allows something
        weight = (1 << torch.arange(32, device=DEV, dtype=torch.int64))
        word = (bits * weight).sum(2)
        allowed = torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)
    return {"logits": torch.empty(n, V, device=DEV).normal_(0.0, 2.0, generator=g), "tokens": tokens,
            "lens": lens, "prompt": lens // 2, "bias_tokens": bias_tokens,
            "bias": torch.empty(n, case["biases"], device=DEV).normal_(0.0, 3.0, generator=g),
            "allowed": allowed, "out": torch.empty(n, V, device=DEV)}


INPUTS = {"attention": _attention_inputs, "fork": _fork_inputs, "import": _import_inputs,
          "logits": _logits_inputs}


def prepare(case, seed):
    s = {"case": case, **INPUTS[case["op"]](case, seed)}
    if case["op"] == "logits":
        # device copies for the plain form, which takes all rows at once
        s["lens_dev"] = torch.from_numpy(s["lens"]).to(DEV)
        s["prompt_dev"] = torch.from_numpy(s["prompt"]).to(DEV)
        s["repetition"] = torch.full((), REPETITION, device=DEV)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a user's program makes once of the framework's objects."""
    import paper_2606_29565_amd as spp

    case = s["case"]
    if case["op"] == "logits":
        rows = [spp.AdjustRow(s["logits"][i], s["out"][i], tokens=s["tokens"][i], n_tokens=int(s["lens"][i]),
                              n_prompt=int(s["prompt"][i]), repetition=REPETITION, frequency=FREQUENCY,
                              presence=PRESENCE, bias_tokens=s["bias_tokens"][i], bias=s["bias"][i],
                              allowed=None if s["allowed"] is None else s["allowed"][i])
                for i in range(case["n"])]
        s["call"] = spp.LogitsAdjust(case["vocab"], rows)
        return
    nq, nkv, dh, fmt = HEADS[case["heads"]]
    layers = case.get("layers", 1)
    s["pool"] = spp.PagePool(layers, nkv, dh, fmt == "bf16", case["page"], s["pages"].shape[0],
                             max_seqs=case["n"] + 1 if case["op"] == "fork" else 4, pages=s["pages"])
    if case["op"] == "attention":
        s["call"] = spp.PagedAttention(s["pool"], 0, nq, s["table"], s["lengths"], io_bf16=fmt == "bf16")
        s["o"] = torch.empty_like(s["q"])
    elif case["op"] == "fork":
        s["seq"] = s["pool"].create(case["cells"])
    else:
        # the sessions of a model with these cells; the copies read nothing else of it
        dt, d, ffn, vocab = _dtype(case), 64, 64, 64
        shapes = {"wq": (nkv * dh, d), "wk": (nkv * dh, d), "wv": (nkv * dh, d), "wo": (d, nkv * dh),
                  "w_gate": (ffn, d), "w_up": (ffn, d), "w_down": (d, ffn), "attn_norm": (d,),
                  "mlp_norm": (d,)}
        w = {k: [torch.zeros(v, dtype=dt, device=DEV)] * layers for k, v in shapes.items()}
        w.update(embed=torch.zeros(vocab, d, dtype=dt, device=DEV),
                 final_norm=torch.zeros(d, dtype=dt, device=DEV),
                 lm_head=torch.zeros(vocab, d, dtype=dt, device=DEV))
        s["model"] = spp.Model(layers, d, nkv, nkv, dh, ffn, vocab, 1e4, fmt == "bf16", w, max_tokens=1)
        s["session"] = spp.Session(s["model"], case["cells"], kv=s["kv"])
        s["session"].restore(case["cells"])
        s["into"] = spp.Session(s["model"], case["cells"], kv=s["other"])


# ---- one pass -------------------------------------------------------------------------------


def run(s):
    if own:
        return {"attention": _own_attention, "fork": _own_fork, "import": _own_import,
                "logits": _own_logits}[s["case"]["op"]](s)
    return {"attention": _plain_attention, "fork": _plain_fork, "import": _plain_import,
            "logits": _plain_logits}[s["case"]["op"]](s)


def _own_attention(s):
    s["call"](s["q"], s["o"])
    return s["o"]


def _own_fork(s):
    """Forks of a state, each made ready for its first own cell, every other one given up, and
    the pages that are left moved together."""
    pool = s["pool"]
    forks = pool.fork(s["seq"], s["case"]["n"])
    pool.reserve(forks, 1)
    for f in forks[1::2]:
        pool.free(f)
    pool.compact()
    last = [pool.table(f)[-1] for f in forks[::2]]
    live = s["pages"][:pool.info().used_pages]
    for f in forks[::2]:
        pool.free(f)
    return {"pages": live, "last": np.array(last, dtype=np.int32)}


def _own_import(s):
    seq = s["pool"].create(0)
    s["pool"].import_session(seq, s["session"])
    s["pool"].export_session(seq, s["into"])
    s["pool"].free(seq)
    return {"pages": s["pages"], "other": s["other"]}


def _own_logits(s):
    r = s["call"]()
    return {"logits": s["out"], "argmax": r.argmax, "top1": r.top1, "top2": r.top2, "lse": r.lse}


def _plain_attention(s):
    case = s["case"]
    nq, nkv, dh, _ = HEADS[case["heads"]]
    n, page = case["n"], case["page"]
    width = s["table"].shape[1]
    listed_page = s["table"] >= 0
    cells = s["pages"][s["table"].clamp(min=0).long(), 0]  # [n, width, 2, elements of a page]
    K = cells[:, :, 0].reshape(n, width, nkv, page, dh).permute(0, 2, 1, 3, 4).reshape(n, nkv, width * page, dh)
    V = cells[:, :, 1].reshape(n, width, nkv, dh, page).permute(0, 2, 1, 4, 3).reshape(n, nkv, width * page, dh)
    live = torch.arange(width * page, device=DEV) < s["lengths"][:, None]
    live = live & listed_page.repeat_interleave(page, dim=1)
    q = s["q"].float().view(n, nkv, nq // nkv, dh)
    scores = torch.matmul(q, K.float().transpose(2, 3).contiguous()) / math.sqrt(dh)
    scores = scores.masked_fill(~live[:, None, None], -math.inf)
    top = scores.amax(3, keepdim=True).clamp(min=-1e30)  # an empty row has no maximum
    e = torch.exp(scores - top)
    total = e.sum(3, keepdim=True)
    out = torch.matmul(e, V.float()) / torch.where(total > 0, total, torch.ones_like(total))
    return out.view(n, nq, dh).to(s["q"].dtype)


def _plain_fork(s):
    n, base, pages = s["case"]["n"], s["base"], s["pages"]
    # the last page of every fork is its own: pages base .. base + n - 1
    pages[base:base + n] = pages[base - 1]
    kept = base + torch.arange(0, n, 2, device=DEV)
    used = base + kept.numel()
    # pages past the live ones move, in order, to the free ones below
    free = base + torch.arange(1, n, 2, device=DEV)
    src, dst = kept[kept >= used], free[free < used]
    pages[dst] = pages[src]
    last = kept.clone()
    last[kept >= used] = dst
    return {"pages": pages[:used], "last": last.to(torch.int32)}


def _plain_import(s):
    case = s["case"]
    _, nkv, dh, _ = HEADS[case["heads"]]
    L, n, page = case["layers"], case["cells"], case["page"]
    cap = s["kv"].shape[2] // (nkv * dh)
    full, rest = n // page, n % page
    for_keys = lambda t: t[:, 0].view(L, nkv, cap, dh)  # noqa: E731
    for_values = lambda t: t[:, 1].view(L, nkv, dh, cap)  # noqa: E731
    K, V, K2, V2 = for_keys(s["kv"]), for_values(s["kv"]), for_keys(s["other"]), for_values(s["other"])
    pk = s["pages"][:, :, 0].view(-1, L, nkv, page, dh)
    pv = s["pages"][:, :, 1].view(-1, L, nkv, dh, page)
    whole = full * page
    pk[:full] = K[:, :, :whole].reshape(L, nkv, full, page, dh).permute(2, 0, 1, 3, 4)
    pv[:full] = V[..., :whole].reshape(L, nkv, dh, full, page).permute(3, 0, 1, 2, 4)
    K2[:, :, :whole] = pk[:full].permute(1, 2, 0, 3, 4).reshape(L, nkv, whole, dh)
    V2[..., :whole] = pv[:full].permute(1, 2, 3, 0, 4).reshape(L, nkv, dh, whole)
    if rest:
        pk[full, :, :, :rest] = K[:, :, whole:n]
        pv[full, :, :, :, :rest] = V[..., whole:n]
        K2[:, :, whole:n] = pk[full, :, :, :rest]
        V2[..., whole:n] = pv[full, :, :, :, :rest]
    return {"pages": s["pages"], "other": s["other"]}


def _plain_logits(s):
    case = s["case"]
    n, V, T = case["n"], case["vocab"], case["history"]
    x = s["logits"]
    at = torch.arange(T, device=DEV)
    tok = s["tokens"].long()
    live = at < s["lens_dev"][:, None]
    answer = live & (at >= s["prompt_dev"][:, None])
    ones = torch.ones_like(tok, dtype=torch.float32)
    seen = torch.zeros(n, V, device=DEV).scatter_add_(1, tok, ones * live)
    count = torch.zeros(n, V, device=DEV).scatter_add_(1, tok, ones * answer)
    x = torch.where(seen > 0, torch.where(x > 0, x / s["repetition"], x * s["repetition"]), x)
    x = x - FREQUENCY * count
    x = x - PRESENCE * (count > 0)
    x = x + torch.zeros(n, V, device=DEV).scatter_(1, s["bias_tokens"].long(), s["bias"])
    ids = torch.arange(V, device=DEV)
    if s["allowed"] is not None:
        bit = (s["allowed"][:, ids >> 5] >> (ids & 31)) & 1
        x = torch.where(bit > 0, x, torch.full_like(x, -math.inf))
    top1 = x.amax(1)
    argmax = torch.where(x == top1[:, None], ids, V).amin(1)
    top2 = torch.where(ids == argmax[:, None], -math.inf, x).amax(1)
    lse = top1 + torch.log(torch.exp(x - top1[:, None]).sum(1))
    return {"logits": x, "argmax": argmax.to(torch.int32), "top1": top1, "top2": top2, "lse": lse}


# ---- what a pass cannot do without --------------------------------------------------------


def work(case):
    if case["op"] == "logits":
        n, V = case["n"], case["vocab"]
        mask = V / 8 if case["allowed"] < 1.0 else 0
        return {"bytes": int(n * (8 * V + mask + 3 * case["history"] + 8 * case["biases"] + 20)),
                "flops": int(n * 6 * V)}
    nq, nkv, dh, fmt = HEADS[case["heads"]]
    elem = 4 if fmt == "f32" else 2
    cell = 2 * nkv * dh * elem
    if case["op"] == "attention":
        cells = int(_lengths(case).sum()) * (1 - case["holes"])
        return {"bytes": int(cells * cell + 2 * case["n"] * nq * dh * elem),
                "flops": int(4 * cells * nq * dh)}
    page = case["page"] * cell * case["layers"]
    if case["op"] == "fork":  # the shared last page read once, a copy for each; a quarter moves
        return {"bytes": int(page * (1 + case["n"] + 2 * (case["n"] // 4))), "flops": 0}
    # a session's cells read, pages written and read, the other session's cells written
    return {"bytes": int(4 * case["cells"] * cell * case["layers"]), "flops": 0}


# ---- the same from the definitions, in 64 bits --------------------------------------------


def exact(case, seed):
    s = INPUTS[case["op"]](case, seed)
    return {"attention": _exact_attention, "fork": _exact_fork, "import": _exact_import,
            "logits": _exact_logits}[case["op"]](case, s)


def _exact_attention(case, s):
    nq, nkv, dh, _ = HEADS[case["heads"]]
    page, G = case["page"], nq // nkv
    out = torch.zeros(case["n"], nq, dh, dtype=torch.float64, device=DEV)
    table, lengths = s["table"].cpu().numpy(), s["lengths"].cpu().numpy()
    for i in range(case["n"]):
        at = np.arange(int(lengths[i]))
        at = at[table[i, at // page] >= 0]
        if not at.size:
            continue
        pg = torch.from_numpy(table[i, at // page].astype(np.int64)).to(DEV)
        cell = torch.from_numpy(at % page).to(DEV)
        for h in range(nkv):
            K = s["pages"][:, 0, 0].view(-1, nkv, page, dh)[pg, h, cell].double()
            V = s["pages"][:, 0, 1].view(-1, nkv, dh, page)[pg, h, :, cell].double()
            for j in range(h * G, (h + 1) * G):
                z = (K * s["q"][i, j].double()).sum(1) / math.sqrt(dh)
                p = torch.exp(z - z.max())
                out[i, j] = (p[:, None] * V).sum(0) / p.sum()
    return out


def _exact_fork(case, s):
    n, base, pages = case["n"], s["base"], s["pages"]
    kept = (n + 1) // 2
    last = []
    # fork 2 j's page is base + 2 j while that is one of the first base + kept, else the next odd one
    odd = 1
    for j in range(0, n, 2):
        if j < kept:
            last.append(base + j)
        else:
            last.append(base + odd)
            odd += 2
    return {"pages": torch.cat([pages[:base]] + [pages[base - 1:base]] * kept), "last": np.array(last, np.int32)}


def _exact_import(case, s):
    _, nkv, dh, _ = HEADS[case["heads"]]
    n, page = case["cells"], case["page"]
    pages, other = s["pages"].clone(), s["other"].clone()
    cap = s["kv"].shape[2] // (nkv * dh)
    for l in range(case["layers"]):
        K, V = s["kv"][l, 0].view(nkv, cap, dh), s["kv"][l, 1].view(nkv, dh, cap)
        other[l, 0].view(nkv, cap, dh)[:, :n] = K[:, :n]
        other[l, 1].view(nkv, dh, cap)[:, :, :n] = V[:, :, :n]
        for j in range(pages.shape[0]):
            m = min(page, n - j * page)
            pages[j, l, 0].view(nkv, page, dh)[:, :m] = K[:, j * page:j * page + m]
            pages[j, l, 1].view(nkv, dh, page)[:, :, :m] = V[:, :, j * page:j * page + m]
    return {"pages": pages, "other": other}


def _exact_logits(case, s):
    n, V = case["n"], case["vocab"]
    x = s["logits"].cpu().double().numpy()
    # the penalties are the 32-bit numbers that a call is given
    rep, freq, pres = (float(np.float32(v)) for v in (REPETITION, FREQUENCY, PRESENCE))
    out = np.empty((n, V))
    res = {"argmax": np.empty(n, np.int32), "top1": np.empty(n), "top2": np.empty(n), "lse": np.empty(n)}
    tokens, bt, bv = s["tokens"].cpu().numpy(), s["bias_tokens"].cpu().numpy(), s["bias"].cpu().double().numpy()
    masks = None if s["allowed"] is None else s["allowed"].cpu().numpy().view(np.uint8).reshape(n, -1)
    for i in range(n):
        h, p = int(s["lens"][i]), int(s["prompt"][i])
        row = x[i].copy()
        seen = np.unique(tokens[i, :h])
        row[seen] = np.where(row[seen] > 0, row[seen] / rep, row[seen] * rep)
        count = np.bincount(tokens[i, p:h], minlength=V)
        row -= freq * count + pres * (count > 0)
        row[bt[i]] += bv[i]
        if masks is not None:
            row[~np.unpackbits(masks[i], bitorder="little")[:V].astype(bool)] = -np.inf
        out[i] = row
        res["argmax"][i] = int(np.argmax(row))
        res["top2"][i], res["top1"][i] = np.sort(row)[-2:]
        res["lse"][i] = row.max() + math.log(np.exp(row - row.max()).sum())
    return {"logits": out, **res}
