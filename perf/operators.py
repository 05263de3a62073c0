"""The operators between the kept visual tokens and a language model's answer: what they are measured on.

A case is a dict of plain values.  `op` names the operator:

  positions        kept_positions: (time, height, width) of kept tokens from their indices in the image's grid
  rotate           Attention.rotate: per-head RMS norm of queries and keys and their rotation by positions of
                   several axes, in one pass
  rotate_backward  Attention.rotate_backward: the gradients of the inputs and of the norms' weights
  append           Attention.append: the same on the way of new keys into a paged cache, values beside them
  attend           Attention.attend: attention of a chunk of new tokens, or of single ones, over that cache

Where `own` is false the operators are computed in elementary torch operations in 32 bits, otherwise by the
library.  `pick` draws the sizes of ragged batches and is part of the case; the values come from the seed.
"""
import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6


# ---- cases -------------------------------------------------------------------------------
def positions_case(name, images, grid, kept, pick=1):
    return {"name": name, "op": "positions", "images": images, "t": grid[0], "h": grid[1], "w": grid[2], "kept": kept, "pick": pick}


def rotate_case(name, op, tokens, heads, kv_heads, head_dim, dtype, sections, rot_dim=0, adjacent=False, norm=True, packed=True,
                start=0, pick=1):
    """`sections`: rotated pairs of each axis, "16,24,24".  `packed`: queries and keys are slices of one projection's output."""
    return {"name": name, "op": op, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype,
            "sections": sections, "rot_dim": rot_dim or head_dim, "adjacent": adjacent, "norm": norm, "packed": packed,
            "start": start, "pick": pick}


def cache_case(name, op, seqs, new, old, heads, kv_heads, head_dim, page, causal=True, window=0, lse=False, norm=True,
               sections="16,24,24", pick=1):
    """`new`, `old`: the range of a sequence's tokens of this step and of those that the cache holds before it."""
    return {"name": name, "op": op, "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "old_lo": old[0], "old_hi": old[1],
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "causal": causal, "window": window,
            "lse": lse, "norm": norm, "sections": sections, "adjacent": False, "rot_dim": head_dim, "dtype": "bf16", "pick": pick}


def listed():
    return [
        # one request: the 64 kept tokens of a 24 x 24 image
        positions_case("positions_one", 1, (1, 24, 24), 64),
        # a batch of clips of 32 frames, 1152 tokens kept of each
        positions_case("positions_clips_64", 64, (32, 24, 24), 1152),
        # a batch of prompts: heads of a width-4096 model, grouped keys, three axes
        rotate_case("rotate_prompts_36864", "rotate", 36864, 32, 8, 128, "bf16", "16,24,24"),
        # one image inside an fp32 encoder of width 1024: two axes, adjacent pairs, no norm
        rotate_case("rotate_image_577_fp32", "rotate", 577, 16, 16, 64, "fp32", "16,16", adjacent=True, norm=False),
        # a training step's prompts, the backward pass
        rotate_case("rotate_back_16384", "rotate_backward", 16384, 32, 8, 128, "bf16", "16,24,24"),
        # an odd number of fp32 tokens, seven queries to a key head, part of each head rotated
        rotate_case("rotate_back_1001_fp32", "rotate_backward", 1001, 28, 4, 128, "fp32", "16,8,8", rot_dim=64, packed=False),
        # a decoding step of 64 requests: one token each
        cache_case("append_tokens_64", "append", 64, (1, 1), (255, 2047), 28, 4, 128, 16),
        # reduced prompts of eight requests: some with an earlier turn in the cache
        cache_case("append_prompts_8", "append", 8, (64, 2048), (0, 1024), 32, 8, 128, 64),
        # one request decoding after a reduced clip, every head with keys of its own: bound by latency
        cache_case("attend_token_one", "attend", 1, (1, 1), (1215, 1215), 32, 32, 128, 16),
        # 64 requests decoding, contexts of very different lengths: bound by the cache's bytes
        cache_case("attend_tokens_64", "attend", 64, (1, 1), (255, 16383), 28, 4, 128, 16),
        # a mixed step: chunks of 1 to 512 tokens over long contexts, pages of 48 tokens
        cache_case("attend_chunks_8", "attend", 8, (1, 512), (256, 18432), 28, 4, 128, 48, lse=True),
        # an unreduced clip's prompt from an empty cache: the largest product
        cache_case("attend_prompt_18432", "attend", 1, (18432, 18432), (0, 0), 32, 8, 128, 64),
    ]


def spread(rng, lo, hi):
    """A whole number in [lo, hi], its logarithm uniform."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def split(rng, pairs, axes):
    cuts = sorted(rng.randint(0, pairs) for _ in range(axes - 1))
    return ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [pairs]))


def draw(rng):
    op = rng.choice(["positions", "rotate", "rotate", "rotate_backward", "rotate_backward", "append", "append",
                     "attend", "attend", "attend", "attend", "attend"])
    if op == "positions":
        images = spread(rng, 1, 64)
        t, h, w = rng.choice([1, 1, spread(rng, 1, 32)]), rng.randint(4, 32), rng.randint(4, 32)
        return {"op": op, "images": images, "t": t, "h": h, "w": w, "kept": spread(rng, 1, min(1152, t * h * w)), "pick": rng.randrange(1 << 20)}
    while True:
        kv_heads = rng.choice([1, 2, 4, 4, 8, 8, 16, 32])
        heads = kv_heads * rng.choice([1, 1, 2, 4, 4, 7, 8])
        head_dim = rng.choice([64, 80, 96, 128, 128, 128, 128])
        if heads > 64:
            continue
        if op in ("rotate", "rotate_backward"):
            rot_dim = rng.choice([head_dim, head_dim, head_dim // 2])
            c = {"op": op, "tokens": spread(rng, 1, 36864), "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
                 "dtype": rng.choice(["bf16", "bf16", "fp32"]), "sections": split(rng, rot_dim // 2, rng.choice([1, 2, 3, 3])),
                 "rot_dim": rot_dim, "adjacent": rng.random() < 0.3, "norm": rng.random() < 0.7, "packed": rng.random() < 0.6,
                 "start": rng.choice([0, 0, spread(rng, 1, 4096)]), "pick": rng.randrange(1 << 20)}
        else:
            new = rng.choice([(1, 1), (1, 1), (0, spread(rng, 1, 32)), (1, spread(rng, 2, 512)), (spread(rng, 16, 2048),) * 2,
                              (spread(rng, 64, 16384),) * 2])
            old_hi = rng.choice([0, spread(rng, 1, 18432), spread(rng, 1, 18432), spread(rng, 64, 32768)])
            if op == "append":
                old_hi = min(old_hi, 4096)
            c = {"op": op, "seqs": spread(rng, 1, 64), "new_lo": new[0], "new_hi": new[1],
                 "old_lo": rng.choice([old_hi, old_hi // 4, old_hi // 64]), "old_hi": old_hi, "heads": heads, "kv_heads": kv_heads,
                 "head_dim": head_dim, "page": rng.choice([1, 16, 16, 32, 48, 64, 64, 100, 256]), "causal": rng.random() < 0.85,
                 "window": rng.choice([0, 0, 0, spread(rng, 1, 4096)]), "lse": rng.random() < 0.3, "norm": rng.random() < 0.6,
                 "sections": split(rng, head_dim // 2, 3), "adjacent": rng.random() < 0.2, "rot_dim": head_dim, "dtype": "bf16",
                 "pick": rng.randrange(1 << 20)}
            if not c["causal"]:
                c["window"] = 0
            new_n, _ = lengths(c)
            if sum(new_n) == 0 or cache_bytes(c) > 2.5e9 or (op == "append" and cache_bytes(c) > 2e8):
                continue
            # the plain form's scores do not stop at the diagonal
            if op == "attend" and sum(n * k for n, k in zip(*lengths(c))) * heads > 18432 * 18432 * 32:
                continue
        w = work(c)
        if w["bytes"] <= 1.2e9 and w["flops"] <= 2.9e12:
            return c


# ---- what a case means -------------------------------------------------------------------
def lengths(case):
    """New tokens of each sequence, and its length in the cache with them."""
    rng = random.Random(case["pick"])
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    return new, [n + rng.randint(case["old_lo"], case["old_hi"]) for n in new]


def pages_of(case):
    return sum((kv + case["page"] - 1) // case["page"] for kv in lengths(case)[1])


def cache_bytes(case):
    return 2 * pages_of(case) * case["page"] * case["kv_heads"] * case["head_dim"] * 2


def element(case):
    return 2 if case["dtype"] == "bf16" else 4


def torch_type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def visible(case, n, kv):
    """(query, key) pairs that are not masked in one sequence, and the keys that some query sees."""
    if not case["causal"]:
        return n * kv, kv if n else 0
    pairs, window = 0, case["window"] or kv + 1
    for i in range(kv - n, kv):
        pairs += min(i + 1, window)
    return pairs, min(kv, window + n - 1) if n else 0


def work(case):
    op = case["op"]
    if op == "positions":
        kept = case["images"] * case["kept"]
        return {"bytes": 16 * kept, "flops": 0}
    e, dim = element(case), case["head_dim"]
    if op in ("rotate", "rotate_backward"):
        axes = case["sections"].count(",") + 1
        heads = case["tokens"] * (case["heads"] + case["kv_heads"])
        moved = 2 if op == "rotate" or not case["norm"] else 3      # without a norm the gradient does not need the inputs
        weights = 2 * dim * (e + (4 if op == "rotate_backward" else 0)) if case["norm"] else 0
        flops = heads * (3 * case["rot_dim"] + (4 * dim if case["norm"] else 0)) * (1 if op == "rotate" else 2)
        return {"bytes": moved * heads * dim * e + 4 * axes * case["tokens"] + weights, "flops": flops}
    new, kv = lengths(case)
    rows = sum(new)
    tables = 4 * (pages_of(case) + 2 * case["seqs"] + 1)
    if op == "append":
        moved = 2 * rows * (case["heads"] + 2 * case["kv_heads"]) * dim * e
        return {"bytes": moved + 12 * rows + 4 * rows + 8 * case["seqs"], "flops": rows * (case["heads"] + case["kv_heads"]) * 7 * dim}
    seen = [visible(case, n, k) for n, k in zip(new, kv)]
    read = 2 * sum(s for _, s in seen) * case["kv_heads"] * dim * e
    out = 2 * rows * case["heads"] * dim * e + (4 * rows * case["heads"] if case["lse"] else 0)
    return {"bytes": read + out + tables, "flops": 4 * dim * case["heads"] * sum(p for p, _ in seen)}


# ---- inputs ------------------------------------------------------------------------------
def generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def kept_indices(case, seed):
    """Kept tokens of each image, ascending, as the reduction returns them."""
    g = generator(seed)
    n = case["t"] * case["h"] * case["w"]
    order = torch.rand(case["images"], n, generator=g, device=DEV).argsort(1)[:, :case["kept"]]
    return order.sort(1)[0].to(torch.int32).flatten().contiguous()


def starts(case):
    """Where each image's positions begin: after the text and the images before it."""
    rng = random.Random(case["pick"])
    at, out = 0, []
    for _ in range(case["images"]):
        at += rng.randint(1, 64)
        out.append((at, at, at))
        at += max(case["t"], case["h"], case["w"])
    return out


def positions_in(case, g, tokens, first=None):
    """int32 [axes, tokens]: text and images in turn; on an image's tokens the axes differ."""
    axes = case["sections"].count(",") + 1
    base = torch.arange(tokens, device=DEV) if first is None else first
    side = torch.randint(0, 24, (axes, tokens), generator=g, device=DEV)
    image = (torch.arange(tokens, device=DEV) // 64) % 2
    return (base + side * image).to(torch.int32).contiguous()


def projected(case, g, tokens, kinds):
    """Outputs of a projection, [tokens, heads of its kind, head_dim] for each kind, slices of one tensor where packed."""
    dt, dim = torch_type(case), case["head_dim"]
    heads = [case["heads"] if kind == "q" else case["kv_heads"] for kind in kinds]
    if case.get("packed", True):
        all_ = (randn(g, tokens, sum(heads), dim) * torch.exp(0.3 * randn(g, 1, sum(heads), 1))).to(dt)
        return list(torch.split(all_, heads, dim=1))
    return [(randn(g, tokens, h, dim) * torch.exp(0.3 * randn(g, 1, h, 1))).to(dt) for h in heads]


def norm_weights(case, g):
    if not case["norm"]:
        return None, None
    return tuple((1.0 + 0.2 * randn(g, case["head_dim"])).to(torch_type(case)) for _ in range(2))


def rotate_inputs(case, seed):
    g = generator(seed)
    x = {"pos": positions_in(case, g, case["tokens"]) + case["start"]}
    x["q"], x["k"] = projected(case, g, case["tokens"], "qk")
    x["wq"], x["wk"] = norm_weights(case, g)
    if case["op"] == "rotate_backward":
        x["gq"], x["gk"] = (1e-2 * randn(g, *t.shape) for t in (x["q"], x["k"]))
        x["gq"], x["gk"] = (t.to(torch_type(case)) for t in (x["gq"], x["gk"]))
    return x


def cache_inputs(case, seed):
    g = generator(seed)
    new, kv = lengths(case)
    seqs, page, dim, total = case["seqs"], case["page"], case["head_dim"], sum(new)
    pages = pages_of(case)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    width = max(1, max((n + page - 1) // page for n in kv))
    counts = torch.tensor([(n + page - 1) // page for n in kv], device=DEV)
    table = torch.zeros(seqs, width, dtype=torch.int32, device=DEV)
    table[torch.arange(width, device=DEV)[None, :] < counts[:, None]] = order
    x = {"q_start": torch.tensor([sum(new[:b]) for b in range(seqs + 1)], dtype=torch.int32, device=DEV),
         "kv_len": torch.tensor(kv, dtype=torch.int32, device=DEV), "table": table}
    shape = (max(1, pages), page, case["kv_heads"], dim)
    # keys as normed and rotated, values as projected
    x["k_cache"], x["v_cache"] = (torch.empty(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for c in (x["k_cache"], x["v_cache"]):
        for part in c.split(max(1, (1 << 27) // (page * case["kv_heads"] * dim))):
            part.copy_(randn(g, *part.shape))
    if case["op"] == "append":
        x["q"], x["k"], x["v"] = projected(case, g, total, "qkv")
        x["wq"], x["wk"] = norm_weights(case, g)
        first = torch.cat([torch.arange(k - n, k, device=DEV) for n, k in zip(new, kv)])
        x["pos"] = positions_in(case, g, total, first)
    else:
        x["q"] = (1.5 * randn(g, total, case["heads"], dim)).to(torch.bfloat16)
    return x


def handle(case):
    import paper_2607_13500_amd as tr
    sections = [int(s) for s in case["sections"].split(",")]
    return tr.Attention(case["heads"], case["kv_heads"], case["head_dim"], torch_type(case), rot_dim=case["rot_dim"],
                        sections=sections, adjacent=case["adjacent"], norm=case["norm"], eps=EPS)


def frequencies(case, dtype):
    """Angle of each rotated pair at position 1, and the pair's axis."""
    pairs = case["rot_dim"] // 2
    i = torch.arange(pairs, dtype=torch.float64, device=DEV)
    axis = [a for a, n in enumerate(case["sections"].split(",")) for _ in range(int(n))]
    return (10000.0 ** (-i / pairs)).to(dtype), torch.tensor(axis, dtype=torch.long, device=DEV)


def prepare(case, seed):
    op = case["op"]
    if op == "positions":
        return {"case": case, "idx": kept_indices(case, seed), "K": [case["kept"]] * case["images"],
                "grid": [(case["t"], case["h"], case["w"])] * case["images"], "start": starts(case)}
    st = cache_inputs(case, seed) if op in ("append", "attend") else rotate_inputs(case, seed)
    st["case"] = case
    if own:
        st["attention"] = handle(case)
        if op in ("append", "attend"):
            import paper_2607_13500_amd as tr
            st["cache"], st["step"] = tr.KVCache(st["k_cache"], st["v_cache"]), tr.Step(st["q_start"], st["kv_len"], st["table"])
    else:
        st["freq"], st["axis"] = frequencies(case, torch.float32)
        if op in ("append", "attend"):
            st["new"], st["kv"] = lengths(case)
    return st


def run(st):
    case = st["case"]
    return run_own(case, st) if own else run_plain(case, st)


def run_own(case, st):
    op, a = case["op"], st.get("attention")
    if op == "positions":
        import paper_2607_13500_amd as tr
        return {"pos": tr.kept_positions(st["idx"], st["K"], st["grid"], st["start"])}
    if op == "rotate":
        q, k = a.rotate(st["q"], st["k"], st["pos"], wq=st["wq"], wk=st["wk"])
        return {"q": q, "k": k}
    if op == "rotate_backward":
        dq, dk, dwq, dwk = a.rotate_backward(st["gq"], st["gk"], st["q"], st["k"], st["pos"], wq=st["wq"], wk=st["wk"])
        return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk} if case["norm"] else {"dq": dq, "dk": dk}
    if op == "append":
        q = a.append(st["q"], st["k"], st["v"], st["pos"], st["cache"], st["step"], wq=st["wq"], wk=st["wk"])
        return {"q": q, "k_cache": st["cache"].k, "v_cache": st["cache"].v}
    out, lse = a.attend(st["q"], st["cache"], st["step"], causal=case["causal"], window=case["window"], want_lse=case["lse"])
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


# ---- the plain forms: elementary operations in 32 bits ------------------------------------
def halves(case, x):
    """The two elements of each rotated pair, and the elements that do not rotate."""
    r = case["rot_dim"]
    if case["adjacent"]:
        return x[..., 0:r:2], x[..., 1:r:2], x[..., r:]
    return x[..., :r // 2], x[..., r // 2:r], x[..., r:]


def joined(case, a, b, rest):
    if case["adjacent"]:
        return torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1)
    return torch.cat([a, b, rest], -1)


def turned(case, x, cos, sin):
    a, b, rest = halves(case, x)
    return joined(case, a * cos - b * sin, b * cos + a * sin, rest)


def angles(st):
    angle = st["pos"].float()[st["axis"]].t() * st["freq"]           # [tokens, pairs]
    return torch.cos(angle)[:, None, :], torch.sin(angle)[:, None, :]


def normed(x, w):
    x = x.float()
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()


def gradient_plain(case, g, x, w, cos, sin):
    g = turned(case, g.float(), cos, -sin)
    if w is None:
        return g, None
    x, w = x.float(), w.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    unit = x * r
    gw = g * w
    return r * (gw - unit * (gw * unit).mean(-1, keepdim=True)), (g * unit).sum((0, 1))


def attend_plain(case, st):
    q, dim, group = st["q"], case["head_dim"], case["heads"] // case["kv_heads"]
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[0], case["heads"], device=DEV) if case["lse"] else None
    t0 = 0
    for b, (n, kv) in enumerate(zip(st["new"], st["kv"])):
        if n == 0:
            continue
        pages = st["table"][b, :(kv + case["page"] - 1) // case["page"]].long()
        at = torch.arange(kv, device=DEV)
        for h in range(case["kv_heads"]):
            k, v = (st[c][pages, :, h].flatten(0, 1)[:kv].float() for c in ("k_cache", "v_cache"))
            for r0 in range(0, n, max(1, (1 << 29) // (kv * group))):
                r1 = min(n, r0 + max(1, (1 << 29) // (kv * group)))
                rows = q[t0 + r0:t0 + r1, h * group:(h + 1) * group].float().flatten(0, 1)
                s = rows @ k.t() * (1.0 / math.sqrt(dim))
                if case["causal"]:
                    i = (torch.arange(r0, r1, device=DEV) + (kv - n)).repeat_interleave(group)[:, None]
                    hide = at > i
                    if case["window"]:
                        hide |= at <= i - case["window"]
                    s.masked_fill_(hide, -math.inf)
                top = s.amax(1, keepdim=True)
                s = torch.exp(s.sub_(top))
                total = s.sum(1, keepdim=True)
                out[t0 + r0:t0 + r1, h * group:(h + 1) * group] = ((s @ v) / total).view(r1 - r0, group, dim).to(q.dtype)
                if lse is not None:
                    lse[t0 + r0:t0 + r1, h * group:(h + 1) * group] = (top + torch.log(total)).view(r1 - r0, group)
        t0 += n
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def run_plain(case, st):
    op = case["op"]
    if op == "positions":
        counts = torch.tensor(st["K"], device=DEV)
        grid, start = (torch.tensor(st[c], device=DEV).repeat_interleave(counts, 0, output_size=st["idx"].numel()) for c in ("grid", "start"))
        i, (_, h, w) = st["idx"].long(), grid.unbind(1)
        return {"pos": (torch.stack([i // (h * w), i // w % h, i % w]) + start.t()).to(torch.int32)}
    if op == "attend":
        return attend_plain(case, st)
    cos, sin = angles(st)
    dt = torch_type(case)
    if op == "rotate_backward":
        dq, dwq = gradient_plain(case, st["gq"], st["q"], st["wq"], cos, sin)
        dk, dwk = gradient_plain(case, st["gk"], st["k"], st["wk"], cos, sin)
        got = {"dq": dq.to(dt), "dk": dk.to(dt)}
        return {**got, "dwq": dwq, "dwk": dwk} if case["norm"] else got
    q, k = (turned(case, normed(st[x], st["w" + x]), cos, sin).to(dt) for x in "qk")
    if op == "rotate":
        return {"q": q, "k": k}
    page, slots = case["page"], []
    for b, (n, kv) in enumerate(zip(st["new"], st["kv"])):
        at = torch.arange(kv - n, kv, device=DEV)
        slots.append(st["table"][b].long()[at // page] * page + at % page)
    slots = torch.cat(slots)
    st["k_cache"].flatten(0, 1)[slots] = k
    st["v_cache"].flatten(0, 1)[slots] = st["v"]
    return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"]}


# ---- the same in 64 bits, from the definitions ---------------------------------------------
def rotation64(case, pos):
    """[tokens, pairs] complex numbers of modulus 1."""
    freq, axis = frequencies(case, torch.float64)
    angle = pos.double().t()[:, axis] * freq
    return torch.polar(torch.ones_like(angle), angle)


def rotate64(case, x, w, turn):
    if w is not None:
        x = x * w / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS)
    r = case["rot_dim"]
    pairs = x[..., :r].unflatten(-1, (r // 2, 2)) if case["adjacent"] else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None, :])
    z = z.flatten(-2) if case["adjacent"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, x[..., r:]], -1)


def slots64(case, x):
    """Rows of the flattened cache that each sequence's tokens lie in."""
    for b, kv in enumerate(lengths(case)[1]):
        j = torch.arange(kv, device=DEV)
        yield x["table"][b].long().gather(0, torch.div(j, case["page"], rounding_mode="floor")) * case["page"] + j.remainder(case["page"])


def attend64(case, x):
    new, _ = lengths(case)
    group = case["heads"] // case["kv_heads"]
    out = torch.zeros(x["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(x["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    t0 = 0
    for n, rows in zip(new, slots64(case, x)):
        kv = rows.numel()
        for head in range(case["heads"] if n else 0):
            k, v = (x[c].flatten(0, 1)[rows, head // group].double() for c in ("k_cache", "v_cache"))
            for r0 in range(0, n, 4096):
                r1 = min(n, r0 + 4096)
                s = torch.matmul(x["q"][t0 + r0:t0 + r1, head].double(), k.t().contiguous()) / math.sqrt(case["head_dim"])
                if case["causal"]:
                    late = torch.arange(kv, device=DEV)[None, :] - (torch.arange(r0, r1, device=DEV) + kv - n)[:, None]
                    s[(late > 0) if not case["window"] else (late > 0) | (late <= -case["window"])] = -math.inf
                total = torch.logsumexp(s, 1)
                lse[t0 + r0:t0 + r1, head] = total
                out[t0 + r0:t0 + r1, head] = torch.matmul(torch.exp(s - total[:, None]), v)
        t0 += n
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def exact(case, seed):
    op = case["op"]
    if op == "positions":
        return None                         # whole numbers
    if op == "attend":
        return attend64(case, cache_inputs(case, seed))
    x = cache_inputs(case, seed) if op == "append" else rotate_inputs(case, seed)
    turn = rotation64(case, x["pos"])
    wq, wk = (None if w is None else w.double().requires_grad_(op == "rotate_backward") for w in (x["wq"], x["wk"]))
    if op == "rotate_backward":
        got = {}
        for name, w in (("q", wq), ("k", wk)):
            v = x[name].double().requires_grad_(True)
            asked = [v] if w is None else [v, w]
            grads = torch.autograd.grad(rotate64(case, v, w, turn), asked, x["g" + name].double())
            got.update(zip(("d" + name, "dw" + name), grads))
        order = ("dq", "dk", "dwq", "dwk") if case["norm"] else ("dq", "dk")
        return {name: got[name] for name in order}
    q, k = rotate64(case, x["q"].double(), wq, turn), rotate64(case, x["k"].double(), wk, turn)
    if op == "rotate":
        return {"q": q, "k": k}
    k_cache, v_cache = x["k_cache"].double(), x["v_cache"].double()
    new, _ = lengths(case)
    rows = torch.cat([r[r.numel() - n:] for r, n in zip(slots64(case, x), new)])
    k_cache.flatten(0, 1).index_copy_(0, rows, k)
    v_cache.flatten(0, 1).index_copy_(0, rows, x["v"].double())
    return {"q": q, "k_cache": k_cache, "v_cache": v_cache}
