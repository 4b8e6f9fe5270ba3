"""The operators of the paged 4-bit key/value cache, as cases that can be timed and compared.

  append     rotated keys and values of new tokens into the pages of their sequences, with the rotation of the queries
  attention  of the rows appended last (single tokens, candidate trees, prompt parts) over such a cache
  read       slots of the cache as values, every layer (export to a 16-bit cache, inspection)
  move       the accepted nodes of a tree to the slots behind their context, every layer

A cached vector x of head_dim numbers is held as codes 0..15 and two bf16 numbers: zero (the largest not above min x) and
scale (the smallest not below (max x - zero) / 15); it stands for zero + scale * code.

Heads and lengths are those of workloads/configs.py (32, 40 and 52 heads of 128, trees of 60 and 64 nodes, contexts of 512
to 2048, batches of 1 to 4) and, for grouped heads, batches and contexts beyond, generic.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
TINY = 2.0 ** -100
TREE = 64           # nodes behind the context of a sequence whose path is moved


def case(op, batch=1, context=512, context_min=0, rows=1, rows_min=0, heads=32, kv_heads=32, head_dim=128, page=64,
         dtype="bf16", tree=False, layers=1):
    """context: tokens that the longest sequence holds before the call, the others going down evenly to context_min; rows: the same of new rows."""
    return {"op": op, "batch": batch, "context": context, "context_min": context_min or context, "rows": rows,
            "rows_min": rows_min or rows, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page,
            "dtype": dtype, "tree": tree, "layers": layers}


def listed():
    out = []

    def add(name, *a, **kw):
        out.append({"name": name, **case(*a, **kw)})

    # one token of one sequence in plain decoding, 7B heads: a few microseconds, so launch and prologue count
    add("attn_decode_577", "attention", context=577, page=16)
    # one token for each of a ragged serving batch, grouped heads: the bytes of the cache are the time
    add("attn_decode_batch32", "attention", batch=32, context=8190, context_min=100, heads=32, kv_heads=8)
    # one token of one very long sequence: too few (sequence, head) pairs for the machine unless keys are split
    add("attn_decode_131071", "attention", context=131071, heads=64, kv_heads=8, page=128, dtype="fp16")
    # verification of a 60-node tree, one sequence, 7B heads, fp32 queries as the engine hands them over
    add("attn_tree60_fp32", "attention", context=1024, rows=60, tree=True, dtype="fp32")
    # verification of the benchmark's batch: 64-node trees of four ragged sequences, 40 heads
    add("attn_tree64_batch4", "attention", batch=4, context=2048, context_min=512, rows=64, heads=40, kv_heads=40, tree=True)
    # a part of a long prompt on top of what is cached: bound by arithmetic
    add("attn_prompt1024", "attention", context=4001, rows=1024, heads=32, kv_heads=8)
    # the new token of each sequence of a batch
    add("append_decode_batch16", "append", batch=16, context=3000, context_min=17, heads=32, kv_heads=8, page=16)
    # a whole prompt batch
    add("append_prompt_8192", "append", batch=4, context=5, rows=2048, heads=32, kv_heads=8)
    # one tree's rows read back, all layers of a small model with heads of 64
    add("read_tree64", "read", context=700, rows=64, heads=16, kv_heads=16, head_dim=64, layers=4, dtype="fp16", page=32)
    # a sequence exported to the 16-bit cache, all layers
    add("read_sequence_2047", "read", context=1, rows=2047, heads=40, kv_heads=40, layers=8)
    # an accepted path of five nodes, 7B heads and layers
    add("move_path5", "move", context=1024, rows=5, layers=32)
    # accepted paths of a large batch
    add("move_batch64", "move", batch=64, context=1000, context_min=40, rows=6, heads=32, kv_heads=8, layers=40, page=16)
    return out


def spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads, kv_heads = rng.choice([(32, 32), (40, 40), (32, 8), (64, 8), (52, 52), (16, 16), (16, 2), (24, 8), (8, 1), (12, 4)])
    common = {"heads": heads, "kv_heads": kv_heads, "head_dim": rng.choice([128, 128, 64]), "page": rng.choice([16, 32, 64, 128]),
              "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"])}
    op = rng.choice(["attention", "attention", "attention", "append", "read", "move"])
    if op == "attention":
        kind = rng.choice(["token", "token", "tree", "few", "prompt"])
        rows = {"token": 1, "tree": rng.randint(17, 128), "few": rng.randint(2, 16), "prompt": spread(rng, 20, 900)}[kind]
        most = (1 << 20) // kv_heads if kind in ("token", "few") else 330000 // heads if kind == "tree" else 4500      # tokens over the batch
        batch = spread(rng, 1, 32) if kind != "prompt" else spread(rng, 1, 3)
        context = spread(rng, 1, max(2, min(131071, most // batch)))
        return case(op, batch, context, spread(rng, 1, context), rows, rng.randint(max(1, rows // 2), rows), tree=kind == "tree", **common)
    if op == "append":
        batch = spread(rng, 1, 32)
        rows = spread(rng, 1, 8192 * 48 // (heads + 2 * kv_heads) // batch)
        return case(op, batch, spread(rng, 1, 4000), 1, rows, rng.randint(max(1, rows // 2), rows), **common)
    layers = spread(rng, 1, 32)
    batch = spread(rng, 1, 32)
    rows = spread(rng, 1, max(1, min(2000, 2047 * 40 * 8 // (kv_heads * layers * batch)))) if op == "read" else rng.randint(1, 8)
    context = spread(rng, 1, max(2, min(2000, 3000000 // (kv_heads * layers * batch))))
    return case(op, batch, context, 1, rows, max(1, rows // 2), layers=layers, **common)


def down(most, least, n):
    return [most - (most - least) * i // max(1, n - 1) for i in range(n)]


def lengths(c):
    """(tokens held before, new rows) of each sequence; for `read` the rows lie behind the context as well."""
    return down(c["context"], min(c["context_min"], c["context"]), c["batch"]), down(c["rows"], min(c["rows_min"], c["rows"]), c["batch"])


def tree_masks(rows, rs):
    """Ancestor sets (own node included) of one random tree a sequence, as two 64-bit words a row."""
    out = []
    for n in rows:
        sets = [1]
        for u in range(1, n):
            sets.append(sets[int(rs.randint(max(0, u - 12), u))] | 1 << u)
        out += [(s & (1 << 64) - 1, s >> 64) for s in sets]
    return np.array(out, dtype=np.uint64).view(np.int64)


def inputs(c, seed):
    """Everything that both the plain form and the 64-bit one are given."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 31))
    t = DTYPES[c["dtype"]]
    ctx, rows = lengths(c)
    B, hq, hk, dh, page = c["batch"], c["heads"], c["kv_heads"], c["head_dim"], c["page"]
    held = [a + (TREE if c["op"] == "move" else r) for a, r in zip(ctx, rows)]
    need = [-(-n // page) for n in held]        # pages of each sequence
    n_pages = sum(need) + 3
    order = rs.permutation(n_pages)
    table = np.full((B, max(need)), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    total = sum(rows)
    ints = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)
    normal = lambda *shape: torch.randn(*shape, generator=g, device=DEV)
    channel = torch.exp(0.4 * normal(1, hk, dh))         # keys have channels of different size
    s = {"table": ints(table), "ctx": ints(ctx), "row_start": ints(np.concatenate([[0], np.cumsum(rows)])),
         "n_pages": n_pages, "total": total, "max_rows": max(rows), "type": t}
    # where each row goes: sequence, slot, position
    seq = np.repeat(np.arange(B), rows)
    inner = np.concatenate([np.arange(r) for r in rows])
    s["seq"], s["inner"] = ints(seq).long(), ints(inner).long()
    slot = np.asarray(ctx)[seq] + inner
    s["slot"] = ints(slot).long()
    s["page_of"] = s["table"][s["seq"], s["slot"] // page].long()
    s["mask"] = torch.from_numpy(tree_masks(rows, rs)).to(DEV) if c["tree"] else None
    if c["op"] == "append":
        s["k"], s["v"], s["q"] = (channel * normal(total, hk, dh)).to(t), normal(total, hk, dh).to(t), normal(total, hq, dh).to(t)
        n_pos = max(a + r for a, r in zip(ctx, rows)) + 1
        angle = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-torch.arange(dh // 2, dtype=torch.float64, device=DEV) * 2 / dh)
        s["rope"] = torch.stack([angle.cos(), angle.sin()], dim=-1).float().contiguous()        # [position][dh/2][cos, sin]
        s["pos"] = s["slot"].int()
        return s
    # what the cache holds: every slot up to the last new row, in the order of (layer, sequence, slot)
    hseq = np.repeat(np.arange(B), held)
    hslot = np.concatenate([np.arange(n) for n in held])
    s["held_seq"], s["held_slot"], s["held_start"] = ints(hseq).long(), ints(hslot).long(), ints(np.concatenate([[0], np.cumsum(held)]))
    s["held_max"] = max(held)
    s["held_page"] = s["table"][s["held_seq"], s["held_slot"] // page].long()
    n = len(hseq)
    s["hk"] = [(channel * normal(n, hk, dh)).bfloat16() for _ in range(c["layers"])]
    s["hv"] = [normal(n, hk, dh).bfloat16() for _ in range(c["layers"])]
    if c["op"] == "attention":
        s["q"] = normal(total, hq, dh).to(t)
    if c["op"] == "move":
        # an accepted path in a tree behind the context: nodes behind the path's own length, so that the call can be repeated
        src, dst = np.full((B, c["rows"]), -1), np.full((B, c["rows"]), -1)
        for b, r in enumerate(rows):
            src[b, :r] = ctx[b] + r + np.sort(rs.permutation(TREE - r)[:r])
            dst[b, :r] = ctx[b] + np.arange(r)
        s["src"], s["dst"] = ints(src), ints(dst)
    return s


# ---------------------------------------------------------------------------------------------- the plain forms

def floor_bf16(x):
    """Largest bf16 not above x (fp32 in, fp32 out): the lower half of the word cut off is towards zero."""
    bits = x.view(torch.int32)
    cut = bits & -65536
    return torch.where((x < 0) & (cut != bits), cut + 65536, cut).view(torch.float32)


def quantise(x):
    """fp32 [..., dh] -> codes (uint8), zero and scale [..., 1] (fp32 that bf16 holds exactly)."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    zero = floor_bf16(lo)
    scale = -floor_bf16(-((hi - zero) / torch.full_like(hi, 15.0)))       # by a tensor: by a number torch multiplies by its rounded inverse
    bad = ~(torch.isfinite(scale) & torch.isfinite(x).all(-1, keepdim=True))
    flat = scale < TINY
    scale = torch.where(flat, torch.zeros_like(scale), scale)
    code = torch.round((x - zero) / torch.where(flat | bad, torch.ones_like(scale), scale)).clamp(0.0, 15.0)
    code = torch.where(flat | bad, torch.zeros_like(code), code)
    nan = torch.full_like(scale, float("nan"))
    return code.to(torch.uint8), torch.where(bad, nan, zero), torch.where(bad, nan, scale)


def rotate(x, cos, sin):
    """Pairs (i, i + dh/2) of [rows, heads, dh] turned, in fp32."""
    a, b = x.float().chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def values(store, page, at):
    """Slots (page, place in it) of a store as fp32."""
    code, zero, scale = store
    return zero[page, at] + scale[page, at] * code[page, at].float()


def store_of(c, n_pages):
    shape = (n_pages, c["page"], c["kv_heads"])
    return [torch.zeros(*shape, c["head_dim"], dtype=torch.uint8, device=DEV), torch.zeros(*shape, 1, device=DEV), torch.zeros(*shape, 1, device=DEV)]


def put(store, page, at, x):
    for part, new in zip(store, quantise(x)):
        part[page, at] = new


def plain_append(s):
    c = s["case"]
    at = s["slot"] % c["page"]
    cs = s["rope"][s["pos"].long()][:, None]
    cos, sin = cs[..., 0], cs[..., 1]
    q = rotate(s["q"], cos, sin).to(s["type"])
    put(s["K"][0], s["page_of"], at, rotate(s["k"], cos, sin))
    put(s["V"][0], s["page_of"], at, s["v"].float())
    return {"q": q, "k": values(s["K"][0], s["page_of"], at).bfloat16(), "v": values(s["V"][0], s["page_of"], at).bfloat16()}


def plain_attention(s):
    c = s["case"]
    B, hq, hk, dh, page, R = c["batch"], c["heads"], c["kv_heads"], c["head_dim"], c["page"], s["max_rows"]
    ctx, count = s["ctx"].long(), (s["row_start"][1:] - s["row_start"][:-1]).long()
    L = s["held_max"]
    slot = torch.arange(L, device=DEV)
    page_of = s["table"][:, slot // page].long().clamp(min=0)                     # [B, L]
    K = values(s["K"][0], page_of, (slot % page).expand(B, L)).permute(0, 2, 3, 1)      # [B, hk, dh, L]
    V = values(s["V"][0], page_of, (slot % page).expand(B, L)).permute(0, 2, 1, 3)      # [B, hk, L, dh]
    q = torch.zeros(B, R, hq, dh, device=DEV)
    q[s["seq"], s["inner"]] = s["q"].float()
    q = q.view(B, R, hk, hq // hk, dh).permute(0, 2, 1, 3, 4).reshape(B, hk, R * (hq // hk), dh)
    score = (q @ K).view(B, hk, R, hq // hk, L) * (1.0 / math.sqrt(dh))
    rel = slot[None, None, :] - ctx[:, None, None]                                 # [B, 1, L]
    if s["mask"] is not None:
        words = torch.zeros(B, R, 2, dtype=torch.int64, device=DEV)
        words[s["seq"], s["inner"]] = s["mask"]
        r = rel.clamp(0, 127).expand(B, R, L)
        word = torch.where(r < 64, words[..., :1], words[..., 1:])
        new = ((word >> (r % 64)) & 1).bool() & (rel < 128)
    else:
        new = rel <= torch.arange(R, device=DEV)[None, :, None]
    sees = ((rel < 0) | new) & (rel < count[:, None, None])
    score = torch.where(sees[:, None, :, None, :], score, torch.full_like(score, float("-inf")))
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    V = torch.where((rel[:, 0] < count[:, None])[:, None, :, None], V, torch.zeros_like(V))
    out = (p.view(B, hk, -1, L) @ V).view(B, hk, R, hq // hk, dh) / torch.where(total > 0, total, torch.ones_like(total))
    return out.permute(0, 2, 1, 3, 4).reshape(B, R, hq, dh)[s["seq"], s["inner"]].to(s["type"])



def layers_read(s):
    """The rows' slots in every layer."""
    at = s["slot"] % s["case"]["page"]
    return {name: (zero[:, s["page_of"], at] + scale[:, s["page_of"], at] * code[:, s["page_of"], at].float()).to(s["read_type"])
            for name, (code, zero, scale) in (("k", s["KL"]), ("v", s["VL"]))}


def plain_move(s):
    page = s["case"]["page"]
    b, i = torch.nonzero(s["dst"] >= 0, as_tuple=True)
    src, dst = s["src"][b, i].long(), s["dst"][b, i].long()
    sp, dp = s["table"][b, src // page].long(), s["table"][b, dst // page].long()
    for parts in (s["KL"], s["VL"]):
        for part in parts:
            part[:, dp, dst % page] = part[:, sp, src % page]
    return layers_read(s)


# ---------------------------------------------------------------------------------------------- the framework's calls

def own_cache(c, s):
    """The handle that a serving program keeps: the cache, filled, and the plan of the forward's rows."""
    from paper_2408_08146_b200 import PagedKV4
    cache = PagedKV4(c["layers"], c["kv_heads"], c["head_dim"], c["page"], s["n_pages"], device=DEV)
    if "hk" in s:
        before = cache.rows(s["table"], torch.zeros_like(s["ctx"]), row_start=s["held_start"], total=len(s["held_seq"]), max_rows=s["held_max"])
        for layer in range(c["layers"]):
            cache.append(layer, before, s["hk"][layer], s["hv"][layer])
    s["cache"] = cache
    s["rows"] = cache.rows(s["table"], s["ctx"], row_start=s["row_start"], total=s["total"], max_rows=s["max_rows"], mask=s["mask"])


def own_run(s):
    cache, rows, op = s["cache"], s["rows"], s["case"]["op"]
    if op == "append":
        cache.append(0, rows, s["k"], s["v"], rope=s["rope"], pos=s["pos"], q=s["q"], q_out=s["q_out"])
        cache.read(rows, layer=0, k_out=s["k_out"], v_out=s["v_out"])
        return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
    if op == "attention":
        return cache.attention(0, rows, s["q"], out=s["out"])
    if op == "move":
        cache.move(s["table"], s["src"], s["dst"])
    cache.read(rows, k_out=s["k_out"], v_out=s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


# ---------------------------------------------------------------------------------------------- what is measured

def prepare(c, seed):
    s = inputs(c, seed)
    s["case"] = c
    s["read_type"] = torch.float16 if c["dtype"] == "fp16" and c["op"] in ("read", "move") else torch.bfloat16
    if own:
        own_cache(c, s)
        if c["op"] == "attention":
            s["out"] = torch.empty_like(s["q"])
        else:
            shape = (s["total"], c["kv_heads"], c["head_dim"])
            shape = shape if c["op"] == "append" else (c["layers"],) + shape
            s["k_out"], s["v_out"] = (torch.empty(shape, dtype=s["read_type"], device=DEV) for _ in range(2))
            s["q_out"] = torch.empty_like(s["q"]) if "q" in s else None
    else:
        s["K"], s["V"] = ([store_of(c, s["n_pages"]) for _ in range(c["layers"])] for _ in range(2))
        if "hk" in s:
            for layer in range(c["layers"]):
                at = s["held_slot"] % c["page"]
                put(s["K"][layer], s["held_page"], at, s["hk"][layer].float())
                put(s["V"][layer], s["held_page"], at, s["hv"][layer].float())
        if c["op"] in ("read", "move"):         # every layer side by side
            s["KL"], s["VL"] = ([torch.stack(p) for p in zip(*s.pop(n))] for n in ("K", "V"))
    s.pop("hk", None)
    s.pop("hv", None)
    return s


def run(s):
    if own:
        return own_run(s)
    return {"append": plain_append, "attention": plain_attention, "read": layers_read, "move": plain_move}[s["case"]["op"]](s)


def work(c):
    ctx, rows = lengths(c)
    hq, hk, dh, total = c["heads"], c["kv_heads"], c["head_dim"], sum(rows)
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[c["dtype"]]
    vector = dh // 2 + 4                         # bytes of one cached key or value of one head
    if c["op"] == "append":                      # q in and out, k, v in; cache written and read; values out
        return {"bytes": total * dh * size * (2 * hq + 2 * hk) + 4 * total * hk * vector + total * hk * dh * 4 + total * dh * 4,
                "flops": total * dh * (3 * (hq + hk) + 8 * hk)}
    if c["op"] == "attention":
        held = sum(a + r for a, r in zip(ctx, rows))
        pairs = sum(r * a + (r * 4 if c["tree"] else r * (r + 1) // 2) for a, r in zip(ctx, rows))
        return {"bytes": held * hk * 2 * vector + 2 * total * hq * dh * size + (16 * total if c["tree"] else 0), "flops": 4 * dh * hq * pairs}
    read = c["layers"] * total * hk * (2 * vector + 2 * dh * 2)
    if c["op"] == "read":
        return {"bytes": read, "flops": c["layers"] * total * hk * dh * 4}
    return {"bytes": read + 2 * c["layers"] * total * hk * 2 * vector, "flops": c["layers"] * total * hk * dh * 4}


# ---------------------------------------------------------------------------------------------- from the definition, in 64 bits

def grid(x, up):
    """x (64 bits) to the bf16 next to it: the smallest not below (up) or the largest not above."""
    near = x.float().bfloat16()
    away = near.double() < x if up else near.double() > x
    step = torch.nextafter(near, torch.full_like(near, float("inf") if up else float("-inf")))
    return torch.where(away, step, near).double()


def held_as(x):
    """What a vector stands for once it is appended (64 bits in and out)."""
    low = grid(x.min(dim=-1, keepdim=True).values, False)
    step = grid((x.max(dim=-1, keepdim=True).values - low) / 15, True)
    some = step >= TINY
    n = torch.where(some, ((x - low) / torch.where(some, step, torch.ones_like(step))).round().clip(0, 15), torch.zeros_like(x))
    return torch.addcmul(low, n, torch.where(some, step, torch.zeros_like(step)))


def held(x):
    """What the cache that is given to `attention`, `read` and `move` stands for: its codes and two numbers a vector are those of prepare()."""
    code, zero, scale = (part.double() for part in quantise(x.float()))
    return torch.addcmul(zero, scale, code)


def exact(c, seed):
    s = inputs(c, seed)
    ctx, rows = lengths(c)
    hq, hk, dh = c["heads"], c["kv_heads"], c["head_dim"]
    if c["op"] == "append":
        turn = torch.view_as_complex(s["rope"].double().contiguous())[s["pos"].long()].unsqueeze(1)
        def turned(x):
            z = torch.complex(x[..., :dh // 2].double(), x[..., dh // 2:].double()) * turn
            return torch.cat([z.real, z.imag], dim=-1)
        return {"q": turned(s["q"]), "k": held_as(turned(s["k"])), "v": held_as(s["v"].double())}
    ends = s["held_start"].tolist()
    if c["op"] == "attention":
        out = []
        first = s["row_start"].tolist()
        for b in range(c["batch"]):
            n, r = ends[b + 1] - ends[b], rows[b]
            q = s["q"][first[b]:first[b + 1]].double()
            bits = torch.ones(r, n, dtype=torch.bool, device=DEV)
            if s["mask"] is None:
                bits = torch.tril(bits, diagonal=n - r)
            else:
                words = s["mask"][first[b]:first[b + 1]].cpu().numpy().view(np.uint8).reshape(r, 16)
                bits[:, n - r:] = torch.from_numpy(np.unpackbits(words, axis=1, bitorder="little")[:, :r].astype(bool)).to(DEV)
            hidden = torch.zeros(r, n, dtype=torch.float64, device=DEV).masked_fill(~bits, -math.inf)
            k, v = (held(s[w][0][ends[b]:ends[b + 1]]) for w in ("hk", "hv"))
            heads = []
            for h in range(hq):
                w = torch.softmax(q[:, h] @ k[:, h * hk // hq].T / dh ** 0.5 + hidden, dim=-1)
                heads.append(w @ v[:, h * hk // hq])
            out.append(torch.stack(heads, dim=1))
        return torch.cat(out)
    got = {}
    for name, parts in (("k", s["hk"]), ("v", s["hv"])):
        full = torch.stack([held(x) for x in parts])
        if c["op"] == "move":
            src, dst, old = s["src"].tolist(), s["dst"].tolist(), full.clone()
            for b in range(c["batch"]):
                for i, j in zip(src[b], dst[b]):
                    if j >= 0:
                        full[:, ends[b] + j] = old[:, ends[b] + i]
        got[name] = torch.cat([full[:, ends[b] + ctx[b]:ends[b] + ctx[b] + rows[b]] for b in range(c["batch"])], dim=1)
    return got
