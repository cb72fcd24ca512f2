"""The operators of a paged KV cache, as cases that can be timed, with their plain forms.

A program that serves several requests keeps their caches in pages: pools ``[pages, page_size, heads, d]``, and for every
request a row of a table that names its pages in order.  A decode step over them is

  attn    attention of the block of new tokens over the pages: one token, a verified chain or a draft tree, with every
          key visible or only the first few and a window of the last
  rope    the new tokens' queries and keys turned to their positions, keys and values written to their pages
  assign  which pages every request holds in the next step: forked, grown, cut short or freed
  copy    rows moved between pages in all layers: a tree's accepted nodes, a draft's pruned cache, the page in which a fork
          goes on on its own

Head shapes are those of the workloads in ``paper_2508_16201_amd.synth`` (4/1, 14/2, 28/4, 40/8, 64/8), lengths too
(1511 keys of a pruned cache, 12806 of a video of 64 frames, 33030 of 128), and generic ones around them.
"""
import math
import random

import numpy as np
import torch

own = False

HEADS = ((4, 1, 64), (14, 2, 64), (28, 4, 128), (40, 8, 128), (64, 8, 128))


# ------------------------------------------------------------------------------------------------- the cases
def attn(name, batch, q_len, kv_len, heads, page_size, **more):
    hq, hkv, d = heads
    case = {"name": name, "kind": "attn", "batch": batch, "q_len": q_len, "kv_len": kv_len, "hq": hq, "hkv": hkv, "d": d,
            "page_size": page_size, "head_major": False, "tree": False, "window": 0, "sinks": 0, "lse": False, "lens": 0}
    case.update(more)
    return case


def rope(name, batch, q_len, kv_len, heads, page_size, **more):
    hq, hkv, d = heads
    case = {"name": name, "kind": "rope", "batch": batch, "q_len": q_len, "kv_len": kv_len, "hq": hq, "hkv": hkv, "d": d,
            "page_size": page_size, "head_major": False, "rot": d, "interleaved": False, "base": 1e6, "factor": 1.0,
            "positions": False, "lens": 0}
    case.update(more)
    return case


def assign(name, batch, kv_len, page_size, n_pages, fork, lens):
    return {"name": name, "kind": "assign", "batch": batch, "kv_len": kv_len, "page_size": page_size, "n_pages": n_pages,
            "fork": fork, "lens": lens}


def copy(name, what, layers, batch, kv_len, hkv, d, page_size, rows, lens, **more):
    case = {"name": name, "kind": "copy", "what": what, "layers": layers, "batch": batch, "kv_len": kv_len, "hkv": hkv,
            "d": d, "page_size": page_size, "rows": rows, "head_major": False, "lens": lens}
    case.update(more)
    return case


def listed():
    return [
        # the draft's next token over its pruned cache: the shortest call of a step, made for every layer and drafted token
        attn("attn-draft", 1, 1, 1511, (14, 2, 64), 16),
        # the verification of a chain block over one 72B-shaped request
        attn("attn-verify", 1, 6, 12806, (64, 8, 128), 64, head_major=True, lse=True),
        # eight requests of very different lengths, up to the longest context, in one call of a serving loop
        attn("attn-serve", 8, 6, 131072, (64, 8, 128), 32, lens=3),
        # streams that go on for ever: four first tokens and a window stay visible, the pages between have been freed
        attn("attn-window", 12, 4, 65000, (40, 8, 128), 16, window=4096, sinks=4, lens=5),
        # draft trees of 26 nodes of four requests: 208 query rows a kv head
        attn("attn-tree", 4, 26, 12826, (64, 8, 128), 128, tree=True, lens=7),
        # the block of a verification, eight requests
        rope("rope-verify", 8, 6, 12806, (64, 8, 128), 64, lens=11),
        # a part of a long prompt, at far positions that are scaled to the trained context
        rope("rope-prompt", 1, 8190, 131072, (28, 4, 128), 16, factor=4.0),
        # eight requests grow by the next block
        assign("assign-grow", 8, 2000, 16, 4096, False, 13),
        # beams or samples: every row goes on from one of another row's prefixes
        assign("assign-fork", 250, 7000, 16, 65536, True, 17),
        # the accepted path of each request's tree moves to the front of its block, in every layer
        copy("copy-accepted", "accepted", 28, 8, 2000, 4, 128, 16, 26, 19),
        # the draft's cache: 10 % of the video's rows, then the text, from the verifier's pages to the draft's
        copy("copy-pruned", "pruned", 80, 1, 12544, 8, 128, 64, 1254, 23),
        # the last page of every fork, which two rows cannot both write
        copy("copy-forked", "forked", 28, 32, 1000, 4, 128, 64, 63, 29),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attn", "attn", "attn", "attn", "rope", "rope", "assign", "copy", "copy"))
    heads = rng.choice(HEADS)
    hq, hkv, d = heads
    page_size = rng.choice((16, 16, 32, 48, 64, 128, 256))
    lens = rng.randint(1, 1 << 20)
    if kind == "attn":
        what = rng.choice(("one", "chain", "chain", "window", "tree"))
        batch = log_int(rng, 1, 16 if what == "tree" else 48)
        kv_len = log_int(rng, 40, min(30000, 50000 // batch) if what == "tree" else min(131072, (1 << 19) // batch))
        q_len = 1 if what == "one" else rng.randint(9, 40) if what == "tree" else rng.randint(1, 8)
        case = attn("", batch, q_len, max(kv_len, q_len), heads, page_size, head_major=rng.random() < 0.5,
                    tree=what == "tree", lse=rng.random() < 0.25, lens=lens)
        if what == "window":
            case.update(window=log_int(rng, 100, 9000), sinks=rng.choice((0, 1, 4, 17, 64)))
    elif kind == "rope":
        batch = log_int(rng, 1, 32)
        q_len = rng.randint(1, 30) if rng.random() < 0.5 else log_int(rng, 30, 8192 // batch)
        case = rope("", batch, q_len, q_len + log_int(rng, 1, 1000000), heads, page_size, head_major=rng.random() < 0.5,
                    rot=rng.choice((d, d, d // 2, d // 4)), interleaved=rng.random() < 0.5,
                    base=rng.choice((1e4, 5e5, 1e6)), factor=rng.choice((1.0, 1.0, 4.0, 32.0)),
                    positions=rng.random() < 0.5, lens=lens)
    elif kind == "assign":
        batch = log_int(rng, 1, 256)
        kv_len = log_int(rng, 20, min(100000, 65536 * page_size // batch // 3))
        pages = batch * (2 * (kv_len // page_size) + 4)
        case = assign("", batch, kv_len, page_size, min(65536, pages + rng.randint(0, 1000)), rng.random() < 0.5, lens)
    else:
        what = rng.choice(("accepted", "pruned", "forked"))
        layers = rng.choice((16, 24, 28, 64, 80))
        batch = log_int(rng, 1, 8 if what == "pruned" else 48)
        kv_len = log_int(rng, 100, 12000)
        kv_len = max(64, min(kv_len, int(4e9 / (4 * layers * batch * hkv * d))))
        rows = {"accepted": rng.randint(6, 40), "pruned": max(1, kv_len * rng.choice((10, 25, 50)) // 100),
                "forked": page_size - 1}[what]
        case = copy("", what, layers, batch, kv_len, hkv, d, page_size, rows, lens, head_major=rng.random() < 0.5)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------- sizes, work
def lengths(case, longest, least):
    """The requests' own lengths: all the same, or (lens: a seed) spread over an eighth of the longest and up."""
    if not case["lens"]:
        return [longest] * case["batch"]
    r = random.Random(case["lens"])
    return [longest] + [max(least, r.randint(max(1, longest // 8), longest)) for _ in range(case["batch"] - 1)]


def first_seen(case, kv_len):
    """The first key behind the sinks that the block's first query sees."""
    return max(0, kv_len - case["q_len"] - case["window"] + 1) if case["window"] else 0


def seen_keys(case, kv_len):
    at = first_seen(case, kv_len)
    return kv_len - at + min(case["sinks"], at)


def accepted_path(r, nodes):
    """Nodes of an accepted path, lowest first, none of which lies where another one moves to."""
    n = r.randint(1, max(1, min(5, nodes // 3)))
    return sorted(r.sample(range(n + 1, nodes), n))


def copied_rows(case):
    """Rows that each request copies."""
    r = random.Random(case["lens"])
    if case["what"] == "accepted":
        return [len(accepted_path(r, case["rows"])) for _ in range(case["batch"])]
    if case["what"] == "forked":
        return [r.randint(1, case["rows"]) for _ in range(case["batch"])]
    return [case["rows"]] * case["batch"]


TEXT = 256  # rows behind the video that a pruned cache keeps


def work(case):
    batch = case["batch"]
    if case["kind"] == "attn":
        hq, hkv, d, q_len = case["hq"], case["hkv"], case["d"], case["q_len"]
        keys = sum(seen_keys(case, n) for n in lengths(case, case["kv_len"], q_len))
        rows = batch * q_len * hq
        return {"bytes": 4 * keys * hkv * d + 4 * rows * d + 4 * case["lse"] * rows + 4 * keys // case["page_size"],
                "flops": 4 * keys * q_len * hq * d}
    if case["kind"] == "rope":
        tokens = batch * case["q_len"]
        return {"bytes": 4 * tokens * (case["hq"] + 2 * case["hkv"]) * case["d"] + 4 * tokens * case["positions"], "flops": 0}
    if case["kind"] == "assign":
        r = assign_inputs(case, 1)
        entries = sum(-(-int(n) // case["page_size"]) for n in np.concatenate([r["keep"], r["new"]]))
        return {"bytes": 4 * entries + 4 * case["n_pages"] + 24 * batch, "flops": 0}
    rows = sum(copied_rows(case)) + (TEXT * batch if case["what"] == "pruned" else 0)
    return {"bytes": 8 * case["layers"] * rows * case["hkv"] * case["d"], "flops": 0}


# ------------------------------------------------------------------------------------------------------ inputs
def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def ints(values):
    return torch.tensor(np.asarray(values, dtype=np.int32), device="cuda")


def pool(g, lead, pages, case):
    """bf16 [*lead, pages, page_size, heads, d] of unit variance, tokens or heads outermost in a page."""
    ps, h, d = case["page_size"], case["hkv"], case["d"]
    if not case["head_major"]:
        return torch.randn((*lead, pages, ps, h, d), generator=g, device="cuda", dtype=torch.bfloat16)
    return torch.randn((*lead, pages, h, ps, d), generator=g, device="cuda", dtype=torch.bfloat16).transpose(-3, -2)


def tables(seed, held, width):
    """int32 [len(held), width]: request b holds the pages at the places held[b] lists, in no order; -1 elsewhere."""
    table = np.full((len(held), width), -1, dtype=np.int32)
    total = sum(len(h) for h in held)
    ids = np.random.default_rng(seed).permutation(total).astype(np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, h] = ids[at:at + len(h)]
        at += len(h)
    return table, total


def prepare(case, seed):
    return {"attn": prepare_attn, "rope": prepare_rope, "assign": prepare_assign, "copy": prepare_copy}[case["kind"]](
        case, seed)


def tree_masks(nodes, seed):
    """Ancestor masks of a tree whose node t hangs under an earlier one, at most four under each."""
    r, parent, below = random.Random(seed), [0], [0]
    masks = [1]
    for t in range(1, nodes):
        p = r.choice([n for n in range(t) if below[n] < 4])
        below[p] += 1
        below.append(0)
        parent.append(p)
        masks.append(masks[p] | 1 << t)
    return [m - (1 << 64) if m >= 1 << 63 else m for m in masks]


def prepare_attn(case, seed):
    g = generator(seed)
    batch, q_len, hq, d, ps = (case[x] for x in ("batch", "q_len", "hq", "d", "page_size"))
    lens = lengths(case, case["kv_len"], q_len)
    held = []
    for n in lens:
        at = first_seen(case, n)
        pages = np.arange(-(-n // ps))
        held.append(pages[((pages + 1) * ps > at) | (pages * ps < case["sinks"])])
    table, total = tables(seed, held, -(-max(lens) // ps))
    s = {"case": case, "scale": 1.0 / math.sqrt(d), "longest": max(lens), "table": ints(table), "lens": ints(lens)}
    s["k"], s["v"] = (pool(g, (), total, case) for _ in range(2))
    s["q"] = torch.randn((batch * q_len, hq, d), generator=g, device="cuda", dtype=torch.bfloat16)
    # a few keys that a query looks for, as trained heads have them
    far = torch.randint(total, (4,), generator=g, device="cuda")
    s["k"][far, 0] = (s["k"][far, 0].float() * 3).to(torch.bfloat16)
    s["masks"] = None
    if case["tree"]:
        s["masks"] = torch.tensor(np.array([tree_masks(q_len, seed + b) for b in range(batch)], dtype=np.int64).reshape(-1),
                                  device="cuda")
    return s


def frequencies(case):
    """The angle a position of each pair, in 64 bits: base^(-2i/rot); with a factor, those that turn less than once over
    the trained context divided by it, those that turn 32 times left as they are, by parts between."""
    f = case["base"] ** (-2.0 * np.arange(case["rot"] // 2, dtype=np.float64) / case["rot"])
    if case["factor"] == 1.0:
        return f, 1.0
    turns = 32768 * f / (2 * math.pi)
    keep = np.clip((turns - 1) / (32 - 1), 0, 1)
    return f * (keep + (1 - keep) / case["factor"]), 0.1 * math.log(case["factor"]) + 1


def prepare_rope(case, seed):
    g = generator(seed)
    batch, q_len, hq, hkv, d, ps = (case[x] for x in ("batch", "q_len", "hq", "hkv", "d", "page_size"))
    lens = lengths(case, case["kv_len"], q_len)
    # (pages before the new tokens are not touched: the pool has those that are)
    held = [np.arange((n - q_len) // ps, -(-n // ps)) for n in lens]
    table, total = tables(seed, held, -(-max(lens) // ps))
    freq, magnitude = frequencies(case)
    s = {"case": case, "table": ints(table), "lens": ints(lens), "magnitude": magnitude, "positions": None}
    s["freq"] = torch.tensor(freq, device="cuda")
    # the same in turns, as 64-bit fractions
    s["turns"] = torch.tensor([int(x / (2 * math.pi) * 2.0 ** 64) for x in freq], device="cuda")
    s["k_pages"], s["v_pages"] = (pool(g, (), total, case) for _ in range(2))
    s["q"], s["k"], s["v"] = (torch.randn((batch * q_len, h, d), generator=g, device="cuda", dtype=torch.bfloat16)
                              for h in (hq, hkv, hkv))
    s["q_out"] = torch.empty_like(s["q"])
    if case["positions"]:
        s["positions"] = torch.randint(1 << 20, (batch * q_len,), generator=g, device="cuda", dtype=torch.int32)
    return s


def assign_inputs(case, seed):
    """The table before, and for every row of the next one the row it goes on from, how much of it, and its new length."""
    batch, ps = case["batch"], case["page_size"]
    r = np.random.default_rng([case["lens"], seed])
    longest = max(lengths(case, case["kv_len"], 1))
    lens = np.array(lengths(case, case["kv_len"], 1))
    held = [np.arange(-(-n // ps)) for n in lens]
    width = -(-(longest + 64) // ps)
    table, total = tables(seed, held, width)
    # the pages held lie anywhere in the pool
    where = r.permutation(max(case["n_pages"], total))[:total].astype(np.int32)
    table = np.where(table >= 0, where[table], -1)
    parent = r.integers(0, batch, batch) if case["fork"] else np.arange(batch)
    keep = lens[parent].copy()
    if case["fork"]:
        cut = r.random(batch) < 0.25           # some go back, some end and leave their row
        keep[cut] = r.integers(0, keep[cut] + 1)
    new = keep + r.integers(1, 9, batch)
    if case["fork"]:
        new[r.random(batch) < 0.05] = 0
        keep = np.minimum(keep, new)
    return {"table": table, "parent": parent, "keep": keep, "new": new}


def prepare_assign(case, seed):
    r = assign_inputs(case, seed)
    return {"case": case, **{k: ints(v) for k, v in r.items()}}


def prepare_copy(case, seed):
    g = generator(seed)
    r = random.Random(case["lens"])
    layers, batch, ps, rows, what = (case[x] for x in ("layers", "batch", "page_size", "rows", "what"))
    n = copied_rows(case)
    s = {"case": case, "n": ints(n), "src_row": None, "idx": None, "most": max(n)}
    if what == "accepted":
        # contexts of any length, the tree's block behind each: node i's row is row context + i
        lens = lengths(case, case["kv_len"], 1)
        table, total = tables(seed, [np.arange(-(-(m + rows) // ps)) for m in lens], -(-(max(lens) + rows) // ps))
        s["src"] = s["dst"] = (pool(g, (layers,), total, case), pool(g, (layers,), total, case))
        s["src_table"] = s["dst_table"] = ints(table)
        paths = [accepted_path(r, rows) for _ in range(batch)]
        s["idx"] = ints([p + [-1] * (rows - len(p)) for p in paths])
        s["src_start"], s["dst_start"] = ints(lens), ints([m + 1 for m in lens])
    elif what == "pruned":
        table, total = tables(seed, [np.arange(-(-(case["kv_len"] + TEXT) // ps))] * batch, -(-(case["kv_len"] + TEXT) // ps))
        s["src"] = (pool(g, (layers,), total, case), pool(g, (layers,), total, case))
        s["src_table"] = ints(table)
        table, total = tables(seed + 1, [np.arange(-(-(rows + TEXT) // ps))] * batch, -(-(rows + TEXT) // ps))
        s["dst"] = (pool(g, (layers,), total, case).zero_(), pool(g, (layers,), total, case).zero_())
        s["dst_table"] = ints(table)
        order = torch.rand((batch, case["kv_len"]), generator=g, device="cuda").argsort(1)[:, :rows]
        s["idx"] = order.sort(1).values.to(torch.int32)
        s["src_start"], s["dst_start"] = ints([0] * batch), ints([0] * batch)
        s["text_n"], s["text_src"], s["text_dst"] = (ints([m] * batch) for m in (TEXT, case["kv_len"], rows))
    else:
        # row b of the next table goes on from row src_row[b] of the last: the same whole pages, a page of its own behind them
        whole = case["kv_len"] // ps
        table, total = tables(seed, [np.arange(whole + 1)] * batch, whole + 2)
        parent = np.array([r.randrange(batch) for _ in range(batch)])
        after = table[parent]
        after[:, whole] = total + np.arange(batch)
        s["src"] = s["dst"] = (pool(g, (layers,), total + batch, case), pool(g, (layers,), total + batch, case))
        s["src_table"], s["dst_table"], s["src_row"] = ints(table), ints(after), ints(parent)
        s["src_start"] = s["dst_start"] = ints([whole * ps] * batch)
    return s


# ----------------------------------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if own:
        return {"attn": own_attn, "rope": own_rope, "assign": own_assign, "copy": own_copy}[case["kind"]](s, case)
    return {"attn": plain_attn, "rope": plain_rope, "assign": plain_assign, "copy": plain_copy}[case["kind"]](s, case)


def own_attn(s, case):
    from paper_2508_16201_amd import binding as B
    return B.paged_attn(s["q"], s["k"], s["v"], s["table"], s["lens"], s["scale"], max_kv_len=s["longest"],
                        window=case["window"], n_sinks=case["sinks"], ancestor_mask=s["masks"], want_lse=case["lse"])


def own_rope(s, case):
    from paper_2508_16201_amd import binding as B
    B.rope_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["lens"], q=s["q"], q_out=s["q_out"],
                  turns=s["turns"], interleaved=case["interleaved"], magnitude=s["magnitude"], positions=s["positions"])
    return s["q_out"], s["k_pages"], s["v_pages"]


def own_assign(s, case):
    from paper_2508_16201_amd import binding as B
    return B.pages_assign(s["table"], s["parent"], s["keep"], s["new"], case["n_pages"], case["page_size"])


def own_copy(s, case):
    from paper_2508_16201_amd import binding as B
    B.pages_copy(*s["src"], s["src_table"], *s["dst"], s["dst_table"], s["n"], s["most"], src_row=s["src_row"],
                 src_start=s["src_start"], dst_start=s["dst_start"], row_idx=s["idx"])
    if case["what"] == "pruned":
        B.pages_copy(*s["src"], s["src_table"], *s["dst"], s["dst_table"], s["text_n"], TEXT, src_start=s["text_src"],
                     dst_start=s["text_dst"])
    return s["dst"]


def plain_attn(s, case):
    batch, q_len, hq, hkv, d, ps = (case[x] for x in ("batch", "q_len", "hq", "hkv", "d", "page_size"))
    table = s["table"].long()
    keys = table.shape[1] * ps
    j = torch.arange(keys, device="cuda")
    t = torch.arange(q_len, device="cuda")
    context = (s["lens"].long() - q_len)[:, None, None]                          # [batch, 1, 1]
    position = context + t[None, :, None]                                        # [batch, q_len, 1]
    if s["masks"] is None:
        visible = j <= position
    else:
        bit = (j - context).clamp(0, 63)
        in_block = (s["masks"].view(batch, q_len, 1) >> bit) & 1
        visible = (j < context) | ((j < context + q_len) & (in_block == 1))
    if case["window"]:
        visible = visible & ((j > position - case["window"]) | (j < case["sinks"]))
    visible = visible & (table >= 0).repeat_interleave(ps, 1)[:, None]
    at = table.clamp(min=0)
    k = s["k"][at].float().reshape(batch, keys, hkv, d).permute(0, 2, 3, 1)          # [batch, heads, d, keys]
    q = s["q"].float().view(batch, q_len, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(batch, hkv, -1, d)
    logits = (torch.matmul(q, k) * s["scale"]).view(batch, hkv, hq // hkv, q_len, keys)
    del k
    logits = logits.masked_fill(~visible[:, None, None], -math.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(logits - top)
    del logits
    total = p.sum(-1, keepdim=True)
    v = s["v"][at].float().reshape(batch, keys, hkv, d).permute(0, 2, 1, 3)
    o = torch.matmul(p.view(batch, hkv, -1, keys), v).view(batch, hkv, hq // hkv, q_len, d) / total
    out = o.permute(0, 3, 1, 2, 4).reshape(batch * q_len, hq, d).to(torch.bfloat16)
    if not case["lse"]:
        return out
    lse = (top + torch.log(total)).view(batch, hkv, hq // hkv, q_len)
    return out, lse.permute(0, 3, 1, 2).reshape(batch * q_len, hq)


def turned(x, cos, sin, case):
    """[tokens, heads, d] with its first `rot` columns turned, in 32 bits, rounded once."""
    x, rot = x.float(), case["rot"]
    cos, sin = cos[:, None], sin[:, None]
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        new = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        new = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((new, x[..., rot:]), -1).to(torch.bfloat16)


def plain_rope(s, case):
    q_len, ps = case["q_len"], case["page_size"]
    at = ((s["lens"].long() - q_len)[:, None] + torch.arange(q_len, device="cuda")).view(-1)
    angle = (at if s["positions"] is None else s["positions"]).double()[:, None] * s["freq"]
    cos, sin = ((f(angle) * s["magnitude"]).float() for f in (torch.cos, torch.sin))
    request = torch.arange(case["batch"], device="cuda").repeat_interleave(q_len)
    page, row = s["table"].long()[request, at // ps], at % ps
    s["q_out"].copy_(turned(s["q"], cos, sin, case))
    s["k_pages"][page, row] = turned(s["k"], cos, sin, case)
    s["v_pages"][page, row] = s["v"]
    return s["q_out"], s["k_pages"], s["v_pages"]


def plain_assign(s, case):
    ps, n_pages, batch = case["page_size"], case["n_pages"], case["batch"]
    table, width = s["table"].long(), s["table"].shape[1]
    keep, new = s["keep"].long(), s["new"].long()
    i = torch.arange(width, device="cuda")[None]
    b = torch.arange(batch, device="cuda")[:, None].expand(batch, width)
    old = table[s["parent"].long().clamp(min=0)]
    old = torch.where((old >= 0) & (old < n_pages) & (i < -(-keep // ps)[:, None]), old, -1)
    written = (i == (keep // ps)[:, None]) & (keep % ps > 0)[:, None]             # the page that a row goes on in
    # the first row that holds a page to go on in, and none where one holds it as a whole page; one place more for "none"
    place = torch.where(old >= 0, old, n_pages).view(-1)
    counts = torch.zeros(n_pages + 1, dtype=torch.long, device="cuda").scatter_add_(0, place, torch.ones_like(place))
    first = torch.full((n_pages + 1,), batch, dtype=torch.long, device="cuda")
    first.scatter_reduce_(0, place, torch.where(written, b, -1).reshape(-1), "amin")
    leaves = written & (old >= 0) & (first[place].view(batch, width) != b)        # goes on in a page of its own
    counts.scatter_add_(0, place, -leaves.view(-1).long())
    wanted = (i < -(-new // ps)[:, None]) & ((i >= -(-keep // ps)[:, None]) | leaves | (written & (old < 0)))
    # the lowest free pages, to the lowest rows
    free = counts[:n_pages] == 0
    rank = torch.where(free, free.cumsum(0) - 1, n_pages)
    by_rank = torch.full((n_pages + 1,), -1, dtype=torch.long, device="cuda").scatter_(0, rank, torch.arange(n_pages, device="cuda"))
    by_rank[n_pages] = -1
    need = wanted.sum(1)
    fits = (need == 0) | (need.cumsum(0) <= free.sum())
    order = (wanted.view(-1).cumsum(0) - 1).view(batch, width)
    given = torch.where(wanted & fits[:, None], by_rank[order.clamp(0, n_pages)], -1)
    after = torch.where(wanted, given, torch.where(leaves, -1, old))
    counts.scatter_add_(0, torch.where(given >= 0, given, n_pages).view(-1), torch.ones_like(place))
    moved = leaves.any(1) & fits
    status = torch.where(fits, 0, -5)
    answers = after, torch.where(moved, keep // ps * ps, 0), torch.where(moved, keep % ps, 0), counts[:n_pages], status
    return tuple(x.to(torch.int32) for x in answers)


def plain_rows(s, n, most, src_start, dst_start, idx):
    """The rows of one copy, read in every layer, then written."""
    ps = s["case"]["page_size"]
    # (behind a request's last row that one again: the same value to the same place)
    i = torch.minimum(torch.arange(most, device="cuda")[None], n.long()[:, None] - 1)
    src = src_start.long()[:, None] + (i if idx is None else idx.long().gather(1, i))
    dst = dst_start.long()[:, None] + i
    from_table = s["src_table"].long() if s["src_row"] is None else s["src_table"].long()[s["src_row"].long()]
    src_page, dst_page = from_table.gather(1, src // ps), s["dst_table"].long().gather(1, dst // ps)
    s["dst"][0][:, dst_page, dst % ps] = s["src"][0][:, src_page, src % ps]
    s["dst"][1][:, dst_page, dst % ps] = s["src"][1][:, src_page, src % ps]


def plain_copy(s, case):
    plain_rows(s, s["n"], s["most"], s["src_start"], s["dst_start"], s["idx"])
    if case["what"] == "pruned":
        plain_rows(s, s["text_n"], TEXT, s["text_src"], s["text_dst"], None)
    return s["dst"]


# --------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": exact_attn, "rope": exact_rope, "assign": exact_assign, "copy": exact_copy}[case["kind"]](s, case)


def exact_attn(s, case):
    batch, q_len, hq, hkv, d, ps = (case[x] for x in ("batch", "q_len", "hq", "hkv", "d", "page_size"))
    out = torch.empty((batch * q_len, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((batch * q_len, hq), dtype=torch.float64, device="cuda")
    table, lens = s["table"].cpu().numpy(), s["lens"].cpu().numpy()
    masks = None if s["masks"] is None else s["masks"].cpu().numpy().reshape(batch, q_len)
    for b in range(batch):
        n = int(lens[b])
        j = np.arange(n)
        j = j[table[b, j // ps] >= 0]
        sees = np.zeros((q_len, len(j)), dtype=bool)
        for t in range(q_len):
            p = n - q_len + t
            sees[t] = j < n - q_len
            in_block = j >= n - q_len
            if masks is None:
                sees[t, in_block] = j[in_block] <= p
            else:
                sees[t, in_block] = [(int(masks[b, t]) >> int(x - (n - q_len))) & 1 for x in j[in_block]]
            if case["window"]:
                sees[t] &= (p - j < case["window"]) | (j < case["sinks"])
        some = sees.any(0)
        j, hidden = j[some], torch.from_numpy(~sees[:, some]).cuda()
        page, row = torch.from_numpy(table[b, j // ps].astype(np.int64)).cuda(), torch.from_numpy(j % ps).cuda()
        k, v = s["k"][page, row].double(), s["v"][page, row].double()             # [keys, heads, d]
        for h in range(hkv):
            heads = slice(h * hq // hkv, (h + 1) * hq // hkv)
            rows = slice(b * q_len, (b + 1) * q_len)
            q = s["q"][rows, heads].double()                                     # [q_len, group, d]
            x = (q.reshape(-1, d) @ k[:, h].t().contiguous() * s["scale"]).view(q_len, -1, len(j))
            x = x.masked_fill(hidden[:, None], -math.inf)
            z = torch.logsumexp(x, -1, keepdim=True)
            out[rows, heads] = (torch.exp(x - z).view(-1, len(j)) @ v[:, h].contiguous()).view(q_len, -1, d)
            lse[rows, heads] = z[..., 0]
    return (out, lse) if case["lse"] else out


def exact_rope(s, case):
    q_len, ps, rot = case["q_len"], case["page_size"], case["rot"]
    freq, magnitude = frequencies(case)
    lens, table = s["lens"].cpu().numpy().astype(np.int64), s["table"].cpu().numpy().astype(np.int64)
    at = np.concatenate([np.arange(n - q_len, n) for n in lens])
    page = np.concatenate([table[b][np.arange(n - q_len, n) // ps] for b, n in enumerate(lens)])
    position = at if s["positions"] is None else s["positions"].cpu().numpy().astype(np.int64)
    z = torch.from_numpy(magnitude * np.exp(1j * np.outer(position, freq))).cuda()[:, None]
    new = []
    for x in (s["q"], s["k"]):
        x = x.double()
        pairs = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
        w = torch.complex(x[..., pairs[0]], x[..., pairs[1]]) * z
        y = x.clone()
        y[..., pairs[0]], y[..., pairs[1]] = w.real, w.imag
        new.append(y)
    k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
    page, row = torch.from_numpy(page).cuda(), torch.from_numpy(at % ps).cuda()
    k_pages[page, row], v_pages[page, row] = new[1], s["v"].double()
    return new[0], k_pages, v_pages


def exact_assign(s, case):
    ps, n_pages = case["page_size"], case["n_pages"]
    table, parent, keep, new = (s[x].cpu().numpy() for x in ("table", "parent", "keep", "new"))
    after, start, count = np.full_like(table, -1), np.zeros_like(keep), np.zeros_like(keep)
    refs, status = np.zeros(n_pages, dtype=np.int32), np.zeros_like(keep)
    whole, going_on = np.zeros(n_pages, dtype=bool), {}
    for b in range(len(parent)):
        n = keep[b] // ps
        after[b, :n] = table[parent[b], :n]
        whole[after[b, :n]] = True
        np.add.at(refs, after[b, :n], 1)
        if keep[b] % ps:
            going_on.setdefault(int(table[parent[b], n]), []).append(b)
    left = []
    for page, rows in going_on.items():
        if not whole[page]:
            refs[page] += 1
            after[rows[0], keep[rows[0]] // ps] = page
            rows = rows[1:]
        left += rows
    free = [int(p) for p in np.flatnonzero(refs == 0)]
    at = 0
    for b in range(len(parent)):
        first = keep[b] // ps if b in left else -(-keep[b] // ps)
        need = max(0, -(-new[b] // ps) - first)
        if need and at + need > len(free):
            status[b] = -5
        elif need:
            after[b, first:first + need] = free[at:at + need]
            refs[free[at:at + need]] = 1
            if b in left:
                start[b], count[b] = first * ps, keep[b] % ps
        at += need
    return after, start, count, refs, status


def exact_copy(s, case):
    ps = case["page_size"]
    new = tuple(x.clone() for x in s["dst"])
    moves = [(s["n"], s["src_start"], s["dst_start"], s["idx"])]
    if case["what"] == "pruned":
        moves.append((s["text_n"], s["text_src"], s["text_dst"], None))
    for n, src_start, dst_start, idx in moves:
        for b in range(case["batch"]):
            i = torch.arange(int(n[b]), device="cuda")
            src = int(src_start[b]) + (i if idx is None else idx[b, :len(i)].long())
            dst = int(dst_start[b]) + i
            row = b if s["src_row"] is None else int(s["src_row"][b])
            for x, y in zip(s["src"], new):
                y[:, s["dst_table"][b].long()[dst // ps], dst % ps] = x[:, s["src_table"][row].long()[src // ps], src % ps]
    return new
