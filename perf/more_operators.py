"""Attention of many texts over one video, as cases that can be timed, with its plain forms.

Several questions about one video go on from the same cache: their rows of the page table begin with the same pages.  And a
model whose text looks at an encoder's states has them beside its own cache, in every layer, of another length than the text.

  groups  which neighbouring requests of a batch share how many tokens, found from the page table
  shared  attention of a block of new tokens (one, a verified chain, a draft tree, a whole question) over paged caches, the
          pages that a group of requests shares taken once for all of them
  cross   attention of texts of any length over encoders' states, every state visible or each query's own range of them

Head shapes are those of the workloads in ``paper_2508_16201_amd.synth`` (4/1, 14/2, 28/4, 40/8, 64/8), lengths too
(1254 kept rows of a pruned cache, 12544 of a video of 64 frames, 32768 of 128), and generic ones around them.
"""
import math
import random

import numpy as np
import torch

own = False

HEADS = ((4, 1, 64), (14, 2, 64), (28, 4, 128), (40, 8, 128), (64, 8, 128))
FRAME = 196        # states of a frame


# ------------------------------------------------------------------------------------------------- the cases
def shared(name, videos, batch, q_len, prefix, text, heads, page_size, lens, **more):
    """batch requests about `videos` videos of up to `prefix` tokens, each with up to `text` tokens of its own, then the block."""
    hq, hkv, d = heads
    case = {"name": name, "kind": "shared", "videos": videos, "batch": batch, "q_len": q_len, "prefix": prefix, "text": text, "hq": hq,
            "hkv": hkv, "d": d, "page_size": page_size, "lens": lens, "head_major": False, "tree": False, "ragged_q": False, "lse": False}
    case.update(more)
    return case


def groups(name, videos, batch, q_len, prefix, text, page_size, lens, min_tokens, **more):
    case = {"name": name, "kind": "groups", "videos": videos, "batch": batch, "q_len": q_len, "prefix": prefix, "text": text,
            "page_size": page_size, "lens": lens, "ragged_q": False, "min_tokens": min_tokens, "common": 0}
    case.update(more)
    return case


def cross(name, batch, q_len, states, heads, lens, **more):
    """batch encoders of up to `states` states, each looked at by up to `q_len` queries (lens 0: all as many)."""
    hq, hkv, d = heads
    case = {"name": name, "kind": "cross", "batch": batch, "q_len": q_len, "states": states, "hq": hq, "hkv": hkv, "d": d, "lens": lens,
            "head_major": False, "ranges": False, "back": 0, "lse": False}
    case.update(more)
    return case


def listed():
    return [
        # four questions about one video: the next token of the draft over its pruned cache, the shortest call of a step
        shared("shared-draft", 1, 4, 1, 1254, 256, (14, 2, 64), 16, 3),
        # sixteen questions about one video, their chain blocks verified
        shared("shared-verify", 1, 16, 6, 12544, 300, (64, 8, 128), 64, 5, head_major=True, lse=True),
        # a service with several videos of different lengths, each with its own questions
        shared("shared-videos", 5, 32, 4, 32768, 700, (40, 8, 128), 32, 7, lse=True),
        # a plain token for each of many viewers of one long stream
        shared("shared-stream", 1, 48, 1, 65536, 1000, (28, 4, 128), 16, 11),
        # draft trees of 26 nodes of eight requests about two videos
        shared("shared-tree", 2, 8, 26, 12544, 260, (64, 8, 128), 128, 13, tree=True),
        # eight questions arrive about a video that is in the cache: their prompts, of any length
        shared("shared-prompts", 1, 8, 256, 12544, 0, (28, 4, 128), 64, 17, ragged_q=True),
        # the plan of a small batch, made once in a step for all layers
        groups("groups-small", 2, 8, 6, 2000, 200, 16, 19, 256),
        # and of a large one: many videos behind one common instruction
        groups("groups-many", 30, 250, 1, 12544, 500, 16, 23, 512, common=96),
        # a step of eight dialogues, each with an encoder's states of its own
        cross("cross-token", 8, 1, 6272, (28, 4, 128), 29),
        # the next token of a small model over one video's pruned states
        cross("cross-small", 1, 1, 1254, (14, 2, 64), 0),
        # texts between the frames of a stream: a token sees the frames before it, the first ones none
        cross("cross-frames", 4, 600, 9800, (40, 8, 128), 31, ranges=True, back=30, lse=True),
        # long prompts, each over the whole of its video
        cross("cross-prompt", 2, 2048, 12544, (64, 8, 128), 0),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(("shared", "shared", "shared", "shared", "groups", "cross", "cross", "cross"))
    heads = rng.choice(HEADS)
    hq, hkv, d = heads
    page_size = rng.choice((16, 16, 32, 48, 64, 128, 256))
    lens = rng.randint(1, 1 << 20)
    pairs = 3_000_000_000 // hq              # queries times keys of a call
    if kind == "cross":
        what = rng.choice(("token", "text", "text", "ranges"))
        batch = log_int(rng, 1, 24)
        q_len = 1 if what == "token" else log_int(rng, 2, 4000 // batch)
        states = log_int(rng, 30, min(65536, pairs // (batch * q_len), (1 << 19) // batch))
        case = cross("", batch, q_len, states, heads, lens if rng.random() < 0.7 else 0, head_major=rng.random() < 0.5,
                     lse=rng.random() < 0.4)
        if what == "ranges":
            case.update(ranges=True, back=rng.choice((0, 0, 8, 40)))
    else:
        videos = log_int(rng, 1, 8)
        batch = videos + log_int(rng, 1, 40)
        ragged_q = rng.random() < 0.2
        tree = kind == "shared" and not ragged_q and rng.random() < 0.25
        q_len = log_int(rng, 10, 3000 // batch) if ragged_q else rng.randint(9, 40) if tree else rng.randint(1, 8)
        prefix = max(page_size, log_int(rng, 100, min(65536, pairs // (batch * q_len) // 2, (1 << 20) // batch)))
        text = rng.choice((0, log_int(rng, 1, 1500)))
        if kind == "shared":
            case = shared("", videos, batch, q_len, prefix, text, heads, page_size, lens, tree=tree, ragged_q=ragged_q,
                          head_major=rng.random() < 0.5, lse=rng.random() < 0.25)
        else:
            case = groups("", videos, batch, q_len, prefix, text, page_size, lens, rng.choice((1, 64, 512, 2000)),
                          ragged_q=ragged_q, common=rng.choice((0, 0, 40, 300)))
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------- sizes, which seeds of inputs leave
def requests(case):
    """Of every request: its video, the whole pages' tokens that it shares with that video's others, its length with the block,
    and the block's."""
    r, ps = random.Random(case["lens"]), case["page_size"]
    batch, videos = case["batch"], case["videos"]
    cuts = sorted(r.sample(range(1, batch), videos - 1))
    video = np.searchsorted(np.array(cuts, dtype=np.int64), np.arange(batch), side="right")
    prefix = [case["prefix"]] + [r.randint(max(1, case["prefix"] // 8), case["prefix"]) for _ in range(videos - 1)]
    whole = np.array([prefix[v] // ps * ps for v in video])
    q_len = np.array([max(1, r.randint(case["q_len"] // 3, case["q_len"])) if case["ragged_q"] else case["q_len"] for _ in range(batch)])
    kept = np.array([prefix[v] % ps + r.randint(case["text"] // 4, case["text"]) for v in video])
    return video, whole, whole + kept + q_len, q_len


def the_groups(video, whole):
    """int32 [3, batch]: each request's first neighbour of the same video, that one's number of them, the tokens they share."""
    batch = len(video)
    first = np.searchsorted(video, video)
    members = np.bincount(first, minlength=batch)
    alone = members[first] == 1
    return np.stack([first, members, np.where(alone, 0, whole)]).astype(np.int32)


def entries(case):
    """Of every encoder: how many queries look at it, and its states.  Some have none of one or the other."""
    r, batch = random.Random(case["lens"]), case["batch"]
    if not case["lens"]:
        return np.full(batch, case["q_len"]), np.full(batch, case["states"])
    q_len, states = np.full(batch, case["q_len"]), np.full(batch, case["states"])
    for b in range(1, batch):
        q_len[b] = r.randint(max(1, case["q_len"] // 4), case["q_len"])
        states[b] = 0 if r.random() < 0.05 else r.randint(max(1, case["states"] // 8), case["states"])
    return q_len, states


def visible_ranges(case):
    """int32 [queries, 2]: the states [from, to) that a query sees: those of the frames before it, the last `back` of them (0: all)."""
    r, out = random.Random(case["lens"] + 1), []
    for n, states in zip(*entries(case)):
        frames = -(-int(states) // FRAME)
        # the text lies in pieces behind some of the frames, a few words before the first
        seen = sorted(0 if r.random() < 0.05 else r.randint(0, frames) for _ in range(int(n)))
        out += [(max(0, f - case["back"]) * FRAME if case["back"] else 0, min(f * FRAME, int(states))) for f in seen]
    return np.array(out, dtype=np.int32).reshape(-1, 2)


def prefix_sums(n):
    return np.concatenate([[0], np.cumsum(n)])


def work(case):
    if case["kind"] == "cross":
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        q_len, states = entries(case)
        rows = int(q_len.sum()) * hq
        if case["ranges"]:
            at, ranges = prefix_sums(q_len), visible_ranges(case)
            pairs = int(np.maximum(ranges[:, 1] - ranges[:, 0], 0).sum())
            keys = 0
            for b in range(case["batch"]):
                mark = np.zeros(int(states[b]) + 1, dtype=np.int64)
                mine = ranges[at[b]:at[b + 1]]
                mine = mine[mine[:, 1] > mine[:, 0]]
                np.add.at(mark, mine[:, 0], 1)
                np.add.at(mark, mine[:, 1], -1)
                keys += int((np.cumsum(mark)[:-1] > 0).sum())
        else:
            pairs, keys = int((q_len * states).sum()), int(states[q_len > 0].sum())
        return {"bytes": 4 * keys * hkv * d + 4 * rows * d + 4 * case["lse"] * rows + 8 * case["ranges"] * int(q_len.sum()),
                "flops": 4 * pairs * hq * d}
    video, whole, lens, q_len = requests(case)
    if case["kind"] == "groups":
        # a row is read as far as it agrees with the one before it, and one entry on (nearly: inputs change a tenth of the rows)
        same = int(np.where(video[1:] == video[:-1], whole[1:] // case["page_size"], 0).sum())
        return {"bytes": 8 * (same + case["batch"]) + 20 * case["batch"], "flops": 0}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    first = np.searchsorted(video, video)
    keys = int((lens - whole).sum() + whole[first == np.arange(case["batch"])].sum())
    rows = int(q_len.sum()) * hq
    pairs = int((q_len * (lens - q_len)).sum() + (q_len * (q_len + 1) // 2).sum())
    return {"bytes": 4 * keys * hkv * d + 4 * rows * d + 4 * case["lse"] * rows + 4 * keys // case["page_size"], "flops": 4 * pairs * hq * d}


# ------------------------------------------------------------------------------------------------------ inputs
def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def ints(values):
    return torch.tensor(np.asarray(values, dtype=np.int32), device="cuda")


def normal(g, shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)


def prepare(case, seed):
    return {"shared": prepare_shared, "groups": prepare_groups, "cross": prepare_cross}[case["kind"]](case, seed)


def shared_table(case, seed):
    """int32 [batch, pages of the longest]: a video's whole pages in the rows of all its requests, then pages of their own, -1
    behind them; in no order.  common: tokens that all the videos begin with."""
    ps = case["page_size"]
    video, whole, lens, _ = requests(case)
    pages = -(-lens // ps)
    table = np.full((case["batch"], int(pages.max())), -1, dtype=np.int64)
    at, common = 0, case.get("common", 0) // ps
    starts = {}
    for b in range(case["batch"]):
        v, n = video[b], whole[b] // ps
        if v not in starts:
            starts[v] = at + common if not starts else at
            at = starts[v] + n
        table[b, :n] = starts[v] + np.arange(n)
        table[b, :min(common, n)] = np.arange(min(common, n))
        table[b, n:pages[b]] = at + np.arange(pages[b] - n)
        at += pages[b] - n
    ids = np.random.default_rng(seed).permutation(at)
    return np.where(table >= 0, ids[table], -1), at


def tree_masks(nodes, seed):
    """Ancestor masks of a tree whose node t hangs under an earlier one, at most four under each."""
    r, below = random.Random(seed), [0]
    masks = [1]
    for t in range(1, nodes):
        p = r.choice([n for n in range(t) if below[n] < 4])
        below[p] += 1
        below.append(0)
        masks.append(masks[p] | 1 << t)
    return [m - (1 << 64) if m >= 1 << 63 else m for m in masks]


def prepare_shared(case, seed):
    g = generator(seed)
    hq, hkv, d, ps = (case[x] for x in ("hq", "hkv", "d", "page_size"))
    video, whole, lens, q_len = requests(case)
    table, total = shared_table(case, seed)
    s = {"case": case, "scale": 1.0 / math.sqrt(d), "longest": int(lens.max()), "most_q": int(q_len.max()), "table": ints(table),
         "lens": ints(lens), "groups": ints(the_groups(video, whole)), "cu_q": ints(prefix_sums(q_len)) if case["ragged_q"] else None,
         "q_lens": ints(q_len), "masks": None}
    shape = (total, hkv, ps, d) if case["head_major"] else (total, ps, hkv, d)
    s["k"], s["v"] = (normal(g, shape).transpose(1, 2) if case["head_major"] else normal(g, shape) for _ in range(2))
    s["q"] = normal(g, (int(q_len.sum()), hq, d))
    # a few keys that a query looks for, as trained heads have them
    far = torch.randint(total, (4,), generator=g, device="cuda")
    s["k"][far, 0] = (s["k"][far, 0].float() * 3).to(torch.bfloat16)
    if case["tree"]:
        s["masks"] = torch.tensor(np.array([tree_masks(case["q_len"], seed + b) for b in range(case["batch"])], dtype=np.int64).reshape(-1),
                                  device="cuda")
    return s


def prepare_groups(case, seed):
    _, _, lens, q_len = requests(case)
    table, total = shared_table(case, seed)
    # a tenth of the dialogues were changed at some place: from there on their pages are their own
    r = np.random.default_rng(seed)
    for b in r.choice(case["batch"], max(1, case["batch"] // 10), replace=False):
        n = int((table[b] >= 0).sum())
        from_page = int(r.integers(0, n))
        table[b, from_page:n] = total + np.arange(n - from_page)
        total += n - from_page
    return {"case": case, "table": ints(table), "lens": ints(lens), "q_lens": ints(q_len), "n_pages": total,
            "cu_q": ints(prefix_sums(q_len)) if case["ragged_q"] else None}


def prepare_cross(case, seed):
    g = generator(seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    q_len, states = entries(case)
    many = case["batch"] > 1
    s = {"case": case, "scale": 1.0 / math.sqrt(d), "cu_q": ints(prefix_sums(q_len)) if many else None,
         "cu_kv": ints(prefix_sums(states)) if many else None, "ranges": ints(visible_ranges(case)) if case["ranges"] else None}
    n = int(states.sum())
    shape = (hkv, n, d) if case["head_major"] else (n, hkv, d)
    s["k"], s["v"] = (normal(g, shape).transpose(0, 1) if case["head_major"] else normal(g, shape) for _ in range(2))
    s["q"] = normal(g, (int(q_len.sum()), hq, d))
    far = torch.randint(n, (40,), generator=g, device="cuda")
    s["k"][far] = (s["k"][far].float() * 3).to(torch.bfloat16)
    # the lengths again, for the plain form's padding
    s["q_lens"], s["kv_lens"] = ints(q_len), ints(states)
    s["most_q"], s["most_kv"] = int(q_len.max()), int(states.max())
    return s


# ----------------------------------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if own:
        return {"shared": own_shared, "groups": own_groups, "cross": own_cross}[case["kind"]](s, case)
    return {"shared": plain_shared, "groups": plain_groups, "cross": plain_cross}[case["kind"]](s, case)


def own_shared(s, case):
    from paper_2508_16201_amd import binding as B
    return B.shared_attn(s["q"], s["k"], s["v"], s["table"], s["lens"], s["scale"], s["groups"], cu_q=s["cu_q"], max_q_len=s["most_q"],
                         max_kv_len=s["longest"], ancestor_mask=s["masks"], want_lse=case["lse"])


def own_groups(s, case):
    from paper_2508_16201_amd import binding as B
    return B.pages_shared(s["table"], s["lens"], s["n_pages"], case["page_size"], case["q_len"], cu_q=s["cu_q"], min_tokens=case["min_tokens"])


def own_cross(s, case):
    from paper_2508_16201_amd import binding as B
    return B.cross_attn(s["q"], s["k"], s["v"], s["scale"], cu_q=s["cu_q"], cu_kv=s["cu_kv"], key_ranges=s["ranges"], want_lse=case["lse"])


def padded_rows(q_lens, most):
    """[batch, most]: the row of the concatenated queries that each place holds (the last one again behind them), and whether
    it holds one."""
    n = q_lens.long()[:, None]
    t = torch.arange(most, device="cuda")[None]
    return n.cumsum(0) - n + torch.minimum(t, (n - 1).clamp(min=0)), t < n


def softmax_attention(q, k, v, visible, scale):
    """q [batch, queries, H_q, d], k, v [batch, keys, H_kv, d], visible [batch, queries or 1, keys], in 32 bits: the outputs, 0
    where nothing is visible, and the logarithms of the sums."""
    batch, queries, hq, d = q.shape
    keys, hkv = k.shape[1:3]
    q = q.float().view(batch, queries, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(batch, hkv, -1, d)
    logits = torch.matmul(q, k.float().permute(0, 2, 3, 1).contiguous()).mul_(scale).view(batch, hkv, hq // hkv, queries, keys)
    logits.masked_fill_(~visible[:, None, None], -math.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=-3e38)
    p = logits.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(batch, hkv, -1, keys), v.float().permute(0, 2, 1, 3).contiguous()).view(batch, hkv, hq // hkv, queries, d)
    o = torch.where(total > 0, o / total, 0.0)
    return o.permute(0, 3, 1, 2, 4).reshape(batch, queries, hq, d), (top + torch.log(total))[..., 0].permute(0, 3, 1, 2).reshape(batch, queries, hq)


def plain_shared(s, case):
    ps, most = case["page_size"], s["most_q"]
    rows, there = padded_rows(s["q_lens"], most)
    table = s["table"].long()
    keys = table.shape[1] * ps
    j = torch.arange(keys, device="cuda")
    context = (s["lens"] - s["q_lens"]).long()[:, None, None]                      # [batch, 1, 1]
    position = context + torch.arange(most, device="cuda")[None, :, None]          # [batch, most, 1]
    if s["masks"] is None:
        visible = j <= position
    else:
        in_block = (s["masks"].view(-1, most, 1) >> (j - context).clamp(0, 63)) & 1
        visible = (j < context) | ((j < context + most) & (in_block == 1))
    visible = visible & (table >= 0).repeat_interleave(ps, 1)[:, None]
    at = table.clamp(min=0)
    k, v = (x[at].reshape(len(at), keys, case["hkv"], case["d"]) for x in (s["k"], s["v"]))
    out, lse = softmax_attention(s["q"][rows], k, v, visible, s["scale"])
    out = out[there].to(torch.bfloat16)
    return (out, lse[there]) if case["lse"] else out


def plain_groups(s, case):
    table, ps, batch = s["table"].long(), case["page_size"], case["batch"]
    whole = (s["lens"] - s["q_lens"]).long() // ps                                  # pages before the block
    i = torch.arange(table.shape[1], device="cuda")
    zero = torch.zeros(1, dtype=torch.long, device="cuda")
    same = (table[1:] == table[:-1]) & (table[1:] >= 0) & (table[1:] < s["n_pages"]) & (i < torch.minimum(whole[1:], whole[:-1])[:, None])
    common = torch.cat([zero, same.long().cumprod(1).sum(1), zero])                 # with the request before; the last: none behind
    mine = common[:batch]
    around = torch.maximum(torch.cat([zero, mine[:-1]]), common[1:])
    linked = (mine > 0) & (mine * ps >= case["min_tokens"]) & (2 * mine >= around)
    b = torch.arange(batch, device="cuda")
    first = torch.where(linked, 0, b).cummax(0).values
    members = torch.zeros(batch, dtype=torch.long, device="cuda").scatter_add_(0, first, torch.ones_like(b))
    least = torch.full((batch,), table.shape[1], dtype=torch.long, device="cuda").scatter_reduce_(0, first, torch.where(linked, mine, table.shape[1]), "amin")
    tokens = torch.where(members[first] > 1, least[first] * ps, 0)
    return torch.stack([first, members, tokens]).to(torch.int32)


def plain_cross(s, case):
    rows, there = padded_rows(s["q_lens"], s["most_q"])
    at, _ = padded_rows(s["kv_lens"], s["most_kv"])
    j = torch.arange(s["most_kv"], device="cuda")[None, None]
    visible = j < s["kv_lens"].long()[:, None, None]
    if s["ranges"] is not None:
        mine = s["ranges"].long()[rows]
        visible = visible & (j >= mine[..., :1]) & (j < mine[..., 1:])
    at = at.clamp(max=len(s["k"]) - 1)
    out, lse = softmax_attention(s["q"][rows], s["k"][at], s["v"][at], visible, s["scale"])
    out = out[there].to(torch.bfloat16)
    return (out, lse[there]) if case["lse"] else out


# --------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"shared": exact_shared, "groups": exact_groups, "cross": exact_cross}[case["kind"]](s, case)


def exact_rows(s, rows, k, v, hidden, out, lse):
    """One request's rows [from, to) over its keys [n, heads, d], hidden [queries, n] or None."""
    hq, d = s["q"].shape[1:]
    hkv, n = k.shape[1], k.shape[0]
    for h in range(hkv):
        heads = slice(h * hq // hkv, (h + 1) * hq // hkv)
        q = s["q"][rows, heads].double()                                         # [queries, group, d]
        x = (q.reshape(-1, d) @ k[:, h].double().t().contiguous() * s["scale"]).view(q.shape[0], -1, n)
        if hidden is not None:
            x = x.masked_fill(hidden[:, None], -math.inf)
        z = torch.logsumexp(x, -1, keepdim=True)
        p = torch.where(z > -math.inf, torch.exp(x - z), 0.0)
        out[rows, heads] = (p.view(-1, n) @ v[:, h].double().contiguous()).view(q.shape)
        lse[rows, heads] = z[..., 0]


def exact_shared(s, case):
    ps = case["page_size"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    table, lens, q_lens = (s[x].cpu().numpy() for x in ("table", "lens", "q_lens"))
    masks = None if s["masks"] is None else s["masks"].cpu().numpy()
    begin = 0
    for b, (n, ql) in enumerate(zip(lens, q_lens)):
        j = np.arange(n)
        sees = np.ones((ql, n), dtype=bool)
        for t in range(ql):
            if masks is None:
                sees[t, n - ql + t + 1:] = False
            else:
                sees[t, n - ql:] = [(int(masks[begin + t]) >> x) & 1 for x in range(ql)]
        page, row = torch.from_numpy(table[b, j // ps].astype(np.int64)).cuda(), torch.from_numpy(j % ps).cuda()
        exact_rows(s, slice(begin, begin + ql), s["k"][page, row], s["v"][page, row], torch.from_numpy(~sees).cuda(), out, lse)
        begin += int(ql)
    return (out, lse) if case["lse"] else out


def exact_groups(s, case):
    ps, batch = case["page_size"], case["batch"]
    table, lens, q_lens = (s[x].cpu().numpy() for x in ("table", "lens", "q_lens"))
    common = [0] * (batch + 1)
    for b in range(1, batch):
        most = min((lens[b] - q_lens[b]) // ps, (lens[b - 1] - q_lens[b - 1]) // ps)
        while common[b] < most and 0 <= table[b, common[b]] == table[b - 1, common[b]] < s["n_pages"]:
            common[b] += 1
    answer = np.zeros((3, batch), dtype=np.int32)
    b = 0
    while b < batch:
        end, least = b + 1, None
        while end < batch and common[end] > 0 and common[end] * ps >= case["min_tokens"] and 2 * common[end] >= max(common[end - 1], common[end + 1]):
            least = common[end] if least is None else min(least, common[end])
            end += 1
        answer[0, b:end], answer[1, b], answer[2, b:end] = b, end - b, (least or 0) * ps
        b = end
    return torch.from_numpy(answer).cuda()


def exact_cross(s, case):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    q_len, states = entries(case)
    q_at, kv_at = prefix_sums(q_len), prefix_sums(states)
    for b in range(case["batch"]):
        rows, keys = slice(int(q_at[b]), int(q_at[b + 1])), slice(int(kv_at[b]), int(kv_at[b + 1]))
        if q_len[b] == 0 or states[b] == 0:
            continue
        hidden = None
        if s["ranges"] is not None:
            j, mine = torch.arange(int(states[b]), device="cuda"), s["ranges"][rows].long()
            hidden = (j[None] < mine[:, :1]) | (j[None] >= mine[:, 1:])
        exact_rows(s, rows, s["k"][keys], s["v"][keys], hidden, out, lse)
    return (out, lse) if case["lse"] else out
