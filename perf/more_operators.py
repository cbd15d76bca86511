"""Performance cases of the paged KV cache: its operators, timed and checked one pass at
a time.

The cache holds the keys and values of many sequences in pages of a common pool (bf16, a
page of a layer laid out as one layer of the single-sequence cache with the page as its
capacity); a table gives every sequence's pages in order, an array its committed slots.
A call serves all sequences at once, each with its own count of new rows (the nodes of
its draft tree, one row without a draft, a prompt's rows):

  append  new queries and keys are rotated, keys and values written to their slots
  attend  attention of the new rows over their sequences' slots, scores capped or not
  mass    the weights that counted rows gave are added up, slot by slot
  commit  accepted tree rows move up behind the committed ones, in all layers
  evict   a sequence over its budget keeps its last slots and the heaviest others

The plain forms below are elementary torch operations on the same buffers, all sequences
padded to the longest.  Shapes are those of perf/cases.py (tiny, 7B, 13B) and generic
ones with grouped heads.
"""
import math
import random

import numpy as np
import torch

own = False

TILE = 32
TINY = dict(heads=4, group=1, hd=64)
SEVEN = dict(heads=32, group=1, hd=128)
THIRTEEN = dict(heads=40, group=1, hd=128)
GROUPED = dict(heads=8, group=4, hd=128)
MOST_BYTES, MOST_FLOPS = 3e9, 1.2e11
PLAIN, LINEAR, TURNS, LOG_TURNS = range(4)


def listed():
    return [
        # two short chats, one token each: nothing but latency
        dict(name="attend-tiny-2x64", kind="attend", dtype="f32", **TINY, page=32, seqs=2, len=64, n=1, cap=0.0),
        # a batch of conversations of all lengths, decoding without a draft
        dict(name="attend-gqa-48x4100", kind="attend", dtype="bf16", **GROUPED, page=64, seqs=48, len=4100, n=1, cap=0.0),
        # the benchmark's step for eight sequences: draft trees behind ragged contexts
        dict(name="attend-13b-8x1037-m16", kind="attend", dtype="f32", **THIRTEEN, page=128, seqs=8, len=1037, n=16,
             cap=0.0),
        # one very long document, many query heads to a KV head, capped scores
        dict(name="attend-gqa-1x130001-cap", kind="attend", dtype="bf16", heads=8, group=8, hd=128, page=256, seqs=1,
             len=130001, n=1, cap=30.0),
        # a layer's new rows of a decoding batch
        dict(name="append-13b-64x1", kind="append", dtype="f32", **THIRTEEN, page=128, seqs=64, len=1037, n=1, rot=128,
             interleaved=False, scaling=PLAIN),
        # the prompts of four new requests, scaled positions in a part of the head
        dict(name="append-gqa-4x1531", kind="append", dtype="bf16", **GROUPED, page=64, seqs=4, len=0, n=1531, rot=96,
             interleaved=True, scaling=TURNS),
        # weights of a decoding batch, on their way to an eviction
        dict(name="mass-gqa-16x4100", kind="mass", dtype="bf16", **GROUPED, page=64, seqs=16, len=4100, n=1, cap=0.0),
        # the accepted nodes of a tree over a long context
        dict(name="mass-7b-2x8191-m16", kind="mass", dtype="f32", **SEVEN, page=128, seqs=2, len=8191, n=16, cap=50.0),
        # the end of an ordinary round of eight sequences, whole model
        dict(name="commit-13b-8x5", kind="commit", layers=40, **THIRTEEN, page=128, seqs=8, len=1037, n=16, path=5),
        # wide trees of which much is accepted
        dict(name="commit-7b-16x38", kind="commit", layers=32, **SEVEN, page=64, seqs=16, len=540, n=64, path=38),
        # one conversation at its budget, some layers
        dict(name="evict-7b-1x2049", kind="evict", layers=4, **SEVEN, page=128, seqs=1, len=2049, budget=1024, recent=32),
        # a batch with ragged lengths, of which some are still below the budget
        dict(name="evict-gqa-16x4500", kind="evict", layers=8, **GROUPED, page=64, seqs=16, len=4500, budget=1500,
             recent=256),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choices(["attend", "append", "mass", "commit", "evict"], [5, 2, 2, 2, 2])[0]
        c = dict(kind=kind, dtype=rng.choice(["f32", "bf16"]), hd=rng.choice([64, 128, 128]),
                 page=rng.choice([32, 64, 96, 128, 256]), heads=_log_int(rng, 1, 40),
                 group=rng.choice([1, 1, 2, 3, 4, 8, 16]), seqs=_log_int(rng, 1, 96), cap=0.0)
        if kind in ("attend", "mass"):
            c.update(len=rng.choice([0] + 5 * [_log_int(rng, 1, 130000)]), n=rng.choice([1, _log_int(rng, 2, 64)]),
                     cap=rng.choice([0.0, 0.0, 20.0, 50.0]))
        elif kind == "append":
            c.update(len=rng.choice([0, _log_int(rng, 1, 20000)]), n=rng.choice([1, _log_int(rng, 2, 64),
                                                                                 _log_int(rng, 65, 3000)]),
                     rot=rng.choice([c["hd"], c["hd"], 32, c["hd"] - 16, 2]), interleaved=rng.random() < 0.5,
                     scaling=rng.randrange(4))
        else:
            c.update(layers=_log_int(rng, 1, 40), len=_log_int(rng, 2, 9000))
            if kind == "commit":
                c["n"] = _log_int(rng, 2, 64)
                c["path"] = rng.randint(1, c["n"])
            else:
                c["budget"] = rng.randint(1, c["len"])
                c["recent"] = rng.randint(0, c["budget"])
        w = work(c)
        # (the second: the plain forms pad every sequence to the longest)
        padded = c["seqs"] * (c["len"] + c.get("n", 0)) * c["heads"] * c.get("layers", 1)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS and padded * c["hd"] <= 1.1e9 \
                and padded * c["group"] * (c["n"] if kind in ("attend", "mass") else 1) <= 8e8:
            return c


def _ragged(most, count):
    """count numbers spread over (most / 20, most], the first the largest; 0 stays 0."""
    return [int(round(most * (1 - 0.95 * (i * 0.6180339887 % 1)))) for i in range(count)]


def _lens(c):
    return _ragged(c["len"], c["seqs"])


def _counts(c):
    """New rows of every sequence."""
    return [max(1, n) for n in _ragged(c["n"], c["seqs"])]


def work(c):
    """Bytes: bf16 keys and values, fp32 masses, queries and outputs in their type, each
    number that the result needs once.  Flops: the products of scores and outputs."""
    lens, slot = _lens(c), 2 * c["heads"] * c["hd"]  # bytes of K's slot, or V's
    if c["kind"] in ("attend", "mass"):
        counts = _counts(c)
        slots = sum(l + n for l, n in zip(lens, counts))
        q = sum(counts) * c["heads"] * c["group"] * c["hd"]
        stats = 8 * sum(counts) * c["heads"] * c["group"]
        products = 2 * c["heads"] * c["group"] * c["hd"] * sum(n * (l + n) for l, n in zip(lens, counts))
        size = 4 if c["dtype"] == "f32" else 2
        if c["kind"] == "attend":
            return dict(bytes=2 * slot * slots + 2 * size * q + stats, flops=2 * products)
        return dict(bytes=(slot + 8 * c["heads"]) * slots + size * q + stats, flops=products)
    if c["kind"] == "append":
        rows, size = sum(_counts(c)), 4 if c["dtype"] == "f32" else 2
        q, kv = rows * c["heads"] * c["group"] * c["hd"], rows * c["heads"] * c["hd"]
        return dict(bytes=2 * size * q + 2 * kv * (size + 2) + 4 * rows * c["heads"], flops=3 * (q + kv))
    layer = c["layers"] * (2 * slot + 4 * c["heads"])  # a slot's bytes in all layers
    if c["kind"] == "commit":
        return dict(bytes=2 * layer * sum(min(c["path"], n) for n in _counts(c)), flops=0)
    over = [l for l in lens if l > c["budget"]]
    return dict(bytes=2 * layer * c["budget"] * len(over) + 4 * c["heads"] * c["layers"] * sum(over), flops=0)


# ---------------------------------------------------------------------------
# inputs


def _tree_masks(rng, n):
    """Per node of a random tree the bits of the nodes on its root path, as signed numbers."""
    masks = []
    for i in range(n):
        m = (masks[rng.randrange(max(0, i - 12), i)] if i else 0) | 1 << i
        masks.append(m)
    return masks


def _signed(bits):
    return [b - (1 << 64) if b >> 63 else b for b in bits]


def _frequencies(c):
    """Radians per position of every pair: base 10000; scaled: a context of 4096 stretched by 8."""
    out = []
    for i in range(c["rot"] // 2):
        f = 10000.0 ** (-2.0 * i / c["rot"])
        if c["scaling"] == LINEAR:
            f /= 8.0
        elif c["scaling"] != PLAIN:
            turns = 4096 * f / (2 * math.pi)
            w = (turns - 1) / (4 - 1) if c["scaling"] == TURNS else math.log(turns / 1) / math.log(32 / 1)
            w = min(1.0, max(0.0, w))
            f *= w + (1 - w) / 8.0
        out.append(f)
    return out


def _magnitude(c):
    return 0.1 * math.log(8.0) + 1 if c["scaling"] == LOG_TURNS else 1.0


def prepare(case, seed):
    c, rng = case, random.Random(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    nl, nh, hd, page, ns = c.get("layers", 2), c["heads"], c["hd"], c["page"], c["seqs"]
    lens, counts = _lens(c), _counts(c) if "n" in c else [0] * c["seqs"]

    def normal(shape, dtype, std=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    def numbers(x, dtype=torch.int32):
        return torch.tensor(x, dtype=dtype, device="cuda")

    # every sequence's pages, in a random order over the pool; entries behind them are -1
    need = [(l + n + page - 1) // page for l, n in zip(lens, counts)]
    n_pages, width = sum(need) + 3, max(need)
    order = rng.sample(range(n_pages), sum(need))
    table = [[order.pop() for _ in range(k)] + [-1] * (width - k) for k in need]
    s = dict(case=c, lens_host=lens, counts_host=counts, table=numbers(table), lens=numbers(lens),
             k=normal((nl, n_pages, nh, page, hd), torch.bfloat16),
             v=normal((nl, n_pages, nh, page // TILE, hd, TILE), torch.bfloat16),
             new_lens=torch.zeros(ns, dtype=torch.int32, device="cuda"))
    # (weights gathered over a conversation: most slots little, a few nearly all)
    s["mass"] = normal((nl, n_pages, nh, page), torch.float32, 3.0 if c["kind"] == "evict" else 1.0).exp_()
    if c["kind"] == "mass":
        s["mass"] /= c["len"] + c["n"]  # the first few rounds' weights
    if c["kind"] in ("commit", "evict"):
        if c["kind"] == "commit":
            paths = [[0] + sorted(rng.sample(range(1, n), min(c["path"], n) - 1)) for n in counts]
            s["path"] = numbers([p + [0] * (c["path"] - len(p)) for p in paths])
            s["path_len"] = numbers([len(p) for p in paths])
        else:
            s["mass"][:, :, :, 5::7] = 0  # slots that nothing looked at: ties
        return s
    rows, dtype = sum(counts), torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    starts = [sum(counts[:i]) for i in range(ns + 1)]
    s["start"] = None if c["n"] == 1 else numbers(starts)
    if c["kind"] == "append":
        # (rows of one projection's output: queries, keys and values behind one another)
        s["qkv"] = normal((rows, (c["group"] + 2) * nh, hd), dtype)
        s["positions"] = numbers([l + i for l, n in zip(lens, counts) for i in range(n)])
        s["freq"] = numbers(_frequencies(c), torch.float64)
        return s
    s["q"] = normal((rows, nh * c["group"], hd), dtype, 1.5)
    s["out"] = torch.zeros_like(s["q"])
    s["stats"] = torch.zeros((rows, nh * c["group"], 2), dtype=torch.float32, device="cuda")
    masks = [_tree_masks(rng, n) for n in counts]
    s["mask"] = None if c["n"] == 1 else numbers(_signed([m for one in masks for m in one]), torch.int64)
    if c["kind"] == "mass":
        s["count"] = numbers(_signed([one[-1] for one in masks]), torch.int64)  # the accepted path
        s["stats"].copy_(_ragged_rows(s, torch.stack(_softmax(s)[1:], dim=-1)))
    return s


# ---------------------------------------------------------------------------
# the framework's calls


def _bound(s):
    """The cache, the rows and the workspace as the calls take them: made once, as a
    program keeps them."""
    if "bound" not in s:
        from paper_2412_18934_amd import dv
        c = s["case"]

        def at(name):
            return s[name].data_ptr() if s.get(name) is not None else 0

        nl, n_pages = s["mass"].shape[:2]
        pg = dv.dv_paged(at("k"), at("v"), at("mass"), at("table"), at("lens"), 0, nl, c["heads"], c["hd"], n_pages,
                         c["page"], c["seqs"], s["table"].shape[1])
        rows = rope = ws = None
        if c["kind"] in ("attend", "mass", "append"):
            q = s["qkv"] if c["kind"] == "append" else s["q"]
            rows = dv.dv_paged_rows(q.data_ptr(), q.stride(0), at("start"), at("mask"), 0.0, c.get("cap", 0.0),
                                    dv.DV_F32 if c["dtype"] == "f32" else dv.DV_BF16, c["heads"] * c["group"],
                                    q.shape[0], min(c["n"], 64), c["len"] + c["n"])
        if c["kind"] == "append":
            low, high = (1, 4) if c["scaling"] == TURNS else (1, 32)
            rope = dv.dv_rope_init(dv.dv_rope(10000.0, 8.0, low, high, _magnitude(c), 4096, c["scaling"], c["rot"],
                                              c["interleaved"]))
        elif c["kind"] == "attend":
            ws = torch.empty(dv.dv_paged_attention_workspace(pg, rows), dtype=torch.uint8, device="cuda")
        s["bound"] = dv, pg, rows, rope, ws
    return s["bound"]


def _own(s):
    c = s["case"]
    dv, pg, rows, rope, ws = _bound(s)
    stream = torch.cuda.current_stream().cuda_stream
    if c["kind"] == "attend":
        dv.dv_paged_attention(pg, 1, rows, s["out"].data_ptr(), s["out"].stride(0), s["stats"].data_ptr(), ws.data_ptr(),
                              ws.numel(), stream)
        return dict(out=s["out"], stats=s["stats"])
    if c["kind"] == "mass":
        dv.dv_paged_mass(pg, 1, rows, s["stats"].data_ptr(), s["count"].data_ptr(), stream)
        return s["mass"][1]
    if c["kind"] == "append":
        x, heads = s["qkv"], c["heads"]
        k = x.data_ptr() + heads * c["group"] * c["hd"] * x.element_size()
        dv.dv_paged_append(pg, 1, rows, rope, s["positions"].data_ptr(), k, x.stride(0),
                           k + heads * c["hd"] * x.element_size(), x.stride(0), stream)
        return dict(q=x[:, :heads * c["group"]], k=s["k"][1], v=s["v"][1], mass=s["mass"][1])
    if c["kind"] == "commit":
        dv.dv_paged_commit(pg, s["path"].data_ptr(), s["path"].stride(0), s["path_len"].data_ptr(), s["new_lens"].data_ptr(),
                           stream)
    else:
        dv.dv_paged_evict(pg, c["budget"], c["recent"], s["new_lens"].data_ptr(), stream)
    return _whole(s)


def _whole(s):
    return dict(k=s["k"], v=s["v"], mass=s["mass"], lens=s["new_lens"])


# ---------------------------------------------------------------------------
# the plain forms


def _row_index(s):
    """[seqs][most rows]: a row's number, and whether there is one."""
    c = s["case"]
    if s["start"] is None:
        at = torch.arange(c["seqs"], device="cuda")[:, None]
        return at, at >= 0
    i = torch.arange(max(s["counts_host"]), device="cuda")
    at = s["start"][:-1, None] + i
    there = at < s["start"][1:, None]
    return torch.where(there, at, 0), there


def _softmax(s, layer=1):
    """Scores of the padded rows [seqs][heads][rows group][slots] as exp(z - max), and max
    and sum of every row."""
    c = s["case"]
    ns, nh, hd = c["seqs"], c["heads"], c["hd"]
    at, _ = _row_index(s)
    n = at.shape[1]
    q = s["q"][at].float().reshape(ns, n, nh, c["group"], hd).transpose(1, 2).reshape(ns * nh, n * c["group"], hd)
    k = s["k"][layer][s["table"].long()].float().transpose(1, 2).reshape(ns * nh, -1, hd)
    z = torch.bmm(q, k.transpose(1, 2).contiguous()).reshape(ns, nh, n, c["group"], -1) / math.sqrt(hd)
    if c["cap"]:
        z = c["cap"] * torch.tanh(z / c["cap"])
    new = torch.arange(z.shape[-1], device="cuda") - s["lens"][:, None]  # [seqs][slots]: which new row a slot is
    if s["mask"] is None:
        sees = (new <= 0)[:, None]
    else:
        bits = s["mask"][at][:, :, None] >> new[:, None].clamp(0, 63) & 1
        sees = (new < 0)[:, None] | (new[:, None] < 64) & (bits == 1)
    z = torch.where(sees[:, None, :, None], z, -math.inf)
    m = z.amax(dim=-1)
    p = torch.exp(z - m[..., None])
    return p, m, p.sum(dim=-1)


def _ragged_rows(s, x):
    """Padded [seqs][heads][rows][group][..] as [all rows][heads group][..]."""
    _, there = _row_index(s)
    x = x.permute(0, 2, 1, 3, *range(4, x.dim()))
    return x[there].reshape(-1, x.shape[2] * x.shape[3], *x.shape[4:])


def _attend(s):
    c = s["case"]
    p, m, l = _softmax(s)
    v = s["v"][1][s["table"].long()].float()  # [seqs][pages][heads][tiles][hd][32]
    v = v.permute(0, 2, 1, 3, 5, 4).reshape(c["seqs"] * c["heads"], -1, c["hd"])
    o = torch.bmm(p.reshape(v.shape[0], -1, v.shape[1]), v).reshape(*l.shape, c["hd"]) / l[..., None]
    return dict(out=_ragged_rows(s, o).to(s["q"].dtype), stats=_ragged_rows(s, torch.stack([m, l], dim=-1)))


def _add_mass(s):
    c = s["case"]
    p, m, l = _softmax(s)
    at, there = _row_index(s)
    stats = s["stats"][at].reshape(*at.shape, c["heads"], c["group"], 2).transpose(1, 2)
    counted = there & ((s["count"][:, None] >> torch.arange(at.shape[1], device="cuda") & 1) == 1)
    w = p * (torch.exp(m - stats[..., 0]) / stats[..., 1] * counted[:, None, :, None])[..., None]
    w = w.sum(dim=(2, 3)).reshape(c["seqs"], c["heads"], -1, c["page"]).transpose(1, 2)  # [seqs][pages][heads][page]
    used = s["table"] >= 0
    s["mass"][1].index_add_(0, s["table"][used].long(), w[used])
    return s["mass"][1]


def _append(s):
    c = s["case"]
    x, nh, half = s["qkv"], c["heads"], c["rot"] // 2
    angle = s["positions"].double()[:, None] * s["freq"]
    cos, sin = ((f(angle) * _magnitude(c)).float()[:, None] for f in (torch.cos, torch.sin))
    turned = x[:, :nh * (c["group"] + 1)].to(torch.float32, copy=True)  # (keys are read only)
    if c["interleaved"]:
        a, b = turned[..., 0:c["rot"]:2], turned[..., 1:c["rot"]:2]
    else:
        a, b = turned[..., :half], turned[..., half:c["rot"]]
    a, b = a * cos - b * sin, b * cos + a * sin
    if c["interleaved"]:
        turned[..., 0:c["rot"]:2], turned[..., 1:c["rot"]:2] = a, b
    else:
        turned[..., :half], turned[..., half:c["rot"]] = a, b
    x[:, :nh * c["group"]] = turned[:, :nh * c["group"]].to(x.dtype)
    row = torch.arange(x.shape[0], device="cuda")
    if s["start"] is None:
        seq, first = row, row
    else:
        seq = (row[:, None] >= s["start"][1:]).sum(dim=1)
        first = s["start"][seq]
    slot = s["lens"][seq] + row - first
    page, at = s["table"][seq, slot // c["page"]].long(), slot % c["page"]
    s["k"][1, page, :, at] = turned[:, nh * c["group"]:].to(torch.bfloat16)
    s["v"][1, page, :, at // TILE, :, at % TILE] = x[:, nh * (c["group"] + 1):].to(torch.bfloat16)
    s["mass"][1, page, :, at] = 0
    return dict(q=x[:, :nh * c["group"]], k=s["k"][1], v=s["v"][1], mass=s["mass"][1])


def _commit(s):
    c = s["case"]
    j = torch.arange(s["path"].shape[1], device="cuda")
    kept = j < s["path_len"][:, None]
    seq = torch.arange(c["seqs"], device="cuda")[:, None].expand_as(kept)[kept]
    to = (s["lens"][:, None] + j)[kept]
    come = (s["lens"][:, None] + s["path"])[kept]
    p, q = s["table"][seq, to // c["page"]].long(), s["table"][seq, come // c["page"]].long()
    to, come = to % c["page"], come % c["page"]
    s["k"][:, p, :, to] = s["k"][:, q, :, come]
    s["v"][:, p, :, to // TILE, :, to % TILE] = s["v"][:, q, :, come // TILE, :, come % TILE]
    s["mass"][:, p, :, to] = s["mass"][:, q, :, come]
    s["new_lens"].copy_(s["lens"] + s["path_len"])
    return _whole(s)


def _evict(s):
    c = s["case"]
    nl, n_pages, nh, page = s["mass"].shape
    table, lens = s["table"].long(), s["lens"].long()
    mass = s["mass"][:, table].transpose(2, 3).reshape(nl, c["seqs"], nh, -1)
    slot = torch.arange(mass.shape[-1], device="cuda")
    rank = torch.where(slot < (lens - c["recent"])[:, None, None], mass, math.inf)
    rank = torch.where(slot < lens[:, None, None], rank, -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices
    come = torch.sort(order[..., :c["budget"]], dim=-1).values
    # (a sequence within its budget keeps its slots: the last stands in for those it has not)
    to = torch.minimum(torch.arange(come.shape[-1], device="cuda").expand_as(come), (lens - 1)[:, None, None].clamp(min=0))
    come = torch.where((lens > c["budget"])[:, None, None], come, to)
    seq = torch.arange(c["seqs"], device="cuda")[:, None, None].expand_as(come)
    head = (torch.arange(nl, device="cuda")[:, None, None, None] * n_pages, torch.arange(nh, device="cuda")[:, None])

    def flat(x):  # an index over [layers][pages][heads][page]
        return ((head[0] + table[seq, x // page]) * nh + head[1]) * page + x % page

    there = (lens > c["budget"])[:, None, None].expand_as(come)
    to, come = flat(to)[there], flat(come)[there]
    k, mass = s["k"].view(-1, c["hd"]), s["mass"].view(-1)
    k[to] = k[come]
    mass[to] = mass[come]
    v = s["v"].view(-1, c["hd"], TILE)
    v[to // TILE, :, to % TILE] = v[come // TILE, :, come % TILE]
    s["new_lens"].copy_(lens.clamp(max=c["budget"]))
    return _whole(s)


def run(state):
    if own:
        return _own(state)
    return dict(attend=_attend, append=_append, mass=_add_mass, commit=_commit, evict=_evict)[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------
# the definitions in 64 bits, sequence by sequence and slot by slot


def _where(s, i, slots):
    """Pages and places of sequence i's slots."""
    pages = s["table"][i].tolist()
    at = torch.tensor([(pages[x // s["case"]["page"]], x % s["case"]["page"]) for x in slots], device="cuda")
    return at.reshape(-1, 2).unbind(1)


def _keys(s, i, n):
    p, at = _where(s, i, range(n))
    return s["k"][1, p, :, at].double().transpose(0, 1), s["v"][1, p, :, at // TILE, :, at % TILE].double().transpose(0, 1)


def _exact_rows(s):
    """Per sequence: its first row, its rows, scores [heads][rows group][slots], values."""
    c, first = s["case"], 0
    masks = None if s["mask"] is None else s["mask"].tolist()
    for i, (length, n) in enumerate(zip(s["lens_host"], s["counts_host"])):
        k, v = _keys(s, i, length + n)
        q = s["q"][first:first + n].double().reshape(n, c["heads"], c["group"], c["hd"]).transpose(0, 1)
        q = q.reshape(c["heads"], n * c["group"], c["hd"])
        z = torch.stack([q[h] @ k[h].T.contiguous() for h in range(c["heads"])]) * c["hd"] ** -0.5
        if c["cap"]:
            z = torch.tanh(z / c["cap"]) * c["cap"]
        hidden = [[0.0 if masks is None or masks[first + a] >> b & 1 else -math.inf for b in range(n)] for a in range(n)]
        hidden = torch.tensor(hidden, dtype=torch.float64, device="cuda").repeat_interleave(c["group"], dim=0)
        z[:, :, length:] += hidden
        yield i, first, n, z, v
        first += n


def exact(case, seed):
    c, s = case, prepare(case, seed)
    nh, group, hd = c["heads"], c["group"], c["hd"]
    if c["kind"] == "attend":
        out, stats = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"), s["stats"].double()
        for _, first, n, z, v in _exact_rows(s):
            o = torch.stack([torch.softmax(z[h], dim=1) @ v[h] for h in range(nh)])
            m = z.amax(dim=2)
            both = torch.stack([m, (z - m[..., None]).exp().sum(dim=2)], dim=2)
            out[first:first + n] = o.reshape(nh, n, group, hd).transpose(0, 1).reshape(n, nh * group, hd)
            stats[first:first + n] = both.reshape(nh, n, group, 2).transpose(0, 1).reshape(n, nh * group, 2)
        return dict(out=out, stats=stats)
    if c["kind"] == "mass":
        mass, count = s["mass"][1].double(), s["count"].tolist()
        for i, first, n, z, _ in _exact_rows(s):
            p, at = _where(s, i, range(z.shape[2]))
            stats = s["stats"][first:first + n].double().reshape(n, nh, group, 2)
            for a in range(n):
                if count[i] >> a & 1:
                    for h in range(nh):
                        w = (z[h, a * group:(a + 1) * group] - stats[a, h, :, :1]).exp() / stats[a, h, :, 1:]
                        mass[p, h, at] += w.sum(dim=0)
        return mass
    if c["kind"] == "append":
        x, freq = s["qkv"].double(), s["freq"]
        k, v, mass = s["k"][1].double(), s["v"][1].double(), s["mass"][1].double()
        angle = s["positions"].double()[:, None] * freq
        turn = torch.polar(torch.full_like(angle, _magnitude(c)), angle)[:, None]
        part = x[:, :nh * (group + 1), :c["rot"]]
        pairs = part.reshape(*part.shape[:2], -1, 2) if c["interleaved"] else part.reshape(*part.shape[:2], 2, -1).transpose(2, 3)
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        x[:, :nh * (group + 1), :c["rot"]] = (pairs if c["interleaved"] else pairs.transpose(2, 3)).reshape(part.shape)
        first = 0
        for i, (length, n) in enumerate(zip(s["lens_host"], s["counts_host"])):
            p, at = _where(s, i, range(length, length + n))
            k[p, :, at] = x[first:first + n, nh * group:nh * (group + 1)]
            v[p, :, at // TILE, :, at % TILE] = x[first:first + n, nh * (group + 1):]
            mass[p, :, at] = 0
            first += n
        return dict(q=x[:, :nh * group], k=k, v=v, mass=mass)
    k, v, mass = s["k"].clone(), s["v"].clone(), s["mass"].clone()  # (moved, not computed)
    if c["kind"] == "commit":
        lens = [n + p for n, p in zip(s["lens_host"], s["path_len"].tolist())]
        for i, path in enumerate(s["path"].tolist()):
            for j in range(int(s["path_len"][i])):
                (p, q), (to, come) = _where(s, i, [s["lens_host"][i] + j, s["lens_host"][i] + path[j]])
                k[:, p, :, to] = s["k"][:, q, :, come]
                v[:, p, :, to // TILE, :, to % TILE] = s["v"][:, q, :, come // TILE, :, come % TILE]
                mass[:, p, :, to] = s["mass"][:, q, :, come]
    else:
        lens = [min(n, c["budget"]) for n in s["lens_host"]]
        if c["layers"] * nh * len(lens) > 6000:  # (every head of every sequence by itself)
            return None
        for i, n in enumerate(s["lens_host"]):
            if n <= c["budget"]:
                continue
            p, at = _where(s, i, range(n))
            b = torch.arange(c["budget"], device="cuda")
            had = s["mass"][:, p, :, at].permute(1, 2, 0).cpu().numpy()  # (indexed dims come first)
            for layer in range(c["layers"]):
                for h in range(nh):
                    # heavier slots stand first, the earlier of equal ones
                    by = np.lexsort((np.arange(n - c["recent"]), -had[layer, h, :n - c["recent"]]))
                    kept = np.concatenate([np.sort(by[:c["budget"] - c["recent"]]), np.arange(n - c["recent"], n)])
                    kept = torch.from_numpy(kept).cuda()
                    q, come = p[kept], at[kept]
                    mass[layer, p[b], h, at[b]] = s["mass"][layer, q, h, come]
                    k[layer, p[b], h, at[b]] = s["k"][layer, q, h, come]
                    v[layer, p[b], h, at[b] // TILE, :, at[b] % TILE] = s["v"][layer, q, h, come // TILE, :, come % TILE]
    return dict(k=k.double(), v=v.double(), mass=mass.double(), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
