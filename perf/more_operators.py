"""Measured calls of the paged cache: rotary positions, the append, attention of new tokens, accumulated attention weights, eviction.

  own                  False: `run` computes the plain forms below; True: it calls the framework's operators
  listed()             the fixed cases
  draw(rng)            one more case of the same ranges
  prepare(case, seed)  inputs, pages, tables, buffers and workspaces a program holds before the call, on the GPU
  run(state)           one pass and its outputs
  work(case)           bytes and operations of one pass that no implementation can do without
  exact(case, seed)    the outputs in 64 bits, from the definitions

A case is a dict of plain values:
  kind      "rope"     queries and keys of a prompt rotated by their positions (bwd: the gradients rotated back)
            "append"   n new tokens per sequence into the pages, keys and queries rotated on the way
            "attn"     attention of a sequence's last n tokens over its pages, causal among the new ones
            "weights"  what every cached token gets of those tokens' attention, summed over them and a group's heads, added to
                       what it had
            "evict"    the budget's rows of each sequence and head with the largest weights, the first and the latest ones among them,
                       into other pages
  batch, seq, seq_min  sequences, the longest and the shortest of them with their new tokens (lengths spread evenly between)
  n, n_min             new tokens of a sequence, the most and the fewest (spread evenly; n_min = 0: all have n)
  hq, hkv, page        query and key-value heads, rows of a page
  rot, interleaved     channels that rotate; pairs (2 j, 2 j + 1) instead of (j, j + rot / 2)
  scaling, factor, original   positions for long contexts: "none", "linear", "ntk", "yarn" or "factors" (one for each pair)
  far                  position of a sequence's first token (-1: 0, and no positions are given)
  budget, first, recent       rows kept; of them the first and the latest tokens
  heavy                keys with log-normal norms

A page holds `page` consecutive tokens of a sequence for all key-value heads; a sequence's table lists its pages, which lie anywhere.
"""
import math

import torch

own = False

D = 128
BASE = 10000.0

_FIELDS = dict(kind="attn", batch=1, seq=1024, seq_min=0, n=1, n_min=0, hq=32, hkv=2, page=64, rot=128, interleaved=False, scaling="none",
               factor=1.0, original=0, far=-1, budget=1, first=0, recent=0, heavy=False, bwd=False)


def _case(**kw):
    c = dict(_FIELDS, **kw)
    c["seq_min"] = c["seq_min"] or c["seq"]
    c["n_min"] = c["n_min"] or c["n"]
    return c


def listed():
    return [
        # a short prompt on a small model, half of the channels rotated in neighbouring pairs
        _case(name="rope_777_g4", kind="rope", seq=777, hq=4, hkv=1, rot=64, interleaved=True),
        # a long document's training step, gradients, positions stretched beyond the trained length
        _case(name="rope_bwd_32k", kind="rope", seq=32768, scaling="yarn", factor=8.0, original=4096, bwd=True),
        # the next token of one chat that has lost its oldest rows: its position is far behind its row
        _case(name="append_b1", kind="append", seq=2049, far=500000, scaling="factors", factor=4.0, original=32768),
        # prompts' pieces of a serving step, ragged
        _case(name="append_4x2000", kind="append", batch=4, seq=9001, seq_min=2500, n=2000, n_min=1777, page=16, scaling="ntk", factor=4.0),
        # the next token of one long chat
        _case(name="attn_b1_20k", kind="attn", seq=20011),
        # the next tokens of a full serving batch
        _case(name="attn_b64", kind="attn", batch=64, seq=32749, seq_min=1501, page=16, heavy=True),
        # two questions of a few words about long documents
        _case(name="attn_n37", kind="attn", batch=2, seq=32749, seq_min=30011, n=37, n_min=21, hq=16, page=32),
        # a piece of a long document's prompt
        _case(name="attn_8k_of_64k", kind="attn", seq=65536, n=8192),
        # a serving batch's next tokens, for the eviction that follows
        _case(name="weights_b64", kind="weights", batch=64, seq=8191, seq_min=4001),
        # a prompt's last piece, for the eviction that follows
        _case(name="weights_4k_of_32k", kind="weights", seq=32749, n=4096, page=128),
        # one long prompt to an eighth
        _case(name="evict_32k", kind="evict", seq=32749, budget=4096, first=4, recent=1024),
        # a serving batch back to its budget
        _case(name="evict_b32", kind="evict", batch=32, seq=9001, seq_min=5001, budget=4501, first=64, recent=2000, page=16),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    kind = rng.choice(["rope", "append", "attn", "attn", "attn", "attn", "weights", "weights", "evict", "evict"])
    group, hkv = rng.choice([16, 16, 8, 4, 2, 1]), rng.choice([1, 2, 2, 4])
    c = dict(kind=kind, hq=group * hkv, hkv=hkv, page=rng.choice([16, 16, 32, 64, 64, 128, 256]), heavy=rng.random() < 0.25)
    if kind in ("rope", "append"):
        c["rot"], c["interleaved"] = rng.choice([128, 128, 96, 64, 32, 16]), rng.random() < 0.4
        c["scaling"] = rng.choice(["none", "none", "linear", "ntk", "yarn", "factors"])
        if c["scaling"] != "none":
            c["factor"], c["original"] = rng.choice([2.0, 3.5, 8.0, 32.0]), rng.choice([2048, 4096, 32768])
        c["far"] = rng.choice([-1, -1, 0, 1, 4097, 131071, 1000003])
    if kind == "rope":
        c["seq"] = _log_int(rng, 1, 32768 * 32 // max(32, c["hq"]))
        c["batch"], c["bwd"] = rng.choice([1, 2, 3, 5]) if c["seq"] <= 4096 else 1, rng.random() < 0.5
    elif kind == "append":
        c["batch"], c["n"] = _log_int(rng, 1, 32), _log_int(rng, 1, 4096)
        c["batch"] = max(1, min(c["batch"], 8192 // c["n"]))
        c["seq"] = c["n"] + _log_int(rng, 1, 16384) - 1
    elif kind == "evict":
        c["seq"] = _log_int(rng, 100, 131072)
        c["batch"] = _log_int(rng, 1, max(1, min(32, 524288 // (c["seq"] * hkv))))
        c["budget"] = _log_int(rng, 1, c["seq"] + 64)
        c["first"] = rng.choice([0, 1, 4, 64])
        c["first"] = min(c["first"], c["budget"])
        c["recent"] = min(c["budget"] - c["first"], rng.choice([0, 1, 16, c["budget"] // 4, c["budget"] // 2]))
    else:
        c["n"] = rng.choice([1, 1, 1, _log_int(rng, 2, 64), _log_int(rng, 64, 4096)])
        context = _log_int(rng, 1, 65536 if c["n"] < 1024 else 32768) - 1
        c["seq"] = c["n"] + context
        c["batch"] = _log_int(rng, 1, max(1, min(64, 1048576 // (c["seq"] * hkv), 4096 // c["n"])))
    if c.get("batch", 1) > 1 and rng.random() < 0.8:
        c["seq_min"] = rng.randint(max(1, c["seq"] // 8), c["seq"])
        if "n" in c:
            c["n_min"] = rng.randint(max(1, c["n"] // 2), c["n"])
            c["seq_min"] = max(c["seq_min"], c["n"])             # a sequence holds its new tokens
    return _case(**c)


# ---- what a case means -----------------------------------------------------------------------------------------

def _spread(most, least, b):
    return [most] if b == 1 else [most - (most - least) * i // (b - 1) for i in range(b)]


def _lengths(c):
    return _spread(c["seq"], c["seq_min"], c["batch"])


def _new(c):
    return _spread(c["n"], c["n_min"], c["batch"])


def _pages(length, page):
    return (length + page - 1) // page


def _pair_factors(c):
    """one divisor for each pair, growing with its wavelength"""
    return [1.0 + (c["factor"] - 1.0) * (2.0 * j / c["rot"]) ** 2 for j in range(c["rot"] // 2)]


def _frequencies(c):
    """angle of each pair from one position to the next, in radians, and what the cosines and sines are multiplied by"""
    rot, factor, kind = c["rot"], c["factor"], c["scaling"]
    base, amplitude = BASE, 1.0
    if kind == "ntk":
        base = BASE * factor ** (rot / (rot - 2.0))
    f = [base ** (-2.0 * j / rot) for j in range(rot // 2)]
    if kind == "linear":
        f = [x / factor for x in f]
    if kind == "yarn":                                           # pairs of 32 turns and more in the trained length stay, those of 1 and less are stretched
        keep = [min(1.0, max(0.0, (c["original"] * x / (2.0 * math.pi) - 1.0) / 31.0)) for x in f]
        f = [x * (k + (1.0 - k) / factor) for x, k in zip(f, keep)]
        amplitude = 0.1 * math.log(factor) + 1.0
    if kind == "factors":
        f = [x / y for x, y in zip(f, _pair_factors(c))]
        amplitude = math.sqrt(1.0 + math.log(factor) / math.log(c["original"]))
    return f, amplitude


# ---- inputs ----------------------------------------------------------------------------------------------------

def _normal(shape, gen):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _page_table(lengths, page, spare, gen):
    """[B, most pages] of pages in random order, and how many pages there are; unused entries are 0"""
    counts = [_pages(x, page) for x in lengths]
    order = torch.randperm(sum(counts) + spare, generator=gen, device="cuda").int()
    table = torch.zeros((len(counts), max(1, max(counts))), dtype=torch.int32, device="cuda")
    at = 0
    for b, x in enumerate(counts):
        table[b, :x] = order[at:at + x]
        at += x
    return table, sum(counts) + spare


def prepare(case, seed):
    c = dict(_FIELDS, **case)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    lengths, kind, b, cap = _lengths(c), c["kind"], c["batch"], c["seq"]
    s = {"c": c, "sl": torch.tensor(lengths, dtype=torch.int32, device="cuda"), "cap": cap, "n_new": None, "positions": None}
    if kind in ("rope", "append"):
        f, s["amplitude"] = _frequencies(c)
        s["frequencies"] = torch.tensor(f, dtype=torch.float64, device="cuda")
    if kind == "rope":
        rows, first = cap, torch.zeros(b, dtype=torch.int64, device="cuda")
        s["q"], s["k"] = _normal((b, cap, c["hq"], D), gen), _normal((b, c["hkv"], cap, D), gen)
    elif kind != "evict":
        rows = c["n"]
        n_new = torch.tensor(_new(c), dtype=torch.int32, device="cuda")
        first = (s["sl"] - n_new).long()
        s["n_new"] = n_new if c["n_min"] < c["n"] else None
        s["q"] = _normal((b, rows, c["hq"], D), gen)
    if kind in ("rope", "append"):
        s["row_positions"] = torch.arange(rows, device="cuda")[None] + (first[:, None] if c["far"] < 0 else c["far"])
        if c["far"] >= 0:
            s["positions"] = s["row_positions"].int()
    if kind != "rope":
        s["table"], count = _page_table(lengths, c["page"], 3, gen)
        s["k_pages"], s["v_pages"] = (_normal((count, c["hkv"], c["page"], D), gen) for _ in range(2))
        if c["heavy"]:
            z = torch.randn((count, c["hkv"], c["page"], 1), generator=gen, device="cuda")
            s["k_pages"] = (s["k_pages"].float() * torch.exp(0.5 * z)).bfloat16()
    if kind == "append":
        s["k_new"], s["v_new"] = (_normal((b, c["hkv"], rows, D), gen) for _ in range(2))
    if kind in ("weights", "evict"):
        s["weights"] = torch.zeros((b, c["hkv"], cap), dtype=torch.float32, device="cuda").exponential_(generator=gen) ** 2
    if kind == "weights":
        s["lse"] = _attn(s)[1]                                   # of the finished attention
        s["weights_out"] = torch.zeros_like(s["weights"])
    if kind == "evict":
        s["to_table"], count = _page_table([min(c["budget"], x) for x in lengths], c["page"], 1, gen)
        s["to_k"], s["to_v"] = (torch.zeros((count, c["hkv"], c["page"], D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """what a program that uses the framework holds besides: parameters, the rotation's table, for serving its buffers and workspace"""
    from paper_2506_07900_amd import binding
    c, b, cap = s["c"], s["c"]["batch"], s["cap"]
    prm = s["prm"] = binding.Params(c["hq"], c["hkv"])
    keep = s["keep"] = {}
    if "frequencies" in s:
        s["rope"] = binding.rope_table(c["rot"], base=BASE, interleaved=c["interleaved"], scaling=c["scaling"], factor=c["factor"],
                                       original_len=c["original"], pair_factors=_pair_factors(c) if c["scaling"] == "factors" else None)
    if s["positions"] is not None:                               # (the call takes one for each row of each sequence)
        s["positions"] = s["positions"].expand(b, -1).contiguous()
    if "k_pages" in s:
        s["cache"] = binding.PagedCache(s["k_pages"], s["v_pages"], s["table"])
    if c["kind"] == "append":
        keep["q_out"] = torch.zeros_like(s["q"])
    if c["kind"] == "attn":
        keep.update(out=torch.zeros_like(s["q"]), lse=torch.zeros((b, c["n"], c["hq"]), dtype=torch.float32, device="cuda"))
    if c["kind"] == "evict":
        s["to"] = binding.PagedCache(s["to_k"], s["to_v"], s["to_table"])
        keep.update(kept=torch.zeros((b, c["hkv"], c["budget"]), dtype=torch.int32, device="cuda"), seqlens_out=torch.zeros_like(s["sl"]),
                    weights_out=torch.zeros((b, c["hkv"], c["budget"]), dtype=torch.float32, device="cuda"))
    op = {"attn": binding.OP_PAGED_ATTN, "weights": binding.OP_PAGED_WEIGHTS, "evict": binding.OP_PAGED_EVICT}.get(c["kind"])
    if op is not None:
        need = binding.paged_workspace_bytes(op, prm, b, cap, c["n"])
        keep["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")


# ---- one pass --------------------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _PLAIN[state["c"]["kind"]](state)


def _run_own(s):
    from paper_2506_07900_amd import binding
    c, prm, cap, keep = s["c"], s["prm"], s["cap"], s["keep"]
    if c["kind"] == "rope":
        return (binding.rope_bwd if c["bwd"] else binding.rope)(prm, s["rope"], s["q"], s["k"], s["sl"], cap, positions=s["positions"])
    if c["kind"] == "append":
        q = binding.paged_append(prm, s["k_new"], s["v_new"], s["cache"], s["sl"], cap, n_new=s["n_new"], rope=s["rope"],
                                 positions=s["positions"], q=s["q"], **keep)
        return q, s["k_pages"], s["v_pages"]
    if c["kind"] == "attn":
        return binding.paged_attn(prm, s["q"], s["cache"], s["sl"], cap, n_new=s["n_new"], **keep)
    if c["kind"] == "weights":
        return binding.paged_attn_weights(prm, s["q"], s["lse"], s["cache"], s["sl"], cap, n_new=s["n_new"], weights=s["weights"],
                                          weights_out=s["weights_out"], **keep)
    kept, weights, lengths = binding.paged_evict(prm, s["weights"], s["cache"], s["sl"], cap, c["budget"], c["first"], c["recent"],
                                                 s["to"], **keep)
    return kept, weights, lengths, s["to_k"], s["to_v"]


# ---- the plain forms, in 32 bits (angles in 64) ------------------------------------------------------------------

def _rotated(x, s, cos, sin):
    """x [.., D] by its row's angles [.., rot / 2]; one rounding at the end"""
    rot, y = s["c"]["rot"], x.float()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if s["c"]["interleaved"] else (y[..., :rot // 2], y[..., rot // 2:rot])
    u, v = a * cos - b * sin, b * cos + a * sin
    u = torch.stack((u, v), -1).flatten(-2) if s["c"]["interleaved"] else torch.cat((u, v), -1)
    return torch.cat((u.to(x.dtype), x[..., rot:]), -1)


def _angles(s):
    """cosines and sines [B, rows, rot / 2]"""
    angle = s["row_positions"].double()[..., None] * s["frequencies"]
    return (torch.cos(angle) * s["amplitude"]).float(), (torch.sin(angle) * s["amplitude"]).float()


def _live(s, rows):
    """rows of a batch that are some sequence's: [B, rows]"""
    counts = s["sl"] if s["c"]["kind"] == "rope" else s["n_new"]
    i = torch.arange(rows, device="cuda")[None]
    return i < counts[:, None] if counts is not None else torch.ones((s["c"]["batch"], rows), dtype=torch.bool, device="cuda")


def _rope(s):
    cos, sin = _angles(s)
    sin = -sin if s["c"]["bwd"] else sin
    live = _live(s, s["cap"])
    q = _rotated(s["q"], s, cos[:, :, None], sin[:, :, None])
    k = _rotated(s["k"], s, cos[:, None], sin[:, None])
    return torch.where(live[:, :, None, None], q, 0), torch.where(live[:, None, :, None], k, 0)


def _first(s):
    """the cache row of a sequence's first new token"""
    return (s["sl"] - (s["n_new"] if s["n_new"] is not None else s["c"]["n"])).long()


def _append(s):
    c = s["c"]
    cos, sin = _angles(s)
    live = _live(s, c["n"])
    q = torch.where(live[:, :, None, None], _rotated(s["q"], s, cos[:, :, None], sin[:, :, None]), 0)
    k = _rotated(s["k_new"], s, cos[:, None], sin[:, None])
    b, i = live.nonzero(as_tuple=True)
    row = _first(s)[b] + i
    page, at = s["table"][b, row // c["page"]].long(), row % c["page"]
    s["k_pages"][page, :, at] = k[b, :, i]
    s["v_pages"][page, :, at] = s["v_new"][b, :, i]
    return q, s["k_pages"], s["v_pages"]


def _cached(s, pages):
    """[B, Hkv, T, D] in 32 bits, T the longest sequence; rows behind a sequence are 0"""
    t = torch.arange(s["cap"], device="cuda")
    rows = pages[s["table"].long()[:, t // s["c"]["page"]], :, t % s["c"]["page"]]                 # [B, T, Hkv, D]
    return torch.where((t[None] < s["sl"][:, None])[..., None, None], rows, 0).transpose(1, 2).float().contiguous()


def _pieces(s):
    """slices of the new tokens whose scores take up to half a GiB"""
    c = s["c"]
    step = max(1, 2 ** 27 // (c["batch"] * c["hq"] * s["cap"]))
    return [slice(i, min(c["n"], i + step)) for i in range(0, c["n"], step)]


def _scores(s, keys, at):
    """scores [B, Hkv, rows, G, T] of the new tokens `at`, hidden ones -inf"""
    c = s["c"]
    q = s["q"][:, at].float().reshape(c["batch"], -1, c["hkv"], c["hq"] // c["hkv"], D).transpose(1, 2)
    x = torch.matmul(q.flatten(2, 3), keys) * D ** -0.5
    i = torch.arange(at.start, at.stop, device="cuda")
    last = torch.where(_live(s, c["n"])[:, at], _first(s)[:, None] + i, -1)                      # the last token that a row sees
    seen = torch.arange(s["cap"], device="cuda") <= last[..., None]
    return torch.where(seen[:, None, :, None], x.reshape(*q.shape[:4], -1), -math.inf)


def _attn(s):
    c = s["c"]
    keys, values = _cached(s, s["k_pages"]).transpose(-1, -2).contiguous(), _cached(s, s["v_pages"])
    out = torch.zeros_like(s["q"])
    lse = torch.zeros((c["batch"], c["n"], c["hq"]), dtype=torch.float32, device="cuda")
    live = _live(s, c["n"])
    for at in _pieces(s):
        x = _scores(s, keys, at)
        top = x.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        p = torch.exp(x - top)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p.flatten(2, 3), values).reshape(*p.shape[:4], D) / torch.where(total > 0, total, 1.0)
        out[:, at] = o.transpose(1, 2).flatten(2, 3).bfloat16()
        z = (top + torch.log(total))[..., 0].transpose(1, 2).flatten(2, 3)
        lse[:, at] = torch.where(live[:, at, None], z, 0.0)
    return out, lse


def _weights(s):
    c = s["c"]
    keys = _cached(s, s["k_pages"]).transpose(-1, -2).contiguous()
    t = torch.arange(s["cap"], device="cuda")[None]
    total = torch.where((t < _first(s)[:, None])[:, None], s["weights"], 0.0)                    # a new token has none yet
    for at in _pieces(s):
        z = s["lse"][:, at].reshape(c["batch"], -1, c["hkv"], c["hq"] // c["hkv"]).transpose(1, 2)
        total += torch.exp(_scores(s, keys, at) - z[..., None]).sum((2, 3))
    return torch.where((t < s["sl"][:, None])[:, None], total, 0.0)


def _evict(s):
    c = s["c"]
    t, length = torch.arange(s["cap"], device="cuda"), s["sl"][:, None, None]
    worth = torch.where((t < c["first"]) | (t >= length - c["recent"]), math.inf, s["weights"])
    worth = torch.where(t < length, worth, -math.inf)
    if c["budget"] > s["cap"]:
        worth = torch.nn.functional.pad(worth, (0, c["budget"] - s["cap"]), value=-math.inf)
    best = torch.sort(worth, dim=-1, descending=True, stable=True)[1][..., :c["budget"]]         # ties: the lowest row first
    best = torch.where(best < length, best, 2 ** 30).sort(-1)[0]
    there = best < 2 ** 30
    kept = torch.where(there, best, -1).int()
    weights = torch.where(there, s["weights"].gather(-1, best.clamp(max=s["cap"] - 1)), 0.0)
    b, h, j = there.nonzero(as_tuple=True)
    row = best[b, h, j]
    page, at = s["table"][b, row // c["page"]].long(), row % c["page"]
    to_page, to_at = s["to_table"][b, j // c["page"]].long(), j % c["page"]
    s["to_k"][to_page, h, to_at] = s["k_pages"][page, h, at]
    s["to_v"][to_page, h, to_at] = s["v_pages"][page, h, at]
    return kept, weights, s["sl"].clamp(max=c["budget"]), s["to_k"], s["to_v"]


_PLAIN = {"rope": _rope, "append": _append, "attn": _attn, "weights": _weights, "evict": _evict}


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    c = dict(_FIELDS, **case)
    wide, kind, hq, hkv = 2 * D, c["kind"], c["hq"], c["hkv"]
    bytes_, flops = 0.0, 0.0
    for length, n in zip(_lengths(c), _new(c)):
        if kind in ("rope", "append"):                           # queries and keys in and out; values too
            rows = length if kind == "rope" else n
            heads = hq + hkv + (hkv if kind == "append" else 0)
            bytes_ += rows * (2.0 * heads * wide + (4 if c["far"] >= 0 else 0)) + 4
            flops += rows * 3.0 * (hq + hkv) * c["rot"]
        elif kind == "evict":                                    # weights in; rows that stay in and out
            stay = min(length, c["budget"])
            bytes_ += hkv * (4.0 * length + stay * (4 * wide + 8)) + 4 * _pages(length, c["page"])
            flops += hkv * length
        else:
            pairs = n * (length - n) + n * (n + 1) // 2
            reads = 2 if kind == "attn" else 1
            bytes_ += length * hkv * reads * wide + n * hq * ((reads if kind == "attn" else 1) * wide + 4) + 4 * _pages(length, c["page"])
            bytes_ += length * hkv * 8 if kind == "weights" else 0
            flops += pairs * hq * 2.0 * D * reads
    return {"bytes": bytes_, "flops": flops}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _turn64(x, position, c, sign):
    """x [rows, heads, D]: each pair as a complex number, times amplitude e^(i position frequency)"""
    f, amplitude = _frequencies(c)
    angle = sign * position.double()[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.full_like(angle, amplitude), angle)[:, None]
    y, half = x.double().clone(), c["rot"] // 2
    j = torch.arange(half, device="cuda")
    first, second = (2 * j, 2 * j + 1) if c["interleaved"] else (j, j + half)
    z = torch.complex(y[..., first], y[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _rows64(s, pages, b, h, length):
    """rows [length, D] of one head"""
    page = s["c"]["page"]
    used = s["table"][b, :_pages(length, page)].long()
    return pages[used, h].reshape(-1, D)[:length].double()


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c, lengths, counts = s["c"], _lengths(s["c"]), _new(s["c"])
    kind, group, page = c["kind"], c["hq"] // c["hkv"], c["page"]
    if kind in ("rope", "append"):
        q = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        k = torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") if kind == "rope" else s["k_pages"].double()
        v = s["v_pages"].double() if kind == "append" else None
        for b, (length, n) in enumerate(zip(lengths, counts)):
            rows = length if kind == "rope" else n
            position = torch.arange(rows, device="cuda") + (c["far"] if c["far"] >= 0 else length - rows)
            sign = -1.0 if c["bwd"] else 1.0
            q[b, :rows] = _turn64(s["q"][b, :rows], position, c, sign)
            new = _turn64((s["k"] if kind == "rope" else s["k_new"])[b, :, :rows].transpose(0, 1), position, c, sign)
            if kind == "rope":
                k[b, :, :rows] = new.transpose(0, 1)
            else:
                for i in range(rows):
                    at = length - rows + i
                    p = s["table"][b, at // page].long()
                    k[p, :, at % page] = new[i]
                    v[p, :, at % page] = s["v_new"][b, :, i].double()
        return (q, k) if kind == "rope" else (q, k, v)
    if kind == "evict":                                          # copies: whole numbers and what the pages held
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((c["batch"], c["n"], c["hq"]), dtype=torch.float64, device="cuda")
    total = torch.zeros((c["batch"], c["hkv"], s["cap"]), dtype=torch.float64, device="cuda")
    for b, (length, n) in enumerate(zip(lengths, counts)):
        first = length - n
        for h in range(c["hkv"]):
            k, v = _rows64(s, s["k_pages"], b, h, length), _rows64(s, s["v_pages"], b, h, length)
            if kind == "weights":
                total[b, h, :first] = s["weights"][b, h, :first]
            for g in range(h * group, (h + 1) * group):
                for i0 in range(0, n, 1024):
                    i1 = min(n, i0 + 1024)
                    score = s["q"][b, i0:i1, g].double() @ k[:first + i1].t() / math.sqrt(D)
                    score[:, first + i0:] += torch.full((i1 - i0, i1 - i0), -math.inf, dtype=torch.float64, device="cuda").triu(1)
                    if kind == "attn":
                        lse[b, i0:i1, g] = torch.logsumexp(score, -1)
                        out[b, i0:i1, g] = torch.softmax(score, -1) @ v[:first + i1]
                    else:
                        total[b, h, :first + i1] += torch.exp(score - s["lse"][b, i0:i1, g].double()[:, None]).sum(0)
    return (out, lse) if kind == "attn" else total
