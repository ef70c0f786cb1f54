"""Measured calls of the 4-bit cache and of the windowed attention: their cases, inputs, plain forms and exact results.

  own                  False: `run` computes the plain forms below; True: it calls the framework's operators
  listed()             the fixed cases, smallest to largest of each kind
  draw(rng)            one more case of the same ranges
  prepare(case, seed)  inputs, caches, lists, buffers and workspaces a program holds before the call, on the GPU
  run(state)           one pass and its outputs
  work(case)           bytes and operations of one pass that no implementation can do without
  exact(case, seed)    the outputs in 64 bits, from the definitions

A case is a dict of plain values:
  kind      "quantize"       a prompt's keys and values into the 4-bit cache, and the whole cache read back
            "append"         n new rows per sequence into the 4-bit cache, with the semantic kernels they complete, and
                             those rows read back
            "sparse_quant"   attention over selected blocks of a 4-bit cache: one query per sequence (n = 0) or n drafted
                             tokens with a tree mask
            "window"         attention over a sliding window and the first tokens, one query per cached token
            "window_bwd"     its gradients
            "window_decode"  the same attention for one query per sequence, cache in bf16 or (quant) in 4 bits
  batch, seq, seq_min        sequences, the longest and the shortest of them (lengths spread evenly between)
  hq, hkv                    query and key-value heads
  n, topk, tree              new or drafted tokens, blocks per query, random tree instead of a chain
  sink, window               first tokens that stay visible, tokens of the window (the query's own among them)
  quant, heavy               4-bit cache; keys with log-normal norms

The 4-bit cache keeps a row of 128 channels as 64 bytes of codes (channel 2 c in the low half of byte c) and 4 bytes of
exponents.  A code is sign and index into 0, 0.5, 1, 1.5, 2, 3, 4, 6; 32 channels share the scale 2^(byte - 127).  The
exponent is that of the group's largest magnitude rounded to two significant bits, less 2 (so nothing is clipped), at
least 2; a group with an infinity or a NaN has byte 255 and reads back NaN.
"""
import math

import torch

own = False

D, BLOCK, GROUP = 128, 64, 32
KERNEL, STRIDE = 32, 16                        # tokens of a semantic kernel, their stride

_FIELDS = dict(kind="", batch=1, seq=0, seq_min=0, hq=32, hkv=2, n=0, topk=16, tree=False, sink=0, window=0, quant=False,
               heavy=False)


def _case(**kw):
    c = dict(_FIELDS, **kw)
    c["seq_min"] = c["seq_min"] or c["seq"]
    return c


def listed():
    return [
        # the next token of one chat on a small model: launches and latency count
        _case(name="append_b1", kind="append", seq=2016, hq=4, hkv=1, n=1),
        # the drafted tokens of a ragged serving batch
        _case(name="append_ragged_b8_n16", kind="append", batch=8, seq=8191, seq_min=77, n=16),
        # a long document's cache after its prompt
        _case(name="quantize_128k", kind="quantize", seq=131071),
        # the next token of a 128K document
        _case(name="sparse_quant_128k", kind="sparse_quant", seq=131047),
        # a full serving batch of ragged documents with many blocks: the bandwidth end
        _case(name="sparse_quant_b32", kind="sparse_quant", batch=32, seq=65521, seq_min=30011, topk=64, heavy=True),
        # speculative decoding: 16 drafted tokens of a tree
        _case(name="sparse_quant_n16", kind="sparse_quant", batch=2, seq=32749, n=16, topk=32, tree=True),
        # a short prompt on a small model
        _case(name="window_777_g4", kind="window", seq=777, hq=4, hkv=1, sink=4, window=256),
        # a long document
        _case(name="window_32k", kind="window", seq=32768, sink=64, window=4096),
        # fine-tuning on two short ragged sequences, eight query heads per key-value head
        _case(name="window_bwd_4k_g8", kind="window_bwd", batch=2, seq=4096, seq_min=3333, hq=16, sink=4, window=1000),
        # a long document's training step
        _case(name="window_bwd_32k", kind="window_bwd", seq=32768, sink=64, window=4096),
        # the next token of one long chat, cache in bf16
        _case(name="window_decode_b1", kind="window_decode", seq=20011, sink=4, window=4096),
        # a serving batch on the 4-bit cache with a long window
        _case(name="window_decode_quant_b64", kind="window_decode", batch=64, seq=32749, seq_min=1501, sink=128, window=8192,
              quant=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    kind = rng.choice(["append", "quantize", "sparse_quant", "sparse_quant", "window", "window", "window_bwd", "window_bwd",
                       "window_decode", "window_decode"])
    group, hkv = rng.choice([16, 16, 8, 4, 2, 1]), rng.choice([1, 2, 2, 4])
    c = dict(kind=kind, hq=group * hkv, hkv=hkv, heavy=rng.random() < 0.25)
    if kind in ("append", "sparse_quant", "window_decode"):
        c["seq"] = _log_int(rng, 100, {"append": 16384, "sparse_quant": 131072, "window_decode": 65536}[kind])
        c["batch"] = _log_int(rng, 1, {"append": max(1, min(32, 131072 // (c["seq"] * hkv))), "sparse_quant": min(32, max(1, 4194304 // (c["seq"] * hkv))),
                                       "window_decode": min(64, max(1, 4194304 // (c["seq"] * hkv)))}[kind])
        if kind == "append":
            c["n"] = rng.choice([1, 1, 2, 5, 16, 33, 64])
        elif kind == "sparse_quant":
            c["topk"] = rng.choice([8, 12, 16, 32, 48, 64])
            if c["batch"] <= 4 and rng.random() < 0.4:
                c.update(n=rng.choice([2, 5, 16, 31, 64]), tree=rng.random() < 0.7)
        else:
            c["quant"] = rng.random() < 0.5
    else:
        c["seq"] = _log_int(rng, 65, {"quantize": 131072, "window": 32768, "window_bwd": 32768}[kind] * 2 // hkv // (2 if hkv == 1 else 1))
        c["batch"] = rng.choice([1, 2, 3, 4]) if c["seq"] * hkv <= 8192 else 1
    if kind.startswith("window"):
        c["sink"] = rng.choice([0, 1, 4, 64, 100, 128])
        c["window"] = _log_int(rng, 1, 8192 if kind == "window_decode" else 4096)
    if c.get("batch", 1) > 1 and rng.random() < 0.8:
        c["seq_min"] = rng.randint(max(1, c["seq"] // 8), c["seq"])
    if c.get("n"):                                               # a sequence holds its new tokens
        c["seq"] = max(c["seq"], c["n"])
        c["seq_min"] = max(c.get("seq_min", 0), c["n"]) if c.get("seq_min") else 0
    return _case(**c)


# ---- what a case means -----------------------------------------------------------------------------------------

def _lengths(c):
    b = c["batch"]
    return [c["seq"]] if b == 1 else [c["seq"] - (c["seq"] - c["seq_min"]) * i // (b - 1) for i in range(b)]


def _kernels(n):
    return 0 if n < KERNEL else (n - KERNEL) // STRIDE + 1


def _visible(c, length):
    """Keys seen by the queries of a sequence, summed over them."""
    full = min(c["window"], length)
    pairs = full * (full + 1) // 2 + (length - full) * full
    beyond = length - full                                       # queries with keys before their window: 1, 2, .. of them
    ramp = min(c["sink"], beyond)
    return pairs + ramp * (ramp + 1) // 2 + (beyond - ramp) * ramp


# ---- the 4-bit format, plainly -----------------------------------------------------------------------------------

_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _encode(x):
    """fp32 [.., 128] -> codes uint8 [.., 64], exponents uint8 [.., 4]"""
    g = x.reshape(*x.shape[:-1], D // GROUP, GROUP)
    most = g.abs().amax(-1)
    exponent = ((most.view(torch.int32) + (1 << 21)) >> 23).clamp(min=4) - 2
    finite = torch.isfinite(g).all(-1)
    exponent = torch.where(finite, exponent, 255)
    y = torch.ldexp(g.abs(), (127 - exponent)[..., None])        # below 7
    index = torch.where(y < 2, torch.round(2 * y), torch.where(y < 4, torch.round(y) + 2, torch.round(y * 0.5) + 4))
    index = torch.where(finite[..., None], index, 0.0).to(torch.uint8) | (torch.signbit(g).to(torch.uint8) << 3)
    index = index.reshape(*x.shape[:-1], D // 2, 2)
    return index[..., 0] | (index[..., 1] << 4), exponent.to(torch.uint8)


def _decode(codes, exponents):
    """the values they stand for, fp32 [.., 128]"""
    table = torch.tensor(_VALUES + tuple(-v for v in _VALUES), dtype=torch.float32, device=codes.device)
    v = table[torch.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], D // GROUP, GROUP).long()]
    e = exponents.int()
    scale = torch.where(e == 255, float("nan"), torch.ldexp(torch.ones_like(e, dtype=torch.float32), e - 127))
    return (v * scale[..., None]).reshape(*codes.shape[:-1], D)


def _encode_cache(x):
    """bf16 [B, H, T, 128] -> (codes, exponents), in pieces"""
    codes = torch.zeros((*x.shape[:-1], D // 2), dtype=torch.uint8, device=x.device)
    exps = torch.zeros((*x.shape[:-1], D // GROUP), dtype=torch.uint8, device=x.device)
    for b in range(x.shape[0]):
        for t in range(0, x.shape[2], 65536):
            codes[b, :, t:t + 65536], exps[b, :, t:t + 65536] = _encode(x[b, :, t:t + 65536].float())
    return codes, exps


# ---- inputs ----------------------------------------------------------------------------------------------------

def _normal(shape, gen):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _cache(c, cap, lengths, gen):
    """k, v [B, Hkv, cap, D]; rows behind a sequence are 0"""
    out = []
    for _ in range(2):
        x = torch.zeros((c["batch"], c["hkv"], cap, D), dtype=torch.bfloat16, device="cuda")
        for b, n in enumerate(lengths):
            x[b, :, :n].normal_(generator=gen)
        out.append(x)
    if c["heavy"]:
        for b, n in enumerate(lengths):
            z = torch.randn((c["hkv"], n, 1), generator=gen, device="cuda")
            out[0][b, :, :n] = (out[0][b, :, :n].float() * torch.exp(0.5 * z)).bfloat16()
    return out


def _block_lists(c, lengths, rows, gen):
    """[B, Hkv, rows, topk]: the first block, the query's own and the one before it, and others by random scores that the
    rows of a sequence mostly share; ascending, padded with -1"""
    idx = torch.full((c["batch"], c["hkv"], rows, c["topk"]), -1, dtype=torch.int32, device="cuda")
    for b, length in enumerate(lengths):
        blocks = (length + BLOCK - 1) // BLOCK
        score = torch.rand((c["hkv"], 1, blocks), generator=gen, device="cuda") + \
            0.05 * torch.rand((c["hkv"], rows, blocks), generator=gen, device="cuda")
        last = (torch.arange(length - rows, length, device="cuda") // BLOCK)[:, None]
        at = torch.arange(blocks, device="cuda")[None, :]
        score = torch.where((at == 0) | (at >= last - 1), 9.0, score)
        score = torch.where(at > last, -1.0, score)
        best, which = score.topk(min(c["topk"], blocks), dim=-1)
        which = torch.where(best < 0, blocks, which).sort(-1)[0]
        idx[b, :, :, :which.shape[-1]] = torch.where(which == blocks, -1, which).int()
    return idx


def _tree(c, gen):
    """mask words [B, n]: a token sees itself and its ancestors"""
    b, n = c["batch"], c["n"]
    parents = torch.rand((b, n), generator=gen, device="cuda").tolist()
    words = []
    for row in parents:
        seen = []
        for t in range(n):
            seen.append((seen[int(row[t] * t)] if t else 0) | 1 << t)
        words.append([w - (1 << 64) if w >> 63 else w for w in seen])
    return torch.tensor(words, dtype=torch.int64, device="cuda")


def prepare(case, seed):
    c = dict(_FIELDS, **case)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    lengths, kind, b = _lengths(c), c["kind"], c["batch"]
    s = {"c": c, "lengths": lengths, "sl": torch.tensor(lengths, dtype=torch.int32, device="cuda")}
    cap = s["cap"] = c["seq"]
    if kind == "quantize":
        s["k"], s["v"] = _cache(c, cap, lengths, gen)
    elif kind == "append":
        k, v = _cache(c, cap, [x - c["n"] for x in lengths], gen)
        s["kq"], s["vq"] = _encode_cache(k), _encode_cache(v)
        s["k_new"], s["v_new"] = (_normal((b, c["hkv"], c["n"], D), gen) for _ in range(2))
        s["ck"] = torch.zeros((b, c["hkv"], max(1, _kernels(cap)), D), dtype=torch.bfloat16, device="cuda")
        for i, x in enumerate(lengths):
            for h in range(c["hkv"]):
                m = _kernels(x - c["n"])
                if m:
                    s["ck"][i, h, :m] = k[i, h, :x - c["n"]].double().unfold(0, KERNEL, STRIDE).mean(-1).bfloat16()
        s["k"], s["v"] = torch.zeros_like(k), torch.zeros_like(v)          # where the new rows are read back
    elif kind == "sparse_quant":
        k, v = _cache(c, cap, lengths, gen)
        s["kq"], s["vq"] = _encode_cache(k), _encode_cache(v)
        rows = max(1, c["n"])
        s["q"] = _normal((b, rows, c["hq"], D), gen)
        s["idx"] = _block_lists(c, lengths, rows, gen)
        s["mask"] = _tree(c, gen) if c["tree"] else None
    else:
        s["k"], s["v"] = _cache(c, cap, lengths, gen)
        rows = 1 if kind == "window_decode" else cap
        s["q"] = _normal((b, rows, c["hq"], D), gen)
        if kind == "window_decode" and c["quant"]:
            s["kq"], s["vq"] = _encode_cache(s.pop("k")), _encode_cache(s.pop("v"))
        if kind == "window_bwd":
            s["dout"] = _normal((b, rows, c["hq"], D), gen)
            s["out"], s["lse"] = _window(s)                      # the finished forward
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """what a program that uses the framework holds besides: parameters, and for serving its buffers and workspace"""
    from paper_2506_07900_amd import binding
    c = s["c"]
    prm = s["prm"] = binding.Params(c["hq"], c["hkv"], topk=c["topk"])
    for name in ("kq", "vq"):
        if name in s:
            s[name] = binding.QuantCache(*s[name])
    keep = s["keep"] = {}
    if c["kind"] in ("sparse_quant", "window_decode"):
        need = (binding.window_workspace_bytes(binding.OP_WINDOW_DECODE, prm, c["sink"], c["window"], c["batch"], s["cap"])
                if c["kind"] == "window_decode" else
                binding.verify_workspace_bytes(binding.OP_ATTN_VERIFY, prm, c["batch"], s["cap"], max(1, c["n"])))
        keep["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        keep["out"] = torch.zeros_like(s["q"])
        keep["lse"] = torch.zeros((c["batch"], c["n"], c["hq"]) if c["n"] else (c["batch"], c["hq"]), dtype=torch.float32,
                                  device="cuda")


# ---- one pass --------------------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _PLAIN[state["c"]["kind"]](state)


def _run_own(s):
    from paper_2506_07900_amd import binding
    c, cap, sl, prm, keep = s["c"], s["cap"], s["sl"], s["prm"], s["keep"]
    kind = c["kind"]
    if kind == "quantize":
        kq, vq = binding.quantize_kv(prm, s["k"], s["v"], sl, cap)
        return binding.dequantize_kv(prm, kq, vq, sl, cap)
    if kind == "append":
        binding.append_kv_quant(prm, s["k_new"], s["v_new"], s["kq"], s["vq"], sl, cap, ck=s["ck"])
        k, v = binding.dequantize_kv(prm, s["kq"], s["vq"], sl, cap, k=s["k"], v=s["v"], n_new_tokens=c["n"])
        return k, v, s["ck"]
    if kind == "sparse_quant":
        if c["n"]:
            return binding.sparse_attn_verify_quant(prm, s["q"], s["kq"], s["vq"], sl, cap, s["idx"], tree_mask=s["mask"], **keep)
        return binding.sparse_attn_decode_quant(prm, s["q"], s["kq"], s["vq"], sl, cap, s["idx"], **keep)
    if kind == "window":
        return binding.window_attn_prefill(prm, c["sink"], c["window"], s["q"], s["k"], s["v"], sl, cap)
    if kind == "window_bwd":
        return binding.window_attn_bwd(prm, c["sink"], c["window"], s["q"], s["k"], s["v"], s["out"], s["dout"], s["lse"], sl, cap)
    if c["quant"]:
        return binding.window_attn_decode_quant(prm, c["sink"], c["window"], s["q"], s["kq"], s["vq"], sl, cap, **keep)
    return binding.window_attn_decode(prm, c["sink"], c["window"], s["q"], s["k"], s["v"], sl, cap, **keep)


# ---- the plain forms, in 32 bits -----------------------------------------------------------------------------------

def _quantize(s):
    k, v = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
    for b, n in enumerate(s["lengths"]):
        for src, dst in ((s["k"], k), (s["v"], v)):
            dst[b, :, :n] = _decode(*_encode(src[b, :, :n].float())).bfloat16()
    return k, v


def _append(s):
    c, n = s["c"], s["c"]["n"]
    for new, (codes, exps), back in ((s["k_new"], s["kq"], s["k"]), (s["v_new"], s["vq"], s["v"])):
        new_codes, new_exps = _encode(new.float())
        values = _decode(new_codes, new_exps).bfloat16()
        for b, length in enumerate(s["lengths"]):
            codes[b, :, length - n:length], exps[b, :, length - n:length] = new_codes[b], new_exps[b]
            back[b, :, length - n:length] = values[b]
    for b, length in enumerate(s["lengths"]):
        for j in range(_kernels(length - n), _kernels(length)):  # sums of 32 values: in 64 bits
            rows = slice(j * STRIDE, j * STRIDE + KERNEL)
            s["ck"][b, :, j] = _decode(s["kq"][0][b, :, rows], s["kq"][1][b, :, rows]).double().mean(1).bfloat16()
    return s["k"], s["v"], s["ck"]


def _softmax_product(score, seen, value):
    """score, seen [.., R, K], value [.., K, D] -> out [.., R, D], lse [.., R]; a row that sees nothing: 0, -inf"""
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    base = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - base)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, value) / torch.where(total > 0, total, 1.0)
    return out, (base + torch.log(total))[..., 0]


def _sparse_quant(s):
    c, cap, n = s["c"], s["cap"], max(1, s["c"]["n"])
    group = c["hq"] // c["hkv"]
    out = torch.zeros_like(s["q"])
    lse = torch.full((c["batch"], n, c["hq"]), -math.inf, dtype=torch.float32, device="cuda")
    for b, length in enumerate(s["lengths"]):
        idx = s["idx"][b].long()                                                       # [Hkv, n, topk]
        tokens = (idx[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")).flatten(-2)
        first = length - n
        pos = torch.arange(first, length, device="cuda")[None, :, None]
        if s["mask"] is None:
            seen = tokens <= pos
        else:
            bit = (s["mask"][b][None, :, None] >> (tokens - first).clamp(0, 63)) & 1
            seen = (tokens < first) | ((tokens < length) & (bit == 1))
        seen &= (idx >= 0).repeat_interleave(BLOCK, -1)
        at = tokens.clamp(0, cap - 1)
        heads = torch.arange(c["hkv"], device="cuda")[:, None, None]
        k, v = (_decode(x[0][b][heads, at], x[1][b][heads, at]) for x in (s["kq"], s["vq"]))     # [Hkv, n, K, D]
        v = torch.where(seen[..., None], v, 0.0)
        q = s["q"][b].float().reshape(n, c["hkv"], group, D).transpose(0, 1)           # [Hkv, n, G, D]
        score = torch.matmul(q, k.transpose(-1, -2).contiguous()) * D ** -0.5
        o, z = _softmax_product(score, seen[:, :, None], v)
        out[b] = o.transpose(0, 1).reshape(n, c["hq"], D).bfloat16()
        lse[b] = z.transpose(0, 1).reshape(n, c["hq"])
    return out, lse if c["n"] else lse[:, 0]


def _window_keys(c, i0, i1):
    """token numbers of the keys that queries i0 .. i1-1 see among them, and who sees which"""
    lo = max(0, i0 - c["window"] + 1)
    t = torch.cat((torch.arange(0, min(c["sink"], lo), device="cuda"), torch.arange(lo, i1, device="cuda")))
    i = torch.arange(i0, i1, device="cuda")[:, None]
    return t, (t[None] <= i) & ((t[None] < c["sink"]) | (i - t[None] < c["window"]))


def _window_pieces(c, length, step=512):
    for i0 in range(0, length, step):
        i1 = min(length, i0 + step)
        t, seen = _window_keys(c, i0, i1)
        yield i0, i1, t, seen


def _window(s):
    c, group = s["c"], s["c"]["hq"] // s["c"]["hkv"]
    out = torch.zeros_like(s["q"])
    lse = torch.zeros((c["batch"], s["cap"], c["hq"]), dtype=torch.float32, device="cuda")
    for b, length in enumerate(s["lengths"]):
        for i0, i1, t, seen in _window_pieces(c, length):
            for h in range(c["hkv"]):
                heads = slice(h * group, (h + 1) * group)
                k, v = s["k"][b, h, t].float(), s["v"][b, h, t].float()
                q = s["q"][b, i0:i1, heads].float().transpose(0, 1)                    # [G, R, D]
                o, z = _softmax_product(torch.matmul(q, k.t().contiguous()) * D ** -0.5, seen, v)
                out[b, i0:i1, heads] = o.transpose(0, 1).bfloat16()
                lse[b, i0:i1, heads] = z.t()
    return out, lse


def _window_bwd(s):
    c, group = s["c"], s["c"]["hq"] // s["c"]["hkv"]
    dq = torch.zeros_like(s["q"])
    dk, dv = (torch.zeros(s["k"].shape, dtype=torch.float32, device="cuda") for _ in range(2))
    for b, length in enumerate(s["lengths"]):
        for i0, i1, t, seen in _window_pieces(c, length):
            for h in range(c["hkv"]):
                heads = slice(h * group, (h + 1) * group)
                k, v = s["k"][b, h, t].float(), s["v"][b, h, t].float()
                q, do, o = (s[x][b, i0:i1, heads].float().transpose(0, 1) for x in ("q", "dout", "out"))
                score = torch.matmul(q, k.t().contiguous()) * D ** -0.5 - s["lse"][b, i0:i1, heads].t()[..., None]
                p = torch.where(seen, torch.exp(score), 0.0)
                ds = p * (torch.matmul(do, v.t().contiguous()) - (do * o).sum(-1, keepdim=True))
                dq[b, i0:i1, heads] = (torch.matmul(ds, k) * D ** -0.5).transpose(0, 1).bfloat16()
                rows = lambda x: x.reshape(-1, x.shape[-1])
                dk[b, h, t] += torch.matmul(rows(ds).t().contiguous(), rows(q)) * D ** -0.5
                dv[b, h, t] += torch.matmul(rows(p).t().contiguous(), rows(do))
    return dq, dk.bfloat16(), dv.bfloat16()


def _window_decode(s):
    c = s["c"]
    out = torch.zeros_like(s["q"])
    lse = torch.zeros((c["batch"], c["hq"]), dtype=torch.float32, device="cuda")
    for b, length in enumerate(s["lengths"]):
        t, seen = _window_keys(c, length - 1, length)
        if c["quant"]:
            k, v = (_decode(x[0][b][:, t], x[1][b][:, t]) for x in (s["kq"], s["vq"]))
        else:
            k, v = s["k"][b][:, t].float(), s["v"][b][:, t].float()
        q = s["q"][b, 0].float().reshape(c["hkv"], -1, D)
        o, z = _softmax_product(torch.matmul(q, k.transpose(-1, -2).contiguous()) * D ** -0.5, seen, v)
        out[b, 0] = o.reshape(c["hq"], D).bfloat16()
        lse[b] = z.reshape(c["hq"])
    return out, lse


_PLAIN = {"quantize": _quantize, "append": _append, "sparse_quant": _sparse_quant, "window": _window, "window_bwd": _window_bwd,
          "window_decode": _window_decode}


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def work(case):
    c = dict(_FIELDS, **case)
    kind, hq, hkv = c["kind"], c["hq"], c["hkv"]
    packed, wide = D // 2 + D // GROUP, 2 * D                    # bytes of a cache row in 4 bits and in bf16
    query = 2 * hq * 2 * D + 4 * hq                              # a query row, its output, its log-sum-exps
    bytes_ = flops = 0.0
    for length in _lengths(c):
        if kind == "quantize":                                   # read bf16, write 4 bits; read those, write bf16
            bytes_ += length * hkv * 2 * 2 * (packed + wide)
            flops += length * hkv * 2 * D * 4
        elif kind == "append":
            done = _kernels(length) - _kernels(length - c["n"])
            bytes_ += c["n"] * hkv * 2 * 2 * (packed + wide) + done * hkv * (wide + KERNEL * packed)
            flops += c["n"] * hkv * 2 * D * 4 + done * hkv * KERNEL * D
        elif kind == "sparse_quant":
            n = max(1, c["n"])
            blocks = min(c["topk"], (length + BLOCK - 1) // BLOCK)
            tokens = (blocks - 1) * BLOCK + (length - 1) % BLOCK + 1
            bytes_ += tokens * hkv * 2 * packed + n * (query + 4 * hkv * c["topk"] + (8 if c["tree"] else 0))
            flops += n * tokens * hq * 4.0 * D
        elif kind == "window_decode":
            tokens = min(length, c["window"]) + min(c["sink"], max(0, length - c["window"]))
            bytes_ += tokens * hkv * 2 * (packed if c["quant"] else wide) + query
            flops += tokens * hq * 4.0 * D
        else:
            products = 10.0 if kind == "window_bwd" else 4.0
            flops += _visible(c, length) * hq * products * D
            bytes_ += length * (query + hkv * 2 * wide)
            if kind == "window_bwd":                             # q, out, dout, lse, k, v in; dq, dk, dv out
                bytes_ += length * (hq * 2 * wide + hkv * 2 * wide)
    return {"bytes": bytes_, "flops": flops}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _nearest(x):
    """the values a row reads back as: of each group's grid the nearest point, of two the one with the even index"""
    x = x.double()
    shape = x.shape
    x = x.reshape(-1, GROUP)
    most = x.abs().amax(-1)
    fraction, e = torch.frexp(most)                              # most = fraction 2^e, 0.5 <= fraction < 1
    e = torch.where(fraction >= 0.875, e, e - 1)                 # 1.75 and more round up to the next power of two
    step = torch.where(most > 0, 2.0 ** (e.double() - 2), 2.0 ** -125.0).clamp(min=2.0 ** -125.0)
    grid = torch.tensor(_VALUES, dtype=torch.float64, device=x.device)
    y = x.abs() / step[:, None]
    upper = torch.searchsorted(grid, y.contiguous()).clamp(1, 7)
    below, above = y - grid[upper - 1], grid[upper] - y
    take = torch.where((below < above) | ((below == above) & ((upper - 1) % 2 == 0)), upper - 1, upper)
    value = grid[take] * step[:, None] * torch.where(x < 0, -1.0, 1.0)
    return torch.where(torch.isfinite(most)[:, None], value, math.nan).reshape(shape)


def _cache_values(x):
    """(codes, exponents) -> fp64 by the definition of a code"""
    codes, exps = x
    nibble = torch.stack((codes % 16, codes // 16), -1).flatten(-2).long()
    magnitude, negative = nibble % 8, nibble >= 8
    small = magnitude.double() / 2                               # indexes 0 to 3: half the index
    big = (2.0 + magnitude % 2) * 2.0 ** (magnitude // 2 - 2).double()   # 4 to 7: 2, 3, 4, 6
    value = torch.where(magnitude < 4, small, big)
    scale = 2.0 ** (exps.double() - 127)
    return torch.where(negative, -value, value) * scale.repeat_interleave(GROUP, -1)


def _attend64(q, k, v, seen):
    """q [R, D], k, v [K, D], seen [R, K]"""
    score = (q.double() @ k.double().t()) / math.sqrt(D)
    score.masked_fill_(~seen, -math.inf)
    z = torch.logsumexp(score, -1)
    p = torch.exp(score - torch.where(torch.isinf(z), torch.zeros_like(z), z)[:, None])
    return p @ v.double(), z


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c, lengths = s["c"], s["lengths"]
    kind, group = c["kind"], c["hq"] // c["hkv"]
    if kind == "quantize":
        k, v = (torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
        for b, n in enumerate(lengths):
            k[b, :, :n], v[b, :, :n] = _nearest(s["k"][b, :, :n]), _nearest(s["v"][b, :, :n])
        return k, v
    if kind == "append":
        k, v, ck = s["k"].double(), s["v"].double(), s["ck"].double()
        cached = _cache_values(s["kq"])
        for b, length in enumerate(lengths):
            first = length - c["n"]
            k[b, :, first:length], v[b, :, first:length] = _nearest(s["k_new"][b]), _nearest(s["v_new"][b])
            whole = torch.cat((cached[b, :, :first], k[b, :, first:length]), 1)
            for j in range(_kernels(first), _kernels(length)):
                ck[b, :, j] = whole[:, j * STRIDE:j * STRIDE + KERNEL].sum(1) / KERNEL
        return k, v, ck
    rows = s["q"].shape[1]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((c["batch"], rows, c["hq"]), dtype=torch.float64, device="cuda")
    if kind == "sparse_quant":
        for b, length in enumerate(lengths):
            t = torch.arange(length, device="cuda")
            for h in range(c["hkv"]):
                for i in range(rows):
                    pos = length - rows + i
                    chosen = torch.zeros((length + BLOCK - 1) // BLOCK, dtype=torch.bool, device="cuda")
                    listed_ = s["idx"][b, h, i]
                    chosen[listed_[listed_ >= 0].long()] = True
                    seen = chosen[t // BLOCK]
                    if s["mask"] is None:
                        seen &= t <= pos
                    else:
                        word = int(s["mask"][b, i]) % (1 << 64)
                        for j in range(rows):
                            if not word >> j & 1:
                                seen[length - rows + j] = False
                    at = t[seen]
                    k, v = (_cache_values((x[0][b, h, at], x[1][b, h, at])) for x in (s["kq"], s["vq"]))
                    heads = slice(h * group, (h + 1) * group)
                    out[b, i, heads], lse[b, i, heads] = _attend64(s["q"][b, i, heads], k, v,
                                                                   torch.ones((group, len(at)), dtype=torch.bool, device="cuda"))
        return out, lse if c["n"] else lse[:, 0]
    if kind == "window_decode":
        for b, length in enumerate(lengths):
            t = torch.arange(length, device="cuda")
            t = t[(t < c["sink"]) | (t > length - 1 - c["window"])]
            for h in range(c["hkv"]):
                k, v = (_cache_values((s[x + "q"][0][b, h, t], s[x + "q"][1][b, h, t])) if c["quant"] else s[x][b, h, t]
                        for x in "kv")
                heads = slice(h * group, (h + 1) * group)
                out[b, 0, heads], lse[b, 0, heads] = _attend64(s["q"][b, 0, heads], k, v,
                                                               torch.ones((group, len(t)), dtype=torch.bool, device="cuda"))
        return out, lse[:, 0]
    grads = [torch.zeros(s[x].shape, dtype=torch.float64, device="cuda") for x in "qkv"]
    for b, length in enumerate(lengths):
        for i0 in range(0, length, 1024):                        # queries i0 .. i1-1 and all keys any of them sees
            i1 = min(length, i0 + 1024)
            t = torch.arange(i1, device="cuda")
            t = t[(t < c["sink"]) | (t > i0 - c["window"])]
            age = torch.arange(i0, i1, device="cuda")[:, None] - t[None]
            seen = (age >= 0) & ((age < c["window"]) | (t[None] < c["sink"]))
            for hq in range(c["hq"]):
                h = hq // group
                q, k, v = s["q"][b, i0:i1, hq], s["k"][b, h, t], s["v"][b, h, t]
                if kind == "window":
                    out[b, i0:i1, hq], lse[b, i0:i1, hq] = _attend64(q, k, v, seen)
                    continue
                q, k, v, do, o = (x.double() for x in (q, k, v, s["dout"][b, i0:i1, hq], s["out"][b, i0:i1, hq]))
                p = torch.exp((q @ k.t()) / math.sqrt(D) - s["lse"][b, i0:i1, hq].double()[:, None])
                p.masked_fill_(~seen, 0.0)
                ds = p * (do @ v.t() - torch.linalg.vecdot(do, o)[:, None]) / math.sqrt(D)
                grads[0][b, i0:i1, hq] = ds @ k
                grads[1][b, h, t] += ds.t() @ q
                grads[2][b, h, t] += p.t() @ do
    return tuple(grads) if kind == "window_bwd" else (out, lse)
