"""Measurable cases of the operators around the verification step: what fills the KV cache, keeps it in eight bits, and attends over it.

Four operators.  `append` writes new tokens' K and V rows into a cache, as they are or as e4m3 codes with one power-of-two scale per
(slot, KV head); `read` brings slots back as dense rows; `attn` is the attention of a chunk of new tokens (or a draft tree) over the
cache that holds them; `compact` moves an accepted path's rows and scales.  Where `own` is false, `run` computes the plain form in 32
bits with elementary torch operations; where it is true, it makes the calls of this library.  Sizes are those of the workload
configurations or generic ones between and beyond them; all inputs are synthetic and made on the GPU.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
PAGE = 16
WORKSPACE = 64 << 20           # bytes a program keeps for attention calls of any shape
STALE_CODE, STALE_SCALE = 0x7F, 255


def listed():
    return [
        # one request without a draft, early in its answer: a single token over a short prefix, latency only
        {"name": "decode_one_short", "kind": "attn", "cache": "bf16", "paged": False, "q_heads": 32, "kv_heads": 32, "head_dim": 128,
         "new": "1", "width": 1, "prefix": "768", "tree": False},
        # continuous batching: sixteen single tokens over prefixes of very different lengths, grouped heads, cache in eight bits
        {"name": "decode_batch_e4m3", "kind": "attn", "cache": "e4m3", "paged": True, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "new": "1,1,1,1,1,1,1,1,1,1,1,1,1,1,1,1", "width": 1,
         "prefix": "4864,3264,768,12001,906,16383,2048,170,9000,350,5120,287,7333,64,1311,2999", "tree": False},
        # one token at the end of a very long prefix, a few KV heads: everything depends on dividing the keys
        {"name": "decode_long", "kind": "attn", "cache": "bf16", "paged": True, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "new": "1", "width": 1, "prefix": "131000", "tree": False},
        # the first chunk of a 7B-shaped target: 2880 visual and 128 text tokens into an empty contiguous cache
        {"name": "chunk_first", "kind": "attn", "cache": "bf16", "paged": False, "q_heads": 32, "kv_heads": 32, "head_dim": 128,
         "new": "3008", "width": 3008, "prefix": "0", "tree": False},
        # chunks of four requests behind long prefixes, one nearly done and one idle, grouped heads, cache in eight bits
        {"name": "chunk_batch_e4m3", "kind": "attn", "cache": "e4m3", "paged": True, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "new": "1024,1024,0,333", "width": 1024, "prefix": "4096,7001,3264,5120", "tree": False},
        # the draft trees of four requests of 8 frames each, 13B-shaped target, cache in eight bits
        {"name": "tree_paged_e4m3", "kind": "attn", "cache": "e4m3", "paged": True, "q_heads": 40, "kv_heads": 40, "head_dim": 128,
         "new": "60,60,60,60", "width": 60, "prefix": "4864,4864,4864,4864", "tree": True},
        # a decoding step's new rows of eight requests, quantised as they are written
        {"name": "append_step_e4m3", "kind": "append", "dtype": "bf16", "cache": "e4m3", "paged": True, "q_heads": 32, "kv_heads": 8,
         "head_dim": 128, "new": "1,1,1,1,1,1,1,1", "width": 1, "prefix": "4864,3264,768,1201,906,2048,170,999"},
        # the rows of four requests' visual prefixes, 7B-shaped, out of the projection's fused buffer
        {"name": "append_prefix_e4m3", "kind": "append", "dtype": "bf16", "cache": "e4m3", "paged": True, "q_heads": 32, "kv_heads": 32,
         "head_dim": 128, "new": "2880,2880,576,2111", "width": 2880, "prefix": "0,33,0,128"},
        # one small image's slots back into dense rows
        {"name": "read_small", "kind": "read", "dtype": "bf16", "cache": "e4m3", "paged": True, "kv_heads": 32, "head_dim": 128,
         "count": "576", "width": 576, "start": "0"},
        # eight requests' visual prefixes back into dense rows, of different lengths and behind different starts
        {"name": "read_batch", "kind": "read", "dtype": "bf16", "cache": "e4m3", "paged": True, "kv_heads": 40, "head_dim": 128,
         "count": "4608,4608,2880,4608,576,4608,1153,4608", "width": 4608, "start": "0,35,0,7,0,0,64,0"},
        # the accepted path of one request in all layers of a contiguous eight-bit cache
        {"name": "compact_one_e4m3", "kind": "compact", "layers": 32, "paged": False, "kv_heads": 32, "head_dim": 128, "nodes": 60,
         "cap": 8, "prefix": "3264"},
        # the accepted paths of eight ragged requests, paged
        {"name": "compact_batch_e4m3", "kind": "compact", "layers": 32, "paged": True, "kv_heads": 32, "head_dim": 128, "nodes": 60,
         "cap": 8, "prefix": "170,390,253,339,350,906,365,287"},
    ]


def _log_int(rng, lo, hi):
    """A whole number of lo .. hi, spread over its logarithm (0 among them where lo is 0)."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi)))) - (lo == 0))))


def _join(numbers):
    return ",".join(str(n) for n in numbers)


def _numbers(text):
    return [int(n) for n in text.split(",")]


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "attn", "append", "append", "read", "compact"])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 8, 16, 32, 40])
    group = rng.choice([g for g in (1, 1, 2, 4, 5, 7, 8) if kv_heads * g <= 64])
    head_dim = rng.choice([64, 128, 128])
    paged = rng.random() < 0.6
    cache = rng.choice(["bf16", "e4m3"])
    batch = _log_int(rng, 1, 16)
    if kind == "attn":
        tree = rng.random() < 0.2
        width = rng.randint(2, 64) if tree else 1 if rng.random() < 0.35 else _log_int(rng, 2, 2048)
        longest = _log_int(rng, 0, 32768)
        spread = rng.random() < 0.5
        prefix = [_log_int(rng, 0, longest) if spread and longest else longest for _ in range(batch)]
        new = [width if rng.random() < 0.6 else rng.randint(1, width) for _ in range(batch)]
        if batch > 1 and rng.random() < 0.3:
            new[rng.randrange(batch)] = 0
        # no more than the largest listed ones: products, bytes of the cache, scores of the plain form
        while len(prefix) > 1 and (len(prefix) * width * (max(prefix) + width) * kv_heads * group > 7.0e8
                                   or len(prefix) * (max(prefix) + width) * kv_heads * head_dim > 2.5e8):
            prefix.pop()
            new.pop()
        while width * (max(prefix) + width) * kv_heads * group > 7.0e8:
            prefix = [prefix[0] // 2]
            width = max(2, width // 2)
            new = [min(new[0], width)]
        new[0] = width
        return {"kind": kind, "cache": cache, "paged": paged, "q_heads": kv_heads * group, "kv_heads": kv_heads, "head_dim": head_dim,
                "new": _join(new), "width": width, "prefix": _join(prefix), "tree": tree}
    if kind == "append":
        width = 1 if rng.random() < 0.3 else _log_int(rng, 2, 4096)
        while batch > 1 and batch * width * kv_heads > 280000:
            batch -= 1
        prefix = [_log_int(rng, 0, 6000) for _ in range(batch)]
        new = [width] + [rng.randint(0, width) for _ in range(batch - 1)]
        return {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f32"]), "cache": rng.choice(["e4m3", "e4m3", "same"]), "paged": paged,
                "q_heads": kv_heads * group, "kv_heads": kv_heads, "head_dim": head_dim, "new": _join(new), "width": width,
                "prefix": _join(prefix)}
    if kind == "read":
        width = _log_int(rng, 1, 4608)
        while batch > 1 and batch * width * kv_heads > 700000:
            batch -= 1
        count = [width] + [rng.randint(0, width) for _ in range(batch - 1)]
        return {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f32"]), "cache": rng.choice(["e4m3", "e4m3", "same"]), "paged": paged,
                "kv_heads": kv_heads, "head_dim": head_dim, "count": _join(count), "width": width,
                "start": _join(_log_int(rng, 0, 500) for _ in range(batch))}
    batch = min(batch, 8)
    prefix = [_log_int(rng, 0, 2000) for _ in range(batch)]
    layers = _log_int(rng, 1, 40)
    while layers > 1 and layers * batch * (max(prefix) + 64) * kv_heads * head_dim > 4.0e8:
        layers -= 1
    return {"kind": kind, "layers": layers, "paged": paged, "kv_heads": kv_heads, "head_dim": head_dim, "nodes": rng.randint(8, 64),
            "cap": rng.randint(2, 9), "prefix": _join(prefix)}


# ---- inputs ------------------------------------------------------------------------------------------
def _i32(numbers):
    return torch.tensor(numbers, dtype=torch.int32, device=DEV)


def _normal(gen, shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, 1.0, generator=gen)


def _rows(gen, rows, heads, dim, dtype, keys):
    """K or V rows [rows, heads, dim]: K has a few channels that are far from zero in every token, V a small mean."""
    mean = _normal(gen, (1, heads, dim), torch.float32)
    return (_normal(gen, (rows, heads, dim), torch.float32).add_(0.5 * mean ** 3 if keys else 0.3 * mean)).to(dtype)


def _two_to(e):
    """2^e in 32 bits for whole e of -126 .. 127, put together from its bits (a power function may be off by a rounding)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """(codes, exponent bytes) of rows x [..., D]: e is the smallest whole number, -100 at least, with max |x| <= 448 * 2^e over the
    row's finite entries; codes are x * 2^-e rounded to e4m3, a code for NaN where x is not finite."""
    x = x.float()
    finite = torch.isfinite(x)
    m, k = torch.frexp(torch.where(finite, x, 0.0).abs().amax(dim=-1, keepdim=True))
    e = torch.where(m == 0, -100, torch.where(m <= 0.875, k - 9, k - 8)).clamp_(min=-100)
    y = x * _two_to(-e)
    y = torch.where((e == 120) & finite, y.clamp(-240.0, 240.0), y)        # (256 * 2^120 would be an infinity)
    return torch.where(finite, y, float("nan")).to(torch.float8_e4m3fn), (e[..., 0] + 127).to(torch.uint8)


def _values(codes, scale):
    if scale is None:
        return codes.float()
    return codes.float() * (scale.int() << 23).view(torch.float32)[..., None]


def _bytes(t):
    """The same memory as whole numbers of its element size (float8 tensors are moved and indexed as such)."""
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _table(gen, need, spare):
    """Block table [B, most blocks] over a pool in random order; entries a request does not use are -1."""
    blocks = [-(-n // PAGE) for n in need]
    pool = sum(blocks) + spare
    order = torch.randperm(pool, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((len(need), max(max(blocks), 1)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at:at + n]
        at += n
    return table, pool


def _cache(gen, case, need, dtype, layers=None, filled=None):
    """K and V caches for requests of need[b] slots, of which filled[b] (all) hold tokens; every other slot holds what is no number."""
    heads, dim = case["kv_heads"], case["head_dim"]
    filled = need if filled is None else filled
    if case["paged"]:
        table, pool = _table(gen, need, 1 + sum(need) // (10 * PAGE))
        rows, per = pool, PAGE
        used = torch.zeros((pool, PAGE), dtype=torch.bool, device=DEV)
        slots = torch.arange(table.shape[1] * PAGE, device=DEV)
        live = slots[None] < _i32(filled)[:, None]
        used.view(-1)[(table.long().repeat_interleave(PAGE, dim=1) * PAGE + slots % PAGE)[live]] = True
    else:
        table, rows, per = None, len(need), -(-max(need) // PAGE) * PAGE
        used = torch.arange(per, device=DEV)[None] < _i32(filled)[:, None]
    out = []
    for keys in (True, False):
        made = []
        for _ in range(layers or 1):
            x = _rows(gen, rows * per, heads, dim, torch.bfloat16 if dtype == "e4m3" else TYPES[dtype], keys)
            x = x.view(rows, per, heads, dim).permute(0, 2, 1, 3)
            if dtype == "e4m3":
                codes, scale = _quantise(x)
                codes = codes.view(torch.uint8).masked_fill_(~used[:, None, :, None], STALE_CODE)
                made.append((codes.contiguous().view(torch.float8_e4m3fn), scale.masked_fill_(~used[:, None], STALE_SCALE).contiguous()))
            else:
                made.append((x.contiguous().masked_fill_(~used[:, None, :, None], float("nan")), None))
        if layers is None:
            out.append(made[0])
        else:
            codes = torch.stack([_bytes(m[0]) for m in made]).view(TYPES[dtype])
            out.append((codes, torch.stack([m[1] for m in made]) if dtype == "e4m3" else None))
    (k, ks), (v, vs) = out
    return {"k": k, "v": v, "ks": ks, "vs": vs, "table": table}


def _tree(gen, nodes):
    """Parents of a random draft tree, in level order near the root and deeper at the end."""
    at = torch.arange(nodes, device=DEV)
    back = 1 + (torch.rand(nodes, generator=gen, device=DEV) ** 2 * 10).long()
    return torch.where(at == 0, -1, (at - back).clamp(min=0)).to(torch.int32)


def _prepare_attn(case, gen):
    prefix, new = _numbers(case["prefix"]), _numbers(case["new"])
    B, N, H, D = len(prefix), case["width"], case["q_heads"], case["head_dim"]
    s = _cache(gen, case, [p + n for p, n in zip(prefix, new)], case["cache"])
    s.update(q=_normal(gen, (B, N, H, D)), out=_normal(gen, (B, N, H, D)), lse=_normal(gen, (B, H, N), torch.float32),
             prefix=_i32(prefix), new=_i32(new), err=_i32([0]),
             parent=torch.stack([_tree(gen, N) for _ in range(B)]) if case["tree"] else None,
             workspace=torch.zeros(WORKSPACE, dtype=torch.uint8, device=DEV))
    return s


def _prepare_append(case, gen):
    prefix, new = _numbers(case["prefix"]), _numbers(case["new"])
    B, N, D = len(prefix), case["width"], case["head_dim"]
    H, kept = case["q_heads"] + 2 * case["kv_heads"], case["kv_heads"]
    dtype = case["dtype"] if case["cache"] == "same" else case["cache"]
    s = _cache(gen, case, [p + n for p, n in zip(prefix, new)], dtype, filled=prefix)
    fused = _rows(gen, B * N, H, D, TYPES[case["dtype"]], True).view(B, N, H, D)           # a projection's q, k and v beside one another
    s.update(fused=fused, k_new=fused[:, :, -2 * kept:-kept], v_new=fused[:, :, -kept:], prefix=_i32(prefix), new=_i32(new), err=_i32([0]))
    return s


def _prepare_read(case, gen):
    start, count = _numbers(case["start"]), _numbers(case["count"])
    B, N = len(start), case["width"]
    dtype = case["dtype"] if case["cache"] == "same" else case["cache"]
    s = _cache(gen, case, [a + n for a, n in zip(start, count)], dtype)
    shape = (B, N, case["kv_heads"], case["head_dim"])
    s.update(start=_i32(start), count=_i32(count), err=_i32([0]), k_out=_normal(gen, shape, TYPES[case["dtype"]]),
             v_out=_normal(gen, shape, TYPES[case["dtype"]]))
    return s


def _prepare_compact(case, gen):
    prefix, N, cap = _numbers(case["prefix"]), case["nodes"], case["cap"]
    B = len(prefix)
    s = _cache(gen, case, [p + N for p in prefix], "e4m3", layers=case["layers"])
    # an accepted path of every length: node numbers that rise from the root's 0
    length = torch.randint(0, min(cap, N), (B,), generator=gen, device=DEV)
    length[0] = min(cap, N) - 1
    picked = torch.rand((B, N), generator=gen, device=DEV)
    picked[:, 0] = -1.0
    path = picked.argsort(dim=1)[:, :min(cap, N)]
    at = torch.arange(path.shape[1], device=DEV)[None]
    path = torch.where(at <= length[:, None], path, N).sort(dim=1).values
    path = torch.where(at <= length[:, None], path, -1)
    path = torch.cat([path, path.new_full((B, cap - path.shape[1]), -1)], dim=1)
    s.update(prefix=_i32(prefix), path=path.to(torch.int32), length=length.to(torch.int32), new_prefix=_i32([0] * B), err=_i32([0]))
    return s


_PREPARE = {"attn": _prepare_attn, "append": _prepare_append, "read": _prepare_read, "compact": _prepare_compact}


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = _PREPARE[case["kind"]](case, gen)
    s["case"] = case
    return s


# ---- the plain forms ---------------------------------------------------------------------------------
def _places(s, slots):
    """Row and slot within it of each request's logical slots [B, n]; a block that a request does not use counts as the pool's first."""
    if s["table"] is None:
        return torch.arange(slots.shape[0], device=DEV)[:, None].expand_as(slots), slots.clamp(max=s["k"].shape[-2] - 1)
    block = (slots // PAGE).clamp(max=s["table"].shape[1] - 1)
    return s["table"].long().gather(1, block).clamp(min=0), slots % PAGE


def _dense(s, slots):
    """K and V of the logical slots [B, n] as 32-bit rows [B, n, heads, D]."""
    row, at = _places(s, slots)
    k, v = (_bytes(c)[row, :, at].view(c.dtype) for c in (s["k"], s["v"]))
    if s["ks"] is None:
        return k.float(), v.float()
    return _values(k, s["ks"][row, :, at]), _values(v, s["vs"][row, :, at])


def _plain_attn(s):
    B, N, H, D = s["q"].shape
    new, prefix = s["new"].long(), s["prefix"].long()
    G = s["k"].shape[-3]
    slots = torch.arange(int(s["case"]["width"]) + max(_numbers(s["case"]["prefix"])), device=DEV).expand(B, -1)
    live = slots < (prefix + new)[:, None]
    k, v = _dense(s, torch.where(live, slots, 0))
    k = torch.where(live[:, :, None, None], k, 0.0).permute(0, 2, 3, 1).contiguous()
    v = torch.where(live[:, :, None, None], v, 0.0).transpose(1, 2).contiguous()
    own_slot = slots[:, None] - prefix[:, None, None]                       # which new token a slot holds, negative in the prefix
    node = torch.arange(N, device=DEV)[None, :, None]
    if s["parent"] is None:
        sees = own_slot <= node
    else:
        one = (torch.arange(N, device=DEV)[None, None] == torch.where(node == 0, 0, s["parent"][:, :, None])) | (torch.arange(N, device=DEV)[None, None] == node)
        step = one.float()
        step = ((step @ step) > 0).float()
        step = ((step @ step) > 0).float()
        step = ((step @ step) > 0).float()
        step = ((step @ step) > 0).float()
        step = ((step @ step) > 0).float()
        reach = (step @ step) > 0                                           # 64 steps up
        sees = (own_slot < 0) | reach.gather(2, own_slot.clamp(0, N - 1).expand(-1, N, -1))
    sees = sees & live[:, None]
    q = s["q"].float().view(B, N, G, H // G, D).permute(0, 2, 3, 1, 4).reshape(B, G, H // G * N, D)
    score = (q @ k).mul_(1.0 / math.sqrt(D)).view(B, G, H // G, N, -1)
    score = score.masked_fill_(~sees[:, None, None], float("-inf"))
    top = score.amax(dim=-1, keepdim=True)
    weight = score.sub_(top).exp_()
    total = weight.sum(dim=-1, keepdim=True)
    o = (weight.view(B, G, H // G * N, -1) @ v).view(B, G, H // G, N, D) / total
    written = node < new[:, None, None]
    s["out"].copy_(torch.where(written[..., None], o.permute(0, 3, 1, 2, 4).reshape(B, N, H, D).to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(written[:, None, :, 0], (top + total.log()).reshape(B, H, N), s["lse"]))
    return {"o": s["out"], "lse": s["lse"], "err": s["err"]}


def _plain_append(s):
    B, N = s["k_new"].shape[:2]
    at = torch.arange(N, device=DEV)[None]
    written = at < s["new"][:, None]
    row, slot = (x[written] for x in _places(s, s["prefix"].long()[:, None] + at))
    if s["ks"] is None:
        s["k"][row, :, slot] = s["k_new"][written]
        s["v"][row, :, slot] = s["v_new"][written]
        return {"k": s["k"], "v": s["v"], "err": s["err"]}
    (k, ks), (v, vs) = _quantise(s["k_new"][written]), _quantise(s["v_new"][written])
    _bytes(s["k"])[row, :, slot] = _bytes(k)
    _bytes(s["v"])[row, :, slot] = _bytes(v)
    s["ks"][row, :, slot] = ks
    s["vs"][row, :, slot] = vs
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"], "err": s["err"]}


def _plain_read(s):
    B, N = s["k_out"].shape[:2]
    at = torch.arange(N, device=DEV)[None]
    taken = at < s["count"][:, None]
    k, v = _dense(s, torch.where(taken, s["start"].long()[:, None] + at, 0))
    s["k_out"].copy_(torch.where(taken[..., None, None], k.to(s["k_out"].dtype), s["k_out"]))
    s["v_out"].copy_(torch.where(taken[..., None, None], v.to(s["v_out"].dtype), s["v_out"]))
    return {"k": s["k_out"], "v": s["v_out"], "err": s["err"]}


def _layer_view(s, name):
    return {"k": s["k"][0], "table": s["table"]}


def _plain_compact(s):
    at = torch.arange(s["path"].shape[1], device=DEV)[None]
    moved = at <= s["length"][:, None]
    base = s["prefix"].long()[:, None]
    one = _layer_view(s, "k")
    row_from, slot_from = (x[moved] for x in _places(one, base + s["path"].long().clamp(min=0)))
    row_to, slot_to = (x[moved] for x in _places(one, base + at))
    for name in ("k", "v", "ks", "vs"):
        t = _bytes(s[name])
        t[:, row_to, :, slot_to] = t[:, row_from, :, slot_from]
    s["new_prefix"].copy_(s["prefix"] + s["length"] + 1)
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"], "new_prefix": s["new_prefix"], "err": s["err"]}


_PLAIN = {"attn": _plain_attn, "append": _plain_append, "read": _plain_read, "compact": _plain_compact}


# ---- the library's calls -----------------------------------------------------------------------------
def _own_attn(s, sv):
    sv.specvlm_chunk_attn(s["q"], s["k"], s["v"], s["prefix"], num_new=s["new"], parent=s["parent"], block_table=s["table"],
                          scales=None if s["ks"] is None else (s["ks"], s["vs"]), out=s["out"], lse=s["lse"], workspace=s["workspace"],
                          err_flag=s["err"])
    return {"o": s["out"], "lse": s["lse"], "err": s["err"]}


def _own_append(s, sv):
    scales = None if s["ks"] is None else (s["ks"], s["vs"])
    sv.specvlm_kv_append(s["k_new"], s["v_new"], s["k"], s["v"], s["prefix"], num_new=s["new"], block_table=s["table"], scales=scales,
                         err_flag=s["err"])
    if scales is None:
        return {"k": s["k"], "v": s["v"], "err": s["err"]}
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"], "err": s["err"]}


def _own_read(s, sv):
    sv.specvlm_kv_read(s["k"], s["v"], s["count"], start=s["start"], block_table=s["table"],
                       scales=None if s["ks"] is None else (s["ks"], s["vs"]), out=(s["k_out"], s["v_out"]), err_flag=s["err"])
    return {"k": s["k_out"], "v": s["v_out"], "err": s["err"]}


def _own_compact(s, sv):
    sv.specvlm_kv_compact_quantized(s["k"], s["v"], (s["ks"], s["vs"]), s["prefix"], s["path"], s["length"], block_table=s["table"],
                                    new_prefix_len=s["new_prefix"], err_flag=s["err"])
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"], "new_prefix": s["new_prefix"], "err": s["err"]}


_OWN = {"attn": _own_attn, "append": _own_append, "read": _own_read, "compact": _own_compact}


def run(state):
    kind = state["case"]["kind"]
    if own:
        import paper_2509_11815_amd as sv
        return _OWN[kind](state, sv)
    return _PLAIN[kind](state)


# ---- from the definition, in 64 bits -----------------------------------------------------------------
def _slots_of(s, b, slots):
    """(row, slot in the row) of request b's logical slots, one after another."""
    if s["table"] is None:
        return [(b, t) for t in slots]
    table = s["table"][b].tolist()
    return [(table[t // PAGE], t % PAGE) for t in slots]


def _take(t, places, head):
    rows = torch.tensor([p[0] for p in places], device=DEV, dtype=torch.long)
    at = torch.tensor([p[1] for p in places], device=DEV, dtype=torch.long)
    return _bytes(t)[rows, head, at].view(t.dtype)


def _two_to64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _take64(s, name, places, head):
    x = _take(s[name], places, head).double()
    scale = s[name + "s"]
    return x if scale is None else x * _two_to64(_take(scale, places, head).long() - 127)[:, None]


def _exact_attn(case, s):
    new, prefix = _numbers(case["new"]), _numbers(case["prefix"])
    o, lse = s["out"].double(), s["lse"].double()
    G = case["kv_heads"]
    group, D = case["q_heads"] // G, case["head_dim"]
    for b, (n, P) in enumerate(zip(new, prefix)):
        if not n:
            continue
        places = _slots_of(s, b, range(P + n))
        hidden = torch.ones((n, P + n), dtype=torch.bool, device=DEV)
        hidden[:, :P] = False
        if s["parent"] is None:
            hidden[:, P:] = torch.ones((n, n), dtype=torch.bool, device=DEV).triu_(1)
        else:
            parent = s["parent"][b].tolist()
            for i in range(n):
                j = i
                while j >= 0:
                    hidden[i, P + j] = False
                    j = parent[j]
        for g in range(G):
            k, v = _take64(s, "k", places, g), _take64(s, "v", places, g)
            for h in range(g * group, (g + 1) * group):
                x = (s["q"][b, :n, h].double() @ k.T) / math.sqrt(D)
                x[hidden] = -math.inf
                lse[b, h, :n] = torch.logsumexp(x, dim=1)
                o[b, :n, h] = torch.softmax(x, dim=1) @ v
    return {"o": o, "lse": lse, "err": None}


def _round_e4m3(y):
    """y (64 bits, |y| <= 464 or NaN) rounded to the nearest e4m3 number, ties to the even code."""
    step = _two_to64(torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 4)
    return torch.round(y / step) * step


def _exact_append(case, s):
    new, prefix = _numbers(case["new"]), _numbers(case["prefix"])
    quantised = s["ks"] is not None
    out = {"err": None, "k": s["k"].double(), "v": s["v"].double()}
    if quantised:
        out.update(ks=s["ks"].clone(), vs=s["vs"].clone())
    for b, (n, P) in enumerate(zip(new, prefix)):
        if not n:
            continue
        places = _slots_of(s, b, range(P, P + n))
        rows = torch.tensor([p[0] for p in places], device=DEV, dtype=torch.long)
        at = torch.tensor([p[1] for p in places], device=DEV, dtype=torch.long)
        for name, source in (("k", s["k_new"]), ("v", s["v_new"])):
            x = source[b, :n].double()
            if quantised:
                a = x.abs().amax(dim=-1, keepdim=True)
                e = torch.where(a > 0, torch.frexp(a).exponent.long() - 10, -100).clamp(min=-100)              # a >= 512 * 2^e: one or two too small
                e = torch.where(a > 448.0 * _two_to64(e), e + 1, e)
                e = torch.where(a > 448.0 * _two_to64(e), e + 1, e)
                out[name + "s"][rows, :, at] = (e[..., 0] + 127).to(torch.uint8)
                x = _round_e4m3(x * _two_to64(-e))
            out[name][rows, :, at] = x
    return out


def _exact_read(case, s):
    start, count = _numbers(case["start"]), _numbers(case["count"])
    out = {"err": None, "k": s["k_out"].double(), "v": s["v_out"].double()}
    for b, (a, n) in enumerate(zip(start, count)):
        if n:
            places = _slots_of(s, b, range(a, a + n))
            for name in ("k", "v"):
                for g in range(case["kv_heads"]):
                    out[name][b, :n, g] = _take64(s, name, places, g)
    return out


def _exact_compact(case, s):
    prefix, path, length = _numbers(case["prefix"]), s["path"].tolist(), s["length"].tolist()
    out = {n: _bytes(s[n]).clone() for n in ("k", "v", "ks", "vs")}
    for b, P in enumerate(prefix):
        m = length[b]
        source, target = _slots_of(s, b, [P + path[b][j] for j in range(m + 1)]), _slots_of(s, b, range(P, P + m + 1))
        for name, t in out.items():
            for (r0, t0), (r1, t1) in zip(source, target):
                t[:, r1, :, t1] = _bytes(s[name])[:, r0, :, t0]
    return {"k": out["k"].view(torch.float8_e4m3fn), "v": out["v"].view(torch.float8_e4m3fn), "ks": out["ks"], "vs": out["vs"],
            "new_prefix": None, "err": None}


_EXACT = {"attn": _exact_attn, "append": _exact_append, "read": _exact_read, "compact": _exact_compact}


def exact(case, seed):
    return _EXACT[case["kind"]](case, prepare(case, seed))


# ---- what a pass cannot do without -------------------------------------------------------------------
def work(case):
    kind, G, D = case["kind"], case["kv_heads"], case["head_dim"]
    if kind == "compact":
        # the rows of a path of half its capacity, read and written in every layer
        rows = len(_numbers(case["prefix"])) * max(1, case["cap"] // 2) * case["layers"] * G * 2
        return {"bytes": 2 * rows * (D + 1), "flops": 0}
    if kind == "attn":
        H, new, prefix = case["q_heads"], _numbers(case["new"]), _numbers(case["prefix"])
        row = (D + 1 if case["cache"] == "e4m3" else 2 * D) * 2 * G
        live = [(n, P) for n, P in zip(new, prefix) if n]
        return {"bytes": sum((P + n) * row + n * H * (4 * D + 4) for n, P in live),
                "flops": sum(4 * H * D * (n * P + n * (n + 1) // 2) for n, P in live)}
    size = 4 if case["dtype"] == "f32" else 2
    rows = sum(_numbers(case["new" if kind == "append" else "count"])) * 2 * G
    return {"bytes": rows * (D * size + (D * size if case["cache"] == "same" else D + 1)), "flops": 0}
