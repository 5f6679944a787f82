"""Performance cases of the operators between the q/k/v linears and the o_proj rotation of a decoder layer.

  rope     rotary positions of the heads of a row (q and k next to each other, as one projection writes them)
  store    new keys and values quantized into the paged cache, and what it now holds read back: a prompt whose own
           attention is to see the values that decoding will see
  read     cached rows read back, as when a cache is moved, checked or handed to another kernel
  attend   attention of new rows over the paged cache, also behind a prefix that all sequences share
  step     store and attend of a decoding step

A page of the cache holds, per key/value head and per sixteen tokens, one block: the codes of the keys, those of the
values, sixteen pairs (scale, least value) of the keys and sixteen of the values.  Codes lie as a warp's matrix
instructions read them: lane 4 r + c, r < 8, c < 4, has words w of 32 bits, word w in 16-byte chunk w / 4 of 512 bytes.
"""
import math

import torch

own = False

PAGE = 64
QMAX = {4: 15.0, 8: 255.0}
PLAIN, LINEAR, NTK, BY_PARTS = "plain", "linear", "ntk", "by_parts"

_ctx = None


def _context():
    """One context per process, as a program that serves a model keeps it."""
    global _ctx
    if _ctx is None:
        from paper_2506_13472_b200 import binding
        _ctx = binding.Context(0)
    return _ctx


# ---------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # decoding: q and k of 64 sequences on the 7B model
        dict(name="rope_7b_decode_m64", kind="rope", rows=64, heads=64, hd=128, rot=128, interleaved=False, scaling=PLAIN, far=4096),
        # a long prompt with grouped key heads, half of each head turned, positions stretched to 131072
        dict(name="rope_prompt_8191", kind="rope", rows=8191, heads=40, hd=128, rot=64, interleaved=True, scaling=BY_PARTS, far=131072),
        # one prompt of the 7B model, four bits
        dict(name="store_7b_prompt_int4", kind="store", seqs=1, old_lo=0, old_hi=0, new_lo=2048, new_hi=2048, hkv=32, hd=128, bits=4),
        # chunks of several prompts that end and begin anywhere, grouped heads, eight bits
        dict(name="store_ragged_int8", kind="store", seqs=13, old_lo=0, old_hi=700, new_lo=1, new_hi=1100, hkv=8, hd=128, bits=8),
        # a 13B cache read back: 16 sequences of ragged length
        dict(name="read_13b_int4", kind="read", seqs=16, old_lo=0, old_hi=0, new_lo=150, new_hi=1500, hkv=40, hd=128, bits=4),
        # the last rows of a few sequences
        dict(name="read_tail_int8", kind="read", seqs=5, old_lo=100, old_hi=900, new_lo=1, new_hi=33, hkv=8, hd=64, bits=8),
        # one user, short context: latency of a decoding step
        dict(name="step_7b_m1_short", kind="step", seqs=1, old_lo=332, old_hi=332, new_lo=1, new_hi=1, hq=32, hkv=32, hd=128, bits=4, prefix=0),
        # a decoding batch of the 7B model, ragged lengths
        dict(name="step_7b_m64", kind="step", seqs=64, old_lo=500, old_hi=4000, new_lo=1, new_hi=1, hq=32, hkv=32, hd=128, bits=4, prefix=0),
        # long contexts, eight query heads to a key head, eight bits
        dict(name="attend_m16_32k_int8", kind="attend", seqs=16, old_lo=20000, old_hi=32767, new_lo=1, new_hi=1, hq=64, hkv=8, hd=128, bits=8, prefix=0),
        # one very long context
        dict(name="attend_m1_131k_int4", kind="attend", seqs=1, old_lo=131070, old_hi=131070, new_lo=1, new_hi=1, hq=32, hkv=8, hd=128, bits=4, prefix=0),
        # several drafted tokens of each sequence at once, heads of 64
        dict(name="attend_drafts_m33", kind="attend", seqs=33, old_lo=3, old_hi=2500, new_lo=1, new_hi=7, hq=32, hkv=8, hd=64, bits=4, prefix=0),
        # 64 sequences behind one system prompt
        dict(name="attend_prefix_m64", kind="attend", seqs=64, old_lo=0, old_hi=400, new_lo=1, new_hi=1, hq=32, hkv=8, hd=128, bits=4, prefix=16001),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _range(rng, lo, hi):
    a, b = sorted((_log_uniform(rng, lo, hi), _log_uniform(rng, lo, hi)))
    return a, b


_MOST_VALUES = 16 * 32768 * 8 * 128          # cached values, and operations, of the largest listed cases
_MOST_FLOPS = 4 * 64 * 16200 * 32 * 128
_MOST_BYTES = 890 * 10 ** 6


def draw(rng):
    kind = rng.choice(["rope", "store", "read", "attend", "attend", "step"])
    hd = rng.choice([64, 128, 128])
    if kind == "rope":
        heads = rng.choice([1, 8, 9, 40, 64, 80])
        rot = rng.choice([hd, hd, hd // 2, hd // 4])
        return dict(kind=kind, rows=_log_uniform(rng, 1, 8191 * 40 // heads // 2), heads=heads, hd=hd, rot=rot,
                    interleaved=rng.random() < 0.5, scaling=rng.choice([PLAIN, LINEAR, NTK, BY_PARTS]),
                    far=_log_uniform(rng, 100, 1 << 20))
    bits = rng.choice([4, 4, 8])
    hkv = rng.choice([1, 2, 8, 8, 32, 40])
    page = rng.choice([16, 32, 64, 64, 128, 256])
    if kind in ("store", "read"):
        seqs = _log_uniform(rng, 1, 64)
        most = max(1, min(4000, 16 * 1500 * 40 * 128 // (seqs * hkv * hd)))
        lo, hi = _range(rng, 1, most)
        return dict(kind=kind, seqs=seqs, old_lo=0, old_hi=_log_uniform(rng, 1, 2000), new_lo=lo, new_hi=hi, hkv=hkv, hd=hd,
                    bits=bits, page=page)
    seqs = _log_uniform(rng, 1, 200)
    hq = hkv * rng.choice([1, 1, 4, 5, 8] if hkv <= 8 else [1])
    most = max(16, min(131072, _MOST_VALUES // (seqs * hkv * 128)))
    new = 1 if kind == "step" or rng.random() < 0.6 else rng.choice([2, 5, 8]) if seqs > 4 else _log_uniform(rng, 2, 300)
    prefix = 0 if kind == "step" or rng.random() < 0.6 else _log_uniform(rng, 16, 16384)
    lo, hi = _range(rng, 1, most)
    c = dict(kind=kind, seqs=seqs, old_lo=lo, old_hi=hi, new_lo=1, new_hi=new, hq=hq, hkv=hkv, hd=hd, bits=bits, page=page, prefix=prefix)
    while work(c)["flops"] > _MOST_FLOPS or work(c)["bytes"] > _MOST_BYTES:   # too many rows over too long a prefix or sequence
        c.update({k: max(1, c[k] * 2 // 3) for k in ("seqs", "old_lo", "old_hi")}, prefix=c["prefix"] * 2 // 3)
    return c


def _spread(lo, hi, n, step):
    """n whole numbers over [lo, hi] in no order, the same for every seed."""
    return [lo + int((hi - lo + 1) * ((0.37 + i * step) % 1.0)) for i in range(n)]


def _lengths(c):
    """(tokens in the cache before the call, new tokens) of every sequence."""
    return _spread(c["old_lo"], c["old_hi"], c["seqs"], 0.6180339887), _spread(c["new_lo"], c["new_hi"], c["seqs"], 0.7548776662)


# ---------------------------------------------------------------------------------------------- the cache's layout
def _block_bytes(hd, bits):
    return 4 * hd * bits + 128


# How a lane's word w of chunk q holds a head of hd values, and the order of axes that the codes [block][token][value] have, as
# token = 8 h + r or 8 h + 2 c + b and value = 16 (words) + 8 p + (2 c + b or r):
#   keys    4 bits  token 8 h + r,       value 16 (4 q + w) + 8 p + 2 c + b        at byte 2 b + h, nibble p
#   values  4 bits  token 8 h + 2 c + b, value 16 (4 q + w) + 8 p + r              at byte 2 b + h, nibble p
#   keys    8 bits  token 8 h + r,       value 16 (2 q + w / 2) + 8 p + 2 c + b    at byte 2 p + b, h = w % 2
#   values  8 bits  token 8 h + 2 c + b, value 16 (2 q + w / 2) + 8 p + r          at byte 2 h + b, p = w % 2
def _codes_of(raw, hd, bits, value):
    """codes [n][16][hd] (uint8) of raw bytes [n][16 * hd * bits / 8]."""
    n = raw.shape[0]
    if bits == 4:
        x = raw.view(n, hd // 64, 8, 4, 4, 2, 2)                                   # q r c w b h
        x = torch.stack([x & 15, x >> 4], -1)                                      # q r c w b h p
        x = x.permute(0, 6, 3, 5, 1, 4, 7, 2) if value else x.permute(0, 6, 2, 1, 4, 7, 3, 5)
    else:
        x = raw.view(n, hd // 32, 8, 4, 2, 2, 2, 2)                                # q r c w (h or p) (p or h) b
        x = x.permute(0, 6, 3, 7, 1, 4, 5, 2) if value else x.permute(0, 5, 2, 1, 4, 6, 3, 7)
    return x.reshape(n, 16, hd)


def _raw_of(codes, bits, value):
    """The inverse of _codes_of."""
    n, _, hd = codes.shape
    if bits == 4:
        if value:
            x = codes.view(n, 2, 4, 2, hd // 64, 4, 2, 8).permute(0, 4, 7, 2, 5, 3, 1, 6)
        else:
            x = codes.view(n, 2, 8, hd // 64, 4, 2, 4, 2).permute(0, 3, 2, 6, 4, 7, 1, 5)
        x = x[..., 0] | (x[..., 1] << 4)
    elif value:
        x = codes.view(n, 2, 4, 2, hd // 32, 2, 2, 8).permute(0, 4, 7, 2, 5, 6, 1, 3)
    else:
        x = codes.view(n, 2, 8, hd // 32, 2, 2, 4, 2).permute(0, 3, 2, 6, 4, 1, 5, 7)
    return x.reshape(n, -1)


def _quantize(x, bits):
    """codes (uint8) and pairs (scale, least value) fp16 of fp16 heads [..., hd]."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    q = torch.full_like(lo, QMAX[bits], dtype=torch.float32)
    scale = torch.div(hi.float() - lo.float(), q).half()
    scale = torch.where(scale == 0, torch.full_like(scale, 2.0 ** -24), scale)
    codes = torch.div(x.float() - lo.float(), scale.float()).round().clamp(0, QMAX[bits]).to(torch.uint8)
    return codes, torch.cat([scale, lo + 0.0], -1)


def _blocks_of(kc, kp, vc, vp, bits):
    """Raw blocks [n][block bytes] of codes [n][16][hd] and pairs [n][16][2]."""
    n = kc.shape[0]
    return torch.cat([_raw_of(kc, bits, False), _raw_of(vc, bits, True), kp.contiguous().view(torch.uint8).reshape(n, 64),
                      vp.contiguous().view(torch.uint8).reshape(n, 64)], 1)


def _split(raw, hd, bits):
    """(key codes, key pairs, value codes, value pairs) of raw blocks."""
    n, cb = raw.shape[0], 2 * hd * bits
    pairs = lambda x: x.contiguous().view(torch.float16).view(n, 16, 2)  # noqa: E731
    return (_codes_of(raw[:, :cb].contiguous(), hd, bits, False), pairs(raw[:, 2 * cb:2 * cb + 64]),
            _codes_of(raw[:, cb:2 * cb].contiguous(), hd, bits, True), pairs(raw[:, 2 * cb + 64:]))


def _views(s):
    """The pages as [page][head][block of 16 tokens][bytes]."""
    return s["pages"].view(s["pages"].shape[0], s["hkv"], s["page"] // 16, -1)


def _held(s, table, n_tokens, dtype=torch.float32):
    """Keys and values [tokens][heads][hd] that the first n_tokens of a page list stand for."""
    np = (n_tokens + s["page"] - 1) // s["page"]
    raw = _views(s)[table[:np].long()]                                             # page, head, block, bytes
    raw = raw.permute(0, 2, 1, 3).reshape(-1, raw.shape[-1])                       # (page, block, head)
    out = []
    kc, kp, vc, vp = _split(raw, s["hd"], s["bits"])
    for codes, pairs in ((kc, kp), (vc, vp)):
        x = codes.to(dtype) * pairs[..., :1].to(dtype) + pairs[..., 1:].to(dtype)
        out.append(x.view(-1, s["hkv"], 16, s["hd"]).transpose(1, 2).reshape(-1, s["hkv"], s["hd"])[:n_tokens])
    return out


# ---------------------------------------------------------------------------------------------- inputs
class _Draw:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, *shape):
        return torch.randn(shape, device="cuda", generator=self.g)

    def loud(self, heads, hd):
        """Per-channel sizes of keys: a few channels of each head are several times larger."""
        size = torch.ones(heads, hd, device="cuda")
        size[torch.rand(heads, hd, device="cuda", generator=self.g) < 0.03] = 6.0
        return size


def _fill(s, dr, n_pages):
    """Pages of quantized keys and values, drawn a stretch at a time."""
    hkv, hd, bits, nb = s["hkv"], s["hd"], s["bits"], s["page"] // 16
    size = dr.loud(hkv, hd)[None, :, None, None]
    s["pages"] = torch.empty((n_pages, hkv * nb * _block_bytes(hd, bits)), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 25) // (hkv * s["page"] * hd))
    for p in range(0, n_pages, step):
        m = min(step, n_pages - p)
        k = (dr.normal(m, hkv, nb, 16, hd).mul_(size[..., None, :].view(1, hkv, 1, 1, hd))).half()
        v = dr.normal(m, hkv, nb, 16, hd).half()
        (kc, kp), (vc, vp) = _quantize(k, bits), _quantize(v, bits)
        s["pages"][p:p + m] = _blocks_of(kc.view(-1, 16, hd), kp.view(-1, 16, 2), vc.view(-1, 16, hd), vp.view(-1, 16, 2),
                                         bits).view(m, -1)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _frequencies(c):
    """Radians per position of each pair, and the size of the turned part, as the case's scaling has them (64 bits, host)."""
    half, base, factor, context = c["rot"] // 2, 10000.0, 8.0, 8192
    if c["scaling"] == NTK:
        base *= factor ** (c["rot"] / (c["rot"] - 2))
    f = [base ** (-i / half) for i in range(half)]
    if c["scaling"] == LINEAR:
        f = [x / factor for x in f]
    if c["scaling"] == BY_PARTS:
        for i, x in enumerate(f):
            keep = min(max((context * x / (2 * math.pi) - 1.0) / (32.0 - 1.0), 0.0), 1.0)
            f[i] = x * (keep + (1.0 - keep) / factor)
    return f, (0.1 * math.log(factor) + 1.0 if c["scaling"] == BY_PARTS else 1.0)


def prepare(case, seed):
    c, dr = case, _Draw(seed)
    if c["kind"] == "rope":
        s = dict(kind="rope", hd=c["hd"], rot=c["rot"], interleaved=c["interleaved"])
        s["x"] = dr.normal(c["rows"], c["heads"] * c["hd"]).half()
        s["positions"] = torch.randint(0, c["far"], (c["rows"],), device="cuda", generator=dr.g, dtype=torch.int32)
        f, s["size"] = _frequencies(c)
        s["freq"] = torch.tensor(f, dtype=torch.float64, device="cuda")
        if own:
            s["ctx"] = _context()
            s["rope"] = s["ctx"].rope_create(c["hd"], c["rot"], interleaved=c["interleaved"], base=10000.0, scaling=c["scaling"],
                                             factor=8.0, low=1.0, high=32.0, context=8192, magnitude=s["size"])
        return s
    page = c.get("page", PAGE)
    s = dict(kind=c["kind"], hkv=c["hkv"], hd=c["hd"], bits=c["bits"], page=page, old=_lengths(c)[0], new=_lengths(c)[1])
    n, lens = c["seqs"], [a + b for a, b in zip(*_lengths(c))]
    need = [(x + page - 1) // page for x in lens]
    extra = (c.get("prefix", 0) + page - 1) // page
    order = torch.randperm(sum(need) + extra, device="cuda", generator=dr.g).to(torch.int32)
    s["table"] = torch.zeros((n, max(need)), dtype=torch.int32, device="cuda")
    at = extra
    for i, m in enumerate(need):
        s["table"][i, :m] = order[at:at + m]
        at += m
    s["prefix"] = (order[:extra].contiguous(), c["prefix"]) if extra else None
    starts = [0]
    for m in s["new"]:
        starts.append(starts[-1] + m)
    s["rows"], s["row_start"], s["kv_len"] = starts[-1], _ints(starts), _ints(lens)
    _fill(s, dr, sum(need) + extra)
    if c["kind"] in ("attend", "step", "store"):
        hq, hkv, hd = c.get("hq", 0), c["hkv"], c["hd"]
        qkv = dr.normal(s["rows"], (hq + 2 * hkv) * hd)
        qkv[:, hq * hd:(hq + hkv) * hd] *= dr.loud(hkv, hd).view(-1)
        qkv = qkv.half()
        s["q"], s["k"], s["v"] = qkv[:, :hq * hd], qkv[:, hq * hd:(hq + hkv) * hd], qkv[:, (hq + hkv) * hd:]
    if own:
        from paper_2506_13472_b200 import binding
        s["ctx"] = _context()
        s["cache"] = binding.KvCache(s["pages"], n_kv_heads=c["hkv"], head_dim=c["hd"], bits=c["bits"], page_tokens=page)
        s["batch"] = binding.KvBatch(s["row_start"], s["kv_len"], s["table"], prefix=s["prefix"])
    return s


# ---------------------------------------------------------------------------------------------- one pass, plain
def _plain_rope(s):
    x, half = s["x"].view(s["x"].shape[0], -1, s["hd"]).float(), s["rot"] // 2
    angle = s["positions"].double()[:, None] * s["freq"][None, :]
    cos, sin = ((f(angle).float() * s["size"])[:, None, :] for f in (torch.cos, torch.sin))
    t = x[..., :s["rot"]]
    a, b = (t[..., 0::2], t[..., 1::2]) if s["interleaved"] else (t[..., :half], t[..., half:])
    u, w = a * cos - b * sin, b * cos + a * sin
    t = torch.stack([u, w], -1).flatten(-2) if s["interleaved"] else torch.cat([u, w], -1)
    return torch.cat([t, x[..., s["rot"]:]], -1).half().view(s["x"].shape)


def _plain_store(s):
    """Writes the new rows' codes into the pages."""
    pages, hkv, hd, at = _views(s), s["hkv"], s["hd"], 0
    for i, (old, new) in enumerate(zip(s["old"], s["new"])):
        b0, b1 = old // 16, (old + new + 15) // 16
        blocks = torch.arange(b0, b1, device="cuda")
        where = (s["table"][i][blocks * 16 // s["page"]].long(), blocks % (s["page"] // 16))
        raw = pages[where[0], :, where[1]].transpose(0, 1).reshape(hkv * (b1 - b0), -1)
        parts = [x.clone().view(hkv, (b1 - b0) * 16, -1) for x in _split(raw, hd, s["bits"])]
        for j, x in enumerate((s["k"], s["v"])):
            codes, pairs = _quantize(x[at:at + new].reshape(new, hkv, hd), s["bits"])
            parts[2 * j][:, old - 16 * b0:old + new - 16 * b0] = codes.transpose(0, 1)
            parts[2 * j + 1][:, old - 16 * b0:old + new - 16 * b0] = pairs.transpose(0, 1)
        raw = _blocks_of(*[x.reshape(hkv * (b1 - b0), 16, -1) for x in parts], s["bits"])
        pages[where[0], :, where[1]] = raw.view(hkv, b1 - b0, -1).transpose(0, 1)
        at += new


def _plain_read(s):
    out = []
    for i, (old, new) in enumerate(zip(s["old"], s["new"])):
        out.append([x[old:].half().reshape(new, -1) for x in _held(s, s["table"][i], old + new)])
    return [torch.cat([x[j] for x in out]) for j in (0, 1)]


def _attention(s, dtype):
    """softmax(q k / sqrt(hd)) v of every new row over the prefix and its sequence up to itself, in `dtype`."""
    hkv, hd, at, out = s["hkv"], s["hd"], 0, []
    group = s["q"].shape[1] // (hkv * hd)
    shared = _held(s, *s["prefix"], dtype) if s["prefix"] else None
    for i, (old, new) in enumerate(zip(s["old"], s["new"])):
        k, v = _held(s, s["table"][i], old + new, dtype)
        ahead = 0
        if shared:
            ahead = s["prefix"][1]
            k, v = torch.cat([shared[0], k]), torch.cat([shared[1], v])
        q = s["q"][at:at + new].reshape(new, hkv, group, hd).to(dtype)
        scores = torch.einsum("nhgd,thd->hgnt", q, k) / math.sqrt(hd)
        seen = torch.arange(k.shape[0], device="cuda")[None, :] <= ahead + old + torch.arange(new, device="cuda")[:, None]
        scores = torch.where(seen, scores, torch.full_like(scores, -math.inf))
        p = torch.exp(scores - scores.amax(-1, keepdim=True))
        o = torch.einsum("hgnt,thd->nhgd", p, v) / p.sum(-1).permute(2, 0, 1)[..., None]
        out.append(o.reshape(new, -1))
        at += new
    return torch.cat(out)


def run(state):
    s, kind = state, state["kind"]
    if own:
        ctx = s["ctx"]
        if kind == "rope":
            return ctx.rope(s["x"], s["positions"], s["rope"])
        if kind in ("store", "step"):
            ctx.kv_write(s["cache"], s["batch"], s["k"], s["v"])
        if kind in ("store", "read"):
            return list(ctx.kv_read(s["cache"], s["batch"], s["rows"]))
        return ctx.attend(s["q"], s["cache"], s["batch"])
    if kind == "rope":
        return _plain_rope(s)
    if kind in ("store", "step"):
        _plain_store(s)
    if kind in ("store", "read"):
        return _plain_read(s)
    return _attention(s, torch.float32).half()


# ---------------------------------------------------------------------------------------------- bounds
def work(case):
    c = case
    if c["kind"] == "rope":
        values = c["rows"] * c["heads"] * c["hd"]
        return {"bytes": 4 * values + 4 * c["rows"], "flops": 3 * c["rows"] * c["heads"] * c["rot"]}
    old, new = _lengths(c)
    head = 2 * (c["hd"] * c["bits"] // 8 + 4)                     # a token's keys and values of one head in the cache
    rows, n = sum(new), sum(old) + sum(new)
    if c["kind"] == "read":
        return {"bytes": rows * c["hkv"] * (head + 4 * c["hd"]), "flops": 4 * rows * c["hkv"] * c["hd"]}
    if c["kind"] == "store":                                      # rows in, blocks out and in again, rows out
        return {"bytes": rows * c["hkv"] * (2 * head + 8 * c["hd"]), "flops": 16 * rows * c["hkv"] * c["hd"]}
    seen = sum(b * (a + c["prefix"]) + b * (b + 1) // 2 for a, b in zip(old, new))
    data = (n + c["prefix"]) * c["hkv"] * head + 4 * rows * c["hq"] * c["hd"]
    if c["kind"] == "step":
        data += 4 * rows * c["hkv"] * c["hd"]
    return {"bytes": data, "flops": 4 * seen * c["hq"] * c["hd"]}


# ---------------------------------------------------------------------------------------------- 64 bits
def _exact_pairs(x, bits):
    """Least value, scale and codes of heads [..., hd] by the definition, all in 64 bits."""
    x = x.double()
    lo = x.min(-1, keepdim=True).values
    scale = ((x.max(-1, keepdim=True).values - lo) / QMAX[bits]).half().double()
    scale = torch.clamp(scale, min=2.0 ** -24)
    return lo + scale * torch.round((x - lo) / scale).clamp(0, QMAX[bits])


def _exact_held(raw, which, hd, bits):
    """Keys (which = 0) or values of raw blocks [n][bytes], looked up code by code."""
    t, d = torch.meshgrid(torch.arange(16, device=raw.device), torch.arange(hd, device=raw.device), indexing="ij")
    # a key's lane goes by token % 8 and the value's place in a pair of pairs, a value's the other way round
    r, o = (t % 8, d % 8) if which == 0 else (d % 8, t % 8)
    lane, b, h, p = 4 * r + o // 2, o % 2, t // 8, d % 16 // 8
    if bits == 4:
        w, byte = d // 16, 2 * b + h
    else:
        w, byte = (2 * (d // 16) + h, 2 * p + b) if which == 0 else (2 * (d // 16) + p, 2 * h + b)
    code = raw[:, which * 2 * hd * bits + 512 * (w // 4) + 16 * lane + 4 * (w % 4) + byte]
    if bits == 4:
        code = torch.where(p == 1, code // 16, code % 16)
    pairs = raw[:, 4 * hd * bits + 64 * which:4 * hd * bits + 64 * which + 64].contiguous().view(torch.float16).view(-1, 16, 2).double()
    return code.double() * pairs[:, :, :1] + pairs[:, :, 1:]


def _exact_rows(s, i, first, last):
    """Keys and values [tokens][heads][hd] of tokens [first, last) of sequence i (of the prefix: i < 0), new rows quantized afresh."""
    table, page = (s["prefix"][0] if i < 0 else s["table"][i]), s["page"]
    b0, b1 = first // 16, (last + 15) // 16
    out = []
    blocks = torch.arange(b0, b1, device="cuda")
    pages = s["pages"].view(s["pages"].shape[0], s["hkv"], page // 16, -1)[table[(blocks * 16) // page].long(), :, blocks % (page // 16)]
    for which in (0, 1):
        x = _exact_held(pages.reshape(-1, pages.shape[-1]), which, s["hd"], s["bits"])
        x = x.view(b1 - b0, s["hkv"], 16, s["hd"]).transpose(1, 2).reshape(-1, s["hkv"], s["hd"])[first - 16 * b0:last - 16 * b0]
        if i >= 0 and s["kind"] in ("store", "step") and last > s["old"][i]:
            fresh = max(first, s["old"][i])
            at = sum(s["new"][:i]) + fresh - s["old"][i]
            rows = s["k" if which == 0 else "v"][at:at + last - fresh]
            x = torch.cat([x[:fresh - first], _exact_pairs(rows.reshape(last - fresh, s["hkv"], s["hd"]), s["bits"])])
        out.append(x)
    return out


_STRETCH = 4096                              # tokens whose 64-bit keys and values are held at a time


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "rope":
        x = s["x"].double().view(s["x"].shape[0], -1, s["hd"])
        y = x.clone()
        f, size = _frequencies(case)
        for i, fi in enumerate(f):
            m, n = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + len(f))
            z = torch.polar(torch.full((x.shape[0],), size, dtype=torch.float64, device="cuda"), s["positions"].double() * fi)
            z = torch.complex(x[..., m], x[..., n]) * z[:, None]
            y[..., m], y[..., n] = z.real, z.imag
        return y.view(s["x"].shape)
    if s["kind"] in ("store", "read"):
        both = [_exact_rows(s, i, a, a + b) for i, (a, b) in enumerate(zip(s["old"], s["new"]))]
        return [torch.cat([x[j].reshape(x[j].shape[0], -1) for x in both]) for j in (0, 1)]
    hq, hd, group, out, at = case["hq"], s["hd"], case["hq"] // case["hkv"], [], 0
    if sum(s["new"]) * (max(s["old"]) + case["prefix"]) * hq > 3 << 30:
        return None
    for i, (old, new) in enumerate(zip(s["old"], s["new"])):
        q = s["q"][at:at + new].double().view(new, hq, hd) / math.sqrt(hd)
        at += new
        scores, parts = [], [(-1, t, min(t + _STRETCH, case["prefix"])) for t in range(0, case["prefix"], _STRETCH)]
        parts += [(i, t, min(t + _STRETCH, old + new)) for t in range(0, old + new, _STRETCH)]
        for which, t0, t1 in parts:
            k = _exact_rows(s, which, t0, t1)[0].repeat_interleave(group, 1)
            x = torch.bmm(q.transpose(0, 1), k.permute(1, 2, 0))                    # head, row, token
            if which >= 0:
                late = torch.arange(t0, t1, device="cuda")[None, :] > old + torch.arange(new, device="cuda")[:, None]
                x = x.masked_fill(late, -math.inf)
            scores.append(x)
        p, at_t, o = torch.softmax(torch.cat(scores, -1), -1), 0, 0.0
        for which, t0, t1 in parts:
            v = _exact_rows(s, which, t0, t1)[1].repeat_interleave(group, 1)
            o = o + torch.bmm(p[..., at_t:at_t + t1 - t0], v.transpose(0, 1))
            at_t += t1 - t0
        out.append(o.transpose(0, 1).reshape(new, -1))
    return torch.cat(out)
