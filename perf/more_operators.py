"""Keys and values of a decoder held in microscaling formats, as cases that can be timed.

Three operators round a paged cache of codes and scales, which a server of quantized weights keeps next to them:

  cache_write       new keys and values quantized along the head, in blocks, on their way into their pages
  cache_read        the tokens of sequences out of their pages, reconstructed
  cache_attention   softmax(scale Q K^T) V of queries over the cache, K and V read as codes: one token per sequence
                    (decoding), a few (speculation) or many (a piece of a prompt)

Pages hold `page` tokens of every head: codes [pages, heads, page, dim * bits / 8], scales [pages, heads, page, dim / block].
A batch is described by its page table [batch, most pages], its lengths in tokens and, where a sequence brings other than
one new token, the places where each sequence's tokens start.  The plain forms below are written from the formulas in
elementary torch operations, in 32 bits, and rounded once to the output's type.  Widths are those of the 8B Llama-shaped
weight set (32 heads over 8 of 128) or generic ones.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
#: format -> (bits, exponent bits, mantissa bits); exponent bits 0: two's complement integers
FMT = {"e4m3": (8, 4, 3), "e2m1": (4, 2, 1), "int8": (8, 0, 0), "int4": (4, 0, 0)}


def _case(name, op, batch, length, new, heads, group, dim, fmt, block=32, page=64, dtype="bf16", window=0, ragged=False, empty=False):
    return {"name": name, "op": op, "batch": batch, "length": length, "new": new, "heads": heads, "group": group, "dim": dim,
            "fmt": fmt, "block": block, "page": page, "dtype": dtype, "window": window, "ragged": ragged, "empty": empty}


def listed():
    return [
        # the keys and values of one decoded token: the smallest call there is, latency counts
        _case("write_token", "write", 1, 1000, 1, 8, 4, 128, "e4m3"),
        # a long prompt on its way into the cache
        _case("write_prompt", "write", 1, 8192, 8192, 8, 4, 128, "int8"),
        # FP32 pieces of prompts of many lengths into a 4-bit cache, and the sequences back for a program with its own attention
        _case("write_read_pieces_f32", "refill", 7, 1500, 300, 5, 1, 64, "e2m1", page=16, dtype="f32", ragged=True),
        # the contexts of a batch reconstructed from 4 bits
        _case("read_contexts", "read", 16, 8192, 1, 8, 4, 128, "e2m1", ragged=True),
        # a short odd batch, one slot of it empty, in FP32
        _case("read_short_f32", "read", 5, 333, 1, 3, 1, 64, "int4", block=64, page=32, dtype="f32", ragged=True, empty=True),
        # one decoded token of one short chat: latency counts
        _case("decode_one_short", "attention", 1, 1000, 1, 8, 4, 128, "e2m1"),
        # a serving step: 64 sequences of many lengths, one token each
        _case("decode_batch", "attention", 64, 8192, 1, 8, 4, 128, "e2m1", ragged=True),
        # one decoded token of one very long context
        _case("decode_one_long", "attention", 1, 131071, 1, 8, 4, 128, "int4"),
        # FP32 queries, small heads, a window over the last tokens, a padded slot
        _case("decode_window_f32", "attention", 33, 3000, 1, 4, 3, 64, "e4m3", block=64, page=32, dtype="f32", window=1024, ragged=True, empty=True),
        # a few tokens per sequence checked at once, as speculation does
        _case("speculate_batch", "attention", 12, 4096, 5, 8, 4, 128, "int8", block=128, ragged=True),
        # a step as a server runs it: the new token's keys and values written, then attended, heads of 256 over one
        _case("step_shared_head", "step", 32, 4096, 1, 1, 8, 256, "e4m3", page=128, ragged=True),
        # the last piece of a long prompt: 2048 queries over 8192 tokens
        _case("prompt_piece", "attention", 1, 8192, 2048, 8, 4, 128, "e2m1"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    op = rng.choice(["write", "refill", "read", "attention", "attention", "attention", "attention", "step"])
    dim = rng.choice([64, 128, 128, 256])
    group = rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16])
    heads = log_int(1, min(8, 32 // group))
    fmt = rng.choice(["e4m3", "int8"] if op in ("write", "step") else sorted(FMT))
    batch = log_int(1, 64)
    length = log_int(1, 8192 if batch < 16 else 2048)
    new, kind = 1, rng.random()
    if op in ("write", "refill"):
        new = log_int(1, max(1, min(length, 4096 // batch)))
    elif op != "read" and kind < 0.3:
        new = min(length, rng.randint(2, 8))
    elif op == "attention" and kind < 0.45:
        batch, new = min(batch, 2), log_int(1, min(length, 256))
    if op == "attention" and new == 1 and kind > 0.8:
        batch, length = 1, log_int(8192, 65536)
    case = _case("", op, batch, length, new, heads, group, dim, fmt, block=rng.choice([b for b in (32, 64, 128) if dim % b == 0]),
                 page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                 window=rng.choice([0, 0, log_int(1, length)]) if op == "attention" else 0, ragged=rng.random() < 0.7,
                 empty=rng.random() < 0.2 and batch > 1)
    del case["name"]
    return case


# ---- what a case says of its batch ----------------------------------------------------------------------------


def _lengths(c):
    """Tokens of each sequence, the new ones among them: from half of `length` to all of it; the last slot may be empty."""
    n = [c["length"] - (b * 7919 % (c["length"] // 2 + 1) if c["ragged"] else 0) for b in range(c["batch"])]
    if c["empty"]:
        n[-1] = 0
    return n


def _news(c):
    """New tokens of each sequence."""
    return [min(n, c["new"] - (b * 31 % (c["new"] // 2 + 1) if c["ragged"] else 0)) for b, n in enumerate(_lengths(c))]


def _queries(c):
    """Queries of each sequence.  A padded slot of a decoding batch has its row all the same."""
    return [1] * c["batch"] if c["new"] == 1 else _news(c)


def _starts(counts):
    got = [0]
    for n in counts:
        got.append(got[-1] + n)
    return got


# ---- inputs ---------------------------------------------------------------------------------------------------


def _keys(g, shape, dtype):
    """N(0, 1) with a few channels of each head several times as large, as keys have them."""
    loud = torch.where(torch.rand(shape[-2:], generator=g, device="cuda") < 0.03, 6.0, 1.0)
    return (torch.randn(shape, generator=g, device="cuda") * loud).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c, dtype = case, DTYPES[case["dtype"]]
    heads, dim, page, fmt, block = c["heads"], c["dim"], c["page"], c["fmt"], c["block"]
    lengths, queries = _lengths(c), _queries(c)
    need = [-(-n // page) for n in lengths]
    pages, most = sum(need) + 3, max(1, *need)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((c["batch"], most), -1, dtype=torch.int32, device="cuda")
    for b, (n, at) in enumerate(zip(need, _starts(need))):
        table[b, :n] = order[at:at + n]
    k = _keys(g, (pages, page, heads, dim), torch.bfloat16).transpose(1, 2).contiguous()
    k = _pack(*_quantize(k.float(), fmt, block), fmt)
    v = torch.randn(pages, heads, page, dim, generator=g, device="cuda")
    v = _pack(*_quantize(v, fmt, block), fmt)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    s = {**c, "dtype": dtype, "cache": (*k, *v), "table": table, "lengths": ints(lengths), "total": sum(lengths),
         "firsts": ints(_starts(lengths)), "starts": None if c["new"] == 1 else ints(_starts(queries)), "row_starts": ints(_starts(queries))}
    rows = sum(queries)
    if c["op"] in ("attention", "step"):
        s["q"] = torch.randn(rows, heads * c["group"], dim, generator=g, device="cuda").to(dtype)
    if c["op"] in ("write", "refill", "step"):        # k and v are slices of one projection's output
        kv = torch.empty(rows, 2, heads, dim, dtype=dtype, device="cuda")
        kv[:, 0] = _keys(g, (rows, heads, dim), dtype)
        kv[:, 1] = torch.randn(rows, heads, dim, generator=g, device="cuda").to(dtype)
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------


def _magnitudes(fmt):
    """The non-negative values of an MXFP element format in the order of their codes."""
    bits, eta, mu = FMT[fmt]
    bias = 2 ** (eta - 1) - 1
    c = torch.arange(2 ** (bits - 1), device="cuda")
    e, m = c >> mu, (c & (2 ** mu - 1)).float() / 2 ** mu
    got = torch.where(e == 0, m * 2.0 ** (1 - bias), (1 + m) * torch.exp2((e - bias).float()))
    return got[:-1] if fmt == "e4m3" else got         # S.1111.111 is NaN in E4M3


def _power(e):
    """2^e as FP32 for whole e in [-127, 127], put together from its bits."""
    e = e.to(torch.int32)
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _quantize(v, fmt, block):
    """Codes (one byte each, in v's shape) and E8M0 bytes of FP32 values, blocks along the last dimension."""
    bits, eta, mu = FMT[fmt]
    e_max = 2 ** (eta - 1) if eta else bits - 2
    parts = v.unflatten(-1, (-1, block))
    amax = parts.abs().amax(-1, keepdim=True)
    shared = (torch.frexp(amax).exponent - 1 - e_max).clamp(-127, 127)
    shared = torch.where(amax == 0, -127, shared)
    p = parts * _power(-shared)
    if eta:
        low = 2 - 2 ** (eta - 1)                       # the exponent of the smallest normal value
        step = _power((torch.frexp(p).exponent - 1).clamp(min=low) - mu)
        mags = _magnitudes(fmt)
        mag = ((p / step).round() * step).abs().clamp(max=float(2 ** e_max * (2 - 2.0 ** -mu) if fmt != "e4m3" else 448))
        code = torch.searchsorted(mags, mag.contiguous())
        code = code.to(torch.uint8) | (torch.signbit(p).to(torch.uint8) << (bits - 1))
    else:
        most = 2 ** (bits - 1) - 1
        whole = (torch.floor(p.abs() + 0.5) * torch.sign(p)).clamp(-most, most)
        code = (whole.to(torch.int32) & (2 ** bits - 1)).to(torch.uint8)
    return code.flatten(-2), (shared.squeeze(-1) + 127).to(torch.uint8)


def _pack(codes, scales, fmt):
    if FMT[fmt][0] == 4:
        codes = codes[..., 0::2] | (codes[..., 1::2] << 4)
    return codes.contiguous(), scales.contiguous()


def _dequantize(codes, scales, fmt, block):
    """FP32 values of packed codes, blocks along the last dimension."""
    bits, eta, _ = FMT[fmt]
    if bits == 4:
        codes = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    if eta:
        mags = _magnitudes(fmt)
        mags = torch.cat((mags, mags.new_full((2 ** (bits - 1) - mags.numel(),), math.nan)))
        v = torch.cat((mags, -mags))[codes.int()]
    else:
        v = (codes.to(torch.int8) if bits == 8 else (codes << 4).to(torch.int8) >> 4).float()
    return (v.unflatten(-1, (-1, block)) * _power(scales.int() - 127).unsqueeze(-1)).flatten(-2)


def _rows(s):
    """Of each new token: its sequence, its position there and whether it has one."""
    starts, lengths = s["row_starts"].long(), s["lengths"].long()
    i = torch.arange(s["q" if "q" in s else "k"].shape[0], device=starts.device)
    b = torch.searchsorted(starts[1:], i, right=True)
    pos = lengths[b] - (starts[b + 1] - i)
    return b, pos, pos >= 0


def _write(s):
    b, pos, there = _rows(s)
    b, pos = b[there], pos[there]
    pages, off = s["table"][b, pos // s["page"]].long(), pos % s["page"]
    for x, codes, scales in ((s["k"], *s["cache"][:2]), (s["v"], *s["cache"][2:])):
        c, e = _pack(*_quantize(x[there].float(), s["fmt"], s["block"]), s["fmt"])
        codes[pages, :, off] = c
        scales[pages, :, off] = e


def _gather(s, b, pos):
    """Keys and values of the tokens at `pos` of the sequences `b`, FP32."""
    pages, off = s["table"][b, pos // s["page"]].long(), pos % s["page"]
    kc, ks, vc, vs = (x[pages, :, off] for x in s["cache"])
    return _dequantize(kc, ks, s["fmt"], s["block"]), _dequantize(vc, vs, s["fmt"], s["block"])


def _read(s):
    firsts = s["firsts"].long()
    i = torch.arange(s["total"], device=firsts.device)
    b = torch.searchsorted(firsts[1:], i, right=True)
    k, v = _gather(s, b, i - firsts[b])
    return k.to(s["dtype"]), v.to(s["dtype"])


def _attention(s):
    lengths, starts = s["lengths"].long(), s["row_starts"].long()
    b, pos, _ = _rows(s)
    batch, heads, group, dim = s["batch"], s["heads"], s["group"], s["dim"]
    most = s["new"]
    q = torch.zeros(batch, most, heads * group, dim, device=b.device)
    at = torch.full((batch, most), -1, device=b.device)
    nth = torch.arange(b.numel(), device=b.device) - starts[b]
    q[b, nth] = s["q"].float()
    at[b, nth] = pos                                   # a query sees the tokens up to its own position
    t = torch.arange(max(1, s["length"]), device=b.device)
    seen = (t <= at.unsqueeze(-1)) & (t < lengths.view(-1, 1, 1))
    if s["window"]:
        seen &= t > at.unsqueeze(-1) - s["window"]
    k, v = _gather(s, torch.arange(batch, device=b.device).view(-1, 1), torch.minimum(t, (lengths - 1).clamp(min=0).view(-1, 1)))
    empty = (lengths == 0).view(-1, 1, 1, 1)
    k, v = k.masked_fill(empty, 0).transpose(1, 2), v.masked_fill(empty, 0).transpose(1, 2)        # [batch, heads, tokens, dim]
    q = q.view(batch, most, heads, group, dim).permute(0, 2, 1, 3, 4).reshape(batch, heads, most * group, dim)
    p = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(dim)
    seen = seen.repeat_interleave(group, 1).unsqueeze(1)
    p = p.masked_fill(~seen, -math.inf)
    p = torch.exp(p - p.amax(-1, keepdim=True).clamp(min=-3e38)).masked_fill(~seen, 0)
    out = torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    out = out.view(batch, heads, most, group, dim).permute(0, 2, 1, 3, 4).reshape(batch, most, heads * group, dim)
    return out[b, nth].to(s["dtype"])


def _held(s):
    """The cache as the values that it holds, 8 bits each, and its scale bytes."""
    kc, ks, vc, vs = s["cache"]
    kind = torch.float8_e4m3fn if s["fmt"] == "e4m3" else torch.int8
    return {"k": kc.view(kind), "k_scales": ks, "v": vc.view(kind), "v_scales": vs}


def run(s):
    op, fmt, block, dtype = s["op"], s["fmt"], s["block"], s["dtype"]
    if own:
        import paper_2604_00529_b200 as mxq
        if op in ("write", "refill", "step"):
            mxq.cache_write(s["k"], s["v"], *s["cache"], s["table"], s["lengths"], fmt, block=block, starts=s["starts"])
        if op in ("attention", "step"):
            out = mxq.cache_attention(s["q"], *s["cache"], s["table"], s["lengths"], fmt, block=block, starts=s["starts"],
                                      window=s["window"])
        if op in ("read", "refill"):
            return mxq.cache_read(*s["cache"], s["table"], s["firsts"], s["total"], fmt, block=block, dtype=dtype)
    else:
        if op in ("write", "refill", "step"):
            _write(s)
        if op in ("attention", "step"):
            out = _attention(s)
        if op in ("read", "refill"):
            return _read(s)
    if op == "write":
        return _held(s)
    return out if op == "attention" else {"out": out, **_held(s)}


# ---- what a pass cannot do without ----------------------------------------------------------------------------


def work(case):
    c = case
    size, row = (2 if c["dtype"] == "bf16" else 4), c["dim"] * FMT[c["fmt"]][0] / 8 + c["dim"] // c["block"]
    token, plain = 2 * c["heads"] * row, 2 * c["heads"] * c["dim"] * size      # keys and values of one token, held and plain
    lengths, queries, op = _lengths(c), _queries(c), c["op"]
    written = sum(_news(c))
    nbytes = flops = 0
    if op in ("write", "refill", "step"):
        nbytes += written * (plain + token)
    if op in ("read", "refill"):
        nbytes += sum(lengths) * (plain + token)
    if op in ("attention", "step"):
        pairs = tokens = 0
        for n, m in zip(lengths, queries):
            if n:
                w = c["window"] or n
                first = n - m                          # the first query's position
                pairs += sum(min(w, first + i + 1) for i in range(m))
                tokens += n - max(0, first + 1 - w)
        nbytes += tokens * token + 2 * sum(queries) * c["heads"] * c["group"] * c["dim"] * size
        flops += 4 * pairs * c["heads"] * c["group"] * c["dim"]
    return {"bytes": int(nbytes), "flops": flops}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------


def _two_to(n):
    """2^n in 64 bits for whole n of a normal value's range."""
    return ((n.to(torch.int64) + 1023) * 2 ** 52).view(torch.float64)


def _binade(v):
    """floor(log2 |v|) of 64-bit values, from the exponent field."""
    return v.contiguous().view(torch.int64) // 2 ** 52 % 2048 - 1023


def _elements64(codes, fmt):
    """Sign, exponent and mantissa fields of packed codes, put together in 64 bits."""
    bits, eta, mu = FMT[fmt]
    c = codes.to(torch.int64)
    if bits == 4:
        c = torch.stack((c % 16, c // 16), -1).flatten(-2)
    if not eta:
        return torch.where(c >= 2 ** (bits - 1), c - 2 ** bits, c).double()
    field = c // 2 ** mu % 2 ** eta
    mant = (c % 2 ** mu).double() / 2 ** mu + (field > 0)
    return (1 - 2 * (c // 2 ** (bits - 1))) * mant * _two_to(field.clamp(min=1) - (2 ** (eta - 1) - 1))


def _stored64(codes, scales, fmt, block):
    return _elements64(codes, fmt) * _two_to(scales.to(torch.int64) - 127).repeat_interleave(block, -1)


def _rounded64(v, fmt, block):
    """Element values and shared exponents of 64-bit values, blocks along the last dimension."""
    bits, eta, mu = FMT[fmt]
    big = v.abs().reshape(*v.shape[:-1], -1, block).max(-1).values
    shared = torch.where(big > 0, _binade(big) - (2 ** (eta - 1) if eta else bits - 2), -127).clamp(-127, 127)
    p = v / _two_to(shared).repeat_interleave(block, -1)
    if not eta:
        top = 2 ** (bits - 1) - 1
        return torch.clamp(torch.trunc(p + torch.copysign(torch.full_like(p, 0.5), p)), -top, top), shared
    top = {"e4m3": 448.0, "e2m1": 6.0}[fmt]
    grid = _two_to(_binade(p.abs().clamp(min=2.0 ** (2 - 2 ** (eta - 1)))) - mu)
    return torch.clamp(torch.round(p / grid) * grid, -top, top), shared


def exact(case, seed):
    s = prepare(case, seed)
    c, fmt, block, page = case, s["fmt"], s["block"], s["page"]
    lengths, queries, news = _lengths(c), _queries(c), _news(c)
    kc, ks, vc, vs = s["cache"]
    wrote = c["op"] in ("write", "refill", "step")

    def new_rows(x, b):                                # what a write keeps of a sequence's new tokens: elements, exponents
        at = sum(queries[:b])
        return _rounded64(x[at:at + news[b]].double(), fmt, block)

    def sequence(b, head=slice(None)):                 # keys and values of a sequence, [tokens, heads, dim]
        t = torch.arange(lengths[b], device=kc.device)
        pages, off = s["table"][b].long()[t // page], t % page
        got = [_stored64(codes[pages, :, off], scales[pages, :, off], fmt, block) for codes, scales in ((kc, ks), (vc, vs))]
        if wrote and news[b]:
            for x, y in zip(got, (s["k"], s["v"])):
                p, e = new_rows(y, b)
                x[lengths[b] - news[b]:] = p * _two_to(e).repeat_interleave(block, -1)
        return [x[:, head] for x in got]

    if c["op"] in ("read", "refill"):
        parts = [sequence(b) for b in range(c["batch"]) if lengths[b]]
        return tuple(torch.cat([p[i] for p in parts]) for i in range(2))
    held = {}
    if wrote:
        held = {"k": _elements64(kc, fmt) if fmt == "e4m3" else None, "k_scales": None,
                "v": _elements64(vc, fmt) if fmt == "e4m3" else None, "v_scales": None}
        for b in range(c["batch"]):
            if news[b] and fmt == "e4m3":
                t = torch.arange(lengths[b] - news[b], lengths[b], device=kc.device)
                pages = s["table"][b].long()[t // page]
                held["k"][pages, :, t % page] = new_rows(s["k"], b)[0]
                held["v"][pages, :, t % page] = new_rows(s["v"], b)[0]
        if c["op"] == "write":
            return held if fmt == "e4m3" else None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=kc.device)
    at, group = 0, c["group"]
    for b in range(c["batch"]):
        if lengths[b] and queries[b]:
            k, v = sequence(b)
            i = torch.arange(lengths[b], device=kc.device)
            mine = torch.arange(lengths[b] - queries[b], lengths[b], device=kc.device).view(-1, 1)
            hidden = i > mine
            if c["window"]:
                hidden |= mine - i >= c["window"]
            for h in range(s["q"].shape[1]):
                score = s["q"][at:at + queries[b], h].double() @ k[:, h // group].T / c["dim"] ** 0.5
                out[at:at + queries[b], h] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ v[:, h // group]
        at += queries[b]
    return out if c["op"] == "attention" else {"out": out, **held}
