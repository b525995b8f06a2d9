"""The operators of a paged key-value pool whose speed is followed: what answers from retained caches is built of.

  write    rows of keys and values into slots of a paged pool, as they are or in 8 bits with a scale per (token, kv-head)
  read     slots of the pool back as rows
  decode   attention of one new token per sequence over its pages, the token's own key and value appended in passing
  prompt   causal attention of whole prompts of different lengths, packed one after the other

Where ``own`` is false a pass takes the plain form: elementary torch operations in 32 bits, rounded once at the end.  Where it
is true it makes the calls that a program makes of ``paper_2604_16734_b200.pool.Pool``.

A case is a dict:

  op                        "write", "read", "decode" or "prompt"
  hq, hkv, d, dtype         query heads, kv-heads, head dimension, "fp32" or "bf16"
  pages                     "plain" (the pages hold the dtype) or "int8"
  page                      tokens per page
  seqs, longest, shape      sequences, the longest one's length; ``shape`` seeds the other lengths
  empty                     how many of the sequences have no entry at all
  append                    decode: the new token's key and value are written to its page by the same call
  heads_first               write: the rows come as a retained cache holds them, [kv-head][row][d], not token by token

In 8 bits a pass of "write" also reads its rows back: what is returned is the values that the pages stand for.
"""
import math
import random

import torch

own = False

SZ = {"fp32": 4, "bf16": 2}
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _case(name, op, heads, d, seqs, longest, dtype="bf16", pages="plain", page=64, shape=0, empty=0, append=False,
          heads_first=False):
    c = dict(op=op, hq=heads[0], hkv=heads[1], d=d, dtype=dtype, pages=pages, page=page, seqs=seqs, longest=longest, shape=shape,
             empty=empty, append=append, heads_first=heads_first)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # One image request's retained cache of one layer (192 entries, as many kv-heads as query heads) handed to the pool.
        _case("write_image", "write", (32, 32), 128, 1, 192, heads_first=True),
        # Packed prompts' keys and values in 8 bits, as after a prefill of sixteen long prompts, and read back.
        _case("write_batch_int8", "write", (32, 8), 128, 16, 4096, pages="int8", shape=1),
        # A small cache at full precision taken out of the pool again, ragged.
        _case("read_tiles_fp32", "read", (28, 4), 128, 3, 1024, dtype="fp32", page=16, shape=2),
        # Requests that leave the pool: 8-bit pages back to bf16 rows.
        _case("read_batch_int8", "read", (32, 8), 128, 12, 4231, pages="int8", shape=3),
        # The smallest decode step: one request at full precision, the repository's smallest configuration.  Latency.
        _case("decode_one_fp32", "decode", (4, 1), 64, 1, 128, dtype="fp32", page=16, append=True),
        # A few image requests (budget 192 and some text), as many kv-heads as query heads.
        _case("decode_image", "decode", (32, 32), 128, 8, 251, page=32, shape=4, append=True),
        # One uncompressed long context: the work has to be split over the length.
        _case("decode_long", "decode", (32, 8), 128, 1, 131149, page=128, append=True),
        # Video requests at a budget of 4096 with answers under way.
        _case("decode_video_batch", "decode", (32, 8), 128, 64, 4600, shape=5, append=True),
        # A large batch on 8-bit pages, seven query heads per kv-head, some requests still empty.
        _case("decode_batch_int8", "decode", (28, 4), 128, 192, 4500, pages="int8", shape=6, empty=3),
        # Short questions that arrive together, a few tokens to two hundred.
        _case("prompt_short", "prompt", (28, 4), 128, 24, 200, shape=7),
        # Long text prompts.
        _case("prompt_long", "prompt", (32, 8), 128, 8, 4096, shape=8),
        # Full precision, for programs that check or calibrate.
        _case("prompt_fp32", "prompt", (8, 2), 64, 6, 600, dtype="fp32", shape=9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w, m = work(c), most.setdefault(c["op"] + ("fp32" if c["op"] == "prompt" and c["dtype"] == "fp32" else ""), [0, 0])
        m[0], m[1] = max(m[0], w["bytes"]), max(m[1], w["flops"])
    while True:
        op = rng.choice(["write", "read", "decode", "decode", "prompt"])
        heads = rng.choice([(4, 1), (8, 2), (12, 4), (16, 4), (28, 4), (32, 8), (32, 32), (16, 1)])
        dtype = "fp32" if rng.random() < 0.25 else "bf16"
        c = _case(None, op, heads, rng.choice([64, 128, 128]), _log(rng, 1, 192 if op == "decode" else 32),
                  _log(rng, 1, {"decode": 131072, "prompt": 4096}.get(op, 8192)), dtype,
                  "plain" if op == "prompt" else rng.choice(["plain", "int8"]), rng.choice([16, 32, 64, 128]), rng.randrange(1 << 20))
        if op == "decode":
            c["empty"] = rng.choice([0, 0, min(2, c["seqs"] - 1)])
            c["append"] = c["pages"] == "plain" and rng.random() < 0.7
        if op == "write":
            c["heads_first"] = rng.random() < 0.5
        w, m = work(c), most[op + ("fp32" if op == "prompt" and dtype == "fp32" else "")]
        padded = c["seqs"] * c["longest"]           # (what the plain forms lay out)
        room = padded * c["longest"] * c["hq"] <= 8 * 4096 * 4096 * 32 if op == "prompt" else padded * c["hkv"] * c["d"] <= 1 << 30
        if w["bytes"] <= m[0] and w["flops"] <= m[1] and room:
            return c


def lengths(c):
    """The sequences' lengths: one has the longest, the others are spread from a twentieth of it on, the last ``empty`` have none."""
    rng = random.Random(c["shape"])
    lens = [c["longest"]] + [rng.randint(max(1, c["longest"] // 20), c["longest"]) for _ in range(c["seqs"] - 1)]
    for i in range(c["empty"]):
        lens[-1 - i] = 0
    return lens


def _rows(gen, c, n, heads):
    """n rows of ``heads`` heads with gains that differ by channel, as projections have them."""
    x = torch.randn(n, heads, c["d"], generator=gen, device="cuda")
    return x * torch.exp(0.4 * torch.randn(heads, c["d"], generator=gen, device="cuda"))


def quantised(x):
    """(codes, scales) of rows in 8 bits: what the pages hold."""
    amax = x.abs().amax(-1, keepdim=True)
    scale = amax * torch.full_like(amax, 1.0 / 127.0)
    scale = torch.where(scale < 2.0 ** -126, torch.zeros_like(scale), scale)
    inv = torch.where(scale > 0, torch.ones_like(scale) / scale, torch.zeros_like(scale))
    return torch.round(x * inv).clamp(-127, 127).to(torch.int8), scale.squeeze(-1)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lens, dtype, ps = lengths(c), TORCH[c["dtype"]], c["page"]
    n = sum(lens)
    s = {"case": c, "lens_list": lens, "scale": 1.0 / math.sqrt(c["d"])}
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    starts = torch.cumsum(s["lens"].long(), 0) - s["lens"].long()
    s["seq"] = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), s["lens"].long())
    s["at"] = torch.arange(n, device="cuda") - starts[s["seq"]]
    if c["op"] == "prompt":
        # the three as a fused projection leaves them: one row of all heads per token
        qkv = torch.cat([_rows(gen, c, n, c["hq"]), _rows(gen, c, n, 2 * c["hkv"])], 1).to(dtype)
        s["q"], s["k"], s["v"] = qkv.split([c["hq"], c["hkv"], c["hkv"]], 1)
    else:
        per_seq = -(-(max(lens) + 1) // ps)
        n_pages = len(lens) * per_seq + 1
        s["table"] = torch.randperm(n_pages, generator=gen, device="cuda")[:len(lens) * per_seq].view(len(lens), per_seq).int()
        s["slots"] = s["table"].long()[s["seq"], s["at"] // ps] * ps + s["at"] % ps
        # one layer of the pool: keys, values and, in 8 bits, their scales, one after the other
        held = (n_pages, c["hkv"], ps, c["d"])
        size = math.prod(held)
        if c["pages"] == "int8":
            up = -(-(size // c["d"] * 4) // 256) * 256
            s["blob"] = torch.zeros(2 * size + 2 * up, dtype=torch.uint8, device="cuda")
            s["k_pages"], s["v_pages"] = (s["blob"][i * size:(i + 1) * size].view(torch.int8).view(held) for i in (0, 1))
            s["k_scales"], s["v_scales"] = (s["blob"][2 * size + i * up:][:size // c["d"] * 4].view(torch.float32).view(held[:3]) for i in (0, 1))
        else:
            size *= SZ[c["dtype"]]
            s["blob"] = torch.zeros(2 * size, dtype=torch.uint8, device="cuda")
            s["k_pages"], s["v_pages"] = (s["blob"][i * size:(i + 1) * size].view(dtype).view(held) for i in (0, 1))
        if c["op"] == "write":
            s["k"], s["v"] = _rows(gen, c, n, c["hkv"]).to(dtype), _rows(gen, c, n, c["hkv"]).to(dtype)
            if c["heads_first"]:
                s["k"], s["v"] = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (s["k"], s["v"]))
        else:
            # pages that are in use are full of earlier rows; what lies behind a sequence's end is stale
            for which in ("k", "v"):
                pages = s[which + "_pages"]
                for first in range(0, n_pages, 512):
                    some = pages[first:first + 512]
                    x = _rows(gen, c, some.shape[0] * ps, c["hkv"]).view(-1, ps, c["hkv"], c["d"]).transpose(1, 2)
                    if c["pages"] == "int8":
                        some.copy_(quantised(x)[0])
                        s[which + "_scales"][first:first + 512] = quantised(x)[1]
                    else:
                        some.copy_(x)
        if c["op"] == "decode":
            s["q"] = _rows(gen, c, len(lens), c["hq"]).to(dtype)
            if c["append"]:
                s["k"], s["v"] = _rows(gen, c, len(lens), c["hkv"]).to(dtype), _rows(gen, c, len(lens), c["hkv"]).to(dtype)
    if own:
        from paper_2604_16734_b200.pool import Pool
        paged = c["op"] != "prompt"
        s["pool"] = Pool(c["hq"], c["hkv"], c["d"], dtype, n_pages if paged else 1, page_size=ps, page_format=c["pages"],
                         max_seqs=len(lens), blob=s["blob"].view(1, -1) if paged else None)
        if not paged:
            s["plan"] = s["pool"].plan(lens)
    return s


def _values(s, which, index):
    """Pages ``index`` ([...] of them) of keys or values in 32 bits."""
    x = s[which + "_pages"][index].float()
    return x * s[which + "_scales"][index].unsqueeze(-1) if s["case"]["pages"] == "int8" else x


def _plain_put(s, k, v, slots):
    ps = s["case"]["page"]
    page, row = slots // ps, slots % ps
    for which, x in (("k", k), ("v", v)):
        if s["case"]["pages"] == "int8":
            s[which + "_pages"][page, :, row], s[which + "_scales"][page, :, row] = quantised(x.float())
        else:
            s[which + "_pages"][page, :, row] = x


def _plain_read(s):
    ps, dtype = s["case"]["page"], TORCH[s["case"]["dtype"]]
    page, row = s["slots"] // ps, s["slots"] % ps
    out = []
    for which in ("k", "v"):
        x = s[which + "_pages"][page, :, row].float()
        out.append((x * s[which + "_scales"][page, :, row].unsqueeze(-1) if s["case"]["pages"] == "int8" else x).to(dtype))
    return out


def _softmax_product(scores, mask, v):
    """Rows of probabilities times values, and the rows' log-sum-exp; nothing comes of a row that sees no key."""
    scores.masked_fill_(~mask, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(torch.isfinite(top), top, torch.zeros_like(top))).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    return out, (torch.where(torch.isfinite(top), top, torch.zeros_like(top)) + total.log()).squeeze(-1)


def _plain_decode(s):
    c = s["case"]
    lens = s["lens"].long()
    if c["append"]:
        slots = s["table"].long().gather(1, (lens // c["page"]).unsqueeze(1)).squeeze(1) * c["page"] + lens % c["page"]
        _plain_put(s, s["k"], s["v"], slots)
        lens = lens + 1
    b, index = len(s["lens_list"]), s["table"].long()
    lay = lambda x: x.transpose(1, 2).reshape(b, c["hkv"], -1, c["d"])  # noqa: E731
    q = s["q"].float().view(b, c["hkv"], -1, c["d"])
    scores = torch.matmul(q, lay(_values(s, "k", index)).transpose(2, 3)) * s["scale"]
    mask = torch.arange(scores.shape[-1], device="cuda") < lens.view(-1, 1, 1, 1)
    out, lse = _softmax_product(scores, mask, lay(_values(s, "v", index)))
    return out.reshape(b, c["hq"], c["d"]).to(TORCH[c["dtype"]]), lse.reshape(b, c["hq"])


def _plain_prompt(s):
    c, b, longest = s["case"], len(s["lens_list"]), max(s["lens_list"])
    group = c["hq"] // c["hkv"]

    def padded(x):
        y = torch.zeros(b, longest, x.shape[1], c["d"], device="cuda")
        y[s["seq"], s["at"]] = x.float()
        return y.transpose(1, 2)

    k, v = (padded(x).repeat_interleave(group, 1) for x in (s["k"], s["v"]))
    scores = torch.matmul(padded(s["q"]), k.transpose(2, 3)).mul_(s["scale"])
    at = torch.arange(longest, device="cuda")
    out, lse = _softmax_product(scores, at.view(-1, 1) >= at, v)
    return out.transpose(1, 2)[s["seq"], s["at"]].to(TORCH[c["dtype"]]), lse.transpose(1, 2)[s["seq"], s["at"]]


def run(state):
    s, c = state, state["case"]
    if c["op"] == "write":
        if own:
            s["pool"].write(0, s["k"], s["v"], s["slots"])
        else:
            _plain_put(s, s["k"], s["v"], s["slots"])
        if c["pages"] == "plain":
            return {"k": s["k_pages"], "v": s["v_pages"]}
    if c["op"] in ("write", "read"):
        k, v = s["pool"].read(0, s["slots"]) if own else _plain_read(s)
        return {"k": k, "v": v}
    if c["op"] == "decode":
        out, lse = s["pool"].decode(0, s["q"], s["table"], s["lens"], s.get("k"), s.get("v")) if own else _plain_decode(s)
        return {"out": out, "lse": lse, **({"k": s["k_pages"], "v": s["v_pages"]} if c["append"] else {})}
    out, lse = s["pool"].prompt(s["q"], s["k"], s["v"], s["plan"]) if own else _plain_prompt(s)
    return {"out": out, "lse": lse}


def work(case):
    c, lens = case, lengths(case)
    sz, n, b = SZ[c["dtype"]], sum(lens), len(lens)
    rows = 2 * n * c["hkv"]                                     # of keys and values
    raw = rows * c["d"] * sz
    held = rows * (c["d"] + 4) if c["pages"] == "int8" else raw
    if c["op"] == "write":
        return {"bytes": 8 * n + raw + held + (held + raw if c["pages"] == "int8" else 0), "flops": 2 * rows * c["d"]}
    if c["op"] == "read":
        return {"bytes": 8 * n + held + raw, "flops": rows * c["d"]}
    if c["op"] == "decode":
        new = 2 * b * c["hkv"] * c["d"] * sz if c["append"] else 0
        return {"bytes": held + 2 * new + b * c["hq"] * (2 * c["d"] * sz + 4) + 4 * b + 4 * sum(-(-x // c["page"]) for x in lens),
                "flops": 4 * c["hq"] * c["d"] * (n + (b if c["append"] else 0))}
    return {"bytes": n * (2 * c["hq"] + 2 * c["hkv"]) * c["d"] * sz + 4 * n * c["hq"],
            "flops": 4 * c["hq"] * c["d"] * sum(x * (x + 1) // 2 for x in lens)}


def exact(case, seed):
    """The definitions in 64 bits, sequence by sequence."""
    c, s, ps = case, prepare(case, seed), case["page"]
    lens, group = s["lens_list"], case["hq"] // case["hkv"]
    wide = torch.float64

    def eight_bit(x):
        step = x.abs().max(-1, keepdim=True).values / 127
        return torch.where(step > 0, torch.round(x / step) * step, x)

    if c["op"] == "write":
        if c["pages"] == "int8":
            return {"k": eight_bit(s["k"].to(wide)), "v": eight_bit(s["v"].to(wide))}
        out = {}
        for which in ("k", "v"):
            flat = s[which + "_pages"].to(wide).transpose(1, 2).contiguous().view(-1, c["hkv"], c["d"])
            flat.index_copy_(0, s["slots"], s[which].to(wide))
            out[which] = flat.view(-1, ps, c["hkv"], c["d"]).transpose(1, 2).contiguous()
        return out

    def rows_of(which, table, count):
        """The first ``count`` rows of a sequence: [kv-head][row][d]."""
        x = s[which + "_pages"][table].to(wide)
        if c["pages"] == "int8":
            x = x * s[which + "_scales"][table].to(wide)[..., None]
        return x.permute(1, 0, 2, 3).reshape(c["hkv"], -1, c["d"])[:, :count]

    if c["op"] == "read":
        return {which: torch.cat([rows_of(which, s["table"][i].long(), m).transpose(0, 1) for i, m in enumerate(lens)]) for which in ("k", "v")}
    outs, lses = [], []
    if c["op"] == "decode":
        for i, m in enumerate(lens):
            k, v = rows_of("k", s["table"][i].long(), m), rows_of("v", s["table"][i].long(), m)
            if c["append"]:
                k, v = torch.cat([k, s["k"][i].to(wide)[:, None]], 1), torch.cat([v, s["v"][i].to(wide)[:, None]], 1)
            q = s["q"][i].to(wide).view(c["hkv"], group, c["d"])
            z = torch.einsum("hgd,hnd->hgn", q, k) * s["scale"]
            lse = torch.logsumexp(z, -1) if z.shape[-1] else torch.full(z.shape[:2], -math.inf, dtype=wide, device="cuda")
            w = torch.exp(z - lse[..., None])
            outs.append(torch.einsum("hgn,hnd->hgd", w, v).reshape(c["hq"], c["d"]))
            lses.append(lse.reshape(c["hq"]))
        return {"out": torch.stack(outs), "lse": torch.stack(lses), **({"k": None, "v": None} if c["append"] else {})}
    first = 0
    for m in lens:
        q, k, v = (x[first:first + m].to(wide) for x in (s["q"], s["k"], s["v"]))
        out = torch.zeros(m, c["hq"], c["d"], dtype=wide, device="cuda")
        lse = torch.zeros(m, c["hq"], dtype=wide, device="cuda")
        later = torch.ones(m, m, dtype=torch.bool, device="cuda").triu(1)
        for h in range(c["hq"]):
            z = (q[:, h] @ k[:, h // group].T * s["scale"]).masked_fill_(later, -math.inf)
            lse[:, h] = torch.logsumexp(z, -1)
            out[:, h] = torch.exp(z - lse[:, h, None]) @ v[:, h // group]
        outs.append(out)
        lses.append(lse)
        first += m
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
