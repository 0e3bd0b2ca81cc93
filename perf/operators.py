"""The language-model side of the prefix, as operators with their plain forms: new tokens' keys and values into a paged
cache (rotated by their positions on the way), and the attention of one new token per sequence over that cache.

Cache layout: K pages [page][KV head][token][head dim], V pages transposed, [page][KV head][head dim][token]; bf16, or
e4m3 with one scale for K and one for V (a value is what is stored times the scale).
"""
import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}


def listed():
    """Sizes: the bundled experts' K/V heads (1 x 256, 2 x 128, 4 x 64), prefixes and fleets; long ones are generic."""
    return [
        # the token that a model decoding a sub-task for one robot has just made: latency alone counts
        _append("append_token", 1, 1, 816, 1, 256, 16, "bf16", "bf16", 256),
        # the same for a fleet of 64, in an 8-bit cache
        _append("append_token_fleet", 64, 1, 1500, 2, 128, 64, "bf16", "e4m3", 128),
        # the small expert's prefix handed over in fp32, neighbouring pairs rotated
        _append("append_small_f32", 1, 64, 0, 4, 64, 16, "f32", "bf16", 64, pairs=True),
        # one robot's new vision-language prefix
        _append("append_prefix", 1, 816, 0, 1, 256, 16, "bf16", "bf16", 256),
        # 16 prompts of uneven length behind a long history, half of each head rotated, rows of padding behind them
        _append("append_ragged", 16, 1021, 50000, 2, 128, 32, "bf16", "e4m3", 64, ragged=True),
        # a fleet's prefixes at once: bandwidth counts
        _append("append_prefix_fleet", 64, 816, 0, 1, 256, 64, "bf16", "bf16", 256),
        # the first tokens of a short prompt
        _attend("attend_short", 3, 61, 4, 4, 64, 16, "f32", "bf16", 64, ragged=True),
        # one robot decoding behind its prefix: latency counts
        _attend("attend_prefix", 1, 817, 8, 1, 256, 16, "bf16", "bf16", 256),
        # a fleet decoding together
        _attend("attend_prefix_fleet", 64, 900, 8, 1, 256, 64, "bf16", "bf16", 256),
        # prompts from a few tokens to thousands in one batch, 8-bit cache
        _attend("attend_ragged", 48, 16383, 12, 2, 128, 32, "bf16", "e4m3", 128, ragged=True),
        # a batch of long conversations without grouped heads, fp32 queries
        _attend("attend_heads", 8, 4001, 16, 16, 64, 128, "f32", "bf16", 32, pairs=True),
        # one very long history
        _attend("attend_long", 1, 131071, 32, 8, 128, 64, "bf16", "bf16", 128),
    ]


def draw(rng):
    """Another case of those ranges, with no more keys and products than the largest listed one (the batch padded to its longest)."""
    wide = lambda a, b: int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))  # noqa: E731
    hkv, hd = rng.choice([1, 1, 2, 4, 8]), rng.choice([64, 128, 256])
    page, cache, given = rng.choice([16, 32, 64, 128]), rng.choice(["bf16", "bf16", "e4m3"]), rng.choice(["bf16", "bf16", "f32"])
    rope, pairs, ragged, seqs = rng.choice([hd, hd, hd // 2, 0]), rng.random() < 0.3, rng.random() < 0.5, wide(1, 64)
    if rng.random() < 0.5:
        rows = 1 if rng.random() < 0.4 else wide(2, max(2, min(4096, 64 * 816 * 256 // (4 if given == "f32" else 1) // (seqs * hkv * hd))))
        return _append(None, seqs, rows, rng.choice([0, wide(1, 100000)]), hkv, hd, page, given, cache, rope, pairs, ragged)
    group = rng.choice([1, 2, 4, 5, 8, 16])
    longest = wide(1, max(1, min(131071, 131071 * 8 * 128 // (seqs * hkv * hd * -(-group // 4)))))
    return _attend(None, seqs, longest, hkv * group, hkv, hd, page, given, cache, rope, pairs, ragged)


def _append(name, seqs, rows, before, kv_heads, head_dim, page, given, cache, rope, pairs=False, ragged=False):
    case = dict(op="append", seqs=seqs, rows=rows, before=before, heads=kv_heads, kv_heads=kv_heads, head_dim=head_dim,
                page=page, given=given, cache=cache, rope=rope, pairs=pairs, ragged=ragged)
    return {"name": name, **case} if name else case


def _attend(name, seqs, longest, heads, kv_heads, head_dim, page, given, cache, rope, pairs=False, ragged=False):
    case = dict(op="attend", seqs=seqs, longest=longest, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page,
                given=given, cache=cache, rope=rope, pairs=pairs, ragged=ragged)
    return {"name": name, **case} if name else case


def _lengths(case):
    """(new rows, length after them) of each sequence: a matter of the case, so that its work is known without inputs."""
    r = random.Random(case["seqs"] * 1000003 + case.get("rows", 0) * 101 + case.get("longest", 0))
    new, after = [], []
    for b in range(case["seqs"]):
        most = case["rows"] if case["op"] == "append" else case["longest"]
        # ragged: from one token to all, spread over the logarithm; else nearly even; the first is the longest
        n = most if b == 0 else int(math.exp(r.uniform(0, math.log(most)))) if case["ragged"] else max(1, most - r.randrange(1 + most // 16))
        if case["op"] == "append":
            new.append(n)
            after.append(n + (r.randrange(case["before"] + 1) if case["ragged"] else case["before"]))
        else:
            new.append(1)
            after.append(n)
    return new, after


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    new, after = _lengths(case)
    seqs, hkv, hd, page = case["seqs"], case["kv_heads"], case["head_dim"], case["page"]
    given, cache = _TYPES[case["given"]], _TYPES[case["cache"]]
    # pages that the call touches get one of their own, in shuffled order; -1 behind the last. Earlier pages of an
    # append are not touched: they stand in for a history that lies elsewhere in the pool.
    wide = max(-(-n // page) for n in after) + 1
    first = [(n - m) // page if case["op"] == "append" else 0 for n, m in zip(after, new)]
    last = [-(-n // page) for n in after]
    count = sum(b - a for a, b in zip(first, last))
    order = torch.randperm(count + 2, generator=g, device="cuda").to(torch.int32)
    table = torch.full((seqs, wide), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(seqs):
        table[b, :first[b]] = order[count]
        table[b, first[b]:last[b]] = order[at:at + last[b] - first[b]]
        at += last[b] - first[b]
    scales = (0.02, 0.02) if case["cache"] == "e4m3" else (1.0, 1.0)
    fill = lambda scale, *shape: (normal(*shape) / scale).clamp(-448, 448).to(cache)  # noqa: E731
    s = dict(case=case, scales=scales, table=table, lens=dev(after), k_pool=fill(scales[0], 1, count + 2, hkv, page, hd),
             v_pool=fill(scales[1], 1, count + 2, hkv, hd, page))
    if case["op"] == "append":
        total = sum(new)
        rows = total + (5 if case["ragged"] else 0)  # rows of padding behind the last sequence
        s["total"] = total
        s["k"], s["v"] = (normal(rows, hkv, hd).to(given) for _ in range(2))
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        s["starts"] = dev(starts)
    else:
        s["q"] = (1.5 * normal(seqs, case["heads"], hd)).to(given)
        s["out"] = torch.empty_like(s["q"])
    if own:  # the handle that a program keeps beside its cache
        import paper_2609_37772_amd as U
        s["kv"] = U.PagedKV(1, case["heads"], hkv, hd, page, count + 2, seqs, dtype=cache, rope_dim=case["rope"],
                            rope_theta=10000.0, rope_pairs=case["pairs"], k_scale=scales[0], v_scale=scales[1],
                            k=s["k_pool"], v=s["v_pool"])
    return s


def run(state):
    s, case = state, state["case"]
    if case["op"] == "append":
        if own:
            # one row per sequence needs no starts
            s["kv"].append(0, s["k"], s["v"], s["table"], s["lens"], None if case["rows"] == 1 and not case["ragged"] else s["starts"])
        else:
            _plain_append(s)
        return {"k": s["k_pool"], "v": s["v_pool"]}
    if own:
        return s["kv"].attend(0, s["q"], s["table"], s["lens"], out=s["out"])
    return _plain_attend(s)


def _rotated(x, positions, case):
    """x [rows][heads][head dim] in fp32, each row rotated by its position; the angles in 64 bits."""
    rd, pairs = case["rope"], case["pairs"]
    if rd == 0:
        return x
    freq = 10000.0 ** (-torch.arange(0, rd, 2, dtype=torch.float64, device=x.device) / rd)
    angle = positions.double()[:, None, None] * freq
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    a, b = (x[..., 0:rd:2], x[..., 1:rd:2]) if pairs else (x[..., :rd // 2], x[..., rd // 2:rd])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((ra, rb), -1).flatten(-2) if pairs else torch.cat((ra, rb), -1)
    return torch.cat((turned, x[..., rd:]), -1)


def _stored(x, scale, cache):
    return (x / scale).clamp(-448, 448).to(cache) if cache == torch.float8_e4m3fn else x.to(cache)


def _plain_append(s):
    case, page, n = s["case"], s["case"]["page"], s["total"]
    cache = _TYPES[case["cache"]]
    starts = s["starts"].long()
    row = torch.arange(n, device=starts.device)
    seq = torch.searchsorted(starts, row, right=True) - 1
    pos = s["lens"].long()[seq] - starts[seq + 1] + row
    where, at = s["table"].long()[seq, pos // page], pos % page
    k = _stored(_rotated(s["k"][:n].float(), pos, case), s["scales"][0], cache)
    v = _stored(s["v"][:n].float(), s["scales"][1], cache)
    bits = torch.uint8 if cache == torch.float8_e4m3fn else torch.int16
    s["k_pool"].view(bits)[0][where, :, at, :] = k.view(bits)
    s["v_pool"].view(bits)[0][where, :, :, at] = v.view(bits)


def _plain_attend(s):
    case, hkv, hd = s["case"], s["case"]["kv_heads"], s["case"]["head_dim"]
    seqs, heads = s["q"].shape[0], s["q"].shape[1]
    lens, table = s["lens"].long(), s["table"].long().clamp(min=0)
    q = _rotated(s["q"].float(), lens - 1, case).view(seqs, hkv, heads // hkv, hd)
    bits = torch.uint8 if case["cache"] == "e4m3" else torch.int16
    cache = _TYPES[case["cache"]]
    k = s["k_pool"].view(bits)[0][table].view(cache).float()  # [seq][page][head][token][dim]
    k = k.permute(0, 2, 1, 3, 4).reshape(seqs, hkv, -1, hd)
    score = torch.matmul(q, k.transpose(2, 3)) * (s["scales"][0] / math.sqrt(hd))
    del k
    hidden = (torch.arange(score.shape[-1], device=lens.device) >= lens[:, None])[:, None, None, :]
    score = score.masked_fill(hidden, -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    v = s["v_pool"].view(bits)[0][table].view(cache).float()  # [seq][page][head][dim][token]
    v = v.permute(0, 2, 1, 4, 3).reshape(seqs, hkv, -1, hd)
    return (torch.matmul(p, v) * s["scales"][1]).view(seqs, heads, hd).to(s["q"].dtype)


def work(case):
    new, after = _lengths(case)
    hkv, hd = case["kv_heads"], case["head_dim"]
    given, cache = _TYPES[case["given"]].itemsize, _TYPES[case["cache"]].itemsize
    pages = lambda n: -(-n // case["page"])  # noqa: E731
    if case["op"] == "append":
        rows = sum(new)
        touched = sum(pages(n) - (n - m) // case["page"] for n, m in zip(after, new))
        return {"bytes": 2 * rows * hkv * hd * (given + cache) + 4 * (touched + 2 * case["seqs"] + 1), "flops": 3 * rows * hkv * case["rope"]}
    keys = sum(after)
    return {"bytes": 2 * keys * hkv * hd * cache + 2 * case["seqs"] * case["heads"] * hd * given + 4 * (sum(map(pages, after)) + case["seqs"]),
            "flops": 4 * keys * case["heads"] * hd}


def exact(case, seed):
    s = prepare(case, seed)
    new, after = _lengths(case)
    hkv, hd, page, rd = case["kv_heads"], case["head_dim"], case["page"], case["rope"]
    group = case["heads"] // hkv
    table = s["table"].cpu()
    # pair i of a rotated head, as complex numbers, is turned by position * 10000^(-2i/rope)
    first = torch.arange(rd // 2, device="cuda") * (2 if case["pairs"] else 1)
    second = first + (1 if case["pairs"] else rd // 2)
    speed = torch.exp(-math.log(10000.0) * 2 * torch.arange(rd // 2, dtype=torch.float64, device="cuda") / max(rd, 1))

    def turn(x, positions):
        x = x.clone()
        z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(speed), positions[:, None] * speed)[:, None]
        x[..., first], x[..., second] = z.real, z.imag
        return x

    if case["op"] == "append":
        # both pools by token, [page * token][head][dim]
        kp = s["k_pool"].double()[0].permute(0, 2, 1, 3).reshape(-1, hkv, hd)
        vp = s["v_pool"].double()[0].permute(0, 3, 1, 2).reshape(-1, hkv, hd)
        row = 0
        for b in range(case["seqs"]):
            pos = torch.arange(after[b] - new[b], after[b], device="cuda")
            k = turn(s["k"][row:row + new[b]].double(), pos.double())
            v = s["v"][row:row + new[b]].double()
            row += new[b]
            if case["cache"] == "e4m3":
                k, v = ((x / scale).clamp(-448, 448) for x, scale in zip((k, v), s["scales"]))
            slot = table[b].to("cuda").long()[pos // page] * page + pos % page
            kp[slot], vp[slot] = k, v
        return {"k": kp.view(-1, page, hkv, hd).permute(0, 2, 1, 3)[None].contiguous(),
                "v": vp.view(-1, page, hkv, hd).permute(0, 2, 3, 1)[None].contiguous()}
    out = torch.empty((case["seqs"], case["heads"], hd), dtype=torch.float64, device="cuda")
    for b in range(case["seqs"]):
        q = turn(s["q"][b:b + 1].double(), torch.tensor([after[b] - 1.0], dtype=torch.float64, device="cuda"))[0]
        ids = table[b, :-(-after[b] // page)].tolist()
        at = torch.tensor(ids, device="cuda")
        bits = torch.uint8 if case["cache"] == "e4m3" else torch.int16
        kb = s["k_pool"].view(bits)[0][at].view(s["k_pool"].dtype)
        vb = s["v_pool"].view(bits)[0][at].view(s["v_pool"].dtype)
        for h in range(hkv):
            k = kb[:, h].reshape(-1, hd)[:after[b]].double() * s["scales"][0]
            v = vb[:, h].transpose(1, 2).reshape(-1, hd)[:after[b]].double() * s["scales"][1]
            w = torch.softmax(q[h * group:(h + 1) * group] @ k.T.contiguous() / math.sqrt(hd), -1)
            out[b, h * group:(h + 1) * group] = w @ v
    return out
