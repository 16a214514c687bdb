"""What the operators of the paged cache are measured on: their calls, their plain forms and their definition in 64 bits.

A sequence's keys and values live in pages, in the context's own type or in 4 bits (e2m1 codes, an e4m3 scale for every 16
channels and one float each for all of K and all of V).  Tokens are appended behind what a sequence holds, with their
rotation; an eviction's retained rows go straight into pages; pages are read back as values; and queries attend to them.
"""
import math
import random

import torch

own = False      # True: run() calls the framework's operators; False: their plain forms

D = 128
FLOAT = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    base = dict(dtype="bf16", format="fp4", page_rows=64, batch=1, len_lo=0, len_hi=0, new_lo=1, new_hi=1, softcap=0.0,
                k_scale=1.0, v_scale=1.0, queries=False, interleaved=False, idle=0, ragged=1)
    llama8, qwen, llama70, tiny = (dict(q_heads=a, kv_heads=b) for a, b in ((32, 8), (28, 4), (64, 8), (8, 2)))
    return [
        # one decode step of 64 sequences whose prompts were evicted to about a thousand rows: latency
        dict(base, **llama8, name="append_step_fp4", op="append", batch=64, len_lo=300, len_hi=1100, page_rows=16, queries=True, ragged=2),
        # eight prompts of a serving batch, whole, into bf16 pages, queries rotated too
        dict(base, **llama8, name="append_prompts_bf16", op="append", format="native", batch=8, new_lo=1000, new_hi=4100, queries=True, ragged=3),
        # one long prompt of the 70B shape into 4 bits
        dict(base, **llama70, name="append_prompt_fp4", op="append", new_lo=32768, new_hi=32768, v_scale=0.25),
        # the retained rows of one 32k prompt (3 %) into 4 bits
        dict(base, **llama8, name="compact_32k_fp4", op="compact", len_lo=32768, len_hi=32768, new_lo=983, new_hi=983),
        # a ragged serving batch, a tenth of every prompt, into bf16 pages
        dict(base, **llama8, name="compact_serving_bf16", op="compact", format="native", batch=8, len_lo=4096, len_hi=32768, new_lo=409, new_hi=3277,
             page_rows=16, ragged=3),
        # the rows of a short evicted cache back as values, before a second eviction
        dict(base, **qwen, name="read_evicted_fp4", op="read", batch=3, len_lo=200, len_hi=1100, page_rows=32, ragged=4),
        # a whole 128k cache back as values
        dict(base, **llama70, name="read_128k_fp4", op="read", len_lo=131072, len_hi=131072, k_scale=2.0),
        # one token of one sequence on an evicted cache: latency
        dict(base, **llama8, name="decode_evicted_fp4", op="attend", len_lo=1021, len_hi=1021),
        # one token on a whole 128k cache in 4 bits
        dict(base, **qwen, name="decode_128k_fp4", op="attend", len_lo=131071, len_hi=131071, page_rows=32),
        # one token of each sequence of a ragged batch in bf16, two of its places idle, scores capped
        dict(base, **llama8, name="decode_batch_bf16_capped", op="attend", format="native", batch=10, len_lo=4096, len_hi=32768, page_rows=16, softcap=30.0,
             idle=2, ragged=3),
        # a few drafted tokens each on fp32 pages
        dict(base, **tiny, name="verify_f32", op="attend", dtype="f32", format="native", batch=3, len_lo=700, len_hi=2048, new_lo=2, new_hi=5, page_rows=16, ragged=5),
        # the next turn of a conversation: a chunk of tokens over what the first turn left
        dict(base, **llama70, name="chunk_fp4", op="attend", batch=2, len_lo=8000, len_hi=16000, new_lo=300, new_hi=500, ragged=6),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "append", "compact", "read", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    hq, hkv = rng.choice([(8, 2), (28, 4), (32, 8), (64, 8), (16, 16), (40, 8), (24, 2), (12, 1)])
    c = dict(op=op, dtype=dtype, format=rng.choice(["native", "fp4"]), q_heads=hq, kv_heads=hkv, page_rows=rng.choice([16, 32, 64, 128, 256]),
             batch=log(1, 64), softcap=rng.choice([0.0, 0.0, round(rng.uniform(10, 60), 2)]), k_scale=rng.choice([1.0, 1.0, 0.37, 2.0]),
             v_scale=rng.choice([1.0, 1.0, 0.21, 0.5]), queries=rng.random() < 0.5, interleaved=rng.random() < 0.3, idle=0, ragged=rng.randrange(1 << 20))
    if c["batch"] > 2 and rng.random() < 0.4:
        c["idle"] = rng.randrange(1, c["batch"])
    if op == "attend":
        new = rng.choice([1, 1, log(1, 8), log(1, 512)])
        most = min(6.0e7 / (c["batch"] * hkv * D) * 8, 9.0e8 / (c["batch"] * hq * new), 131072)
        c["len_hi"] = log(1, max(2, most))
        c["len_lo"] = rng.choice([0, c["len_hi"] // 3, c["len_hi"]])
        c["new_hi"], c["new_lo"] = new, max(1, new // 2)
    elif op == "append":
        c["new_hi"] = log(1, max(2, 2.0e7 / (c["batch"] * (hkv + (hq if c["queries"] else 0)) * D)))
        c["new_lo"] = rng.choice([0 if c["batch"] > 1 else 1, c["new_hi"]])
        c["len_lo"], c["len_hi"] = 0, log(1, 1000)
    elif op == "compact":
        c["len_hi"] = log(2, max(4, 2.0e7 / (c["batch"] * hkv * D)))
        c["len_lo"] = max(1, c["len_hi"] // 2)
        c["new_hi"] = log(1, c["len_hi"])
        c["new_lo"] = max(1, c["new_hi"] // 3)
    else:
        c["len_hi"] = log(1, max(2, 2.0e7 / (c["batch"] * hkv * D)))
        c["len_lo"] = max(1, c["len_hi"] // 2)
        c["new_lo"] = c["new_hi"] = 1
    return c


def _lengths(case):
    """Rows that each sequence holds before the step (-1: it takes no part), new rows of each."""
    r = random.Random(case["ragged"])
    n = case["batch"]
    lens = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(n)]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(n)]
    if not any(new):
        new[0] = 1
    for b in r.sample(range(n), case["idle"]):
        lens[b] = -1
    if case["op"] == "compact":
        lens = [max(1, x) for x in lens]
        new = [min(k, x) for k, x in zip(new, lens)]
    if case["op"] == "read":
        lens = [max(0, x) for x in lens]
        new = list(lens)
        if not any(new):
            new[0] = lens[0] = 1
    return lens, new


def _cu(counts):
    cu = [0]
    for n in counts:
        cu.append(cu[-1] + n)
    return cu


def work(case):
    lens, new = _lengths(case)
    hq, hkv = case["q_heads"], case["kv_heads"]
    e = 2 if case["dtype"] == "bf16" else 4
    row = 72 if case["format"] == "fp4" else D * e
    live = [(a, n) for a, n in zip(lens, new) if a >= 0]
    t = sum(n for _, n in live)
    flops = 0
    if case["op"] == "attend":
        pairs = sum(n * a + n * (n + 1) // 2 for a, n in live)
        b = sum(2 * hkv * (a + n) * row for a, n in live) + sum(new) * hq * (2 * D * e + 4)
        flops = 4 * pairs * hq * D
    elif case["op"] == "append":
        b = t * (2 * hkv * (D * e + row) + 4) + (2 * t * hq * D * e if case["queries"] else 0)
        b += 2 * t * hkv * D * e if case["format"] == "fp4" else 0          # (the values that are returned)
        flops = 6 * t * (hkv + (hq if case["queries"] else 0)) * D // 2
    elif case["op"] == "compact":
        t = sum(new)
        b = t * hkv * (2 * (D * e + row) + 4)
        b += 2 * t * hkv * D * e if case["format"] == "fp4" else 0
    else:
        b = 2 * t * hkv * (row + D * e)
    return {"bytes": b, "flops": flops}


# ---- the 4-bit format -----------------------------------------------------------------------------------------------
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantise(x, kappa):
    """fp32 [.., 128] -> codes uint8 [.., 64] (even channel in the low half), scales e4m3 as uint8 [.., 8]."""
    g = x.unflatten(-1, (8, 16))
    six = torch.full((), 6.0, device=x.device) * kappa
    top = g.abs().amax(-1)
    fine = torch.isfinite(top)
    s = (top / six).clamp(max=448.0).to(torch.float8_e4m3fn)
    step = s.float().unsqueeze(-1) * torch.full((), 1.0, device=x.device).mul(kappa)
    y = torch.where(step > 0, g.abs() / step, torch.zeros_like(g))
    y = torch.where(fine.unsqueeze(-1), y, torch.zeros_like(y))
    code = (y > 0.25).to(torch.uint8)
    code += y >= 0.75
    code += y > 1.25
    code += y >= 1.75
    code += y > 2.5
    code += y >= 3.5
    code += y > 5.0
    code += ((g < 0) & (code > 0)).to(torch.uint8) * 8
    code = code.flatten(-2)
    scales = torch.where(fine, s.view(torch.uint8), torch.full((), 0x7F, dtype=torch.uint8, device=x.device))
    return code[..., 0::2] + code[..., 1::2] * 16, scales


def _values(codes, scales, kappa, dtype=torch.float32):
    """What codes and scales stand for, [.., 128]."""
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=dtype, device=codes.device)
    both = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    x = table[both.int()].unflatten(-1, (8, 16)) * scales.view(torch.float8_e4m3fn).to(dtype).unsqueeze(-1)
    return (x * kappa).flatten(-2)


def _inv_freq(device):
    return torch.tensor([5.0e5 ** (-2.0 * c / D) for c in range(D // 2)], dtype=torch.float64, device=device)


# ---- a user's program before the call -------------------------------------------------------------------------------
_contexts = {}


def _context(case):
    """The library's context of a model's shape, which a program keeps."""
    import paper_2603_11564_b200 as dq
    key = (case["q_heads"], case["kv_heads"], case["dtype"], case["interleaved"])
    if key not in _contexts:
        _contexts[key] = dq.dapq_create(case["q_heads"], case["kv_heads"], 32, 128, 1 << 18, dq.DAPQ_BF16 if case["dtype"] == "bf16" else dq.DAPQ_F32, 5.0e5,
                                        flags=dq.DAPQ_FLAG_ROPE_INTERLEAVED if case["interleaved"] else 0)
    return _contexts[key]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    f = FLOAT[case["dtype"]]
    hq, hkv, rows = case["q_heads"], case["kv_heads"], case["page_rows"]
    lens, new = _lengths(case)
    held = [0] * len(lens) if case["op"] == "compact" else lens
    ends = [n if case["op"] == "read" else max(0, a) + n for a, n in zip(held, new)]
    pages = [-(-e // rows) for e in ends]
    room, total = max(max(pages), 1), sum(pages) + 1
    order = torch.randperm(total, generator=g, device=dev).int()
    table = torch.full((len(lens), room), -1, dtype=torch.int32)
    cu = _cu(pages)
    at = order.cpu()
    for b, n in enumerate(pages):
        table[b, :n] = at[cu[b]:cu[b] + n]
    first = lens if case["op"] == "append" else [0] * len(lens)
    s = dict(case=case, dev=dev, new=new, first=first, cu=_cu(new), table=table.to(dev), held=torch.tensor(held, dtype=torch.int32, device=dev), room=room, spare=order[-1].long())

    def drawn(*shape):
        # a few channels are far larger than the others, as in keys of real models
        x = torch.randn(*shape, generator=g, device=dev)
        x[..., 5::37] *= 4.0
        return x.to(f)

    for name, scale in (("k", case["k_scale"]), ("v", case["v_scale"])):
        pool = drawn(total, hkv, rows, D)
        if case["format"] == "fp4":
            s[name], s[name + "_scales"] = _quantise(pool.float(), scale)
        else:
            s[name], s[name + "_scales"] = pool, None
    t = s["cu"][-1]
    s["cu_dev"], s["inv_freq"] = torch.tensor(s["cu"], device=dev), _inv_freq(dev)
    if case["op"] == "append":
        s["qkv"] = drawn(t, hq + 2 * hkv, D)                     # as a fused projection leaves them
        s["q_new"], s["k_new"], s["v_new"] = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:]
        first = torch.randint(0, 100000, (len(lens),), generator=g, device=dev)
        n = torch.tensor(new, device=dev)
        step = torch.arange(t, device=dev) - torch.repeat_interleave(s["cu_dev"][:-1], n, output_size=t)
        s["positions"] = (torch.repeat_interleave(first, n, output_size=t) + step).int()
        s["q_rot"] = torch.empty((t, hq, D), dtype=f, device=dev)
    elif case["op"] == "compact":
        s["lens"], s["cu_rows"] = lens, _cu([x + 32 for x in lens])
        s["cu_rows_dev"] = torch.tensor(s["cu_rows"], device=dev)
        s["k_dense"], s["v_dense"] = drawn(hkv, s["cu_rows"][-1], D), drawn(hkv, s["cu_rows"][-1], D)
        picks = [torch.rand(hkv, x, generator=g, device=dev).topk(k, -1).indices.sort(-1).values for x, k in zip(lens, new)]
        s["idx"] = torch.cat(picks, -1).int()
    elif case["op"] == "attend":
        s["q"] = drawn(t, hq, D)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((t, hq), dtype=torch.float32, device=dev)
    if case["op"] == "read" or case["format"] == "fp4":
        s["k_back"], s["v_back"] = (torch.zeros((hkv, t, D), dtype=f, device=dev) for _ in "kv")
    if own:
        import paper_2603_11564_b200 as dq
        s["ctx"] = _context(case)
        s["pages"] = dq.dapq_paged_cache(s["k"], s["v"], s["table"], s["held"], s["k_scales"], s["v_scales"], case["k_scale"], case["v_scale"])
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        _own(s)
    else:
        PLAIN[case["op"]](s)
    if case["op"] == "attend":
        return {"out": s["out"], "lse": s["lse"]}
    got = {"k": s["k_back"], "v": s["v_back"]} if "k_back" in s else {"k": s["k"], "v": s["v"]}
    if case["op"] == "append" and case["queries"]:
        got["q"] = s["q_rot"]
    return got


def _own(s):
    import paper_2603_11564_b200 as dq
    case, ctx, pages = s["case"], s["ctx"], s["pages"]
    if case["op"] == "attend":
        dq.dapq_paged_attend(ctx, pages, s["cu"], s["q"], s["out"], s["lse"], softcap=case["softcap"])
        return
    if case["op"] == "append":
        q = (s["q_new"], s["q_rot"]) if case["queries"] else (None, None)
        dq.dapq_paged_append(ctx, pages, s["cu"], s["k_new"], s["v_new"], s["positions"], *q)
    elif case["op"] == "compact":
        dq.dapq_paged_compact(ctx, s["k_dense"], s["v_dense"], s["cu_rows"], s["lens"], s["idx"], s["new"], pages)
    if "k_back" in s:
        dq.dapq_paged_read(ctx, pages, s["first"], s["new"], s["cu"][:-1], s["k_back"], s["v_back"])


def _sequence_of(s):
    """Sequence of every new row, and its number within it."""
    t = s["cu"][-1]
    row = torch.arange(t, device=s["dev"])
    b = torch.searchsorted(s["cu_dev"], row, right=True) - 1
    return b, row - s["cu_dev"][b]


def _places(s, first):
    """Page and row of every new row, and whether its sequence takes part (the others: those of a page that no sequence has)."""
    b, i = _sequence_of(s)
    at = first[b].long() + i
    rows = s["case"]["page_rows"]
    live = first[b] >= 0
    page = torch.where(live, s["table"].long()[b, at.clamp(min=0) // rows % s["room"]], s["spare"])
    return page, at.clamp(min=0) % rows, live


def _rotated(x, positions, inv_freq, interleaved):
    angle = positions.double()[:, None] * inv_freq
    c, sn = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = x.float()
    lo, hi = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :D // 2], x[..., D // 2:])
    a, b = lo * c - hi * sn, hi * c + lo * sn
    return torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)


def _stored(s, name, place, x):
    """Rows x [rows, H_kv, 128] (fp32) to their places; rows of sequences that take no part stay out."""
    page, row, live = place
    scale = s["case"][name + "_scale"]
    if s["case"]["format"] == "fp4":
        codes, scales = _quantise(x, scale)
        keep = live[:, None, None]
        s[name][page, :, row] = torch.where(keep, codes, s[name][page, :, row])
        s[name + "_scales"][page, :, row] = torch.where(keep, scales, s[name + "_scales"][page, :, row])
    else:
        s[name][page, :, row] = torch.where(live[:, None, None], x.to(s[name].dtype), s[name][page, :, row])


def _read_back(s, first):
    place = _places(s, first)
    for name in "kv":
        x = s[name][place[0], :, place[1]]
        if s["case"]["format"] == "fp4":
            x = _values(x, s[name + "_scales"][place[0], :, place[1]], s["case"][name + "_scale"])
        back = s[name + "_back"]
        back.copy_(torch.where(place[2][:, None, None], x, torch.zeros_like(x)).transpose(0, 1).to(back.dtype))


def _append(s):
    case, place = s["case"], _places(s, s["held"])
    _stored(s, "k", place, _rotated(s["k_new"], s["positions"], s["inv_freq"], case["interleaved"]))
    _stored(s, "v", place, s["v_new"].float())
    if case["queries"]:
        s["q_rot"].copy_(_rotated(s["q_new"], s["positions"], s["inv_freq"], case["interleaved"]))
    if "k_back" in s:
        _read_back(s, s["held"])


def _compact(s):
    b, _ = _sequence_of(s)
    row = s["idx"].long() + s["cu_rows_dev"][b]                          # [H_kv, KT]
    for name in "kv":
        x = torch.gather(s[name + "_dense"], 1, row[..., None].expand(-1, -1, D)).transpose(0, 1)
        _stored(s, name, _places(s, s["held"]), x.float())
    if "k_back" in s:
        _read_back(s, s["held"])


def _read(s):
    _read_back(s, torch.zeros_like(s["held"]))


def _dense(s, name):
    """A cache's values [B, H_kv, room * page_rows, 128] in fp32."""
    table = s["table"].long().clamp(min=0)
    x = s[name][table]
    if s["case"]["format"] == "fp4":
        x = _values(x, s[name + "_scales"][table], s["case"][name + "_scale"])
    return x.float().transpose(1, 2).flatten(2, 3)


def _attend(s):
    case, dev = s["case"], s["dev"]
    hq, hkv, n = case["q_heads"], case["kv_heads"], max(s["new"])
    held, i = s["held"].long(), torch.arange(n, device=dev)
    token = (s["cu_dev"][:-1, None] + i).clamp(max=s["cu"][-1] - 1)                                          # [B, n]
    sees = torch.where((held >= 0)[:, None], held[:, None] + i + 1, 0)                              # rows that a query sees
    q = s["q"].float()[token].unflatten(2, (hkv, hq // hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)   # [B, H_kv, G n, 128]
    k, v = _dense(s, "k"), _dense(s, "v")
    score = q @ k.transpose(-1, -2) * (1.0 / math.sqrt(D))
    if case["softcap"]:
        score = torch.tanh(score / case["softcap"]) * case["softcap"]
    hidden = torch.arange(k.shape[2], device=dev) >= sees[..., None]                                # [B, n, rows]
    score = score.unflatten(2, (hq // hkv, n)).masked_fill(hidden[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = (p.flatten(2, 3) @ v).unflatten(2, (hq // hkv, n)) / total.clamp(min=torch.finfo(torch.float32).tiny)
    lse = (torch.log(total) + top).squeeze(-1)
    lse = torch.where((sees > 0)[:, None, None], lse, -math.inf)
    b, i = _sequence_of(s)
    s["out"].copy_(out.permute(0, 3, 1, 2, 4).flatten(2, 3)[b, i])
    s["lse"].copy_(lse.permute(0, 3, 1, 2).flatten(2, 3)[b, i])


PLAIN = {"append": _append, "compact": _compact, "read": _read, "attend": _attend}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------
def _nearest(x, kappa):
    """What 4 bits hold of x (float64 [.., 128]): the nearest multiple of the nearest scale, ties to the even code."""
    g = x.reshape(*x.shape[:-1], 8, 16)
    s = (g.abs().amax(-1) / (6.0 * kappa)).clamp(max=448.0)
    bits = torch.floor(torch.log2(s.clamp(min=2.0 ** -60))).clamp(min=-6.0)          # e4m3: 3 bits of fraction, exponents from -6
    unit = torch.exp2(bits - 3.0)
    s = torch.round(s / unit) * unit
    size = s[..., None] * kappa
    y = torch.where(size > 0, g.abs() / size, 0.0).clamp(max=6.0)
    unit = torch.where(y < 2.0, 0.5, torch.where(y < 4.0, 1.0, 2.0))                 # e2m1: steps of a half, one and two
    y = torch.round(y / unit) * unit
    return (y * size * torch.sign(g)).reshape(x.shape)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    f64, dev = torch.float64, s["dev"]
    lens, new = _lengths(case)
    rows, hq, hkv = case["page_rows"], case["q_heads"], case["kv_heads"]
    held = s["held"].tolist()
    fp4 = case["format"] == "fp4"

    def sequence(name, b, lo, hi):
        """Rows lo .. hi of sequence b, [H_kv, hi - lo, 128]."""
        at = torch.arange(lo, hi, device=dev)
        page, row = s["table"][b].long()[at // rows], at % rows
        x = s[name][page, :, row]
        if fp4:
            lv = torch.tensor(LEVELS, dtype=f64, device=dev)
            nib = torch.stack((x & 15, x >> 4), -1).flatten(-2).long()
            x = torch.where(nib >= 8, -lv[nib % 8], lv[nib % 8])
            sc = s[name + "_scales"][page, :, row].view(torch.float8_e4m3fn).to(f64).repeat_interleave(16, -1)
            x = x * sc * case[name + "_scale"]
        return x.to(f64).transpose(0, 1)

    if case["op"] == "attend":
        out, lse = torch.zeros((s["cu"][-1], hq, D), dtype=f64, device=dev), torch.full((s["cu"][-1], hq), -math.inf, dtype=f64, device=dev)
        for b, n in enumerate(new):
            if held[b] < 0 or n == 0:
                continue
            k, v = sequence("k", b, 0, held[b] + n), sequence("v", b, 0, held[b] + n)
            sees = torch.arange(held[b] + n, device=dev) <= held[b] + torch.arange(n, device=dev)[:, None]
            for h in range(hq):
                kv = h // (hq // hkv)
                z = s["q"][s["cu"][b]:s["cu"][b + 1], h].to(f64) @ k[kv].T / math.sqrt(D)
                if case["softcap"]:
                    z = case["softcap"] * torch.tanh(z / case["softcap"])
                z = torch.where(sees, z, -math.inf)
                lse[s["cu"][b]:s["cu"][b + 1], h] = torch.logsumexp(z, -1)
                out[s["cu"][b]:s["cu"][b + 1], h] = torch.softmax(z, -1) @ v[kv]
        return {"out": out, "lse": lse}
    t = s["cu"][-1]
    fresh = {}
    if case["op"] == "append":
        z = s["positions"].to(f64)[:, None, None] * 5.0e5 ** (-2.0 * torch.arange(D // 2, dtype=f64, device=dev) / D)
        turn = torch.polar(torch.ones_like(z), z)

        def rotate(x):
            x = x.to(f64)
            pair = x.reshape(*x.shape[:-1], D // 2, 2) if case["interleaved"] else x.reshape(*x.shape[:-1], 2, D // 2).transpose(-1, -2)
            y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
            return (y if case["interleaved"] else y.transpose(-1, -2)).reshape(x.shape)

        fresh = {"k": rotate(s["k_new"]), "v": s["v_new"].to(f64)}
    elif case["op"] == "compact":
        for name in "kv":
            parts = []
            for b in range(len(new)):
                pick = s["idx"][:, s["cu"][b]:s["cu"][b + 1]].long() + s["cu_rows"][b]
                parts.append(torch.stack([s[name + "_dense"][h, pick[h]] for h in range(hkv)], 1))
            fresh[name] = torch.cat(parts).to(f64)
    got = {}
    for name in "kv":
        kappa = float(torch.tensor(case[name + "_scale"]))
        if "k_back" in s:
            parts = []
            for b in range(len(new)):
                if case["op"] == "read":
                    parts.append(sequence(name, b, 0, new[b]))
                else:
                    x = fresh[name][s["cu"][b]:s["cu"][b + 1]].transpose(0, 1)
                    x = _nearest(x, kappa) if fp4 else x
                    parts.append(x if held[b] >= 0 else torch.zeros_like(x))
            got[name] = torch.cat(parts, 1)
        else:
            pool = s[name].to(f64)
            for b in range(len(new)):
                if held[b] >= 0 and new[b]:
                    at = torch.arange(held[b], held[b] + new[b], device=dev)
                    pool[s["table"][b].long()[at // rows], :, at % rows] = fresh[name][s["cu"][b]:s["cu"][b + 1]]
            got[name] = pool
    if case["op"] == "append" and case["queries"]:
        got["q"] = rotate(s["q_new"])
    return got
