"""The paged cache: appending, compacting into pages, reading back and attending, against plain 64-bit statements of include/dapq.h.

Tolerances count roundings.  A rounding to type t is off by at most finfo(t).eps / 2 relative to the value (bf16 2^-8, fp16 2^-11,
fp32 2^-24).
  * rotation: cos, sin, two products and a sum in fp32 are five roundings of terms of at most |lo| + |hi|: 5 * 2^-24 (|lo| + |hi|), then
    the rounding to the stored type.
  * 4 bits, unrotated bf16 values, kappa a power of two: every quotient is either exact or far from a tie: equal to the 64-bit formula.
    Otherwise: within half the distance of the neighbouring codes, which is at most step / 4, / 2, 1 below 2, 4 and above,
    of a step that is the group's largest magnitude / 6 kappa to nearest in e4m3 (2^-4 relative: the top of a group may lie
    6.4 steps up, 0.4 from its code).
  * attention: a logit (128 products summed in fp32, whatever the order) is off by at most dz = 140 * 2^-24 * scale * sum |q k|, the
    exponential and its argument's rounding by 2^-22 + |z - max| 2^-23 relative, a weight's rounding by 2^-11 (4 bits: fp16), 2^-8
    (bf16) or not at all (fp32), sums of fp32 by 2^-18 relative: out is off by rel * sum_j w_j |v_j| with rel twice the sum of
    these (numerator and normaliser), plus the rounding of the output."""
import ctypes as C
import math

import pytest
import torch

D = 128
F64 = torch.float64
LEVELS = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=F64)


@pytest.fixture(scope="module")
def dq():
    import paper_2603_11564_b200 as lib
    lib.load_library()
    return lib


def half(dtype):
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------------------------------- plain statements (64 bits)
def nearest_fp4(x, kappa):
    """(values, steps) of x [.., 128] in 4 bits, float64, ties to even codes."""
    g = x.unflatten(-1, (8, 16))
    s = (g.abs().amax(-1) / (6 * kappa)).clamp(max=448.0)
    unit = torch.exp2(torch.floor(torch.log2(s.clamp(min=2.0 ** -30))).clamp(min=-6) - 3)
    s = torch.round(s / unit) * unit
    step = (s * kappa).unsqueeze(-1)
    y = torch.where(step > 0, g.abs() / step, 0.0)
    lv = LEVELS.to(x.device)
    mid = (lv[1:] + lv[:-1]) / 2
    code = torch.zeros_like(y, dtype=torch.long)
    for i, m in enumerate(mid):                       # a tie goes to the even one of codes i and i + 1
        code += (y > m) | ((y == m) & (i % 2 == 1))
    return (lv[code] * step * torch.sign(g)).flatten(-2), step.expand_as(g).flatten(-2)


def decode(codes, scales, kappa):
    both = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    x = LEVELS.to(codes.device)[both % 8] * torch.where(both >= 8, -1.0, 1.0)
    return x * scales.view(torch.float8_e4m3fn).to(F64).repeat_interleave(16, -1) * kappa


def rotated(x, pos, interleaved, base):
    x = x.to(F64)
    a = pos.to(F64)[:, None, None] * base ** (-2.0 * torch.arange(D // 2, dtype=F64, device=x.device) / D)
    lo, hi = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :64], x[..., 64:])
    y0, y1 = lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()
    size = lo.abs() + hi.abs()
    if interleaved:
        return torch.stack((y0, y1), -1).flatten(-2), torch.stack((size, size), -1).flatten(-2)
    return torch.cat((y0, y1), -1), torch.cat((size, size), -1)


class Cache:
    """Pools with pages in random order, poisoned where nothing was written; `layout` chooses the strides."""

    def __init__(self, dq, dtype, fmt, hkv, page_rows, lens, room, seed=0, layout="plain", k_scale=1.0, v_scale=1.0, extra=3, wide=0):
        g = torch.Generator().manual_seed(seed)
        self.dq, self.dtype, self.fmt, self.rows, self.lens, self.hkv = dq, dtype, fmt, page_rows, list(lens), hkv
        self.k_scale, self.v_scale = k_scale, v_scale
        need = [-(-max(0, r) // page_rows) for r in room]
        n = sum(need) + extra
        order = torch.randperm(n, generator=g).int()
        stride = max(max(need) + 1, 2, wide)                  # (wide: room for long sequences, as which kernel takes a call goes by the room)
        table = torch.full((len(lens), stride), n + 7, dtype=torch.int32)
        table[::2] = -3
        at = 0
        for b, m in enumerate(need):
            table[b, :m] = order[at:at + m]
            at += m
        self.n, self.table = n, table.cuda()
        width, el = (64, torch.uint8) if fmt == "fp4" else (D, dtype)
        poison = 0xFF if fmt == "fp4" else math.nan

        def pool(w, t):
            if layout == "interleaved":                       # K and V of a page side by side, rows outside heads
                x = torch.full((n, 2, page_rows, hkv, w), poison, dtype=t, device="cuda").transpose(2, 3)
                return x[:, 0], x[:, 1]
            if layout == "padded":
                a, b = (torch.full((n, hkv + 1, page_rows, 2 * w), poison, dtype=t, device="cuda")[:, :hkv, :, :w] for _ in "kv")
                return a, b
            return tuple(torch.full((n, hkv, page_rows, w), poison, dtype=t, device="cuda") for _ in "kv")

        self.k, self.v = pool(width, el)
        self.ks, self.vs = pool(8, torch.uint8) if fmt == "fp4" else (None, None)
        self.len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.view = dq.dapq_paged_cache(self.k, self.v, self.table, self.len, self.ks, self.vs, k_scale, v_scale)

    def where(self, b, lo, hi):
        at = torch.arange(lo, hi, device="cuda")
        return self.table[b].long()[at // self.rows], at % self.rows

    def fill(self, b, k, v):
        """Rows 0 .. of sequence b: [H_kv, n, 128] values, stored by the plain statement."""
        page, row = self.where(b, 0, k.shape[1])
        for name, x, kap in (("k", k, self.k_scale), ("v", v, self.v_scale)):
            p, sc = (self.k, self.ks) if name == "k" else (self.v, self.vs)
            if self.fmt == "fp4":
                val, step = nearest_fp4(x.to(F64), kap)
                s = (step.unflatten(-1, (8, 16))[..., 0] / kap).to(torch.float32).to(torch.float8_e4m3fn)
                y = torch.where(step > 0, val.abs() / step, 0.0)
                code = torch.searchsorted(LEVELS.cuda(), y.contiguous()) + 8 * (val < 0)
                p[page, :, row] = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8).transpose(0, 1)
                sc[page, :, row] = s.view(torch.uint8).transpose(0, 1)
            else:
                p[page, :, row] = x.to(self.dtype).transpose(0, 1)

    def values(self, b, lo, hi):
        """K and V rows lo .. hi of sequence b as float64 [H_kv, n, 128]."""
        page, row = self.where(b, lo, hi)
        out = []
        for p, sc, kap in ((self.k, self.ks, self.k_scale), (self.v, self.vs, self.v_scale)):
            x = p[page, :, row]
            x = decode(x, sc[page, :, row], kap) if self.fmt == "fp4" else x.to(F64)
            out.append(x.transpose(0, 1))
        return out

    def bits(self):
        return [x.contiguous().view(torch.uint8).clone() for x in (self.k, self.v, self.ks, self.vs) if x is not None]


def context(dq, hq, hkv, dtype, max_batch=8, **kw):
    return dq.dapq_create(hq, hkv, 32, max_batch, 4096, dq.DAPQ_BF16 if dtype == torch.bfloat16 else dq.DAPQ_F32, 5.0e5, **kw)


def attend_reference(cache, q, cu, scale, softcap=0.0):
    """(out, lse, their tolerances) of every new query, float64."""
    T, hq, _ = q.shape
    G = hq // cache.hkv
    out, lse = torch.zeros(T, hq, D, dtype=F64, device="cuda"), torch.full((T, hq), -math.inf, dtype=F64, device="cuda")
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    weight = 0.0 if cache.dtype == torch.float32 else 2.0 ** (-11 if cache.fmt == "fp4" else -8)
    for b, held in enumerate(cache.lens):
        n = cu[b + 1] - cu[b]
        if held < 0 or n == 0:
            continue
        k, v = cache.values(b, 0, held + n)
        k, v = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
        x = q[cu[b]:cu[b + 1]].to(F64).transpose(0, 1)
        sees = torch.arange(held + n, device="cuda") <= held + torch.arange(n, device="cuda")[:, None]
        z = x @ k.transpose(1, 2) * scale
        dz = 140 * 2.0 ** -24 * scale * (x.abs() @ k.abs().transpose(1, 2))
        if softcap:
            z = softcap * torch.tanh(z / softcap)
            # bf16: tanh through an exponential and a quotient (base 2: a quarter of 2^y's 2^-22 twice, the quotient's 2^-22 twice, a sum's 2^-24);
            # fp32: its own 2^-22, products and the argument's factor 3 times 2^-24
            dz = dz + (z.abs() * 2.0 ** -21 if cache.dtype == torch.float32 else softcap * 2.0 ** -21)
        z = torch.where(sees, z, -math.inf)
        top = z.amax(-1, keepdim=True)
        w = torch.softmax(z, -1)
        rel = torch.where(sees, dz + (top - z) * 2.0 ** -23, 0.0).amax(-1, keepdim=True) + top.abs() * 2.0 ** -23 + 2.0 ** -21
        out[cu[b]:cu[b + 1]] = (w @ v).transpose(0, 1)
        lse[cu[b]:cu[b + 1]] = torch.logsumexp(z, -1).T
        tol[cu[b]:cu[b + 1]] = ((2 * rel + weight + 2.0 ** -18) * (w @ v.abs())).transpose(0, 1)
        ltol[cu[b]:cu[b + 1]] = rel.squeeze(-1).T + 2.0 ** -18
    tol += half(cache.dtype) * out.abs()
    ltol += 2.0 ** -22 * lse.abs().nan_to_num(posinf=0.0)
    return out, lse, tol, ltol


def check_attend(dq, ctx, cache, q, cu, softcap=0.0, stream=None):
    out, lse = torch.full_like(q, math.nan).contiguous(), torch.full(q.shape[:2], math.nan, device="cuda")
    dq.dapq_paged_attend(ctx, cache.view, cu, q, out, lse, softcap=softcap, stream=stream)
    dq.dapq_poll_status(ctx, stream)
    ref, rlse, tol, ltol = attend_reference(cache, q, cu, 1 / math.sqrt(D), softcap)
    bad = ~((out.to(F64) - ref).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), float(((out.to(F64) - ref).abs() / tol.clamp(min=1e-300)).max()))
    gone = torch.isinf(rlse)
    assert torch.equal(gone, torch.isinf(lse)) and not (lse[gone] > 0).any()
    assert ((lse.to(F64) - rlse)[~gone].abs() <= ltol[~gone]).all()
    return out, lse


# ----------------------------------------------------------------------------------------------------------- on the CPU
def test_struct_layouts(dq):
    assert C.sizeof(dq.dapq_paged_cache) == 104 and dq.dapq_paged_cache.page_table.offset == 56 and dq.dapq_paged_cache.k_scale.offset == 88
    assert C.sizeof(dq.dapq_new_tokens) == 64 and dq.dapq_new_tokens.positions.offset == 56


def test_null_context_is_an_error(dq):
    lib = dq.load_library()
    for fn, n in ((lib.dapq_paged_append, 5), (lib.dapq_paged_compact, 6), (lib.dapq_paged_read, 9)):
        args = [None] * n
        if fn is lib.dapq_paged_read:
            args[7] = 0
        assert fn(*args) == dq.DAPQ_ERR_INVALID_ARG
    assert lib.dapq_paged_attend(None, None, None, None, 0, 0.0, None, None, None) == dq.DAPQ_ERR_INVALID_ARG


def test_the_view_takes_only_what_the_library_reads(dq):
    pool = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t)
    table, held = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    v = dq.dapq_paged_cache(pool(5, 2, 16, 128), pool(5, 2, 16, 128), table, held)
    assert (v.page_stride, v.head_stride, v.row_stride, v.n_pages, v.page_rows, v.batch, v.table_stride, v.format) == (4096, 2048, 128, 5, 16, 2, 3, 0)
    u8 = lambda w: pool(5, 2, 16, w, t=torch.uint8)
    v = dq.dapq_paged_cache(u8(64), u8(64), table, held, u8(8), u8(8), 2.0, 0.5)
    assert (v.page_stride, v.head_stride, v.row_stride, v.format, v.k_scale, v.v_scale) == (4096, 2048, 128, 1, 2.0, 0.5)
    for bad in (lambda: dq.dapq_paged_cache(pool(5, 2, 16, 64), pool(5, 2, 16, 64), table, held),              # head_dim
                lambda: dq.dapq_paged_cache(pool(5, 2, 16, 128), pool(5, 2, 32, 128), table, held),            # K and V differ
                lambda: dq.dapq_paged_cache(u8(64), u8(64), table, held, u8(8), u8(16)[..., ::2]),             # strides of the scales
                lambda: dq.dapq_paged_cache(pool(5, 2, 16, 128), pool(5, 2, 16, 128), table.long(), held),     # type of the table
                lambda: dq.dapq_paged_cache(pool(5, 2, 16, 128), pool(5, 2, 16, 128), table[:, ::2], held),    # its strides
                lambda: dq.dapq_paged_cache(pool(5, 2, 16, 128), pool(5, 2, 16, 128), table, held[:1])):       # its batch
        with pytest.raises(AssertionError):
            bad()


def test_the_plain_4_bit_statement():
    """Hand-worked groups: a top of 6 gives scale 1 and every code itself; ties go to even codes."""
    x = torch.zeros(1, 128, dtype=F64)
    x[0, :8] = torch.tensor([6, 0.25, 0.75, -1.25, 1.75, 2.5, 3.5, -5.0], dtype=F64)
    val, step = nearest_fp4(x, 1.0)
    assert val[0, :8].tolist() == [6, 0, 1, -1, 2, 2, 4, -4] and step[0, 0] == 1 and not val[0, 8:].any()
    x[0, 16] = 2000.0 * 6                                     # beyond the largest scale: the largest code
    assert nearest_fp4(x, 1.0)[0][0, 16] == 448 * 6 and nearest_fp4(x, 8.0)[0][0, 16] == 12288                 # (2000 / 8 = 250: e4m3 has 256)


# ------------------------------------------------------------------------------------------------------------ on the GPU
gpu = pytest.mark.gpu
TYPES = [(torch.bfloat16, "native"), (torch.bfloat16, "fp4"), (torch.float32, "native"), (torch.float32, "fp4")]


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
@pytest.mark.parametrize("interleaved,layout,rows,kappas", [(False, "plain", 16, (1.0, 1.0)), (True, "interleaved", 32, (0.5, 4.0)), (False, "padded", 128, (0.37, 1.7))])
def test_append(dq, dtype, fmt, interleaved, layout, rows, kappas):
    hq, hkv = 12, 3
    lens, new = [0, 130, -1, 15, 63, 7], [5, 1, 4, 0, 67, 9]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    T = cu[-1]
    g = torch.Generator().manual_seed(3)
    ctx = context(dq, hq, hkv, dtype, flags=dq.DAPQ_FLAG_ROPE_INTERLEAVED if interleaved else 0)
    cache = Cache(dq, dtype, fmt, hkv, rows, lens, [max(0, a) + n for a, n in zip(lens, new)], layout=layout, k_scale=kappas[0], v_scale=kappas[1])
    qkv = torch.randn(T, hq + 2 * hkv, D, generator=g).to(dtype).cuda()
    qkv[3, hq + 1, 16:32] = 0.0                                # a group of zeros
    pos = torch.randint(0, 131072, (T,), generator=g).int().cuda()
    q_rot = torch.full((T, hq, D), math.nan, dtype=dtype, device="cuda")
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    before = cache.bits()
    dq.dapq_paged_append(ctx, cache.view, cu, k, v, pos, q, q_rot)
    dq.dapq_poll_status(ctx)
    want, size = rotated(q, pos, interleaved, 5.0e5)
    assert ((q_rot.to(F64) - want).abs() <= half(dtype) * want.abs() + 5 * 2.0 ** -24 * size * (1 + half(dtype))).all()
    want, size = rotated(k, pos, interleaved, 5.0e5)
    touched = []
    for b, (a, n) in enumerate(zip(lens, new)):
        if a < 0 or n == 0:
            continue
        touched.append(cache.where(b, a, a + n))
        gk, gv = (x.transpose(0, 1) for x in cache.values(b, a, a + n))
        wk, wv, sz = want[cu[b]:cu[b + 1]], v[cu[b]:cu[b + 1]].to(F64), size[cu[b]:cu[b + 1]]
        if fmt == "native":
            assert ((gk - wk).abs() <= half(dtype) * wk.abs() + 5 * 2.0 ** -24 * sz * (1 + half(dtype))).all() and torch.equal(gv, wv)
            continue
        kap = torch.tensor(kappas, dtype=torch.float32).tolist()
        for got, x, kappa, noise in ((gk, wk, kap[0], 5 * 2.0 ** -24 * sz), (gv, wv, kap[1], 0.0)):
            # the kernel's step may be the other side of a border of e4m3 from this one, a factor 8/9 .. 9/8: codes up to 1.5 are
            # then below 1.6875 of this step and 2 above 1.77, codes up to 3 below 3.375 and 4 above 3.55; what a code stands
            # for reaches halfway to the next one up, so 2 belongs to the gap of 0.5 and 4 to that of 1
            step = nearest_fp4(x, kappa)[1]
            gap = torch.where(got.abs() < 1.75 * step, 0.25, torch.where(got.abs() < 3.5 * step, 0.5, 1.0)) * step * (1 + 2.0 ** -3)
            assert ((got - x).abs() <= gap * (1 + 2.0 ** -20) + noise).all()
        if dtype == torch.bfloat16 and kappas[1] == 2.0 ** round(math.log2(kappas[1])):
            assert torch.equal(gv, nearest_fp4(wv, kappas[1])[0])
    keep = torch.ones(cache.n, rows, dtype=torch.bool, device="cuda")
    for page, row in touched:
        keep[page, row] = False
    for x, y in zip(before, cache.bits()):                     # rows of other sequences, idle ones, tails: as they were
        assert torch.equal(x.transpose(1, 2)[keep], y.transpose(1, 2)[keep])
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_append_without_rotation_one_token_each(dq, dtype, fmt):
    ctx = context(dq, 8, 8, dtype)
    cache = Cache(dq, dtype, fmt, 8, 16, [15, 16, 0], [16, 17, 1])
    k, v = (torch.randn(3, 8, D, generator=torch.Generator().manual_seed(s)).to(dtype).cuda() for s in (1, 2))
    dq.dapq_paged_append(ctx, cache.view, None, k, v)
    dq.dapq_poll_status(ctx)
    for b, a in enumerate(cache.lens):
        for got, x in zip(cache.values(b, a, a + 1), (k[b], v[b])):
            x = x.to(F64)
            want = x if fmt == "native" else nearest_fp4(x, 1.0)[0]
            if fmt == "fp4" and dtype == torch.float32:        # fp32 values may lie within a rounding of a border
                assert (got[:, 0] == want).double().mean() > 0.99
            else:
                assert torch.equal(got[:, 0], want)
    dq.dapq_destroy(ctx)


@gpu
def test_4_bits_of_extreme_values(dq):
    """Groups with an infinity or NaN read back as NaN, values beyond the largest scale as the largest code, tiny ones as zero."""
    ctx = context(dq, 1, 1, torch.float32)
    cache = Cache(dq, torch.float32, "fp4", 1, 16, [0], [1])
    x = torch.ones(1, 1, D, device="cuda")
    x[0, 0, 3], x[0, 0, 20], x[0, 0, 37] = math.inf, math.nan, -3.0e38
    x[0, 0, 64:80], x[0, 0, 80:96], x[0, 0, 96:112] = 1e-30, 0.0, -0.0
    dq.dapq_paged_append(ctx, cache.view, None, x, -x)
    k, v = (y[0, 0] for y in cache.values(0, 0, 1))
    one = 6 * 11 / 64                                         # 1 / 6 lies between 10 / 64 and 11 / 64 in e4m3
    assert k[:32].isnan().all() and k[37] == -2688 and (k[32:37] == 0).all() and (k[48:64] == one).all() and (k[64:112] == 0).all() and (k[112:] == one).all()
    assert v[:32].isnan().all() and torch.equal(v[32:], -k[32:])
    out = torch.empty(1, 1, D, device="cuda")
    back = torch.empty_like(out)
    dq.dapq_paged_read(ctx, cache.view, None, [1], [0], out, back)
    assert torch.equal(out[0, 0].to(F64).nan_to_num(nan=9.0), k.nan_to_num(nan=9.0))
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
@pytest.mark.parametrize("hkv,rows", [(1, 16), (4, 64)])
def test_compact_into_pages(dq, dtype, fmt, hkv, rows):
    """Against dapq_compact_kv's own rows; the second sequence already holds 20, the third takes no part."""
    L, keep, held = [70, 300, 40, 1], [70, 99, 5, 1], [0, 20, -1, 0]
    ctx = context(dq, 2 * hkv, hkv, dtype)
    cu_rows, cu_keep = [0], [0]
    for a, b in zip(L, keep):
        cu_rows.append(cu_rows[-1] + a + 32)
        cu_keep.append(cu_keep[-1] + b)
    g = torch.Generator().manual_seed(5)
    big = torch.randn(2, hkv, cu_rows[-1], 256, generator=g).to(dtype).cuda()
    k, v = big[0, ..., :128], big[1, ..., 128:]
    idx = torch.cat([torch.rand(hkv, a, generator=g).topk(b, -1).indices.sort(-1).values for a, b in zip(L, keep)], -1).int().cuda()
    dense = [torch.empty(hkv, cu_keep[-1], D, dtype=dtype, device="cuda") for _ in "kv"]
    dq.dapq_compact_kv(ctx, k, v, cu_rows, L, idx, keep, *dense)
    cache = Cache(dq, dtype, fmt, hkv, rows, held, [h + b for h, b in zip([0, 20, 0, 0], keep)])
    before = cache.bits()
    dq.dapq_paged_compact(ctx, k, v, cu_rows, L, idx, keep, cache.view)
    dq.dapq_poll_status(ctx)
    touched = torch.ones(cache.n, rows, dtype=torch.bool, device="cuda")
    for b in (0, 1, 3):
        touched[cache.where(b, held[b], held[b] + keep[b])] = False
        for got, x in zip(cache.values(b, held[b], held[b] + keep[b]), dense):
            x = x[:, cu_keep[b]:cu_keep[b + 1]].to(F64)
            if fmt == "native" or dtype == torch.bfloat16:
                assert torch.equal(got, x if fmt == "native" else nearest_fp4(x, 1.0)[0])
            else:
                assert (got == nearest_fp4(x, 1.0)[0]).double().mean() > 0.9999
    for x, y in zip(before, cache.bits()):
        assert torch.equal(x.transpose(1, 2)[touched], y.transpose(1, 2)[touched])
    bad = idx.clone()
    bad[0, 3], bad[0, 80] = -1, 300
    dq.dapq_paged_compact(ctx, k, v, cu_rows, L, bad, keep, cache.view)
    with pytest.raises(dq.DapqError) as e:
        dq.dapq_poll_status(ctx)
    assert e.value.status == dq.DAPQ_ERR_INVALID_ARG and "indices" in str(e.value)
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
@pytest.mark.parametrize("layout", ["plain", "interleaved", "padded"])
def test_read(dq, dtype, fmt, layout):
    lens, first, n, at = [200, 33, 64, 5], [17, 0, -1, 2], [100, 33, 3, 0], [3, 110, 0, 0]
    ctx = context(dq, 4, 2, dtype)
    cache = Cache(dq, dtype, fmt, 2, 32, lens, lens, layout=layout, k_scale=0.5, v_scale=0.3)
    for b, m in enumerate(lens):
        cache.fill(b, *(torch.randn(2, m, D, device="cuda") for _ in "kv"))
    out = [torch.full((2, 150, D), 7.0, dtype=dtype, device="cuda") for _ in "kv"]
    dq.dapq_paged_read(ctx, cache.view, first, n, at, *out)
    dq.dapq_poll_status(ctx)
    left = torch.ones(150, dtype=torch.bool, device="cuda")
    for b in (0, 1):
        left[at[b]:at[b] + n[b]] = False
        for got, want in zip(out, cache.values(b, first[b], first[b] + n[b])):
            # a product by kappa in fp32 and the rounding to the type
            assert ((got[:, at[b]:at[b] + n[b]].to(F64) - want).abs() <= (half(dtype) + 2.0 ** -22) * want.abs()).all()
    assert all((x[:, left] == 7).all() for x in out)
    dq.dapq_destroy(ctx)


SHAPES = [
    # (H_q, H_kv, page_rows, rows held, new rows, softcap)
    (8, 2, 16, [0], [1], 0.0),
    (8, 1, 16, [1, 14, 15, 16, 17], [1] * 5, 0.0),
    (4, 4, 32, [126, 127, 128, 129, 255, 256], [1] * 6, 0.0),
    (28, 4, 64, [5000, 3, -1, 1111], [1] * 4, 30.0),
    (12, 1, 16, [700, 0, 31], [1] * 3, 0.0),
    (48, 2, 128, [900, 64], [1, 1], 5.0),
    (8, 8, 16, [200, 0, 17], [9, 5, 1], 0.0),
    (32, 8, 16, [64, -1, 0, 333], [3, 2, 0, 40], 50.0),
    (16, 2, 1024, [2500], [130], 0.0),
    (6, 2, 256, [0, 0], [257, 33], 0.0),
]


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_attend(dq, dtype, fmt, shape):
    hq, hkv, rows, lens, new, cap = shape
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    g = torch.Generator(device="cuda").manual_seed(7)
    ctx = context(dq, hq, hkv, dtype)
    layout = ["plain", "interleaved", "padded"][hq % 3]
    cache = Cache(dq, dtype, fmt, hkv, rows, lens, [a + n if a >= 0 else 0 for a, n in zip(lens, new)], layout=layout, k_scale=0.5, v_scale=0.3)
    for b, (a, n) in enumerate(zip(lens, new)):
        if a + n > 0 and a >= 0:
            cache.fill(b, *(torch.randn(hkv, a + n, D, device="cuda", generator=g) for _ in "kv"))
    q = (2.0 * torch.randn(cu[-1], hq + 2, D, device="cuda", generator=g)).to(dtype)[:, :hq]      # (tokens further apart than their heads)
    first = check_attend(dq, ctx, cache, q, cu, cap)
    again = check_attend(dq, ctx, cache, q, cu, cap)
    assert all(torch.equal(a, b) for a, b in zip(first, again))           # whoever arrives last
    dq.dapq_destroy(ctx)


WIDE = 131072                                                 # rows of room: the kernel for many query rows takes 48 and more


MANY = [
    (48, 2, 128, [900, 64], [2, 2], 5.0),
    (32, 8, 16, [64, -1, 0, 333], [30, 20, 0, 40], 50.0),
    (16, 2, 1024, [2500], [130], 0.0),
    (6, 2, 256, [0, 0], [257, 33], 0.0),
    (64, 8, 16, [5, 300], [64, 17], 0.0),
    (8, 1, 32, [127, 128, 129, 255], [16, 17, 15, 48], 0.0),
    (12, 4, 64, [3000], [100], 20.0),
    (8, 2, 16, [120, 20, 4000, 7], [33, 1, 3, 200], 0.0),     # sequences for either kernel in one call
    (8, 8, 64, [500, 90, 0, 1300, 40, 700, 260, 3], [600] * 8, 0.0),
    (16, 16, 32, [2000, 100, -1, 3000], [200, 100, 64, 130], 8.0),
]


@gpu
@pytest.mark.parametrize("fmt", ["native", "fp4"])
@pytest.mark.parametrize("shape", MANY, ids=[str(i) for i in range(len(MANY))])
def test_attend_with_many_query_rows(dq, fmt, shape):
    hq, hkv, rows, lens, new, cap = shape
    bf = torch.bfloat16
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    g = torch.Generator(device="cuda").manual_seed(13)
    ctx = context(dq, hq, hkv, bf)
    cache = Cache(dq, bf, fmt, hkv, rows, lens, [a + n if a >= 0 else 0 for a, n in zip(lens, new)], layout=["plain", "interleaved", "padded"][hkv % 3],
                  k_scale=0.5, v_scale=0.3, wide=WIDE // rows)
    for b, (a, n) in enumerate(zip(lens, new)):
        if a + n > 0 and a >= 0:
            cache.fill(b, *(torch.randn(hkv, a + n, D, device="cuda", generator=g) for _ in "kv"))
    q = (2.0 * torch.randn(cu[-1], hq + 2, D, device="cuda", generator=g)).to(bf)[:, :hq]
    first = check_attend(dq, ctx, cache, q, cu, cap)
    again = check_attend(dq, ctx, cache, q, cu, cap)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("fmt", ["native", "fp4"])
def test_many_query_rows_and_maxima_that_move(dq, fmt):
    """Keys along the queries, ever larger, then far below, over several tiles; a page in the middle that does not exist."""
    bf = torch.bfloat16
    ctx = context(dq, 4, 1, bf)
    held, n = 1500, 40
    cache = Cache(dq, bf, fmt, 1, 32, [held], [held + n], wide=WIDE // 32)
    d = torch.randn(D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    d = d / d.norm()
    z = torch.cat((torch.linspace(-60, 60, 1000, device="cuda"), torch.linspace(60, -200, held + n - 1000, device="cuda")))
    cache.fill(0, (z[:, None] * d + 0.01 * torch.randn(held + n, D, device="cuda"))[None], torch.randn(1, held + n, D, device="cuda"))
    f = torch.linspace(-1.5, 1.5, 4 * n, device="cuda").view(n, 4, 1)
    q = (f * d * math.sqrt(D)).to(bf)
    good, _ = check_attend(dq, ctx, cache, q, [0, n])
    page = int(cache.table[0, 5])
    cache.table[0, 5] = -2                                    # rows 160 .. 191
    out = torch.empty_like(q)
    dq.dapq_paged_attend(ctx, cache.view, [0, n], q, out)
    with pytest.raises(dq.DapqError) as e:
        dq.dapq_poll_status(ctx)
    assert e.value.status == dq.DAPQ_ERR_INVALID_ARG and out.isfinite().all()
    k, v = cache.values(0, 0, 160)[0][0], cache.values(0, 0, 160)[1][0]
    cache.table[0, 5] = page
    k2, v2 = (x[0] for x in cache.values(0, 192, held + n))
    k, v = torch.cat((k, k2)), torch.cat((v, v2))
    seen = torch.cat((torch.arange(160), torch.arange(192, held + n))).cuda()
    x = q.to(F64) @ k.T / math.sqrt(D)
    x = torch.where(seen <= held + torch.arange(n, device="cuda")[:, None, None], x, -math.inf)
    w = torch.softmax(x, -1)
    # logits reach 140: dz = 140 * 2^-24 * 140 and the exponent's rounding of as much again
    assert ((out.to(F64) - w @ v).abs() <= (2.0 ** -8 + half(bf) + 4 * 140 * 140 * 2.0 ** -24 + 2.0 ** -12) * (w @ v.abs()) + 1e-6).all()
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_attend_to_peaks_that_move_the_maximum(dq, dtype, fmt):
    """Keys along the query, ever larger, then far below: the running maximum moves at every tile; queries from 2^-20 to 2^10."""
    ctx = context(dq, 4, 1, dtype)
    n = 700
    cache = Cache(dq, dtype, fmt, 1, 16, [n - 1], [n])
    d = torch.randn(D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    d = d / d.norm()
    z = torch.cat((torch.linspace(-60, 60, 350, device="cuda"), torch.linspace(60, -200, 350, device="cuda")))
    k = z[:, None] * d + 0.01 * torch.randn(n, D, device="cuda")
    cache.fill(0, k[None], torch.randn(1, n, D, device="cuda"))
    q = torch.stack([d * math.sqrt(D) * f for f in (1.0, -1.0, 2.0 ** -20, 0.0)])[None].to(dtype)
    check_attend(dq, ctx, cache, q, [0, 1])
    if dtype == torch.bfloat16:
        check_attend(dq, ctx, cache, q * 2.0 ** 10, [0, 1], softcap=20.0)
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_attend_reports_bad_pages_and_goes_on(dq, dtype, fmt):
    ctx = context(dq, 8, 2, dtype)
    lens = [100, 50]
    cache = Cache(dq, dtype, fmt, 2, 16, lens, [101, 51])
    for b, a in enumerate(lens):
        cache.fill(b, *(torch.randn(2, a + 1, D, device="cuda") for _ in "kv"))
    q = torch.randn(2, 8, D, device="cuda").to(dtype)
    good, _ = check_attend(dq, ctx, cache, q, None if False else [0, 1, 2])
    sound = cache.table.clone()
    for page in (-1, cache.n, 1 << 30):
        cache.table[0, 2] = page
        out, lse = torch.empty_like(q), torch.empty(2, 8, device="cuda")
        dq.dapq_paged_attend(ctx, cache.view, None, q, out, lse)
        with pytest.raises(dq.DapqError) as e:
            dq.dapq_poll_status(ctx)
        assert e.value.status == dq.DAPQ_ERR_INVALID_ARG and torch.equal(out[1], good[1]) and out.isfinite().all()
        back = [torch.full((2, 101, D), 5.0, dtype=dtype, device="cuda") for _ in "kv"]
        dq.dapq_paged_read(ctx, cache.view, None, [101, 0], [0, 0], *back)
        with pytest.raises(dq.DapqError):
            dq.dapq_poll_status(ctx)
        assert all((x[:, 32:48] == 0).all() and x.isfinite().all() for x in back)
        cache.table.copy_(sound)
    before = cache.bits()
    cache.len.copy_(torch.tensor([cache.view.table_stride * 16, 51]))       # no room for one more row
    kv = [torch.randn(2, 2, D, device="cuda").to(dtype) for _ in "kv"]
    dq.dapq_paged_append(ctx, cache.view, [0, 1, 1], *(x[:1] for x in kv))
    with pytest.raises(dq.DapqError):
        dq.dapq_poll_status(ctx)
    assert all(torch.equal(x, y) for x, y in zip(before, cache.bits()))
    out = torch.empty(1, 8, D, dtype=dtype, device="cuda")
    cache.len[0] = (1 << 31) - 1
    dq.dapq_paged_attend(ctx, cache.view, [0, 1, 1], q[:1], out)
    with pytest.raises(dq.DapqError):
        dq.dapq_poll_status(ctx)
    dq.dapq_poll_status(ctx)
    dq.dapq_destroy(ctx)


UNITS = (8, 8, 64, [500, 90, 0, 1300, 40, 700, 260, 3], [600] * 8)     # more units than a third of the CTAs: joined where they are computed


@gpu
@pytest.mark.parametrize("fmt", ["native", "fp4"])
@pytest.mark.parametrize("shape", [(8, 2, 16, [3000, 70], [100, 100]), (4, 2, 16, [2500], [30]), UNITS], ids=["parts", "both tiles", "units"])
def test_giving_up_in_the_kernel_for_many_rows(dq, fmt, shape):
    """A limit of a cycle on its waits: a status, no hang, and the next call is right (its arrival counters are back at 0)."""
    hq, hkv, rows, lens, new = shape
    bf = torch.bfloat16
    ctx = context(dq, hq, hkv, bf)
    cache = Cache(dq, bf, fmt, hkv, rows, lens, [a + n for a, n in zip(lens, new)], wide=WIDE // rows)
    cu = [0]
    for b, (a, n) in enumerate(zip(lens, new)):
        cache.fill(b, *(torch.randn(hkv, a + n, D, device="cuda") for _ in "kv"))
        cu.append(cu[-1] + n)
    q = torch.randn(cu[-1], hq, D, device="cuda").to(bf)
    out = torch.empty_like(q)
    times = 0
    for _ in range(10):
        dq.dapq_set_wait_limit(ctx, 1)
        dq.dapq_paged_attend(ctx, cache.view, cu, q, out)
        try:
            dq.dapq_poll_status(ctx)
            gave_up = False
        except dq.DapqError as e:
            assert e.status == dq.DAPQ_ERR_TIMEOUT
            gave_up = True
        dq.dapq_set_wait_limit(ctx, 0)
        right, _ = check_attend(dq, ctx, cache, q, cu)
        # (a barrier is tried once before the clock is looked at, and the hardware may hold that try for as long as a short run's waits take: then
        # nothing runs out, and the result has to be right)
        assert gave_up or torch.equal(out, right)
        times += gave_up
        if times == 2:
            break
    assert times > 0 or len(cu) == 2
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("fmt", ["native", "fp4"])
@pytest.mark.parametrize("shape", [(8, 2, 16, [3000, 70], [100, 1]), UNITS], ids=["parts", "units"])
def test_many_query_rows_in_a_graph(dq, fmt, shape):
    """Replayed twice, behind another capture that uses the same workspace."""
    hq, hkv, rows, lens, new = shape
    bf = torch.bfloat16
    ctx = context(dq, hq, hkv, bf)
    cache = Cache(dq, bf, fmt, hkv, rows, lens, [a + n for a, n in zip(lens, new)], wide=WIDE // rows)
    cu = [0]
    for b, (a, n) in enumerate(zip(lens, new)):
        cache.fill(b, *(torch.randn(hkv, a + n, D, device="cuda") for _ in "kv"))
        cu.append(cu[-1] + n)
    q = [torch.randn(cu[-1], hq, D, device="cuda").to(bf) for _ in range(2)]
    want = [check_attend(dq, ctx, cache, x, cu, 30.0)[0] for x in q]
    outs, graphs, stream = [torch.empty_like(x) for x in q], [torch.cuda.CUDAGraph() for _ in q], torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for x, out, graph in zip(q, outs, graphs):
            with torch.cuda.graph(graph, stream=stream):
                dq.dapq_paged_attend(ctx, cache.view, cu, x, out, softcap=30.0)
        for _ in range(2):
            for out, graph in zip(outs, graphs):
                out.zero_()
                graph.replay()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    dq.dapq_poll_status(ctx, stream)
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_attend_with_more_sequences_than_ctas_and_more_ctas_than_tiles(dq, dtype, fmt):
    """128 sequences of all lengths, a third of them idle or without new tokens, some with many query rows."""
    g = torch.Generator().manual_seed(9)
    lens = [int(x) for x in torch.randint(0, 400, (128,), generator=g)]
    new = [int(x) for x in torch.randint(0, 4, (128,), generator=g)]
    lens[7], lens[50], lens[127], lens[3] = 9000, -1, -1, -1
    new[9], new[50], new[3] = 70, 40, 1
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    ctx = context(dq, 8, 2, dtype, max_batch=128)
    cache = Cache(dq, dtype, fmt, 2, 16, lens, [a + n if a >= 0 else 0 for a, n in zip(lens, new)], wide=WIDE // 16)
    for b, (a, n) in enumerate(zip(lens, new)):
        if a + n > 0 and a >= 0:
            cache.fill(b, *(torch.randn(2, a + n, D, device="cuda") for _ in "kv"))
    check_attend(dq, ctx, cache, torch.randn(cu[-1], 8, D, device="cuda").to(dtype), cu)
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("fmt", ["native", "fp4"])
@pytest.mark.parametrize("n", [1, 30])
def test_infinities_and_nan_behind_the_cache_and_in_it(dq, fmt, n):
    """In rows that nobody sees they do not matter; a NaN key that is seen makes its queries NaN, those of other heads and sequences not."""
    bf = torch.bfloat16
    ctx = context(dq, 4, 2, bf)
    cache = Cache(dq, bf, fmt, 2, 16, [40, 40], [40 + n, 40 + n], wide=WIDE // 16)
    for b in range(2):
        cache.fill(b, *(torch.randn(2, 40 + n, D, device="cuda") for _ in "kv"))
    q = torch.randn(2 * n, 4, D, device="cuda").to(bf)
    good, lse = check_attend(dq, ctx, cache, q, [0, n, 2 * n])
    page, row = cache.where(1, 5, 6)
    (cache.ks if fmt == "fp4" else cache.k)[page, 1, row] = 0x7F if fmt == "fp4" else math.nan
    out = torch.empty_like(q)
    dq.dapq_paged_attend(ctx, cache.view, [0, n, 2 * n], q, out)
    dq.dapq_poll_status(ctx)
    assert torch.equal(out[:n], good[:n]) and torch.equal(out[n:, :2], good[n:, :2]) and out[n:, 2:].isnan().all()
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_attend_to_the_largest_and_smallest_queries(dq, dtype, fmt):
    """Queries near the ends of their type's range: logits of 0 stay 0, others saturate the softmax on the largest key."""
    ctx = context(dq, 4, 1, dtype)
    cache = Cache(dq, dtype, fmt, 1, 16, [49], [50])
    k = torch.zeros(1, 50, D, device="cuda")
    k[0, :, 0] = torch.arange(50, device="cuda") % 7 - 3.0
    v = torch.randn(1, 50, D, device="cuda")
    cache.fill(0, k, v)
    v = cache.values(0, 0, 50)[1][0]
    q = torch.zeros(1, 4, D, device="cuda")
    q[0, 0, 1] = 3e38                                          # no key has this channel: all logits 0
    q[0, 1, 0] = 1e30
    q[0, 2, 0] = -1e-38
    out, lse = torch.empty(1, 4, D, dtype=dtype, device="cuda"), torch.empty(1, 4, device="cuda")
    dq.dapq_paged_attend(ctx, cache.view, None, q.to(dtype), out, lse)
    dq.dapq_poll_status(ctx)
    mean, best = v.mean(0), v[k[0, :, 0] == 3].mean(0)
    # equal weights: sums of 50 products, roundings of the weights and of the output
    tol = (half(dtype) + 2.0 ** -8 + 2.0 ** -18) * v.abs().mean(0) + 2.0 ** -20
    for h in (0, 2, 3):
        assert ((out[0, h].to(F64) - mean).abs() <= tol).all() and abs(lse[0, h].item() - math.log(50)) < 1e-5
    assert ((out[0, 1].to(F64) - best).abs() <= (half(dtype) + 2.0 ** -8 + 2.0 ** -18) * v.abs().amax(0) + 2.0 ** -20).all()
    dq.dapq_destroy(ctx)


@gpu
def test_two_contexts_on_two_streams(dq):
    """Each context orders its own calls only: two of them side by side, many times."""
    bf = torch.bfloat16
    pairs = []
    for seed in (1, 2):
        ctx = context(dq, 8, 2, bf)
        cache = Cache(dq, bf, "fp4", 2, 16, [2500, 300], [2501, 301], seed=seed)
        for b, a in enumerate((2501, 301)):
            cache.fill(b, *(torch.randn(2, a, D, device="cuda") for _ in "kv"))
        q = torch.randn(2, 8, D, device="cuda").to(bf)
        want, _ = check_attend(dq, ctx, cache, q, [0, 1, 2])
        pairs.append((ctx, cache, q, want, torch.cuda.Stream(), [torch.empty_like(q) for _ in range(40)]))
    torch.cuda.synchronize()
    for i in range(40):
        for ctx, cache, q, _, stream, outs in pairs:
            dq.dapq_paged_attend(ctx, cache.view, None, q, outs[i], stream=stream)
    torch.cuda.synchronize()
    for ctx, _, _, want, stream, outs in pairs:
        assert all(torch.equal(o, want) for o in outs)
        dq.dapq_poll_status(ctx, stream)
        dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
@pytest.mark.parametrize("wide", [0, WIDE // 64])
def test_more_new_rows_than_room_for_a_sequence_that_takes_no_part(dq, dtype, fmt, wide):
    """Its table has two pages: nothing of it is skipped, as nothing of it is there; one that takes part is flagged."""
    ctx = context(dq, 3, 3, dtype)
    cache = Cache(dq, dtype, fmt, 3, 64, [0, -1], [6, 0], wide=wide)
    cache.fill(0, *(torch.randn(3, 6, D, device="cuda") for _ in "kv"))
    n = cache.table.shape[1] * 64 + 100 if wide == 0 else 300
    q = torch.randn(6 + n, 3, D, device="cuda").to(dtype)
    check_attend(dq, ctx, cache, q, [0, 6, 6 + n])
    dq.dapq_paged_append(ctx, cache.view, [0, 0, n], *(torch.zeros(2, n, 3, D, dtype=dtype, device="cuda")))
    dq.dapq_poll_status(ctx)
    if wide == 0:
        held = torch.tensor([0, 0], dtype=torch.int32, device="cuda")
        cache.view.cache_len = held.data_ptr()
        dq.dapq_paged_attend(ctx, cache.view, [0, 6, 6 + n], q, torch.empty_like(q))
        with pytest.raises(dq.DapqError):
            dq.dapq_poll_status(ctx)
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
@pytest.mark.parametrize("cap", [1e-18, 0.3, 1000.0, 1024.0])
def test_smallest_and_largest_caps(dq, dtype, fmt, cap):
    ctx = context(dq, 8, 2, dtype)
    cache = Cache(dq, dtype, fmt, 2, 16, [90, 7], [91, 57], wide=WIDE // 16)
    for b, n in enumerate((91, 57)):
        cache.fill(b, *(torch.randn(2, n, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(b)) for _ in "kv"))
    q = torch.randn(51, 8, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(9)).to(dtype)
    check_attend(dq, ctx, cache, q, [0, 1, 51], cap)
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_logits_whose_factor_underflows(dq, dtype, fmt):
    """All of them 0 to fp32: every row seen weighs the same, those not seen nothing."""
    ctx = dq.dapq_create(8, 2, 32, 4, 4096, dq.DAPQ_BF16 if dtype == torch.bfloat16 else dq.DAPQ_F32, 5.0e5, softmax_scale=1e-30)
    cache = Cache(dq, dtype, fmt, 2, 16, [90, 7], [91, 57], wide=WIDE // 16, k_scale=2.0 ** -60)
    v = [torch.randn(2, n, D, device="cuda") for n in (91, 57)]
    for b in range(2):
        cache.fill(b, torch.randn(*v[b].shape, device="cuda") * 2.0 ** -60, v[b])
    q = (torch.randn(51, 8, D, device="cuda") * 2.0 ** -110).to(dtype)
    out = torch.full_like(q, math.nan)
    dq.dapq_paged_attend(ctx, cache.view, [0, 1, 51], q, out)
    dq.dapq_poll_status(ctx)
    for t, (b, n) in enumerate([(0, 91)] + [(1, 8 + i) for i in range(50)]):
        x = cache.values(b, 0, n)[1]
        want = x.mean(1).repeat_interleave(4, 0)
        # weights 1 / n exactly (in 16 bits too: a power of two each), sums of n products
        assert ((out[t].to(F64) - want).abs() <= half(dtype) * want.abs() + (n + 8) * 2.0 ** -24 * x.abs().mean(1).repeat_interleave(4, 0)).all(), t
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_queries_rotated_and_answered_in_place(dq, dtype, fmt):
    ctx = context(dq, 8, 2, dtype)
    cache = Cache(dq, dtype, fmt, 2, 16, [2000, 300, 5], [2001, 400, 5], wide=WIDE // 16)
    for b, n in enumerate((2000, 300, 5)):
        cache.fill(b, *(torch.randn(2, n, D, device="cuda") for _ in "kv"))
    cu = [0, 1, 101, 101]
    q = torch.randn(101, 8, D, device="cuda").to(dtype)
    kv = torch.randn(2, 101, 2, D, device="cuda").to(dtype)
    pos = torch.arange(101, dtype=torch.int32, device="cuda") + 7
    turned, out = torch.empty_like(q), torch.empty_like(q)
    dq.dapq_paged_append(ctx, cache.view, cu, kv[0], kv[1], pos, q, turned)
    dq.dapq_paged_attend(ctx, cache.view, cu, turned, out)
    dq.dapq_paged_append(ctx, cache.view, cu, kv[0], kv[1], pos, q, q)
    assert torch.equal(q, turned)
    dq.dapq_paged_attend(ctx, cache.view, cu, q, q)
    assert torch.equal(q, out)
    dq.dapq_poll_status(ctx)
    dq.dapq_destroy(ctx)


@gpu
def test_refusals(dq):
    bf = torch.bfloat16
    ctx = context(dq, 8, 2, bf, max_batch=2)
    cache = Cache(dq, bf, "native", 2, 16, [3, 4], [4, 5])
    four = Cache(dq, bf, "fp4", 2, 16, [3, 4], [4, 5])
    kv, q = torch.zeros(2, 2, D, dtype=bf, device="cuda"), torch.zeros(2, 8, D, dtype=bf, device="cuda")
    out, pos = torch.empty_like(q), torch.zeros(2, dtype=torch.int32, device="cuda")

    def refused(status, fn, view=None, **fields):
        keep = {}
        for k, x in fields.items():
            keep[k] = getattr(view, k)
            setattr(view, k, x)
        n = dq.dapq_launch_count(ctx)
        with pytest.raises(dq.DapqError) as e:
            fn()
        assert e.value.status == status and dq.dapq_launch_count(ctx) == n, (fields, str(e.value))
        for k, x in keep.items():
            setattr(view, k, x)

    attend = lambda c=cache, cu=None, **kw: lambda: dq.dapq_paged_attend(ctx, c.view, cu, q, out, **kw)
    for fields, status in ((dict(k=None), 1), (dict(page_table=None), 1), (dict(cache_len=None), 1), (dict(format=2), 1), (dict(reserved=1), 1),
                           (dict(batch=0), 1), (dict(batch=3), 3), (dict(n_pages=0), 1), (dict(table_stride=0), 1), (dict(page_rows=8), 2),
                           (dict(page_rows=48), 2), (dict(page_rows=2048), 2), (dict(row_stride=64), 1), (dict(row_stride=132), 2),
                           (dict(head_stride=-8), 1), (dict(k=cache.view.k + 2), 2), (dict(table_stride=1 << 28), 2)):
        refused(status, attend(), cache.view, **fields)
    for fields, status in ((dict(k_scales=None), 1), (dict(k_scale=0.0), 1), (dict(v_scale=math.nan), 1), (dict(k_scale=-1.0), 1), (dict(row_stride=160), 2),
                           (dict(v_scales=four.view.v_scales + 4), 2)):
        refused(status, attend(four), four.view, **fields)
    refused(1, attend(cu=[1, 2, 2]))
    refused(1, attend(cu=[0, 2, 1]))
    refused(2, attend(cu=[0, 1, 1 << 30]))
    for cap in (-1.0, math.nan, math.inf, 1e-19, 1025.0, 1e19):
        refused(1, attend(softcap=cap))
    refused(2, lambda: dq.dapq_paged_attend(ctx, cache.view, None, q, out.view(-1)[4:4 + 128].view(1, 1, D)))
    refused(1, lambda: dq.dapq_paged_append(ctx, cache.view, None, kv, kv, None, q, out))                       # queries without positions
    refused(1, lambda: dq.dapq_paged_append(ctx, cache.view, None, kv, kv, pos, q, None))
    refused(1, lambda: dq.dapq_paged_append(ctx, cache.view, [0, 5, 4], kv, kv, pos))
    refused(2, lambda: dq.dapq_paged_append(ctx, cache.view, None, kv.view(-1)[4:260].view(1, 2, D), kv, pos))
    dense = torch.zeros(2, 80, D, dtype=bf, device="cuda")
    idx = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    refused(1, lambda: dq.dapq_paged_compact(ctx, dense, dense, [0, 42], [10], idx, [1], cache.view))           # another batch
    refused(1, lambda: dq.dapq_paged_compact(ctx, dense, dense, [0, 40, 80], [10, 8], idx, [1, 1], cache.view))
    back = torch.empty(2, 6, D, dtype=bf, device="cuda")
    refused(1, lambda: dq.dapq_paged_read(ctx, cache.view, None, [3, 4], [0, 3], back, back.clone()))           # one row too many
    refused(1, lambda: dq.dapq_paged_read(ctx, cache.view, None, [-1, 4], [0, 0], back, back.clone()))
    for fn in (lambda: dq.dapq_paged_attend(ctx, cache.view, [0, 1], q, out), lambda: dq.dapq_paged_append(ctx, cache.view, [0, 1, 2, 2], kv, kv),
               lambda: dq.dapq_paged_read(ctx, cache.view, None, [1], [0, 0], back, back.clone())):
        with pytest.raises(AssertionError):                                                                     # offsets of another number of sequences
            fn()
    n = dq.dapq_launch_count(ctx)
    dq.dapq_paged_attend(ctx, cache.view, [0, 0, 0], q, out)                                                    # nothing to do
    dq.dapq_paged_append(ctx, cache.view, [0, 0, 0], kv, kv)
    dq.dapq_paged_read(ctx, cache.view, None, [0, 0], [0, 0], back, back.clone())
    assert dq.dapq_launch_count(ctx) == n
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("fmt", ["native", "fp4"])
def test_captured_steps_grow_with_the_cache(dq, fmt):
    """Append and attend of one decode step in a graph on a stream of its own, replayed as cache_len grows."""
    bf, hq, hkv = torch.bfloat16, 8, 2
    ctx = context(dq, hq, hkv, bf)
    lens, steps = [120, 7], 20
    cache = Cache(dq, bf, fmt, hkv, 16, lens, [a + steps for a in lens])
    for b, a in enumerate(lens):
        cache.fill(b, *(torch.randn(hkv, a, D, device="cuda") for _ in "kv"))
    side = torch.cuda.Stream()
    qkv, pos = torch.zeros(2, hq + 2 * hkv, D, dtype=bf, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    q_rot, out, lse = torch.zeros(2, hq, D, dtype=bf, device="cuda"), torch.zeros(2, hq, D, dtype=bf, device="cuda"), torch.zeros(2, hq, device="cuda")

    def step():
        dq.dapq_paged_append(ctx, cache.view, None, qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], pos, qkv[:, :hq], q_rot)
        dq.dapq_paged_attend(ctx, cache.view, None, q_rot, out, lse)

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        cache.len.fill_(-1)
        step()                                                  # (kernels loaded before the capture; nothing takes part)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for i in range(steps):
            cache.lens = [a + i for a in lens]
            cache.len.copy_(torch.tensor(cache.lens, dtype=torch.int32))
            qkv.normal_()
            pos.fill_(5000 + i)
            graph.replay()
            side.synchronize()
            if i % 6 == 5 or i < 2:
                ref, rlse, tol, ltol = attend_reference(cache, q_rot, [0, 1, 2], 1 / math.sqrt(D))
                assert ((out.to(F64) - ref).abs() <= tol).all() and ((lse.to(F64) - rlse).abs() <= ltol).all()
    dq.dapq_poll_status(ctx, side)
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("fmt", ["native", "fp4"])
def test_pages_past_32_bit_offsets(dq, fmt):
    """Pages 1.3e9 channels apart, rows at both ends."""
    bf = torch.bfloat16
    ctx = context(dq, 4, 1, bf)
    far = 1_300_000_000 // 128 * 128
    per = 2 if fmt == "fp4" else 1
    el = torch.uint8 if fmt == "fp4" else bf
    flat = [torch.zeros((2 * far + 16 * 128) // per, dtype=el, device="cuda") for _ in "kv"]
    k, v = (x.as_strided((3, 1, 16, 128 // per), (far // per, 2048 // per, 128 // per, 1)) for x in flat)
    sc = [None, None]
    if fmt == "fp4":
        sc = [torch.zeros((2 * far + 16 * 128) // 16, dtype=el, device="cuda").as_strided((3, 1, 16, 8), (far // 16, 128, 8, 1)) for _ in "kv"]
    cache = Cache(dq, bf, fmt, 1, 16, [40], [41])
    cache.table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda")
    cache.k, cache.v, cache.ks, cache.vs, cache.n = k, v, *sc, 3
    cache.len.fill_(0)
    cache.view = dq.dapq_paged_cache(k, v, cache.table, cache.len, *sc)
    kv = [torch.randn(41, 1, D, device="cuda").to(bf) for _ in "kv"]
    dq.dapq_paged_append(ctx, cache.view, [0, 41], *kv)
    for got, x in zip(cache.values(0, 0, 41), kv):
        want = x.to(F64).transpose(0, 1)
        assert torch.equal(got, nearest_fp4(want, 1.0)[0] if fmt == "fp4" else want)
    cache.len.fill_(40)
    check_attend(dq, ctx, cache, torch.randn(1, 4, D, device="cuda").to(bf), [0, 1])
    back = [torch.empty(1, 41, D, dtype=bf, device="cuda") for _ in "kv"]
    dq.dapq_paged_read(ctx, cache.view, None, [41], [0], *back)
    assert all(torch.equal(b.to(F64), g) for b, g in zip(back, cache.values(0, 0, 41)))
    dq.dapq_destroy(ctx)


@gpu
@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_evict_decode_and_evict_again(dq, dtype, fmt):
    """A prompt scored and selected, its rows into pages, eight tokens decoded, the pages read back and evicted again."""
    hq, hkv, N = 8, 2, 32
    L, keep = [400, 90], [60, 17]
    ctx = context(dq, hq, hkv, dtype)
    g = torch.Generator(device="cuda").manual_seed(11)
    cu_rows = [0, L[0] + N, L[0] + L[1] + 2 * N]
    k, v = (torch.randn(hkv, cu_rows[-1], D, device="cuda", generator=g).to(dtype) for _ in "kv")
    pseudo = torch.randn(2, hq, N, D, device="cuda", generator=g).to(dtype)
    rot, scores = torch.empty_like(pseudo), torch.empty(hkv, sum(L), device="cuda")
    idx = torch.empty(hkv, sum(keep), dtype=torch.int32, device="cuda")
    dq.dapq_rope_pseudo_q(ctx, pseudo, L, rot)
    dq.dapq_score(ctx, rot, k, cu_rows, L, scores)
    dq.dapq_topk_select(ctx, scores, [0, L[0], sum(L)], keep, idx)
    cache = Cache(dq, dtype, fmt, hkv, 16, [0, 0], [a + 8 for a in keep])
    dq.dapq_paged_compact(ctx, k, v, cu_rows, L, idx, keep, cache.view)
    held = list(keep)
    for step in range(8):
        cache.lens = list(held)
        cache.len.copy_(torch.tensor(held, dtype=torch.int32))
        qkv = torch.randn(2, hq + 2 * hkv, D, device="cuda", generator=g).to(dtype)
        pos = torch.tensor([a + step for a in L], dtype=torch.int32, device="cuda")
        q_rot = torch.empty(2, hq, D, dtype=dtype, device="cuda")
        dq.dapq_paged_append(ctx, cache.view, None, qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], pos, qkv[:, :hq], q_rot)
        check_attend(dq, ctx, cache, q_rot, [0, 1, 2])
        held = [a + 1 for a in held]
    rows = [0, held[0] + N, sum(held) + 2 * N]
    dense = [torch.zeros(hkv, rows[-1], D, dtype=dtype, device="cuda") for _ in "kv"]
    dq.dapq_paged_read(ctx, cache.view, None, held, rows[:2], *dense)
    for b in range(2):
        for got, want in zip(dense, cache.values(b, 0, held[b])):
            assert torch.equal(got[:, rows[b]:rows[b] + held[b]].to(F64), want)
    out = [torch.empty(hkv, 20, D, dtype=dtype, device="cuda") for _ in "kv"]
    second = torch.empty(hkv, 20, dtype=torch.int32, device="cuda")
    dq.dapq_evict(ctx, pseudo, *dense, rows, held, [10, 10], *out, second)
    dq.dapq_poll_status(ctx)
    for h in range(hkv):
        for b in range(2):
            pick = second[h, 10 * b:10 * b + 10].long() + rows[b]
            assert torch.equal(out[0][h, 10 * b:10 * b + 10], dense[0][h, pick])
    dq.dapq_destroy(ctx)
