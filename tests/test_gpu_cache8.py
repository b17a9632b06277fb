"""Caches held in 8 bits on the GPU: appended rows byte for byte, values read back, attention over them against the plain 64-bit form."""
import math

import pytest
import torch

from paper_2604_22808_amd import binding as B
from tests import heads_util as H
from tests import tokens_util as U

pytestmark = pytest.mark.gpu


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32).cuda()


class Cache:
    """Device tensors of a cache and their copy on the host.  pad: bytes between rows; order "heads": head-major."""

    def __init__(self, seed, n, cap, heads, d, block, pad=0, lead=0, order="rows", clean=False):
        gen = torch.Generator().manual_seed(seed)
        self.block, self.shape = block, (n, cap, heads, d)
        codes = [torch.randint(0, 256, self.shape, generator=gen).to(torch.uint8) for _ in range(2)]
        if clean:      # no NaN codes
            codes = [torch.where((c & 0x7f) == 0x7f, c - 1, c) for c in codes]
        scales = [torch.randint(117, 135, (n, -(-cap // block), heads), generator=gen).to(torch.uint8) for _ in range(2)]
        self.codes, self.scales = codes, scales

        def place(c):
            a, b = (heads, cap) if order == "heads" else (cap, heads)
            x = torch.full((lead + n * a * b * (d + pad),), 0x55, dtype=torch.uint8, device="cuda")[lead:].view(n, a, b, d + pad)[..., :d]
            x = x.transpose(1, 2) if order == "heads" else x
            x.copy_(c)
            return x

        self.dev = [place(c) for c in codes]
        self.dev_scales = [s.cuda() for s in scales]

    def args(self):
        return (*self.dev, *self.dev_scales, self.block)

    def values(self, which):
        return U.cache_values(self.codes[which], self.scales[which], self.block)

    def append(self, which, rows, lengths):
        """The same on the host; rows[i]: [new rows, heads, d] of sequence i."""
        n, cap, heads, d = self.shape
        for i, r in enumerate(rows):
            for h in range(heads):
                c, s = self.codes[which][i, :, h].tolist(), self.scales[which][i, :, h].tolist()
                U.append(c, s, self.block, r[:, h].double().tolist(), max(0, min(cap, lengths[i])))
                self.codes[which][i, :, h] = torch.tensor(c, dtype=torch.uint8)
                self.scales[which][i, :, h] = torch.tensor(s, dtype=torch.uint8)


def new_rows(seed, n, heads, d, io):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(n, heads, d, generator=gen) * torch.exp2(torch.randint(-6, 7, (n, 1, 1), generator=gen).float())
    return x.to(io)


def same(c):
    for which in range(2):
        got, want = (torch.where((x & 0x7f) == 0x7f, 0x7f, x) for x in (c.dev[which].cpu(), c.codes[which]))     # (either NaN will do)
        off = (got != want).nonzero().tolist()
        first = [(i, int(got[tuple(i)]), int(want[tuple(i)])) for i in off[:5]]
        assert not off, (which, len(off), first)
        off = (c.dev_scales[which].cpu() != c.scales[which]).nonzero().tolist()
        assert not off, (which, "scales", off[:5])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block,heads,d,cap,new,lengths", [
    (16, 2, 64, 100, [1, 1, 1, 1], [1, 17, 40, 100]), (16, 1, 8, 33, [33, 5, 0], [33, 20, 9]), (32, 3, 40, 70, [40, 31, 33], [70, 63, 64]),
    (64, 1, 128, 300, [250, 64, 65, 1], [300, 64, 129, 65]), (128, 2, 7, 260, [259, 100], [260, 229]), (256, 1, 96, 600, [600, 10], [600, 300]), (64, 1, 1, 5, [5], [5])])
def test_appended_rows(block, heads, d, cap, new, lengths, dtype):
    io, n = U.TYPES[dtype], len(new)
    for packed, pad, lead, order in ((True, 0, 0, "rows"), (False, 0, 0, "heads"), (True, 5, 3, "rows")):
        c = Cache(d + cap, n, cap, heads, d, block, pad, lead, order)
        data = [new_rows(i + 10 * w, max(new), heads, d, io) for w in range(2) for i in range(n)]
        if packed:
            off = [0]
            for x in new:
                off.append(off[-1] + x)
            k, v = (torch.cat([data[w * n + i][:new[i]] for i in range(n)] + [torch.full((2, heads, d), math.nan).to(io)]).cuda() for w in range(2))
            how = dict(q_offsets=ints(off))
        else:
            k, v = (torch.stack(data[w * n:w * n + n]).cuda() for w in range(2))
            how = dict(q_lengths=ints(new))
        B.cache8_append(k, v, *c.args(), k_lengths=ints(lengths), **how)
        for w in range(2):
            c.append(w, [data[w * n + i][:new[i]] for i in range(n)], lengths)
        same(c)
        for t in c.dev:
            if pad:
                at = t.as_strided((n, cap, heads, pad), t.stride(), t.storage_offset() + d)
                assert bool((at == 0x55).all())


@pytest.mark.parametrize("n", [63, 64, 65, 90])
def test_rows_of_about_as_many_sequences_as_lanes(n):
    new = [(5 * i) % 19 for i in range(n)]
    test_appended_rows(16, 2, 24, 40, new, [x + i % 21 for i, x in enumerate(new)], "bf16")


def test_a_row_at_a_time_is_what_growing_scales_make_it():
    """Fifty single rows of growing and shrinking sizes, each after the other, and the same rows in pieces."""
    n, heads, d, block, cap = 2, 2, 16, 16, 60
    rows = [new_rows(50 + i, cap, heads, d, torch.bfloat16) for i in range(2 * n)]
    c = Cache(1, n, cap, heads, d, block)
    for step in range(1, 51):
        lengths = [step, max(step - 3, 0)]
        new = [1, 1 if step > 3 else 0]
        part = [[rows[w * n + i][lengths[i] - new[i]:lengths[i]] for i in range(n)] for w in range(2)]
        k, v = (torch.cat(p).cuda() for p in part)
        B.cache8_append(k, v, *c.args(), q_offsets=ints([0, new[0], sum(new)]), k_lengths=ints(lengths))
        for w in range(2):
            c.append(w, part[w], lengths)
    same(c)


def test_every_code_and_values_beside_borders():
    """All finite values of 16 bits at one scale, and values beside the borders between codes in fp32."""
    bits = torch.arange(0, 0x7f80, dtype=torch.int32)
    x = (bits << 16).view(torch.float32)
    x = x[(x <= 448.0)]
    x = torch.cat([x, -x, torch.tensor([448.0])])
    x = torch.cat([x, torch.zeros(-len(x) % 128)]).view(-1, 1, 128).to(torch.bfloat16)
    lists = [x]
    t = U.TABLE[:127]
    mid = ((t[1:] + t[:-1]) / 2).float()
    near = torch.cat([torch.nextafter(mid, torch.tensor(0.0)), mid, torch.nextafter(mid, torch.tensor(1e9)), -mid, torch.tensor([448.0])])
    lists.append(torch.cat([near, torch.zeros(-len(near) % 128)]).view(-1, 1, 128))
    for x in lists:
        x[:, 0, 0] = 448.0       # every block has the scale 1
        n = x.shape[0]
        c = Cache(2, 1, n, 1, 128, 256)
        B.cache8_append(x[None].cuda(), x[None].cuda(), *c.args())
        for w in range(2):
            c.append(w, [x], [n])
        same(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sizes_at_the_ends_and_values_that_are_not_finite(dtype):
    io, d, cap = U.TYPES[dtype], 24, 16 * 12
    x = torch.randn(cap, 1, d, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
    for i, e in enumerate((-140, -126, -120, -115, -100, 0, 8, 9, 100, 126)):
        at = x[16 * i:16 * i + 16]
        x[16 * i:16 * i + 16] = at / at.abs().max() * 2.0 ** e * (1.75 if i % 2 else 1.7500001)
    x[160:176] = 0.0
    x[180, 0, 3], x[185, 0, 4], x[190, 0, 5] = math.inf, math.nan, -math.inf
    x = x.to(io)
    c = Cache(4, 1, cap, 1, d, 16)
    B.cache8_append(x[None].cuda(), x[None].cuda(), *c.args())
    for w in range(2):
        c.append(w, [x], [cap])
    same(c)
    k, v = (torch.empty(1, cap, 1, d, dtype=io, device="cuda") for _ in range(2))
    B.cache8_read(*c.args(), k, v)
    U.check("values", k, c.values(0), torch.zeros(1, cap, 1, d))      # exact, NaN where they were


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,cap,heads,d,block,lengths", [(3, 70, 2, 40, 16, [70, 0, 33]), (1, 1000, 8, 128, 64, None), (2, 9, 3, 5, 256, [9, 1]), (2, 40, 1, 1, 32, [40, 7])])
def test_values_read_back(n, cap, heads, d, block, lengths, dtype):
    io = U.TYPES[dtype]
    for pad, lead, order in ((0, 0, "rows"), (0, 0, "heads"), (3, 1, "rows")):
        c = Cache(5, n, cap, heads, d, block, pad, lead, order)
        c.scales[0][0, 0, 0] = 255
        c.dev_scales[0].copy_(c.scales[0])
        k, v = (torch.full((n, cap, heads, d + pad), U.MARK, dtype=io, device="cuda")[..., pad:] for _ in range(2))
        B.cache8_read(*c.args(), k, v, k_lengths=ints(lengths))
        inside = torch.arange(cap)[None] < torch.tensor(lengths if lengths else [cap] * n)[:, None]
        for w, t in enumerate((k, v)):
            got, want = t.cpu().double(), c.values(w)
            U.check("inside", got[inside], want[inside], torch.zeros_like(want[inside]))
            assert bool((got[~inside] == U.MARK).all())


def test_lengths_that_are_wrong_stay_inside():
    """Lengths beyond the cache, below zero, offsets that do not ascend: what a call may not touch stays."""
    c = Cache(6, 3, 40, 2, 16, 16)
    before = [t.clone() for t in c.dev]
    x = new_rows(1, 60, 2, 16, torch.bfloat16).cuda()
    B.cache8_append(x, x, *c.args(), q_offsets=ints([0, 5, 5, 20]), k_lengths=ints([-4, 1000, 6]))
    torch.cuda.synchronize()
    for w in range(2):
        got = c.dev[w]
        assert torch.equal(got[0], before[w][0]) and torch.equal(got[1], before[w][1]) and torch.equal(got[2, 6:], before[w][2, 6:])
    host = x[5:20].cpu()
    for w in range(2):
        c.append(w, [host[:0], host[:0], host], [0, 40, 6])      # rows before row 0 are dropped
    same(c)
    B.cache8_append(x, x, *c.args(), q_offsets=ints([30, 10, 50, 2]), k_lengths=ints([40, 40, 40]))
    torch.cuda.synchronize()


# ---- attention

def bounds(res, d, io):
    """What heads_util takes the kernel to do, and more: fp32 queries and probabilities are three bf16 operands each, so sums have three times the terms."""
    if io is torch.float32:
        return {n: (v, 3 * b, inside) for n, (v, b, inside) in res.items()}
    return res


def attend(seed, dtype, n, heads, kv_heads, d, block, cap, q_rows, lengths, q_offsets=None, q_lengths=None, causal=True, pad=0, lead=0, order="rows", spoil=True,
           scale=0.0, workspace=None, q_pad=0):
    io, gen = U.TYPES[dtype], torch.Generator().manual_seed(seed)
    c = Cache(seed, n, cap, kv_heads, d, block, pad, lead, order, clean=True)
    c.scales[0] = torch.randint(117, 120, c.scales[0].shape, generator=gen).to(torch.uint8)      # keys of up to 7, so that scores stay moderate
    c.dev_scales[0].copy_(c.scales[0])
    # codes with mass around a half of the range
    k_len = [cap] * n if lengths is None else lengths
    q_host = torch.randn(1 if q_offsets else n, q_rows, heads, d, generator=gen, dtype=torch.float64).to(io)
    kv = [c.values(w) for w in range(2)]
    q_spans, k_spans = H.spans(q_offsets, q_lengths, q_rows, n), H.spans(None, k_len, cap, n)
    if spoil:      # rows that belong to nobody hold NaN
        for w in range(2):
            for i in range(n):
                c.dev[w][i, k_len[i]:] = 0x7f
        inside = torch.zeros(q_host.shape[:2], dtype=torch.bool)
        for b, first, count in q_spans:
            inside[b, first:first + count] = True
        q_host[~inside] = math.nan
    q = torch.empty(*q_host.shape[:3], d + q_pad, dtype=io, device="cuda")[..., q_pad:]
    q.copy_(q_host)
    out = torch.full((*q_host.shape[:3], d + q_pad), U.MARK, dtype=io, device="cuda")[..., q_pad:]
    lse = torch.full((heads, q_host.shape[0] * q_rows), U.MARK, device="cuda")
    packed = q_offsets is not None
    how = dict(causal=causal, scale=scale, q_offsets=ints(q_offsets), q_lengths=ints(q_lengths), k_lengths=ints(lengths), workspace=workspace)
    B.cache8_attention(q[0] if packed else q, *c.args(), out[0] if packed else out, lse=lse, **how)
    torch.cuda.synchronize()
    # in fp64 from values that bf16 and fp32 hold exactly
    s = scale if scale > 0 else 1.0 / math.sqrt(d)
    res = bounds(H.attend_all(q_host, kv[0].to(io), kv[1].to(io), causal, s, q_spans, k_spans), d, io)
    value, bound, inside = res["out"]
    U.check("out", out.cpu().double()[inside], value[inside], bound[inside])
    assert bool((out.cpu()[~inside] == U.MARK).all())
    value, bound, inside = res["lse"]
    got = lse.cpu().double().view(heads, *q_host.shape[:2]).permute(1, 2, 0)
    U.check("lse", got[inside], value[inside], bound[inside])
    assert bool((got[~inside] == U.MARK).all())
    return out, lse


ONE = [(1, 1, 1, 16, [1]), (3, 4, 1, 64, [1, 40, 64]), (2, 8, 2, 200, [200, 77]), (4, 6, 3, 333, [0, 1, 333, 32]), (1, 16, 2, 1000, [777]), (2, 32, 1, 130, [129, 31]),
       (1, 4, 4, 3000, [2999])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,block", [(128, 64), (64, 16), (96, 32), (72, 128), (8, 256), (40, 16)])
def test_one_token(d, block, dtype):
    for i, (n, heads, kv_heads, cap, lengths) in enumerate(ONE):
        attend(100 + i, dtype, n, heads, kv_heads, d, block, cap, 1, lengths)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,block", [(128, 64), (64, 32), (88, 16), (24, 128)])
def test_rows_of_prompts(d, block, dtype):
    attend(1, dtype, 2, 4, 2, d, block, 300, 60, [300, 111], causal=True)
    attend(2, dtype, 3, 4, 1, d, block, 170, 90, [170, 64, 0], q_offsets=[0, 50, 51, 90], causal=True)
    attend(3, dtype, 2, 2, 2, d, block, 200, 140, [200, 33], q_lengths=[140, 70], causal=False)
    attend(4, dtype, 2, 3, 3, d, block, 65, 200, [65, 64], causal=True)       # more queries than keys: the first see nothing
    attend(5, dtype, 1, 2, 1, d, block, 700, 300, [650], causal=True, scale=0.02)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64, 20, 33, 1])
def test_rows_of_any_address_and_order(d, dtype):
    for kw in (dict(order="heads"), dict(pad=8, lead=8), dict(pad=3, lead=1), dict(q_pad=3)):
        attend(7, dtype, 2, 4, 2, d, 16, 90, 1, [90, 35], **kw)
        attend(8, dtype, 2, 4, 2, d, 32, 150, 70, [150, 35], **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_caches_in_pieces(dtype):
    attend(9, dtype, 1, 8, 2, 128, 64, 5000, 1, [4999])
    attend(10, dtype, 2, 4, 4, 64, 16, 2100, 5, [2100, 70])
    attend(11, dtype, 1, 4, 1, 128, 256, 3000, 40, [2900])
    attend(12, dtype, 40, 2, 2, 64, 64, 500, 1, list(range(1, 500, 13))[:38] + [500, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,cap,heads,kv_heads,d,lengths", [(1, 20003, 8, 1, 64, [20003]), (1, 24577, 4, 2, 128, None), (2, 20064, 4, 1, 72, [19278, 12312]), (3, 20001, 2, 1, 40, [6085, 20001, 0])])
def test_caches_of_more_steps_than_pieces(n, cap, heads, kv_heads, d, lengths, dtype):
    attend(60 + d, dtype, n, heads, kv_heads, d, 64, cap, 1, lengths)
    attend(61 + d, dtype, n, heads, kv_heads, d, 64, cap, 5, lengths)


def test_workspaces_hold_no_more_than_64_pieces():
    for cap in (8192, 8193, 16640, 20064, 100000):
        for n in (1, 2, 3, 64, 65):
            for rows in (1, 30, 1000):
                shape = B.SequenceShape(n, 8, 1, 64, rows, cap, B.BF16, 1, 0.0)
                need = B.lib().freqattn_cache8_attention_workspace(shape, B.SequenceRows(None, None, None, 16))
                assert need <= 64 * 8 * n * rows * 65 * 4 + 16, (cap, n, rows)      # 64 results and log sums a row and head; 16 bytes for the length of a piece


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences_and_uneven_ones(dtype):
    """More sequences than lanes of a wave; rows of a few sequences that fill tiles unevenly; caches whose lengths differ by all there is."""
    lengths = [(37 * i) % 301 for i in range(70)]
    attend(20, dtype, 70, 2, 1, 64, 16, 300, 1, lengths)
    attend(21, dtype, 66, 4, 2, 32, 64, 120, 66 * 2, [min(120, 3 + 2 * i) for i in range(66)], q_offsets=[2 * i for i in range(67)])
    attend(22, dtype, 5, 8, 2, 128, 32, 3000, 23, [3000, 1, 0, 1500, 20], q_offsets=[0, 1, 2, 2, 20, 23])
    attend(23, dtype, 3, 4, 1, 72, 64, 2500, 8, [2500, 100, 2400])
    attend(24, dtype, 2, 4, 2, 128, 64, 4200, 330, [4200, 300])
    attend(25, dtype, 3, 4, 4, 64, 128, 2600, 400, [2600, 900, 0], q_offsets=[0, 300, 390, 400], causal=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_caches_of_no_rows_and_calls_of_none(dtype):
    io = U.TYPES[dtype]
    q = torch.randn(2, 3, 4, 64, device="cuda").to(io)
    out, lse = torch.full_like(q, U.MARK), torch.full((4, 6), U.MARK, device="cuda")
    none = torch.empty(2, 0, 2, 64, dtype=torch.uint8, device="cuda")
    scales = torch.empty(2, 0, 2, dtype=torch.uint8, device="cuda")
    B.cache8_attention(q, none, none, scales, scales, 64, out, lse=lse, causal=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    B.cache8_append(q[:, :, :2], q[:, :, :2], none, none, scales, scales, 64)
    c = Cache(1, 2, 20, 2, 64, 16)
    B.cache8_append(q[:, :0, :2], q[:, :0, :2], *c.args())
    B.cache8_attention(q[:, :0], *c.args(), out[:, :0])
    B.cache8_attention(q[:0], *(t[:0] for t in (*c.dev, *c.dev_scales)), 16, out[:0])
    B.cache8_read(*(t[:0] for t in (*c.dev, *c.dev_scales)), 16, *(torch.empty(0, 20, 2, 64, dtype=io, device="cuda") for _ in range(2)))
    torch.cuda.synchronize()
    same(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_workspaces_hold_does_not_matter_and_calls_repeat(dtype):
    """Pieces joined from a workspace of NaN; equal calls give equal bits, also one after the other on one workspace."""
    io = U.TYPES[dtype]
    for n, rows, cap, lengths in ((3, 1, 6000, [6000, 100, 2500]), (1, 2, 5000, [4000]), (2, 300, 4000, [4000, 1000])):
        c = Cache(30, n, cap, 2, 64, 64, clean=True)
        q = torch.randn(n, rows, 4, 64, generator=torch.Generator().manual_seed(1)).to(io).cuda()
        need = B.lib().freqattn_cache8_attention_workspace(B.SequenceShape(n, 4, 2, 64, rows, cap, B.BF16 if dtype == "bf16" else B.F32, 1, 0.0), B.SequenceRows(None, None, None, 16))
        assert need > 0
        res = []
        for fill in (math.nan, math.inf, 0.0):
            ws = torch.full((need // 4 + 64,), fill, device="cuda")
            for _ in range(2):
                out, lse = torch.empty_like(q), torch.empty(4, n * rows, device="cuda")
                B.cache8_attention(q, *c.args(), out, lse=lse, causal=True, k_lengths=ints(lengths), workspace=ws[:need // 4])
                res.append((out, lse))
            assert torch.equal(ws[need // 4:].nan_to_num(1.0), torch.full((64,), fill, device="cuda").nan_to_num(1.0))
        for out, lse in res[1:]:
            assert torch.equal(out, res[0][0]) and torch.equal(lse, res[0][1])
        with pytest.raises(B.FreqAttnError):
            B.cache8_attention(q, *c.args(), out, causal=True, k_lengths=ints(lengths), workspace=ws[:need // 4 - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 20, 150])
def test_nan_behind_the_diagonal_and_keys_that_are_seen(rows, dtype):
    """NaN codes among the keys of a causal call reach the queries that see them and no others; a scale byte of 255 spoils its block alone."""
    io, n, heads, d, cap, block = U.TYPES[dtype], 1, 2, 64, 256, 16
    c = Cache(13, n, cap, heads, d, block, clean=True)
    for w in range(2):
        c.scales[w].fill_(118)
        c.dev_scales[w].copy_(c.scales[w])
    q = torch.randn(n, rows, heads, d, generator=torch.Generator().manual_seed(1)).to(io).cuda()
    length = 200
    clean, out = torch.empty_like(q), torch.empty_like(q)
    B.cache8_attention(q, *c.args(), clean, causal=True, k_lengths=ints([length]))
    for which, at in ((0, length - 1), (1, length - 1), (1, length - 2)):
        keep = c.dev[which][0, at, 0, 3].clone()
        c.dev[which][0, at, 0, 3] = 0x7f
        B.cache8_attention(q, *c.args(), out, causal=True, k_lengths=ints([length]))
        c.dev[which][0, at, 0, 3] = keep
        hit = rows - (length - at)                     # the first query that sees the key
        assert torch.equal(out[0, :, 1], clean[0, :, 1])
        if hit > 0:
            assert bool(((out[0, :hit, 0].float() - clean[0, :hit, 0].float()).abs() <= 0.02 * clean[0, :hit, 0].float().abs().max()).all())
        row = out[0, hit:, 0]
        assert bool(torch.isnan(row if which == 0 else row[:, 3]).all())
        if which == 1:
            assert not bool(torch.isnan(row[:, 4:]).any())
    c.dev_scales[1][0, 3, 1] = 255
    B.cache8_attention(q, *c.args(), out, causal=True, k_lengths=ints([length]))
    assert torch.equal(out[0, :, 0], clean[0, :, 0])
    first = max(0, 48 - (length - rows))
    assert bool(torch.isnan(out[0, first:, 1]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_that_are_not_finite_and_large_scores(dtype):
    io, heads, d, cap = U.TYPES[dtype], 2, 64, 300
    for rows in (1, 40):
        c = Cache(14, 1, cap, heads, d, 64, clean=True)
        q = 30 * torch.randn(1, rows, heads, d, generator=torch.Generator().manual_seed(2), dtype=torch.float64).to(io)
        kv = [c.values(w) for w in range(2)]
        out, lse = torch.empty_like(q, device="cuda"), torch.empty(heads, rows, device="cuda")
        B.cache8_attention(q.cuda(), *c.args(), out, lse=lse)
        res = bounds(H.attend_all(q, kv[0].to(io), kv[1].to(io), False, 1 / math.sqrt(d), H.spans(None, None, rows, 1), H.spans(None, None, cap, 1)), d, io)
        U.check("out", out, *res["out"][:2])
        U.check("lse", lse.T[None], *res["lse"][:2])
        bad = q.clone()
        bad[0, 0, 0, 5], bad[0, rows - 1, 1, 6] = math.inf, math.nan
        o2 = torch.empty_like(out)
        B.cache8_attention(bad.cuda(), *c.args(), o2)
        assert bool(torch.isnan(o2[0, 0, 0]).all()) and bool(torch.isnan(o2[0, rows - 1, 1]).all())
        if rows > 1:
            assert torch.equal(o2[0, 1:rows - 1], out[0, 1:rows - 1])


def test_rows_behind_2_31_bytes():
    """A cache of 4.5 GB: the last sequence's rows lie behind 32 bits."""
    n, cap, heads, d = 9, 1 << 16, 64, 128
    codes = [torch.zeros(n, cap, heads, d, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((n, cap // 64, heads), 120, dtype=torch.uint8, device="cuda") for _ in range(2)]
    rows = new_rows(5, 70, heads, d, torch.bfloat16)
    lengths = ints([0] * (n - 1) + [cap])
    off = ints([0] * n + [70])
    B.cache8_append(rows.cuda(), rows.cuda(), *codes, *scales, 64, q_offsets=off, k_lengths=lengths)
    c, s = [[0] * d for _ in range(128)], [120, 120]
    U.append(c, s, 64, rows[:, 7].double().tolist(), 128)
    assert codes[0][n - 1, cap - 128:, 7].tolist() == c and scales[1][n - 1, -2:, 7].tolist() == s
    q = torch.randn(1, heads, d, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    out = torch.zeros(1, heads, d, dtype=torch.bfloat16, device="cuda")
    B.cache8_attention(q.cuda(), *codes, *scales, 64, out, q_offsets=ints([0] * n + [1]), k_lengths=lengths)
    value = U.cache_values(torch.tensor(c, dtype=torch.uint8)[None, :, None], torch.tensor(s, dtype=torch.uint8)[None, :, None], 64)[0, :, 0]
    kv = torch.cat([torch.zeros(cap - 128, d, dtype=torch.float64), value])
    want, bound = H.attend(q[:, 7], kv, kv, False, 1 / math.sqrt(d), torch.bfloat16)["out"]
    U.check("far", out[:, 7], want, bound)
