"""The 8-bit cache: quantising as it is written, reading back, attention over it - each against its definition in 64 bits
(tests/kv8ref.py, where the bounds are derived) - and the draft/verify path on such a cache."""
import math

import numpy as np
import pytest
import torch

import kv8ref
from paper_2505_08600_amd import api
from paper_2505_08600_amd import datagen as dg

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
i32 = lambda *a: torch.tensor(a, dtype=torch.int32)


def starts(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32)


# ---------------------------------------------------------------- append and read
def rows_with_edges(g, n, heads, dim, dtype):
    x = torch.randn(n, heads, dim, generator=g) * torch.exp(2 * torch.randn(n, heads, 1, generator=g))
    f = x.view(-1, dim)
    special = [torch.zeros(dim), torch.full((dim,), 1e-30), torch.full((dim,), -0.0), torch.full((dim,), 2.0 ** -60 * 0.5),
               torch.arange(dim).float() - dim / 2, torch.full((dim,), 3e38), torch.full((dim,), 1e-44)]
    ties = torch.arange(dim).float() % 120 + 0.5
    ties[0] = 127.0                                      # scale 1: every other element lies on a half
    special += [ties, -ties]
    bad = torch.ones(dim)
    bad[dim // 3] = math.nan
    worse = torch.ones(dim)
    worse[-1] = -math.inf
    for k, s in enumerate(special + [bad, worse]):
        f[(k * 7) % f.shape[0]] = s
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,dim", [(1, 16), (12, 64), (32, 128), (3, 80), (2, 256), (5, 48)])
def test_append_and_read(dtype, heads, dim):
    print(f"append/read {dtype} {heads} x {dim}", flush=True)
    g = torch.Generator().manual_seed(heads * 1000 + dim)
    caps, counts, lens = [40, 9, 30, 70], [17, 0, 30, 33], [5, 9, 0, 37]
    ref = kv8ref.Cache(caps, heads, dim, gap=3)
    for t in (ref.k, ref.v):
        t.random_(-127, 128, generator=g)
    cache = ref.to_gpu()
    n = sum(counts)
    k, v = rows_with_edges(g, n + 2, heads, dim, dtype), rows_with_edges(g, n + 2, heads, dim, dtype)
    rs = starts(counts)
    api.sd_kv8_append(cache, i32(*lens).cuda(), k.cuda(), v.cuda(), row_start=rs.cuda())   # two rows behind the last sequence
    for x, codes, scales in ((k, ref.k, ref.ks), (v, ref.v, ref.vs)):
        c, s = kv8ref.quantise(x)
        for b, (l, m) in enumerate(zip(lens, counts)):
            at, r = ref.off[b] + l, int(rs[b])
            codes[:, at:at + m] = c[r:r + m].transpose(0, 1).to(torch.int8)
            scales[:, at:at + m] = s[r:r + m].T
    got_v, got_ks, got_vs, _, _, status = [t.cpu() for t in cache._keep]
    assert torch.equal(cache.k.cpu(), ref.k) and torch.equal(got_v, ref.v)
    assert torch.equal(got_ks.view(torch.int32) & 0x7fffffff, ref.ks.view(torch.int32) & 0x7fffffff)   # (a NaN's bits too)
    assert torch.equal(torch.nan_to_num(got_vs), torch.nan_to_num(ref.vs)) and status.item() == 0
    for out_t in (F32, BF16):
        ko, vo = (torch.full((n + 2, heads, dim), 5.0, dtype=out_t).cuda() for _ in range(2))
        api.sd_kv8_read(cache, i32(*lens).cuda(), ko, vo, row_start=rs.cuda())
        for x, y in ((k, ko), (v, vo)):
            c, s = kv8ref.quantise(x[:n])
            want = (c.float() * s.unsqueeze(-1)).to(out_t)       # one product in 32 bits, one rounding
            assert torch.equal(torch.nan_to_num(y[:n].cpu(), nan=1e3), torch.nan_to_num(want, nan=1e3))
            assert (y[n:] == 5.0).all()


def test_read_one_of_two_strided_and_unaligned():
    ref = kv8ref.Cache([20, 20], 3, 64).fill(1)
    cache = ref.to_gpu()
    for dtype in (F32, BF16):
        buf = torch.full((1 + 8 * 5 * 70,), 9.0, dtype=dtype).cuda()
        k = buf[1:].view(8, 5, 70)[:, 1:4, 3:67]
        api.sd_kv8_read(cache, i32(4, 11).cuda(), k, None)
        want = torch.cat([ref.k[:, 4:8].float() * ref.ks[:, 4:8, None], ref.k[:, 31:35].float() * ref.ks[:, 31:35, None]], 1)
        assert torch.equal(k.cpu(), want.transpose(0, 1).to(dtype))
        k[:] = 9.0
        assert (buf == 9.0).all()
        v = torch.zeros(3, 8, 64, dtype=dtype).cuda().transpose(0, 1)
        api.sd_kv8_read(cache, i32(4, 11).cuda(), None, v)
        want = torch.cat([ref.v[:, 4:8].float() * ref.vs[:, 4:8, None], ref.v[:, 31:35].float() * ref.vs[:, 31:35, None]], 1)
        assert torch.equal(v.cpu(), want.transpose(0, 1).to(dtype))


def test_rows_outside_their_sequence_are_dropped_and_flagged():
    ref = kv8ref.Cache([8, 8, 8], 2, 64)
    cache = ref.to_gpu()
    k = torch.ones(9, 2, 64)
    api.sd_kv8_append(cache, i32(6, -1, 2 ** 31 - 2).cuda(), k.cuda(), k.cuda())      # tokens 6 7 8, -1 0 1, far away
    assert cache.status.item() == 1
    written = cache.k.cpu().ne(0).any(-1)
    assert written[:, [6, 7, 8, 9]].all() and written.sum() == 2 * 4
    cache.status.zero_()
    out = torch.full((9, 2, 64), 5.0).cuda()
    api.sd_kv8_read(cache, i32(6, -1, 2 ** 31 - 2).cuda(), out, None)
    assert cache.status.item() == 1
    assert [bool((out[r] == 1.0).all()) for r in range(9)] == [True, True, False, False, True, True, False, False, False]
    assert (out[[2, 3, 6, 7, 8]] == 5.0).all()
    cache.status.zero_()
    api.sd_kv8_append(cache, i32(0, 0, 0).cuda(), 2 * k[:6].cuda(), 2 * k[:6].cuda(), seq_ids=i32(3, 1).cuda())
    assert cache.status.item() == 4 and cache.k.cpu().ne(0).any(-1).sum() == 2 * (2 + 3)   # sequence 1 only: tokens 0..2


def test_offsets_behind_32_bits():
    """A cache of 5.2e9 codes: the last sequence's codes lie behind 2^32 in every head but the first."""
    heads, dim, caps = 3, 128, [13_500_000, 333]
    n = sum(caps)
    k, v = (torch.empty(heads, n, dim, dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.empty(heads, n, device="cuda") for _ in range(2))
    assert k.numel() > 2 ** 32
    for t in (k, v, ks, vs):
        t[:, -400:] = 0
        t[:, :8] = 0
    cache = api.Kv8Cache(k, v, ks, vs, torch.tensor([0, caps[0]]).cuda(), i32(*caps).cuda())
    g = torch.Generator().manual_seed(4)
    new = torch.randn(2 * 300, heads, dim, generator=g)
    far = caps[0] - 300
    api.sd_kv8_append(cache, i32(far, 30).cuda(), new.cuda(), (2 * new).cuda())
    back, back_v = torch.zeros(600, heads, dim).cuda(), torch.zeros(600, heads, dim).cuda()
    api.sd_kv8_read(cache, i32(far, 30).cuda(), back, back_v)
    c, s = kv8ref.quantise(new)
    assert torch.equal(back.cpu(), c.float() * s[..., None]) and torch.equal(back_v.cpu(), c.float() * (2 * s)[..., None])
    small = kv8ref.Cache([333], heads, dim)
    for a, b in ((small.k, k), (small.v, v), (small.ks, ks), (small.vs, vs)):
        a.copy_(b[:, caps[0]:].cpu())
    for dtype in (F32, BF16):
        q = torch.randn(2, heads, dim, generator=g).to(dtype)
        out = torch.zeros_like(q).cuda()
        api.sd_kv8_attend(cache, i32(0, 328).cuda(), q.cuda(), out, dim ** -0.5, seq_ids=i32(1).cuda(), max_len=328)
        want, _, bound, _ = kv8ref.attend(small, q, [(0, 328, 0, 2)], dim ** -0.5)
        assert ((out.cpu().double() - want).abs() <= bound).all()


# ---------------------------------------------------------------- attention
def run_attend(cache, q, lens, counts, scale, causal=True, window=0, sinks=0, ragged=True, seq_ids=None, extra=2, max_len=None):
    """-> (out, lse) with `extra` rows behind the last sequence, which have to stay as they were."""
    rows, heads, dim = q.shape
    pad = torch.full((extra if ragged else 0, heads, dim), 3.0, dtype=q.dtype)
    qd = torch.cat([q, pad]).cuda()
    out, lse = torch.full_like(qd, 3.0), torch.full((qd.shape[0], heads), 3.0).cuda()
    api.sd_kv8_attend(cache, i32(*lens).cuda(), qd, out, scale, row_start=starts(counts).cuda() if ragged else None, max_rows=max(counts),
                      max_len=max(max(lens), 0) if max_len is None else max_len, causal=causal, window=window, sinks=sinks, lse=lse,
                      seq_ids=None if seq_ids is None else i32(*seq_ids).cuda())
    assert (out[rows:] == 3.0).all() and (lse[rows:] == 3.0).all()
    return out[:rows].cpu(), lse[:rows].cpu()


def close(got, want):
    out, lse, b_out, b_lse = want
    d = (got[0].double() - out).abs()
    assert (d <= b_out).all(), f"out: {(d / b_out.clamp_min(1e-300)).max():.3g} of its bound"
    assert torch.equal(torch.isinf(got[1]), torch.isinf(lse))
    e = torch.nan_to_num((got[1].double() - lse).abs())
    assert (e <= b_lse).all(), f"lse: {(e / b_lse.clamp_min(1e-300)).max():.3g} of its bound"


SHAPES = [  # heads, cache heads, dim, lengths, rows of each
    (1, 1, 64, [0], [1]),
    (12, 12, 64, [100], [1]),
    (4, 4, 128, [31, 32, 33, 63], [1, 1, 1, 1]),
    (2, 2, 128, [511, 0, 64, 1], [6, 6, 6, 6]),
    (8, 2, 128, [200, 95], [5, 5]),
    (16, 1, 64, [77, 300], [3, 3]),
    (5, 1, 128, [40, 129], [16, 16]),
    (2, 1, 16, [33, 5], [2, 2]),
    (3, 3, 80, [60, 61], [4, 4]),
    (4, 2, 256, [70, 1], [3, 3]),
    (6, 3, 96, [130], [2]),
    (6, 3, 32, [130], [2]),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv,dim,lens,rows", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (40, 0), (33, 5)])
def test_attention_of_a_step(dtype, heads, kv, dim, lens, rows, window, sinks):
    print(f"attend {dtype} {heads}/{kv} x {dim} lens {lens} rows {rows} window {window} sinks {sinks}", flush=True)
    g = torch.Generator().manual_seed(sum(lens) + dim)
    ref = kv8ref.Cache([a + b + 2 for a, b in zip(lens, rows)], kv, dim, gap=1).fill(dim + heads)
    q = (1.5 * torch.randn(sum(rows), heads, dim, generator=g)).to(dtype)
    first = starts(rows).tolist()
    parts = [(b, lens[b], first[b], rows[b]) for b in range(len(lens))]
    got = run_attend(ref.to_gpu(), q, lens, rows, dim ** -0.5, window=window, sinks=sinks, ragged=False)
    close(got, kv8ref.attend(ref, q, parts, dim ** -0.5, True, window, sinks))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 64), (3, 3, 128), (8, 1, 128), (2, 2, 48)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3), (7, 0)])
def test_attention_of_prompts(dtype, heads, kv, dim, window, sinks):
    """Ragged pieces of prompts: none, one row, some with a context, rows past several tiles."""
    print(f"prompts {dtype} {heads}/{kv} x {dim} window {window} sinks {sinks}", flush=True)
    g = torch.Generator().manual_seed(dim + heads)
    lens, rows = [0, 37, 300, 64, 5], [130, 0, 65, 1, 33]
    ref = kv8ref.Cache([a + b + 1 for a, b in zip(lens, rows)], kv, dim, gap=2).fill(7 * dim + heads)
    q = (1.5 * torch.randn(sum(rows), heads, dim, generator=g)).to(dtype)
    first = starts(rows).tolist()
    parts = [(b, lens[b], first[b], rows[b]) for b in range(len(lens))]
    got = run_attend(ref.to_gpu(), q, lens, rows, dim ** -0.5, window=window, sinks=sinks)
    close(got, kv8ref.attend(ref, q, parts, dim ** -0.5, True, window, sinks))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [1, 5, 40])
def test_attention_over_a_cache_the_rows_are_not_part_of(dtype, rows):
    lens = [0, 1, 77, 260]
    ref = kv8ref.Cache([max(l, 1) for l in lens], 2, 64).fill(3)
    q = torch.randn(rows * 4, 4, 64, generator=torch.Generator().manual_seed(rows)).to(dtype)
    got = run_attend(ref.to_gpu(), q, lens, [rows] * 4, 0.2, causal=False, ragged=False)
    assert (got[0][:rows] == 0).all() and (got[1][:rows] == -math.inf).all()          # an empty context
    close(got, kv8ref.attend(ref, q, [(b, lens[b], b * rows, rows) for b in range(4)], 0.2, causal=False))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128, 48])
def test_unseen_tokens_leave_no_trace(dtype, dim):
    """NaN scales in front of the window, behind the last token and in the neighbours: not one bit of the result changes."""
    lens, rows, heads = [150, 90], [3, 40], 2
    clean = kv8ref.Cache([200, 200], heads, dim, gap=40).fill(11)
    q = torch.randn(43, heads, dim, generator=torch.Generator().manual_seed(1)).to(dtype)
    for window, sinks in ((0, 0), (45, 3)):
        dirty = kv8ref.Cache([200, 200], heads, dim, gap=40)
        for a, b in ((dirty.k, clean.k), (dirty.v, clean.v), (dirty.ks, clean.ks), (dirty.vs, clean.vs)):
            a.copy_(b)
        seen = torch.zeros(dirty.tokens, dtype=torch.bool)
        for b in range(2):
            for i in range(rows[b]):
                seen[[dirty.off[b] + t for t in kv8ref.visible(lens[b], i, 200, True, window, sinks)]] = True
        for s in (dirty.ks, dirty.vs):
            s[:, ~seen] = math.nan
        got = [run_attend(c.to_gpu(), q, lens, rows, 0.125, window=window, sinks=sinks) for c in (clean, dirty)]
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        assert torch.isfinite(got[1][0]).all()
    dirty.vs[0, dirty.off[0] + 149] = math.nan            # ... and a token that is seen does show, in the rows of its sequence and head
    dirty.ks[1, dirty.off[1] + 95] = math.nan
    out, lse = run_attend(dirty.to_gpu(), q, lens, rows, 0.125, window=window, sinks=sinks)
    assert torch.isnan(out[:3, 0]).all() and torch.isfinite(out[:3, 1]).all() and torch.isfinite(out[3:, 0]).all()
    assert torch.isfinite(out[3:8, 1]).all() and torch.isnan(out[8:, 1]).all() and torch.isnan(lse[8:, 1]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (45, 3)])
def test_unseen_tokens_leave_no_trace_in_prompts(dtype, dim, window, sinks):
    """The same with more rows: NaN scales of every token that no row sees, and of one that only the last rows see."""
    lens, rows, heads = [150, 33], [70, 131], 2
    clean = kv8ref.Cache([300, 300], heads, dim, gap=40).fill(11)
    dirty = kv8ref.Cache([300, 300], heads, dim, gap=40)
    for a, b in ((dirty.k, clean.k), (dirty.v, clean.v), (dirty.ks, clean.ks), (dirty.vs, clean.vs)):
        a.copy_(b)
    seen = torch.zeros(dirty.tokens, dtype=torch.bool)
    for b in range(2):
        for i in range(rows[b]):
            seen[[dirty.off[b] + t for t in kv8ref.visible(lens[b], i, 300, True, window, sinks)]] = True
    for s in (dirty.ks, dirty.vs):
        s[:, ~seen] = math.nan
    q = torch.randn(sum(rows), heads, dim, generator=torch.Generator().manual_seed(1)).to(dtype)
    got = [run_attend(c.to_gpu(), q, lens, rows, 0.125, window=window, sinks=sinks) for c in (clean, dirty)]
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and torch.isfinite(got[1][0]).all()
    dirty.vs[0, dirty.off[0] + 200] = math.nan            # seen from row 50 of the first sequence on
    dirty.ks[1, dirty.off[1] + 160] = math.nan            # seen from row 127 of the second one on
    out, lse = run_attend(dirty.to_gpu(), q, lens, rows, 0.125, window=window, sinks=sinks)
    last = 70 if not window else min(70, 50 + 45)
    assert torch.isnan(out[50:last, 0]).all() and torch.equal(out[:50, 0], got[0][0][:50, 0]) and torch.equal(out[:70, 1], got[0][0][:70, 1])
    assert torch.isnan(out[70 + 127:, 1]).all() and torch.equal(out[70:70 + 127, 1], got[0][0][70:70 + 127, 1]) and torch.equal(out[70:, 0], got[0][0][70:, 0])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_ids_and_rows_left_alone(dtype):
    """q inside a packed buffer, out with gaps, sequences out of order, one id out of range."""
    heads, kv, dim, lens = 4, 2, 64, [20, 90, 45]
    ref = kv8ref.Cache([100] * 3, kv, dim).fill(5)
    cache = ref.to_gpu()
    g = torch.Generator().manual_seed(2)
    for shift in (0, 1):
        packed = torch.randn(1 + 12 * 8 * 72, generator=g).to(dtype)
        q = packed[shift:shift + 12 * 8 * 72].view(12, 8, 72)[:, 2:6, :64]
        buf = torch.full((1 + 12 * 5 * 66,), 3.0, dtype=dtype).cuda()
        out = buf[shift:shift + 12 * 5 * 66].view(12, 5, 66)[:, 1:, 2:]
        qd = packed.cuda()[shift:shift + 12 * 8 * 72].view(12, 8, 72)[:, 2:6, :64]
        api.sd_kv8_attend(cache, i32(*lens).cuda(), qd, out, 0.125, seq_ids=i32(2, 7, 0).cuda(), max_len=90)
        assert cache.status.item() == 4
        cache.status.zero_()
        want, _, bound, _ = kv8ref.attend(ref, q.contiguous(), [(2, 45, 0, 4), (0, 20, 8, 4)], 0.125)
        assert (out[4:8] == 3.0).all()
        live = [0, 1, 2, 3, 8, 9, 10, 11]
        assert ((out.cpu().double() - want).abs() <= bound)[live].all()
        out[:] = 3.0
        assert (buf == 3.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128])
def test_wide_ranges(dtype, dim):
    """Values whose scales span many powers of two, rows of zeros, large and small queries, scores far from zero."""
    ref = kv8ref.Cache([400], 2, dim).fill(1, spread=0.5)
    g = torch.Generator().manual_seed(8)
    ref.vs *= 2.0 ** torch.randint(-12, 13, ref.vs.shape, generator=g).float()
    ref.v[:, 5], ref.vs[:, 5] = 0, kv8ref.SCALE_MIN
    ref.v[:, 200:230], ref.vs[:, 200:230] = 0, kv8ref.SCALE_MIN
    ref.ks[:, 300:] *= 3.0
    q = torch.randn(6, 2, dim, generator=g)
    q[1] *= 1e-6
    q[2] *= 8.0
    q[3] *= 1e-30
    q[4, :, 1:] = 0
    q[5] = 0
    q = q.to(dtype)
    close(run_attend(ref.to_gpu(), q, [380], [6], dim ** -0.5), kv8ref.attend(ref, q, [(0, 380, 0, 6)], dim ** -0.5))
    close(run_attend(ref.to_gpu(), q, [380], [6], -0.3), kv8ref.attend(ref, q, [(0, 380, 0, 6)], -0.3))
    ref.vs *= 1e-12                                       # all of them small, all of them large
    close(run_attend(ref.to_gpu(), q, [380], [6], 0.1), kv8ref.attend(ref, q, [(0, 380, 0, 6)], 0.1))
    ref.vs *= 1e24
    close(run_attend(ref.to_gpu(), q, [380], [6], 0.1), kv8ref.attend(ref, q, [(0, 380, 0, 6)], 0.1))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv,dim,length,rows,window,sinks", [(2, 2, 128, 5000, 6, 0, 0), (4, 1, 64, 9001, 1, 0, 0), (8, 2, 128, 3333, 16, 0, 0),
                                                                   (2, 1, 64, 7000, 3, 2500, 70), (2, 1, 128, 2100, 200, 0, 0)])
def test_long_contexts_split_or_not(dtype, heads, kv, dim, length, rows, window, sinks):
    """With a workspace (split over blocks) and without one, and whatever the caller takes the longest context for."""
    print(f"long {dtype} {heads}/{kv} x {dim} len {length} rows {rows} window {window}", flush=True)
    ref = kv8ref.Cache([length + rows, 50 + rows], kv, dim).fill(9)
    cache, lens, n = ref.to_gpu(), [length, 50], 2 * rows
    q = (1.5 * torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(6))).to(dtype)
    show = sorted({0, rows // 2, rows - 1})
    want = kv8ref.attend(ref, q, [(0, length + i, i, 1) for i in show] + [(1, 50 + i, rows + i, 1) for i in show], dim ** -0.5, True, window, sinks)
    live = show + [rows + i for i in show]
    pick = lambda t: tuple(x[live] for x in t)
    first = None
    for max_len in (length, 0, 100_000):
        got = run_attend(cache, q, lens, [rows] * 2, dim ** -0.5, window=window, sinks=sinks, ragged=False, max_len=max_len)
        close(pick(got), pick(want))
        again = run_attend(cache, q, lens, [rows] * 2, dim ** -0.5, window=window, sinks=sinks, ragged=False, max_len=max_len)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])     # the same call, the same bits
        first = first or got
    # without a workspace
    qd, out, lse = q.cuda(), torch.zeros_like(q).cuda(), torch.zeros(n, heads).cuda()
    ld = i32(*lens).cuda()
    a = api._Kv8Attn(None, ld.data_ptr(), None, 2, n, 0, length, heads, api._DTYPES[dtype], *api._rows3(qd, "q"), *api._rows3(out, "out"),
                     lse.data_ptr(), dim ** -0.5, 1, window, sinks, None, 0)
    api._check(api.lib().sd_kv8_attend(api.C.byref(cache.c), api.C.byref(a), api._stream()))
    close(pick((out.cpu(), lse.cpu())), pick(want))
    need = api.lib().sd_kv8_attend_workspace(api.C.byref(cache.c), api.C.byref(a))
    if need > 16:
        ws = torch.empty(need, dtype=torch.uint8).cuda()
        a.workspace, a.workspace_bytes = ws.data_ptr(), need - 1
        assert api.lib().sd_kv8_attend(api.C.byref(cache.c), api.C.byref(a), api._stream()) == api.SD_ECAP


KINDS = [(2, 2, 64, 6), (2, 2, 128, 6), (4, 1, 128, 5), (4, 1, 64, 7), (2, 1, 128, 40), (3, 3, 64, 70), (2, 1, 48, 9)]  # heads, cache heads, dim, rows


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv,dim,rows", KINDS)
def test_rows_of_very_different_size(dtype, heads, kv, dim, rows):
    """A row's precision is that of its own elements, whatever the rows beside it hold."""
    ref = kv8ref.Cache([400], kv, dim).fill(dim)
    q = torch.randn(rows, heads, dim, generator=torch.Generator().manual_seed(rows))
    for i, f in ((1, 1e6), (2, 1e-3), (3, 1e30), (4, 1e12), (6, 1e-25), (33, 1e5), (36, 1e35)):
        q[i:i + 1] *= f
    q = q.to(dtype)
    for scale in (dim ** -0.5, -0.2):
        close(run_attend(ref.to_gpu(), q, [330], [rows], scale), kv8ref.attend(ref, q, [(0, 330, 0, rows)], scale))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv,dim,rows", KINDS)
@pytest.mark.parametrize("length", [330, 1])
def test_queries_that_are_not_numbers(dtype, heads, kv, dim, rows, length):
    """A NaN or an infinity makes its own row and head NaN and no other; a row that sees nothing stays zeros."""
    ref = kv8ref.Cache([length + rows, 1], kv, dim).fill(dim)
    q = torch.randn(2 * rows, heads, dim, generator=torch.Generator().manual_seed(rows))
    good = q.clone()
    bad = torch.zeros(2 * rows, heads, dtype=torch.bool)
    for r, h, d, x in ((1, 0, 5, math.nan), (3, heads - 1, dim - 1, math.inf), (4, 0, 0, -math.inf), (rows - 1, 1, dim // 2, math.nan)):
        q[r, h, d], bad[r, h] = x, True
    q[rows:, :, 3] = math.nan
    q, good = q.to(dtype), good.to(dtype)
    out, lse = run_attend(ref.to_gpu(), q, [length, 0], [rows, rows], 0.1, causal=False, ragged=False)
    assert (out[rows:] == 0).all() and (lse[rows:] == -math.inf).all()
    assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all()
    want = kv8ref.attend(ref, good, [(0, length, 0, rows), (1, 0, rows, rows)], 0.1, causal=False)
    live = ~bad
    live[rows:] = False
    close((out[live], lse[live]), tuple(t[live] for t in want))


@pytest.mark.parametrize("rows,max_rows", [(3, 3), (3, 1), (1, 60), (40, 1), (40, 40)])
@pytest.mark.parametrize("dim", [64, 128])
def test_many_sequences(dim, rows, max_rows):
    """150 of them, short and long, in another order, some with no row, one id out of range; max_rows right, too small, too large."""
    rng = np.random.default_rng(rows)
    n = 150
    lens = [int(x) for x in rng.integers(0, 90, n)]
    lens[77], lens[140] = 2500, 1300
    ref = kv8ref.Cache([x + rows for x in lens], 2, dim).fill(4)
    ids = [int(x) for x in rng.permutation(n)]
    counts = [int(x) for x in rng.integers(0, rows + 1, n)]
    for b in (77, 140):
        counts[ids.index(b)] = rows
    lost = ids.index(5)
    counts[lost], ids[lost] = 1, n + 3
    first = starts(counts).tolist()
    q = torch.randn(first[-1], 4, dim, generator=torch.Generator().manual_seed(rows)).to(BF16)
    cache = ref.to_gpu()
    qd, out, lse = q.cuda(), torch.full_like(q, 3.0).cuda(), torch.zeros(first[-1], 4).cuda()
    api.sd_kv8_attend(cache, i32(*lens).cuda(), qd, out, 0.1, row_start=starts(counts).cuda(), max_rows=max_rows, max_len=2500, lse=lse, seq_ids=i32(*ids).cuda())
    assert cache.status.item() == 4
    out, lse = out.cpu(), lse.cpu()
    assert (out[first[lost]] == 3.0).all()
    parts = [(b, lens[b], first[j], counts[j]) for j, b in enumerate(ids) if b < n and (rows < 10 or j % 9 == 0 or b in (77, 140))]
    live = [r for _, _, r0, m in parts for r in range(r0, r0 + m)]
    close((out[live], lse[live]), tuple(t[live] for t in kv8ref.attend(ref, q, parts, 0.1)))


@pytest.mark.parametrize("workspace", [True, False])
def test_one_long_context_among_very_many(workspace):
    """A million tokens beside 65535 short sequences: the tiles of all, each as long as the longest, would not fit 31 bits."""
    n, long = 65536, 1 << 20
    lens = torch.arange(n, dtype=torch.int32) % 3
    at = 40_000
    lens[at] = long - 1
    ref = kv8ref.Cache((lens + 1).tolist(), 1, 64).fill(6)
    cache = ref.to_gpu()
    q = torch.randn(n, 1, 64, generator=torch.Generator().manual_seed(1))
    qd, out, lse = q.cuda(), torch.full_like(q, math.nan).cuda(), torch.full((n, 1), math.nan).cuda()
    if workspace:
        api.sd_kv8_attend(cache, lens.cuda(), qd, out, 0.1, max_len=long - 1, lse=lse)
    else:
        ld = lens.cuda()
        a = api._Kv8Attn(None, ld.data_ptr(), None, n, n, 1, 0, 1, api.SD_FP32, *api._rows3(qd, "q"), *api._rows3(out, "out"), lse.data_ptr(), 0.1,
                         1, 0, 0, None, 0)
        api._check(api.lib().sd_kv8_attend(api.C.byref(cache.c), api.C.byref(a), api._stream()))
    out, lse = out.cpu(), lse.cpu()
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    some = [0, 1, 2, 64, 127, at - 1, at, at + 1, n - 1]
    want = kv8ref.attend(ref, q, [(b, int(lens[b]), b, 1) for b in some], 0.1)
    close((out[some], lse[some]), tuple(t[some] for t in want))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_context_in_the_most_parts(dtype):
    """A token over 200000 others, one cache head: 4096 tiles and more."""
    n = 200_000
    ref = kv8ref.Cache([n + 1], 1, 64).fill(12)
    q = torch.randn(1, 2, 64, generator=torch.Generator().manual_seed(2)).to(dtype)
    close(run_attend(ref.to_gpu(), q, [n], [1], 0.125, ragged=False), kv8ref.attend(ref, q, [(0, n, 0, 1)], 0.125))


@pytest.mark.parametrize("rows,dim", [(3, 128), (5, 64), (100, 128)])
def test_workspace_contents_do_not_matter(rows, dim):
    lens = [4000, 30, 1500]
    ref = kv8ref.Cache([x + rows for x in lens], 2, dim).fill(3)
    cache, ld = ref.to_gpu(), i32(*lens).cuda()
    q = torch.randn(3 * rows, 4, dim, generator=torch.Generator().manual_seed(1)).cuda()
    first = None
    for fill in (0, 1, 127, 255):
        out, lse = torch.zeros_like(q), torch.zeros(3 * rows, 4).cuda()
        a = api._Kv8Attn(None, ld.data_ptr(), None, 3, 3 * rows, 0, max(lens), 4, api.SD_FP32, *api._rows3(q, "q"), *api._rows3(out, "out"), lse.data_ptr(),
                         0.1, 1, 0, 0, None, 0)
        need = api.lib().sd_kv8_attend_workspace(api.C.byref(cache.c), api.C.byref(a))
        assert need > 0
        ws = torch.full((need + 4096,), fill, dtype=torch.uint8).cuda()
        a.workspace, a.workspace_bytes = ws.data_ptr(), need
        api._check(api.lib().sd_kv8_attend(api.C.byref(cache.c), api.C.byref(a), api._stream()))
        assert (ws[need:] == fill).all()
        first = first or (out, lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    show = [0, rows - 1]
    want = kv8ref.attend(ref, q.cpu(), [(b, lens[b] + i, b * rows + i, 1) for b in range(3) for i in show], 0.1)
    live = [b * rows + i for b in range(3) for i in show]
    close((first[0].cpu()[live], first[1].cpu()[live]), tuple(t[live] for t in want))


def test_row_starts_behind_the_rows():
    """Rows that row_start gives a sequence beyond the call's rows are not touched."""
    ref = kv8ref.Cache([100, 100], 1, 64).fill(3)
    q = torch.randn(6, 1, 64, generator=torch.Generator().manual_seed(1))
    for max_rows in (2, 60):
        out = torch.full((40, 1, 64), 3.0).cuda()
        api.sd_kv8_attend(ref.to_gpu(), i32(40, 50).cuda(), q.cuda(), out[:6], 0.1, row_start=i32(0, 4, 100_000).cuda(), max_rows=max_rows, max_len=50)
        assert (out[6:] == 3.0).all()
        want, _, bound, _ = kv8ref.attend(ref, q, [(0, 40, 0, 4), (1, 50, 4, 2)], 0.1)
        assert ((out[:6].cpu().double() - want).abs() <= bound).all()


def test_plain_kernel_agrees():
    """Option force_generic = 2 (attention): the plain kernel, within the same bounds."""
    ref = kv8ref.Cache([300], 2, 128).fill(2)
    q = torch.randn(5, 4, 128, generator=torch.Generator().manual_seed(3))
    want = kv8ref.attend(ref, q, [(0, 290, 0, 5)], 0.1)
    api.set_option("force_generic", 2)
    try:
        close(run_attend(ref.to_gpu(), q, [290], [5], 0.1), want)
    finally:
        api.set_option("force_generic", 0)


# ---------------------------------------------------------------- together, as a step uses them
def step(cache, lens, packed, freq, heads, kv, out, lse, window=0, sinks=0):
    """Turn q and k inside the packed projection, append k and v, attend."""
    rows = packed.shape[0]
    pos = (lens.view(-1, 1) + torch.arange(rows // lens.numel(), device="cuda", dtype=torch.int32)).view(-1)
    qk = packed[:, :heads + kv]
    api.sd_rope(qk, pos, freq, out=qk)
    api.sd_kv8_append(cache, lens, packed[:, heads:heads + kv], packed[:, heads + kv:])
    api.sd_kv8_attend(cache, lens, packed[:, :heads], out, 0.125, max_len=600, lse=lse, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,dim,window", [(F32, 64, 0), (BF16, 128, 0), (BF16, 64, 30)])
def test_a_step_captured_and_replayed(dtype, dim, window):
    """rope, append and attend in one graph on a stream of its own, replayed while the sequences grow, with eager work between."""
    heads, kv, caps = 4, 2, [700, 90]
    g = torch.Generator().manual_seed(dim)
    caches = [api.Kv8Cache.empty(caps, kv, dim) for _ in range(2)]
    lens = i32(500, 3).cuda()
    for c in caches:
        for t, s in ((c.k, c._keep[1]), (c._keep[0], c._keep[2])):
            gg = torch.Generator(device="cuda").manual_seed(1)
            t.copy_(torch.randint(-127, 128, t.shape, generator=gg, device="cuda", dtype=torch.int8))
            s.fill_(0.01)
    freq = torch.from_numpy(api.rope_freqs(dim)).cuda()
    packed, out, lse = torch.zeros(6, heads + 2 * kv, dim, dtype=dtype).cuda(), torch.zeros(6, heads, dim, dtype=dtype).cuda(), torch.zeros(6, heads).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[0], lens, packed.clone(), freq, heads, kv, out.clone(), lse.clone(), window, 2 if window else 0)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(caches[0], lens, packed, freq, heads, kv, out, lse, window, 2 if window else 0)
    for turn in range(5):
        x = torch.randn(packed.shape, generator=g).to(dtype).cuda()
        packed.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        o, l = torch.zeros_like(out), torch.zeros_like(lse)
        y = x.clone()
        step(caches[1], lens, y, freq, heads, kv, o, l, window, 2 if window else 0)
        torch.cuda.synchronize()
        assert torch.equal(packed, y) and torch.equal(out, o) and torch.equal(lse, l), turn
        assert torch.isfinite(o).all() and o.abs().sum() > 0
        lens += i32(3, 1).cuda()                          # a rejected candidate: its rows are written over
    assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0]._keep[2], caches[1]._keep[2])


def test_two_calls_at_once():
    """Two streams, two caches, workspaces of their own: the results of one after the other."""
    refs = [kv8ref.Cache([4000], 1, 128).fill(k) for k in (1, 2)]
    q = torch.randn(2, 4, 128, generator=torch.Generator().manual_seed(3)).cuda()
    caches, lens = [r.to_gpu() for r in refs], i32(3990).cuda()
    alone = [torch.zeros_like(q) for _ in refs]
    for c, o in zip(caches, alone):
        api.sd_kv8_attend(c, lens, q, o, 0.1, max_len=3990)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in refs], [torch.zeros_like(q) for _ in refs]
    for _ in range(20):
        for s, c, o in zip(streams, caches, outs):
            with torch.cuda.stream(s):
                api.sd_kv8_attend(c, lens, q, o, 0.1, max_len=3990)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))


# ---------------------------------------------------------------- the path on a cache in 8 bits
def plain_forward(shape, w, tokens, kv_of, window=0, sinks=0):
    """Logits of every position in float64, with the keys and values that the library's cache holds (kv_of(layer) -> k, v of the
    positions)."""
    f = lambda a: torch.from_numpy(dg.bf16_bits_to_f32(a) if a.dtype == np.uint16 else np.asarray(a)).double()
    H, D, n = shape.n_heads, shape.head_dim, len(tokens)
    x = f(w["embed"])[tokens]
    norm = lambda t, gain: t / torch.sqrt((t * t).mean(-1, keepdim=True) + shape.rms_eps) * f(gain)
    freq, pos = api.rope_freqs(D, base=shape.rope_base), np.arange(n)
    made = []
    for l in range(shape.n_layers):
        a = norm(x, w["norm_attn"][l])
        q, k, v = ((a @ f(w[m][l]).T).view(n, H, D) for m in ("wq", "wk", "wv"))
        q, k = kv8ref.rope(q, pos, freq), kv8ref.rope(k, pos, freq)
        made.append((k, v))
        kc, vc = kv_of(l)
        m = len(kc)
        s = torch.einsum("qhd,khd->hqk", q, kc) / math.sqrt(D)
        t, p = torch.arange(m), torch.arange(n)[:, None]
        hide = t > p
        if window:
            hide |= (t <= p - window) & (t >= sinks)
        o = torch.einsum("hqk,khd->qhd", torch.softmax(s.masked_fill(hide, -math.inf), -1), vc).reshape(n, H * D)
        x = x + o @ f(w["wo"][l]).T
        a = norm(x, w["norm_ffn"][l])
        gate, up = a @ f(w["wgate"][l]).T, a @ f(w["wup"][l]).T
        x = x + (gate * torch.sigmoid(gate) * up) @ f(w["wdown"][l]).T
    return norm(x, w["final_norm"]) @ f(w["lm_head"]).T, made


@pytest.mark.parametrize("name,window,sinks,tol", [("tiny_target", 0, 0, 1e-4), ("tiny_target", 24, 3, 1e-4), ("tiny_target_bf16", 0, 0, 2e-2),
                                                   ("small_target_bf16", 0, 0, 2e-2), ("small_target_bf16", 24, 3, 2e-2)])
def test_path_on_an_8_bit_cache(name, window, sinks, tol):
    """Prefill, verify, a second verify after a rollback: logits against float64 over the keys and values the cache holds (tol: the
    path's own bounds on logits, relative to a row's largest), and those against quantised projections."""
    shape = dg.SHAPES[name]
    w = dg.make_weights(shape, 21)
    m = api.Model(shape, w, max_rows=64, max_pos=256)
    ctx = api.Context([200, 128])
    ctx.attach_kv8(m, window, sinks)
    rng = np.random.default_rng(5)
    seqs = [rng.integers(0, shape.vocab, n).tolist() for n in (101, 38)]
    ctx.set_tokens(seqs)
    api.sd_prefill(m, ctx, None, 2, 100)
    gamma = 4
    for turn in range(2):
        cand = torch.from_numpy(rng.integers(0, shape.vocab, (2, gamma)).astype(np.int32)).cuda()
        na, nx = torch.zeros(2, dtype=torch.int32).cuda(), torch.zeros(2, dtype=torch.int32).cuda()
        api.sd_verify(m, ctx, None, 2, gamma, 0.0, cand, None, None, na, nx, commit=False)
        logits = m.last_logits().cpu().view(2, gamma + 1, -1).double()
        q_read = m.debug_read("q", 2 * (gamma + 1))
        assert np.isfinite(q_read).all() and np.abs(q_read).max() > 0
        for b in range(2):
            tokens = seqs[b] + cand[b].tolist()
            n = len(tokens)
            held = [ctx.get_kv(m, l, b, n) for l in range(shape.n_layers)]
            vals = [tuple(torch.from_numpy(dg.bf16_bits_to_f32(a) if a.dtype == np.uint16 else a).double() for a in kv) for kv in held]
            want, made = plain_forward(shape, w, tokens, lambda l: vals[l], window, sinks)
            want = want[-(gamma + 1):]
            err = (logits[b] - want).abs().amax(-1) / want.abs().amax(-1)
            assert (err < tol).all(), (b, err)
            for l in range(shape.n_layers):               # the cache: within half a scale, the read's rounding and the path's error
                for x, y in zip(made[l], vals[l]):
                    amax = x.abs().amax(-1, keepdim=True)
                    assert ((x - y).abs() <= amax * (0.5 / 127 + tol / 4 + (2 ** -8 if shape.dtype == dg.BF16 else 0))).all(), (b, l)
        seqs = [s + [int(c[0]), 7] for s, c in zip(seqs, cand.cpu())]      # one candidate accepted, then token 7
        api.sd_commit(ctx, None, 2, gamma, cand, torch.ones_like(na), torch.full_like(nx, 7))
    ctx.sync(m)


def test_speculation_on_8_bit_caches_follows_plain_decoding():
    """Greedy draft / verify / commit with target and draft on 8-bit caches gives the tokens of the target decoding alone on one: a
    token's codes do not depend on the candidates that were tried before it."""
    shape, dshape = dg.SHAPES["tiny_target"], dg.SHAPES["tiny_draft"]
    w = dg.make_weights(shape, 31)
    target, draft = api.Model(shape, w, max_rows=64, max_pos=256), api.Model(dshape, dg.make_weights(dshape, 32), max_rows=64, max_pos=256)
    rng = np.random.default_rng(6)
    prompts = [rng.integers(0, shape.vocab, n).tolist() for n in (33, 50)]

    def decode(gamma, steps):
        ctx = api.Context([200, 200])
        ctx.attach_kv8(target)
        ctx.attach_kv8(draft, 32, 2)
        ctx.set_tokens(prompts)
        api.sd_prefill(target, ctx, None, 2, 50)
        api.sd_prefill(draft, ctx, None, 2, 50)
        na, nx = torch.zeros(2, dtype=torch.int32).cuda(), torch.zeros(2, dtype=torch.int32).cuda()
        cand = torch.zeros(2, max(gamma, 1), dtype=torch.int32).cuda()
        for _ in range(steps):
            if gamma:
                api.sd_draft(draft, ctx, None, 2, gamma, 0.0, None, cand, None)
            api.sd_verify(target, ctx, None, 2, gamma, 0.0, cand if gamma else None, None, None, na, nx, commit=True)
        ctx.sync(target)
        return [ctx.get_tokens(b).tolist() for b in range(2)]
    alone, spec = decode(0, 40), decode(3, 20)
    for a, s in zip(alone, spec):
        n = min(len(a), len(s))
        assert n > 60 - 10 and a[:n] == s[:n]


def test_adapters_on_an_8_bit_cache():
    """Sequences of one batch with different low-rank adapters: logits against the merged weights in float64 over the keys and values the
    cache holds."""
    shape = dg.SHAPES["tiny_target"]
    w = dg.make_weights(shape, 41)
    lora, scale, gamma = dg.make_lora(shape, 42, n_adapters=2, rank=4, std_a=0.05, std_b=0.05), 2.0, 3
    m = api.Model(shape, w, max_rows=64, max_pos=128)
    m.set_lora(lora, scale)
    ctx = api.Context([100, 100, 60])
    ctx.attach_kv8(m)
    ids = [1, -1, 0]
    ctx.set_adapters(m, ids)
    rng = np.random.default_rng(7)
    seqs = [rng.integers(0, shape.vocab, n).tolist() for n in (70, 33, 20)]
    ctx.set_tokens(seqs)
    api.sd_prefill(m, ctx, None, 3, 69)
    cand = torch.from_numpy(rng.integers(0, shape.vocab, (3, gamma)).astype(np.int32)).cuda()
    na, nx = torch.zeros(3, dtype=torch.int32).cuda(), torch.zeros(3, dtype=torch.int32).cuda()
    api.sd_verify(m, ctx, None, 3, gamma, 0.0, cand, None, None, na, nx, commit=False)
    logits = m.last_logits().cpu().view(3, gamma + 1, -1).double()
    for b, a in enumerate(ids):
        wm = dict(w)
        if a >= 0:
            for pnm, key in (("q", "wq"), ("k", "wk"), ("v", "wv"), ("o", "wo")):
                wm[key] = [w[key][l].astype(np.float64) + scale * lora["b_" + pnm][l][a].astype(np.float64) @ lora["a_" + pnm][l][a].astype(np.float64)
                           for l in range(shape.n_layers)]
        tokens = seqs[b] + cand[b].tolist()
        vals = [tuple(torch.from_numpy(x).double() for x in ctx.get_kv(m, l, b, len(tokens))) for l in range(shape.n_layers)]
        want, made = plain_forward(shape, wm, tokens, lambda l: vals[l])
        err = (logits[b] - want[-(gamma + 1):]).abs().amax(-1) / want[-(gamma + 1):].abs().amax(-1)
        assert (err < 1e-4).all(), (b, err)               # (the path's bound on fp32 logits)
        for x, y in zip(made[0], vals[0]):
            assert ((x - y).abs() <= x.abs().amax(-1, keepdim=True) * (0.5 / 127 + 1e-4 / 4)).all()
    ctx.sync(m)


@pytest.mark.parametrize("name,dname", [("tiny_target", "tiny_draft"), ("small_target_bf16", "small_draft_bf16")])
def test_path_on_8_bit_caches_captured_and_replayed(name, dname):
    """A committing greedy step in a graph, captured at 20 tokens and replayed far past that: the tokens of the same steps launched eagerly."""
    shape, dshape = dg.SHAPES[name], dg.SHAPES[dname]
    target, draft = (api.Model(s, dg.make_weights(s, 51), max_rows=64, max_pos=1600) for s in (shape, dshape))
    prompt, gamma, steps = [np.random.default_rng(8).integers(0, shape.vocab, n).tolist() for n in (20, 1400)], 3, 24
    cand = torch.zeros(2, gamma, dtype=torch.int32).cuda()
    na, nx = torch.zeros(2, dtype=torch.int32).cuda(), torch.zeros(2, dtype=torch.int32).cuda()

    def new_ctx():
        c = api.Context([160, 1560])
        c.attach_kv8(target)
        c.attach_kv8(draft, 16, 2)
        c.set_tokens(prompt)
        api.sd_prefill(target, c, None, 2, 1399)
        api.sd_prefill(draft, c, None, 2, 1399)
        return c

    def step(c):
        api.sd_draft(draft, c, None, 2, gamma, 0.0, None, cand, None)
        api.sd_verify(target, c, None, 2, gamma, 0.0, cand, None, None, na, nx, commit=True)

    eager = new_ctx()
    for _ in range(steps):
        step(eager)
    eager.sync()
    want = [list(eager.get_tokens(b)) for b in range(2)]
    ctx = new_ctx()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(ctx)
    torch.cuda.synchronize()
    for k in range(steps):
        graph.replay()
        torch.cuda.synchronize()
    ctx.sync()
    assert [list(ctx.get_tokens(b)) for b in range(2)] == want and len(want[0]) >= 20 + steps


def test_attach_and_cache_rows():
    shape = dg.SHAPES["small_target_bf16"]
    m = api.Model(shape, dg.make_weights(shape, 3), max_rows=32, max_pos=128)
    ctx, plain = api.Context([64, 64]), api.Context([64, 64])
    ctx.attach_kv8(m)
    ctx.attach_kv8(m)                                     # the same form again: fine
    plain.attach(m)
    for bad in (lambda: ctx.attach_kv8(m, 8), lambda: plain.attach_kv8(m), lambda: api.Context([64]).attach_kv8(m, 0, 3),
                lambda: api.Context([64]).attach_kv8(m, -1), lambda: ctx.attach(m)):
        with pytest.raises(api.SdError):
            bad()
    rows = [dg.f32_to_bf16_bits(np.random.default_rng(k).standard_normal((50, shape.n_heads, shape.head_dim)).astype(np.float32)) for k in range(2)]
    for c in (ctx, plain):
        c.set_kv(m, 1, 1, *rows)
        assert c.sync(m)[1].tolist() == [0, 50]
    for got, src in zip(plain.get_kv(m, 1, 1, 50), rows):
        assert np.array_equal(got, src)
    for got, src in zip(ctx.get_kv(m, 1, 1, 50), rows):
        codes, s = kv8ref.quantise(torch.from_numpy(dg.bf16_bits_to_f32(src)))
        assert np.array_equal(got, dg.f32_to_bf16_bits((codes.float() * s[..., None]).numpy()))
    assert not np.any(ctx.get_kv(m, 0, 1, 50)[0]) and not np.any(ctx.get_kv(m, 1, 0, 64)[0])     # other layers and sequences
    with pytest.raises(api.SdError):
        ctx.get_kv(m, 2, 0, 1)
    with pytest.raises(api.SdError):
        ctx.get_kv(m, 0, 0, 65)
