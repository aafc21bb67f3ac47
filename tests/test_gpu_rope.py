"""sd_rope against the rotation in 64 bits."""
import numpy as np
import pytest
import torch

import kv8ref
from paper_2505_08600_amd import api

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def check(y, want, x, gain=1.0):
    """The angle's fraction of a turn is rounded to 24 bits (2 pi 2^-26 of an angle), sine and cosine to a few 2^-24, products and
    the sum to 2^-24 each: 2^-20 of |a| + |b| times the gain is above all of it together; then the half step of the type."""
    y, x = y.double().cpu(), x.double()
    mag = x.abs().amax(-1, keepdim=True) * 2 * abs(gain)
    bound = 2.0 ** -20 * mag + HALF[check.dtype] * want.abs()
    bad = (y - want).abs() > bound
    assert not bad.any(), ((y - want).abs() / bound).max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,heads,dim,rot,inter", [(1, 1, 64, 64, False), (6, 64, 128, 128, False), (77, 3, 64, 32, True), (1003, 24, 64, 32, False),
                                                      (5, 7, 80, 40, True), (9, 2, 6, 2, False), (9, 2, 6, 4, True), (33, 5, 512, 512, True),
                                                      (2500, 8, 128, 64, True), (4, 1, 2, 2, True)])
def test_rotation(dtype, rows, heads, dim, rot, inter):
    print(f"rope {dtype} {rows} x {heads} x {dim}, {rot} turning, interleaved {inter}", flush=True)
    check.dtype = dtype
    g = torch.Generator().manual_seed(rows * 131 + dim)
    x = torch.randn(rows, heads, dim, generator=g).to(dtype)
    pos = torch.randint(0, 5000, (rows,), generator=g, dtype=torch.int32)
    f = api.rope_freqs(rot)
    for inverse, gain in ((False, 1.0), (True, 1.25)):
        y = api.sd_rope(x.cuda(), pos.cuda(), torch.from_numpy(f).cuda(), interleaved=inter, inverse=inverse, gain=gain)
        check(y, kv8ref.rope(x, pos.numpy(), f, inter, inverse, gain), x, gain)
        assert torch.equal(y[..., rot:].cpu(), x[..., rot:])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_in_place_packed_and_unaligned(dtype):
    check.dtype = dtype
    g = torch.Generator().manual_seed(5)
    rows, f = 19, api.rope_freqs(48)
    pos = torch.arange(100, 100 + rows, dtype=torch.int32)
    fd, pd = torch.from_numpy(f).cuda(), pos.cuda()
    for shift, width in ((0, 64), (1, 64), (0, 65), (3, 67)):      # element offset of the buffer, row pitch of a head
        buf = torch.randn(shift + rows * 6 * width, generator=g).to(dtype)
        view = lambda b: b[shift:].view(rows, 6, width)
        want = kv8ref.rope(view(buf)[:, :4, :64], pos.numpy(), f, False)
        dev = buf.cuda()
        x = view(dev)[:, :4, :64]
        assert api.sd_rope(x, pd, fd, out=x) is x
        check(x, want, view(buf)[:, :4, :64])
        rest, was = dev.cpu(), buf.clone()
        view(rest)[:, :4, :48] = 0
        view(was)[:, :4, :48] = 0
        assert torch.equal(rest, was)                              # nothing else has moved
        out = torch.full((4, rows, 64), 7.0, dtype=dtype).cuda().transpose(0, 1)   # heads outside rows
        api.sd_rope(view(buf.cuda())[:, :4, :64], pd, fd, out=out)
        check(out, want, view(buf)[:, :4, :64])


def test_far_and_negative_positions():
    check.dtype = torch.float32
    g = torch.Generator().manual_seed(9)
    pos = torch.tensor([0, -1, 131071, 1 << 20, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    x, f = torch.randn(6, 2, 128, generator=g), api.rope_freqs(128)
    y = api.sd_rope(x.cuda(), pos.cuda(), torch.from_numpy(f).cuda())
    check(y, kv8ref.rope(x, pos.numpy(), f), x)


def test_gradient_is_the_inverse_and_agrees_with_differences():
    check.dtype = torch.float32
    g = torch.Generator().manual_seed(3)
    rows, heads, dim, rot = 7, 3, 64, 32
    x, w = torch.randn(rows, heads, dim, generator=g), torch.randn(rows, heads, dim, generator=g)
    pos, f, gain = torch.arange(40, 47, dtype=torch.int32), api.rope_freqs(rot), 1.5
    run = lambda t, **kw: api.sd_rope(t.cuda(), pos.cuda(), torch.from_numpy(f).cuda(), gain=gain, **kw).cpu()
    grad = run(w, inverse=True)
    # d/dx sum(w . rope(x)) along a direction e: the map is linear, so a whole step is as exact as the sums
    for k in range(4):
        e = torch.zeros_like(x)
        e[k % rows, k % heads, 5 * k] = 1.0
        diff = ((run(x + e) - run(x)).double() * w.double()).sum()
        # each of the at most two outputs that move is off by 2^-20 of its inputs' size (above), times |w|
        assert abs(diff - (grad.double() * e.double()).sum()) < 2 ** -18 * gain * w.abs().max() * (x.abs().max() + 1) * 4
    check(grad, kv8ref.rope(w, pos.numpy(), f, inverse=True, gain=gain), w, gain)


def test_model_positions_follow_the_scaling():
    """sd_model_set_rope: keys that a prefill appends are turned by the scaled angles."""
    from paper_2505_08600_amd import datagen as dg
    shape = dg.SHAPES["tiny_draft"]
    m = api.Model(shape, dg.make_weights(shape, 11), max_rows=64, max_pos=128)
    ctx = api.Context([64])
    ctx.attach(m)
    tokens = list(range(5, 25))

    def keys():
        ctx.set_tokens([tokens])
        api.sd_prefill(m, ctx, None, 1, len(tokens))
        return ctx.get_kv(m, 0, 0, len(tokens) - 1)[0]
    plain = keys()
    m.set_rope("linear", factor=4.0, gain=1.0)
    scaled = keys()
    m.set_rope("plain")
    assert np.array_equal(keys(), plain)
    f0, f1 = api.rope_freqs(shape.head_dim), api.rope_freqs(shape.head_dim, "linear", factor=4.0)
    pos = np.arange(len(tokens) - 1)
    unturned = kv8ref.rope(torch.from_numpy(plain), pos, f0, inverse=True)
    want = kv8ref.rope(unturned, pos, f1).numpy()
    # table, products and sums in 32 bits, once forward and once back: 8 steps of 2^-24 of the largest element
    assert np.abs(scaled - want).max() < 2 ** -20 * np.abs(plain).max() * 2
    with pytest.raises(api.SdError):
        api._check(api.lib().sd_model_set_rope(m.h, api.C.byref(api._RopeConfig(32, 0, 1e4, 1, 1, 4, 8192)), 1.0))
