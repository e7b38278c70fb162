"""Rotary positions and page plans on the GPU against their plain statements."""
import numpy as np
import pytest
import torch

import _cache4 as plain
import paper_2606_10944_b200 as elm

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _check_rotation(got, x, pos, rope, layout, inverse, dtype):
    """Cosine, sine, two products and a sum, each within half a step of fp32, then the storage type's half step."""
    freq = np.array(rope.inv_freq)
    xf = x.double().cpu().numpy()
    ref = plain.rotate(xf, pos, freq, rope.scale, layout, inverse)
    r = 2 * len(freq)
    size = np.abs(xf).copy()
    a, b = (size[..., :r // 2], size[..., r // 2:r]) if layout == "halves" else (size[..., 0:r:2], size[..., 1:r:2])
    both = a + b
    if layout == "halves":
        size[..., :r // 2] = size[..., r // 2:r] = both
    else:
        size[..., 0:r:2] = size[..., 1:r:2] = both
    tol = 4 * 2.0 ** -24 * size * abs(rope.scale) + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * np.abs(ref) + 1e-38
    tol[..., r:] = 0
    err = np.abs(got.double().cpu().numpy() - ref)
    assert (err <= tol).all(), float((err - tol).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("B,H,n,d,rotary", [(1, 1, 1, 64, 64), (2, 3, 17, 128, 128), (1, 5, 33, 128, 64), (3, 2, 7, 64, 48), (2, 2, 9, 64, 6),
                                            (1, 2, 5, 10, 2), (1, 1, 3, 256, 256), (2, 1, 11, 96, 96), (4, 32, 300, 128, 128), (1, 300, 3, 128, 128),
                                            (2, 70, 2, 256, 32)])
def test_rotation(dtype, layout, B, H, n, d, rotary):
    g = torch.Generator().manual_seed(B * 1000 + d + rotary)
    x = torch.randn(B, H, n, d, generator=g).to(DTYPES[dtype]).cuda()
    pos = torch.randint(-5, 200000, (B, n), generator=g, dtype=torch.int32)
    rope = elm.Rope(rotary, layout=layout)
    for inverse in (False, True):
        got = elm.rope(x, pos.cuda(), rope, inverse=inverse)
        _check_rotation(got, x, pos.numpy()[:, None], rope, layout, inverse, x.dtype)


@pytest.mark.parametrize("scaling,kw", [("linear", dict(factor=4.0)), ("base", dict(factor=8.0)), ("ramp", dict(factor=16.0, original=4096)),
                                        ("smooth", dict(factor=8.0, original=8192, low=1.0, high=4.0))])
def test_far_positions(scaling, kw):
    """The largest positions of an int32, where an angle in fp32 has lost every bit."""
    rope = elm.Rope(128, scaling=scaling, **kw)
    x = torch.randn(1, 2, 6, 128, generator=torch.Generator().manual_seed(2)).cuda()
    pos = torch.tensor([[0, 1, 2 ** 31 - 1, -2 ** 31, 131071, 10 ** 9]], dtype=torch.int32)
    got = elm.rope(x, pos.cuda(), rope)
    # (an angle of 2^31 radians is known to 2^-22 in double: the statement's own angle is formed in long double from double
    # frequencies, which the library takes exactly)
    _check_rotation(got, x, pos.numpy()[:, None], rope, "halves", False, x.dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("rotary", [128, 96, 34])
def test_strided_in_place_and_first_position(dtype, layout, rotary):
    rope = elm.Rope(rotary, layout=layout)
    wide = torch.randn(2, 21, 7, 128, generator=torch.Generator().manual_seed(4)).to(DTYPES[dtype]).cuda()
    x = wide[:, :, 1:5].transpose(1, 2)                       # [B, H, n, d] inside [B, n, heads, d]
    ref = elm.rope(x.contiguous(), 77, rope)
    assert torch.equal(elm.rope(x, 77, rope), ref)
    pos = (torch.arange(21, dtype=torch.int32) + 77).expand(2, 21).contiguous().cuda()
    assert torch.equal(elm.rope(x, pos, rope), ref)
    before = wide.clone()
    out = torch.empty_like(wide)[:, :, 1:5].transpose(1, 2)
    assert torch.equal(elm.rope(x, 77, rope, out=out), ref) and torch.equal(wide, before)
    assert elm.rope(x, 77, rope, out=x) is x
    assert torch.equal(x, ref)
    assert torch.equal(wide[:, :, 0], before[:, :, 0]) and torch.equal(wide[:, :, 5:], before[:, :, 5:])
    # rows that start on odd addresses
    odd = torch.randn(1, 3, 5, 129, generator=torch.Generator().manual_seed(5)).to(DTYPES[dtype]).cuda()[..., 1:]
    assert torch.equal(elm.rope(odd, 5, rope), elm.rope(odd.contiguous(), 5, rope))


def test_broadcast_heads_read_once_each():
    rope = elm.Rope(64)
    x = torch.randn(2, 1, 9, 64, generator=torch.Generator().manual_seed(6)).cuda()
    assert torch.equal(elm.rope(x.expand(2, 4, 9, 64), 3, rope), elm.rope(x, 3, rope).expand(2, 4, 9, 64))
    one = torch.randn(64, generator=torch.Generator().manual_seed(7)).cuda().expand(2, 3, 4, 64)
    assert torch.equal(elm.rope(one, 3, rope), elm.rope(one.contiguous(), 3, rope))


def test_inverse_is_the_gradient():
    """<rope(x), y> = <x, inverse(y)>, and a difference of the rotation along a direction is the rotation of it."""
    rope = elm.Rope(128, scaling="ramp", factor=4.0, original=1000)
    g = torch.Generator().manual_seed(8)
    x, y = torch.randn(2, 4, 50, 128, generator=g).cuda(), torch.randn(2, 4, 50, 128, generator=g).cuda()
    fx, by = elm.rope(x, 9, rope), elm.rope(y, 9, rope, inverse=True)
    left, right = (fx.double() * y.double()).sum().item(), (x.double() * by.double()).sum().item()
    # 51200 products of numbers off by at most 4 half steps of (|a| + |b|) scale
    tol = 4 * 2.0 ** -24 * rope.scale * ((x.double().abs().sum() * 2 * y.abs().max()) + (y.double().abs().sum() * 2 * x.abs().max())).item()
    assert abs(left - right) <= tol
    h = 2.0 ** -6
    diff = (elm.rope(x + h * y, 9, rope).double() - elm.rope(x - h * y, 9, rope).double()) / (2 * h)
    err = (diff - elm.rope(y, 9, rope).double()).abs().max().item()
    size = (x.abs().max() + h * y.abs().max()).item() * 2 * rope.scale
    assert err <= (2 * (4 + 1) * 2.0 ** -24 * size) / (2 * h) + 5 * 2.0 ** -24 * size


def test_first_position_of_any_size():
    """A first position past 32 bits turns by the angle modulo a turn: a frequency of a quarter turn a position comes back every four."""
    rope = elm.Rope(64)
    rope._freq[:] = [np.pi / 2] * 32
    x = torch.randn(1, 2, 8, 64, generator=torch.Generator().manual_seed(3)).cuda()
    near, far = elm.rope(x, 1, rope), elm.rope(x, 2 ** 45 + 1, rope)
    # (the frequency is off by 2^-53 of a radian: 2^-8 radians at 2^45)
    assert (near - far).abs().max().item() <= 2 * x.abs().max().item() * 2.0 ** -7
    assert torch.equal(elm.rope(x, -7, rope, inverse=True)[:, :, 0], elm.rope(x, 7, rope)[:, :, 0])


def test_rope_other_stream_and_graph():
    rope = elm.Rope(128)
    x = torch.randn(1, 8, 64, 128, generator=torch.Generator().manual_seed(9)).cuda()
    ref = elm.rope(x, 5, rope)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = elm.rope(x, 5, rope)
    s.synchronize()
    assert torch.equal(got, ref)
    out, pos = torch.empty_like(x), torch.zeros(1, 64, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        elm.rope(x, pos, rope, out=out)
    pos.copy_(torch.arange(64, dtype=torch.int32)[None] + 5)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ref)


# ------------------------------------------------------------------------------------------------
def _ints(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def _plan_both(table, length, n_new, free, count, page, T):
    want = plain.plan(table, length, n_new, free, count, page, T)
    tab = _ints(table)
    got = elm.page_plan(tab, _ints(length), _ints(n_new), _ints(free), _ints([count]), page, T)
    out = [got.start, got.length, got.free_count, got.cu, got.positions, got.slots, tab]
    for name, a, b in zip(("start", "length", "free", "cu", "positions", "slots", "table"), out, want):
        assert np.array_equal(a.cpu().numpy().reshape(-1), np.asarray(b).reshape(-1)), name
    return got, tab


@pytest.mark.parametrize("B", [1, 2, 33, 1024, 1025, 5000, 65536])
@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("most,share", [(1, 1.0), (3, 0.5), (100, 0.7)])
def test_plan(B, page, most, share):
    r = np.random.default_rng(B + page + most)
    max_pages = 9
    length = r.integers(0, max_pages * page // 2, B)
    n_new = r.integers(0, most + 1, B)
    if B > 4:
        n_new[r.integers(0, B, B // 5)] = 0
        length[r.integers(0, B, B // 5)] = 0
        length[0] = max_pages * page                          # full: only a step without tokens fits
        length[1] = -3
        n_new[2] = -1
    held = np.clip(-(-length // page), 0, None)
    need = (-(-(length + np.clip(n_new, 0, None)) // page) - held).clip(0).sum()
    pages = r.permutation(int(held.sum() + need + 5))
    table = np.full((B, max_pages), -1)
    at = 0
    for b in range(B):
        table[b, :held[b]] = pages[at:at + held[b]]
        at += held[b]
    free = pages[at:]
    T = int(np.clip(n_new, 0, None).sum())
    for tokens in {T, T + 3, max(0, T - 2)}:
        _plan_both(table, length, n_new, free, int(len(free) * share), page, tokens)
    _plan_both(table, length, n_new, free, len(free) + 100, page, T)      # a count beyond the list


def test_plan_of_long_prompts():
    length, n_new = np.array([5, 0, 70000, 0, 0, 3]), np.array([20000, 0, 1, 0, 65536, 0])
    held = -(-length // 16)
    table = np.full((6, 8192), -1)
    pages = np.random.default_rng(1).permutation(60000)
    at = 0
    for b in range(6):
        table[b, :held[b]] = pages[at:at + held[b]]
        at += held[b]
    for count in (len(pages) - at, 1300, 1, 0):
        _plan_both(table, length, n_new, pages[at:], count, 16, int(n_new.sum()) + 1000)


def test_plan_in_place_and_release():
    B, page, max_pages = 40, 16, 20
    r = np.random.default_rng(3)
    table, length = np.full((B, max_pages), -1), np.zeros(B, np.int64)
    free = r.permutation(500)
    count = 500
    t, n, f, c = _ints(table), _ints(length), _ints(free), _ints([count])
    for step in range(6):
        n_new = r.integers(0, 60, B)
        start, length, count, cu, pos, slot, table = plain.plan(table, length, n_new, free, count, page, int(n_new.sum()))
        got = elm.page_plan(t, n, _ints(n_new), f, c, page, int(n_new.sum()), length_out=n, free_count_out=c)
        assert np.array_equal(got.slots.cpu().numpy(), slot) and np.array_equal(got.start.cpu().numpy(), start)
        done = r.random(B) < 0.3
        free = free.copy()
        for b in np.nonzero(done)[0]:
            for i in range(-(-length[b] // page)):
                free[count] = table[b, i]
                count += 1
                table[b, i] = -1
            length[b] = 0
        elm.page_release(t, n, _ints(done.astype(np.int32)), f, c, page)
        assert np.array_equal(t.cpu().numpy(), table) and np.array_equal(n.cpu().numpy(), length)
        assert int(c.item()) == count and np.array_equal(f.cpu().numpy()[:count], free[:count])
    assert sorted(free[:count].tolist() + table[table >= 0].tolist()) == list(range(500))


def test_release_without_room_and_bad_entries():
    t, n, c = _ints([[3, -1, 7, 9], [1, 2, -1, -1]]), _ints([50, 20]), _ints([1])
    f = _ints([5, 0, 0])
    elm.page_release(t, n, _ints([1, 1]), f, c, 16)
    assert f.tolist() == [5, 3, 7] and c.item() == 3 and n.tolist() == [0, 0]
    assert t.tolist() == [[-1, -1, -1, -1], [-1, -1, -1, -1]]


def test_plan_captured():
    t, n, f, c = _ints(np.full((3, 4), -1)), _ints([0, 0, 0]), _ints(np.arange(12)), _ints([12])
    new = _ints([1, 1, 1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = elm.page_plan(t, n, new, f, c, 16, 3, length_out=n, free_count_out=c)
    for step in range(33):
        graph.replay()
    torch.cuda.synchronize()
    assert n.tolist() == [33, 33, 33] and c.item() == 3 and r.positions.tolist() == [32, 32, 32]
    assert sorted(t.cpu()[:, :3].reshape(-1).tolist()) == list(range(3, 12))


@pytest.mark.parametrize("tokens", [40, 5000])                # one launch, two launches
@pytest.mark.parametrize("page", [16, 32, 1024])
def test_pages_that_no_pool_holds(page, tokens):
    """Page numbers whose rows' numbers would pass 2^31 - 1, in a table and among the free ones: their tokens are in no slot, instead of in that of
    another page modulo 2^32; given back, they are dropped.  The last page that a pool can hold is one."""
    most = (2 ** 31 - 1) // page                              # pages of the largest pool
    bad = [most, most + 1, 2 ** 32 // page // 2, 2 ** 31 - 1]
    if page == 32:
        bad += [1 << 27, (1 << 27) + 1]
    table = np.full((len(bad) + 2, 9), -1)
    table[:len(bad), 0] = bad
    table[len(bad), 0] = most - 1
    length = np.array([5] * len(bad) + [7, 0])
    n_new = np.array([3] * len(bad) + [2, 3])
    free = np.array([4, bad[-1], bad[0]])                     # (the last request's page)
    t, n, f, c = _ints(table), _ints(length), _ints(free), _ints([3])
    got = elm.page_plan(t, n, _ints(n_new), f, c, page, tokens, length_out=n, free_count_out=c)
    slots = got.slots.tolist()
    at = 3 * len(bad)
    assert slots[:at] == [-1] * at and got.positions[:at].tolist() == [5, 6, 7] * len(bad)
    assert slots[at:at + 2] == [(most - 1) * page + 7, (most - 1) * page + 8] and set(slots[at + 2:]) == {-1}
    assert c.item() == 2
    # nothing is stored through them
    pool = torch.full((4, 1, page, 80), 0xa5, dtype=torch.uint8, device="cuda")
    x = torch.randn(tokens, 1, 64, generator=torch.Generator().manual_seed(1)).cuda()
    elm.cache4_append(pool, x, x, got.slots)
    assert (pool == 0xa5).all()
    elm.page_release(t, n, _ints([1] * len(table)), f, c, page)
    assert c.item() == 3 and f.tolist() == [4, bad[-1], most - 1] and (t == -1).all() and (n == 0).all()


def test_plan_of_as_many_places_as_there_can_be():
    """A step of 2^31 - 1 places (17 GB of results): tokens in the first of them, all others marked."""
    most = 2 ** 31 - 1
    t, n = _ints(np.full((2, 400), -1)), _ints([3, 0])
    t[0, 0] = 7
    got = elm.page_plan(t, n, _ints([4, 6000]), _ints(np.arange(400) + 10), _ints([400]), 16, most)
    assert got.cu.tolist() == [0, 4, 6004] and got.start.tolist() == [3, 0] and got.free_count.item() == 400 - 375
    assert got.positions[:6004].tolist() == [3, 4, 5, 6] + list(range(6000))
    assert got.slots[:4].tolist() == [7 * 16 + i for i in (3, 4, 5, 6)]
    table = t[1].tolist()
    assert got.slots[4:6004].tolist() == [table[i // 16] * 16 + i % 16 for i in range(6000)]
    for x in (got.positions, got.slots):
        assert all(bool((part == -1).all()) for part in x[6004:].split(1 << 28))


@pytest.mark.parametrize("eighth", range(8))
def test_angles_next_to_the_eighths_of_a_turn(eighth):
    """Positions of a frequency of 2 pi / 4096: the angle's nearest quarter changes at its eighths, and at half a turn the fraction's sign does."""
    rope = elm.Rope(64)
    rope._freq[:] = [2 * np.pi / 4096] * 32
    x = torch.randn(1, 1, 9, 64, generator=torch.Generator().manual_seed(3)).cuda()
    for turns in (0, 1, -3, 1 << 40):
        got = elm.rope(x, 4096 * turns + 512 * eighth - 4, rope)
        # (the frequency is a double off by 2^-53 of itself, and so is an angle)
        pos = np.arange(9) + 512 * eighth - 4
        freq = np.array([2 * np.pi / 4096] * 32)
        ref = plain.rotate(x.double().cpu().numpy(), pos, freq)
        a = np.abs(x.double().cpu().numpy())
        size = np.concatenate([a[..., :32] + a[..., 32:]] * 2, -1)
        off = 4 * 2.0 ** -24 + abs(turns) * 2 * np.pi * 2.0 ** -53
        assert (np.abs(got.double().cpu().numpy() - ref) <= off * size + 2.0 ** -24 * np.abs(ref)).all(), turns


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("inverse", [False, True])
def test_gradient_by_autograd(dtype, layout, inverse):
    """Where X requires a gradient the result has it: the transposed rotation of the incoming one, against the 64-bit statement and
    against differences; through strided, broadcast and other-stream uses, and again through itself."""
    rope = elm.Rope(96, layout=layout, scaling="ramp", factor=4.0, original=1000)
    g = torch.Generator().manual_seed(11)
    wide = torch.randn(2, 13, 7, 128, generator=g).to(DTYPES[dtype]).cuda().requires_grad_()
    x = wide[:, :, 1:5].transpose(1, 2)
    pos = torch.randint(0, 5000, (2, 13), generator=g, dtype=torch.int32).cuda()
    y = elm.rope(x, pos, rope, inverse=inverse)
    with torch.no_grad():
        assert torch.equal(y, elm.rope(x, pos, rope, inverse=inverse))
    assert y.requires_grad
    dy = torch.randn(y.shape, generator=g).to(DTYPES[dtype]).cuda()
    got, = torch.autograd.grad(y, wide, dy, retain_graph=True)
    assert (got[:, :, :1] == 0).all() and (got[:, :, 5:] == 0).all()
    _check_rotation(got[:, :, 1:5].transpose(1, 2), dy, pos.cpu().numpy()[:, None], rope, layout, not inverse, wide.dtype)
    # an incoming gradient that is one number, one with the numbers of a head apart, and one taken on another stream
    one, = torch.autograd.grad(y.sum(), wide, retain_graph=True)
    ref, = torch.autograd.grad(y, wide, torch.ones_like(y), retain_graph=True)
    assert torch.equal(one, ref)
    apart, = torch.autograd.grad(y, wide, dy.transpose(2, 3).contiguous().transpose(2, 3), retain_graph=True)
    assert torch.equal(apart, got)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other, = torch.autograd.grad(elm.rope(x, pos, rope, inverse=inverse), wide, dy)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(other, got)
    # the gradient's own gradient is the rotation
    v = dy.clone().requires_grad_()
    back, = torch.autograd.grad(y, wide, v, create_graph=True)
    u = torch.randn(wide.shape, generator=g).to(DTYPES[dtype]).cuda()
    again, = torch.autograd.grad(back, v, u)
    with torch.no_grad():
        assert torch.equal(again, elm.rope(u[:, :, 1:5].transpose(1, 2), pos, rope, inverse=inverse))


def test_gradient_against_differences():
    rope = elm.Rope(64, scaling="ramp", factor=4.0, original=1000)
    g = torch.Generator().manual_seed(12)
    x = torch.randn(1, 2, 9, 64, generator=g).cuda().requires_grad_()
    weight, step = torch.randn(1, 2, 9, 64, generator=g).cuda(), torch.randn(1, 2, 9, 64, generator=g).cuda()
    value = lambda z: (elm.rope(z, 40, rope).double() * weight.double()).sum()      # noqa: E731
    grad, = torch.autograd.grad(value(x), x)
    h = 2.0 ** -4
    with torch.no_grad():
        diff = (value(x + h * step) - value(x - h * step)).item() / (2 * h)
        # linear: each number of a rotation is off by 4 half steps of (|a| + |b|) scale, x +- h step by one more; so is the gradient's
        size = rope.scale * 2 * weight.abs().max().item()
        tol = 1152 * size * (2 * 5 * 2.0 ** -24 * (x.abs().max() + h * step.abs().max()).item() / (2 * h) + 4 * 2.0 ** -24 * step.abs().max().item())
        assert abs((grad.double() * step.double()).sum().item() - diff) <= tol


def test_gradient_refused_and_kept_apart():
    rope = elm.Rope(64)
    x = torch.randn(1, 2, 5, 64, generator=torch.Generator().manual_seed(1)).cuda().requires_grad_()
    with pytest.raises(elm.ElmError):                         # a given place for the result has no gradient
        elm.rope(x, 3, rope, out=torch.empty_like(x))
    with torch.no_grad():
        out = torch.empty_like(x)
        assert torch.equal(elm.rope(x, 3, rope, out=out), elm.rope(x, 3, rope)) and not elm.rope(x, 3, rope).requires_grad
    # positions that were changed between the two directions are noticed
    pos = torch.arange(5, dtype=torch.int32)[None].cuda()
    y = elm.rope(x, pos, rope)
    pos += 1
    with pytest.raises(RuntimeError):
        y.sum().backward()


def test_gradient_captured():
    """Both directions in one graph, replayed over other numbers."""
    rope = elm.Rope(64)
    g = torch.Generator().manual_seed(2)
    x = torch.randn(1, 2, 9, 64, generator=g).cuda().requires_grad_()
    dy = torch.randn(1, 2, 9, 64, generator=g).cuda()
    pos = torch.arange(9, dtype=torch.int32)[None].cuda()
    torch.autograd.grad(elm.rope(x, pos, rope), x, dy)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = elm.rope(x, pos, rope)
        dx, = torch.autograd.grad(y, x, dy)
    with torch.no_grad():
        x.copy_(torch.randn(x.shape, generator=g))
    dy.copy_(torch.randn(x.shape, generator=g))
    graph.replay()
    torch.cuda.synchronize()
    with torch.no_grad():
        assert torch.equal(y, elm.rope(x, pos, rope)) and torch.equal(dx, elm.rope(dy, pos, rope, inverse=True))
