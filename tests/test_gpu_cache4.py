"""Rows held in 4 bits on the GPU: stored, read back and attended over, against plain statements in 64 bits."""
import numpy as np
import pytest
import torch

import _cache4 as plain
import paper_2606_10944_b200 as elm

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _np(x):
    return x.double().cpu().numpy()


def _ints(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def _pool(r, n_pages, H, page, d, spread=0.5):
    k = r.standard_normal((n_pages, H, page, d)) * np.exp(spread * r.standard_normal(d))
    v = r.standard_normal((n_pages, H, page, d))
    return torch.as_tensor(plain.pack(k, v)).cuda()


def _tables(r, lengths, page, max_pages, spare=2):
    held = [-(-int(n) // page) for n in lengths]
    order = r.permutation(sum(held) + spare)
    table = np.full((len(lengths), max_pages), -1)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    return table, len(order)


def _rows_of(pool, table, b, h, rows, page, d):
    p = pool.cpu().numpy()
    return plain.unpack(np.stack([p[table[b, r // page], h, r % page] for r in rows]) if len(rows) else np.zeros((0, p.shape[-1]), np.uint8), d)


# ------------------------------------------------------------------------------------------------
# storing
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("T,H,Hq,d,rotary", [(1, 1, 1, 64, 64), (1, 8, 32, 128, 128), (33, 3, 6, 128, 96), (70, 2, 2, 64, 48), (19, 1, 3, 128, 34),
                                             (40, 2, 0, 128, 64), (600, 2, 4, 64, 32), (7, 2, 4, 128, 0)])
def test_append_bits(dtype, layout, T, H, Hq, d, rotary):
    """Every bit of the rows: scales and codes are whole numbers.  Only slots that are given are written."""
    r = np.random.default_rng(T * 7 + d + rotary)
    page, n_pages = 16, T // 16 + 3
    g = torch.Generator().manual_seed(T + rotary)
    wide = torch.randn(T, Hq + 2 * H, d, generator=g) * torch.exp(2 * torch.randn(T, Hq + 2 * H, d // 16, 1, generator=g)).expand(-1, -1, -1, 16).reshape(T, -1, d)
    wide = wide.to(DTYPES[dtype]).cuda()
    Q, K, V = wide[:, :Hq], wide[:, Hq:Hq + H], wide[:, Hq + H:]
    slots = r.permutation(n_pages * page)[:T]
    slots[T // 2] = [-1, n_pages * page, 2 ** 31 - 1][T % 3] if T > 1 else slots[0]
    pos = r.integers(0, 100000, T)
    rope = elm.Rope(rotary, layout=layout) if rotary else None
    rows = torch.full((n_pages, H, page, plain.row_bytes(d)), 0xa5, dtype=torch.uint8, device="cuda")
    out = elm.cache4_append(rows, K, V, _ints(slots), rope=rope, positions=_ints(pos) if rotary else None, Q=Q if Hq else None,
                            q_out=torch.full((T, Hq, d), 7.0, dtype=DTYPES[dtype], device="cuda") if Hq else None)
    want = np.full(rows.shape, 0xa5, np.uint8)
    k = K.float().cpu().numpy()
    if rotary:
        k = plain.rotate(k, pos[:, None], rope.inv_freq, 1.0, layout, single=True)
    packed = plain.pack(k.astype(np.float64), _np(V))
    for t in range(T):
        if 0 <= slots[t] < n_pages * page:
            want[slots[t] // page, :, slots[t] % page] = packed[t]
    assert np.array_equal(rows.cpu().numpy(), want)
    if Hq:
        q = Q.float().cpu().numpy()
        if rotary:
            q = plain.rotate(q, pos[:, None], rope.inv_freq, 1.0, layout, single=True)
        q = torch.as_tensor(q).to(DTYPES[dtype])
        q[[t for t in range(T) if not 0 <= slots[t] < n_pages * page]] = 7.0
        assert torch.equal(out.cpu(), q)


@pytest.mark.parametrize("d", [64, 128])
def test_scales_ties_and_edges(d):
    """Ties of scales and codes, the smallest and largest numbers, zeros of both signs, infinities, NaN."""
    rows = []
    for s in (1.0, 1.125, 1.875, 2.0 ** -14, 3 * 2.0 ** -17, 2.0 ** -17, 10240.0, 0.75 * 2.0 ** 13):
        tie = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, 0.5]) * s
        rows += [tie, tie * (1 + 2.0 ** -20), tie * (1 - 2.0 ** -20)]
    for q in (1 + 1 / 16, 1 + 3 / 16, 2.0 ** -17 * 0.5, 2.0 ** -17 * 1.5, 2.0 ** -14 * (1 - 1 / 16)):      # scales halfway between two
        rows.append(np.array([6 * q] + [q * i / 3 for i in range(15)]))
    rows += [np.zeros(16), -np.zeros(16), np.full(16, 1e-30), np.full(16, 3e38), np.array([np.inf, -np.inf, 1.0, -2.0] * 4),
             np.array([np.nan] + [1.0] * 15), np.array([1.0] * 15 + [-np.nan]), np.full(16, -61440.0), np.array([65536.0, 70000.0, -1.0, 20000.0] * 4)]
    while len(rows) % (d // 16):
        rows.append(np.arange(16) - 8.0)
    x = np.concatenate(rows).reshape(-1, 1, d).astype(np.float32)
    T = len(x)
    pool = elm.cache4_pool(T // 16 + 1, 1, 16, d)
    pool.zero_()
    t = torch.as_tensor(x).cuda()
    elm.cache4_append(pool, t, t.flip(0).contiguous(), _ints(np.arange(T)))
    with np.errstate(invalid="ignore", over="ignore"):
        want = plain.pack(x.astype(np.float64), x[::-1].astype(np.float64))
    assert np.array_equal(pool.cpu().numpy().reshape(-1, plain.row_bytes(d))[:T], want[:, 0])
    k, v = elm.cache4_read(pool, _ints([np.arange(T // 16 + 1)]), T, dtype=torch.float32)
    back = plain.unpack(want[:, 0], d)
    assert np.array_equal(_np(k)[0, 0], back[0], equal_nan=True) and np.array_equal(_np(v)[0, 0], back[1], equal_nan=True)


def test_append_strides_and_in_place():
    d, T, H, Hq = 128, 21, 2, 4
    g = torch.Generator().manual_seed(1)
    rope = elm.Rope(128)
    for dtype in (torch.float32, torch.bfloat16):
        for first in (0, 1):                                  # rows on 16-byte boundaries, and not
            wide = torch.randn(T, Hq + 2 * H, d + 8, generator=g).to(dtype).cuda()[..., first:first + d]
            Q, K, V = wide[:, :Hq], wide[:, Hq:Hq + H], wide[:, Hq + H:]
            slots, pos = _ints(np.random.default_rng(2).permutation(64)[:T]), _ints(np.arange(T) + 9)
            a, b = (torch.zeros(4, H, 16, 144, dtype=torch.uint8, device="cuda") for _ in range(2))
            ref = elm.cache4_append(a, K.contiguous(), V.contiguous(), slots, rope=rope, positions=pos, Q=Q.contiguous())
            before = wide.clone()
            got = elm.cache4_append(b, K, V, slots, rope=rope, positions=pos, Q=Q, q_out=Q)
            assert got is Q and torch.equal(Q, ref) and torch.equal(a, b)
            assert torch.equal(wide[:, Hq:], before[:, Hq:])
            c = elm.cache4_append(b, K.permute(1, 0, 2).contiguous().permute(1, 0, 2), V, slots, rope=rope, positions=pos)
            assert c is None and torch.equal(a, b)


# ------------------------------------------------------------------------------------------------
# reading
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 128])
def test_read(dtype, d, page):
    r = np.random.default_rng(d + page)
    lengths = [0, 1, page, page + 1, 3 * page - 1]
    table, n_pages = _tables(r, lengths, page, 4)
    table[4, 1] = n_pages                                     # bad pages: past the pool, negative
    table[3, 1] = -7
    H = 3
    pool = _pool(r, n_pages, H, page, d)
    n = 4 * page + 5
    k, v = elm.cache4_read(pool, _ints(table), n, length=_ints(lengths), dtype=DTYPES[dtype])
    wk, wv = np.zeros((5, H, n, d)), np.zeros((5, H, n, d))
    for b in range(5):
        there = [i for i in range(lengths[b]) if 0 <= table[b, i // page] < n_pages]
        for h in range(H):
            wk[b, h, there], wv[b, h, there] = _rows_of(pool, table, b, h, there, page, d)
    assert np.array_equal(_np(k), wk) and np.array_equal(_np(v), wv)
    idx = r.integers(-3, 5 * page, (5, H, 40))
    k, v = elm.cache4_read(pool, _ints(table), 40, idx=_ints(idx), length=_ints(lengths), dtype=DTYPES[dtype])
    for b in range(5):
        for h in range(H):
            for i, x in enumerate(idx[b, h]):
                ok = 0 <= x < lengths[b]
                assert np.array_equal(_np(k)[b, h, i], wk[b, h, x] if ok else np.zeros(d))
                assert np.array_equal(_np(v)[b, h, i], wv[b, h, x] if ok else np.zeros(d))


# ------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------
def _check(got, o, size, reach, most, dtype, n, what=""):
    got = _np(got)
    assert np.array_equal(np.isnan(got), np.isnan(o)), what
    with np.errstate(invalid="ignore"):
        err, tol = np.abs(got - o), plain.attend_bound(o, size, reach, most, dtype, n)
    ok = np.isnan(o) | (err <= tol)
    assert ok.all(), (what, float(np.nanmax(err / np.maximum(tol, 1e-300))))


def _check_lengths(pool, table, lengths, Q, got, cu, page, d, causal=True):
    """Q, got [T, Hq, d] and cu, or [B, Hq, n, d]."""
    H, B = pool.shape[1], len(lengths)
    n_pages = pool.shape[0]
    Hq = Q.shape[1]
    rep = Hq // H
    for b in range(B):
        q = _np(Q[cu[b]:cu[b + 1]].transpose(0, 1)) if cu is not None else _np(Q[b])       # [Hq, n, d]
        o = got[cu[b]:cu[b + 1]].transpose(0, 1) if cu is not None else got[b]
        n_q = q.shape[1]
        n = max(0, int(lengths[b]))
        there = np.array([0 <= table[b, i // page] < n_pages for i in range(n)], bool)
        for h in range(H):
            rows = np.nonzero(there)[0]
            k, v = _rows_of(pool, table, b, h, rows, page, d)
            for j in range(n_q):
                upto = n - n_q + 1 + j if causal else n
                ref = plain.attend(q[h * rep:(h + 1) * rep, j], k, v, np.broadcast_to(rows < upto, (rep, len(rows))))
                _check(o[h * rep:(h + 1) * rep, j], *ref, Q.dtype, max(n, 1), (b, h, j))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("H,rep,n_q", [(1, 1, 1), (2, 4, 1), (1, 8, 1), (2, 3, 2), (1, 16, 1), (2, 2, 5), (1, 5, 7)])
def test_attend_lengths(dtype, d, H, rep, n_q):
    r = np.random.default_rng(d + 10 * H + rep)
    page = [16, 32, 64][n_q % 3]
    lengths = [0, 1, 2, 15, 16, 17, 31, 33, 64, 100, 129, 300, 511]
    table, n_pages = _tables(r, lengths, page, 511 // page + 2)
    pool = _pool(r, n_pages, H, page, d)
    g = torch.Generator().manual_seed(n_q)
    Q = torch.randn(len(lengths), H * rep, n_q, d, generator=g).to(DTYPES[dtype]).cuda()
    got = elm.cache4_attend(Q, pool, _ints(table), length=_ints(lengths))
    _check_lengths(pool, table, lengths, Q, got, None, page, d)
    got = elm.cache4_attend(Q, pool, _ints(table), length=_ints(lengths), causal=False)
    _check_lengths(pool, table, lengths, Q, got, None, page, d, causal=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_kv", [None, 2500])
def test_attend_ragged_tokens(dtype, n_kv):
    """Different numbers of new tokens, some none; one long request among short ones; tokens behind the last as they were."""
    r = np.random.default_rng(5)
    d, H, rep, page = 128, 2, 4, 32
    lengths, new = [7, 2500, 0, 64, 33, 40, 1], [3, 9, 0, 0, 33, 1, 1]
    table, n_pages = _tables(r, lengths, page, 100)
    pool = _pool(r, n_pages, H, page, d)
    cu = np.concatenate([[0], np.cumsum(new)])
    T = cu[-1] + 4
    Q = torch.randn(T, H * rep, d, generator=torch.Generator().manual_seed(6)).to(DTYPES[dtype]).cuda()
    out = torch.full_like(Q, 5.0)
    got = elm.cache4_attend(Q, pool, _ints(table), length=_ints(lengths), cu=_ints(cu), max_q=33, n_kv=n_kv, out=out)
    assert got is out and (out[cu[-1]:] == 5.0).all()
    _check_lengths(pool, table, lengths, Q, got, cu, page, d)
    # a queue that names more tokens than there are, or more than max_q: those that are there, and no others
    out = torch.full_like(Q, 5.0)
    elm.cache4_attend(Q[:10], pool, _ints(table), length=_ints(lengths), cu=_ints(cu), max_q=33, out=out[:10])
    assert (out[12:] == 5.0).all() and not (out[:10] == 5.0).all(-1).any()


@pytest.mark.parametrize("d", [64, 128])
def test_attend_bad_pages_and_garbage(d):
    """Rows on no page, and whatever bytes lie behind a request's last row (NaN scales among them), are not seen."""
    r = np.random.default_rng(9)
    page, H, rep = 16, 2, 2
    lengths = [40, 40, 16, 5, 200]
    table, n_pages = _tables(r, lengths, page, 13)
    pool = _pool(r, n_pages, H, page, d)
    for b, n in enumerate(lengths):
        for i in range(n, -(-n // page) * page):
            pool[table[b, i // page], :, i % page] = 0xff
    table[0, 1] = n_pages + 3
    table[1, 0] = -1
    table[2, 0] = 2 ** 31 - 1
    Q = torch.randn(5, H * rep, 2, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    got = elm.cache4_attend(Q, pool, _ints(table), length=_ints(lengths))
    _check_lengths(pool, table, lengths, Q, got, None, page, d)
    assert (got[2] == 0).all()
    # lengths past the table are the table's rows (here with the garbage of the last page), negative ones none
    got = elm.cache4_attend(Q, pool, _ints(table), length=_ints([40, -5, 16, 5, 10 ** 9]))
    ref = elm.cache4_attend(Q, pool, _ints(table), length=_ints([40, 0, 16, 5, 13 * page]))
    assert (got[1] == 0).all() and torch.equal(got[:4], ref[:4]) and torch.equal(torch.isnan(got[4]), torch.isnan(ref[4]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_nan_rows_and_queries(dtype, d):
    """NaN in a row that a query sees gives NaN in the numbers it reaches; in one that it does not see, nothing."""
    r = np.random.default_rng(d)
    page, H, rep, n_q, n = 16, 1, 2, 6, 45
    table, n_pages = _tables(r, [n, n, n], page, 3)
    pool = _pool(r, n_pages, H, page, d)
    value_scales = d + d // 16                                # in a row's bytes
    pool[table[0, 42 // page], 0, 42 % page, value_scales + 1] = 0xff      # a group of the value of row 42
    pool[table[1, 43 // page], 0, 43 % page, d] = 0xff                     # a group of the key of row 43
    Q = torch.randn(3, rep, n_q, d, generator=torch.Generator().manual_seed(2)).to(DTYPES[dtype]).cuda()
    Q[2, 1, 3, 5] = float("nan")
    got = elm.cache4_attend(Q, pool, _ints(table), length=_ints([n, n, n]))
    _check_lengths(pool, table, [n, n, n], Q, got, None, page, d)
    bad = torch.isnan(got)
    # query j sees the rows below 40 + j
    assert bad[0, :, 3:, 16:32].all() and not bad[0, :, :3].any() and not bad[0, :, :, :16].any() and not bad[0, :, :, 32:].any()
    assert bad[1, :, 4:].all() and not bad[1, :, :4].any()
    assert bad[2, 1, 3].all() and bad[2].sum() == d


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_sizes_of_numbers(dtype):
    """Logits in the thousands, queries of any size, a far larger row late in the list: the running reference moves."""
    r = np.random.default_rng(12)
    d, page, H, n = 128, 64, 1, 700
    table, n_pages = _tables(r, [n] * 6, page, 11)
    pool = _pool(r, n_pages, H, page, d, spread=1.5)
    Q = torch.randn(6, 8, 1, d, generator=torch.Generator().manual_seed(3))
    Q[1] *= 30
    Q[2] *= 1e-30
    Q[3] = 0
    Q[4] *= 1e4
    Q[5, :, :, ::2] *= 1e-6
    Q = Q.to(DTYPES[dtype]).cuda()
    got = elm.cache4_attend(Q, pool, _ints(table), length=_ints([n] * 6))
    # (one query large enough for a logit's error to be a factor: there the bound says nothing, and only that it is finite is asked)
    _check_lengths(pool, table, [n] * 6, Q, got, None, page, d)
    assert torch.isfinite(got).all()


def _list(r, B, H, n, n_core):
    idx = np.stack([[r.integers(0, n, n_core) for _ in range(H)] for _ in range(B)])
    w = 2.0 ** r.integers(-17, -8, (B, H, n_core))
    return idx, w


def _check_list(pool, table, idx, w, Q, got, page, d):
    B, H = idx.shape[:2]
    rep = Q.shape[1] // H
    n_pages = pool.shape[0]
    cap = table.shape[1] * page
    for b in range(B):
        for h in range(H):
            i = idx[b, h]
            there = np.array([0 <= x < cap and 0 <= table[b, x // page] < n_pages for x in i]) & (w[b, h] > 0)
            k, v = _rows_of(pool, table, b, h, i[there], page, d)
            q = _np(Q[b, h * rep:(h + 1) * rep]).reshape(-1, d)
            ref = plain.attend(q, k, v, np.ones((len(q), len(k)), bool), np.log(w[b, h][there]))
            _check(got[b, h * rep:(h + 1) * rep].reshape(-1, d), *ref, Q.dtype, len(i), (b, h))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("n_core,n_q,rep", [(1, 1, 1), (31, 1, 4), (33, 3, 2), (257, 1, 8), (1000, 2, 4), (2048, 1, 4)])
def test_attend_list(dtype, d, n_core, n_q, rep):
    r = np.random.default_rng(n_core + d)
    B, H, page, n = 2, 2, 32, 1500
    table, n_pages = _tables(r, [n] * B, page, 50)
    pool = _pool(r, n_pages, H, page, d)
    idx, w = _list(r, B, H, n, n_core)
    if n_core > 30:
        idx[0, 0, 3], idx[0, 1, 5], idx[1, 0, 7] = -1, 10 ** 9, 50 * page - 1              # rows that are not there
        w[1, 1, 9], w[0, 0, 11] = 0.0, -1.0
        idx[1, 1, 9] = n - 1
        pool[table[1, (n - 1) // page], 1, (n - 1) % page] = 0xff                          # NaN in a row of weight 0
        idx[1, 1][idx[1, 1] == n - 1] = 3
        idx[1, 1, 9] = n - 1
    Q = torch.randn(B, H * rep, n_q, d, generator=torch.Generator().manual_seed(n_core)).to(DTYPES[dtype]).cuda()
    got = elm.cache4_attend(Q, pool, _ints(table), idx=_ints(idx), w=torch.as_tensor(w, dtype=torch.float32).cuda())
    _check_list(pool, table, idx, w, Q, got, page, d)


def _by_tensor_cores(Q, pool, table, n_core):
    """Whether a call takes the tensor-core form, by the workspace it asks for."""
    p = elm.Cache4Params(Q.shape[0], Q.shape[1], pool.shape[1], Q.shape[3], 1, pool.shape[2], pool.shape[0], table.shape[1], n_core, Q.shape[2])
    need = elm.cache4_attend_workspace_bytes(p, True)
    p.dtype = 0                                               # (fp32 queries do not)
    return need != elm.cache4_attend_workspace_bytes(p, True)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("n_core", [1, 100, 128, 500])
def test_attend_list_of_many_queries(d, n_core):
    """The tensor-core form of bf16 lists: probabilities are bf16 there (half a step 2^-8 of each)."""
    r = np.random.default_rng(n_core)
    B, H, rep, page, n, n_q = 2, 2, 2, 64, 900, 3001
    table, n_pages = _tables(r, [n] * B, page, 16)
    pool = _pool(r, n_pages, H, page, d)
    idx, w = _list(r, B, H, n, n_core)
    if n_core > 30:
        idx[0, 0, 3], w[1, 1, 9], idx[0, 0, 60] = -1, 0.0, 10 ** 9
    Q = torch.randn(B, H * rep, n_q, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    assert _by_tensor_cores(Q, pool, table, n_core)
    tw = torch.as_tensor(w, dtype=torch.float32).cuda()
    got = elm.cache4_attend(Q, pool, _ints(table), idx=_ints(idx), w=tw)
    for b in range(B):
        for h in range(H):
            there = (idx[b, h] >= 0) & (idx[b, h] < 16 * page) & (w[b, h] > 0)
            k, v = _rows_of(pool, table, b, h, idx[b, h][there], page, d)
            q = _np(Q[b, h * rep:(h + 1) * rep]).reshape(-1, d)
            o, size, reach, most = plain.attend(q, k, v, np.ones((len(q), len(k)), bool), np.log(w[b, h][there]))
            err = np.abs(_np(got[b, h * rep:(h + 1) * rep]).reshape(-1, d) - o)
            # probabilities 2^-8 (numerator; the denominator sums them unrounded), their exponentials partly by a cubic: 1e-4 twice
            tol = plain.attend_bound(o, size, reach, most, torch.bfloat16, n_core) + (2.0 ** -8 + 2e-4) * size
            assert (err <= tol).all()
    # the same with few queries: the other form
    assert not _by_tensor_cores(Q[:, :, :3], pool, table, n_core)
    few = elm.cache4_attend(Q[:, :, :3].contiguous(), pool, _ints(table), idx=_ints(idx), w=tw)
    assert (few.float() - got[:, :, :3].float()).abs().max() <= 0.05 * got.float().abs().max()


def test_attend_list_nothing_seen():
    r = np.random.default_rng(0)
    pool = _pool(r, 4, 1, 16, 128)
    idx, w = np.full((1, 1, 40), -1), np.ones((1, 1, 40))
    for n_q in (1, 200, 20000):
        Q = torch.randn(1, 2, n_q, 128).bfloat16().cuda()
        assert _by_tensor_cores(Q, pool, np.zeros((1, 2)), 40) == (n_q == 20000)
        got = elm.cache4_attend(Q, pool, _ints([[0, 1]]), idx=_ints(idx), w=torch.as_tensor(w, dtype=torch.float32).cuda())
        assert (got == 0).all()


def test_attend_strides():
    r = np.random.default_rng(20)
    d, H, rep, page, n = 64, 2, 3, 16, 90
    table, n_pages = _tables(r, [n, 30], page, 6)
    pool = _pool(r, n_pages, H, page, d)
    Q = torch.randn(2, 4, H * rep + 2, d, generator=torch.Generator().manual_seed(1)).cuda()[:, :, 1:1 + H * rep].transpose(1, 2)
    ref = elm.cache4_attend(Q.contiguous(), pool, _ints(table), length=_ints([n, 30]))
    wide = torch.full((2, 4, H * rep + 2, d), 3.0, device="cuda")
    out = wide[:, :, 2:].transpose(1, 2)
    assert torch.equal(elm.cache4_attend(Q, pool, _ints(table), length=_ints([n, 30]), out=out), ref)
    assert (wide[:, :, :2] == 3.0).all()
    assert torch.equal(elm.cache4_attend(Q, pool, _ints(table), length=_ints([n, 30]), out=Q), ref)      # over the queries themselves


def test_attend_long_and_repeatable():
    """Many stretches per request; the same bits every time, on another stream, and from a captured graph whose lengths change."""
    r = np.random.default_rng(30)
    d, H, rep, page = 128, 2, 4, 256
    lengths = [40000, 17, 3000]
    table, n_pages = _tables(r, lengths, page, 160)
    small = _pool(r, 8, H, page, d)
    pool = small[torch.as_tensor(r.integers(0, 8, n_pages))].contiguous()
    Q = torch.randn(3, H * rep, 1, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    t, n = _ints(table), _ints(lengths)
    ref = elm.cache4_attend(Q, pool, t, length=n)
    _check_lengths(pool, table, lengths, Q, ref, None, page, d)
    for _ in range(3):
        assert torch.equal(elm.cache4_attend(Q, pool, t, length=n), ref)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs.append([elm.cache4_attend(Q, pool, t, length=n) for _ in range(5)])
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for part in outs for o in part)
    live = _ints([1, 1, 1])
    out = torch.empty_like(Q)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    elm.cache4_attend(Q, pool, t, length=live, workspace=ws, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        elm.cache4_attend(Q, pool, t, length=live, workspace=ws, out=out)
    for want in (lengths, [1, 0, 2], lengths):
        live.copy_(_ints(want))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, elm.cache4_attend(Q, pool, t, length=_ints(want)))


def test_row_numbers_past_32_bits():
    """A pool of more than 2^32 bytes: the last page's rows are where they belong."""
    d, H, page = 128, 8, 1024
    n_pages = (5 << 30) // (H * page * 144)
    pool = torch.empty(n_pages, H, page, 144, dtype=torch.uint8, device="cuda")
    r = np.random.default_rng(2)
    last = _pool(r, 1, H, page, d)
    pool[n_pages - 1] = last[0]
    table = np.array([[n_pages - 1]])
    Q = torch.randn(1, 2 * H, 1, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    got = elm.cache4_attend(Q, pool, _ints(table), length=_ints([777]))
    assert torch.equal(got, elm.cache4_attend(Q, last, _ints([[0]]), length=_ints([777])))
    K = torch.randn(3, H, d, generator=torch.Generator().manual_seed(2)).cuda()
    slots = [(n_pages - 1) * page + 5, 1, (n_pages - 1) * page + 1023]
    elm.cache4_append(pool, K, K, _ints(slots))
    k, _ = elm.cache4_read(pool, _ints(table), 2, idx=_ints(np.broadcast_to([5, 1023], (1, H, 2)).copy()), dtype=torch.float32)
    assert np.array_equal(_np(k[0]), plain.unpack(plain.pack(_np(K), _np(K)), d)[0][[0, 2]].swapaxes(0, 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("H,rep,n_q,page", [(1, 2, 1, 16), (2, 4, 2, 32), (1, 3, 5, 128), (1, 20, 1, 1024)])
def test_attend_stretches(dtype, d, H, rep, n_q, page):
    """Tables of so many pages that the rows are one line cut into equal stretches: problems inside one, and over several, of every
    form of the kernel, with rows that are on no page."""
    r = np.random.default_rng(d + page)
    lengths = [3000, 5, 0, 700, 4097, 64, 1]
    table, n_pages = _tables(r, lengths, page, 9216 // page + 1)
    small = _pool(r, 4, H, page, d)
    pool = small[torch.as_tensor(r.integers(0, 4, n_pages))].contiguous()
    table[0, 1], table[4, 4096 // page] = n_pages, -1
    Q = torch.randn(len(lengths), H * rep, n_q, d, generator=torch.Generator().manual_seed(d)).to(DTYPES[dtype]).cuda()
    got = elm.cache4_attend(Q, pool, _ints(table), length=_ints(lengths))
    _check_lengths(pool, table, lengths, Q, got, None, page, d)


@pytest.mark.parametrize("B,cap", [(33, 40), (130, 600), (600, 300), (1024, 9000)])
def test_attend_many_requests(B, cap):
    """As many requests as a call takes, most of them short, some without queries."""
    r = np.random.default_rng(B)
    d, H, rep, page = 64, 1, 2, 16
    lengths = r.integers(0, 30, B)
    lengths[B // 2], lengths[B - 1] = cap - 7, cap // 2
    new = r.integers(0, 3, B)
    table, n_pages = _tables(r, lengths, page, -(-cap // page))
    pool = _pool(r, n_pages, H, page, d)
    cu = np.concatenate([[0], np.cumsum(new)])
    Q = torch.randn(int(cu[-1]), H * rep, d, generator=torch.Generator().manual_seed(B)).bfloat16().cuda()
    wide = torch.full((int(cu[-1]), H * rep + 1, d), 9.0, dtype=torch.bfloat16, device="cuda")
    got = elm.cache4_attend(Q, pool, _ints(table), length=_ints(lengths), cu=_ints(cu), max_q=2, out=wide[:, 1:])
    assert (wide[:, 0] == 9.0).all()
    _check_lengths(pool, table, lengths, Q, got, cu, page, d)


@pytest.mark.parametrize("n_kv", [200, 6000])
def test_attend_far_bound_of_queries(n_kv):
    """max_q far above the tokens that requests have."""
    r = np.random.default_rng(3)
    d, H, rep, page, B = 128, 4, 4, 16, 40
    lengths = r.integers(1, 190, B)
    if n_kv > 200:
        lengths[7] = 5600
    new = r.integers(0, 6, B)
    table, n_pages = _tables(r, lengths, page, -(-n_kv // page))
    small = _pool(r, 8, H, page, d)
    pool = small[torch.as_tensor(r.integers(0, 8, n_pages))].contiguous()
    cu = np.concatenate([[0], np.cumsum(new)])
    Q = torch.randn(int(cu[-1]), H * rep, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    args = dict(length=_ints(lengths), cu=_ints(cu))
    ref = elm.cache4_attend(Q, pool, _ints(table), max_q=5, **args)
    _check_lengths(pool, table, lengths, Q, ref, cu, page, d)
    for max_q in (50, 3000):
        got = elm.cache4_attend(Q, pool, _ints(table), max_q=max_q, **args)
        _check_lengths(pool, table, lengths, Q, got, cu, page, d)


def test_append_of_many_heads():
    """More heads than a block has threads for at once, of keys and of queries."""
    r = np.random.default_rng(7)
    T, H, Hq, d = 9, 70, 300, 128
    x = torch.randn(T, Hq + 2 * H, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    Q, K, V = x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
    for rotary in (128, 48):
        rope = elm.Rope(rotary)
        rows = torch.zeros(1, H, 16, 144, dtype=torch.uint8, device="cuda")
        slots, pos = r.permutation(16)[:T], r.integers(0, 9999, T)
        q = elm.cache4_append(rows, K, V, _ints(slots), rope=rope, positions=_ints(pos), Q=Q)
        k = plain.rotate(K.float().cpu().numpy(), pos[:, None], rope.inv_freq, single=True)
        assert np.array_equal(rows.cpu().numpy()[0][:, slots].swapaxes(0, 1), plain.pack(k.astype(np.float64), _np(V)))
        assert torch.equal(q.cpu(), torch.as_tensor(plain.rotate(Q.float().cpu().numpy(), pos[:, None], rope.inv_freq, single=True)).bfloat16())


# ------------------------------------------------------------------------------------------------
# as they are used together
# ------------------------------------------------------------------------------------------------
def test_a_generation():
    """Prompts come in, their pages are planned, rows stored and attended over; then steps of a token each; a request ends and its
    pages go to a new one.  Against attention in 64 bits over the rows as a plain statement stores them."""
    torch.manual_seed(0)
    r = np.random.default_rng(1)
    B, H, rep, d, page, n_pages, max_pages = 3, 2, 4, 128, 16, 24, 10
    rope = elm.Rope(d)
    pool = elm.cache4_pool(n_pages, H, page, d)
    table, length, free, count = _ints(np.full((B, max_pages), -1)), _ints([0] * B), _ints(np.arange(n_pages)), _ints([n_pages])
    kept = [[] for _ in range(B)]                             # per request the rows [Hkv] as stored
    for step, new in enumerate([[37, 1, 80], [1, 1, 1], [1, 1, 1], [4, 0, 2], [1, 50, 1]]):
        if step == 4:
            elm.page_release(table, length, _ints([0, 1, 0]), free, count, page)
            kept[1] = []
        T = sum(new) + 2
        plan = elm.page_plan(table, length, _ints(new), free, count, page, T, length_out=length, free_count_out=count)
        x = torch.randn(T, H * (rep + 2), d, device="cuda").bfloat16()
        Q, K, V = x[:, :H * rep], x[:, H * rep:H * (rep + 1)], x[:, H * (rep + 1):]
        q = elm.cache4_append(pool, K, V, plan.slots, rope=rope, positions=plan.positions, Q=Q)
        o = elm.cache4_attend(q, pool, table, length=length, cu=plan.cu, max_q=max(new))
        k = plain.rotate(K.float().cpu().numpy(), plan.positions.cpu().numpy()[:, None], rope.inv_freq, single=True)
        back = plain.unpack(plain.pack(k.astype(np.float64), _np(V)), d)
        cu = np.concatenate([[0], np.cumsum(new)])
        for b in range(B):
            n0 = len(kept[b])
            kept[b] += [(back[0][t], back[1][t]) for t in range(cu[b], cu[b + 1])]
            assert plan.positions[cu[b]:cu[b + 1]].tolist() == list(range(n0, len(kept[b])))
            if not kept[b]:
                continue
            ks, vs = np.stack([a for a, _ in kept[b]]), np.stack([a for _, a in kept[b]])
            for j, t in enumerate(range(cu[b], cu[b + 1])):
                for h in range(H):
                    n = n0 + j + 1
                    qq = _np(q[t, h * rep:(h + 1) * rep])
                    ref = plain.attend(qq, ks[:n, h], vs[:n, h], np.ones((rep, n), bool))
                    _check(o[t, h * rep:(h + 1) * rep], *ref, torch.bfloat16, n, (step, b, j))
        assert length.tolist() == [len(x) for x in kept]


def test_coreset_of_a_stored_prompt():
    """A prompt's rows read back, compressed by elm_compress, and attended over in 4 bits: as elm_attend over the rows read back."""
    B, H, rep, d, n, page = 1, 2, 2, 128, 4096, 64
    pool = elm.cache4_pool(n // page, H, page, d)
    g = torch.Generator().manual_seed(3)
    K, V = torch.randn(n, H, d, generator=g).bfloat16().cuda(), torch.randn(n, H, d, generator=g).bfloat16().cuda()
    order = np.random.default_rng(4).permutation(n // page)
    slots = (order[np.arange(n) // page] * page + np.arange(n) % page)
    elm.cache4_append(pool, K, V, _ints(slots), rope=elm.Rope(d), positions=_ints(np.arange(n)))
    table = _ints(order[None])
    k, v = elm.cache4_read(pool, table, n)
    idx, w = elm.compress(k, v, 8, 4, seed=5)
    for n_q in (1, 5, 400, 8000):
        Q = torch.randn(B, H * rep, n_q, d, generator=g).bfloat16().cuda()
        got, ref = elm.cache4_attend(Q, pool, table, idx=idx, w=w), elm.attend(Q, k, v, idx, w)
        # two bf16 outputs, and probabilities of 2^-8 in either, of values whose mean size is the bound's
        size = float(v.float().abs().mean()) * 4
        assert (got.float() - ref.float()).abs().max().item() <= 2 * 2.0 ** -8 * size * 2
    assert _by_tensor_cores(Q, pool, table, 256)
    many = elm.cache4_attend(Q, pool, table, idx=idx, w=w)
    assert torch.equal(many, elm.attend(Q, k, v, idx, w))     # the same kernel over the same bf16 rows


def test_a_captured_decode_step():
    """Plan, append and attention of a decode step in one graph, replayed as the requests grow over pages' ends: as the same calls made
    one by one."""
    B, H, rep, d, page, n_pages, max_pages = 5, 2, 4, 128, 16, 40, 8
    rope = elm.Rope(d, layout="pairs")
    x = torch.zeros(B, H * (rep + 2), d, dtype=torch.bfloat16, device="cuda")
    Q, K, V = x[:, :H * rep], x[:, H * rep:H * (rep + 1)], x[:, H * (rep + 1):]
    one = _ints([1] * B)

    def state():
        return dict(pool=torch.zeros(n_pages, H, page, 144, dtype=torch.uint8, device="cuda"), table=_ints(np.full((B, max_pages), -1)),
                    length=_ints([0] * B), free=_ints(np.arange(n_pages)), count=_ints([n_pages]))

    def step(s, out):
        plan = elm.page_plan(s["table"], s["length"], one, s["free"], s["count"], page, B, length_out=s["length"], free_count_out=s["count"])
        q = elm.cache4_append(s["pool"], K, V, plan.slots, rope=rope, positions=plan.positions, Q=Q)
        return elm.cache4_attend(q, s["pool"], s["table"], length=s["length"], cu=plan.cu, max_q=1, out=out)

    eager, kept = state(), state()
    out, ref = torch.zeros_like(Q.contiguous()), torch.zeros_like(Q.contiguous())
    step(state(), out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(kept, out)
    g = torch.Generator().manual_seed(5)
    for i in range(40):
        x.copy_(torch.randn(x.shape, generator=g))
        graph.replay()
        step(eager, ref)
        torch.cuda.synchronize()
        assert torch.equal(out, ref), i
    assert kept["length"].tolist() == [40] * B and torch.equal(kept["pool"], eager["pool"]) and torch.equal(kept["table"], eager["table"])


def _check_many(pool, table, idx, w, Q, got, page, d):
    """Lists met by many queries: probabilities 2^-8 (numerator; the denominator sums them unrounded), their exponentials partly by a cubic:
    1e-4 twice."""
    B, H = idx.shape[:2]
    rep = Q.shape[1] // H
    for b in range(B):
        for h in range(H):
            i = idx[b, h]
            there = np.array([0 <= x < table.shape[1] * page and 0 <= table[b, x // page] < pool.shape[0] for x in i]) & (w[b, h] > 0)
            k, v = _rows_of(pool, table, b, h, i[there], page, d)
            q = _np(Q[b, h * rep:(h + 1) * rep]).reshape(-1, d)
            o, size, reach, most = plain.attend(q, k, v, np.ones((len(q), len(k)), bool), np.log(w[b, h][there]))
            out = _np(got[b, h * rep:(h + 1) * rep]).reshape(-1, d)
            assert np.isfinite(out).all(), (b, h)
            assert (np.abs(out - o) <= plain.attend_bound(o, size, reach, most, torch.bfloat16, len(i)) + (2.0 ** -8 + 2e-4) * size).all(), (b, h)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("hidden", [(0, 127), (0, 128), (0, 200), (0, 256), (0, 499), (128, 256), (200, 500), (1, 500)])
def test_attend_list_of_many_queries_blocks_not_seen(d, hidden):
    """Whole blocks of 128 entries that are not seen, the first among them: by weights of 0 and below, by negative numbers, by pages that are
    none; one problem of which everything is seen, with one weight, beside them."""
    r = np.random.default_rng(d + hidden[1])
    B, H, rep, page, n, n_q, n_core = 3, 2, 2, 64, 900, 701, 500
    table, n_pages = _tables(r, [n] * B, page, 16)
    pool = _pool(r, n_pages, H, page, d)
    idx, w = _list(r, B, H, n, n_core)
    a, e = hidden
    table[1, 2] = n_pages + 1
    idx[1][idx[1] // page == 2] = 5
    w[0, 0, a:e] = 0.0
    w[0, 1, a:e] = -1.0
    idx[1, 0, a:e] = -1
    idx[1, 1, a:e] = 2 * page + np.arange(e - a) % page
    w[2, 0] = 2.0 ** -9
    w[2, 1] = np.nan
    w[2, 1, e - 1] = 1.0
    Q = torch.randn(B, H * rep, n_q, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    assert _by_tensor_cores(Q, pool, table, n_core)
    args = dict(idx=_ints(idx), w=torch.as_tensor(w, dtype=torch.float32).cuda())
    got = elm.cache4_attend(Q, pool, _ints(table), **args)
    _check_many(pool, table, idx, w, Q, got, page, d)
    few = elm.cache4_attend(Q[:, :, :2].contiguous(), pool, _ints(table), **args)
    _check_list(pool, table, idx, w, Q[:, :, :2].contiguous(), few, page, d)


def test_append_of_as_many_tokens_as_there_can_be():
    """2^31 - 1 places (8.6 GB of slots) of which four are tokens, keys and values one row for all: the four are stored."""
    T, d, page = 2 ** 31 - 1, 64, 16
    k = torch.randn(1, 1, d, generator=torch.Generator().manual_seed(1)).cuda()
    rows = torch.full((2, 1, page, 80), 0xa5, dtype=torch.uint8, device="cuda")
    slots = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    for t, slot in ((0, 3), (1 << 30, 17), (T - 64, 9), (T - 1, 31)):
        slots[t] = slot
    elm.cache4_append(rows, k.expand(T, 1, d), k.expand(T, 1, d), slots)
    want = np.full((2 * page, 80), 0xa5, np.uint8)
    want[[3, 17, 9, 31]] = plain.pack(_np(k), _np(k))[0, 0]
    assert np.array_equal(rows.cpu().numpy()[:, 0].reshape(-1, 80), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("held,max_q", [(10, 33), (100, 5), (7, 5), (41, 33)])
def test_attend_tokens_cut_off(dtype, held, max_q):
    """Requests of which Q holds the first tokens only, or that have more than max_q: those see the rows that they would see among all
    of them."""
    r = np.random.default_rng(5)
    d, H, rep, page = 128, 2, 4, 32
    lengths, new = [7, 2500, 64, 33, 40, 1], [3, 9, 0, 33, 4, 1]
    table, n_pages = _tables(r, lengths, page, 100)
    pool = _pool(r, n_pages, H, page, d)
    cu = np.concatenate([[0], np.cumsum(new)])
    Q = torch.randn(held, H * rep, d, generator=torch.Generator().manual_seed(6)).to(DTYPES[dtype]).cuda()
    for causal in (True, False):
        out = torch.full_like(Q, 5.0)
        elm.cache4_attend(Q, pool, _ints(table), length=_ints(lengths), cu=_ints(cu), max_q=max_q, causal=causal, out=out)
        written = np.zeros(held, bool)
        for b, n in enumerate(lengths):
            for j in range(min(new[b], max_q, max(0, held - cu[b]))):
                t = cu[b] + j
                written[t] = True
                for h in range(H):
                    k, v = _rows_of(pool, table, b, h, np.arange(n), page, d)
                    upto = n - new[b] + 1 + j if causal else n
                    ref = plain.attend(_np(Q[t, h * rep:(h + 1) * rep]), k, v, np.broadcast_to(np.arange(n) < upto, (rep, n)))
                    _check(out[t, h * rep:(h + 1) * rep], *ref, Q.dtype, n, (b, h, j))
        assert (out[torch.as_tensor(~written)] == 5.0).all()


# ------------------------------------------------------------------------------------------------
# forms that the calls above do not meet
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("n_core", [130, 2100])               # one CTA or a cluster, clusters
@pytest.mark.parametrize("hidden", [(0, 32), (0, 64), (32, 64), (31, 129), (0, 129), (64, 2100)])
def test_attend_list_tiles_not_seen(dtype, d, n_core, hidden):
    """Whole tiles of 32 entries that are not seen: by weight, by number, by page, the first, the last and all but one among them."""
    r = np.random.default_rng(n_core + hidden[1])
    B, H, rep, page, n = 2, 2, 4, 32, 1500
    table, n_pages = _tables(r, [n] * B, page, 50)
    pool = _pool(r, n_pages, H, page, d)
    idx, w = _list(r, B, H, n, n_core)
    a, e = hidden[0], min(hidden[1], n_core)
    table[1, 2] = -1
    idx[1, 1][idx[1, 1] // page == 2] = 5
    w[0, 0, a:e], w[0, 1, a:e] = 0.0, np.nan
    idx[1, 0, a:e], idx[1, 1, a:e] = -5, 2 * page + 3
    Q = torch.randn(B, H * rep, 1, d, generator=torch.Generator().manual_seed(2)).to(DTYPES[dtype]).cuda()
    got = elm.cache4_attend(Q, pool, _ints(table), idx=_ints(idx), w=torch.as_tensor(w, dtype=torch.float32).cuda())
    _check_list(pool, table, idx, w, Q, got, page, d)


@pytest.mark.parametrize("d", [128, 64])
def test_attend_list_of_many_queries_in_place_and_status(d):
    """The tensor-core form over its own queries, and its status: 0, or what a bounded wait left that ran out (made to by a test hook; the
    launch ends by itself), and 0 again after the next call."""
    from paper_2606_10944_b200 import binding
    lib = binding.load_library()
    r = np.random.default_rng(d)
    H, rep, page, n, n_core, n_q = 2, 2, 64, 900, 300, 3001
    table, n_pages = _tables(r, [n], page, 16)
    pool = _pool(r, n_pages, H, page, d)
    idx, w = _list(r, 1, H, n, n_core)
    Q = torch.randn(1, H * rep, n_q, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    assert _by_tensor_cores(Q, pool, table, n_core)
    p = elm.Cache4Params(1, H * rep, H, d, 1, page, n_pages, 16, n_core, n_q)
    ws = torch.empty(elm.cache4_attend_workspace_bytes(p, True), dtype=torch.uint8, device="cuda")
    args = dict(idx=_ints(idx), w=torch.as_tensor(w, dtype=torch.float32).cuda(), workspace=ws)
    t = _ints(table)
    ref = elm.cache4_attend(Q, pool, t, **args)
    assert elm.cache4_attend_status(ws, p, True) == 0
    try:
        assert lib.elm_debug_set(0, 20_000_000) == 0          # waits give up after 20 ms
        assert lib.elm_debug_set(1, 1) == 0                   # the next launch misses one arrival per barrier
        elm.cache4_attend(Q, pool, t, **args)
        torch.cuda.synchronize()
        assert elm.cache4_attend_status(ws, p, True) != 0
    finally:
        assert lib.elm_debug_set(0, 2_000_000_000) == 0
    assert elm.cache4_attend(Q, pool, t, out=Q, **args) is Q
    assert elm.cache4_attend_status(ws, p, True) == 0 and torch.equal(Q, ref)
    p = elm.Cache4Params(1, H * rep, H, d, 1, page, n_pages, 16, 0, 1)
    ws = torch.empty(elm.cache4_attend_workspace_bytes(p, False), dtype=torch.uint8, device="cuda")
    elm.cache4_attend(Q[:, :, :1].contiguous(), pool, t, length=_ints([n]), workspace=ws)
    assert elm.cache4_attend_status(ws, p, False) == 0


def test_threads_that_share_a_rotation():
    """Steps of many sizes from two threads on streams of their own, with one Rope: what each does alone."""
    import threading
    d, H, page = 128, 2, 16
    rope = elm.Rope(d)
    sizes = list(range(1, 41))
    g = torch.Generator().manual_seed(1)
    x = torch.randn(40, H, d, generator=g).cuda()
    table, length = _ints(np.arange(4)[None]), _ints([40])

    def steps(rope):
        rows = elm.cache4_pool(4, H, page, d)
        rows.zero_()
        for n in sizes:
            k = x[:n]
            q = elm.cache4_append(rows, k, k, _ints(np.arange(n)), rope=rope, positions=_ints(np.arange(n)), Q=k)
            y = elm.rope(k[None].transpose(1, 2), 5, rope)
        o = elm.cache4_attend(q.transpose(0, 1)[None].contiguous(), rows, table, length=length)
        return rows, q, y, o

    want = steps(elm.Rope(d))
    torch.cuda.synchronize()
    found = {}

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            found[i] = steps(rope)
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(found[i], want))


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("n_q", [2, 20000])
def test_attend_list_nan_queries(d, n_q):
    """Over a list a query with a NaN gets NaN, whether it sees anything or not, and no other query does."""
    r = np.random.default_rng(d)
    pool = _pool(r, 4, 2, 16, d)
    idx, w = _list(r, 1, 2, 60, 40)
    idx[0, 1] = -1
    Q = torch.randn(1, 4, n_q, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    Q[:, :, 1, 3] = float("nan")
    assert _by_tensor_cores(Q, pool, np.zeros((1, 4)), 40) == (n_q == 20000)
    got = elm.cache4_attend(Q, pool, _ints([[0, 1, 2, 3]]), idx=_ints(idx), w=torch.as_tensor(w, dtype=torch.float32).cuda())
    bad = torch.isnan(got).any(-1)
    assert bad[:, :, 1].all() and bad.sum() == 4 and torch.isnan(got[:, :, 1]).all()
    assert (got[:, 2:, 0] == 0).all() and (got[:, :2, 0] != 0).any(-1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rep", [1, 3])
def test_attend_prompt_chunks(dtype, rep):
    """Hundreds of new tokens to a request, behind rows that were there and at its beginning; some of the tokens against 64 bits."""
    r = np.random.default_rng(rep)
    d, H, page = 64, 2, 32
    lengths, new = [2900, 701, 1, 40], [513, 701, 1, 39]
    table, n_pages = _tables(r, lengths, page, 100)
    pool = _pool(r, n_pages, H, page, d)
    cu = np.concatenate([[0], np.cumsum(new)])
    Q = torch.randn(cu[-1], H * rep, d, generator=torch.Generator().manual_seed(1)).to(DTYPES[dtype]).cuda()
    got = elm.cache4_attend(Q, pool, _ints(table), length=_ints(lengths), cu=_ints(cu), max_q=max(new))
    for b, n in enumerate(lengths):
        k, v = zip(*[_rows_of(pool, table, b, h, np.arange(n), page, d) for h in range(H)])
        for j in sorted({0, 1, 31, 32, new[b] // 2, new[b] - 2, new[b] - 1} & set(range(new[b]))):
            t, upto = cu[b] + j, n - new[b] + 1 + j
            for h in range(H):
                ref = plain.attend(_np(Q[t, h * rep:(h + 1) * rep]), k[h], v[h], np.broadcast_to(np.arange(n) < upto, (rep, n)))
                _check(got[t, h * rep:(h + 1) * rep], *ref, Q.dtype, n, (b, h, j))
