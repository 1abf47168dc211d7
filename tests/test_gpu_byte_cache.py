"""The operators over a cache of keys and values in 8 bits against tests/byte_cache_util.py."""

import math

import numpy as np
import pytest

import byte_cache_util as u

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DEV = "cuda:0"


def cache_of(req, heads, dim, tokens):
    """A cache whose buffers hold anything: NaN halves, codes and scales of a block that nobody stored."""
    from paper_2506_23431_amd import ByteCache
    c = ByteCache(req, heads, dim, tokens, device=DEV)
    c.k.fill_(77), c.v.fill_(-99)
    for t in (c.k_scale, c.v_scale, c.k_tail, c.v_tail):
        t.fill_(float("nan"))
    return c


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def data(seed, req, n, heads, dim, kind, spread=1.0):
    """Tokens of the type, and the same as float32 numpy."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((req, n, heads, dim)).astype(np.float32) * spread
    x *= np.where(rng.random((1, 1, heads, dim)) < 0.05, 8, 1).astype(np.float32)
    t = torch.from_numpy(x).to(TYPES[kind])
    return t.to(DEV), t.float().numpy()


def fill(cache, k, v, lens):
    cache.append(k, v, ints(lens), counts=ints(lens))


def check_contents(cache, req, k, v, n):
    """Codes, scales and tail of one request bit for bit."""
    held = cache.to_tensors()
    for name, x in (("k", k), ("v", v)):
        codes, scales, rest, values = u.contents(x[:n])
        whole = n // u.BLOCK
        got = held[name][req, :, :whole].cpu().numpy()
        tail = held[name + "_tail"][req, :, whole % 2].cpu().numpy()
        if name == "v":
            got, tail = got.swapaxes(-1, -2), tail.swapaxes(-1, -2)
        assert np.array_equal(got, codes), name
        assert np.array_equal(held[name + "_scale"][req, :, :whole].cpu().numpy(), scales, equal_nan=True), name
        assert np.array_equal(tail[:, :n % u.BLOCK].view(np.uint16), rest.view(np.uint16)), name


PIECES = [[1] * 3 + [60, 1, 1, 130, 200, 64, 129, 2], [64, 63, 1, 192], [700], [50, 150, 14, 128, 65]]


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_contents_do_not_depend_on_the_pieces(dim, kind):
    req, heads = 4, 3
    total = max(sum(p) for p in PIECES)
    k, kn = data(dim, req, total, heads, dim, kind)
    v, vn = data(dim + 1, req, total, heads, dim, kind)
    cache = cache_of(req, heads, dim, total)
    at = [0] * req
    for i in range(max(len(p) for p in PIECES)):
        counts = [p[i] if i < len(p) else 0 for p in PIECES]
        most = max(counts)
        piece_k, piece_v = torch.full((2, req, most, heads, dim), float("nan"), dtype=k.dtype, device=DEV)   # padding is not read
        for r, n in enumerate(counts):
            piece_k[r, :n], piece_v[r, :n] = k[r, at[r]:at[r] + n], v[r, at[r]:at[r] + n]
            at[r] += n
        cache.append(piece_k, piece_v, ints(at), counts=ints(counts))
    for r in range(req):
        check_contents(cache, r, kn[r], vn[r], at[r])
    got = cache.read(ints(at), total)
    for g, x in zip(got, (kn, vn)):
        for r in range(req):
            want = np.zeros(x[r].shape)
            want[:at[r]] = u.contents(x[r][:at[r]])[3]
            assert np.array_equal(g[r].cpu().numpy(), want.astype(np.float32))


@pytest.mark.parametrize("held,new", [(0, 0), (0, 1), (63, 1), (64, 1), (0, 64), (10, 128), (63, 66), (130, 62)])
def test_every_request_new_tokens_without_counts(held, new):
    k, kn = data(3, 2, held + new + 1, 2, 64, "bf16")
    cache = cache_of(2, 2, 64, held + new + 1)
    if held:
        cache.append(k[:, :held], k[:, :held], ints([held] * 2))
    cache.append(k[:, held:held + new], k[:, held:held + new], ints([held + new] * 2))
    for r in range(2):
        check_contents(cache, r, kn[r], kn[r], held + new)


def test_strides_and_unaligned_tokens():
    req, n, heads, dim = 2, 150, 3, 64
    base, basen = data(5, req, n, heads, dim, "f16")
    fused = torch.zeros(req, n, 3 * heads * dim + 1, dtype=torch.float16, device=DEV)      # rows at odd places
    fused[:, :, 1:heads * dim + 1] = base.flatten(2)
    by_head = base.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    odd = fused[:, :, 1:heads * dim + 1].unflatten(2, (heads, dim))
    assert odd.stride(1) % 8 and not by_head.is_contiguous()
    for k, v in ((odd, by_head), (by_head, odd), (by_head, by_head), (base[:1].expand(2, -1, -1, -1), base)):
        cache = cache_of(req, heads, dim, n)
        cache.append(k, v, ints([n] * req))
        for r in range(req):
            check_contents(cache, r, k[r].float().cpu().numpy(), basen[r], n)


def test_requests_that_do_not_fit_are_left_as_they_are():
    cache = cache_of(6, 2, 32, 128)
    k, _ = data(7, 6, 70, 2, 32, "f32")
    was = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.k_tail, cache.v_tail)]
    # fewer held than new; beyond the blocks; no new ones; negative; more than the batch has; negative length
    cache.append(k, k, ints([5, 129, 64, 64, 128, -3]), counts=ints([6, 70, 0, -1, 71, 1]))
    for a, b in zip(was, (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.k_tail, cache.v_tail)):
        assert torch.equal(torch.nan_to_num(a.float(), nan=-7), torch.nan_to_num(b.float(), nan=-7))


def test_ties_zeros_infinities_and_nan():
    dim, x = 32, np.zeros((320, 1, 32), dtype=np.float32)
    # block 0: scale 1 / 127 * 127 = 1 exactly, values on half steps; block 1: zeros; block 2: an infinity; block 3: a NaN
    x[:64, 0] = (np.arange(64 * dim).reshape(64, dim) % 253 - 126) / 2
    x[5, 0, 3] = 127
    x[130, 0, 1], x[131, 0, 2], x[132, 0, 0] = np.inf, -np.inf, 1e30
    x[200, 0, 4], x[201, 0, 4] = np.nan, 3
    x[256:, 0] = np.random.default_rng(1).standard_normal((64, dim)) * 6e-8        # halves at the end of their range
    k = torch.from_numpy(x)[None].to(DEV)
    cache = cache_of(1, 1, dim, 320)
    cache.append(k, k, ints([320]))
    check_contents(cache, 0, x, x, 320)
    got = cache.read(ints([320]), 320)[0][0].cpu().numpy()
    assert np.isnan(got[192:256]).all() and np.isfinite(np.delete(got, slice(192, 256), 0)).all()
    assert got[130, 0, 1] == 65504 and got[131, 0, 2] == -65504 and got[132, 0, 0] == 65504
    # in the tail a NaN stays one value
    cache = cache_of(1, 1, dim, 320)
    cache.append(k[:, 192:202], k[:, 192:202], ints([10]))
    assert np.isnan(cache.read(ints([10]), 10)[1].cpu().numpy()).sum() == 1


def test_scales_that_do_not_divide_exactly_pick_the_nearest_code():
    """Every half against scales where value / scale comes closest to a border between two codes."""
    rng = np.random.default_rng(11)
    tops = rng.integers(0x0400, 0x7bff, 200).astype(np.uint16).view(np.float16).astype(np.float64)
    x = np.zeros((200 * 64, 1, 32), dtype=np.float32)
    for b, top in enumerate(tops):
        scale = np.float64(np.float32(top / 127))
        n = rng.integers(0, 127, 64 * 32)
        near = np.float16((n + 0.5) * scale)                   # the half next to the border, on either side of it
        x[b * 64:(b + 1) * 64, 0] = np.clip(near.astype(np.float64), -top, top).reshape(64, 32)
        x[b * 64, 0, 0] = top
    k = torch.from_numpy(x)[None].to(DEV)
    cache = cache_of(1, 1, 32, len(x))
    cache.append(k, -k, ints([len(x)]))
    check_contents(cache, 0, x, -x, len(x))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("first,n", [(None, 1), ([0, 63, 64], 65), ([130, 0, 500], 200), ([-5, 199, 200], 1), ([7, 70, 190], 0)])
def test_read_ranges(kind, first, n):
    lens = [200, 64, 0]
    k, kn = data(13, 3, 200, 2, 96, "f32", spread=30)
    cache = cache_of(3, 2, 96, 256)
    fill(cache, k, -k, lens)
    got = cache.read(ints(lens), n, first=None if first is None else ints(first), dtype=TYPES[kind])
    assert got[0].shape == (3, n, 2, 96) and got[0].dtype == TYPES[kind]
    for r in range(3):
        at = 0 if first is None else max(first[r], 0)
        all_ = np.zeros((1000, 2, 96))
        all_[:lens[r]] = u.contents(kn[r, :lens[r]])[3]
        want = torch.from_numpy(all_[at:at + n].astype(np.float32)).to(TYPES[kind])
        assert torch.equal(got[0][r].cpu(), want) and torch.equal(got[1][r].cpu(), -want)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def check_attention(kind, lens, rows, heads, kv, dim, row_limit=None, tags=None, scale=None, q_spread=2.0, max_len=0, seed=0,
                    room=0, strided=False):
    req, most = len(lens), max(max(lens), 1)
    k, kn = data(seed + 1, req, most, kv, dim, "f32")
    v, vn = data(seed + 2, req, most, kv, dim, "f32")
    cache = cache_of(req, kv, dim, most + room)
    fill(cache, k, v, lens)
    q, qn = data(seed + 3, req, rows, heads, dim, kind, spread=q_spread)
    if strided:
        wide = torch.zeros(req, rows, heads, dim + 1, dtype=q.dtype, device=DEV)
        wide[..., 1:] = q
        q = wide[..., 1:]
    key_tag = row_tag = None
    if tags is not None:
        kt = np.zeros((req, cache.n_block * 64), dtype=np.uint16)
        for r in range(req):
            kt[r, :lens[r]] = tags[0][r][:lens[r]]
            kt[r, lens[r]:] = 0
        key_tag, row_tag = torch.from_numpy(kt).to(DEV), ints(tags[1])
    out, lse = cache.attention(q, ints(lens), row_limit=None if row_limit is None else ints(row_limit), key_tag=key_tag,
                               row_tag=row_tag, scale=scale, max_len=max_len, with_lse=True)
    assert out.shape == q.shape and out.dtype == TYPES[kind]
    out, lse = out.float().cpu().numpy(), lse.cpu().numpy()
    for r in range(req):
        n = lens[r]
        sees = np.ones((rows, n), dtype=bool)
        if row_limit is not None:
            sees &= np.arange(n)[None] < np.array(row_limit[r])[:, None]
        if tags is not None:
            sees &= np.array(tags[0][r])[None, :n].astype(int) <= np.array(tags[1][r])[:, None]
        kk, vv = u.contents(kn[r, :n])[3], u.contents(vn[r, :n])[3]
        want, wl, mag, scores = u.attend(qn[r].astype(np.float64), kk, vv, sees, 1 / math.sqrt(dim) if scale is None else scale)
        tol, tl = u.tolerance(kind, want, mag, scores, dim, n, np.abs(vv).max(initial=0))
        bad = np.abs(out[r] - want) - tol
        assert not (bad > 0).any() and np.isfinite(out[r]).all(), (r, bad.max(), np.abs(out[r] - want).max())
        none = ~sees.any(axis=1)
        assert (out[r][none] == 0).all() and np.isneginf(lse[r][none]).all()
        assert (np.abs(lse[r][~none] - wl[~none]) <= tl[~none]).all()
    return cache


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,heads,kv", [(1, 2, 2), (5, 6, 2), (17, 3, 3), (70, 2, 1)])
def test_attention(dim, kind, rows, heads, kv):
    check_attention(kind, [333, 64, 1, 0, 200], rows, heads, kv, dim, seed=dim + rows)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 1000, 4097])
@pytest.mark.parametrize("kind,dim", [("f32", 128), ("bf16", 64), ("f16", 96)])
def test_attention_lengths(n, kind, dim):
    check_attention(kind, [n, n - 1], 3, 2, 1, dim, seed=n)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n", [(40, 40), (100, 333), (33, 129), (300, 300), (64, 70)])
def test_attention_causal_piece(kind, rows, n):
    lens = [n, max(n - 25, 1)]
    limits = [[max(m - rows + i + 1, 0) for i in range(rows)] for m in lens]
    check_attention(kind, lens, rows, 4, 2, 64, row_limit=limits, seed=rows)


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_attention_subsequences_limits_and_rows_that_see_nothing(dim, kind):
    rng = np.random.default_rng(dim)
    lens, rows = [700, 65, 130], 6
    tags = [np.concatenate([np.zeros(n // 2), rng.integers(1, rows + 1, n - n // 2)]).astype(np.uint16) for n in lens]
    tags[1][:] = 3                                             # rows 1 and 2 of this request see nothing
    limits = [[700, 0, -4, 10, 10 ** 9, 351], [65] * 6, [130, 64, 65, 1, 129, 2]]
    check_attention(kind, lens, rows, 4, 4, dim, row_limit=limits, tags=(tags, [[1, 2, 3, 4, 5, 6]] * 3), seed=1)
    tags = [t.copy() for t in tags]
    tags[2][:] = 65535                                         # the largest tag, and rows that see only it, or all but it
    check_attention(kind, lens, rows, 4, 4, dim, tags=(tags, [[0, 1, 2, 3, 4, 5], [-1, 0, 3, 2, 65535, 70000],
                                                              [65534, 65535, 1, 0, 65536, 2]]), seed=2)


LENS28 = [0, 1, 2, 31, 63, 64, 65, 90, 127, 128, 129, 130, 150, 190, 191, 192, 193, 200, 255, 256, 257, 320, 333, 64, 5, 128, 448, 100]


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("rows,heads,kv,strided", [(100, 8, 8, False), (130, 4, 4, True), (50, 24, 8, False)])
def test_attention_pieces_that_fill_the_chip(dim, rows, heads, kv, strided):
    """Half queries, 128 columns to a work-group: ragged requests, causal limits with rows that see nothing, grouped heads."""
    limits = [[max(n - rows + i + 1 - 3 * (r % 2), 0) for i in range(rows)] for r, n in enumerate(LENS28)]
    check_attention("f16", LENS28, rows, heads, kv, dim, row_limit=limits, strided=strided, seed=dim, room=70)


@pytest.mark.parametrize("dim", [64, 128])
def test_attention_pieces_that_fill_the_chip_by_tags(dim):
    rows, rng = 100, np.random.default_rng(8)
    tags = [[int(x) for x in np.sort(rng.integers(0, 5, max(n, 1)))] for n in LENS28]
    check_attention("f16", LENS28, rows, 8, 8, dim, tags=(tags, [[i % 6 - 1 for i in range(rows)] for _ in LENS28]), scale=-0.2, seed=3)
    check_attention("f16", [200] * 28, rows, 8, 8, dim, max_len=230, seed=4)


def test_attention_pieces_that_fill_the_chip_keep_nan_where_it_is():
    k, _ = data(96, 28, 190, 8, 64, "f16")
    q, _ = data(97, 28, 100, 8, 64, "f16")
    limit = ints([[64 if i < 30 else 128 if i < 60 else 190 for i in range(100)]] * 28)
    lens, out = ints([190] * 28), []
    for bad in (False, True):
        kk, vv, qq = k.clone(), k.flip(1).contiguous(), q.clone()
        if bad:
            kk[3, 100, 2, 5] = vv[4, 70, 1, 7] = vv[5, 150, 0, 9] = qq[6, 40, 3, 1] = float("nan")
            qq[7, 50, 4, 2] = float("inf")
        cache = cache_of(28, 8, 64, 200)
        cache.append(kk, vv, lens)
        out.append(cache.attention(qq, lens, row_limit=limit))
    moved = (out[0] != out[1]).any(dim=3)
    want = torch.zeros_like(moved)
    want[3, 30:, 2] = want[4, 30:, 1] = want[5, 60:, 0] = want[6, 40, 3] = want[7, 50, 4] = True
    assert torch.equal(moved, want)
    assert torch.isnan(out[1][3, 30:, 2]).all() and torch.isnan(out[1][6, 40, 3]).all() and torch.isnan(out[1][7, 50, 4]).all()
    assert torch.isnan(out[1][5, 60:, 0, 9]).all()


def test_attention_few_rows_of_long_caches_are_split():
    check_attention("f32", [5000, 3], 2, 2, 2, 128, seed=4)
    check_attention("bf16", [9000], 8, 4, 4, 64, seed=5)
    check_attention("f16", [70, 6001], 1, 8, 1, 96, seed=6)
    check_attention("f16", [70, 601], 1, 8, 1, 96, seed=6, max_len=601, room=20000)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_attention_scales_and_magnitudes(kind):
    check_attention(kind, [150], 2, 2, 2, 64, scale=0.0)
    check_attention(kind, [150], 2, 2, 2, 64, scale=-0.3)
    check_attention(kind, [150], 2, 2, 2, 64, scale=1e-3, q_spread=2000.0)
    check_attention(kind, [150], 2, 2, 2, 64, scale=30.0, q_spread=2e-3)
    if kind != "f16":
        check_attention(kind, [150], 2, 2, 2, 64, scale=1e30, q_spread=1e-31)
        check_attention(kind, [150], 2, 2, 2, 64, scale=1e-30, q_spread=1e30)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_attention_strided_queries(kind):
    check_attention(kind, [300, 20], 4, 6, 3, 96, strided=True)


def test_unseen_nan_and_infinities_stay_out():
    """A NaN in block 1 and in the tail: rows that see nothing of their block are what they would be without them."""
    dim, n = 64, 200
    k, _ = data(21, 1, n, 2, dim, "f32")
    v, _ = data(22, 1, n, 2, dim, "f32")
    bad_k, bad_v = k.clone(), v.clone()
    bad_k[0, 70, 0, 5], bad_v[0, 80, 1, 6] = float("nan"), float("inf")
    bad_v[0, 90, 0, 6], bad_v[0, 195, 1, 2], bad_k[0, 199, 0, 0] = float("nan"), float("nan"), float("inf")
    q, _ = data(23, 1, 4, 2, dim, "f32")
    limits = ints([[64, 64, 10, 128]])
    key_tag = torch.zeros(1, 256, dtype=torch.int32, device=DEV)
    key_tag[0, 64:] = 2
    for kw in (dict(row_limit=limits), dict(key_tag=key_tag.to(torch.uint16), row_tag=ints([[1, 1, 0, 2]]))):
        outs = []
        for kk, vv in ((k, v), (bad_k, bad_v)):
            cache = cache_of(1, 2, dim, 256)
            cache.append(kk, vv, ints([n]))
            outs.append(cache.attention(q, ints([n]), **kw))
        assert torch.equal(outs[0][:, :3], outs[1][:, :3])
        assert torch.isnan(outs[1][0, 3, 0]).all()             # this row sees the block with NaN in its keys and values


def test_queries_that_are_no_numbers_stay_in_their_row():
    cache = cache_of(1, 1, 64, 300)
    k, _ = data(31, 1, 300, 1, 64, "f32")
    cache.append(k, k, ints([300]))
    q, _ = data(32, 1, 5, 1, 64, "f32")
    bad = q.clone()
    bad[0, 1, 0, 7], bad[0, 3, 0, 0] = float("nan"), float("inf")
    a, b = cache.attention(q, ints([300])), cache.attention(bad, ints([300]))
    assert torch.equal(a[:, [0, 2, 4]], b[:, [0, 2, 4]]) and torch.isnan(b[0, 1]).all() and torch.isnan(b[0, 3]).all()


def test_rows_and_requests_do_not_depend_on_the_batch():
    """The same request alone, and among others: the same numbers where the launch has the same shape, within tolerance else."""
    cache = cache_of(3, 2, 64, 500)
    k, kn = data(41, 3, 500, 2, 64, "f16")
    fill(cache, k, k, [500, 17, 129])
    q, _ = data(42, 3, 2, 2, 64, "f16")
    whole = cache.attention(q, ints([500, 17, 129]))
    for lens in ([500, 0, 129], [500, 500, 129]):
        if lens[1] == 500:
            cache.append(k[:, 17:], k[:, 17:], ints(lens), counts=ints([0, 483, 0]))
        again = cache.attention(q, ints(lens))
        assert torch.equal(whole[0], again[0]) and torch.equal(whole[2], again[2])


def test_store_attend_read_as_a_program_does_captured_and_replayed():
    """A prompt, then tokens one by one from a graph that appends, attends and counts by itself, with other work in between."""
    req, heads, kv, dim, start, steps = 2, 4, 2, 128, 61, 9
    total = start + steps
    k, kn = data(51, req, total, kv, dim, "bf16")
    v, vn = data(52, req, total, kv, dim, "bf16")
    q, qn = data(53, req, total, heads, dim, "bf16")
    cache = cache_of(req, kv, dim, total)
    cache.append(k[:, :start], v[:, :start], ints([start] * req))
    lens = ints([start] * req)
    tok = [x[:, :1].clone() for x in (k, v, q)]

    def step():
        lens.add_(1)
        cache.append(tok[0], tok[1], lens)
        return cache.attention(tok[2], lens), cache.read(lens, 3, first=lens - 2)

    side = torch.cuda.Stream()
    saved = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.k_tail, cache.v_tail)]
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        step()
        lens.fill_(start)
        for t, w in zip((cache.k, cache.v, cache.k_scale, cache.v_scale, cache.k_tail, cache.v_tail), saved):
            t.copy_(w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, back = step()
    for i in range(start, total):
        for t, x in zip(tok, (k, v, q)):
            t.copy_(x[:, i:i + 1])
        graph.replay()
        torch.cuda.synchronize()
        other = torch.ones(1000, device=DEV).sum()
        for r in range(req):
            check_contents(cache, r, kn[r], vn[r], i + 1)
            kk, vv = u.contents(kn[r, :i + 1])[3], u.contents(vn[r, :i + 1])[3]
            want, _, mag, scores = u.attend(qn[r, i:i + 1].astype(np.float64), kk, vv, np.ones((1, i + 1), bool), dim ** -0.5)
            tol, _ = u.tolerance("bf16", want, mag, scores, dim, i + 1, np.abs(vv).max())
            assert (np.abs(out[r].float().cpu().numpy() - want) <= tol).all()
            assert np.array_equal(back[0][r, :2].cpu().numpy(), kk[i - 1:].astype(np.float32))
            assert (back[0][r, 2] == 0).all()
        assert int(other) == 1000 and lens.tolist() == [i + 1] * req


def test_two_streams_at_once_have_workspaces_of_their_own():
    a = cache_of(1, 2, 64, 6000)
    k, _ = data(61, 1, 6000, 2, 64, "f16")
    a.append(k, k, ints([6000]))
    q, _ = data(62, 8, 1, 2, 64, "f16")
    lens = ints([6000])
    want = [a.attention(q[i:i + 1], lens) for i in range(8)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None] * 8
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(8):
            with torch.cuda.stream(streams[i % 2]):
                got[i] = a.attention(q[i:i + 1], lens)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, got))


def test_offsets_beyond_32_bits():
    """One request with 2^25 tokens: codes of 4 GiB, tags of 64 MiB; only the last 100 tokens and one at the start are seen."""
    from paper_2506_23431_amd import ByteCache
    dim, n_block = 128, 2 ** 19 + 1
    n = n_block * 64 - 30
    cache = ByteCache(1, 1, dim, n_block * 64, device=DEV)
    cache.k_scale.fill_(1), cache.v_scale.fill_(1)
    k, kn = data(71, 1, 300, 1, dim, "f32")
    v, vn = data(72, 1, 300, 1, dim, "f32")
    cache.append(k[:, :64], v[:, :64], ints([64]))
    at = (n - 136) // 64 * 64
    cache.append(k[:, 64:64 + n - at], v[:, 64:64 + n - at], ints([n]))
    m = 64 + n - at
    held = [np.concatenate([u.contents(x[0, :64])[3], u.contents(x[0, 64:m])[3]]) for x in (kn, vn)]
    got = cache.read(ints([n]), n - at, first=ints([at]))
    assert np.array_equal(got[0][0].cpu().numpy(), held[0][64:].astype(np.float32))
    assert np.array_equal(got[1][0].cpu().numpy(), held[1][64:].astype(np.float32))
    tag = torch.ones(1, n_block * 64, dtype=torch.uint8, device=DEV)
    tag[0, 5] = 0
    tag[0, n - 100:] = 0
    tag = tag.to(torch.uint16)
    q, qn = data(73, 1, 1, 2, dim, "f32")
    out = cache.attention(q, ints([n]), key_tag=tag, row_tag=ints([[0]]))
    sees = np.zeros((1, m), dtype=bool)
    sees[0, 5], sees[0, m - 100:] = True, True
    want, _, mag, scores = u.attend(qn[0].astype(np.float64), held[0], held[1], sees, dim ** -0.5)
    tol, _ = u.tolerance("f32", want, mag, scores, dim, 2048, np.abs(held[1]).max())
    assert (np.abs(out[0].cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
def test_plain_tensors_go_in_and_come_out(dim):
    """A cache made from plain codes reads as code times scale, and gives the same tensors back."""
    from paper_2506_23431_amd import ByteCache
    rng = np.random.default_rng(dim)
    plain = {"k": rng.integers(-127, 128, (2, 3, 4, 64, dim)).astype(np.int8),
             "v": rng.integers(-127, 128, (2, 3, 4, dim, 64)).astype(np.int8),
             "k_scale": rng.random((2, 3, 4)).astype(np.float32), "v_scale": rng.random((2, 3, 4)).astype(np.float32),
             "k_tail": rng.standard_normal((2, 3, 2, 64, dim)).astype(np.float16),
             "v_tail": rng.standard_normal((2, 3, 2, dim, 64)).astype(np.float16)}
    cache = ByteCache.from_tensors(**{n: torch.from_numpy(x).to(DEV) for n, x in plain.items()})
    for n, t in cache.to_tensors().items():
        assert np.array_equal(t.cpu().numpy(), plain[n]), n
    lens = [200, 129]
    k, v = cache.read(ints(lens), 200)
    for r, n in enumerate(lens):
        whole = n // 64
        want_k = (plain["k"][r].astype(np.float32) * plain["k_scale"][r][..., None, None]).astype(np.float32)
        want_v = (plain["v"][r].astype(np.float32) * plain["v_scale"][r][..., None, None]).astype(np.float32).swapaxes(-1, -2)
        for got, want, tail in ((k, want_k, plain["k_tail"][r, :, whole % 2]),
                                (v, want_v, plain["v_tail"][r, :, whole % 2].swapaxes(-1, -2))):
            flat = np.concatenate([want[:, :whole].reshape(3, whole * 64, dim), tail[:, :n - whole * 64].astype(np.float32)], axis=1)
            assert np.array_equal(got[r, :n].cpu().numpy(), flat.transpose(1, 0, 2))
            assert (got[r, n:] == 0).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_tokens_and_queries_that_repeat_along_an_axis(kind):
    """Strides of zero: one token for all heads, one prompt for all requests, one query for all rows and heads."""
    x, _ = data(91, 1, 150, 1, 64, kind)
    for shown in (x.expand(2, 150, 3, 64), x[:, :1].expand(2, 150, 3, 64)):
        caches = [cache_of(2, 3, 64, 200) for _ in range(2)]
        caches[0].append(shown, -shown, ints([150, 150]))
        caches[1].append(shown.contiguous(), (-shown).contiguous(), ints([150, 150]))
        q = x[:, 3:4].expand(2, 20, 6, 64)
        outs = [c.attention(y, ints([150, 149]), with_lse=True) for c in caches for y in (q, q.contiguous())]
        assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(outs[0], o))
        assert all(torch.equal(a, b) for a, b in zip(*(c.read(ints([150, 150]), 150) for c in caches)))


@pytest.mark.parametrize("rows", [1, 40])
def test_lengths_beyond_what_there_is(rows):
    """Lengths above the room count as the room, below zero as zero; what lies behind max_len may be left out, in whole blocks."""
    k, _ = data(92, 2, 256, 2, 64, "bf16")
    cache = cache_of(2, 2, 64, 256)
    cache.append(k, k, ints([256, 256]))
    q, _ = data(93, 2, rows, 2, 64, "bf16")
    want = cache.attention(q, ints([256, 256]))
    for lens in ([257, 1 << 30], [256, (1 << 31) - 1]):
        assert torch.equal(cache.attention(q, ints(lens)), want)
        assert torch.equal(cache.read(ints(lens), 300)[0], cache.read(ints([256, 256]), 300)[0])
    for lens in ([-1, -(1 << 31)], [0, -64]):
        out, lse = cache.attention(q, ints(lens), with_lse=True)
        assert (out == 0).all() and torch.isneginf(lse).all() and (cache.read(ints(lens), 70)[1] == 0).all()
    assert torch.equal(cache.attention(q, ints([256, 200]), max_len=100), cache.attention(q, ints([128, 128]), max_len=128))
    limit = torch.full((2, rows), 1 << 30, dtype=torch.int32, device=DEV)
    assert torch.equal(cache.attention(q, ints([256, 256]), row_limit=limit), want)
    assert (cache.attention(q, ints([256, 256]), row_limit=-limit) == 0).all()


@pytest.mark.parametrize("rows", [1, 40])
def test_tags_at_the_ends_of_their_range(rows):
    k, _ = data(94, 1, 130, 1, 32, "bf16")
    cache = cache_of(1, 1, 32, 192)
    cache.append(k, k, ints([130]))
    q, _ = data(95, 1, rows, 1, 32, "bf16")
    tags = np.full((1, 192), 65535, dtype=np.uint16)
    tags[:, :70] = 32768
    tags = torch.from_numpy(tags).to(DEV)

    def seen(tag):
        return cache.attention(q, ints([130]), key_tag=tags, row_tag=torch.full((1, rows), tag, dtype=torch.int32, device=DEV))
    everything, first = cache.attention(q, ints([130])), cache.attention(q, ints([130]), row_limit=torch.full((1, rows), 70, dtype=torch.int32, device=DEV))
    for tag, want in ((65535, everything), ((1 << 31) - 1, everything), (65534, first), (32768, first)):
        assert torch.equal(seen(tag), want), tag
    for tag in (32767, 0, -1, -(1 << 31)):
        assert (seen(tag) == 0).all(), tag


def test_refusals_of_the_binding():
    from paper_2506_23431_amd import ByteCache, PdError
    cache = cache_of(2, 2, 64, 128)
    k, _ = data(81, 2, 3, 2, 64, "f32")
    lens = ints([3, 3])
    for call in (lambda: cache.append(k, k.half(), lens), lambda: cache.append(k[:1], k[:1], lens),
                 lambda: cache.append(k.double(), k.double(), lens), lambda: cache.append(k.cpu(), k.cpu(), lens),
                 lambda: cache.append(k, k, lens.long()), lambda: cache.append(k, k, lens[:1]),
                 lambda: cache.append(k, k, lens, counts=lens.cpu()), lambda: cache.append(k.transpose(2, 3), k, lens),
                 lambda: cache.append(k.repeat(1, 50, 1, 1), k.repeat(1, 50, 1, 1), lens),
                 lambda: cache.read(lens, -1), lambda: cache.read(lens, 3, dtype=torch.float64),
                 lambda: cache.read(lens, 3, first=lens.long()),
                 lambda: cache.attention(k[:, :, :1], lens), lambda: cache.attention(k, lens, key_tag=torch.zeros(2, 128, dtype=torch.uint16, device=DEV)),
                 lambda: cache.attention(k, lens, row_limit=lens), lambda: cache.attention(k, lens, scale=float("nan")),
                 lambda: cache.attention(k, lens, scale=float("inf")), lambda: cache.attention(k, lens, max_len=-1),
                 lambda: cache.attention(k[..., :32], lens), lambda: cache.attention(k.cpu(), lens),
                 lambda: ByteCache(1, 1, 48, 64), lambda: ByteCache(0, 1, 64, 64), lambda: ByteCache(1, 1, 64, 0),
                 lambda: ByteCache(1, 1, 64, 64, device="cpu"),
                 lambda: ByteCache.from_tensors(**{**cache.to_tensors(), "v": cache.v}),
                 lambda: ByteCache.from_tensors(**{**cache.to_tensors(), "k_scale": cache.k_scale.half()}),
                 lambda: ByteCache.from_tensors(**{n: t.cpu() for n, t in cache.to_tensors().items()})):
        with pytest.raises(PdError):
            call()
    # no rows, no tokens: nothing to do
    assert cache.attention(k[:, :0], lens).shape == (2, 0, 2, 64) and cache.read(lens, 0)[0].shape == (2, 0, 2, 64)
