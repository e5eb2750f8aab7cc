"""The cache in 8 bits on the GPU, against the oracle in 64 bits: decode attention over codes, storing whole slabs and appended rows, and
the way back to bf16."""
import numpy as np
import pytest
import torch

import oracle
from q8_common import Cache, bf16, random_slab

pytestmark = pytest.mark.gpu
FORMATS = ["e4m3", "int8"]


@pytest.fixture(scope="module")
def B():
    from paper_2512_07993_b200 import binding, build
    build.build()
    return binding


# ------------------------------------------------------------------ decode attention
def filled(B, lens, caps, hk, fmt, block, paged, seed, general=False, sigma=1.0, **kw):
    c = Cache(B, lens, caps, hk, fmt, block, paged, seed, **kw)
    codes, scales = ([], []), ([], [])
    for s in range(c.slabs):
        for i in range(2):
            x, f = random_slab(c.r, int(c.lens.reshape(-1)[s]), block, fmt, sigma, general)
            codes[i].append(x)
            scales[i].append(f)
    c.put(codes, scales)
    c.rows64 = [[oracle.q8_rows(codes[i][s], scales[i][s], len(codes[i][s]), block, fmt) for s in range(c.slabs)] for i in range(2)]
    return c


def check_attention(c, q, out, only=None):
    """out against 64 bits.  Bound: a logit of the 128 products q k is off by at most 2^-23 (128 + 8) sum |q k| / sqrt(d) =: e (sums of
    32 bits that may truncate, a few factors), so a probability by 2 e + 2^-19 relative (exponential, two parts of 22 bits, sums over up to
    some thousand rows of which 64 lie in one chain), the result by that times sum p |v|, and its rounding to bf16 by 2^-8 of it.  Small
    probabilities have an absolute floor: 2^15 p goes in as two f16 parts, whose last rounding is half of the smallest f16 (2^-25), so
    p, relative to the largest one, is off by up to 2^-40, and the result by 2^-40 sum |v|."""
    n = q.shape[1] // c.hk
    q64, got = q.double().cpu().numpy(), out.double().cpu().numpy()
    for s in range(c.slabs) if only is None else only:
        b, h = divmod(s, c.hk)
        K, V = c.rows64[0][s], c.rows64[1][s]
        for j in range(n):
            qq = q64[b, h * n + j][None]
            want = oracle.attn_rows(qq, K, V)[0]
            mine = got[b, h * n + j]
            if len(K) == 0:
                assert (mine == 0).all()
                continue
            e = 2.0 ** -23 * 136 * (np.abs(qq) @ np.abs(K).T).max() / np.sqrt(128)
            room = 2.0 ** -8 * np.abs(want) + (2 * e + 2.0 ** -19) * oracle.attn_rows(qq, K, np.abs(V))[0] + 2.0 ** -40 * np.abs(V).sum(0)
            far = float((np.abs(mine - want) / np.maximum(room, 1e-300)).max())
            assert far <= 1, (s, j)


def queries(c, nq, seed, scale=1.0):
    return bf16(np.random.default_rng(seed).normal(0, scale, (c.bt, nq, 128))).cuda()


def attend(c, q, **kw):
    out = torch.full_like(q, float("nan"))
    c.B.skipkv_decode_attn_q8(c.shape, c.cache, q, c.kv_len, out, kw.get("hidden"), kw.get("vec"), kw.get("alpha"), kw.get("flag"), c.ws,
                              kw.get("stream"))
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 6, 7, 8])
def test_attention(B, fmt, paged, group):
    """Lengths around the rows of a warp and of a page, none and one among them, other ones in every head."""
    lens = [[0, 1, 15], [16, 17, 127], [128, 129, 300], [1000, 2, 255]]
    c = filled(B, lens, [16, 131, 333, 1003], 3, fmt, [16, 32, 64, 128][group % 4], paged, group, n_q=3 * group)
    q = queries(c, 3 * group, 40 + group)
    out = attend(c, q)
    assert c.status() == 0
    check_attention(c, q, out)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("block", [16, 128])
def test_attention_over_slabs_of_many_blocks(B, fmt, paged, block):
    """Slabs that are split over many CTAs, with scales that are no powers of two."""
    c = filled(B, [[40000], [9001]], [40003, 9001], 1, fmt, block, paged, 3, general=True, n_q=4)
    q = queries(c, 4, 5)
    check_attention(c, q, attend(c, q))
    assert c.status() == 0


def test_attention_over_more_slabs_than_blocks(B):
    lens = np.random.default_rng(1).integers(0, 70, (150, 8))
    c = filled(B, lens, [70] * 150, 8, "e4m3", 32, False, 2, n_q=16)
    q = queries(c, 16, 6)
    check_attention(c, q, attend(c, q))
    c.kv_len.zero_()
    c.rows64 = [[x[:0] for x in y] for y in c.rows64]
    check_attention(c, q, attend(c, q))


@pytest.mark.parametrize("paged", [False, True])
def test_many_slabs_replayed_with_other_lengths_and_steered(B, paged):
    """The table of the slabs belongs to a call: a captured one makes it anew from the lengths that it finds."""
    r = np.random.default_rng(3)
    c = filled(B, r.integers(0, 260, (150, 8)), [260] * 150, 8, "int8", 32, paged, 2, n_q=40, d_model=64)
    q, out = queries(c, 40, 6), torch.zeros(150, 40, 128, dtype=torch.bfloat16, device="cuda")
    start, vec = bf16(r.normal(0, 1, (150, 64))).cuda(), bf16(r.normal(0, 1, 64)).cuda()
    alpha, flag = torch.from_numpy(r.random(150).astype(np.float32)).cuda(), torch.from_numpy(r.integers(0, 2, 150).astype(np.uint8)).cuda()
    want, hidden = start.clone(), start.clone()
    B.skipkv_steer(150, 64, want, vec, alpha, flag)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.skipkv_decode_attn_q8(c.shape, c.cache, q, c.kv_len, out, hidden, vec, alpha, flag, c.ws)
    full = c.kv_len.clone()
    for lens in (full, torch.zeros_like(full), full // 2, full * (torch.arange(1200, device="cuda").view(150, 8) % 97 == 0).int()):
        c.kv_len.copy_(lens)
        out.fill_(float("nan"))
        hidden.copy_(start)
        g.replay()
        torch.cuda.synchronize()
        assert c.status() == 0 and torch.equal(hidden, want) and torch.equal(out, attend(c, q))
        n = lens.view(-1).tolist()
        d, c.rows64 = c.rows64, [[x[:k] for x, k in zip(y, n)] for y in c.rows64]
        check_attention(c, q, out, only=range(0, 1200, 97))
        c.rows64 = d


@pytest.mark.parametrize("paged", [False, True])
def test_attention_where_few_of_many_slabs_have_rows(B, paged):
    """A block's range goes from one slab over hundreds of empty ones to the next."""
    lens = np.zeros((700, 2), np.int64)
    for s, n in ((3, 20000), (4, 1), (5, 129), (300, 40000), (301, 700), (1000, 5), (1007, 128), (1398, 9000), (1399, 1)):
        lens[s // 2, s % 2] = n
    caps = np.maximum(lens.max(1), 1)
    c = filled(B, lens, caps, 2, "e4m3", 64, paged, 2, n_q=4)
    q = queries(c, 4, 6)
    check_attention(c, q, attend(c, q))
    assert c.status() == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("q_size,sigma", [(0.0, 1.0), (1e30, 1e-30), (1e-30, 1e30), (2e4, 2.0 ** -9), (1e-38, 1.0), (30.0, 1.0)])
def test_attention_over_extreme_magnitudes(B, fmt, q_size, sigma):
    """Queries and keys of any size whose products are ordinary; one with peaked softmax; zero queries."""
    c = filled(B, [[600, 77]], [600], 2, fmt, 16, False, 9, sigma=sigma, n_q=6)
    q = queries(c, 6, 7, q_size)
    if q_size == 2e4:
        q[0, 0, ::2] *= 2.0 ** -25                        # small elements beside large ones
    check_attention(c, q, attend(c, q))


def test_attention_with_a_nan_in_one_head(B):
    """A live NaN comes out in the heads that meet it and nowhere else."""
    c = filled(B, [[200, 200]], [200], 2, "e4m3", 16, False, 9, n_q=8)
    c.V[c.places(0, 200)[0][33], 5] = 0x7f
    q = queries(c, 8, 7)
    out = attend(c, q).float()
    assert bool(torch.isnan(out[0, :4, 5]).all()) and int(torch.isnan(out).sum()) == 4


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_attention_with_a_query_that_is_not_finite(B, fmt, value):
    """Its head is NaN, as the products would make it; the others are what they are."""
    c = filled(B, [[200, 200]], [200], 2, fmt, 16, False, 9, n_q=12)
    q = queries(c, 12, 7)
    q[0, 4, 17] = value
    out = attend(c, q)
    assert bool(torch.isnan(out[0, 4].float()).all())
    q[0, 4, 17] = 0
    keep = torch.arange(12, device="cuda") != 4
    assert torch.equal(out[:, keep], attend(c, q)[:, keep])


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_over_as_many_slabs_as_there_may_be(B, fmt):
    lens = np.random.default_rng(1).integers(0, 4, (1024, 8))
    c = Cache(B, lens, [3] * 1024, 8, fmt, 16, False, 2, n_q=8)
    x = values(c.r, c.rows16).cuda()
    B.skipkv_pack_q8(c.shape, c.cache, x, x, c.kv_len, c.ws)
    back = torch.zeros_like(x)
    B.skipkv_unpack_q8(c.shape, c.cache, c.kv_len, back, None, c.ws)
    q = queries(c, 8, 6)
    out = attend(c, q)
    assert c.status() == 0
    host = back.double().cpu().numpy()
    c.rows64 = [[host[c.row0[s]:c.row0[s] + int(lens.reshape(-1)[s])] for s in range(c.slabs)]] * 2
    check_attention(c, q, out)


@pytest.mark.parametrize("paged", [False, True])
def test_two_streams_with_a_workspace_each(B, paged):
    """Calls over two caches that run at the same time give what they give alone."""
    cs = [filled(B, [[3000, 33], [200, 1500]], [3000, 1500], 2, "e4m3", 64, paged, 20 + i, n_q=8) for i in range(2)]
    qs = [queries(c, 8, 30 + i) for i, c in enumerate(cs)]
    alone = [attend(c, q) for c, q in zip(cs, qs)]
    outs = [[torch.zeros_like(qs[i]) for _ in range(20)] for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for k in range(20):
        for i in range(2):
            B.skipkv_decode_attn_q8(cs[i].shape, cs[i].cache, qs[i], cs[i].kv_len, outs[i][k], None, None, None, None, cs[i].ws, streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert cs[i].status() == 0
        for o in outs[i]:
            assert torch.equal(o, alone[i])


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("replayed", [False, True])
def test_steps_behind_one_another_see_the_lengths_that_the_step_before_left(B, paged, replayed):
    """Append and attention without a pause, lengths that cross rows, blocks and tiles: the same bits as with a pause behind every call.  (The
    attention derives its work from the lengths before the append ahead of it has finished, and has to notice.)"""
    lens = [[120, 3], [250, 384]]
    runs = []
    for pause in (True, False):
        c = filled(B, lens, [700, 700], 2, "int8", 16, paged, 5, n_q=8)
        r = np.random.default_rng(6)
        k, v = (bf16(r.normal(0, 1, (150, 2, 2, 128)) * np.exp2(np.arange(150) % 5)[:, None, None, None]).cuda() for _ in range(2))
        q = bf16(r.normal(0, 1, (150, 2, 8, 128))).cuda()
        out = torch.zeros_like(q)
        a, b = c.kv_len.clone(), torch.zeros_like(c.kv_len)

        def step(i):
            src, dst = (a, b) if i % 2 == 0 else (b, a)
            B.skipkv_append_q8(c.shape, c.cache, k[i], v[i], None, 2, src, dst, c.ws)
            if pause:
                torch.cuda.synchronize()
            B.skipkv_decode_attn_q8(c.shape, c.cache, q[i], dst, out[i], None, None, None, None, c.ws)
            if pause:
                torch.cuda.synchronize()

        if replayed and not pause:
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                for i in range(150):
                    step(i)
            g.replay()
        else:
            for i in range(150):
                step(i)
        torch.cuda.synchronize()
        assert c.status() == 0 and (a if 150 % 2 == 0 else b).tolist() == [[n + 150 for n in x] for x in lens]
        runs.append((out, c.K.clone(), c.V.clone()))
    for x, y in zip(*runs):
        assert torch.equal(x, y)


@pytest.mark.parametrize("paged", [False, True])
def test_attention_steers_in_the_same_launch(B, paged):
    c = filled(B, [[100, 90]] * 5, [100] * 5, 2, "int8", 64, paged, 9, n_q=4, d_model=264)
    r = torch.Generator(device="cuda").manual_seed(4)
    hidden, vec = (torch.randn(*s, generator=r, device="cuda").bfloat16() for s in ((5, 264), (264,)))
    alpha, flag = torch.rand(5, generator=r, device="cuda"), torch.tensor([1, 0, 1, 1, 0], dtype=torch.uint8, device="cuda")
    want = hidden.clone()
    B.skipkv_steer(5, 264, want, vec, alpha, flag)
    q = queries(c, 4, 8)
    out = attend(c, q, hidden=hidden, vec=vec, alpha=alpha, flag=flag)
    check_attention(c, q, out)
    assert torch.equal(hidden, want)


@pytest.mark.parametrize("paged", [False, True])
def test_attention_repeats_and_replays_to_the_same_bits(B, paged):
    """Twice in a row, on another stream, and captured into a graph that is replayed with other queries."""
    c = filled(B, [[5000, 33]], [5000], 2, "e4m3", 64, paged, 19, n_q=8)
    q = queries(c, 8, 8)
    first = attend(c, q)
    assert torch.equal(first, attend(c, q))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert torch.equal(first, attend(c, q, stream=side))
    torch.cuda.synchronize()
    static_q, out = q.clone(), torch.zeros_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(3):                                # one workspace: launches that follow one another
            B.skipkv_decode_attn_q8(c.shape, c.cache, static_q, c.kv_len, out, None, None, None, None, c.ws)
    for seed in (8, 9):
        static_q.copy_(queries(c, 8, seed))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, attend(c, static_q))


def test_attention_leaves_bad_pages_out(B):
    """Pages outside the pool: reported, and the other rows are attended to; a slab of bad pages alone gives zeros."""
    c = filled(B, [[300, 300], [300, 100]], [300, 300], 2, "e4m3", 32, True, 5, n_q=6)
    table = c.block_table.clone()
    table[0, 1, 1] = c.pool
    table[1, 0, 0] = -5
    table[1, 1, 0] = 2 ** 31 - 1
    c.cache = B.make_q8_cache(c.K.view(torch.float8_e4m3fn), c.V.view(torch.float8_e4m3fn), c.ks, c.vs, 32, table)
    q = queries(c, 6, 1)
    out = attend(c, q)
    assert c.status() == 4
    for i in range(2):
        c.rows64[i][1] = np.concatenate([c.rows64[i][1][:128], c.rows64[i][1][256:]])
        c.rows64[i][2] = c.rows64[i][2][128:]
        c.rows64[i][3] = c.rows64[i][3][:0]
    check_attention(c, q, out)
    assert c.status() == 0


def test_attention_takes_lengths_beyond_the_room_as_the_room(B):
    c = filled(B, [[64, 40]], [64], 2, "int8", 16, False, 5, n_q=6)
    c.kv_len[0, 0] = 1 << 30
    c.kv_len[0, 1] = -7
    c.rows64 = [[c.rows64[i][0], c.rows64[i][1][:0]] for i in range(2)]
    q = queries(c, 6, 1)
    check_attention(c, q, attend(c, q))


# ------------------------------------------------------------------ storing
def values(r, n, wild=False):
    """bf16 rows whose magnitudes differ from row to row by a few powers of two, zeros and a whole row of them among them."""
    x = r.normal(0, 1, (n, 128)) * np.exp2(r.integers(-4, 4, (n, 1)))
    if n:
        x[r.integers(0, n)] = 0
        x[r.integers(0, n, 5), r.integers(0, 128, 5)] = 0
    if wild and n > 2:
        x[0, 3], x[0, 4], x[1, 5] = np.inf, -np.inf, np.nan
        x[n - 1] = 0
        x[n - 1, 0] = np.inf
    return bf16(x)


def same(c, s, n, want_codes, want_scales):
    for (codes, scale), wc, wsc in zip(c.get(s, n), want_codes, want_scales):
        assert np.array_equal(scale, wsc[:len(scale)]), s
        assert np.array_equal(oracle.q8_values(c.fmt)[codes], oracle.q8_values(c.fmt)[wc[:n]]), s


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("wild", [False, True])
def test_pack(B, fmt, paged, block, wild):
    lens = np.array([[0, 1, 15], [16, 17, 127], [128, 129, 300]])
    c = Cache(B, lens, [20, 131, 300], 3, fmt, block, paged, block)
    src = [torch.full((c.rows16, 128), float("nan"), dtype=torch.bfloat16) for _ in range(2)]
    for s in range(c.slabs):
        for x in src:
            n = int(lens.reshape(-1)[s])
            x[c.row0[s]:c.row0[s] + n] = values(c.r, n, wild)
    dev = [x.cuda() for x in src]
    B.skipkv_pack_q8(c.shape, c.cache, dev[0], dev[1], c.kv_len, c.ws)
    torch.cuda.synchronize()
    assert c.status() == (8 if wild else 0)
    for s in range(c.slabs):
        n = int(lens.reshape(-1)[s])
        want = []
        for x in src:
            codes, scale = np.zeros((n, 128), np.uint8), np.zeros(-(-max(n, 1) // block))
            oracle.q8_append(codes, scale, 0, x[c.row0[s]:c.row0[s] + n].double().numpy(), block, fmt)
            want.append((codes, scale))
        same(c, s, n, [w[0] for w in want], [w[1] for w in want])
    c.untouched(lens.reshape(-1))
    # and back: powers of two times codes are bf16 values, so nothing is rounded
    out = [torch.full((c.rows16, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.skipkv_unpack_q8(c.shape, c.cache, c.kv_len, out[0], out[1], c.ws)
    alone = torch.full_like(out[1], 7.0)
    B.skipkv_unpack_q8(c.shape, c.cache, c.kv_len, None, alone, c.ws)
    torch.cuda.synchronize()
    assert c.status() == 0 and torch.equal(alone, out[1])
    for i in range(2):
        got, live = out[i].double().cpu().numpy(), np.zeros(c.rows16, bool)
        for s in range(c.slabs):
            n = int(lens.reshape(-1)[s])
            codes, scale = c.get(s, n)[i]
            assert np.array_equal(got[c.row0[s]:c.row0[s] + n], oracle.q8_rows(codes, scale, n, block, fmt))
            live[c.row0[s]:c.row0[s] + n] = True
        assert (got[~live] == 7).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_pack_magnitudes_from_the_smallest_to_the_largest(B, fmt):
    """Every bf16 magnitude as the largest of its block, the edges of the scales' steps among them."""
    bits = np.arange(0, 0x7f80, 1, dtype=np.uint16)
    n = len(bits)
    x = torch.zeros(n * 16, 128, dtype=torch.bfloat16)
    top = torch.from_numpy(bits.astype(np.int32)).to(torch.int16).view(torch.bfloat16)
    x[::16, 0] = top
    x[::16, 1] = -top
    x[5::16, 2] = (top.float() / 3).bfloat16()
    c = Cache(B, [[n * 16]], [n * 16], 1, fmt, 16, False, 1)
    B.skipkv_pack_q8(c.shape, c.cache, x.cuda(), x.cuda(), c.kv_len, c.ws)
    torch.cuda.synchronize()
    assert c.status() == 0
    codes, scale = c.get(0, n * 16)[0]
    amax = np.abs(top.double().numpy())
    want = np.array([oracle.q8_scale([a], fmt) for a in amax])
    assert np.array_equal(scale, want)
    for row, col in ((0, 0), (0, 1), (5, 2)):
        y = x[row::16, col].double().numpy() / want
        assert np.array_equal(oracle.q8_values(fmt)[codes[row::16, col]], oracle.q8_values(fmt)[oracle.q8_nearest(y, fmt)])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_append(B, fmt, paged, block):
    """Parts of prompts of different lengths (none, one, several pages) and then single tokens, into blocks that have rows and whose scales grow."""
    hk, bt = 2, 5
    caps = [300, 300, 300, 400, 129]
    c = Cache(B, np.zeros((bt, hk)), caps, hk, fmt, block, paged, 10 + block)
    host = [([np.zeros((400, 128), np.uint8) for _ in range(c.slabs)], [np.zeros(-(-400 // block)) for _ in range(c.slabs)]) for _ in range(2)]
    lens = np.zeros(c.slabs, np.int32)
    lens[3], lens[6] = 0, 0
    a, b = torch.zeros(bt, hk, dtype=torch.int32, device="cuda"), torch.full((bt, hk), -1, dtype=torch.int32, device="cuda")
    parts = [[0, 1, 100, 250, 128], [17, 0, 28, 129, 1], [1, 5, 3, 1, 0]] + [[1] * bt] * 20
    for i, part in enumerate(parts):
        part = [min(p, caps[k] - int(lens[k * hk])) for k, p in enumerate(part)]
        off = np.concatenate([[0], np.cumsum(part)])
        x = [bf16(values(c.r, max(int(off[-1]), 1) * hk).double().numpy().reshape(-1, hk, 128) * 2.0 ** (i % 7 - 3)) for _ in range(2)]
        single = part == [1] * bt
        B.skipkv_append_q8(c.shape, c.cache, x[0].cuda(), x[1].cuda(), None if single else torch.from_numpy(off.astype(np.int32)).cuda(), int(off[-1]),
                           a, b, c.ws)
        torch.cuda.synchronize()
        assert c.status() == 0
        for s in range(c.slabs):
            q, h = divmod(s, hk)
            for k in range(2):
                rows = x[k][int(off[q]):int(off[q + 1]), h].double().numpy()
                n = oracle.q8_append(host[k][0][s], host[k][1][s], int(lens[s]), rows, block, fmt)
            lens[s] = n
        assert np.array_equal(b.cpu().numpy().reshape(-1), lens)
        for s in range(c.slabs):
            same(c, s, int(lens[s]), [host[0][0][s], host[1][0][s]], [host[0][1][s], host[1][1][s]])
        a, b = b, a
    c.untouched(lens)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("block", [16, 128])
def test_append_no_more_rows_than_sequences(B, fmt, paged, block):
    """A few rows in all, however they fall to the sequences: across blocks and pages, with scales that grow, NaN and infinities among them."""
    hk, bt = 2, 7
    c = Cache(B, np.zeros((bt, hk)), [300] * bt, hk, fmt, block, paged, 11)
    host = [([np.zeros((400, 128), np.uint8) for _ in range(c.slabs)], [np.zeros(-(-400 // block)) for _ in range(c.slabs)]) for _ in range(2)]
    lens = np.zeros(c.slabs, np.int32)
    a, b = torch.zeros(bt, hk, dtype=torch.int32, device="cuda"), torch.full((bt, hk), -1, dtype=torch.int32, device="cuda")
    parts = [[120, 125, 14, 15, 16, 250, 0], [7, 0, 0, 0, 0, 0, 0], [0, 5, 1, 1, 0, 0, 0], [0, 0, 3, 4, 0, 0, 0], [0] * 7, [0, 0, 0, 0, 0, 6, 1], [1] * 7,
             [2, 0, 2, 0, 2, 0, 1]]
    for i, part in enumerate(parts):
        off = np.concatenate([[0], np.cumsum(part)])
        x = [values(c.r, max(int(off[-1]), 1) * hk, wild=i == 5).double().numpy().reshape(-1, hk, 128) * 2.0 ** (i % 5 - 2) for _ in range(2)]
        x = [bf16(y) for y in x]
        B.skipkv_append_q8(c.shape, c.cache, x[0].cuda(), x[1].cuda(), torch.from_numpy(off.astype(np.int32)).cuda(), int(off[-1]), a, b, c.ws)
        torch.cuda.synchronize()
        assert c.status() == (8 if i == 5 else 0)
        for s in range(c.slabs):
            q, h = divmod(s, hk)
            for k in range(2):
                n = oracle.q8_append(host[k][0][s], host[k][1][s], int(lens[s]), x[k][int(off[q]):int(off[q + 1]), h].double().numpy(), block, fmt)
            lens[s] = n
            same(c, s, n, [host[0][0][s], host[1][0][s]], [host[0][1][s], host[1][1][s]])
        assert np.array_equal(b.cpu().numpy().reshape(-1), lens)
        a, b = b, a
    c.untouched(lens)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("block", [16, 64, 128])
def test_append_up_to_four_rows_per_sequence(B, fmt, paged, block):
    """As many rows as a call may have whose slabs are shared out by blocks, and one more: equal parts, one sequence with all of them, scales that grow."""
    hk, bt = 2, 21
    c = Cache(B, np.zeros((bt, hk)), [400] * bt, hk, fmt, block, paged, 13)
    host = [([np.zeros((400, 128), np.uint8) for _ in range(c.slabs)], [np.zeros(-(-400 // block)) for _ in range(c.slabs)]) for _ in range(2)]
    lens = np.zeros(c.slabs, np.int32)
    a, b = torch.zeros(bt, hk, dtype=torch.int32, device="cuda"), torch.full((bt, hk), -1, dtype=torch.int32, device="cuda")
    parts = [[4] * 21, [84] + [0] * 20, [5] * 16 + [4, 0, 0, 0, 0], [61, 0, 3] + [1] * 18, [0] * 20 + [85], [1] * 20 + [64], [0, 22] + [0] * 19]
    for i, part in enumerate(parts):
        off = np.concatenate([[0], np.cumsum(part)])
        x = [bf16(values(c.r, int(off[-1]) * hk, wild=i == 3).double().numpy().reshape(-1, hk, 128) * 2.0 ** (2 * i - 6)) for _ in range(2)]
        B.skipkv_append_q8(c.shape, c.cache, x[0].cuda(), x[1].cuda(), torch.from_numpy(off.astype(np.int32)).cuda(), int(off[-1]), a, b, c.ws)
        torch.cuda.synchronize()
        assert c.status() == (8 if i == 3 else 0)
        for s in range(c.slabs):
            q, h = divmod(s, hk)
            for k in range(2):
                n = oracle.q8_append(host[k][0][s], host[k][1][s], int(lens[s]), x[k][int(off[q]):int(off[q + 1]), h].double().numpy(), block, fmt)
            lens[s] = n
            same(c, s, n, [host[0][0][s], host[1][0][s]], [host[0][1][s], host[1][1][s]])
        assert np.array_equal(b.cpu().numpy().reshape(-1), lens)
        a, b = b, a
    c.untouched(lens)


@pytest.mark.parametrize("paged", [False, True])
def test_many_slabs_stored_appended_and_loaded(B, paged):
    """So many slabs that their table has a launch of its own; most are empty.  The calls behind one another leave what they leave with a pause after each."""
    hk, bt, block, fmt = 2, 1100, 16, "e4m3"
    r = np.random.default_rng(5)
    lens = np.where(r.random((bt, hk)) < 0.1, r.integers(0, 140, (bt, hk)), 0)
    lens[-1] = 140
    part = np.where(r.random(bt) < 0.3, r.integers(0, 30, bt), 0)
    part[7] = 25
    part[9] += max(0, 4 * bt + 1 - int(part.sum()))
    room = int((lens.max(1) + part).max()) + 20
    off = np.concatenate([[0], np.cumsum(part)]).astype(np.int32)
    new = [values(r, int(off[-1]) * hk).view(-1, hk, 128) for _ in range(2)]
    got = []
    for pause in (True, False):
        c = Cache(B, lens, [room] * bt, hk, fmt, block, paged, 2, n_q=2 * hk)
        src = [torch.from_numpy(np.random.default_rng(8 + i).normal(0, 1, (c.rows16, 128)).astype(np.float32)).bfloat16().cuda() for i in range(2)]
        n1, n2 = torch.full_like(c.kv_len, -1), torch.full_like(c.kv_len, -1)
        dev, offs = [x.cuda() for x in new], torch.from_numpy(off).cuda()
        out, back, q = torch.full((bt, 2 * hk, 128), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full_like(src[0], 7.0), queries(c, 2 * hk, 3)
        torch.cuda.synchronize()
        calls = [lambda: B.skipkv_pack_q8(c.shape, c.cache, src[0], src[1], c.kv_len, c.ws),
                 lambda: B.skipkv_append_q8(c.shape, c.cache, dev[0], dev[1], offs, int(off[-1]), c.kv_len, n1, c.ws),
                 lambda: B.skipkv_decode_attn_q8(c.shape, c.cache, q, n1, out, None, None, None, None, c.ws),
                 lambda: B.skipkv_append_q8(c.shape, c.cache, dev[0][:bt], dev[1][:bt], None, bt, n1, n2, c.ws),
                 lambda: B.skipkv_unpack_q8(c.shape, c.cache, n2, None, back, c.ws)]
        for f in calls:
            f()
            if pause:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert c.status() == 0
        got.append([out, back, n1, n2, c.K, c.V, c.ks.view(torch.int32), c.vs.view(torch.int32)])
        if not pause:
            break
        host = [x.double().cpu().numpy() for x in src]
        want_n1, want_n2 = lens + part[:, None], lens + part[:, None] + 1
        assert np.array_equal(n1.cpu().numpy(), want_n1) and np.array_equal(n2.cpu().numpy(), want_n2)
        V = back.double().cpu().numpy()
        x64, live = [x.double().numpy() for x in new], np.zeros(c.rows16, bool)
        c.rows64 = [[], []]
        for s in range(c.slabs):
            b, h = divmod(s, hk)
            n = int(want_n2[b, h])
            codes, scale = np.zeros((room, 128), np.uint8), np.zeros(-(-room // block))
            end = []
            for k in range(2):
                old = int(lens[b, h])
                oracle.q8_append(codes, scale, 0, host[k][c.row0[s]:c.row0[s] + old], block, fmt)
                m = oracle.q8_append(codes, scale, old, x64[k][off[b]:off[b + 1], h], block, fmt)
                c.rows64[k].append(oracle.q8_rows(codes, scale, m, block, fmt))
                if k == 1:
                    oracle.q8_append(codes, scale, m, x64[k][b:b + 1, h], block, fmt)
                    assert np.array_equal(V[c.row0[s]:c.row0[s] + n], oracle.q8_rows(codes, scale, n, block, fmt)), s
            live[c.row0[s]:c.row0[s] + n] = True
        assert (V[~live] == 7).all()
        check_attention(c, q, out)
        # a length without room is reported, its slab left out
        bad = c.kv_len.clone()
        bad[3, 1] = room + 200
        B.skipkv_pack_q8(c.shape, c.cache, src[0], src[1], bad, c.ws)
        torch.cuda.synchronize()
        assert c.status() == 4
        c2 = got[0]
        got[0] = [x.clone() for x in c2[:4]]
    for x, y in zip(got[0], got[1]):
        assert torch.equal(x, y)


def test_append_where_heads_differ_in_length(B):
    """After an eviction the heads of a sequence have lengths of their own."""
    c = Cache(B, [[5, 130], [64, 0]], [200, 200], 2, "e4m3", 64, False, 3)
    codes, scales = ([], []), ([], [])
    for s in range(4):
        for i in range(2):
            x, f = random_slab(c.r, int(c.lens.reshape(-1)[s]), 64, "e4m3")
            codes[i].append(x)
            scales[i].append(f)
    c.put(codes, scales)
    x = [bf16(c.r.normal(0, 3, (50, 2, 128))) for _ in range(2)]
    off = torch.tensor([0, 20, 50], dtype=torch.int32).cuda()
    out = torch.zeros_like(c.kv_len)
    B.skipkv_append_q8(c.shape, c.cache, x[0].cuda(), x[1].cuda(), off, 50, c.kv_len, out, c.ws)
    torch.cuda.synchronize()
    assert c.status() == 0 and out.tolist() == [[25, 150], [94, 30]]
    for s in range(4):
        b, h = divmod(s, 2)
        old = int(c.lens.reshape(-1)[s])
        want = []
        for i in range(2):
            cc, ff = np.zeros((200, 128), np.uint8), np.zeros(4)
            cc[:old], ff[:len(scales[i][s])] = codes[i][s], scales[i][s]
            n = oracle.q8_append(cc, ff, old, x[i][[0, 20][b]:[20, 50][b], h].double().numpy(), 64, "e4m3")
            want.append((cc, ff))
        same(c, s, n, [w[0] for w in want], [w[1] for w in want])


@pytest.mark.parametrize("paged", [False, True])
def test_append_without_room_leaves_the_slab(B, paged):
    """One slab too full, offsets that go down, a bad page: reported, left as they were, and the others are served."""
    c = filled(B, [[120], [10], [10]], [128, 128, 128], 1, "int8", 32, paged, 3)
    before = [c.get(s, int(c.lens[s, 0])) for s in range(3)]
    x = bf16(c.r.normal(0, 1, (30, 1, 128))).cuda()
    out = torch.full_like(c.kv_len, -1)
    B.skipkv_append_q8(c.shape, c.cache, x, x, torch.tensor([0, 9, 20, 30], dtype=torch.int32).cuda(), 30, c.kv_len, out, c.ws)
    torch.cuda.synchronize()
    assert c.status() == 4 and out.view(-1).tolist() == [120, 21, 20]
    for (x0, f0), (x1, f1) in zip(before[0], c.get(0, 120)):
        assert np.array_equal(x0, x1) and np.array_equal(f0, f1)
    for off, want in (([0, 5, 3, 8], [120, 10, 15]), ([0, 2, 4, 31], [122, 12, 10]), ([-1, 2, 4, 8], [120, 12, 14])):
        c = filled(B, [[120], [10], [10]], [128, 128, 128], 1, "int8", 32, paged, 3)
        B.skipkv_append_q8(c.shape, c.cache, x, x, torch.tensor(off, dtype=torch.int32).cuda(), 30, c.kv_len, out, c.ws)
        torch.cuda.synchronize()
        got = out.view(-1).tolist()
        assert c.status() == 4
        assert got == [g if o0 >= 0 and o0 <= o1 <= 30 and n + o1 - o0 <= 128 else n
                       for n, o0, o1, g in zip([120, 10, 10], off, off[1:], [n + o1 - o0 for n, o0, o1 in zip([120, 10, 10], off, off[1:])])]
    if paged:
        c = filled(B, [[100], [10]], [256, 256], 1, "int8", 32, True, 3)
        table = c.block_table.clone()
        table[0, 0, 1] = c.pool + 3
        cache = B.make_q8_cache(c.K.view(torch.int8), c.V.view(torch.int8), c.ks, c.vs, 32, table)
        kept = c.K.clone()
        kept[torch.from_numpy(c.places(0, 128)[0]).cuda()] = 0
        B.skipkv_append_q8(c.shape, cache, x[:29].repeat(5, 1, 1), x[:29].repeat(5, 1, 1), torch.tensor([0, 100, 100], dtype=torch.int32).cuda(), 145,
                           c.kv_len, out[:2], c.ws)
        torch.cuda.synchronize()
        assert c.status() == 4
        now = c.K.clone()
        now[torch.from_numpy(c.places(0, 128)[0]).cuda()] = 0
        assert torch.equal(now, kept)                     # nothing outside the good page


def test_pack_and_unpack_report_lengths_without_room(B):
    c = filled(B, [[100], [50]], [100, 60], 1, "e4m3", 32, False, 3)
    K, V = (torch.ones(c.rows16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    before = c.get(1, 50)
    kv = torch.tensor([[100], [61]], dtype=torch.int32, device="cuda")
    B.skipkv_pack_q8(c.shape, c.cache, K, V, kv, c.ws)
    torch.cuda.synchronize()
    assert c.status() == 4 and np.array_equal(before[0][0], c.get(1, 50)[0][0])
    assert (oracle.q8_rows(*c.get(0, 100)[0], 100, 32, "e4m3") == 1).all()
    B.skipkv_unpack_q8(c.shape, c.cache, torch.tensor([[100], [-1]], dtype=torch.int32, device="cuda"), K, V, c.ws)
    torch.cuda.synchronize()
    assert c.status() == 4 and bool((K == 1).all())


@pytest.mark.parametrize("fmt", FORMATS)
def test_unpack_with_general_scales_rounds_once(B, fmt):
    """Code times scale in 32 bits, then bf16: off by at most half a step of bf16 and one of fp32."""
    c = filled(B, [[700, 13]], [700], 2, fmt, 32, False, 3, general=True)
    K = torch.zeros(c.rows16, 128, dtype=torch.bfloat16, device="cuda")
    B.skipkv_unpack_q8(c.shape, c.cache, c.kv_len, K, None, c.ws)
    torch.cuda.synchronize()
    for s, n in ((0, 700), (1, 13)):
        want = c.rows64[0][s]
        got = K[c.row0[s]:c.row0[s] + n].double().cpu().numpy()
        assert (np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -23) * np.abs(want)).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_to_scales_that_are_no_powers_of_two(B, fmt):
    """Such a scale goes up to the next power of two, and the block's codes are rounded under it."""
    c = filled(B, [[20]], [64], 1, fmt, 32, False, 3, general=True)
    old = c.get(0, 20)
    x = bf16(np.full((1, 1, 128), 1e-3)).cuda()
    out = torch.zeros_like(c.kv_len)
    B.skipkv_append_q8(c.shape, c.cache, x, x, None, 1, c.kv_len, out, c.ws)
    torch.cuda.synchronize()
    for (x0, f0), (x1, f1) in zip(old, c.get(0, 20)):
        up = 2.0 ** np.ceil(np.log2(f0[0]))
        assert f1[0] == up
        v = oracle.q8_values(fmt)
        y = v[x0] * (f0[0] / up)
        step = 1.0 if fmt == "int8" else np.maximum(np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3), 2.0 ** -9)
        assert (np.abs(v[x1] - y) <= step / 2 + 2.0 ** -22 * np.abs(y)).all()


# ------------------------------------------------------------------ large buffers, steps
@pytest.mark.parametrize("paged", [False, True])
def test_rows_beyond_two_gigabytes(B, paged):
    """Slabs whose bytes lie behind 2^31 and 2^32, in 8 bits and in 16."""
    n, far = 200, 35_000_000                              # 4.5 GB of codes, 9 GB of bf16 rows
    rows = (far + n + 127) // 128 * 128                # (whole pages that hold the last slab)
    K, V = (torch.zeros(rows, 128, dtype=torch.int8, device="cuda") for _ in range(2))
    r = np.random.default_rng(2)
    off, cap = torch.tensor([0, far], dtype=torch.int64).cuda(), torch.tensor([256, 200], dtype=torch.int32).cuda()
    shape = B.make_shape(2, 4, 1, 128, 1, 0, 1, 256, off, cap, far + 200)
    ws = torch.empty(B.skipkv_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    B.skipkv_workspace_init(shape, ws)
    table = torch.tensor([[[1, 0]], [[rows // 128 - 1, rows // 128 - 2]]], dtype=torch.int32).cuda() if paged else None
    sc = torch.full((rows // 128, 1) if paged else (2, 1, 2), 0.0, device="cuda")
    sv = sc.clone()
    cache = B.make_q8_cache(K, V, sc, sv, 128, table)
    src = torch.zeros(far + 200, 128, dtype=torch.bfloat16, device="cuda")
    x = bf16(r.normal(0, 1, (n, 128)))
    src[far:far + n] = x.cuda()
    kv = torch.tensor([[0], [n]], dtype=torch.int32, device="cuda")
    B.skipkv_pack_q8(shape, cache, src, src, kv, ws)
    back = torch.zeros_like(src)
    B.skipkv_unpack_q8(shape, cache, kv, back, None, ws)
    q = bf16(r.normal(0, 1, (2, 4, 128))).cuda()
    out = torch.zeros_like(q)
    B.skipkv_decode_attn_q8(shape, cache, q, kv, out, None, None, None, None, ws)
    torch.cuda.synchronize()
    assert B.skipkv_status(ws) == 0
    codes, scale = np.zeros((n, 128), np.uint8), np.zeros(2)
    oracle.q8_append(codes, scale, 0, x.double().numpy(), 128, "int8")
    want = oracle.q8_rows(codes, scale, n, 128, "int8")
    assert np.array_equal(back[far:far + n].double().cpu().numpy(), want) and not bool(back[:far].any())
    c = type("C", (), dict(hk=1, slabs=2, rows64=[[want[:0], want]] * 2))
    check_attention(c, q, out)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
def test_append_step_keeps_the_tables_that_append_step_keeps(B, fmt, paged):
    """Range list, window and lengths as skipkv_append_step leaves them beside a bf16 cache; a full slab and a full list are reported."""
    bt, hk, hq, window, ms = 4, 2, 6, 4, 6
    c = Cache(B, np.zeros((bt, hk)), [5, 9, 9, 9], hk, fmt, 16, paged, 1, n_q=hq, window=window, max_sent=ms)
    if paged:                                             # room is that of whole pages: the first slabs' room is what cap says
        c.cap.copy_(torch.tensor([5, 9, 9, 9], dtype=torch.int32))
    ref_cap = torch.tensor([5, 9, 9, 9], dtype=torch.int32).cuda()
    ref_off = torch.tensor([0, 5, 14, 23], dtype=torch.int64).cuda()
    ref = B.make_shape(bt, hq, hk, 128, window, 0, ms, 9, ref_off, ref_cap, 32 * hk)
    K16, V16 = (torch.zeros(32 * hk, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mk = lambda: (torch.zeros(bt, hk, ms + 1, dtype=torch.int32, device="cuda"), torch.full((bt, hk, ms), -1, dtype=torch.int32, device="cuda"),  # noqa: E731
                  torch.zeros(bt, hk, dtype=torch.int32, device="cuda"), torch.zeros(bt, hq, window, 128, dtype=torch.bfloat16, device="cuda"))
    a, b = mk(), mk()
    len16, n0, n1 = (torch.zeros(bt, hk, dtype=torch.int32, device="cuda") for _ in range(3))
    host = [[(np.zeros((9, 128), np.uint8), np.zeros(1)) for _ in range(c.slabs)] for _ in range(2)]
    g = torch.Generator().manual_seed(3)
    for step in range(9):
        k, v = (torch.randn(bt, hk, 128, generator=g).mul(2.0 ** (step % 4)).bfloat16() for _ in range(2))
        q = torch.randn(bt, hq, 128, generator=g).bfloat16().cuda()
        opens = torch.tensor([1, step % 2, step % 3 == 0, 0], dtype=torch.uint8).cuda()
        gid = torch.full((bt,), 70 + step, dtype=torch.int32, device="cuda")
        B.skipkv_append_step(ref, K16, V16, k.cuda(), v.cuda(), len16, a[0], a[1], a[2], opens, gid, a[3], q, step % window, c.ws)
        torch.cuda.synchronize()
        bits = c.status()
        B.skipkv_append_step_q8(c.shape, c.cache, k.cuda(), v.cuda(), n0, n1, b[0], b[1], b[2], opens, gid, b[3], q, step % window, c.ws)
        torch.cuda.synchronize()
        assert c.status() == bits == (4 if step >= 5 else 0)
        for x, y in zip(a, b):
            assert torch.equal(x, y), step
        assert torch.equal(n1, len16)
        old = n0.cpu().numpy().reshape(-1)
        for s in range(c.slabs):
            if int(n1.view(-1)[s]) > old[s]:
                for i, x in enumerate((k, v)):
                    oracle.q8_append(*host[i][s], int(old[s]), x.view(-1, 128)[s:s + 1].double().numpy(), 16, fmt)
            same(c, s, int(n1.view(-1)[s]), [host[0][s][0], host[1][s][0]], [host[0][s][1], host[1][s][1]])
        n0, n1 = n1, n0
    torch.cuda.synchronize()
    # without a window nothing of it is written
    B.skipkv_append_step_q8(c.shape, c.cache, k.cuda(), v.cuda(), n0, n1, b[0], b[1], b[2], opens, gid, None, None, 0, c.ws)
    torch.cuda.synchronize()
    assert torch.equal(a[3], b[3])


def test_another_device_is_refused(B):
    c = filled(B, [[10]], [16], 1, "e4m3", 16, False, 3)
    c.cache.device = 1
    with pytest.raises(B.SkipKVError) as e:
        attend(c, queries(c, 1, 1))
    assert e.value.code == -1
