"""The 8-bit cache at the ends of its ranges: infinities beside the largest magnitudes, sums and logits near the largest numbers, queries of very
unequal elements, slabs that reach beyond their buffers, range lists that make no sense, tables of other slabs."""
import numpy as np
import pytest
import torch

import oracle
from q8_common import DT, Cache, bf16, random_slab
from test_gpu_q8 import B, FORMATS, attend, check_attention, filled, queries, same  # noqa: F401

pytestmark = pytest.mark.gpu
LARGEST = float(torch.finfo(torch.bfloat16).max)


# ------------------------------------------------------------------ infinities
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("block", [16, 128])
def test_infinities_beside_the_largest_magnitude(B, fmt, paged, block):
    """Stored as the largest codes of their signs under the largest scale there is too: packed, and joining a block that has it (a row at a time,
    and more rows than go without tiles)."""
    r = np.random.default_rng(4)
    first = r.normal(0, 1, (21, 128))
    first[3, :5] = LARGEST, np.inf, -np.inf, -LARGEST, np.nan
    first[20, 7] = -LARGEST
    later = []
    for n in (1, 4, 5, 30):
        x = r.normal(0, 1, (n, 128))
        x[n - 1, 9:12] = np.inf, -np.inf, LARGEST / 2
        x[0, 100] = -np.inf
        later.append(bf16(x))
    first = bf16(first)
    c = Cache(B, [[21]], [200], 1, fmt, block, paged, 1)
    src = torch.zeros(c.rows16, 128, dtype=torch.bfloat16)
    src[:21] = first
    B.skipkv_pack_q8(c.shape, c.cache, src.cuda(), src.cuda(), c.kv_len, c.ws)
    torch.cuda.synchronize()
    assert c.status() == 8
    codes, scale = np.zeros((200, 128), np.uint8), np.zeros(-(-200 // block))
    n = oracle.q8_append(codes, scale, 0, first.double().numpy(), block, fmt)
    assert scale[0] == 2.0 ** (122 if fmt == "int8" else 120)
    same(c, 0, n, [codes] * 2, [scale] * 2)
    a, b = c.kv_len.clone(), torch.zeros_like(c.kv_len)
    for x in later:
        rows = x.view(-1, 1, 128).cuda()
        B.skipkv_append_q8(c.shape, c.cache, rows, rows, torch.tensor([0, len(x)], dtype=torch.int32).cuda(), len(x), a, b, c.ws)
        torch.cuda.synchronize()
        assert c.status() == 8
        n = oracle.q8_append(codes, scale, n, x.double().numpy(), block, fmt)
        assert b.item() == n
        same(c, 0, n, [codes] * 2, [scale] * 2)
        a, b = b, a


# ------------------------------------------------------------------ attention near the ends of 32 bits
def slab_cache(B, lens, hk, fmt, paged, k_scale, v_scale, seed, n_q, general=False):
    """Slabs of ordinary codes whose scales are the given ones, times up to two."""
    bt = len(lens)
    c = Cache(B, lens, [int(max(x)) for x in lens], hk, fmt, 32, paged, seed, n_q=n_q)
    codes, scales = ([], []), ([], [])
    for s in range(bt * hk):
        n = int(c.lens.reshape(-1)[s])
        for i, base in enumerate((k_scale, v_scale)):
            x, f = random_slab(c.r, n, 32, fmt)
            f = np.full_like(f, base)
            codes[i].append(x)
            scales[i].append(np.asarray(f * c.r.uniform(1, 2, len(f)), np.float32).astype(np.float64) if general else f)
    c.put(codes, scales)
    c.rows64 = [[oracle.q8_rows(codes[i][s], scales[i][s], len(codes[i][s]), 32, fmt) for s in range(c.slabs)] for i in range(2)]
    return c


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("group", [3, 7])
def test_attention_over_values_near_the_largest(B, fmt, paged, group):
    """Sums of p |v| (p relative to the largest) below 2^127, as a cache in 32 bits would have them: 600 rows of up to 448 * 2^108 < 2^117 (1e35), and
    one row of the largest value there is."""
    k = 2.0 ** -8 if fmt == "e4m3" else 2.0 ** -6
    c = slab_cache(B, [[600, 77], [5000, 1]], 2, fmt, paged, k, 2.0 ** 108, 3, 2 * group)
    q = queries(c, 2 * group, 7)
    check_attention(c, q, attend(c, q))
    c = slab_cache(B, [[1, 1]], 2, fmt, paged, k, 2.0 ** (118 if fmt == "e4m3" else 120), 3, 2 * group)
    q = queries(c, 2 * group, 8)
    check_attention(c, q, attend(c, q))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("general", [False, True])
@pytest.mark.parametrize("group", [3, 7])
def test_attention_over_the_least_scales(B, fmt, general, group):
    """2^-111, where products with 2^-15 are normal numbers still, and queries that make ordinary logits of such keys."""
    c = slab_cache(B, [[600, 77], [5000, 1]], 2, fmt, False, 2.0 ** -111, 2.0 ** -111, 3, 2 * group, general)
    q = queries(c, 2 * group, 7, 2.0 ** (103 if fmt == "e4m3" else 105))
    check_attention(c, q, attend(c, q))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("group", [2, 6])
@pytest.mark.parametrize("n", [1, 100, 300, 9000])
def test_attention_with_logits_far_below_zero(B, fmt, paged, group, n):
    """Logits of -2^122 and below, all of them: the largest has all of the weight, wherever its row lies."""
    c = slab_cache(B, [[n]], 1, fmt, paged, 1.0, 1.0, 5, group)
    top = (n * 2) // 3
    v = c.rows64[1][0]
    codes = np.zeros((n, 128), np.uint8)
    codes[:, 0] = oracle.q8_nearest(np.array([-64.0]), fmt)[0]
    codes[top, 0] = oracle.q8_nearest(np.array([-32.0]), fmt)[0]
    old = c.get(0, n)
    c.put(([codes], [old[1][0]]), ([np.full(-(-n // 32), 2.0 ** 60)], [old[1][1]]))
    q = torch.zeros(1, group, 128)
    q[:, :, 0] = 2.0 ** 60
    out = attend(c, q.bfloat16().cuda()).double().cpu().numpy()
    assert np.array_equal(out[0], np.broadcast_to(bf16(v[top]).double().numpy(), (group, 128)))


# ------------------------------------------------------------------ queries of unequal elements
@pytest.mark.parametrize("fmt,steps", [("e4m3", (9, 14, 16, 18, 30)), ("int8", (20, 31, 33, 35, 60))])
@pytest.mark.parametrize("group", [3, 7])
def test_attention_where_large_query_elements_meet_zeros(B, fmt, steps, group):
    """One element is 2^step times the others and meets keys that are 0, so the others make the logits.  They are exact from 2^-14 (int8: 2^-31) of
    the largest on; below that off by at most 2^-22 (2^-39) of it, which moves a logit by that times sum |k| / sqrt(d)."""
    for step in steps:
        c = filled(B, [[600, 77]], [600], 2, fmt, 16, False, 9, n_q=2 * group)
        for s in range(2):
            rows = torch.from_numpy(c.places(s, len(c.rows64[0][s]))[0]).cuda()
            c.K[rows, 17] = 0
            c.rows64[0][s][:, 17] = 0
        q = queries(c, 2 * group, 7)
        # others in [1, 2) in magnitude
        q = (1 + q.float().abs().frac()).bfloat16().clamp(max=1.9921875) * torch.where(q < 0, -1, 1).bfloat16()
        q[:, :, 17] = 2.0 ** step
        out = attend(c, q)
        if step <= (14 if fmt == "e4m3" else 31):
            check_attention(c, q, out)
            continue
        lost = 2.0 ** step * (2.0 ** -22 if fmt == "e4m3" else 2.0 ** -39)
        q64, got = q.double().cpu().numpy(), out.double().cpu().numpy()
        for s in range(c.slabs):
            K, V = c.rows64[0][s], c.rows64[1][s]
            for j in range(group):
                qq = q64[0, s * group + j][None]
                want, mine = oracle.attn_rows(qq, K, V)[0], got[0, s * group + j]
                e = (2.0 ** -23 * 136 * (np.abs(qq) @ np.abs(K).T).max() + lost * np.abs(K).sum(1).max()) / np.sqrt(128)
                # a probability is off by a factor of at most exp(2 e)
                room = 2.0 ** -8 * np.abs(want) + (1 + 2.0 ** -8) * ((np.expm1(min(2 * e, 50)) + 2.0 ** -19) * oracle.attn_rows(qq, K, np.abs(V))[0] + 2.0 ** -40 * np.abs(V).sum(0))
                assert (np.abs(mine - want) <= room).all(), (step, s, j)


# ------------------------------------------------------------------ slabs that reach beyond the buffers
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("inside", [0, 1, 17, 31, 32, 33, 100, 127, 128, 129, 160, 299, -20])
def test_attention_over_the_rows_inside_the_buffer(B, fmt, inside):
    """A slab of which the buffer has the first rows only: those are attended to, however few of a tile they are, and it is reported."""
    c = filled(B, [[200, 250], [300, 301]], [256, 301], 2, fmt, 16, False, 5, n_q=6)
    rows = c.row0[3] + inside
    c.cache = B.make_q8_cache(c.K[:rows].view(DT[fmt]), c.V[:rows].view(DT[fmt]), c.ks, c.vs, 16)
    for i in range(2):
        c.rows64[i][3] = c.rows64[i][3][:max(inside, 0)]
        c.rows64[i][2] = c.rows64[i][2][:min(300, rows - c.row0[2])]
    q = queries(c, 6, 1)
    check_attention(c, q, attend(c, q))
    assert c.status() == 4
    check_attention(c, q, attend(c, q))


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("inside", [0, 1, 100, 128, 149, -20, -60])
def test_slabs_have_no_room_beyond_the_buffer(B, many, inside):
    """Slabs that would reach beyond the buffer: packing leaves them out, appending leaves them and their lengths as they were, loading takes the rows
    that are there; all report it."""
    bt, fmt = 2100 if many else 2, "int8"
    lens, caps = np.zeros(bt, np.int64), np.ones(bt, np.int64)
    lens[-2:], caps[-2:] = 150, 200
    c = filled(B, lens[:, None], caps, 1, fmt, 32, False, 5)
    rows = c.row0[-1] + inside
    room = np.minimum(caps, np.maximum(rows - np.array(c.row0), 0))
    state = (c.K, c.V, c.ks.view(torch.int32), c.vs.view(torch.int32))
    before = [x.clone() for x in state]
    c.cache = B.make_q8_cache(c.K[:rows].view(DT[fmt]), c.V[:rows].view(DT[fmt]), c.ks, c.vs, 32)

    def changed_alone(first, last):
        """Rows [first, last) of the slabs and the scales of those that have any are other ones; the rest is what it was.  Then all is put back."""
        for x, y in zip(state[:2], before):
            keep = torch.ones(len(x), dtype=torch.bool, device="cuda")
            for s in np.flatnonzero(last > first):
                at = slice(c.row0[s] + int(first[s]), c.row0[s] + int(last[s]))
                assert bool((x[at] != y[at]).any(1).all())
                keep[at] = False
            assert torch.equal(x[keep], y[keep])
        same_scales = torch.from_numpy(last <= first).cuda()
        for x, y in zip(state[2:], before[2:]):
            assert torch.equal(x[same_scales], y[same_scales])
        for x, y in zip(state, before):
            x.copy_(y)

    src = torch.full((c.rows16, 128), 2.0 ** -40, dtype=torch.bfloat16, device="cuda")
    B.skipkv_pack_q8(c.shape, c.cache, src, src, c.kv_len, c.ws)
    torch.cuda.synchronize()
    assert c.status() == 4
    changed_alone(np.zeros(bt, int), np.where(lens <= room, lens, 0))
    # a few rows, without tiles, and so many (most of no sequence) that they go by tiles
    for extra in (0, 4 * bt):
        count = np.where(lens > 0, 2, 0)
        off = torch.from_numpy(np.concatenate([[0], np.cumsum(count)]).astype(np.int32)).cuda()
        n = int(count.sum()) + extra
        x = torch.full((n, 1, 128), 2.0 ** -40, dtype=torch.bfloat16, device="cuda")
        out = torch.full_like(c.kv_len, -1)
        B.skipkv_append_q8(c.shape, c.cache, x, x, off, n, c.kv_len, out, c.ws)
        torch.cuda.synchronize()
        assert c.status() == 4
        want = np.where(lens + count <= room, lens + count, lens)
        assert np.array_equal(out.view(-1).cpu().numpy(), want)
        changed_alone(lens, want)

    def loaded(i):
        y = np.full((c.rows16, 128), 7.0)
        for s in np.flatnonzero(lens):
            m = min(int(lens[s]), int(room[s]))
            y[c.row0[s]:c.row0[s] + m] = c.rows64[i][s][:m]
        return y

    # the codes' buffer ends, then the one that they are loaded into
    whole = B.make_q8_cache(c.K.view(DT[fmt]), c.V.view(DT[fmt]), c.ks, c.vs, 32)
    short = B.make_shape(bt, 1, 1, 128, 1, 0, 1, c.max_cap, c.slab_off, c.cap, rows)
    for shape, cache in ((c.shape, c.cache), (short, whole)):
        back = [torch.full((c.rows16, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        B.skipkv_unpack_q8(shape, cache, c.kv_len, back[0], back[1], c.ws)
        torch.cuda.synchronize()
        assert c.status() == 4
        for i in range(2):
            assert np.array_equal(back[i].double().cpu().numpy(), loaded(i))
    # bf16 slabs that reach beyond their buffer are not packed
    B.skipkv_pack_q8(short, whole, src, src, c.kv_len, c.ws)
    torch.cuda.synchronize()
    assert c.status() == 4
    changed_alone(np.zeros(bt, int), np.where(lens <= room, lens, 0))


# ------------------------------------------------------------------ range lists that make no sense
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("paged", [False, True])
def test_append_step_with_a_bad_sentence_count(B, fmt, paged):
    """As skipkv_append_step beside a bf16 cache: reported, the length and the list as they were, the other slabs served.  The block's codes and scale
    stay too, although the row would raise it."""
    bt, hk, ms = 3, 2, 4
    c = filled(B, [[5, 20], [7, 8], [16, 9]], [40] * bt, hk, fmt, 16, paged, 3, window=2, max_sent=ms)
    row0 = [s * 40 for s in range(bt * hk)]
    ref = B.make_shape(bt, hk, hk, 128, 2, 0, ms, 40, torch.tensor([0, 40, 80]).cuda(), torch.tensor([40] * bt, dtype=torch.int32).cuda(), 40 * bt * hk)
    K16 = torch.zeros(40 * bt * hk, 128, dtype=torch.bfloat16, device="cuda")
    counts = torch.tensor([[-1, 1], [ms + 1, 2], [ms, 1 << 30]], dtype=torch.int32)
    mk = lambda: (torch.full((bt, hk, ms + 1), 77, dtype=torch.int32, device="cuda"), torch.full((bt, hk, ms), -1, dtype=torch.int32, device="cuda"),  # noqa: E731
                  counts.clone().cuda())
    a, b = mk(), mk()
    len16, out = c.kv_len.clone(), torch.full_like(c.kv_len, -1)
    x = torch.full((bt, hk, 128), 1000.0, dtype=torch.bfloat16, device="cuda")
    opens, gid = torch.tensor([1, 0, 0], dtype=torch.uint8).cuda(), torch.full((bt,), 5, dtype=torch.int32, device="cuda")
    before = [c.get(s, int(c.lens.reshape(-1)[s])) for s in range(c.slabs)]
    B.skipkv_append_step(ref, K16, K16.clone(), x, x, len16, a[0], a[1], a[2], opens, gid, None, None, 0, c.ws)
    torch.cuda.synchronize()
    assert c.status() == 4
    B.skipkv_append_step_q8(c.shape, c.cache, x, x, c.kv_len, out, b[0], b[1], b[2], opens, gid, None, None, 0, c.ws)
    torch.cuda.synchronize()
    assert c.status() == 4
    for u, v in zip(a, b):
        assert torch.equal(u, v)
    assert torch.equal(out, len16)
    ok = (counts >= 0) & (counts <= ms)
    assert torch.equal(out.cpu(), torch.from_numpy(c.lens) + ok.int())
    for s in range(c.slabs):
        n = int(c.lens.reshape(-1)[s])
        if ok.view(-1)[s]:
            assert all((row[0][n] == row[0][n][0]).all() for row in c.get(s, n + 1))
        else:
            for (x0, f0), (x1, f1) in zip(before[s], c.get(s, n)):
                assert np.array_equal(x0, x1) and np.array_equal(f0, f1)


# ------------------------------------------------------------------ tables of other slabs
@pytest.mark.parametrize("paged", [False, True])
def test_tables_of_more_sequences_are_taken(B, paged):
    """A cache laid out for five sequences serves the first three of them; one of fewer, or with other heads, is refused."""
    c = filled(B, [[100, 90]] * 5, [100] * 5, 2, "int8", 32, paged, 3, n_q=4)
    q = queries(c, 4, 5)
    whole = attend(c, q)
    few = B.make_shape(3, 4, 2, 128, 1, 0, 1, c.max_cap, c.slab_off, c.cap, c.rows16)
    out = torch.zeros(3, 4, 128, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(B.skipkv_workspace_bytes(few), dtype=torch.uint8, device="cuda")
    B.skipkv_workspace_init(few, ws)
    B.skipkv_decode_attn_q8(few, c.cache, q[:3], c.kv_len[:3], out, None, None, None, None, ws)
    torch.cuda.synchronize()
    assert B.skipkv_status(ws) == 0 and torch.equal(out, whole[:3])
    for batch, heads in ((6, 2), (5, 1), (5, 4)):
        shape = B.make_shape(batch, 2 * heads, heads, 128, 1, 0, 1, c.max_cap, c.slab_off, c.cap, c.rows16)
        with pytest.raises(B.SkipKVError) as e:
            B.skipkv_decode_attn_q8(shape, c.cache, q, c.kv_len, whole, None, None, None, None, c.ws)
        assert e.value.code == -1
