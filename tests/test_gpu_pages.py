"""Block tables and slot maps built on the GPU, against the oracle's one-slab-after-the-other form, and a run of the 8-bit and the paged
calls together as a server makes them."""
import numpy as np
import pytest
import torch

import oracle
from q8_common import DT, bf16
from test_gpu_q8 import check_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2512_07993_b200 import binding, build
    build.build()
    return binding


class Server:
    """Page state on the GPU and the oracle's beside it."""

    def __init__(self, B, bt, hk, max_pages, pool, seed, head=0):
        self.B, self.bt, self.hk, self.max_pages, self.pool = B, bt, hk, max_pages, pool
        r = np.random.default_rng(seed)
        ring = r.permutation(pool).astype(np.int32)
        self.ring_h, self.head, self.free = np.roll(ring, head % pool), head % pool, pool
        self.table_h, self.held = np.full((bt * hk, max_pages), -1, np.int32), np.zeros(bt * hk, np.int32)
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        self.ring, self.table = dev(self.ring_h), dev(self.table_h.reshape(bt, hk, max_pages))
        self.state, self.state2 = torch.tensor([self.head, self.free], dtype=torch.int32).cuda(), torch.full((2,), -9, dtype=torch.int32).cuda()
        self.n, self.n2 = (torch.zeros(bt, hk, dtype=torch.int32, device="cuda") for _ in range(2))
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def ask(self, need, bits=0):
        need = np.asarray(need, np.int32).reshape(self.bt, self.hk)
        self.B.skipkv_page_tables(self.bt, self.hk, self.max_pages, self.pool, torch.from_numpy(need).cuda(), self.n, self.n2, self.table, self.ring,
                                  self.state, self.state2, self.status)
        self.n, self.n2, self.state, self.state2 = self.n2, self.n, self.state2, self.state
        self.held, self.head, self.free, short = oracle.page_tables(need.reshape(-1), self.held, self.table_h, self.ring_h, self.head, self.free)
        torch.cuda.synchronize()
        assert int(self.status) == (0x10 if short else 0) | bits
        self.status.zero_()
        assert np.array_equal(self.n.cpu().numpy().reshape(-1), self.held)
        assert np.array_equal(self.table.cpu().numpy().reshape(-1, self.max_pages), self.table_h)
        assert np.array_equal(self.ring.cpu().numpy(), self.ring_h)
        assert self.state.tolist() == [self.head, self.free]


@pytest.mark.parametrize("bt,hk,max_pages,pool", [(1, 1, 1, 1), (2, 3, 5, 20), (16, 8, 520, 66000), (700, 4, 7, 9000), (1, 1, 3000, 3001)])
def test_tables(B, bt, hk, max_pages, pool):
    """Growing, shrinking, leaving and coming back, too few pages now and then, round the ring more than once."""
    r = np.random.default_rng(pool)
    sv = Server(B, bt, hk, max_pages, pool, 5, head=pool - 1)
    full = max_pages * 128
    sv.ask(np.zeros(bt * hk))
    sv.ask(np.ones(bt * hk))
    for _ in range(12):
        need = r.integers(0, full + 1, bt * hk)
        kind = r.random(bt * hk)
        need = np.where(kind < 0.3, sv.held * 128, np.where(kind < 0.5, 0, need))
        sv.ask(need)
    sv.ask(np.full(bt * hk, full))
    sv.ask(np.zeros(bt * hk))
    assert sv.free == pool


def test_tables_refuse_what_makes_no_sense(B):
    """Lengths below zero and beyond the table, counts outside it: that slab is left, the others are served."""
    sv = Server(B, 2, 2, 4, 12, 1)
    sv.ask([128, 256, 0, 300])
    need = torch.tensor([[-1, 4 * 128 + 1], [129, 2 ** 31 - 1]], dtype=torch.int32).cuda()
    before = sv.n.clone()
    B.skipkv_page_tables(2, 2, 4, 12, need, sv.n, sv.n2, sv.table, sv.ring, sv.state, sv.state2, sv.status)
    torch.cuda.synchronize()
    assert int(sv.status) == 4
    assert sv.n2.tolist() == [[int(before[0, 0]), int(before[0, 1])], [2, int(before[1, 1])]]
    assert sv.state2.tolist() == [sv.head + 2, sv.free - 2]
    # a ring that cannot be: nothing moves
    for ring in ([-1, 3], [12, 3], [0, 13], [0, -2]):
        sv.status.zero_()
        table = sv.table.clone()
        B.skipkv_page_tables(2, 2, 4, 12, need.clamp(0, 512), sv.n, sv.n2, sv.table, sv.ring, torch.tensor(ring, dtype=torch.int32).cuda(), sv.state2, sv.status)
        torch.cuda.synchronize()
        assert int(sv.status) == 4 and torch.equal(sv.n2, sv.n) and torch.equal(table, sv.table) and sv.state2.tolist() == ring
    # more pages come back than the pool has; pages in the ring that are none
    sv.status.zero_()
    B.skipkv_page_tables(2, 2, 4, 12, torch.zeros_like(need), sv.n, sv.n2, sv.table, sv.ring, torch.tensor([0, 10], dtype=torch.int32).cuda(), sv.state2, None)
    B.skipkv_page_tables(2, 2, 4, 12, torch.zeros_like(need), sv.n, sv.n2, sv.table, sv.ring, torch.tensor([0, 10], dtype=torch.int32).cuda(), sv.state2, sv.status)
    torch.cuda.synchronize()
    assert int(sv.status) == 4 and sv.state2.tolist() == [0, 12]
    sv.status.zero_()
    ring = torch.full((12,), 12, dtype=torch.int32, device="cuda")
    B.skipkv_page_tables(2, 2, 4, 12, torch.full_like(need, 512), torch.zeros_like(need), sv.n2, sv.table, ring, torch.tensor([0, 12], dtype=torch.int32).cuda(), sv.state2, sv.status)
    torch.cuda.synchronize()
    assert int(sv.status) == 4 | 0x10 and sv.table.view(-1)[:12].tolist() == [-1] * 12 and sv.n2.view(-1).tolist() == [4, 4, 4, 0]


@pytest.mark.parametrize("hk", [1, 2, 3, 8])
@pytest.mark.parametrize("lens", [[1], [0, 3, 0, 200, 1], [700] * 3, list(range(40)), [5000, 1, 1, 9000]])
def test_slots(B, hk, lens):
    """Ragged new tokens behind lengths that differ by head; tokens without a page; rows before and behind the sequences' are left."""
    bt, max_pages = len(lens), 90
    r = np.random.default_rng(hk)
    table = r.integers(0, 1 << 20, (bt * hk, max_pages)).astype(np.int32)
    start = r.integers(0, 700, bt * hk).astype(np.int32)
    n_pages = np.array([r.integers(max(0, -(-(int(start[s]) + lens[s // hk]) // 128) - 1), max_pages + 1) for s in range(bt * hk)], np.int32)
    for first in (0, 3):
        off = first + np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        n_new = int(off[-1]) + 4
        slots = torch.full((n_new, hk), -77, dtype=torch.int64, device="cuda")
        d = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()  # noqa: E731
        B.skipkv_slot_map(bt, hk, max_pages, d(table), d(n_pages), d(start), d(off), n_new, slots)
        torch.cuda.synchronize()
        want = oracle.slot_map(table, n_pages, start, off, hk, n_new, -77)
        assert np.array_equal(slots.cpu().numpy(), want)
    one = torch.full((bt + 1, hk), -77, dtype=torch.int64, device="cuda")
    B.skipkv_slot_map(bt, hk, max_pages, d(table), d(n_pages), d(start), None, bt, one)
    torch.cuda.synchronize()
    assert np.array_equal(one.cpu().numpy(), oracle.slot_map(table, n_pages, start, np.arange(bt + 1), hk, bt + 1, -77))
    # an odd place in memory: entries eight bytes at a time
    if hk % 2 == 0:
        buf = torch.full((bt * hk + 1,), -77, dtype=torch.int64, device="cuda")
        B.skipkv_slot_map(bt, hk, max_pages, d(table), d(n_pages), d(start), None, bt, buf[1:].view(bt, hk))
        torch.cuda.synchronize()
        assert torch.equal(buf[1:].view(bt, hk), one[:bt]) and int(buf[0]) == -77


def test_captured_tables_and_slots(B):
    """Both calls in a graph, replayed as lengths change in place."""
    sv = Server(B, 4, 2, 6, 60, 3)
    need, start = (torch.zeros(4, 2, dtype=torch.int32, device="cuda") for _ in range(2))
    slots = torch.zeros(4, 2, dtype=torch.int64, device="cuda")
    B.skipkv_slot_map(4, 2, 6, sv.table, sv.n, start, None, 4, slots)         # (loads the code before the capture)
    B.skipkv_page_tables(4, 2, 6, 60, need, sv.n, sv.n2, sv.table, sv.ring, sv.state, sv.state2, sv.status)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        torch.add(start, 1, out=need)
        B.skipkv_page_tables(4, 2, 6, 60, need, sv.n, sv.n2, sv.table, sv.ring, sv.state, sv.state2, sv.status)
        B.skipkv_slot_map(4, 2, 6, sv.table, sv.n2, start, None, 4, slots)
        sv.n.copy_(sv.n2)
        sv.state.copy_(sv.state2)
        start.add_(1)
    for step in range(300):
        g.replay()
        if step % 37 == 0 or step > 297:
            torch.cuda.synchronize()
            while int(sv.held[0]) * 128 < step + 1:
                need_h = np.full(8, int(sv.held[0]) * 128 + 1)
                sv.held, sv.head, sv.free, _ = oracle.page_tables(need_h, sv.held, sv.table_h, sv.ring_h, sv.head, sv.free)
            assert np.array_equal(sv.table.cpu().numpy().reshape(8, 6), sv.table_h)
            assert np.array_equal(slots.cpu().numpy(), oracle.slot_map(sv.table_h, sv.held, np.full(8, step), np.arange(5), 2, 4, 0))
    assert int(sv.status) == 0 and sv.state.tolist() == [sv.head, sv.free]


@pytest.mark.parametrize("pause", [True, False])
def test_pages_slots_append_and_attention_behind_one_another(B, pause):
    """A decode loop in which every call's input is what the call before it wrote, with and without a pause between them: pages are taken as
    slabs grow, and rows of a pool that no slab holds stay as they were."""
    bt, hk, max_pages, pool = 3, 2, 4, 30
    sv = Server(B, bt, hk, max_pages, pool, 9)
    K, V = (torch.full((pool * 128, 128), -128, dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((pool, 4), float("nan"), device="cuda") for _ in range(2))
    cache = B.make_q8_cache(K, V, ks, vs, 32, sv.table)
    off16 = torch.zeros(bt, dtype=torch.int64, device="cuda")
    cap = torch.full((bt,), max_pages * 128, dtype=torch.int32, device="cuda")
    shape = B.make_shape(bt, hk * 2, hk, 128, 1, 0, 1, max_pages * 128, off16, cap, pool * 128)
    ws = torch.empty(B.skipkv_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    B.skipkv_workspace_init(shape, ws)
    g = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.randn(260, bt, hk, 128, generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(260, bt, hk * 2, 128, generator=g, device="cuda").bfloat16()
    out, slots = torch.zeros_like(q), torch.full((260, bt, hk), -5, dtype=torch.int64, device="cuda")
    n, n2 = sv.n, sv.n2
    state, state2 = sv.state, sv.state2
    kv = torch.zeros(261, bt, hk, dtype=torch.int32, device="cuda")
    kv[0] = torch.tensor([[100, 120], [0, 127], [128, 250]], dtype=torch.int32)
    need = kv[0].clone()
    B.skipkv_page_tables(bt, hk, max_pages, pool, need, n, n2, sv.table, sv.ring, state, state2, sv.status)
    n, n2, state, state2 = n2, n, state2, state
    torch.cuda.synchronize()
    for i in range(260):
        torch.add(kv[i], 1, out=need)
        for call in (lambda: B.skipkv_page_tables(bt, hk, max_pages, pool, need, n, n2, sv.table, sv.ring, state, state2, sv.status),
                     lambda: B.skipkv_slot_map(bt, hk, max_pages, sv.table, n2, kv[i], None, bt, slots[i]),
                     lambda: B.skipkv_append_q8(shape, cache, k[i], v[i], None, bt, kv[i], kv[i + 1], ws),
                     lambda: B.skipkv_decode_attn_q8(shape, cache, q[i], kv[i + 1], out[i], None, None, None, None, ws)):
            call()
            if pause:
                torch.cuda.synchronize()
        n, n2, state, state2 = n2, n, state2, state
    torch.cuda.synchronize()
    # (the tokens before the first step were never stored: junk codes of scale NaN, so those slabs' results are NaN; slab (1, 0) began empty)
    assert int(sv.status) == 0 and B.skipkv_status(ws, raise_on_error=False) == 0
    assert kv[260].tolist() == [[360, 380], [260, 387], [388, 510]] and n.tolist() == [[3, 3], [3, 4], [4, 4]]
    assert state.tolist()[1] == pool - 21
    table, sl = sv.table.cpu().numpy(), slots.cpu().numpy()
    held = {int(p) for b in range(bt) for h in range(hk) for p in table[b, h, :int(n[b, h])]}
    assert len(held) == 21
    for i in (0, 1, 27, 28, 127, 128, 259):
        for b in range(bt):
            for h in range(hk):
                t = int(kv[0, b, h]) + i
                assert sl[i, b, h] == table[b, h, t // 128] * 128 + t % 128
    free = torch.ones(pool, dtype=torch.bool)
    free[list(held)] = False
    assert bool((K.view(pool, 128, 128)[free.cuda()] == -128).all()) and bool(torch.isnan(ks[free.cuda()]).all())
    host = [[np.zeros((512, 128), np.uint8), np.zeros(16)] for _ in range(2)]
    for j, x in enumerate((k, v)):
        for i in range(260):
            oracle.q8_append(*host[j], i, x[i, 1, 0][None].double().cpu().numpy(), 32, "int8")
            if i in (0, 130, 259):
                rows = oracle.q8_rows(*host[j], i + 1, 32, "int8")
                if j == 0:
                    keys = getattr(sv, "keys", {})
                    keys[i] = rows
                    sv.keys = keys
                else:
                    check_attention(type("C", (), dict(hk=1, slabs=1, rows64=[[sv.keys[i]], [rows]])), q[i, 1:2, :2], out[i, 1:2, :2])


def test_slots_scatter_a_prompt_into_a_bf16_pool(B):
    """Pages for prompts, their slots as an index for torch's copy, and the paged bf16 attention over the result."""
    bt, hk, group, lens = 3, 2, 4, [300, 1, 129]
    sv = Server(B, bt, hk, 3, 20, 3)
    sv.ask(np.repeat(lens, hk))
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()
    n = int(off[-1])
    slots = torch.full((n, hk), -1, dtype=torch.int64, device="cuda")
    B.skipkv_slot_map(bt, hk, 3, sv.table, sv.n, torch.zeros_like(sv.n), off, n, slots)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(n, hk, 128, generator=g, device="cuda").bfloat16() for _ in range(2))
    K, V = (torch.full((20 * 128, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    K[slots] = k
    V[slots] = v
    kv = torch.from_numpy(np.repeat(np.array(lens, np.int32)[:, None], hk, 1).copy()).cuda()
    off64, cap = torch.zeros(bt, dtype=torch.int64, device="cuda"), torch.full((bt,), 384, dtype=torch.int32, device="cuda")
    shape = B.make_shape(bt, hk * group, hk, 128, 1, 0, 1, 384, off64, cap, 20 * 128)
    ws = torch.empty(B.skipkv_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    B.skipkv_workspace_init(shape, ws)
    q = torch.randn(bt, hk * group, 128, generator=g, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    B.skipkv_decode_attn_paged(shape, q, K, V, sv.table, 3, kv, out, None, None, None, None, ws)
    torch.cuda.synchronize()
    assert B.skipkv_status(ws) == 0
    rows = [[], []]
    for s in range(bt * hk):
        b, h = divmod(s, hk)
        for i, x in enumerate((k, v)):
            rows[i].append(x[int(off[b]):int(off[b + 1]), h].double().cpu().numpy())
    check_attention(type("C", (), dict(hk=hk, slabs=bt * hk, rows64=rows)), q, out)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("block", [16, 128])
def test_server_loop(B, fmt, block):
    """As a program uses them together: pages for the prompts, the prompts in two parts into the paged 8-bit cache, decode steps
    with page tables, append and attention, an eviction through bf16 (unpack, score, select, compact, pack), pages given back, and on."""
    bt, hk, group, window, budget = 3, 2, 4, 4, 150
    hq, ms, max_pages, pool = hk * group, 40, 5, 34
    cap_rows = max_pages * 128
    r = np.random.default_rng(block)
    sv = Server(B, bt, hk, max_pages, pool, 2)
    K, V = (torch.zeros(pool * 128, 128, dtype=torch.uint8, device="cuda").view(DT[fmt]) for _ in range(2))
    ks, vs = (torch.full((pool, 128 // block), float("nan"), device="cuda") for _ in range(2))
    cache = B.make_q8_cache(K, V, ks, vs, block, sv.table)
    off16 = torch.arange(bt, dtype=torch.int64, device="cuda") * cap_rows
    cap = torch.full((bt,), cap_rows, dtype=torch.int32, device="cuda")
    shape = B.make_shape(bt, hq, hk, 128, window, 0, ms, cap_rows, off16, cap, bt * hk * cap_rows)
    params = B.make_params(0.1, 0.95, 1e-6, budget, window)
    ws = torch.empty(B.skipkv_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    B.skipkv_workspace_init(shape, ws)
    K16, V16 = (torch.zeros(bt * hk * cap_rows, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    host = [[(np.zeros((cap_rows, 128), np.uint8), np.zeros(cap_rows // block)) for _ in range(bt * hk)] for _ in range(2)]
    lens = np.zeros(bt * hk, np.int64)
    kv, kv2 = (torch.zeros(bt, hk, dtype=torch.int32, device="cuda") for _ in range(2))

    def add(x, counts):
        at = 0
        for b, n in enumerate(counts):
            for h in range(hk):
                s = b * hk + h
                for i in range(2):
                    oracle.q8_append(*host[i][s], int(lens[s]), x[i][at:at + n, h].double().numpy(), block, fmt)
                lens[s] += n
            at += n

    def check():
        rows = [[oracle.q8_rows(*host[i][s], int(lens[s]), block, fmt) for s in range(bt * hk)] for i in range(2)]
        q = bf16(r.normal(0, 1, (bt, hq, 128))).cuda()
        out = torch.full_like(q, float("nan"))
        B.skipkv_decode_attn_q8(shape, cache, q, kv, out, None, None, None, None, ws)
        torch.cuda.synchronize()
        assert B.skipkv_status(ws) == 0 and np.array_equal(kv.cpu().numpy().reshape(-1), lens)
        check_attention(type("C", (), dict(hk=hk, slabs=bt * hk, rows64=rows)), q, out)
        return q

    for counts in ([200, 131, 77], [100, 0, 128]):
        sv.ask(lens + np.repeat(counts, hk))
        n = sum(counts)
        x = [bf16(r.normal(0, 1, (n, hk, 128)) * np.exp2(r.integers(-2, 3, (n, 1, 1)))) for _ in range(2)]
        off = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
        B.skipkv_append_q8(shape, cache, x[0].cuda(), x[1].cuda(), off, n, kv, kv2, ws)
        kv, kv2 = kv2, kv
        add(x, counts)
        check()
    # sentences of 13 tokens
    so = np.minimum(np.arange(ms + 1)[None] * 13, lens[:, None]).astype(np.int32).reshape(bt, hk, ms + 1)
    sent_off = torch.from_numpy(so).cuda()
    n_sent = torch.from_numpy((-(-lens // 13)).astype(np.int32).reshape(bt, hk)).cuda()
    sent_id = torch.arange(ms, dtype=torch.int32, device="cuda").repeat(bt, hk, 1)
    q_win = bf16(r.normal(0, 1, (bt, hq, window, 128))).cuda()
    opens = torch.zeros(bt, dtype=torch.uint8, device="cuda")
    gid = torch.full((bt,), 99, dtype=torch.int32, device="cuda")

    def steps(count):
        nonlocal kv, kv2
        for i in range(count):
            sv.ask(lens + 1)
            x = [bf16(r.normal(0, 1 + i, (bt, hk, 128))) for _ in range(2)]
            q = check() if i % 3 == 0 else bf16(r.normal(0, 1, (bt, hq, 128))).cuda()
            B.skipkv_append_step_q8(shape, cache, x[0].cuda(), x[1].cuda(), kv, kv2, sent_off, sent_id, n_sent, opens, gid, q_win, q, i % window, ws)
            torch.cuda.synchronize()
            assert torch.equal(q_win[:, :, i % window], q)
            kv, kv2 = kv2, kv
            add(x, [1] * bt)

    steps(8)
    # eviction
    B.skipkv_unpack_q8(shape, cache, kv, K16, V16, ws)
    torch.cuda.synchronize()
    for s in range(bt * hk):
        for i, x in enumerate((K16, V16)):
            assert np.array_equal(x[s * cap_rows:s * cap_rows + int(lens[s])].double().cpu().numpy(), oracle.q8_rows(*host[i][s], int(lens[s]), block, fmt))
    f32 = [torch.zeros(bt, hk, ms, device="cuda") for _ in range(4)]
    B.skipkv_score(shape, params, K16, q_win, kv, sent_off, n_sent, None, *f32, ws)
    keep = torch.zeros(bt, hk, ms, dtype=torch.uint8, device="cuda")
    B.skipkv_select(shape, params, f32[3], sent_off, n_sent, keep, None, None, None, ws)
    B.skipkv_compact(shape, K16, V16, keep, sent_off, sent_id, n_sent, kv, None, ws)
    torch.cuda.synchronize()
    assert B.skipkv_status(ws) == 0
    lens = kv.cpu().numpy().reshape(-1).astype(np.int64)
    assert (lens <= budget).all() and (lens > 0).all()
    sv.ask(lens)
    B.skipkv_pack_q8(shape, cache, K16, V16, kv, ws)
    torch.cuda.synchronize()
    for s in range(bt * hk):
        for i, x in enumerate((K16, V16)):
            host[i][s] = (np.zeros((cap_rows, 128), np.uint8), np.zeros(cap_rows // block))
            oracle.q8_append(*host[i][s], 0, x[s * cap_rows:s * cap_rows + int(lens[s])].double().cpu().numpy(), block, fmt)
    check()
    steps(4)
    check()
    sv.ask(np.zeros(bt * hk))
    assert sv.free == pool


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two devices")
def test_tensors_of_another_device_are_refused(B):
    here, there = (torch.zeros(1, 1, dtype=torch.int32, device=f"cuda:{i}") for i in (0, 1))
    slots = torch.zeros(1, 1, dtype=torch.int64, device="cuda:0")
    with torch.cuda.device(0):
        for k in range(3):
            a = [here] * 3
            a[k] = there
            with pytest.raises(ValueError, match="another device"):
                B.skipkv_slot_map(1, 1, 1, *a, None, 1, slots)
