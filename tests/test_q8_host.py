"""The 8-bit cache and the page tables without a GPU: the oracle's pins, the argument checks of the C entries, and the kernels' address
arithmetic (bad pages, slabs that reach beyond their buffers) compiled for the host."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import oracle

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def binding():
    from paper_2512_07993_b200 import build, binding
    build.build()
    return binding


# ------------------------------------------------------------------ oracle
def test_e4m3_values_are_those_of_the_type():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = oracle.q8_values("e4m3")
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])
    assert np.nanmax(got) == 448 and got[1] == 2.0 ** -9


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_nearest_code(fmt):
    """All codes stand for themselves, every midpoint of neighbours goes to the even one, and (e4m3) a cast of the type agrees."""
    v = oracle.q8_values(fmt)
    good = np.array([c for c in range(256) if np.isfinite(v[c]) and abs(v[c]) <= oracle.Q8_TOP[fmt]])
    assert np.array_equal(oracle.q8_nearest(v[good], fmt)[v[good] != 0], good[v[good] != 0])
    grid = np.sort(np.unique(v[good]))
    mid = (grid[1:] + grid[:-1]) / 2
    picked = oracle.q8_nearest(mid, fmt)
    assert (picked % 2 == 0).all()
    assert (np.abs(v[picked] - mid) == np.diff(grid) / 2).all()
    for side in (-1, 1):
        near = oracle.q8_nearest(mid + side * np.diff(grid) * 0.01, fmt)
        assert np.array_equal(v[near], grid[1:] if side > 0 else grid[:-1])
    y = np.random.default_rng(3).normal(0, oracle.Q8_TOP[fmt] / 4, 20000).astype(np.float32).clip(-oracle.Q8_TOP[fmt], oracle.Q8_TOP[fmt])
    if fmt == "e4m3":
        want = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    else:
        want = np.rint(y).astype(np.int8).view(np.uint8)
    assert np.array_equal(oracle.q8_nearest(y, fmt), want)
    assert np.array_equal(v[oracle.q8_nearest([np.inf, -np.inf, np.nan], fmt)], [oracle.Q8_TOP[fmt], -oracle.Q8_TOP[fmt], 0])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_scale_is_the_least_power_of_two(fmt):
    top = oracle.Q8_TOP[fmt]
    for amax in (1.0, top, top * 1.0001, 2 * top, 3e38, 1e-20, np.float64(top) / 3):
        s = oracle.q8_scale([amax, -amax / 2, 0], fmt)
        assert amax <= top * s and amax > top * s / 2 and np.log2(s) == np.round(np.log2(s))
    assert oracle.q8_scale([0.0], fmt) == 2.0 ** -100 == oracle.q8_scale([], fmt)
    assert oracle.q8_scale([np.inf, np.nan, 2.0], fmt) == oracle.q8_scale([2.0], fmt)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_appending_rows_one_by_one_stays_within_the_roundings(fmt):
    """A value is rounded once as it comes and once more each time its block's scale doubles: with powers of two the half steps of the
    smaller scales add up to less than one half step of the last, so the error is below one step in all."""
    r = np.random.default_rng(5)
    x = r.normal(0, 1, (40, 128)) * np.exp(r.normal(0, 1, (40, 1)))
    codes, scale, n = np.zeros((40, 128), np.uint8), np.ones(3), 0
    for row in x:
        n = oracle.q8_append(codes, scale, n, row[None], 16, fmt)
    got = oracle.q8_rows(codes, scale, n, 16, fmt)
    s = scale[np.arange(40) // 16][:, None]
    step = s if fmt == "int8" else np.maximum(np.abs(got) * 2.0 ** -2, s * 2.0 ** -9)
    assert (np.abs(got - x) <= step).all()
    whole, ws = np.zeros((40, 128), np.uint8), np.ones(3)
    oracle.q8_append(whole, ws, 0, x, 16, fmt)
    assert np.array_equal(ws, scale)


def test_pages_are_neither_lost_nor_given_twice():
    r = np.random.default_rng(11)
    slabs, max_pages, pool = 12, 9, 40
    table, ring = np.full((slabs, max_pages), -1), r.permutation(pool)
    held, head, free = np.zeros(slabs, np.int32), 7, pool
    ring = np.roll(ring, 7)
    for _ in range(60):
        need = r.integers(0, max_pages * 128 + 1, slabs)
        need = np.where(r.random(slabs) < 0.4, held * 128, need)
        held, head, free, short = oracle.page_tables(need, held, table, ring, head, free)
        out = [int(table[s][j]) for s in range(slabs) for j in range(held[s])]
        rest = [int(ring[(head + i) % pool]) for i in range(free)]
        assert sorted(out + rest) == list(range(pool))
        assert short or (held == -(-need // 128)).all()


# ------------------------------------------------------------------ argument checks of the C entries
def _args(binding, **over):
    """A shape and a cache whose pointers are never followed: every call here is refused before a launch."""
    shape = binding.make_shape(2, 8, 2, 128, 8, 256, 16, 256, None, None, 1024)
    shape.slab_off, shape.cap = 256, 256
    c = binding.Q8Cache(0, 64, 4, 0, -1, 0, 1024, 4096, 8192, 256, 512, None)
    for k, v in over.items():
        setattr(c, k, v)
    return shape, c


BAD_CACHES = [(dict(K=None), -1), (dict(V=None), -1), (dict(k_scale=None), -1), (dict(v_scale=None), -1), (dict(rows=0), -1),
              (dict(format=2), -2), (dict(format=-1), -2), (dict(block_rows=8), -2), (dict(block_rows=48), -2), (dict(block_rows=256), -2),
              (dict(K=4097), -1), (dict(V=4104), -1), (dict(k_scale=258), -1), (dict(max_blocks=0), -1),
              (dict(block_table=256, max_pages=0), -1), (dict(block_table=256, max_pages=2, rows=1000), -1), (dict(rows=1 << 31), -2)]


@pytest.mark.parametrize("over,code", BAD_CACHES)
def test_bad_caches_are_refused(binding, over, code):
    lib = binding.lib()
    shape, c = _args(binding, **over)
    s, k, p = C.byref(shape), C.byref(c), C.c_void_p(4096)
    none = C.c_void_p(None)
    assert lib.skipkv_pack_q8(s, k, p, p, p, p, none) == code
    assert lib.skipkv_append_q8(s, k, p, p, p, 2, p, C.c_void_p(8192), p, none) == code
    assert lib.skipkv_append_step_q8(s, k, p, p, p, C.c_void_p(8192), p, p, p, p, p, none, none, 0, p, none) == code
    assert lib.skipkv_decode_attn_q8(s, k, p, p, p, none, none, none, none, p, none) == code
    assert lib.skipkv_unpack_q8(s, k, p, p, p, p, none) == code


def test_bad_arguments_are_refused(binding):
    lib = binding.lib()
    shape, c = _args(binding)
    s, k, p, q, none, odd = C.byref(shape), C.byref(c), C.c_void_p(4096), C.c_void_p(8192), C.c_void_p(None), C.c_void_p(4100)
    for a in ((s, none, p, p, p, p), (s, k, none, p, p, p), (s, k, p, none, p, p), (s, k, p, p, none, p), (none, k, p, p, p, p), (s, k, odd, p, p, p)):
        assert lib.skipkv_pack_q8(*a, none) == -1
    assert lib.skipkv_pack_q8(s, k, p, p, p, none, none) == -3
    assert lib.skipkv_pack_q8(s, k, p, p, p, odd, none) == -3
    bad = [(none, p, p, 2, p, q), (p, none, p, 2, p, q), (p, p, p, 2, none, q), (p, p, p, 2, p, none), (p, p, p, 2, p, p), (p, p, p, -1, p, q),
           (p, p, none, 3, p, q), (odd, p, p, 2, p, q)]
    for kn, vn, off, n, li, lo in bad:
        assert lib.skipkv_append_q8(s, k, kn, vn, off, n, li, lo, p, none) == -1
    assert lib.skipkv_append_q8(s, k, p, p, p, 2, p, q, none, none) == -3
    step = lambda *a: lib.skipkv_append_step_q8(s, k, p, p, p, q, *a, p, none)  # noqa: E731
    for i in range(5):
        a = [p] * 5
        a[i] = none
        assert step(*a, none, none, 0) == -1
    assert step(p, p, p, p, p, p, none, 0) == -1 and step(p, p, p, p, p, none, p, 0) == -1        # a window without queries, queries without one
    assert step(p, p, p, p, p, p, p, 8) == -1 and step(p, p, p, p, p, p, p, -1) == -1             # slots outside the window
    attn = lambda q_, kv, out, hid=none, st=none, al=none, fl=none, ws=p: lib.skipkv_decode_attn_q8(s, k, q_, kv, out, hid, st, al, fl, ws, none)  # noqa: E731
    assert attn(none, p, p) == -1 and attn(p, none, p) == -1 and attn(p, p, none) == -1 and attn(odd, p, p) == -1
    assert attn(p, p, p, hid=p) == -1 and attn(p, p, p, hid=C.c_void_p(4104), st=p, al=p, fl=p) == -1
    assert attn(p, p, p, ws=none) == -3
    assert lib.skipkv_unpack_q8(s, k, p, none, none, p, none) == -1
    assert lib.skipkv_unpack_q8(s, k, none, p, p, p, none) == -1
    many, _ = _args(binding)
    many.batch = 5000                                                                            # 10000 slabs
    assert lib.skipkv_pack_q8(C.byref(many), k, p, p, p, p, none) == -2
    assert lib.skipkv_decode_attn_q8(C.byref(many), k, p, p, p, none, none, none, none, p, none) == -2
    assert lib.skipkv_unpack_q8(C.byref(many), k, p, p, p, p, none) == -2


@pytest.mark.parametrize("over", [dict(max_blocks=1 << 28), dict(block_table=256, max_pages=1 << 28)])
def test_tables_beyond_32_bits_are_refused(binding, over):
    """Four slabs: 2^30 scales or pages, whose places and tiles (K and V) would not be numbers of 32 bits."""
    lib = binding.lib()
    shape, c = _args(binding, **over)
    s, k, p, none = C.byref(shape), C.byref(c), C.c_void_p(4096), C.c_void_p(None)
    assert lib.skipkv_pack_q8(s, k, p, p, p, p, none) == -2
    assert lib.skipkv_append_q8(s, k, p, p, p, 2, p, C.c_void_p(8192), p, none) == -2
    assert lib.skipkv_decode_attn_q8(s, k, p, p, p, none, none, none, none, p, none) == -2
    assert lib.skipkv_unpack_q8(s, k, p, p, p, p, none) == -2
    # a range of tokens whose end and one pass of a warp more is no number of 32 bits
    assert lib.skipkv_slot_map(1, 1, 4, p, p, p, p, (1 << 31) - 1, p, none) == -2


def test_page_calls_refuse_bad_arguments(binding):
    lib = binding.lib()
    p, q, none = C.c_void_p(4096), C.c_void_p(8192), C.c_void_p(None)
    tables = lambda bt=2, hk=2, mp=4, pool=16, a=(p, p, q, p, p, p, q): lib.skipkv_page_tables(bt, hk, mp, pool, *a, none, none)  # noqa: E731
    for over in (dict(bt=0), dict(hk=0), dict(mp=0), dict(pool=0)):
        assert tables(**over) == -1
    for i in range(7):
        a = [p, C.c_void_p(256), q, p, p, p, q]
        a[i] = none
        assert tables(a=a) == -1
    assert tables(a=(p, q, q, p, p, p, q)) == -1              # counts in place
    assert tables(a=(q, p, q, p, p, p, q)) == -1              # over the lengths
    assert tables(a=(p, p, q, p, p, p, p)) == -1              # ring state in place
    assert tables(bt=5000) == -2 and tables(pool=1 << 25) == -2 and tables(bt=4096, mp=1 << 20) == -2
    slots = lambda bt=2, hk=2, mp=4, t=p, n=p, st=p, off=p, new=3, out=p: lib.skipkv_slot_map(bt, hk, mp, t, n, st, off, new, out, none)  # noqa: E731
    for over in (dict(bt=0), dict(hk=0), dict(mp=0), dict(t=none), dict(n=none), dict(st=none), dict(new=-1), dict(out=none), dict(off=none)):
        assert slots(**over) == -1
    assert slots(new=0, out=none) == 0
    assert slots(new=1 << 30, hk=4) == -2


def test_make_q8_cache_checks_its_tensors(binding):
    K = torch.zeros(256, 128, dtype=torch.int8)
    sc = torch.zeros(1, 2, 2)
    with pytest.raises(ValueError, match="float8_e4m3fn or torch.int8"):
        binding.make_q8_cache(K.to(torch.uint8), K, sc, sc, 64)
    with pytest.raises(ValueError, match="alike"):
        binding.make_q8_cache(K, K.view(torch.float8_e4m3fn), sc, sc, 64)
    with pytest.raises(ValueError, match=r"\[rows\]\[128\]"):
        binding.make_q8_cache(K.view(512, 64), K.view(512, 64), sc, sc, 64)
    with pytest.raises(ValueError, match="block_rows"):
        binding.make_q8_cache(K, K, sc, sc, 8)
    with pytest.raises(ValueError, match="different shapes"):
        binding.make_q8_cache(K, K, sc, sc[:, :1], 64)
    with pytest.raises(ValueError, match="max_blocks"):
        binding.make_q8_cache(K, K, sc[0], sc[0], 64)
    table = torch.zeros(1, 2, 1, dtype=torch.int32)
    with pytest.raises(ValueError, match="pages"):
        binding.make_q8_cache(K, K, sc, sc, 64, table)
    with pytest.raises(ValueError, match="whole pages"):
        binding.make_q8_cache(K[:200], K[:200], sc, sc, 64, table)
    with pytest.raises(ValueError, match="device-resident"):
        binding.make_q8_cache(K, K, sc, sc, 64)                # host memory


# ------------------------------------------------------------------ the kernels' addresses, compiled for the host
ADDRESSES = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "q8.cuh"
using namespace skipkv;
static long long rnd(long long n) { return n > 0 ? ((long long)rand() << 16 ^ rand()) % n : 0; }
int main() {
    srand(7);
    long long checked = 0, refused = 0;
    for (int trial = 0; trial < 20000; ++trial) {
        const int Hk = 1 + int(rnd(4)), batch = 1 + int(rnd(3)), log2 = 4 + int(rnd(4));
        const bool paged = rnd(2);
        Q8View v{};
        v.block_log2 = log2;
        v.max_pages = 1 + int(rnd(5));
        v.rows = paged ? 128 * (1 + rnd(20)) : 1 + rnd(6000);
        v.max_blocks = paged ? 128 >> log2 : 1 + int(rnd(60));
        std::vector<int32_t> table(size_t(batch) * Hk * v.max_pages), cap(batch);
        for (auto& p : table) p = rnd(4) ? int32_t(rnd(v.rows / 128 + 1)) : int32_t(rnd(8) == 0 ? rnd(1ll << 31) : -1 - rnd(1ll << 31));
        std::vector<int64_t> off(batch);
        for (int b = 0; b < batch; ++b) { cap[b] = int32_t(rnd(900)) - 20; off[b] = rnd(6) ? rnd(1500) : -rnd(1ll << 40); }
        v.table = paged ? table.data() : nullptr;
        for (int s = 0; s < batch * Hk; ++s) {
            const int room = q8_room(v, cap.data(), Hk, s);
            const long long most = paged ? 128ll * v.max_pages : (long long)v.max_blocks << log2;
            if (room < 0 || room > most || (room > 0 && room > cap[s / Hk])) { printf("room %d\n", room); return 1; }
            for (int j = 0; j * 128 < room; ++j) {
                const int rows = room - j * 128 < 128 ? room - j * 128 : 128;
                const Q8Tile t = q8_tile(v, s, j, rows, q8_row0(off.data(), cap.data(), Hk, s));
                ++checked;
                if (t.row < 0) { ++refused; continue; }
                if (t.row + rows > v.rows) { printf("row %lld of %lld\n", t.row, v.rows); return 1; }
                const size_t scales = paged ? size_t(v.rows / 128) << (7 - log2) : size_t(batch) * Hk * v.max_blocks;
                const size_t blocks = size_t(rows + (1 << log2) - 1) >> log2;
                if (t.scale + blocks > scales) { printf("scale %zu + %zu of %zu\n", t.scale, blocks, scales); return 1; }
            }
        }
    }
    printf("ok %lld %lld\n", checked, refused);
    return 0;
}
"""


def test_addresses_stay_inside_the_buffers(tmp_path):
    """Random caches with bad pages, short scale tables and slabs beyond the buffers: a tile is either refused or lies inside."""
    src, exe = tmp_path / "addresses.cu", tmp_path / "addresses"
    src.write_text(ADDRESSES)
    from paper_2512_07993_b200 import build
    subprocess.run([build.NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(ROOT, "include"), "-I", build.CSRC,
                    str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True)
    assert got.returncode == 0, got.stdout
    word, checked, refused = got.stdout.split()
    assert word == "ok" and int(checked) > 50000 and int(refused) > 1000
