"""Calls on the 8-bit cache and the page tables that would reach beyond their tables: refused before a launch, without a GPU."""
import ctypes as C
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def binding():
    from paper_2512_07993_b200 import build, binding
    build.build()
    return binding


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("batch,heads,code", [(1, 2, -1), (2, 1, -1), (2, 4, -1), (4, 1, -1), (0, 2, -1), (2, 0, -1)])
def test_tables_of_other_slabs_are_refused(binding, paged, batch, heads, code):
    """Scales or a block table for fewer sequences than the shape has, or for other KV heads.  (The pointers are never followed.)"""
    lib = binding.lib()
    shape = binding.make_shape(2, 8, 2, 128, 8, 256, 16, 256, None, None, 1024)
    shape.slab_off, shape.cap = 256, 256
    c = binding.Q8Cache(0, 64, 4, 2, -1, 0, 1024, 4096, 8192, 256, 512, 256 if paged else None, batch, heads)
    s, k, p, q, none = C.byref(shape), C.byref(c), C.c_void_p(4096), C.c_void_p(8192), C.c_void_p(None)
    assert lib.skipkv_pack_q8(s, k, p, p, p, p, none) == code
    assert lib.skipkv_append_q8(s, k, p, p, p, 2, p, q, p, none) == code
    assert lib.skipkv_append_step_q8(s, k, p, p, p, q, p, p, p, p, p, none, none, 0, p, none) == code
    assert lib.skipkv_decode_attn_q8(s, k, p, p, p, none, none, none, none, p, none) == code
    assert lib.skipkv_unpack_q8(s, k, p, p, p, p, none) == code


def test_make_q8_cache_keeps_the_slabs_of_its_tables(binding, monkeypatch):
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype=None: None)
    K = torch.zeros(256, 128, dtype=torch.int8)
    c = binding.make_q8_cache(K, K, torch.zeros(3, 5, 2), torch.zeros(3, 5, 2), 64)
    assert (c.batch, c.n_kv_heads) == (3, 5)
    c = binding.make_q8_cache(K, K, torch.zeros(2, 2), torch.zeros(2, 2), 64, torch.zeros(4, 7, 1, dtype=torch.int32))
    assert (c.batch, c.n_kv_heads) == (4, 7)


@pytest.mark.parametrize("slabs,max_pages,pool", [(1, (1 << 31) - 8, 16), (4, (1 << 29) - 1, 1 << 20), (8192, (1 << 18) - 1, 1 << 23)])
def test_page_tables_whose_places_pass_32_bits_are_refused(binding, slabs, max_pages, pool):
    """Counts that claim whole rows of the block table, given back behind the free pages: a place of the ring would be a sum beyond 2^31."""
    assert slabs * max_pages < 1 << 31 <= slabs * max_pages + pool
    p, q = C.c_void_p(4096), C.c_void_p(8192)
    assert binding.lib().skipkv_page_tables(slabs, 1, max_pages, pool, p, p, q, p, p, p, q, None, None) == -2


@pytest.mark.parametrize("over", [dict(max_blocks=(1 << 28) - 2), dict(block_table=256, max_pages=(1 << 28) - 2)])
def test_tables_whose_last_step_passes_32_bits_are_refused(binding, over):
    """Four slabs with all but eight of 2^30 places: a CTA's step behind the last tile of K and V would be a number beyond 2^31."""
    lib = binding.lib()
    shape = binding.make_shape(2, 8, 2, 128, 8, 256, 16, 256, None, None, 1024)
    shape.slab_off, shape.cap = 256, 256
    c = binding.Q8Cache(0, 64, 4, 2, -1, 0, 1024, 4096, 8192, 256, 512, None)
    for k, v in over.items():
        setattr(c, k, v)
    s, k, p, q, none = C.byref(shape), C.byref(c), C.c_void_p(4096), C.c_void_p(8192), C.c_void_p(None)
    assert lib.skipkv_unpack_q8(s, k, p, p, p, p, none) == -2
    assert lib.skipkv_pack_q8(s, k, p, p, p, p, none) == -2
    assert lib.skipkv_append_q8(s, k, p, p, p, 2, p, q, p, none) == -2
    assert lib.skipkv_decode_attn_q8(s, k, p, p, p, none, none, none, none, p, none) == -2


# ------------------------------------------------------------------ the kernels' counts, compiled for the host
COUNTS = r"""
#include <climits>
#include <cstdio>
#include "q8.cuh"
using namespace skipkv;
int main() {
    const int caps[] = {INT_MIN, -1, 0, 1, 128, 0x7ffffeff, 0x7fffff00, 0x7fffff01, INT_MAX - 1, INT_MAX};
    for (int paged = 0; paged < 2; ++paged)
        for (int log2 = 4; log2 <= 7; ++log2)
            for (int most : {1, 1 << 20, 1 << 24, 1 << 25, (1 << 30) - 5000})
                for (int cap : caps) {
                    Q8View v{};
                    int32_t table = 0;
                    v.table = paged ? &table : nullptr;
                    v.block_log2 = log2; v.max_blocks = v.max_pages = most;
                    const int room = q8_room(v, cap);
                    // the tiles of a slab that is full, as the kernels count them
                    const unsigned tiles = unsigned(room) + unsigned(kQ8Tile) - 1u;
                    if (room < 0 || room > (cap < 0 ? 0 : cap) || tiles > unsigned(INT_MAX)) { printf("%d %d %d %d: %d\n", paged, log2, most, cap, room); return 1; }
                }
    return 0;
}
"""


def test_tiles_of_the_longest_slab_are_numbers_of_32_bits(binding, tmp_path):
    """Whatever a table of capacities says: 127 rows more than a slab's room, the sum from which its tiles are counted, stay below 2^31."""
    from paper_2512_07993_b200 import build
    src, exe = tmp_path / "counts.cu", tmp_path / "counts"
    src.write_text(COUNTS)
    subprocess.run([build.NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(ROOT, "include"), "-I", build.CSRC,
                    str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True)
    assert got.returncode == 0, got.stdout
