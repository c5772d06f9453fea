"""The paged cache without a device: how its attention deals key steps out and finds the parts again, what the library refuses, and the
reference's eviction on small cases worked out by hand."""
import ctypes as C
import os
import random
import re
import subprocess

import pytest

import paged_ref as pr
from paper_2406_13170_amd import binding as B
from paper_2406_13170_amd.build import CSRC
from test_boundary_cpu import base_cfg

HARNESS = r"""
#define __host__
#define __device__
#include <vector>
#include "paged_plan.h"
using namespace amph;
// The pieces of the workgroups over walks of the given steps (U a sequence): every step in one piece, every cut part in the place where
// the walk's list has it, no place used twice.  Returns 0, or the number of the rule that fails.
extern "C" int deal(const int *steps, int n_seq, int U) {
  const int wgs = PAGED_WGS;
  long long total = 0;
  std::vector<long long> first;
  for (int b = 0; b < n_seq; ++b) for (int u = 0; u < U; ++u) { first.push_back(total); total += steps[b]; }
  const PagedDeal d = paged_deal(total);
  if (d.begin(0) != 0 || d.begin(wgs) < total) return 1;
  std::vector<int> seen(total, 0), place(2 * wgs, -1), at(2 * wgs, -1);
  for (int w = 0; w < wgs; ++w) {
    const long long pos = d.begin(w), end = d.begin(w + 1) < total ? d.begin(w + 1) : total;
    if (pos >= total) continue;
    if (end <= pos || d.piece(pos) != w || d.piece(end - 1) != w) return 7;
    int b = 0;
    long long before = 0;
    while (!(pos >= before * U && pos < (before + steps[b]) * (long long)U)) before += steps[b++];
    int off = (int)(pos - before * U), u = off / steps[b], s = off % steps[b], left = (int)(end - pos);
    bool head = true;
    while (left > 0) {
      if (b >= n_seq || steps[b] <= 0) return 2;
      const int n = steps[b] - s < left ? steps[b] - s : left;
      for (int i = 0; i < n; ++i) seen[first[(long long)b * U + u] + s + i]++;
      if (n != steps[b]) {
        const int p = 2 * w + (head ? 0 : 1);
        if (place[p] >= 0) return 3;
        place[p] = b * U + u;
      }
      head = false; left -= n; s = 0;
      if (++u == U) { u = 0; do ++b; while (left > 0 && b < n_seq && steps[b] <= 0); }
    }
  }
  for (int x : seen) if (x != 1) return 4;
  int used = 0, listed = 0;
  for (int p : place) used += p >= 0;
  for (int b = 0; b < n_seq; ++b) for (int u = 0; u < U && steps[b] > 0; ++u) {
    const PagedWalk wk = paged_walk(first[(long long)b * U + u], steps[b], d);
    if (wk.w0 == wk.w1) continue;
    for (int w = wk.w0; w <= wk.w1; ++w, ++listed) if (w >= wgs || place[wk.place(w)] != b * U + u) return 5;
  }
  return used == listed ? 0 : 6;
}
extern "C" int far() {
  for (long long total : {(1ll << 32) - 1, (1ll << 32) + 77, (1ll << 36) - 3, (1ll << 36) - 511}) {
    const PagedDeal d = paged_deal(total);
    for (int w = 0; w < PAGED_WGS; ++w) {
      const long long a = d.begin(w), b = d.begin(w + 1);
      if (b <= a || d.piece(a) != w || d.piece(b - 1) != w || (w == PAGED_WGS - 1 && b != total)) return w + 1;
    }
  }
  return 0;
}
extern "C" int rows(int len, int n_new, int valid, int cap) { return paged_rows(len, valid == -99 ? n_new : paged_new(n_new, valid), cap); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged_plan")
    (d / "harness.cpp").write_text(HARNESS)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(d / "harness.cpp"), "-o", str(d / "harness.so")], check=True)
    return C.CDLL(str(d / "harness.so"))


def deal(plan, steps, U):
    return plan.deal((C.c_int * len(steps))(*steps), len(steps), U)


@pytest.mark.parametrize("steps,U", [
    ([1], 1), ([32], 32), ([4096], 8), ([0, 0, 5, 0], 4), ([1] * 1024, 1), ([0] * 1023 + [7], 3), ([100000], 1), ([3, 0, 4096, 1, 0], 8),
    ([129] * 64, 8), ([5, 6], 2), ([2047], 1), ([2048], 1), ([2049], 1), ([2559], 1), ([2560], 1), ([1] * 700, 40),
])
def test_every_step_is_walked_once_and_found_again(plan, steps, U):
    assert deal(plan, steps, U) == 0


def test_pieces_beyond_32_bits(plan):
    """The most steps that a call can have, every piece's first and last step."""
    assert plan.far() == 0


def test_random_lengths_are_dealt_out(plan):
    rng = random.Random(3)
    for _ in range(400):
        n = rng.choice([1, 2, 5, 33, 200])
        top = rng.choice([1, 9, 130, 2000 if n < 10 else 50])
        steps = [rng.choice([0, 1, top, rng.randint(0, top)]) for _ in range(n)]
        assert deal(plan, steps, rng.choice([1, 2, 7, 40])) == 0, steps


def test_no_steps_at_all(plan):
    assert deal(plan, [0, 0, 0], 4) == 0


@pytest.mark.parametrize("len_,n_new,valid,cap,expect", [
    (0, 0, -99, 32, 0), (31, 1, -99, 32, 32), (32, 1, -99, 32, -1), (32, 5, 0, 32, 32), (-1, 1, -99, 32, -1), (33, 0, -99, 32, -1),
    (2 ** 31 - 1, 2 ** 24, -99, 2 ** 24, -1), (2 ** 24, 2 ** 24, -99, 2 ** 24, -1), (-2 ** 31, 1, -99, 32, -1), (4, 3, 7, 32, 7), (4, 3, -5, 32, 4),
])
def test_rows_of_a_sequence(plan, len_, n_new, valid, cap, expect):
    assert plan.rows(len_, n_new, valid, cap) == expect


def fault(n_layers=1, cfg=None, null=False, **kw):
    f = B.lib()["_ZN4amph14paged_kv_faultERK11amph_configPK13amph_paged_kviPb"]
    f.restype, f.argtypes = C.c_char_p, [C.POINTER(B.amph_config), C.POINTER(B.amph_paged_kv), C.c_int, C.POINTER(C.c_bool)]
    base = dict(k_pages=4096, v_pages=8192, page_table=64, n_seq=2, n_kv_heads=2, page_rows=64, n_pages=9, table_pages=4, max_pages=4,
                page_stride=2 * 64 * 64, head_stride=64 * 64, layer_stride=9 * 2 * 64 * 64)
    base.update(kw)
    kv, shape, c = B.amph_paged_kv(*base.values()), C.c_bool(), cfg or base_cfg()
    text = f(C.byref(c), None if null else C.byref(kv), n_layers, C.byref(shape))
    return None if text is None else (text.decode(), shape.value)


def test_a_sound_cache_is_taken():
    assert fault() is None and fault(n_layers=0) is None and fault(max_pages=1, n_kv_heads=1, page_rows=32) is None
    assert fault(n_seq=128, table_pages=2 ** 18, max_pages=2 ** 18) is None and fault(n_layers=2 ** 20, n_seq=1, layer_stride=64) is None and fault(layer_stride=0) is None
    assert fault(page_stride=2 ** 42, layer_stride=2 ** 45, n_layers=2) is None
    assert fault(cfg=base_cfg(dtype=B.AMPH_BF16)) is None


@pytest.mark.parametrize("kw,shape", [
    (dict(k_pages=0), False), (dict(v_pages=None), False), (dict(page_table=0), False), (dict(k_pages=4104), False), (dict(page_table=66), False),
    (dict(n_seq=0), False), (dict(n_kv_heads=0), False), (dict(page_rows=0), False), (dict(n_pages=0), False), (dict(table_pages=0), False),
    (dict(max_pages=0), False), (dict(max_pages=-3), False), (dict(page_stride=-4), False), (dict(head_stride=6), False),
    (dict(layer_stride=2), False), (dict(n_layers=-1), False),
    (dict(n_seq=1025), True), (dict(n_kv_heads=3), True), (dict(page_rows=48), True), (dict(page_rows=16), True), (dict(max_pages=5), True),
    (dict(table_pages=2 ** 18 + 1), True), (dict(page_stride=2 ** 43), True), (dict(head_stride=2 ** 46), True), (dict(layer_stride=2 ** 45, n_layers=3), True), (dict(n_layers=2 ** 30), True),
    (dict(n_layers=2 ** 20 + 1, n_seq=1, layer_stride=64), True), (dict(n_seq=129, table_pages=2 ** 18, max_pages=2 ** 18), True),
    (dict(n_seq=1024, table_pages=2 ** 18, max_pages=2 ** 18, cfg=base_cfg(n_heads=128, d_model=8192)), True),
])
def test_an_unsound_cache_is_refused(kw, shape):
    got = fault(**kw)
    assert got is not None and got[1] == shape, got


def test_no_cache_is_refused():
    assert fault(null=True)[1] is False


def test_calls_without_a_context_are_refused():
    lib, n = B.lib(), C.c_size_t()
    kv = B.amph_paged_kv()
    assert lib.amph_paged_bytes(None, C.byref(kv), 0, C.byref(n)) == B.AMPH_EINVAL
    assert lib.amph_paged_append(None, C.byref(kv), 0, 1, None, None, None, None, 0, None, 0, None, 0, None, None, None) == B.AMPH_EINVAL
    assert lib.amph_paged_attn(None, C.byref(kv), 0, None, 0, 0, None, None, None, None, None, None) == B.AMPH_EINVAL
    assert lib.amph_paged_evict(None, C.byref(kv), 1, 1, 0, 0, None, None, None, None, None, None, None, None) == B.AMPH_EINVAL


def test_struct_is_the_header_s():
    assert C.sizeof(B.amph_paged_kv) == 3 * 8 + 6 * 4 + 3 * 8
    text = open(os.path.join(CSRC, "..", "..", "include", "amph.h")).read()
    body = re.sub(r"/\*.*?\*/", "", text[text.index("typedef struct amph_paged_kv {"):text.index("} amph_paged_kv;")], flags=re.S)
    at = [body.index(name) for name, _ in B.amph_paged_kv._fields_]
    assert at == sorted(at) and "AMPH_MAX_SEQ = %d" % B.AMPH_MAX_SEQ in text and "AMPH_DEV_BAD_PAGE = %d" % B.AMPH_DEV_BAD_PAGE in text


nan = float("nan")


@pytest.mark.parametrize("w,pos,budget,recent,expect", [
    ([5, 1, 4, 2, 3], [0, 1, 2, 3, 4], 5, 2, [0, 1, 2, 3, 4]),             # nothing to drop
    ([5, 1, 4, 2, 3], [0, 1, 2, 3, 4], 3, 0, [0, 4, 2]),                   # row 1 goes, row 4 moves in
    ([5, 1, 4, 2, 3], [0, 1, 2, 3, 4], 3, 1, [0, 4, 2]),                   # the newest is kept anyway
    ([5, 4, 3, 2, 0], [0, 1, 2, 3, 4], 3, 2, [0, 3, 4]),                   # the two newest, then the largest
    ([1, 1, 1, 1], [3, 2, 1, 0], 2, 0, [0, 1]),                            # ties: the lower rows
    ([1, 1, 1, 1], [0, 1, 2, 9], 2, 2, [0, 3]),                            # positions with gaps: one row is recent
    ([nan, 0, nan, -1], [0, 1, 2, 3], 2, 0, [3, 1]),                       # NaN last
    ([0, 0, 7], [0, 1, 2], 1, 1, [2]),
])
def test_reference_eviction_by_hand(w, pos, budget, recent, expect):
    assert pr.evict_rows(w, pos, len(w), budget, recent) == expect
