"""Launches of the cache's operators, on the CPU: a small host program against the library's own helpers."""
import ctypes as C
import itertools
import os
import subprocess

import pytest

from paper_2512_17917_amd import binding as kvr
from paper_2512_17917_amd import build as B

PROBE = r"""
#include <cstdio>
#include "kvr_prompt.h"
// g n -> workgroups a row, rows | p B heads G rows keys -> the scores' pass: workgroups, those that add, most parts, 1 if more pieces may
// follow, bytes of workspace, of those before the parts' sums | s blocks longest units most wgs -> parts | t window n_sink lo hi end ->
// tiles of 256 tokens that start before `end`, all
int main() {
  char kind;
  while (std::scanf(" %c", &kind) == 1) {
    long long n;
    if (kind == 'g') {
      if (std::scanf("%lld", &n) != 1) return 1;
      const kvr::GridRows r = kvr::grid_rows(n);
      std::printf("%u %u\n", r.x, r.rows);
    } else if (kind == 'p') {
      kvr::DevDesc d = {};
      long long rows, keys;
      if (std::scanf("%d %d %d %lld %lld", &d.B, &d.Hkv, &d.G, &rows, &keys) != 5) return 1;
      d.Hq = d.Hkv * d.G;
      const kvr::ScoresPlan p = kvr::prompt_scores_plan(d, rows, keys);
      std::printf("%d %d %d %d %zu %zu\n", p.wgs, p.add_wgs, p.most_splits, (int)p.walk, p.bytes, p.off_part);
    } else if (kind == 's') {
      int x[5];
      for (int& y : x)
        if (std::scanf("%d", &y) != 1) return 1;
      std::printf("%d\n", kvr::scores_splits(x[0], x[1], x[2], x[3], x[4]));
    } else if (kind == 't') {
      kvr::Visible v;
      int lo, hi, end;
      if (std::scanf("%d %d %d %d %d", &v.window, &v.n_sink, &lo, &hi, &end) != 5) return 1;
      const kvr::TileRange r = kvr::tile_range<256>(v, lo, hi);
      std::printf("%d ", kvr::tiles_before<256>(r, end));
      for (int i = 0; i < r.n; ++i) std::printf("%d ", kvr::tile_token<256>(r, i));
      std::printf("\n");
    }
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("launch")
    src, exe = str(d / "probe.hip"), str(d / "probe")
    open(src, "w").write(PROBE)
    subprocess.run([B._hipcc(), "--offload-host-only", "-std=c++17", "-I", B.CSRC, src, "-L", os.path.dirname(B.OUT),
                    "-l:" + os.path.basename(B.OUT), f"-Wl,-rpath,{os.path.dirname(B.OUT)}", "-o", exe], check=True, capture_output=True)

    def run(lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, x.split())) for x in out.splitlines()]
    return run


def test_no_dimension_of_a_launch_wraps(ask):
    """Every workgroup is there, in dimensions that hold them with 512 threads each."""
    cases = [1, 2, 255, 1 << 22, (1 << 22) + 1, 1 << 24, (1 << 24) + 3, (1 << 27) + 65535, 1 << 31]
    for n, (x, rows) in zip(cases, ask([f"g {n}" for n in cases])):
        assert x * 512 < 1 << 32 and rows <= 65535 and n <= x * rows < n + (1 << 22)
        assert rows == 1 or n > 1 << 22


SIZES = [(b, h, g, rows, keys) for b, h, g in ((1, 8, 4), (1, 1, 1), (2, 8, 4), (64, 8, 4), (512, 8, 1), (8000, 8, 8)) for rows in (1, 16, 200, 5000, 1 << 24)
         for keys in (1, 256, 300, 2048, 32768, 131072, 1 << 20, 1 << 30) if b * h * keys <= 1 << 37]


def test_scores_pass_is_as_large_as_its_work(ask):
    """Launches and workspace within bounds, whatever there is room for; room for the sums of every cut that the device may choose."""
    for (b, h, g, rows, keys), (wgs, add, most, walk, size, off) in zip(SIZES, ask([f"p {b} {h} {g} {rows} {keys}" for b, h, g, rows, keys in SIZES])):
        blocks = b * h * -(-keys // 256)
        assert 1 <= wgs <= 16384 and walk == (blocks > 16384) and most == min(64, max(1, -(-rows * g // 128)))
        assert add == (min(blocks, 767) if most > 1 else 0) and off >= 12 + 4 * b and off % 256 == 0 and size - off <= 1535 * 1024
        counts = sorted({x for x in (1, 2, 3, 7, 8, 12, 50, 255, 256, 383, 384, 400, 766, 767, 768, 5000) if x <= blocks} | {min(blocks, 767)})
        for n, (s,) in zip(counts, ask([f"s {n} 1 1 {most} {wgs}" for n in counts])):
            assert 1 <= s <= most and (s == 1 or (n <= add and n * s * 1024 <= size - off))


def test_parts_go_by_the_tokens_that_there_are(ask):
    """About 768 pieces, none beyond the launch; the same for a cache with room for more."""
    def parts(blocks, longest, units, rows, g, b, h, keys):
        (wgs, _, most, _, _, _), = ask([f"p {b} {h} {g} {rows} {keys}"])
        return ask([f"s {blocks} {longest} {units} {most} {wgs}"])[0][0]
    for keys in (2048, 32768, 131072):
        assert parts(64, 8, 8, 2048, 4, 1, 8, keys) == 12             # 2k tokens, 32 heads on 8
        assert parts(256, 8, 32, 8192, 4, 4, 8, keys) == 3            # 4 x 2k
        assert parts(8, 1, 8, 200, 4, 1, 8, keys) == 7                # 200 tokens: two tiles of columns a part
    for blocks, longest, units, most, wgs, want in ((0, 0, 8, 64, 800, 1), (768, 96, 8, 64, 2000, 1), (767, 96, 8, 64, 2000, 2), (10, 5, 128, 64, 640, 1),
                                                    (10, 5, 128, 64, 1280, 2), (10, 5, 128, 64, 16384, 25), (1, 1, 8000, 64, 16384, 2), (5, 5, 8000, 9, 16384, 1)):
        assert ask([f"s {blocks} {longest} {units} {most} {wgs}"])[0][0] == want


def test_workspace_of_a_prompt_does_not_grow_with_room_for_scores():
    """2048 rows of 32 heads on 8: the same workspace for caches of 2k and of 1M tokens."""
    d, n = kvr.make_desc(1, 32, 8, 1, 1, kvr.KVR_BF16), C.c_size_t(0)
    sizes = []
    for cap in (2048, 32768, 1 << 20):
        p = kvr.kvr_pages(None, None, 0x10000, 10, 64, cap // 64)
        both = []
        for scores in (0, 1):
            assert kvr.lib().kvr_attend_prompt_workspace_size(C.byref(d), 2048, C.byref(p), 0, 0, scores, C.byref(n)) == kvr.KVR_OK
            both.append(n.value)
        sizes.append(both[1] - both[0])
    assert sizes[1] == sizes[2] and sizes[0] <= sizes[1] <= 2 << 20


def test_tiles_that_start_before_a_token(ask):
    cases = [(w, s, lo, lo + more, end) for w, s, lo, more, end in itertools.product(
        (0, 1, 300, 1000), (0, 1, 256, 700, 5000), (-3, 0, 255, 1500, 4000), (0, 255, 900), (1, 256, 257, 1400, 2000, 9000))]
    for case, (n, *tiles) in zip(cases, ask([("t " + " ".join(map(str, c))) for c in cases])):
        assert n == sum(t < case[4] for t in tiles), case


def test_more_rows_and_heads_than_attention_is_launched_for_are_refused():
    """2^30 rows times heads: 256 GiB of queries in bf16, twice that with the outputs."""
    d, n = kvr.make_desc(1, 12, 3, 1, 1, kvr.KVR_BF16), C.c_size_t(0)
    p = kvr.kvr_pages(0x10000, 0x10000, 0x10000, 10, 64, 100)
    P = 0x10000
    for rows, want, call in (((1 << 30) // 12, kvr.KVR_OK, kvr.KVR_ERR_WORKSPACE_TOO_SMALL), ((1 << 30) // 12 + 1, kvr.KVR_ERR_INVALID_ARG, kvr.KVR_ERR_INVALID_ARG),
                             (1 << 27, kvr.KVR_ERR_INVALID_ARG, kvr.KVR_ERR_INVALID_ARG)):
        assert kvr.lib().kvr_attend_prompt_workspace_size(C.byref(d), rows, C.byref(p), 0, 0, 1, C.byref(n)) == want
        assert kvr.lib().kvr_attend_prompt(C.byref(d), P, rows, P, P, C.byref(p), 0, 0, P + 16, P, 64, P, 0, None) == call
