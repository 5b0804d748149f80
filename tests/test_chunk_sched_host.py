"""The deal of the chunk attention's work, compiled for the CPU and compared with loops over every item: units, cuts, the walk of
every CTA through its share, and who holds the parts of an item that is cut; up to the largest line of units that 31 bits count."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#define __host__
#define __device__
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include "chunk_sched.cuh"
using namespace earn;

#define CHECK(x) do { if (!(x)) { printf("line %d: %s (call %d)\n", __LINE__, #x, g_call); exit(1); } } while (0)
static int g_call = 0;
struct Item { int b, h, m, units, cost; uint32_t start; };

// The line of the call: every item with its units, in the order of the line (cols = 1: (sequence, head block, item)).
static std::vector<Item> line(const ChunkSched& s, const std::vector<int>& cu, const std::vector<int>& len, int cols) {
  std::vector<Item> own, out;
  for (int b = 0; b < s.n_seq; ++b) {
    const long n = cu[b + 1] - cu[b], base = std::min(std::max(len[b], 0), s.max_len) - n;
    for (int h = 0; h < s.heads; ++h)
      for (long m = 0; m * s.item_tok < n; ++m) {
        const long keys = std::max(0l, base + std::min((m + 1) * s.item_tok, n)), tile = 1l << s.key_shift;
        const int cost = n - m * s.item_tok <= s.free_tok ? 0 : s.item_cost;
        own.push_back({b, h, (int)m, (int)std::max(1l, (keys + tile - 1) / tile) + cost, cost, 0});
      }
  }
  for (int c = 0; c < cols; ++c)
    for (size_t i = c; i < own.size(); i += cols) out.push_back(own[i]);
  uint32_t at = 0;
  for (auto& x : out) { x.start = at; at += x.units; }
  return out;
}

static void check(ChunkSched s, const std::vector<int>& cu, const std::vector<int>& len, bool columns) {
  ++g_call;
  s.cu_new = cu.data(); s.seq_len = len.data(); s.table = nullptr;
  uint32_t total = 0, items = 0, lists = 0;
  std::vector<int> first(1, 0);
  for (int b = 0; b < s.n_seq; ++b) {
    const ChunkSeq q = chunk_seq(s, b);
    const uint32_t per_head = q.n > 0 ? chunk_units_before(s, q, q.items) : 0;
    total += s.heads * per_head;
    items += q.items;
    lists += q.n > 0;
    first.push_back((int)(items * s.heads));
    uint32_t sum = 0;   // every prefix of a short sequence's items
    if (q.items <= 300)
      for (int m = 0; m < q.items; ++m) { CHECK(chunk_units_before(s, q, m) == sum); sum += chunk_units(s, q, m); }
  }
  s.first = first.data();
  ChunkWalk w{};
  w.total = total;
  if (total == 0) return;
  chunk_cuts(s, w);
  w.cols = columns ? chunk_columns(items * s.heads, lists * s.heads, s.n_seq, w.shares, 640) : 1;
  const std::vector<Item> all = line(s, cu, len, w.cols);
  CHECK(total < 0x80000000u && all.back().start + all.back().units == total);
  // every CTA's cut, and where it lies
  std::vector<uint32_t> cut;
  std::vector<ChunkWalk> at;
  for (int c = 0; c <= w.shares; ++c) {
    const uint32_t x = chunk_cut(w, c);
    ChunkWalk v = w;
    if (x >= total) { v.b = s.n_seq; cut.push_back(total); at.push_back(v); continue; }
    const size_t k = std::upper_bound(all.begin(), all.end(), x, [](uint32_t y, const Item& i) { return y < i.start; }) - all.begin() - 1;
    ChunkSeq q;
    if (w.cols > 1) {
      size_t left = k;   // the column and the place in it
      for (v.col = 0; left >= ((size_t)first.back() - v.col + w.cols - 1) / w.cols; ++v.col) left -= ((size_t)first.back() - v.col + w.cols - 1) / w.cols;
      v.i = v.col + (int)left * w.cols;
      chunk_place(s, v, q);
      CHECK(v.b == all[k].b && v.h == all[k].h && v.m == all[k].m);
      v.off = (int)(x - all[k].start);
    } else {
      v.b = all[k].b; v.h = all[k].h;
      q = chunk_seq(s, v.b);
      const uint32_t per_head = chunk_units_before(s, q, q.items), head0 = all[k].start - chunk_units_before(s, q, all[k].m);
      CHECK(x - head0 < per_head);
      chunk_find(s, v, q, x - head0);
      CHECK(v.m == all[k].m && (uint32_t)v.off == x - all[k].start);
    }
    cut.push_back(chunk_settle(s, v, q, x));
    at.push_back(v);
  }
  CHECK(cut[0] == 0);
  // the walks: what every CTA holds of every item
  std::vector<std::vector<int>> holders(all.size());
  size_t k = 0;
  for (int c = 0; c < w.shares; ++c) {
    CHECK(cut[c] <= cut[c + 1]);
    ChunkWalk v = at[c];
    v.pos = cut[c]; v.end = cut[c + 1];
    ChunkSeq q{};
    if (v.pos < v.end) q = chunk_seq(s, v.b);
    while (v.pos < v.end) {
      CHECK(v.b == all[k].b && v.h == all[k].h && v.m == all[k].m && v.pos - v.off == all[k].start);
      const int units = chunk_units(s, q, v.m);
      CHECK(units == all[k].units && chunk_cost(s, q, v.m) == all[k].cost);
      const int stop = v.off + (int)std::min((uint32_t)(units - v.off), v.end - v.pos);
      CHECK(stop > all[k].cost);                        // a part has a key tile
      holders[k].push_back(c);
      v.pos += stop - v.off;
      if (stop == units) { chunk_next(s, v, q); ++k; }
      else v.off = stop;
    }
  }
  CHECK(k == all.size());
  std::vector<int> starts(w.shares, 0), ends(w.shares, 0);
  for (k = 0; k < all.size(); ++k) {
    const ChunkParts p = chunk_parts(w, all[k].start, all[k].units, all[k].cost);
    CHECK(p.parts == (int)holders[k].size());
    for (int i = 0; i < p.parts && p.parts > 1; ++i) CHECK(holders[k][i] == p.first + i);
    // a place in the scratch per CTA and side
    if (p.parts > 1) {
      CHECK(starts[p.first]++ == 0);
      for (int i = 1; i < p.parts; ++i) CHECK(ends[p.first + i]++ == 0);
    }
  }
}

int main(int argc, char** argv) {
  std::mt19937 r(atoi(argv[1]));
  auto pick = [&](int lo, int hi) { return lo + (int)(r() % (uint32_t)(hi - lo + 1)); };
  const int calls = atoi(argv[2]);
  for (int i = 0; i < calls; ++i) {
    ChunkSched s{};
    s.n_seq = pick(1, i % 3 == 0 ? 90 : 12);
    s.heads = pick(1, 8);
    const int tile_tok = pick(1, 128), kind = pick(0, 2);   // tensor cores, few rows, fp32
    s.item_tok = kind == 0 ? 2 * tile_tok : tile_tok;
    s.key_shift = kind == 2 ? 6 : 7;
    s.item_cost = kind == 0 ? 2 : 0; s.free_tok = kind == 0 ? tile_tok : 0;
    s.min_share = kind == 0 ? 2 : 1;
    s.grid = pick(1, kind == 2 ? 296 : 148);
    s.max_len = pick(1, 1 << pick(4, 15));
    const int longest = pick(1, 1 << pick(0, 11));
    std::vector<int> cu(1, 0), len;
    for (int b = 0; b < s.n_seq; ++b) {
      cu.push_back(cu.back() + (pick(0, 4) == 0 ? 0 : pick(0, longest)));
      len.push_back(pick(0, 5) == 0 ? pick(-3, longest) : cu.back() - cu[b] + pick(0, s.max_len));
    }
    s.n_tokens = cu.back() + pick(0, 5);
    check(s, cu, len, false);
    check(s, cu, len, true);
  }
  // long lines: one list of two million rows, or several, with so many new tokens that the line is just short of 2^31 units
  for (int tile_tok : {128, 32, 8, 1})
    for (int n_seq : {1, 7})
      for (int grid : {148, 3, 1}) {
        ChunkSched s{};
        s.n_seq = n_seq; s.heads = 8;
        s.item_tok = 2 * tile_tok; s.free_tok = tile_tok; s.item_cost = 2; s.key_shift = 7; s.min_share = 2; s.grid = grid;
        s.max_len = 1 << 21;
        const long items = (long)(0x7fffffff / 8) / ((1 << 14) + 2) / n_seq;
        std::vector<int> cu(1, 0), len;
        for (int b = 0; b < n_seq; ++b) { cu.push_back(cu.back() + (int)(items * s.item_tok) - b); len.push_back(s.max_len); }
        s.n_tokens = cu.back();
        check(s, cu, len, false);
        check(s, cu, len, true);
      }
  printf("%d calls\n", g_call);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    folder = tmp_path_factory.mktemp("sched")
    (folder / "sched.cpp").write_text(SOURCE)
    csrc = os.path.join(ROOT, "paper_2507_00715_b200", "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", csrc, "-o", str(folder / "sched"),
                    str(folder / "sched.cpp")], check=True)
    return str(folder / "sched")


@pytest.mark.parametrize("seed", range(4))
def test_every_share_against_loops(program, seed):
    r = subprocess.run([program, str(seed), "1500"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
