"""How the attention of a few rows of each sequence is shared out over workgroups (rows_units.h), walked on the host: every
step of every unit is taken once, partial sums lie where the merge looks for them, and no walk leaves its sequences;
with sequences without rows or context, ranges and lengths that are inconsistent, and contexts that are cut short."""

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_09590_amd", "csrc")

PROGRAM = r"""
#include "rows_units.h"

#include <cstdio>
#include <map>
#include <tuple>
#include <vector>

using namespace bros;
using namespace bros::ra;

#define wrong(msg, ...) (snprintf(msg, 256, __VA_ARGS__), 1)

// Takes the shares of every workgroup one after another, as the kernels do. 0: all is as it has to be.
template <class P, int CT, int KS, int THREADS, int TEAM>
int walk(const RowsArgs& a, int group, char* msg) {
  const int S = a.num_seqs, H = a.num_kv_heads;
  // From the definition: the rows of each sequence, its units, and the keys that each unit's rows may see.
  struct Rows {
    int n;
    int64_t c0, ctx, row0;
  };
  std::vector<Rows> seqs(S);
  int64_t dense = 0;
  for (int s = 0; s < S; ++s) {
    const int64_t lo = a.cu_q[s], hi = a.cu_q[s + 1], ctx = a.ctx_lens[s];
    Rows& r = seqs[s];
    r.n = lo < 0 || hi > a.num_q_tokens || hi < lo ? 0 : (int)(hi - lo);
    r.c0 = ctx - r.n;
    r.ctx = r.c0 < 0 ? 0 : std::min<int64_t>(std::min<int64_t>(ctx, a.max_ctx), (int64_t)a.max_blocks_per_seq * 16);
    r.row0 = dense;
    dense += (r.ctx + 31) / 32 * 32;
  }
  struct Unit {
    std::vector<int> taken;                     // of each step
    std::map<int, std::pair<int, int>> parts;   // steps [first, last) by the partial's slot
    int noted = -1, last = -1;                  // the workgroup that noted it for the merge, and the last share's
  };
  std::map<std::tuple<int, int, int>, Unit> units;
  const int groups = a.workers * TEAM;
  std::vector<int> used(2 * groups, 0);
  for (int me = 0; me < groups; ++me) {
    const int team = me / TEAM, member = me % TEAM;
    int64_t total = 0;
    std::vector<int64_t> steps(THREADS), rows(THREADS);
    for (int i = 0; i < THREADS; ++i) {
      count_run<P, CT * TEAM, KS>(a, group, Run(S, THREADS, i), steps[i], rows[i]);
      if (steps[i] < 0) return wrong(msg, "thread %d counts %lld steps", i, (long long)steps[i]);
      total += steps[i];
    }
    const Shares shares(a, total);
    const int64_t wanted = team < shares.n ? shares.begin(team) : -1;
    Place at{-1, 0, 0, 0, total, 0};
    int64_t first = 0, row = 0;
    for (int i = 0; i < THREADS; ++i) {
      if (wanted >= first && wanted < first + steps[i])
        place_in_run<P, CT * TEAM, KS>(a, group, Run(S, THREADS, i), wanted - first, row, total, &at);
      first += steps[i];
      row += rows[i];
    }
    if (at.s < 0) {
      if (wanted >= 0 && wanted < total) return wrong(msg, "share %d has steps and no place", team);
      continue;
    }
    int64_t x = wanted;
    const int64_t x_end = shares.begin(team + 1);
    while (x < x_end) {
      if (at.s < 0 || at.s >= S) return wrong(msg, "share %d walks to sequence %d of %d", team, at.s, S);
      const Rows& r = seqs[at.s];
      const int64_t tiles = ((int64_t)r.n * group + CT * TEAM - 1) / (CT * TEAM);
      if (r.n == 0 || at.g >= H || at.t >= tiles || at.step < 0)
        return wrong(msg, "share %d at sequence %d head %d unit %d step %d, of %d rows", team, at.s, at.g, at.t, at.step, r.n);
      if (!P::kPaged && at.row0 != r.row0) return wrong(msg, "share %d: dense row %lld of sequence %d", team, (long long)at.row0, at.s);
      const Segment<P, CT, KS, TEAM> seg(a, at, group, member, x, x_end);
      if (seg.next <= x) return wrong(msg, "share %d stands still", team);
      if (seg.count > 0) {
        if ((int64_t)seg.t * CT >= (int64_t)r.n * group) return wrong(msg, "share %d: unit %d of %d columns", team, seg.t, r.n * group);
        Unit& u = units[{at.s, at.g, seg.t}];
        if (u.taken.empty()) u.taken.resize(seg.steps, 0);
        if ((int)u.taken.size() != seg.steps || seg.first < 0 || seg.last > seg.steps) return wrong(msg, "share %d: steps %d to %d", team, seg.first, seg.last);
        for (int i = seg.first; i < seg.last; ++i) ++u.taken[i];
        if (seg.whole != (seg.first == 0 && seg.last == seg.steps)) return wrong(msg, "share %d: whole", team);
        if (!seg.whole) {
          const int slot = 2 * me + (seg.first == 0 ? 1 : 0);
          if (used[slot]++) return wrong(msg, "slot %d written twice", slot);
          u.parts[slot] = {seg.first, seg.last};
          if (seg.first == 0) {
            u.noted = me;
            u.last = seg.last_share(shares) * TEAM + member;
          }
        }
      }
      x = seg.next;
      at.step = 0;
      if (x < x_end) next_unit<P>(a, at, seg.tiles);
    }
    if (x != x_end) return wrong(msg, "share %d ends at %lld, not %lld", team, (long long)x, (long long)x_end);
  }
  // Every unit, and every step of it, once.
  size_t n_units = 0;
  for (int s = 0; s < S; ++s) {
    const Rows& r = seqs[s];
    const int64_t columns = (int64_t)r.n * group;
    for (int g = 0; g < H; ++g) {
      for (int64_t t = 0; t * CT < columns; ++t) {
        ++n_units;
        const auto it = units.find({s, g, (int)t});
        if (it == units.end()) return wrong(msg, "unit %d of sequence %d head %d: taken by nobody", (int)t, s, g);
        const Unit& u = it->second;
        for (size_t i = 0; i < u.taken.size(); ++i)
          if (u.taken[i] != 1) return wrong(msg, "step %d of unit %d of sequence %d: taken %d times", (int)i, (int)t, s, u.taken[i]);
        const int64_t keys = P::kCausalUnits ? std::min<int64_t>(r.ctx, r.c0 + std::min<int64_t>(r.n, (t + 1) * CT)) : r.ctx;
        if ((int64_t)u.taken.size() * KS < keys) return wrong(msg, "unit %d of sequence %d: too few steps", (int)t, s);
        if ((int64_t)u.taken.size() > std::max<int64_t>(1, (r.ctx + KS - 1) / KS)) return wrong(msg, "unit %d of sequence %d: too many steps", (int)t, s);
        if (u.parts.empty()) continue;
        // the merge's pieces, in the order of their keys
        if (u.noted < 0 || u.noted >= std::max(1, groups - 1)) return wrong(msg, "cut unit without a note: %d", u.noted);
        int at = 0;
        size_t pieces = 0;
        for (int w = u.noted; w <= u.last; w += TEAM, ++pieces) {
          const auto p = u.parts.find(2 * w + (w == u.noted ? 1 : 0));
          if (p == u.parts.end() || p->second.first != at) return wrong(msg, "piece of share %d is missing", w / TEAM);
          at = p->second.second;
        }
        if (at != (int)u.taken.size() || pieces != u.parts.size()) return wrong(msg, "pieces do not make the unit");
      }
    }
  }
  if (n_units != units.size()) return wrong(msg, "units that are none");
  return 0;
}

extern "C" int walk_batch(int shape, int group, int heads, int seqs, const int* cu_q, const int* ctx_lens, int tokens, int width, int max_ctx, int workers,
                          int min_steps, int whole, int start, char* msg) {
  RowsArgs a{};
  a.cu_q = cu_q;
  a.ctx_lens = ctx_lens;
  a.num_q_tokens = tokens;
  a.num_seqs = seqs;
  a.max_blocks_per_seq = width;
  a.max_ctx = max_ctx;
  a.num_kv_heads = heads;
  a.workers = workers;
  a.min_steps = min_steps;
  a.whole_units = whole;
  a.start_steps = start;
  switch (shape) {
    case 0: return walk<KvPool, 32, 64, 128, 1>(a, group, msg);
    case 1: return walk<KvPool, 64, 64, 256, 1>(a, group, msg);
    case 2: return walk<KvPool, 128, 32, 256, 1>(a, group, msg);
    case 3: return walk<KvPool, 128, 32, 256, 2>(a, group, msg);
    case 4: return walk<KvPool, 128, 32, 256, 4>(a, group, msg);
    case 5: return walk<LatentPool, 16, 32, 256, 1>(a, group, msg);
    case 6: return walk<LatentPool, 32, 32, 256, 1>(a, group, msg);
    case 7: return walk<LatentPool, 64, 32, 256, 1>(a, group, msg);
    case 8: return walk<LatentPool, 128, 32, 512, 1>(a, group, msg);
    case 9: return walk<Expanded, 64, 64, 256, 1>(a, 1, msg);
    case 10: return walk<Expanded, 128, 32, 256, 1>(a, 1, msg);
    case 11: return walk<Expanded, 128, 32, 256, 2>(a, 1, msg);
    default: return walk<Expanded, 128, 32, 256, 4>(a, 1, msg);
  }
}
"""
SHAPES = 13


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("units")
    (d / "units.cpp").write_text(PROGRAM)
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-ftrapv", "-shared", "-fPIC", "-I", CSRC, str(d / "units.cpp"),
                    "-o", str(d / "units.so")], check=True)
    lib = ctypes.CDLL(str(d / "units.so"))

    def call(shape, ranges, ctx, tokens, width, max_ctx, group=1, heads=1, workers=512, min_steps=4, whole=0, start=4):
        """ranges: the offsets [S + 1]. What lies behind the arrays would be a sequence with rows."""
        cu = np.concatenate([ranges, [tokens]]).astype(np.int32)
        lens = np.concatenate([ctx, [77]]).astype(np.int32)
        msg = ctypes.create_string_buffer(256)
        P = lambda x: x.ctypes.data_as(ctypes.POINTER(ctypes.c_int))  # noqa: E731
        off = lib.walk_batch(shape, group, heads, len(ctx), P(cu), P(lens), tokens, width, max_ctx, workers, min_steps, whole, start, msg)
        assert off == 0, f"{msg.value.decode()} (shape {shape}, offsets {ranges}, lengths {ctx}, bound {max_ctx}, {workers} shares)"
    return call


def offsets(n):
    return np.concatenate([[0], np.cumsum(n)])


@pytest.mark.parametrize("shape", range(SHAPES))
@pytest.mark.parametrize("n,ctx", [([0, 1400, 601], [0, 4400, 6601]), ([1400, 0, 601], [4400, 0, 6601]), ([1400, 601, 0, 0], [4400, 6601, 0, 0]),
                                   ([0, 0, 1400], [9000, 5, 4400]), ([300, 0], [300, 2]), ([0], [0]), ([0, 0], [0, 40])])
def test_sequences_without_rows(walk, shape, n, ctx):
    """Before, between and behind the others, as in a batch padded to a fixed number; with and without context."""
    for workers in (256 // (1, 2, 4)[shape % 3], 7, 1):
        for start in (0, 4, 8):
            walk(shape, offsets(n), ctx, sum(n), 600, 6601, heads=2, workers=workers, start=start)
    walk(shape, offsets(n), ctx, sum(n), 600, 6601, heads=3, workers=60, min_steps=1, whole=1)


@pytest.mark.parametrize("shape", range(SHAPES))
def test_ranges_and_lengths_that_are_inconsistent(walk, shape):
    """Ranges outside the rows (a sequence of no rows), lengths below the rows there are or below zero, or near the ends of
    32 bits, and contexts above the bound and above what a row of the table holds."""
    for ctx in ([300, 50, 900], [-5, 50, 0], [2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 20], [-2 ** 31, -2 ** 31, 900], [5000, 4000, 3000]):
        for ranges in ([0, 100, 150, 400], [-3, 100, 150, 400], [0, 400, 150, 380], [0, 100, 401, 400], [0, 0, 2 ** 31 - 1, 400], [400, 400, 400, 400]):
            for max_ctx in (0, 700, 2 ** 31 - 1):
                walk(shape, np.array(ranges), ctx, 400, 100, max_ctx, heads=2, workers=33)


@pytest.mark.parametrize("shape", range(SHAPES))
def test_random_batches(walk, shape):
    rng = np.random.default_rng(shape)
    for _ in range(150):
        S = int(rng.integers(1, 40))
        n = np.where(rng.random(S) < 0.3, 0, (2 ** rng.uniform(0, 10, S)).astype(int))
        c0 = np.where(rng.random(S) < 0.3, 0, (2 ** rng.uniform(0, 13, S)).astype(int))
        ctx = n + c0 - np.where(rng.random(S) < 0.1, rng.integers(0, 50, S), 0)
        ranges = offsets(n)
        tokens = int(ranges[-1]) - (int(rng.integers(0, 9)) if rng.random() < 0.2 else 0)   # (the last range may lie outside)
        max_ctx = int(max(1, ctx.max())) if rng.random() < 0.6 else int(rng.integers(0, 4000))
        whole = int(rng.random() < 0.2)
        walk(shape, ranges, ctx, max(tokens, 0), int(rng.integers(1, 600)), max_ctx, group=int(rng.choice([1, 2, 4, 8])), heads=int(rng.integers(1, 5)),
             workers=int(rng.choice([1, 5, 64, 128, 256, 512])), min_steps=1 if whole else int(rng.choice([1, 4, 6])), whole=whole,
             start=int(rng.choice([0, 4, 6, 8])))
