"""Host paths of the page calls and of the beam selection without a GPU: the plans of forks are compiled on their own, those of
compactions read from what the library copies to the device (a stand-in for the HIP runtime, fake_hip.cpp), and both are carried out
here; and every refusal."""
import ctypes as C
import os
import subprocess
import sys
from types import SimpleNamespace

import numpy as np
import pytest

from test_host_runtime_paths import MODEL, ROOT, Child, fake  # noqa: F401  (the fixture builds the stand-in)

INVALID, RANGE, BATCH, CONFLICT, MEMORY, HIP = -1, -2, -3, -4, -5, -6


def up(n):
    return (n + 15) // 16 * 16


def i32(a):
    return np.ascontiguousarray(a, dtype=np.int32)


def at(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def last_image(c, ctx):
    ctx.synchronize()
    return c.copies()[-1]


PLAN = r"""
#include <map>

#include "page_plans.h"
// src, dst [n]; pages [p]: carries the plan out, the runs of a launch one after the other from the last to the first; what a launch
// holds at most; returns launches, or -1 where one holds more moves than it may
extern "C" int carry_out(const int32_t* src, const int32_t* dst, int n, int32_t* pages, int32_t* counts) {
  const ForkPlan plan(src, dst, n);
  counts[0] = (int)plan.moves.size();
  counts[1] = (int)plan.runs.size();
  for (const ForkPlan::Launch& l : plan.launches) {
    if (l.n_moves > FORK_MOVES || l.n_moves < 1) return -1;
    int next = 0;
    for (int r = 0; r < l.n_runs; ++r) {
      const PageRun& run = plan.runs[l.run0 + r];
      if (run.first != next || run.n < 1) return -1;
      next += run.n;
    }
    if (next != l.n_moves) return -1;
    std::map<int32_t, int> writer;  // runs of a launch may go at the same time: what one writes no other touches
    for (int r = 0; r < l.n_runs; ++r)
      for (int i = 0; i < plan.runs[l.run0 + r].n; ++i) writer[plan.moves[l.move0 + plan.runs[l.run0 + r].first + i].dst] = r;
    for (int r = 0; r < l.n_runs; ++r) {
      const PageRun& run = plan.runs[l.run0 + r];
      if (run.keep >= 0 && writer.count(run.keep) && writer[run.keep] != r) return -2;
      for (int i = 0; i < run.n; ++i) {
        const PageMove m = plan.moves[l.move0 + run.first + i];
        if (writer[m.dst] != r || (m.src >= 0 && writer.count(m.src) && writer[m.src] != r)) return -2;
      }
    }
    for (int r = l.n_runs; r-- > 0;) {
      const PageRun& run = plan.runs[l.run0 + r];
      const int32_t kept = run.keep >= 0 ? pages[run.keep] : -1;
      for (int i = run.first; i < run.first + run.n; ++i) {
        const PageMove m = plan.moves[l.move0 + i];
        pages[m.dst] = m.src < 0 ? kept : pages[m.src];
      }
    }
  }
  return (int)plan.launches.size();
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    where = tmp_path_factory.mktemp("plan")
    src, so = where / "plan.cpp", str(where / "plan.so")
    src.write_text(PLAN)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-Wall", "-Werror", "-D_GLIBCXX_ASSERTIONS", "-I", os.path.join(ROOT, "paper_2510_24051_amd", "csrc"),
                    "-o", so, str(src)], check=True)
    return C.CDLL(so)


@pytest.mark.parametrize("form", ["random", "permutation", "rotation", "two cycles", "chain", "fan", "wide fans on a cycle", "beams", "pairs", "one", "swap", "none"])
def test_fork_plans(form, plans):
    """Carried out in order, whichever run of a launch goes first, a plan gives every page what its source was; no move more than pages
    change but one for a cycle and one for each launch that it runs into."""
    rng = np.random.default_rng(5)
    every = np.arange(2000)
    for trial in range(40):
        n = int(rng.integers(1, 900))
        dst = rng.permutation(2000)[:n]
        others = np.setdiff1d(every, dst)
        if form == "random":
            src = rng.integers(0, 2000, n)
        elif form == "permutation":
            src = rng.permutation(dst)
        elif form == "rotation":
            src = np.roll(dst, 1)
        elif form == "two cycles":
            src = np.concatenate([np.roll(dst[:n // 2], 1), np.roll(dst[n // 2:], -1)])
        elif form == "chain":
            src = np.concatenate([others[:1], dst[:-1]])
        elif form == "fan":
            src = rng.choice(others, 3)[rng.integers(0, 3, n)]
        elif form == "wide fans on a cycle":
            k = max(2, n // 8)  # a cycle of k pages, every other destination a copy of one of them or of a copy
            k = min(k, n)
            src = np.concatenate([np.roll(dst[:k], 1), dst[rng.integers(0, np.arange(k, n))]]) if n > k else np.roll(dst[:k], 1)
        elif form == "beams":
            src = dst[np.arange(n) // 8 * 8 + np.minimum(rng.integers(0, 8, n), n - 1 - np.arange(n) // 8 * 8)]
        elif form == "pairs":
            src = others[:n]
            dst = dst[:len(src)]
        elif form == "one":
            src, dst = others[:1], dst[:1]
        elif form == "swap":
            dst = np.array([3, 9])
            src = dst[::-1]
        else:
            src = dst
        src, dst = i32(src), i32(dst)
        want, got, counts = every.copy(), i32(every).copy(), np.zeros(2, np.int32)
        want[dst] = every[src]
        launches = plans.carry_out(at(src), at(dst), len(src), at(got), at(counts))
        assert launches >= 0 and np.array_equal(got, want), (form, n)
        moving = int((src != dst).sum())
        # each cycle saves one load and needs no move more; what it puts down at the end of a launch is one
        assert moving <= counts[0] <= moving + launches and launches <= moving // 159 + 1, (form, n, counts, launches)


def fork_masks(c):
    """Masks go with the pages, as they were before the call; also where nothing is copied to the device."""
    for page_size in (16, 32):
        m = SimpleNamespace(**{**vars(MODEL), "page_size": page_size})
        ctx = c.context(n_pages=64, m=m)
        ctx.mask_kvpage([0, 1, 2], [0x1, 0x3, 0x7])
        ctx.fork_kvpage([0, 1, 2, 2], [1, 2, 0, 9])  # a cycle and a copy
        # page 1 now has one visible token, 2 two, 0 and 9 three: a decode request over each sees one page of them
        lens = {0: 3, 1: 1, 2: 2, 9: 3, 5: page_size}
        for p, n in lens.items():
            out = np.zeros(1, np.int32)
            assert ctx.compact_kvpage([0, 1], [p], [page_size], dst_page_indptr=[0, 1], dst_page_ids=[40])[0] == n
        ctx.close()


def compact_plans(c):
    """Ragged sequences, both page sizes, in place and apart, with shifts: the chains, carried out in any order, leave what a
    simultaneous move leaves, and tiles of a chain that has to go in order never read what an earlier one wrote."""
    rng = np.random.default_rng(8)
    checked = scratched = 0
    c.fake.fake_watch(b"compact_kernel", 5)  # waves of a layer: chains x kv heads x 2 (head_dim 64)
    for trial in range(40):
        P = int(rng.choice([16, 32]))
        F = P // 16
        m = SimpleNamespace(**{**vars(MODEL), "page_size": P})
        ctx = c.context(n_pages=1600, m=m)
        S = int(rng.integers(1, 5))
        lens = rng.integers(0, 250 * P // F, S)
        lens[rng.integers(0, S)] = rng.choice([0, 1, 15, 16, 17, P, 6 * P])
        n_pages = -(-lens // P) + rng.integers(0, 2, S)
        ids = rng.permutation(1600)
        ip = np.concatenate([[0], np.cumsum(n_pages)])
        table = ids[:ip[-1]]
        bits = rng.integers(0, 1 << 32, len(table), dtype=np.uint64) & (rng.integers(0, 1 << 32, len(table), dtype=np.uint64) | np.uint64(0xFF))
        bits[rng.random(len(table)) < 0.3] = 0xFFFFFFFF
        bits[rng.random(len(table)) < 0.2] = 0
        if len(table):
            ctx.mask_kvpage(table, bits)
        visible = [np.array([(int(bits[ip[s] + j // P]) >> (j % P)) & 1 for j in range(lens[s])], bool) for s in range(S)]
        shifts = np.concatenate([np.where(rng.random(n) < 0.5, 0, rng.integers(-3, 4, n)) for n in lens] or [[]]) if trial % 3 else None
        apart = trial % 2 == 0
        kept = [int(v.sum()) for v in visible]
        dp = np.concatenate([[0], np.cumsum([-(-k // P) for k in kept])]) if apart else None
        di = ids[ip[-1]:ip[-1] + dp[-1]] if apart else None
        n0 = len(c.copies())
        if trial % 4 == 1:  # no room for scratch blocks: the same in order
            c.fake.fake_malloc_limit(1 << 19)
        c.launches()
        got = ctx.compact_kvpage(ip, table, lens, shifts=shifts, dst_page_indptr=dp, dst_page_ids=di)
        c.fake.fake_malloc_limit(1 << 62)
        assert got.tolist() == kept
        pool = np.arange(1600 * P).astype(object)
        want = pool.copy()
        off = 0
        for s in range(S):
            into = di[dp[s]:dp[s + 1]] if apart else table[ip[s]:ip[s + 1]]
            for i, j in enumerate(np.nonzero(visible[s])[0]):
                by = 0 if shifts is None else int(shifts[off + j])
                token = int(table[ip[s] + j // P]) * P + j % P
                want[int(into[i // P]) * P + i % P] = (token, by) if by else token
            off += lens[s]
        ctx.synchronize()
        if len(c.copies()) == n0:  # nothing moves, or the plan is small and travels as kernel arguments
            ctx.close()
            continue
        checked += 1
        phases = [int(x.split()[1]) // (2 * m.n_kv_heads) for x in c.launches() if "compact_kernel" in x]
        # into destinations at once; or into scratch blocks, and from there; or both
        n_direct, n_in, n_back = {1: phases + [0, 0], 2: [0] + phases, 3: phases}[len(phases)]
        assert trial % 4 != 1 or n_in == 0
        scratched += n_in > 0
        image = c.copies()[-1]
        # chains (entries from, to; first destination block), entries (block, mask, first kept token, row of the table or -1, -2),
        # destination blocks, then, where a block's keys turn differently, rows of the table, and the shifts, each at a multiple of 16
        ints = np.frombuffer(image, np.int32)
        k = n_entries = 0
        while 3 * k < len(ints) and ints[3 * k] == n_entries and ints[3 * k + 1] > n_entries:
            n_entries, k = int(ints[3 * k + 1]), k + 1
        chains = ints[:3 * k].reshape(-1, 3)
        o = up(12 * k) // 4
        entries = ints[o:o + 4 * n_entries].reshape(-1, 4)
        o += 4 * n_entries
        tiles = ints[o:]
        turning = any(isinstance(x, tuple) for x in want)
        turn = np.full(sum(kept), -1)
        if turning:
            n_tiles = max(c0[2] + -(-sum(bin(m).count("1") for _, m, _, _ in entries[c0[0]:c0[1]]) // 16) for c0 in chains)
            o = up(4 * (o + n_tiles)) // 4
            mixed = (entries[:, 3] == -2).any()
            if mixed:
                turn = ints[o:o + len(turn)]
                o = up(4 * (o + len(turn))) // 4
            else:
                for _, mask, k, row in entries[:chains[k - n_back - 1][1]]:
                    turn[k:k + bin(mask).count("1")] = row
            turns = ints[o:]
            assert turn.max() == len(turns) - 1
        have, scratch = pool.copy(), np.full(20000, -1, object)
        order = [x for a, b in ((0, n_direct), (n_direct, n_direct + n_in), (n_direct + n_in, len(chains))) for x in range(b - 1, a - 1, -1)]
        assert len(chains) == n_direct + n_in + n_back
        # chains of a phase may go at the same time: a block that one writes no other reads or writes
        for a, b in ((0, n_direct), (n_direct, n_direct + n_in), (n_direct + n_in, len(chains))):
            writer = {}
            for x in range(a, b):
                e0, e1, tile = chains[x]
                for i in range(-(-sum(bin(mask).count("1") for _, mask, _, _ in entries[e0:e1]) // 16)):
                    assert writer.setdefault(int(tiles[tile + i]), x) == x
            for x in range(a, min(b, n_direct)):  # (what goes through scratch blocks reads one memory and writes the other)
                for block, _, _, _ in entries[chains[x][0]:chains[x][1]]:
                    assert writer.get(int(block), x) == x
        for x in order:
            e0, e1, tile = chains[x]
            back = x >= n_direct + n_in
            source, dest = (scratch if back else have), (scratch if n_direct <= x < n_direct + n_in else have)
            ring, n_stored = [], 0
            for block, mask, k, row in entries[e0:e1]:
                assert 0 < mask < 1 << 16
                some = {-1} if back else set(turn[k:k + bin(mask).count("1")].tolist())
                assert row == (some.pop() if len(some) == 1 else -2)
                for slot in range(16):
                    if mask >> slot & 1:
                        x = source[block * 16 + slot]  # (block * 16 + slot counts tokens as page * P + slot does)
                        ring.append((x, int(turns[turn[k]])) if not back and turn[k] >= 0 else x)
                        k += 1
                while len(ring) >= 16 * (n_stored + 1):
                    b0 = int(tiles[tile + n_stored]) * 16
                    dest[b0:b0 + 16] = ring[16 * n_stored:16 * n_stored + 16]
                    n_stored += 1
            rest = ring[16 * n_stored:]
            if rest:
                b0 = int(tiles[tile + n_stored]) * 16
                dest[b0:b0 + len(rest)] = rest
        assert all(x == y for x, y in zip(have, want)), trial
        ctx.close()
    c.fake.fake_watch(None, 0)
    assert checked > 20 and scratched > 5, (checked, scratched)


def compact_masks(c):
    """Pages that are written become visible throughout; what stays keeps its mask, also where another sequence sees more of it."""
    for P in (16, 32):
        ctx = c.context(n_pages=64, m=SimpleNamespace(**{**vars(MODEL), "page_size": P}))
        every = (1 << P) - 1
        visible = lambda p: int(ctx.compact_kvpage([0, 1], [p], [P], dst_page_indptr=[0, 1], dst_page_ids=[40])[0])  # noqa: E731
        ctx.mask_kvpage([1, 2, 3], [every & ~(1 << (P - 2)), every & ~2, every & ~4])
        # 4 tokens of page 1 (its hidden one is behind them) stay; page 2 loses one, pages 3's first token moves into it
        assert ctx.compact_kvpage([0, 1, 3], [1, 2, 3], [4, P + 1]).tolist() == [4, P]
        assert visible(1) == P - 1 and visible(2) == P and visible(3) == P - 1
        assert ctx.compact_kvpage([0, 1], [3], [P]).tolist() == [P - 1] and visible(3) == P
        ctx.close()


def raw(ctx, name, *args):
    return getattr(ctx.lib, name)(ctx.ctx, *args)


def page_refusals(c):
    ctx = c.context(n_pages=32, layers=2)
    a, b, one = i32([0, 1]), i32([2, 3]), i32([0, 1])
    big = np.zeros(64, np.int8)
    image = C.c_void_p((big.ctypes.data + 15) // 16 * 16)
    odd = C.c_void_p(image.value + 2)
    p = c.Pie.planner(MODEL, 32, 16, 8, 4)
    assert c.status(lambda: p.fork_kvpage([0], [1]))[0] == INVALID
    assert c.status(lambda: p.compact_kvpage([0, 1], [0], [3]))[0] == INVALID
    assert raw(p, "pie_save_kvpage", at(a), 2, image) == INVALID and raw(p, "pie_restore_kvpage", at(a), 2, image) == INVALID
    assert raw(ctx, "pie_fork_kvpage", None, at(b), 2) == INVALID and raw(ctx, "pie_fork_kvpage", at(a), at(b), -1) == INVALID
    assert raw(ctx, "pie_fork_kvpage", None, None, 0) == 0
    assert c.status(lambda: ctx.fork_kvpage([0, 32], [1, 2]))[0] == RANGE and c.status(lambda: ctx.fork_kvpage([0, 1], [-1, 2]))[0] == RANGE
    assert c.status(lambda: ctx.fork_kvpage([0, 1], [2, 2]))[0] == CONFLICT
    for name in ("pie_save_kvpage", "pie_restore_kvpage"):
        assert raw(ctx, name, at(a), 2, None) == INVALID and raw(ctx, name, at(a), 2, odd) == INVALID and raw(ctx, name, at(a), -1, image) == INVALID
        assert raw(ctx, name, None, 0, None) == 0
        assert raw(ctx, name, at(i32([0, 32])), 2, image) == RANGE
    assert raw(ctx, "pie_restore_kvpage", at(i32([4, 4])), 2, image) == CONFLICT and raw(ctx, "pie_save_kvpage", at(i32([4, 4])), 2, image) == 0
    com = lambda *x, **k: c.status(lambda: ctx.compact_kvpage(*x, **k))  # noqa: E731
    assert com([0, 1], [32], [3])[0] == RANGE and com([0, 1], [-1], [3])[0] == RANGE
    assert com([0, 1], [0], [17])[0] == INVALID and com([0, 1], [0], [-1])[0] == INVALID and com([1, 1], [0], [0])[0] == INVALID
    assert com([0, 2, 1, 2], [0, 1], [0, 0, 0])[0] == INVALID
    assert com([0, 1], [0], [16], dst_page_indptr=[0, 0], dst_page_ids=[])[0] == INVALID  # (16 tokens kept, no page for them)
    assert com([0, 1], [0], [16], dst_page_indptr=[0, 1], dst_page_ids=[33])[0] == RANGE
    lens, out = i32([3]), i32([0])
    assert raw(ctx, "pie_compact_kvpage", 1, at(i32([0, 1])), at(a), at(lens), at(i32([0, 1])), None, None, at(out)) == INVALID
    assert raw(ctx, "pie_compact_kvpage", 1, at(i32([0, 1])), None, at(lens), None, None, None, at(out)) == INVALID
    assert raw(ctx, "pie_compact_kvpage", 1, at(i32([0, 1])), at(a), at(lens), None, None, None, None) == INVALID
    assert raw(ctx, "pie_compact_kvpage", -1, None, None, None, None, None, None, None) == INVALID
    assert raw(ctx, "pie_compact_kvpage", 0, None, None, None, None, None, None, None) == 0
    # pages that two sequences share may stay, but not be written
    ctx.mask_kvpage([5], [0xFFFE])
    assert com([0, 2, 4], [4, 5, 4, 6], [32, 32])[0] == 0
    ctx.mask_kvpage([5], [0xFFFE])
    assert com([0, 2, 4], [4, 5, 5, 6], [32, 32])[0] == CONFLICT  # page 5 is written by the first and read by the second
    assert com([0, 2, 4], [4, 5, 7, 6], [32, 32], shifts=np.r_[np.zeros(32), np.ones(32)])[0] == 0
    assert com([0, 2, 4], [4, 6, 4, 7], [32, 32], shifts=np.ones(64))[0] == CONFLICT
    assert com([0, 1, 2], [4, 5], [16, 16], dst_page_indptr=[0, 1, 2], dst_page_ids=[8, 8])[0] == CONFLICT
    assert com([0, 2], [8, 9], [32], dst_page_indptr=[0, 2], dst_page_ids=[9, 8])[0] == CONFLICT
    assert com([0, 2], [8, 9], [32], dst_page_indptr=[0, 2], dst_page_ids=[8, 10])[0] == 0  # (the first page is its own destination)
    # nothing of a refused call has happened: the mask of page 5 is as it was set
    ctx.mask_kvpage([5], [0x00FF])
    assert com([0, 2], [5, 5], [32])[0] == CONFLICT
    assert ctx.compact_kvpage([0, 1], [5], [16], dst_page_indptr=[0, 1], dst_page_ids=[20])[0] == 8
    ctx.close()


def captured(c):
    """While the stream is captured, calls whose plans fit the kernel arguments are taken and the others refused before the runtime is
    asked for anything."""
    ctx = c.context(n_pages=1024)
    ctx.compact_kvpage([0, 4], [0, 1, 2, 3], [60], shifts=np.ones(60))  # a copy is in flight
    c.fake.fake_capturing(1)
    calls = c.fake.fake_event_syncs(), c.fake.fake_allocations()
    ctx.fork_kvpage(np.arange(400), 500 + np.arange(400))
    for n in (16, 1000):
        st, msg = c.status(lambda: ctx.compact_kvpage([0, 70], np.arange(70), [n], shifts=np.ones(n)))
        assert st == HIP and "captured" in msg
    assert calls == (c.fake.fake_event_syncs(), c.fake.fake_allocations())
    c.fake.fake_capturing(0)
    ctx.compact_kvpage([0, 70], np.arange(70), [1000], shifts=np.ones(1000))
    ctx.close()


def images_in_flight(c):
    """Batches and page plans share the host image: each copy gets what its call wrote."""
    from test_host_runtime_paths import batch_of
    ctx = c.context(n_pages=2000)
    shifts = [np.arange(6000), np.arange(6000)[::-1]]
    compact = lambda k: ctx.compact_kvpage([0, 375], np.arange(375), [6000], shifts=shifts[k])  # noqa: E731
    compact(0)
    want = [last_image(c, ctx)]
    ctx.batch_create(batch_of([(1, 40), (20, 5)])).destroy()
    want.append(last_image(c, ctx))
    compact(1)
    want.append(last_image(c, ctx))
    n0 = len(c.copies())
    compact(0)
    b = ctx.batch_create(batch_of([(1, 40), (20, 5)]))
    c.fake.fake_fail_event_syncs(1)
    assert c.status(lambda: compact(1))[0] == HIP
    compact(1)
    ctx.synchronize()
    assert c.copies()[n0:] == want
    b.destroy()
    ctx.close()


def no_memory(c):
    """Every C++ allocation of a call in turn fails, and the device block: PIE_ENOMEM, and the next call does its work."""
    for call in (lambda x: x.fork_kvpage(np.roll(np.arange(200), 1), np.arange(200)),
                 lambda x: x.compact_kvpage([0, 20], np.arange(20), [300], shifts=np.arange(300))):
        failed = 0
        for k in range(1, 4000):
            ctx = c.context(n_pages=1024)
            ctx.mask_kvpage([0], [0xFFF0])
            c.fake.fake_fail_new_at(k)
            st = c.status(lambda: call(ctx))[0]
            hit = c.fake.fake_new_failed()
            c.fake.fake_fail_new_at(0)
            assert st == (MEMORY if hit else 0), (k, st)
            if hit:
                call(ctx)
            ctx.close()
            if not hit:
                break
            failed += 1
        assert failed > 3
        ctx = c.context(n_pages=1024)
        ctx.mask_kvpage([0], [0xFFF0])
        if "compact" not in call.__code__.co_names[0]:
            continue  # (a fork allocates nothing on the device)
        c.fake.fake_malloc_limit(1)
        assert c.status(lambda: call(ctx))[0] == MEMORY
        c.fake.fake_malloc_limit(1 << 62)
        call(ctx)
        ctx.close()


def beam_refusals(c):
    m = SimpleNamespace(**{**vars(MODEL), "vocab": 512})
    ctx = c.loaded(m=m, dist=(8, 4))
    B = c.binding.BeamSearchC
    room = np.zeros(4096, np.int32)
    o = C.c_void_p(room.ctypes.data)

    def search(indptr=(0, 4, 8), n_out=4, t=1.0, finished=None, eos=0):
        ip = i32(indptr)
        s = B(len(ip) - 1, ip.ctypes.data, None, finished, eos, n_out, t)
        s.keep = ip
        return s

    def select(s, z=o, dtype=0, stride=512, n_vocab=512, outs=(o, o, o)):
        return raw(ctx, "pie_beam_select", None if s is None else C.byref(s), z, dtype, stride, n_vocab, *outs)

    assert select(search()) == 0 and select(search(finished=o.value, eos=511)) == 0
    assert select(None) == INVALID and select(search((0,))) == INVALID
    for k in range(3):
        assert select(search(), outs=tuple(None if i == k else o for i in range(3))) == INVALID
    assert select(search(), z=None) == INVALID and select(search((0, 0, 0)), z=None) == 0
    for t in (0.0, -1.0, float("nan"), float("inf"), 9e-31, 1.1e30):
        assert select(search(t=t)) == INVALID
    assert select(search(t=1.1e-30)) == 0 and select(search(t=9e29)) == 0
    assert select(search((1, 4))) == INVALID and select(search((0, 4, 3))) == INVALID
    assert select(search((0, 9))) == BATCH
    assert select(search(n_out=0)) == RANGE and select(search(n_out=257)) == RANGE and select(search(n_out=256)) == 0
    assert select(search(), n_vocab=0) == RANGE and select(search(), n_vocab=513, stride=513) == RANGE and select(search(), stride=511) == INVALID
    assert select(search(), n_vocab=1, stride=1) == 0
    assert select(search(), dtype=3) == INVALID and select(search(), dtype=-1) == INVALID
    assert select(search(), z=C.c_void_p(o.value + 2)) == INVALID and select(search(), z=C.c_void_p(o.value + 2), dtype=1) == 0
    assert select(search(), z=C.c_void_p(o.value + 1), dtype=2) == INVALID
    assert select(search(finished=o.value, eos=512)) == RANGE and select(search(finished=o.value, eos=-1)) == RANGE and select(search(eos=-1)) == 0
    wide = c.loaded(m=m, dist=(300, 4))
    ip = i32([0, 257])
    assert raw(wide, "pie_beam_select", C.byref(B(1, ip.ctypes.data, None, None, 0, 4, 1.0)), o, 0, 512, 512, o, o, o) == BATCH
    beams = lambda s, ids: raw(ctx, "pie_get_next_beams", None if s is None else C.byref(s), at(ids), o, o, o)  # noqa: E731
    assert beams(search(), i32(np.arange(8))) == 0
    assert beams(search(), None) == INVALID and beams(search((0, 0)), i32([0])) == INVALID and beams(None, i32([0])) == INVALID
    assert beams(search((0, 1)), i32([1024])) == RANGE and beams(search((0, 1)), i32([-1])) == RANGE and beams(search((0, 9)), i32(np.arange(9))) == BATCH
    no_head = c.context(m=m, dist=(8, 4))
    assert raw(no_head, "pie_get_next_beams", C.byref(search()), at(i32(np.arange(8))), o, o, o) == INVALID
    no_vocab = c.context()
    assert raw(no_vocab, "pie_beam_select", C.byref(search()), o, 0, 512, 512, o, o, o) == RANGE
    p = c.Pie.planner(m, 32, 16, 8, 4)
    assert raw(p, "pie_beam_select", C.byref(search()), o, 0, 512, 512, o, o, o) == INVALID
    assert raw(p, "pie_get_next_beams", C.byref(search()), at(i32([0])), o, o, o) == INVALID


CASES = {f.__name__: f for f in (fork_masks, compact_masks, compact_plans, page_refusals, captured, images_in_flight, no_memory, beam_refusals)}

if __name__ == "__main__":
    CASES[sys.argv[2]](Child(sys.argv[1]))
    print("case passed")
    sys.exit(0)


@pytest.mark.parametrize("case", list(CASES))
def test_host_path(fake, case):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), fake, case], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "case passed" in r.stdout, f"exit {r.returncode}\n{r.stdout}\n{r.stderr}"
