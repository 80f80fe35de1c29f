"""The attention over full caches as index arithmetic: how rows, tiles and keys are shared out among workgroups, and every
address that the kernels form from it, worked out on the CPU from the same expressions and constants and held against the
buffers.  The expressions are checked to stand in the sources as they are written down here: where one changes, the model has to
change with it."""
import bisect
import os
import random
import re

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2403_09636_amd", "csrc")
HIP, HDR, API = (open(os.path.join(CSRC, n)).read() for n in ("dmc_full.hip", "dmc_full.h", "dmc_api.cpp"))


def _const(text, name):
    return eval(re.search(r"\b%s = ([0-9<() ]+)[,;]" % name, text).group(1))


PLACES = _const(HDR, "kFullPlaces")
NARROW, CHUNK, WIDE, EQUAL, JOIN, JOIN_PAIRS, WIDE_COLS, FEW, MANY = (
    _const(HIP, n) for n in ("kNarrowRange", "kChunkRange", "kWideRange", "kEqualKeys", "kJoin", "kJoinPairs", "kWideCols",
                             "kAloneFew", "kAloneMany"))
COUNTERS = int(re.search(r"#define DMC_FULL_COUNTER_BYTES (\d+)", open(os.path.join(ROOT, "include", "dmc.h")).read()).group(1))

# What the model below takes from the sources, as they have it.
EXPRESSIONS = {
    HDR: ["return cols <= 16 || group > 64 ? 16 : 64;", "return cols <= 16 ? 16 : cols <= 32 || group > 128 ? 32 : 128;",
          "return tiles * hkv * capacity <= int64_t(1) << 18;"],
    API: ["const int narrow = std::min(L.tile_cols, es == 4 ? 16 : 32);",
          "cu ? int64_t(total) * G / narrow + cfg->batch : int64_t(cfg->batch) * ((G + narrow - 1) / narrow);",
          "p.tile_cols = p.one_launch ? narrow : L.tile_cols;", "p.tile_tokens = std::max(1, p.tile_cols / G);",
          "return int64_t(tile_cols) * (head_dim + 2);", "size_t(dmc::kFullPlaces) * 2 * full_record_floats(L.tile_cols, c.head_dim) * 4",
          "p.capacity = cfg->max_pages * cfg->page_size;"],
    HIP: [
        "r.n = min(n, capacity);", "r.m = n < 0 ? 0 : min(r.given, capacity - r.n);",
        "step = TRI ? tokens : cols;", "const int all = TRI ? m : m * G;", "count = all <= step ? 1 : (all + step - 1) / step;",
        "return TRI ? n + min(m, (t + 1) * step) : n + m;",
        "return TRI ? int64_t(t) * n + int64_t(step) * t * (t + 1) / 2 : int64_t(t) * (n + m);",
        "return m > 0 ? before(count - 1) + keys(count - 1) : 0;", "return TRI ? t * step * G : t * step;",
        "equal = count <= grid && sum <= (4 * count <= grid ? kEqualKeys : kEqualKeys / 2) * grid;",
        "const int each = max(small_div(sum, max(grid - count, 1)) + 1, LEAST);", "pieces = (keys + each - 1) / each;",
        "per = equal ? 1 : max((all + grid - 1) / grid, int64_t(LEAST));",
        "static constexpr int kSnap = TRI && ES == 2 ? 512 : 128;", "const int64_t v = min(i * per, all);",
        "return v - u.begin <= kSnap ? u.begin : u.begin + u.keys - v <= kSnap ? u.begin + u.keys : v;",
        "const int o = static_cast<int>(off), unit = small_div(o, u.pieces);", "u.index = o - unit * u.pieces;",
        "u.h = small_div(unit, ts.count);", "u.t = unit - u.h * ts.count;", "u.begin = v - in_head + ts.before(u.t);",
        "x.first = range - x.index;", "const int size = (small_div(x.keys + x.pieces - 1, x.pieces) + 31) & ~31;",
        "x.k0 = min(x.index * size, x.keys);", "x.k1 = min(x.k0 + size, x.keys);",
        "x.k1 = static_cast<int>(min(int64_t(x.keys), x.k0 + (hi - pos)));",
        "x.first = static_cast<int>((u.begin + min(kSnap, x.keys - 1)) / per);",
        "x.pieces = max(static_cast<int>((u.begin + x.keys - kSnap - 1) / per) - x.first, 0) + 1;", "x.index = range - x.first;",
        "x.cols = min(TRI ? ts.step * G : ts.step, u.m * G - x.col0);",
        "return 2 * (first + index) + (index == 0 ? 1 : 0);",
        # addresses
        "const int col0 = x.col0 + (SPLIT_KEYS ? 0 : wave * 16 * NT), cols = min(16 * NT, x.col0 + x.cols - col0);",
        "const int keys = SPLIT_KEYS ? x.keys : cols > 0 ? x.n + div_group(p, col0 + cols - 1) + 1 : 0;",
        "const int i = div_group(p, col0 + c), head = x.h * G + (col0 + c) - i * G;",
        "const int kb1 = (min(x.k1, keys) + KEYS - 1) / KEYS;", "int kb = (x.k0 + KEYS - 1) / KEYS + (SPLIT_KEYS ? wave : 0);",
        "pg.x[u] = table[min(kb * KEYS + u * 16 + c16, keys - 1) >> p.log2p];",
        "pg.x[U + u] = table[min(kb * KEYS + u * 16 + g4 * 4, keys - 1) >> p.log2p];",
        "pg.x[0] = table_entry(table, min(kb * KEYS, keys - 1) >> p.log2p);",
        "((int64_t(checked_page(p, page)) * p.hkv + x.h) << p.log2p) * RB;", "int64_t((kb * KEYS) & mask) * RB);",
        "(min(kb * KEYS + u * 16 + c16, keys - 1) & mask) * RB + X::key_offset(g4));",
        "at + (min(kb * KEYS + u * 16 + g4 * 4 + i, keys - 1) & mask) * RB);", "const uint32_t last = keys - 1 - kb * KEYS;",
        "at + (min(uint32_t(u * 16 + c16), last) * RB + X::key_offset(g4)));",
        "at + (min(uint32_t((i >> 2) * 16 + g4 * 4 + (i & 3)), last) * RB + c16 * (E * ES)));", "next = pages_of(min(kb + STEP, kb1 - 1));",
        "next = pages_of(min(kb + 2 * STEP, kb1 - 1));", "if (key >= keys) break;",
        "put2(p, rec + 2 * (e2 * COLS + col), a, bb);", "put2(p, rec + COLS * D + 2 * col, top, sum);",
        "const int blk0 = (x.k0 + 31) >> 5, nblk = (x.k1 + 31) >> 5;",
        "table_entry(table, min(min(kb, nblk - 1) * 32 + (i * kWaves + wave) * RPI, x.keys - 1) >> p.log2p);",
        "const int first = min(kb * 32 + (i * kWaves + wave) * RPI, x.keys - 1);", "const uint32_t row = min(lrow, x.keys - 1 - first);",
        "(((int64_t(checked_page(p, pg.x[i])) * p.hkv + x.h) << p.log2p) + (first & mask)) * RB;",
        "x = part * STEP + lane / VPR; x < items; x += parts * STEP", "(blockIdx.x + gridDim.x - b % gridDim.x) % gridDim.x",
    ],
}


@pytest.mark.parametrize("i", range(3))
def test_the_sources_have_the_expressions(i):
    text = re.sub(r"\s+", " ", list(EXPRESSIONS)[i])
    for e in list(EXPRESSIONS.values())[i]:
        assert re.sub(r"\s+", " ", e) in text, e


class Tiles:
    def __init__(self, tri, n, m, G, cols, tokens):
        self.tri, self.n, self.m, self.G = tri, n, m, G
        self.step = tokens if tri else cols
        every = m if tri else m * G
        self.count = 1 if every <= self.step else -(-every // self.step)

    def keys(self, t):
        return self.n + min(self.m, (t + 1) * self.step) if self.tri else self.n + self.m

    def before(self, t):
        return t * self.n + self.step * t * (t + 1) // 2 if self.tri else t * (self.n + self.m)

    def all(self):
        return self.before(self.count - 1) + self.keys(self.count - 1) if self.m > 0 else 0

    def at(self, off):
        lo, hi = 0, self.count
        while hi - lo > 1:
            mid = (lo + hi) // 2
            lo, hi = (mid, hi) if self.before(mid) <= off else (lo, mid)
        return lo

    def first_col(self, t):
        return t * self.step * self.G if self.tri else t * self.step


def small_div(a, b):
    assert 0 <= a < 1 << 22 and b > 0
    return a // b


class Call:
    """One call and all of its pieces, by workgroup."""

    def __init__(self, held, lens, hq, hkv, d, es, page, max_pages, table, num_pages, packed, max_chunk, total):
        self.held, self.hq, self.hkv, self.d, self.es, self.page, self.table = held, hq, hkv, d, es, page, table
        self.max_pages, self.num_pages, self.total, self.max_chunk = max_pages, num_pages, total, max_chunk
        self.G = G = hq // hkv
        self.rows, self.capacity = len(held), max_pages * page
        cols = max_chunk * G
        layout = (16 if cols <= 16 or G > 64 else 64) if es == 4 else (16 if cols <= 16 else 32 if cols <= 32 or G > 128 else 128)
        narrow = min(layout, 16 if es == 4 else 32)
        tiles = total * G // narrow + self.rows if packed else self.rows * -(-G // narrow)
        self.one = tiles * hkv * self.capacity <= 1 << 18
        self.cols = narrow if self.one else layout
        self.tokens = max(1, self.cols // G)
        self.split = self.cols <= (16 if es == 4 else 32)     # whole rows, each wave a fourth of the keys
        self.tri = not self.split
        self.least = NARROW if self.split else CHUNK if es == 4 else WIDE
        self.snap = 512 if self.tri and es == 2 else 128
        self.record = self.cols * (d + 2)
        cu = [0]
        for m in lens:
            cu.append(cu[-1] + m)
        self.row = []
        for b, n in enumerate(held):
            start, given = (cu[b], lens[b]) if packed else (b, 1)
            n = min(n, self.capacity)
            self.row.append((start, given, n, 0 if n < 0 else min(given, self.capacity - n)))
        self.share_out()

    def tiles(self, b):
        _, _, n, m = self.row[b]
        return Tiles(self.tri, n, min(m, self.max_chunk), self.G, self.cols, self.tokens)

    def share_out(self):
        few, self.equal, share = self.rows <= 64, False, []
        if few:
            units, keys = [], []
            for b, (_, _, n, m) in enumerate(self.row):
                m = min(m, self.max_chunk)
                units.append(min(self.hkv * self.tiles(b).count, 1 << 24) if m > 0 else 0)
                keys.append(n + m)
            count, total = sum(units), sum(min(u * k, 1 << 24) for u, k in zip(units, keys))
            self.equal = count <= PLACES and total <= (EQUAL if 4 * count <= PLACES else EQUAL // 2) * PLACES
            if self.equal:
                each = max(small_div(total, max(PLACES - count, 1)) + 1, self.least)
                self.pieces = [-(-k // each) if u else 0 for u, k in zip(units, keys)]
                share = [u * x for u, x in zip(units, self.pieces)]
        if not self.equal:
            share = [self.hkv * self.tiles(b).all() if self.row[b][3] > 0 else 0 for b in range(self.rows)]
        self.before = [0]
        for x in share:
            self.before.append(self.before[-1] + x)
        self.all = self.before[-1]
        self.per = 1 if self.equal else max(-(-self.all // PLACES), self.least)
        if self.equal:
            assert self.all <= PLACES
        self.ranges = [list(self.range(r)) for r in range(PLACES)]

    def unit(self, v):
        b = bisect.bisect_right(self.before, v) - 1
        assert self.before[b] <= v < self.before[b + 1]
        ts, off = self.tiles(b), v - self.before[b]
        if self.equal:
            u = small_div(off, self.pieces[b])
            h = small_div(u, ts.count)
            return b, ts, h, u - h * ts.count, off - u * self.pieces[b], None
        h, inside = divmod(off, ts.all())
        t = ts.at(inside)
        return b, ts, h, t, None, v - inside + ts.before(t)

    def boundary(self, i):
        v = min(i * self.per, self.all)
        if self.equal or v in (0, self.all):
            return v
        _, ts, _, t, _, begin = self.unit(v)
        end = begin + ts.keys(t)
        return begin if v - begin <= self.snap else end if end - v <= self.snap else v

    def range(self, r):
        pos, hi = self.boundary(r), self.boundary(r + 1)
        while pos < hi:
            b, ts, h, t, index, begin = self.unit(pos)
            keys = ts.keys(t)
            if self.equal:
                n = self.pieces[b]
                first = r - index
                size = (small_div(keys + n - 1, n) + 31) & ~31
                k0 = min(index * size, keys)
                k1 = min(k0 + size, keys)
                pos = hi
            else:
                k0 = pos - begin
                k1 = min(keys, k0 + hi - pos)
                first = (begin + min(self.snap, keys - 1)) // self.per
                n = max((begin + keys - self.snap - 1) // self.per - first, 0) + 1
                index = r - first
                pos += k1 - k0
            col0 = ts.first_col(t)
            start, _, held, m = self.row[b]
            cols = min(ts.step * self.G if self.tri else ts.step, min(m, self.max_chunk) * self.G - col0)
            yield dict(b=b, n=held, start=start, h=h, t=t, col0=col0, cols=cols, keys=keys, k0=k0, k1=k1, first=first, index=index,
                       pieces=n, m=min(m, self.max_chunk))

    # ------------------------------------------------------------------
    def check(self):
        seen, units, records, joins = {}, {}, set(), []
        every = max(sum(map(len, self.ranges)) // 200, 1)   # (of many pieces some, and all that are cut)
        number = 0
        for r, pieces in enumerate(self.ranges):
            cut = [x for x in pieces if x["pieces"] != 1]
            assert len(cut) <= 2, r
            for x in pieces:
                units.setdefault((x["b"], x["h"], x["col0"]), []).append(x)
                number += 1
                if number % every == 0 or x["pieces"] != 1 and len(units) < 300:
                    self.check_piece(x)
                if x["pieces"] != 1:
                    self.check_record(x, records)
            if not self.one and cut and cut[-1]["index"] == 0:
                joins.append(cut[-1])
        assert max((x["first"] for x in joins), default=0) < PLACES and len({x["first"] for x in joins}) == len(joins)
        joined = {(x["b"], x["h"], x["col0"]): x["pieces"] for x in joins}
        for u, parts in units.items():
            parts.sort(key=lambda x: x["index"])
            assert [x["index"] for x in parts] == list(range(parts[0]["pieces"])), u
            assert parts[0]["k0"] == 0 and parts[-1]["k1"] == parts[0]["keys"]
            assert all(x["k1"] == y["k0"] for x, y in zip(parts, parts[1:])), u
            if not self.one:
                assert joined.get(u, 1) == len(parts), u
            b, h, col0 = u
            for c in range(col0, col0 + parts[0]["cols"]):
                i = c // self.G
                key = parts[0]["start"] + i, h * self.G + c - i * self.G
                assert key not in seen and 0 <= key[0] < self.total and 0 <= key[1] < self.hq, key
                assert parts[0]["n"] + i < parts[0]["keys"]   # the token's last key is among the unit's
                seen[key] = b
        for b, (start, given, n, m) in enumerate(self.row):
            for i in range(min(m, self.max_chunk)):
                assert all((start + i, h) in seen for h in range(self.hq)), (b, i)
        assert len(seen) == self.hq * sum(min(m, self.max_chunk) for _, _, _, m in self.row)
        self.check_dropped()

    def check_record(self, x, records):
        at = 2 * (x["first"] + x["index"]) + (x["index"] == 0)
        assert 0 <= at < 2 * PLACES and at not in records
        records.add(at)
        # the last float that is written and read: of the statistics, of the accumulator (two columns at once)
        assert self.cols * self.d + 2 * (x["cols"] - 1) + 1 < self.record
        assert 2 * ((self.d // 2 - 1) * self.cols + ((x["cols"] - 1) & ~1)) + 3 < self.cols * self.d
        assert JOIN_PAIRS // x["pieces"] & ~1 >= 2
        if self.one:
            begin = x["index"] // JOIN * JOIN
            group = 2 * (x["first"] + begin) + (begin == 0)
            assert 0 <= group < 2 * PLACES and 4 * (2 * PLACES + x["first"] + 1) <= COUNTERS and x["first"] >= 0

    def in_pool(self, page, h, slot, offset, size):
        row = self.d * self.es
        at = ((page * self.hkv + h) * self.page + slot) * row + offset
        assert (page >= 0).all() and (page < self.num_pages).all() and (at >= 0).all()
        assert (at + size <= self.num_pages * self.hkv * self.page * row).all() and ((offset + size) <= row).all()

    def pages(self, b, index):
        assert (index >= 0).all() and (index < self.max_pages).all()
        return self.table[b][index]

    def check_piece(self, x):
        wide = not self.split and self.es == 2
        waves = range(4) if self.tri else [0]
        assert x["keys"] > 0 and x["cols"] > 0 and 0 <= x["k0"] <= x["k1"] <= x["keys"] and 0 <= x["h"] < self.hkv
        assert x["cols"] <= self.cols and x["keys"] <= self.capacity
        if wide:
            return self.check_wide(x)
        U = 2 if self.es == 2 or self.d == 64 else 1
        K, E, row = 16 * U, self.d // 16, self.d * self.es
        lane = np.arange(64)
        c16, g4 = lane & 15, lane >> 4
        small = self.page < K
        slices = row // 64
        for w in waves:
            col0 = x["col0"] + (0 if self.split else w * 16)
            nt = self.cols // 16 if self.split else 1
            cols = min(16 * nt, x["col0"] + x["cols"] - col0)
            for c in range(max(cols, 0)):
                i = (col0 + c) // self.G
                head = x["h"] * self.G + col0 + c - i * self.G
                assert 0 <= x["start"] + i < self.total and 0 <= head < self.hq
            keys = x["keys"] if self.split else x["n"] + (col0 + cols - 1) // self.G + 1 if cols > 0 else 0
            assert keys <= x["keys"]
            kb1 = -(-min(x["k1"], keys) // K)
            blocks = range(-(-x["k0"] // K), kb1)
            for kb in sorted({*blocks[:2], *blocks[-2:]}):
                for u in range(U):
                    key = np.minimum(kb * K + u * 16 + c16, keys - 1)
                    page = self.pages(x["b"], key // self.page if small else np.full(64, min(kb * K, keys - 1) // self.page))
                    slot = key % self.page if small else (kb * K) % self.page + np.minimum(u * 16 + c16, keys - 1 - kb * K)
                    assert (slot < self.page).all()
                    self.in_pool(page, x["h"], slot, 16 * g4 + 64 * (slices - 1), 16)
                    for i in range(4):
                        key = np.minimum(kb * K + u * 16 + g4 * 4 + i, keys - 1)
                        if small:   # one page for a lane's four values
                            page = self.pages(x["b"], np.minimum(kb * K + u * 16 + g4 * 4, keys - 1) // self.page)
                            assert (page == self.table[x["b"]][key // self.page]).all()
                            slot = key % self.page
                        else:
                            slot = (kb * K) % self.page + np.minimum(u * 16 + g4 * 4 + i, keys - 1 - kb * K)
                            assert (self.table[x["b"]][key // self.page] == page).all() and (slot == key % self.page).all()
                        self.in_pool(page, x["h"], slot, c16 * E * self.es, E * self.es)

    def check_wide(self, x):
        assert self.cols == WIDE_COLS
        row = self.d * 2
        chunks = row // 16
        per_instr = 64 // chunks                     # rows of one transfer
        transfers = 32 * row // 16 // 256            # of a wave, of a block of 32 keys
        lane = np.arange(64)
        blk0, nblk = (x["k0"] + 31) >> 5, (x["k1"] + 31) >> 5
        blocks = list(range(blk0, nblk))
        for kb in sorted({*blocks[:2], *blocks[-2:]}) + ([nblk, nblk + 4] if blocks else []):
            for i in range(transfers):
                for w in range(4):
                    place = (i * 4 + w) * per_instr
                    page = self.pages(x["b"], np.array([min(min(kb, nblk - 1) * 32 + place, x["keys"] - 1) // self.page]))
                    if kb >= nblk:                   # switched off
                        continue
                    first = min(kb * 32 + place, x["keys"] - 1)
                    r = np.minimum(lane // chunks, x["keys"] - 1 - first)
                    slot = first % self.page + r
                    assert (slot < self.page).all() and (self.table[x["b"]][(first + r) // self.page] == page).all()
                    self.in_pool(np.broadcast_to(page, 64), x["h"], slot, 16 * (lane % chunks), 16)
        for c in range(x["cols"]):
            i = (x["col0"] + c) // self.G
            assert 0 <= x["start"] + i < self.total

    def check_dropped(self):
        """Every dropped (token, head) once, each by the workgroups that share the row."""
        row = self.d * self.es // 16
        for b, (start, given, n, m) in enumerate(self.row):
            items = (given - m) * self.hq
            if items <= 0:
                continue
            few = self.rows <= 64
            alone = items <= (FEW if few else MANY)
            lanes = 256 if few or alone else 64
            step, parts = lanes // row, 1 if alone else PLACES
            taken = np.zeros(items, dtype=int)
            for block in range(PLACES):
                if alone and block != b % PLACES:
                    continue
                part = 0 if alone else (block + PLACES - b % PLACES) % PLACES
                for lane in range(0, lanes, row):
                    taken[part * step + lane // row::parts * step] += 1
            assert (taken == 1).all(), b
            assert 0 <= start + m and start + given <= self.total


def make(held, lens, hq, hkv, d, es, page, room=0, packed=True, tail=0, max_chunk=None, rng=None):
    need = [-(-(n + m) // page) if n >= 0 else 0 for n, m in zip(held, lens)]
    width = max(max(need), 1, room // page)
    order = list(range(2, sum(need) + 2))
    (rng or random.Random(1)).shuffle(order)
    table = []
    for k in need:
        table.append(np.array(order[:k] + [-1] * (width - k)))
        order = order[k:]
    chunk = max(max(lens), 1) if max_chunk is None else max_chunk
    return Call(held, lens, hq, hkv, d, es, page, width, table, sum(need) + 2, packed, chunk, sum(lens) + tail)


STEP = [0, 1, 30, 31, 32, 63, 64, -1, 127, 255, 256, 300, 511, 700]


@pytest.mark.parametrize("room", [0, 1 << 19])
@pytest.mark.parametrize("es,d", [(4, 128), (4, 64), (2, 128)])
@pytest.mark.parametrize("hq,hkv", [(34, 2), (8, 1)])
@pytest.mark.parametrize("page", [8, 32])
def test_steps(room, es, d, hq, hkv, page):
    """Among them the step that is not run on the GPU: fp32, 34 query heads on 2 of 128, pages of 8 tokens."""
    c = make(STEP, [1] * len(STEP), hq, hkv, d, es, page, room, packed=False)
    if (es, d, hq) == (4, 128, 34):
        assert c.cols == (16 if room == 0 else 64) and c.one == (room == 0)
    c.check()


@pytest.mark.parametrize("room", [0, 1 << 19])
@pytest.mark.parametrize("es", [2, 4])
@pytest.mark.parametrize("held,lens,hq,hkv,page", [([0, 700, 77, 1300, 20], [300, 129, 0, 257, 1], 8, 8, 32), ([0, 4000, 0], [0, 200, 0], 8, 1, 8),
                                                   ([90, 20, 64], [150, 40, 1], 16, 2, 16), ([140001], [1], 8, 1, 64), ([100, -1, 3], [70, 900, 5], 71, 1, 8)])
def test_chunks(room, es, held, lens, hq, hkv, page):
    for d in (64, 128):
        make(held, lens, hq, hkv, d, es, page, room, tail=2).check()


@pytest.mark.parametrize("seed", range(48))
def test_any_mix_of_rows(seed):
    rng = random.Random(seed)
    rows = rng.choice([1, 2, 5, 30, 64, 65, 90])
    es, d, page = rng.choice([2, 2, 4]), rng.choice([64, 128]), rng.choice([8, 16, 32, 128])
    G, hkv = rng.choice([1, 2, 3, 4, 8, 17, 64, 65, 129]), rng.choice([1, 2, 5, 8])
    long, most = rng.choice([20, 300, 3000]), rng.choice([1, 1, 4, 40, 200]) if rows < 30 else rng.choice([1, 1, 4, 20])
    held = [rng.randint(-long // 8 - 1, long) for _ in range(rows)]
    packed = most > 1 or rng.random() < 0.5
    lens = [rng.randint(0, most) if packed else 1 for _ in range(rows)]
    c = make([max(n, -1) for n in held], lens, G * hkv, hkv, d, es, page, rng.choice([0, 0, 1 << 16]), packed, rng.randint(0, 3) if packed else 0, rng=rng)
    c.check()
