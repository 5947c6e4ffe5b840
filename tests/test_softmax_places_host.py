"""Softmax attention's index arithmetic that the compiler can check without a GPU: the headers
are compiled for the host with static assertions (in a constant expression an overflow of int32
is an error)."""
import glob
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def host_compile(tmp_path, body):
    src = tmp_path / "check.hip"
    src.write_text('#include "paper_2012_01170_amd/csrc/softmax_kernels.hpp"\nusing namespace sbc;\n'
                   + body)
    return subprocess.run([HIPCC, "-std=c++17", f"-I{ROOT}", "--offload-arch=gfx950",
                           "--cuda-host-only", "-fsyntax-only", str(src)],
                          capture_output=True, text=True, timeout=300)


needs_hipcc = pytest.mark.skipif(not (os.path.exists(HIPCC) or shutil.which(HIPCC)),
                                 reason="hipcc is not installed")


@needs_hipcc
def test_search_over_splits(tmp_path):
    """The sequence that a place belongs to: the last that begins at or before it where splits
    are in order, and where they fall one that does, so that no tile begins before its rows."""
    r = host_compile(tmp_path, """
constexpr int32_t kN = 300;  // sequences, in up to two rounds of 64 lanes
struct Splits { int32_t at[kN + 1]; };
constexpr int32_t begin(const Splits &s, int32_t group, int32_t b) {
    return (int32_t)((int64_t)s.at[b] * group / 128) + b;
}
constexpr int32_t find(const Splits &s, int32_t group, int32_t n, int32_t x) {
    return last_beginning(n, [&](int32_t lo, int32_t step, int32_t hi) {
        uint64_t bits = 0;
        for (int lane = 0; lane < 64; ++lane) {
            const int64_t b = lo + (int64_t)lane * step;
            if (b < hi && begin(s, group, (int32_t)b) <= x) bits |= (uint64_t)1 << lane;
        }
        return bits;
    });
}
// whether every place's sequence begins at or before it, or is the last such one (`last`)
constexpr bool holds(const Splits &s, int32_t group, int32_t n, int32_t places, bool last) {
    for (int32_t x = 0; x < places; ++x) {
        const int32_t b = find(s, group, n, x);
        if (b < -1 || b >= n || (b >= 0 && begin(s, group, b) > x)) return false;
        if (!last) continue;
        int32_t want = -1;
        for (int32_t i = 0; i < n && begin(s, group, i) <= x; ++i) want = i;
        if (b != want) return false;
    }
    return true;
}
constexpr Splits kFall{{0, 12800, 0, 0, 0, 20000}};
static_assert(holds(kFall, 2, 5, 330, false), "splits that fall, 5 sequences");
static_assert(find(kFall, 2, 5, 2) == 0, "place 2 of them");
constexpr Splits mixed() {
    Splits s{};
    uint32_t r = 1;
    for (int i = 0; i <= kN; ++i) s.at[i] = (r = r * 1664525u + 1013904223u) >> 18;
    return s;
}
static_assert(holds(mixed(), 3, kN, 90, false), "splits in no order, 300 sequences");
constexpr Splits rising() {
    Splits s{};
    for (int i = 1; i <= kN; ++i) s.at[i] = s.at[i - 1] + (i % 7 == 0 ? 0 : i % 5 * 9);
    return s;
}
static_assert(holds(rising(), 2, kN, 90, true) && holds(rising(), 5, kN, 120, true) &&
              holds(rising(), 1, 64, 70, true) && holds(rising(), 1, 65, 70, true) &&
              holds(rising(), 1, 1, 9, true), "splits in order");
static_assert(find(rising(), 2, 0, 3) == -1, "no sequence");
""")
    assert r.returncode == 0, r.stderr


# lengths next to the most keys that a call takes, and whether the parts of `lk` keys cover those up
# to `limit` once each
PARTS = """
constexpr int32_t kMost = (int32_t)kMostRows;
static_assert(kMostRows == 2147482624, "keys that a call takes");
constexpr bool covers(int32_t lk, int32_t parts, int32_t limit) {
    const int32_t size = part_keys(lk, parts);
    int32_t next = 0;
    for (int32_t part = 0; part < parts; ++part) {
        const int32_t first = part * size;
        if (part > 0 && first >= limit) break;
        const int32_t end = part_end(first, size, limit);
        if (first != next || end < first) return false;
        next = end;
    }
    return next == limit;
}
constexpr int32_t kNear[] = {0, 1, 127, 128, 129, 5000, 1440000000, 2120000000, kMost - 8192, kMost - 8191,
                             kMost - 129, kMost - 128, kMost - 1, kMost};
"""


@needs_hipcc
def test_parts_cover_the_keys(tmp_path):
    r = host_compile(tmp_path, PARTS + """
constexpr bool all() {
    for (int32_t parts = 2; parts <= 64; ++parts)
        for (int32_t lk : kNear)
            for (int32_t limit : kNear)
                if (limit <= lk && !covers(lk, parts, limit)) return false;
    return true;
}
static_assert(all(), "each key is in one part");
""")
    assert r.returncode == 0, r.stderr


@needs_hipcc
def test_parts_are_counted(tmp_path):
    """The parts that are joined: those that begin below a row's limit."""
    r = host_compile(tmp_path, PARTS + """
constexpr bool all() {
    for (int32_t parts = 2; parts <= 64; ++parts)
        for (int32_t lk : kNear)
            for (int32_t limit : kNear) {
                if (limit > lk) continue;
                const int32_t size = part_keys(lk, parts);
                int32_t want = 0;
                while (want < parts && (int64_t)want * size < limit) ++want;
                if (parts_below(limit, size) != want) return false;
            }
    return true;
}
static_assert(all(), "the parts that begin below the limit");
""")
    assert r.returncode == 0, r.stderr


def test_assembly_names_what_it_overwrites():
    """Each piece of assembly that sets m0 names it to the compiler, which may keep a value there."""
    found = 0
    for path in glob.glob(os.path.join(ROOT, "paper_2012_01170_amd", "csrc", "*.h*")):
        for text in re.findall(r"asm\b.*?;", open(path).read(), re.S):
            if re.search(r"\bm0\s*,\s*%", text):
                found += 1
                assert '"m0"' in text.rsplit(":", 1)[1], (path, text)
    assert found > 0
