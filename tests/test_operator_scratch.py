"""The layer operators' scratch (csrc/heddle_scratch.cuh) with memory of its
own that records what is released and when (no GPU): a block whose address a
captured graph holds outlives every growth.  And how much attention asks for."""

import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2609_34244_gb300")
CSRC = os.path.join(PKG, "csrc")

HEAD = r'''
#include <cstdio>
#include <cstdlib>
#include <set>
#include "heddle_scratch.cuh"

#define CHECK(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)

static size_t room = 0;  // bytes left
static std::set<void*> live;
static bool in_capture = false, released_in_capture = false;
struct Memory {  // the size is held ahead of the block
    static void* allocate(size_t n) {
        if (n > room) return nullptr;
        size_t* p = static_cast<size_t*>(std::malloc(16 + n));
        p[0] = n;
        room -= n;
        live.insert(p + 2);
        return p + 2;
    }
    static void release(void* v) {
        if (in_capture) released_in_capture = true;
        if (!live.erase(v)) { std::printf("released twice\n"); std::exit(2); }
        size_t* p = static_cast<size_t*>(v) - 2;
        room += p[0];
        std::free(p);
    }
};
static bool take(hd::Scratch<Memory>& s, size_t n, bool captured, bool or_keep = false) {
    in_capture = captured;
    const bool ok = s.reserve(n, captured, or_keep);
    in_capture = false;
    return ok;
}
int main() {
    hd::Scratch<Memory> s;
'''

CASES = {
    "grows and gives back what no graph holds": r'''
    room = 1000;
    CHECK(take(s, 100, false));
    void* a = s.get();
    CHECK(take(s, 60, false) && s.get() == a && s.size() == 100);
    CHECK(take(s, 300, false) && s.size() == 300 && live.size() == 1 && room == 700);
''',
    "keeps what a graph holds": r'''
    room = 1000;
    CHECK(take(s, 100, true));
    void* a = s.get();
    CHECK(take(s, 200, false) && s.get() != a && live.count(a));
    CHECK(take(s, 400, false) && live.count(a) && live.size() == 2 && room == 500);
''',
    "keeps what a graph holds that grew before": r'''
    room = 1000;
    CHECK(take(s, 100, false));
    CHECK(take(s, 50, true));  // captured in the block that was there
    void* a = s.get();
    CHECK(take(s, 200, true));
    void* b = s.get();
    CHECK(take(s, 300, false) && live.count(a) && live.count(b) && live.size() == 3);
''',
    "releases nothing during a capture, and later what no graph holds": r'''
    room = 1000;
    CHECK(take(s, 100, false));
    CHECK(take(s, 200, true) && live.size() == 2 && !released_in_capture);
    void* b = s.get();
    CHECK(take(s, 300, false) && live.count(b) && live.size() == 2);
''',
    "without room the old block is given up for the new one, unless it is kept": r'''
    room = 1000;
    CHECK(take(s, 600, false));
    void* a = s.get();
    CHECK(!take(s, 900, false, true) && s.get() == a && s.size() == 600);
    CHECK(take(s, 900, false) && s.size() == 900 && live.size() == 1);
    CHECK(!take(s, 2000, false) && !s.get() && s.size() == 0 && live.empty());
    CHECK(take(s, 10, false) && s.size() == 10);
''',
    "without room a captured block stays": r'''
    room = 1000;
    CHECK(take(s, 600, true));
    void* a = s.get();
    CHECK(!take(s, 700, false) && s.get() == a && live.count(a) && s.size() == 600);
    CHECK(!take(s, 700, true) && s.get() == a && live.count(a));
    CHECK(take(s, 500, false) && s.get() == a);
''',
}


REFUSALS = {
    "is asked for again after some calls": r'''
    CHECK(r.worth_asking(100));
    r.refused(100);
    int asked = 0;
    for (int i = 0; i < 10 * hd::Refusal::kAgain; ++i) asked += r.worth_asking(i % 2 ? 100 : 200);
    CHECK(asked == 10);
''',
    "less than what was refused is asked for at once": r'''
    r.refused(100);
    CHECK(r.worth_asking(99) && !r.worth_asking(100));
    r.refused(50);
    CHECK(!r.worth_asking(99) && r.worth_asking(49));
    r.refused(80);
    CHECK(!r.worth_asking(50));
''',
    "is forgotten once granted": r'''
    r.refused(100);
    r.granted(60);  // less than was refused says nothing of it
    CHECK(!r.worth_asking(100));
    r.granted(100);
    CHECK(r.worth_asking(100) && r.worth_asking(200));
''',
}


@pytest.mark.parametrize("name", REFUSALS)
def test_refusal(name, tmp_path):
    src, exe = tmp_path / "refusal.cpp", tmp_path / "refusal"
    src.write_text(HEAD.split("static size_t room")[0] + "int main() {\n    hd::Refusal r;\n" + REFUSALS[name]
                   + "    return 0;\n}\n")
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", CSRC, str(src), "-o", str(exe)])
    p = subprocess.run([str(exe)], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout + p.stderr


@pytest.mark.parametrize("name", CASES)
def test_scratch(name, tmp_path):
    src, exe = tmp_path / "scratch.cpp", tmp_path / "scratch"
    src.write_text(HEAD + CASES[name] + r'''
    s.release_all();
    CHECK(live.empty() && !s.get() && !released_in_capture);
    return 0;
}
''')
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined", "-I",
                           CSRC, str(src), "-o", str(exe)])
    p = subprocess.run([str(exe)], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout + p.stderr


def test_scratch_of_tokens_that_stay_visible(heddle_lib, tmp_path):
    """Sums of parts of the gradients' key tiles stay within 0.35 GB (two of 128
    x 128 floats a part, 16 parts an SM at most, where a ceiling doubles eight)
    beside delta and dS, whatever the first tokens and lengths are."""
    from paper_2609_34244_gb300 import _build
    src, exe = tmp_path / "sizes.cu", tmp_path / "sizes"
    src.write_text(r"""
#include <cstdio>
#include "heddle_attn.cuh"
int main() {
    hd::OpContext x;
    x.num_sms = 152;
    const long long lengths[] = {1, 100, 4095, 8192, 32768, 131072};
    for (long long t : lengths)
        for (long long window : {0ll, 1ll, 256ll, 5000ll})
            for (long long sinks : {0ll, 4ll, 300ll, 4096ll, 16384ll, 100000ll})
                for (int group : {1, 4, 128})
                    for (int heads : {1, 8})
                        for (int batch : {1, 16}) {
                            heddle_attention_args a{};
                            a.batch = batch, a.q_len = a.kv_len = t;
                            a.q_heads = group * heads, a.kv_heads = heads, a.head_dim = 128;
                            a.window = window, a.sinks = sinks, a.scale = 0.1f;
                            std::printf("%lld %lld %lld %d %d %d %zu\n", t, window, sinks, group, heads, batch,
                                        hd::attn_tc_grad_scratch(x, a, false));
                        }
    return 0;
}
""")
    subprocess.check_call([_build.nvcc(), *_build.ARCH, "-std=c++17", "-I", _build.INCLUDE, "-I", CSRC, str(src), "-o",
                           str(exe), "-L", PKG, "-lheddle", "-Xlinker", "-rpath", "-Xlinker", PKG])
    sizes = [tuple(map(int, line.split())) for line in subprocess.check_output([str(exe)], text=True).splitlines()]
    assert len(sizes) == 6 * 4 * 6 * 3 * 2 * 2
    assert max(s[-1] for s in sizes) <= 0.35e9, max(sizes, key=lambda s: s[-1])
    assert any(s[-1] > 1e6 for s in sizes)
