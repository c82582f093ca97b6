"""The memory that the calls of a layer share (csrc/arena.h), without a GPU: what a recorded launch was given stays allocated while the arena
lives, what no recorded launch has is given back when it is outgrown, and everything is given back once at the end."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cassert>
#include <cstdio>
#include <cstdlib>
#include <set>

#include "arena.h"

static std::set<char *> live;
static bool full = false;
static char *take(int64_t n) {
    if (full) return nullptr;
    char *p = static_cast<char *>(std::malloc(static_cast<size_t>(n)));
    live.insert(p);
    return p;
}
static void give(char *p) {
    assert(live.erase(p) == 1);
    std::free(p);
}

int main() {
    mqg::Arena a;
    assert(a.grow(100, take, give) && a.bytes == 100 && live.count(a.data));
    assert(a.grow(200, take, give) && a.bytes == 200 && live.size() == 1);         // nobody has the first
    a.recorded = true;
    char *first = a.data;
    assert(a.grow(300, take, give) && a.data != first && live.count(first) && live.size() == 2);
    assert(!a.recorded);                                                         // nobody has the new one yet
    char *between = a.data;
    assert(a.grow(400, take, give) && live.count(first) && !live.count(between) && live.size() == 2);
    a.recorded = true;
    char *second = a.data;
    full = true;                                                                 // no memory: the recorded ones stay, the arena is empty
    assert(!a.grow(500, take, give) && !a.data && a.bytes == 0 && live.count(first) && live.count(second));
    full = false;
    assert(a.grow(50, take, give) && a.bytes == 50 && live.size() == 3);
    a.end(give);
    assert(live.empty() && !a.data && a.bytes == 0 && a.kept.empty());
    a.end(give);
    std::puts("ok");
}
"""


def test_recorded_memory_is_kept(tmp_path):
    src, exe = tmp_path / "arena.cpp", tmp_path / "arena"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2601_04707_amd", "csrc"), "-o", str(exe), str(src)])
    assert subprocess.check_output([str(exe)], text=True).strip() == "ok"
