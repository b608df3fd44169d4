"""Host memory that a blocking call reads back into (host_block.hpp) where the heap has none left, or the runtime throws: a runtime that is at work is
asked for pinned memory, one that may not be is left alone, and nothing is thrown."""
import subprocess

from paper_2510_24273_amd import build

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <new>
#include "host_block.hpp"
static bool no_heap = false, throws = false;
static int asked = 0;
void* operator new(size_t n, const std::nothrow_t&) noexcept { return no_heap ? nullptr : std::malloc(n); }
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }
struct Alloc {
    static void* pin(size_t n) { ++asked; if (throws) throw std::bad_alloc(); return std::malloc(n); }
    static void unpin(void* p) { std::free(p); }
};
typedef sals::HostBlock<Alloc, 4096, 1> Block;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main()
{
    no_heap = true;
    { Block b; CHECK(!b.p && asked == 0); }                    // nothing is known of the runtime
    { Block b(true); CHECK(b.p && asked == 1); }               // at work: there may be pinned memory (not idle: freed)
    { Block b; CHECK(b.p && asked == 2); b.idle = true; }      // it was, before
    { Block b, c; CHECK(b.p && c.p && b.p != c.p && asked == 3); }   // a kept one and a new one
    throws = true;
    { Block b(true); CHECK(!b.p && asked == 4); }
    no_heap = false;
    { Block b; CHECK(b.p && asked == 5); b.idle = true; }      // ordinary memory
    std::printf("ok\n");
}
"""


def test_blocks_without_a_heap(tmp_path):
    (tmp_path / "b.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-I", build.CSRC, "-o", str(tmp_path / "b"), str(tmp_path / "b.cpp")], check=True)
    assert subprocess.run([str(tmp_path / "b")], capture_output=True, text=True, timeout=60).stdout.strip() == "ok"
