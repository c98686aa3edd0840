"""The table that keeps tensor maps, compiled alone: values belong to their keys whatever is pushed out, a stack of layers fits."""
import os
import subprocess


ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cassert>
#include <cstdio>
#include <thread>
#include "tmap_table.cuh"
using namespace laga;
struct Key {
    uint64_t base, rows; uint32_t box;
    bool operator==(const Key& o) const { return base == o.base && rows == o.rows && box == o.box; }
    uint64_t hash() const { return hash_add(hash_add(hash_add(0, base), rows), box); }
};
struct Value { uint64_t of[16]; };
static bool fill(const Key& k, Value* v) { for (auto& x : v->of) x = k.base + 3 * k.rows + 5 * k.box; return true; }
static bool right(const Key& k, const Value& v) { for (auto x : v.of) if (x != k.base + 3 * k.rows + 5 * k.box) return false; return true; }
template <class Table> static int misses(Table& t, int layers, int maps) {
    int made = 0;
    for (uint64_t l = 0; l < (uint64_t)layers; ++l)
        for (uint64_t m = 0; m < (uint64_t)maps; ++m) {      // tensors a few MB apart, several maps on one base
            const Key k{0x7f0000000000ull + l * (37ull << 20) + (m / 2) * (4ull << 20), 576 + 64 * (m % 3), (uint32_t)(16 << (m % 4))};
            Value v;
            assert(t.get(k, &v, [&](Value* p) { ++made; return fill(k, p); }) && right(k, v));
        }
    return made;
}
static MapTable<Key, Value, 256, 8> big;
static MapTable<Key, Value, 1, 2> tiny;
int main() {
    assert(misses(big, 61, 16) == 61 * 16);
    const int again = misses(big, 61, 16);
    printf("again %d of %d\n", again, 61 * 16);
    assert(again <= 61 * 16 / 20);
    assert(misses(tiny, 3, 4) > 0 && misses(tiny, 3, 4) == 12 && misses(tiny, 1, 2) == 2 && misses(tiny, 1, 2) == 0);
    Value v;
    const Key bad{1, 2, 3};
    assert(!tiny.get(bad, &v, [](Value*) { return false; }));
    assert(tiny.get(bad, &v, [&](Value* p) { return fill(bad, p); }) && right(bad, v));      // a failure is not kept
    std::thread a([] { for (int i = 0; i < 200; ++i) misses(tiny, 5, 4); }), b([] { for (int i = 0; i < 200; ++i) misses(tiny, 7, 4); });
    a.join(); b.join();
    puts("ok");
}
"""


def test_table_of_maps(tmp_path):
    source, binary = tmp_path / "t.cpp", tmp_path / "t"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-Wall", "-Werror", f"-I{os.path.join(ROOT, 'paper_2607_17644_b200', 'csrc')}", str(source), "-o", str(binary)],
                   check=True)
    out = subprocess.run([str(binary)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout.endswith("ok\n"), out.stdout + out.stderr
