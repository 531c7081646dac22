"""The barriers of the prompt attention kernel, without a GPU: the kernel's own initialisation is compiled for the host, with a
stand-in that records what it does.  Every barrier is initialised once (on one that is valid already it would be undefined), lies
on its own 8 bytes, and meets neither the tensor-memory slot nor the exponents of the decoding warps."""
import os
import re
import subprocess

import pytest

SOURCE = os.path.join(os.path.dirname(__file__), "..", "paper_2412_01034_b200", "csrc", "attn_many.cu")

PROGRAM = """
#include <cstdint>
#include <cstdio>
static unsigned char smem_bytes[4096];
static uint32_t smem_u32(const void* p) { return (uint32_t)(static_cast<const unsigned char*>(p) - smem_bytes); }
static void mbar_init(uint32_t bar, uint32_t count) { std::printf("%%u:%%u ", bar, count); }
struct Shape { static constexpr int kBars = 0; };
template <int kBits, int kStages>
static void barriers() {
    unsigned char* smem = smem_bytes;
    const int tid = 0;
    %s
    }
    (void)raw_free;
    std::printf("slot:%%u exponents:%%u\\n", smem_u32(tmem_slot), smem_u32(exponents));
}
int main() {
    barriers<16, 2>(); barriers<16, 4>(); barriers<8, 2>(); barriers<8, 4>(); barriers<4, 2>(); barriers<4, 4>();
}
"""


@pytest.fixture(scope="module")
def lines(tmp_path_factory):
    with open(SOURCE) as f:
        block = re.search(r"uint64_t\* bars = .*?(?=asm volatile\(\"fence\.mbarrier_init)", f.read(), re.S).group(0)
    here = tmp_path_factory.mktemp("barriers")
    (here / "b.cpp").write_text(PROGRAM % block)
    subprocess.run(["g++", "-std=c++17", "-O0", "-o", str(here / "b"), str(here / "b.cpp")], check=True)
    return subprocess.run([str(here / "b")], check=True, capture_output=True, text=True).stdout.splitlines()


@pytest.mark.parametrize("at,bits,stages", [(0, 16, 2), (1, 16, 4), (2, 8, 2), (3, 8, 4), (4, 4, 2), (5, 4, 4)])
def test_every_barrier_is_initialised_once(lines, at, bits, stages):
    made = [tuple(part.split(":")) for part in lines[at].split()]
    places = {name: int(v) for name, v in made if not name.isdigit()}
    bars = [int(name) for name, _ in made if name.isdigit()]
    assert len(bars) == len(set(bars)), f"initialised more than once: {sorted(b for b in set(bars) if bars.count(b) > 1)}"
    assert all(b % 8 == 0 for b in bars) and max(bars) + 8 <= (256 if bits == 16 else 512)
    # S, Q, O and two halves of P for two row tiles; the cleared V and the end; K, V and free for each stage
    assert len(bars) == 10 + 2 + 3 * stages + (0 if bits == 16 else 2 + 2 + 2 + 1)
    taken = {b + i for b in bars for i in range(8)}
    assert not taken & set(range(places["slot"], places["slot"] + 4))
    if bits != 16:
        assert not taken & set(range(places["exponents"], places["exponents"] + 4 * 10))
        assert places["exponents"] + 4 * 10 <= 512
