"""The tables of tensors that the clipping kernels are launched with (built with the host compiler; needs no GPU): every element once, in order, in launches of
fewer than 2^32 threads."""
import os
import shutil
import subprocess

import pytest

from conftest import ROOT

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "grad_table.h"
using namespace abt;
// addresses that nothing is read from
char* base_of(int i, bool out) { return reinterpret_cast<char*>((uintptr_t)(2 * i + out + 1) << 44); }
int check(const std::vector<int64_t>& counts, int chunk, int limit) {
    std::vector<GradTensor> t;
    for (size_t i = 0; i < counts.size(); ++i) t.push_back(GradTensor{base_of((int)i, false), i % 3 ? base_of((int)i, true) : nullptr, counts[i], i % 2 == 1});
    std::vector<int64_t> seen(counts.size(), 0);
    GradTables tables(t.data(), (int)t.size());
    GradTable a;
    int chunks, launches = 0;
    size_t at = 0;
    while (tables.next(a, chunk, limit, chunks)) {
        if (++launches > 100000 || chunks < 1 || chunks > limit || a.n < 1 || a.n > kGradMaxTensors || a.first[0] != 0 || a.first[a.n] != chunks) return 1;
        for (int i = 0; i < a.n; ++i) {
            while (at < counts.size() && seen[at] == counts[at]) ++at;
            if (at == counts.size()) return 2;
            const int64_t size = t[at].bf16 ? 2 : 4;
            if ((((a.bf16[i >> 6] >> (i & 63)) & 1) != 0) != t[at].bf16) return 3;
            if (a.grad[i] != base_of((int)at, false) + seen[at] * size) return 4;
            if (t[at].out ? a.out[i] != base_of((int)at, true) + seen[at] * size : a.out[i] != nullptr) return 5;
            if (seen[at] % chunk) return 6;                        // (whole chunks, so that 16-byte pieces stay aligned)
            if (a.count[i] < 1 || a.first[i + 1] - a.first[i] != (a.count[i] + chunk - 1) / chunk) return 7;
            seen[at] += a.count[i];
            if (seen[at] > counts[at]) return 8;
        }
    }
    for (size_t i = 0; i < counts.size(); ++i) if (seen[i] != counts[i]) { std::printf("tensor %zu: %lld of %lld\n", i, (long long)seen[i], (long long)counts[i]); return 9; }
    return 0;
}
int main() {
    const int64_t big = 1ll << 40;
    std::vector<int64_t> many;
    for (int i = 0; i < 700; ++i) many.push_back(i % 7 * 5000);
    const std::vector<std::vector<int64_t>> sets = {{}, {0, 0}, {1}, {0, 5, 0, 4096, 4097}, {(1ll << 36) - 1}, {1ll << 36}, {(1ll << 36) + 1}, {17, 0, big, 3, (1ll << 37) + 4099}, many};
    for (size_t s = 0; s < sets.size(); ++s)
        for (int k = 0; k < 3; ++k) {
            const int chunk = k == 1 ? 16384 : 4096, limit = k == 2 ? 3 : (int)kGradMaxBlocks;
            if (k == 2 && s > 3 && s < 8) continue;
            const int r = check(sets[s], chunk, limit);
            if (r) { std::printf("set %zu chunk %d limit %d: %d\n", s, chunk, limit, r); return 1; }
        }
    return (uint64_t)kGradMaxBlocks * 256 < (1ull << 32) ? 0 : 2;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_every_element_once_and_launches_that_fit(tmp_path):
    src = tmp_path / "tables.cpp"
    src.write_text(PROGRAM)
    exe = str(tmp_path / "tables")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2405_01067_amd", "csrc"), str(src), "-o", exe], check=True)
    r = subprocess.run([exe], stdout=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stdout
