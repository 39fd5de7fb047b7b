"""How a batch of drafted tokens is cut into chunks of cached tokens: the host
and device function of the library's internal header, compiled by the host
compiler and run on the CPU, at every size that a call may have."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2504_16083_amd", "csrc", "cache.hpp")
MOST = 1 << 30                   # cached tokens of a sequence


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    """cut([(Hkv, target, [(sequences, tiles, tokens)])]) -> [(chunk, items, cut)]: the chunk length of each batch,
    the items it makes (-1 where the length is not positive) and those of sequences that are cut."""
    if not shutil.which("g++") or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("no host compiler or HIP headers")
    d = tmp_path_factory.mktemp("cut")
    src, exe = str(d / "t.cpp"), str(d / "t")
    with open(src, "w") as f:
        f.write(f'''#include "{HEADER}"
#include <cstdio>
#include <vector>
int main() {{
  long long Hkv, target, n;
  while (scanf("%lld %lld %lld", &Hkv, &target, &n) == 3) {{
    std::vector<long long> k(n), tiles(n), L(n);
    long long work = 0, all = 0;
    for (int i = 0; i < n; ++i) {{
      if (scanf("%lld %lld %lld", &k[i], &tiles[i], &L[i]) != 3) return 1;
      work += k[i] * tiles[i] * L[i];
      all += k[i] * tiles[i];
    }}
    auto count = [&](int chunk) {{
      long long s = 0;
      for (int i = 0; i < n && chunk > 0; ++i) s += k[i] * tiles[i] * mmi::chunks_of((int)L[i], chunk);
      return s;
    }};
    const int chunk = mmi::choose_chunk(work, all, (int)Hkv, (int)target, count);
    long long cut = 0;
    for (int i = 0; i < n && chunk > 0; ++i)
      if (L[i] > chunk) cut += k[i] * tiles[i] * mmi::chunks_of((int)L[i], chunk);
    printf("%d %lld %lld\\n", chunk, chunk > 0 ? count(chunk) * Hkv : -1, cut * Hkv);
  }}
}}
''')
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", src, "-o", exe], check=True, capture_output=True, text=True)

    def go(batches):
        text = "\n".join(f"{h} {t} {len(s)} " + " ".join("%d %d %d" % x for x in s) for h, t, s in batches)
        r = subprocess.run([exe], input=text, check=True, capture_output=True, text=True, timeout=60)
        got = [tuple(int(x) for x in line.split()) for line in r.stdout.splitlines()]
        assert len(got) == len(batches)
        return got
    return go


def holds(batches, got):
    for (Hkv, target, seqs), (chunk, items, cut) in zip(batches, got):
        what = (Hkv, target, seqs, chunk, items, cut)
        units = Hkv * sum(n * t for n, t, _ in seqs)
        work = Hkv * sum(n * t * L for n, t, L in seqs)
        assert chunk > 0 and chunk % 128 == 0, what
        assert chunk <= MOST, what
        assert items <= units + target, what                     # a workgroup each is launched
        if units < target:
            assert items <= target, what                         # they all start together
        assert items >= units, what
        assert cut < 2 * target, what                            # partials of cut sequences
        if units + work // 128 < target:
            assert chunk == 128, what


@pytest.mark.parametrize("Hkv,target,tiles,L", [(1, 256, 255, 8500000), (4, 256, 63, 35000000), (1, 256, 255, MOST),
                                                (1, 512, 511, MOST), (1, 768, 767, MOST), (1024, 256, 1, MOST),
                                                (1, 256, 1, MOST), (1, 256, 128, MOST), (255, 256, 1, MOST)])
def test_longest_sequences(cut, Hkv, target, tiles, L):
    """One sequence of this many tiles, and as many sequences of one tile each: up to one unit of work less than
    workgroups, where the rest of them would be given all of it."""
    batches = [(Hkv, target, [(1, tiles, L)]), (Hkv, target, [(tiles, 1, L)]), (Hkv, target, [(tiles, 1, L), (1, 1, 0)])]
    holds(batches, cut(batches))


def test_batches_of_every_size(cut):
    rng = random.Random(0)
    batches = []
    for _ in range(3000):
        target = rng.choice([8, 64, 256, 512, 768])
        Hkv = rng.choice([1, 1, 2, 4, 8, 64, 1024])
        top = rng.choice([1, 200, 5000, 1 << 20, MOST])
        seqs = [(rng.choice([1, 1, 2, 63, 500]), rng.choice([0, 1, 1, 2, 7, 300]), int(top ** rng.random()) if rng.random() < 0.9 else rng.choice([0, top]))
                for _ in range(rng.randint(1, 5))]
        batches.append((Hkv, target, seqs))
    holds(batches, cut(batches))
