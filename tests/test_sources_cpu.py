"""Rules of the CUDA sources that no run would show to be broken."""
import glob
import os
import re
import shutil
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2503_03588_b200", "csrc")


def test_no_read_only_loads():
    """The kernels may start while the kernel that writes their inputs still runs, so nothing may be read by the loads
    that are for data unchanged over a kernel's whole life (they are not ordered by the wait for that kernel)."""
    for path in glob.glob(os.path.join(CSRC, "*.cu*")):
        code = re.sub(r"//[^\n]*", "", open(path).read())
        assert not re.search(r"__ldg\b|ld\.global(\.\w+)*\.nc|__restrict__", code), path


def test_a_wait_behind_a_wait_is_as_long_as_the_row(tmp_path):
    """A CTA of kv4_cluster_kernel whose wait ran out stays for its peers' stores: long enough for a wait for each block of a
    peer's share, and no longer than a few of these, whatever the table's rows hold."""
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    source, program = tmp_path / "wait.cpp", tmp_path / "wait"
    source.write_text('#include "kv4.cuh"\n#include <stdio.h>\n#include <stdlib.h>\n'
                      "int main(int n, char **x) { for (int i = 1; i + 2 < n; i += 3) "
                      'printf("%lld\\n", pa::kv4_outlast_cycles(atoll(x[i]), atoi(x[i + 1]), atoi(x[i + 2]))); }\n')
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, "-I", os.path.join(os.path.dirname(os.path.dirname(CSRC)), "include"),
                    "-isystem", os.path.join(os.path.dirname(os.path.dirname(nvcc)), "include"), "-o", str(program), str(source)], check=True)
    cases = [(limit, n, r) for limit in (1, 2 * 10 ** 9) for n in (0, 1, 20, 45, 8216) for r in range(1, 9)]
    out = subprocess.run([str(program)] + [str(x) for c in cases for x in c], check=True, capture_output=True, text=True).stdout.split()
    for (limit, n, r), cycles in zip(cases, map(int, out)):
        blocks = -(-n // r)
        assert (blocks + 1) * limit < cycles <= (blocks + 2) * (limit + 2 * 10 ** 6), (limit, n, r, cycles)
    kernel = re.search(r"kv4_cluster_kernel\(const Kv4Args a\)\n\{.*?\n\}\n", open(os.path.join(CSRC, "kv4_decode.cu")).read(), re.S).group(0)
    limits = re.findall(r"\bmost = ([^;]*);", kernel)
    assert limits == ["kv4_outlast_cycles(a.wait_cycles, n, R)"], limits   # n: blocks of this row's list
