"""The arithmetic by which the kernels of the decoder's attention block cut their work, compiled for the host with checks for overflows."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2301_01333_amd", "csrc")


def runs(tmp_path, program):
    src, exe = tmp_path / "p.cpp", tmp_path / "p"
    src.write_text(program)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-Wno-unused-function", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC,
                    str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert (out.returncode, out.stdout.strip()) == (0, "ok"), out.stdout + out.stderr


def test_splits_cover_a_sequence_once_up_to_the_longest(tmp_path):
    """Also where the last split would end beyond 2^31."""
    runs(tmp_path, r"""
#include "ogc_kv4_layout.h"
#include <stdio.h>
#include <initializer_list>
int main() {
    const int longest = 0x7fff0000;
    for (int len : {0, 1, 127, 128, 129, 4000, 98305, 1 << 30, longest - 2796288, longest - 1, longest})
        for (int chunk : {128, 256, 1408, 2796288, 1 << 30, 0x7fffffff / 512 * 512}) {
            const int n = kv4_splits_of(len, chunk);
            if (n != ((int64_t)len + chunk - 1) / chunk) return printf("%d splits of %d by %d\n", n, len, chunk), 1;
            int64_t to = 0;
            for (int i = 0; i < n; ++i) {
                const int end = kv4_split_end(len, chunk, i * chunk);
                if (to != (int64_t)i * chunk || end <= to || end > len || end - to > chunk) return printf("split %d of %d by %d ends at %d\n", i, len, chunk, end), 1;
                to = end;
            }
            if (to != len) return printf("%d by %d ends at %lld\n", len, chunk, (long long)to), 1;
        }
    if (kv4_split_end(0, 128, 0) != 0) return puts("empty"), 1;
    puts("ok");
    return 0;
}
""")
