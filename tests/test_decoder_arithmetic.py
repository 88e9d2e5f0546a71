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


def test_tiles_by_how_far_they_reach(tmp_path):
    """Against a count where there are few; and where there are more queries than keys by far, fewer tiles from level to level, and none twice."""
    runs(tmp_path, r"""
#include "ogc_prompt_tiles.h"
#include <stdio.h>
#include <initializer_list>
int main() {
    for (int n : {0, 1, 5, 33, 200})
        for (int m : {0, 1, 4, 64, 65, 300, 1000})
            for (int group : {1, 3, 8})
                for (int rows : {32, 128})
                    for (int causal : {0, 1})
                        for (int max_k : {0, 64, 1000, 0x7fff0000}) {
                            const int keys = prompt_level_keys(max_k, 1000), off = m - n;
                            for (int level = 0; level <= PROMPT_LEVELS; ++level) {
                                int count = 0;
                                for (int t = 0; t * rows < n * group; ++t) {
                                    const int last = t * rows + rows < n * group ? t * rows + rows - 1 : n * group - 1;
                                    const int reach = causal ? last / group + off : m - 1;
                                    count += level == 0 || (level < PROMPT_LEVELS && reach >= level * keys);
                                }
                                const int got = prompt_tiles_from(n, m, off, group, causal, level, keys, rows);
                                if (got != count) return printf("%d queries, %d keys, group %d: %d tiles from level %d, not %d\n", n, m, group, got, level, count), 1;
                            }
                        }
    for (int n : {1 << 20, 1 << 30, 0x7fff0000 - 100})
        for (int m : {0, 100, 1 << 20})
            for (int whole : {n, 0x7fff0000})  // of queries: those beyond the announced longest are left out
                for (int keys : {prompt_level_keys(0x7fff0000, m), prompt_level_keys(0x7fff0000, 0x7fff0000)}) {
                    int last = prompt_tiles_from(n, m, m - whole, 1, 1, 0, keys, 128);
                    if (last != (n + 127) / 128) return puts("all"), 1;
                    for (int level = 1; level <= PROMPT_LEVELS; ++level) {
                        const int got = prompt_tiles_from(n, m, m - whole, 1, 1, level, keys, 128);
                        const int64_t first = (int64_t)level * keys - (m - whole), want = level == PROMPT_LEVELS || first >= n ? 0 : first <= 0 ? last : (n + 127) / 128 - first / 128;
                        if (got > last || got != want) return printf("%d queries, %d keys: %d tiles from level %d after %d\n", n, m, got, level, last), 1;
                        last = got;
                    }
                }
    if (prompt_level_keys(0x7fff0000, 640) != 11 || prompt_level_keys(640, 0x7fff0000) != 11) return puts("levels"), 1;
    puts("ok");
    return 0;
}
""")
