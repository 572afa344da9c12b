"""How the requests of a step are shared among a workgroup's threads (csrc/shares.h), on the host: every request is
some thread's at every number of requests that the entry points take, the largest ones among them, where the number
of requests rounded up to whole shares no longer is a 32-bit number with a sign."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHECK = r"""
#include <cstdio>
#include <initializer_list>
#include "shares.h"

// thread i takes items i * share .. (i + 1) * share, cut at n
template <uint32_t THREADS> bool covers(int32_t n) {
    const int64_t share = craft::share_of<THREADS>(n);
    return share >= 0 && share * THREADS >= n && (share - 1) * THREADS < n;
}

int main() {
    const int64_t most = 0x7fffffff;
    int bad = 0;
    for (int64_t back = 0; back <= 3000; ++back)
        for (int64_t n : {back, most - back, most / 2 + back, most / 2 - back})
            if (!covers<256>((int32_t)n) || !covers<1024>((int32_t)n)) {
                if (++bad <= 5) std::printf("%lld requests: shares of %d and %d\n", (long long)n, craft::share_of<256>((int32_t)n), craft::share_of<1024>((int32_t)n));
            }
    return bad ? 1 : 0;
}
"""


def test_every_request_is_some_threads(tmp_path):
    (tmp_path / "check.cpp").write_text(CHECK)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I",
                           os.path.join(ROOT, "paper_2603_28768_amd", "csrc"), str(tmp_path / "check.cpp"), "-o", str(tmp_path / "check")])
    res = subprocess.run([str(tmp_path / "check")], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
