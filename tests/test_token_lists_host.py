"""Host arrays of the token calls on the CPU: a call that is to be refused reads none of its lists past their ends.

The lists lie at the end of a page behind which no access is allowed, and the library's own checks run on them, compiled
here from its source: no device is needed up to a refusal."""
import os
import subprocess

import pytest

from paper_2607_18582_gb300 import build, mure

HEAD = r"""
#include <sys/mman.h>
#include <unistd.h>
#include <cstdio>
#include <cstring>

// n numbers, right before a page that cannot be read
static int32_t *at_the_end(std::initializer_list<int32_t> x)
{
    const size_t page = sysconf(_SC_PAGESIZE);
    char *m = static_cast<char *>(mmap(nullptr, 2 * page, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0));
    mprotect(m + page, page, PROT_NONE);
    int32_t *p = reinterpret_cast<int32_t *>(m + page) - x.size();
    memcpy(p, x.begin(), x.size() * sizeof(int32_t));
    return p;
}

static mure_tokens_desc geometry()
{
    mure_tokens_desc d{};
    d.n_kv_heads = 1; d.head_dim = 64; d.page_size = 16; d.dtype = MURE_F32; d.n_pages = 100;
    return d;
}
"""


def run(tmp_path, source, program):
    """What a program says that holds one of the library's sources."""
    src, exe = tmp_path / "lists.cu", tmp_path / "lists"
    src.write_text(f'#include "{source}"\n' + HEAD + program)
    lib, nvcc = build.build(), build._nvcc()
    r = subprocess.run([nvcc] + build.ARCH + ["-std=c++17", "-cudart", "shared", "--expt-relaxed-constexpr", "-I", build.CSRC, "-I", build.INCLUDE, "-o", str(exe),
                                              str(src), lib], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "lib64") if os.path.isabs(nvcc) else ""
    env = dict(os.environ, LD_LIBRARY_PATH=":".join(p for p in (cuda, os.path.dirname(lib), os.environ.get("LD_LIBRARY_PATH", "")) if p))
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60, env=env)
    assert r.returncode == 0, (r.returncode, r.stderr)
    return r.stdout.splitlines()


def test_parents_are_read_after_all_lengths(tmp_path):
    """Lengths of which a later one is negative name more parents than there are: the length is refused first."""
    said = run(tmp_path, "tokens.cu", r"""
int main()
{
    mure_ctx c;
    mure_tokens_plan p;
    p.ctx = &c;
    p.d = geometry();
    const int32_t sizes[][3] = {{1024, -1023, 0}, {1, 1000, -1000}, {1000, -1001, 2}};
    for (auto &s : sizes) {
        const int32_t pos[3] = {0, 0, 0}, kv[3] = {0, 0, 0};
        mure_tokens_batch b{};
        b.n_seqs = 3; b.n_heads = 1; b.new_len = s; b.pos = pos; b.kv_len = kv;
        int status = 0;
        try {
            set_plan(&p, &b, true, at_the_end({-1}));
        } catch (const Fail &f) {
            status = f.st;
        }
        printf("%d %s\n", status, c.err.c_str());
        fflush(stdout);
    }
    return 0;
}
""")
    assert said == [f"1 sequence {s}: a negative length or position" for s in (1, 2, 1)]


@pytest.mark.parametrize("new,parents", [([1024, -1023], [-1]), ([-1, 2], [-1]), ([3, -3], [])])
def test_negative_lengths_of_trees_are_refused(new, parents):
    """The binding counts the parents, so that their number says nothing where a length is negative.  (Looked at before the cache is.)"""

    class Cache:
        ctx = h = None

    with pytest.raises(ValueError):
        mure.mure_tokens_plan(Cache, 1, new, [0] * len(new), [0] * len(new), [[0]] * len(new), parents=parents)


def test_kept_indexes_are_read_after_all_counts(tmp_path):
    """Counts of which a later one cannot be name more indexes than there are: the count is refused first."""
    said = run(tmp_path, "tokens_step.cu", r"""
int main()
{
    mure_ctx c;
    mure_tokens t;
    mure_tokens_plan p;
    t.ctx = p.ctx = &c;
    t.d = p.d = geometry();
    p.ready = true;
    p.seq = {{0, 50, 0, 50, 0, 0}, {50, 50, 0, 50, 4, 50}};
    const int32_t counts[][2] = {{50, -49}, {-1, 2}, {50, -50}, {50, 51}};
    for (auto &n : counts) {
        const int status = mure_tokens_keep(&t, &p, n, at_the_end({0}));
        printf("%d %s\n", status, c.err.c_str());
        fflush(stdout);
    }
    return 0;
}
""")
    assert said == [f"1 sequence {s}: {n} kept of 50 new tokens" for s, n in ((1, -49), (0, -1), (1, -50), (1, 51))]


def test_sets_of_ids_far_apart(tmp_path):
    """Page ids that are multiples of a power of two, or any distance apart, lie few slots behind the first one that they look
    at: linear probing of a set half full looks at 1.5 slots on average if ids fall on them by chance, and 16 are
    allowed here (all on one slot, 2^15 ids look at 2^14 each)."""
    said = run(tmp_path, "tokens_host.cuh", r"""
int main()
{
    const int32_t n = 1 << 15;
    for (int32_t step : {1, 3, 1 << 4, 1 << 9, 1 << 12, 1 << 16, (1 << 16) - 1, 10007}) {
        mure::IdSet ids(n), empty(n);
        bool ok = true;
        int64_t probes = 0;
        for (int32_t i = 0; i < n; ++i) ok = ids.insert((n - 1 - i) * step) && ok;
        for (int32_t i = 0; i < n; ++i) {
            ok = ok && ids.has(i * step) && !ids.insert(i * step) && (step == 1 || !ids.has(i * step + 1));
            probes += 1 + ((ids.at(i * step) - empty.at(i * step)) & ids.mask);
        }
        printf("%d %d\n", ok, probes <= 16 * n);
    }
    mure::IdSet few(0);
    const bool first = few.insert(INT32_MAX), again = few.insert(INT32_MAX);
    printf("%d %d %d\n", first, again, few.has(0));
    return 0;
}
""")
    assert said == ["1 1"] * 8 + ["1 0 0"]
