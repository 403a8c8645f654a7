"""What the host code of the embedding's gradient and of distillation launches, and whether the grids and the kernels' arithmetic of indices hold there: the host code
by itself, whose launches are looked at instead of made (no GPU needed)."""
import os
import subprocess

import pytest

from paper_2605_29517_amd import build as B

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
F32, F16 = 0, 1

# The runtime's entry points that a launch goes through; look() sees the kernel's name, its grid and its arguments.
RUNTIME = r"""
#include <cstdio>
#include <cstring>
#include <map>
#include <string>
static std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> all;
    return all;
}
static dim3 grid_, block_;
static void look(const std::string &kernel, dim3 grid, dim3 block, void **args);
extern "C" {
void **__hipRegisterFatBinary(const void *)
{
    static void *any;
    return &any;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { names()[host] = name; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t)
{
    grid_ = grid;
    block_ = block;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    *grid = grid_;
    *block = block_;
    *lds = 0;
    *stream = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **args, size_t, hipStream_t)
{
    look(names()[f], grid, block, args);
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
}
"""

EMBED = r"""
#include "%(csrc)s/embed.hip"
""" + RUNTIME + r"""
using namespace maxsim;
static uint64_t looks; // at tokens, of all workgroups that sort
// Whether the quotients of all x below n are right: at the largest x of which the remainder is the largest they go wrong first.
static bool right(const Divisor &y, int64_t n)
{
    const int64_t x = n / y.d * y.d - 1;
    for (int64_t at : {x, n - 1})
        if (at >= 0 && at < (int64_t(1) << 32) && (y.m ? (int64_t)(((uint64_t)at * y.m) >> 32) : at) != at / y.d)
            return false;
    return n <= int64_t(1) << 32;
}
static bool right(const Order &o, int64_t vocab, int64_t rows) { return o.ranges == 0 || (right(o.by_ranges, ((vocab - 1) >> o.block) + 1) && right(o.by_range, rows)); }
static void look(const std::string &kernel, dim3 grid, dim3 block, void **args)
{
    const char *name = "";
    bool ok = (uint64_t)grid.x * block.x < uint64_t(1) << 32 && grid.y < 1u << 16;
    const uint64_t wgs = (uint64_t)grid.x * grid.y;
    if (kernel.find("embed_small") != std::string::npos) {
        const SortParams &s = *static_cast<SortParams *>(args[0]);
        const SumParams &p = *static_cast<SumParams *>(args[1]);
        name = "small";
        ok = ok && right(p.by_chunks, (int64_t)s.range * p.chunks) && right(p.order, p.vocab, p.rows);
    } else if (kernel.find("embed_scan") != std::string::npos) {
        const SortParams &s = *static_cast<SortParams *>(args[0]);
        name = "scan";
        looks += wgs * s.n;
        ok = ok && right(s.order, s.vocab, s.rows);
    } else if (kernel.find("embed_split") != std::string::npos || kernel.find("embed_place") != std::string::npos) {
        const SplitParams &s = *static_cast<SplitParams *>(args[0]);
        name = kernel.find("embed_split") != std::string::npos ? "split" : "place";
        looks += s.n;
        ok = ok && right(s.order, s.vocab, (int64_t)s.order.range * s.order.ranges);
    } else if (kernel.find("embed_sum") != std::string::npos) {
        const SumParams &p = *static_cast<SumParams *>(args[0]);
        name = "sum";
        ok = ok && right(p.by_chunks, (int64_t)p.per_wg * p.chunks) && right(p.by_chunks, (int64_t)p.slices_per_wg * p.chunks) && right(p.order, p.vocab, p.rows);
    } else if (kernel.find("embed_join") != std::string::npos) {
        const SumParams &p = *static_cast<SumParams *>(args[0]);
        name = "join";
        ok = ok && right(p.order, p.vocab, p.rows);
    } else {
        const LookupParams &p = *static_cast<LookupParams *>(args[0]);
        name = "lookup";
        ok = ok && right(p.by_chunks, (int64_t)p.per_wg * p.chunks);
    }
    printf("%%s %%d ", name, ok);
}
int main()
{
    static int32_t any[4];
    long n, vocab;
    int d, dtype, w_dtype, accumulate;
    while (scanf("%%ld %%ld %%d %%d %%d %%d", &n, &vocab, &d, &dtype, &w_dtype, &accumulate) == 6) {
        const hipError_t e = accumulate < 0 ? embed_launch(any, vocab, d, dtype, any, true, n, 1.0f, any, w_dtype, nullptr)
                                            : embed_backward_launch(any, dtype, any, true, n, vocab, d, 1.0f, accumulate, any, w_dtype, any, nullptr);
        printf("%%lu%%s\n", (unsigned long)looks, e == hipSuccess ? "" : " error");
        looks = 0;
    }
    return 0;
}
"""


DISTILL = r"""
#include "%(csrc)s/distill.hip"
""" + RUNTIME + r"""
using namespace maxsim;
static void look(const std::string &kernel, dim3 grid, dim3 block, void **args)
{
    const DistillParams &p = *static_cast<DistillParams *>(args[0]);
    printf("%%s %%lu %%lu %%u %%d ", kernel.find("stats") != std::string::npos ? "stats" : "rows", (unsigned long)grid.x, (unsigned long)grid.y * grid.z, block.x, p.pieces);
}
int main()
{
    static float any[4], out[4];
    long n, b;
    int k, dtype, indexed, how;
    while (scanf("%%ld %%ld %%d %%d %%d %%d", &n, &b, &k, &dtype, &indexed, &how) == 6) {
        const hipError_t e = distill_launch(any, (int)n, (int)b, b, dtype, any, dtype, indexed ? reinterpret_cast<int32_t *>(any) : nullptr, k, 1.0f, any, nullptr, how == 2 ? any : nullptr, 1.0f,
                                            how ? out : nullptr, b, any, 256, nullptr);
        printf("%%s\n", e == hipSuccess ? "" : "error");
    }
    return 0;
}
"""


def program(tmp_path_factory, name, text):
    at = tmp_path_factory.mktemp(name)
    (at / "harness.hip").write_text(text % {"csrc": B.CSRC})
    subprocess.run([HIPCC, "-std=c++17", "-O1", "--cuda-host-only", "-Wl,--unresolved-symbols=ignore-all", str(at / "harness.hip"), "-o", str(at / "harness")], check=True, stderr=subprocess.DEVNULL)

    def run(calls):
        text = "".join(" ".join(str(int(v)) for v in c) + "\n" for c in calls)
        out = subprocess.run([str(at / "harness")], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(calls)
        return [line.split() for line in out]
    return run


@pytest.fixture(scope="module")
def embed(tmp_path_factory):
    """(n, vocab, d, dtype, w_dtype, accumulate; -1: the lookup) -> kernels by name, each followed by 1 where its grid and its divisions of indices are right, and how often sorting
    workgroups look at a token."""
    return program(tmp_path_factory, "embed", EMBED)


def wrong(embed, calls):
    return [(c, r) for c, r in zip(calls, embed(calls)) if "error" in r or any(ok != "1" for ok in r[1:-1:2])]


def test_quotients_of_wide_rows(embed):
    """Added to what is there, rows of an odd number of entries are taken entry by entry: the divisor is the row's length. Every odd one, with the largest
    vocabulary of which one launch takes the gradient."""
    calls = [(40, ((256 << 20) - 1) // (w * d), d, dtype, w_dtype, 1) for w_dtype, w in ((F16, 2), (F32, 4)) for dtype in (F16, F32) for d in range(1, 65536, 2) if ((256 << 20) - 1) // (w * d) > 0]
    assert wrong(embed, calls) == []
    assert wrong(embed, [(63, 4352, 16385, F16, F16, 1), (40, 8000, 16383, F16, F16, 1), (64, 16386, 8191, F16, F16, 1), (16, 2000, 65535, F16, F16, 1)]) == []


def test_quotients(embed):
    """Few and many tokens, small and large vocabularies, narrow and wide rows, both directions."""
    calls = [(n, vocab, d, dtype, w_dtype, how) for n in (1, 60, 4000, 8192, 8193, 300_000, 20_000_000) for vocab in (1, 255, 1000, 50_001, 131_072, 524_288) for d in (1, 3, 8, 100, 1023, 8190, 65_535, 65_536)
             for dtype in (F32, F16) for w_dtype in (F32, F16) for how in (-1, 0, 1)]
    assert wrong(embed, calls) == []


def test_one_launch_for_few_tokens(embed):
    for call in ((1440, 1000, 256, F32, F32, 0), (1440, 1000, 256, F32, F32, 1), (40, 5000, 1023, F16, F16, 1), (20, 1000, 8191, F16, F16, 1)):
        assert embed([call])[0][:-1:2] == ["small"], call


def test_sorting_takes_a_bounded_time(embed):
    """Up to 2^27 - 1 tokens and 2^31 - 2 ids: what all sorting workgroups look at is a few times the tokens for every 2^19 ids."""
    calls = [(n, vocab, 1, F16, F16, how) for n in (1, 8192, 8193, 100_000, 1 << 20, 1 << 24, (1 << 24) + 1, (1 << 27) - 1) for vocab in (1, 50_001, 524_288, 524_289, 700_000, 10_000_000, 1 << 30, (1 << 31) - 2)
             for how in (0, 1)]
    assert wrong(embed, calls) == []
    for call, r in zip(calls, embed(calls)):
        n, vocab = call[:2]
        assert int(r[-1]) <= max(4 * n * -(-vocab // 524_288), 49_152 * 1024 * -(-vocab // 524_288)), (call, r)


@pytest.fixture(scope="module")
def distill(tmp_path_factory):
    """(n, b, k, dtype, whether columns are named, what: 0 the losses, 1 both, 2 the gradient) -> kernels by name, each followed by its grid's row, rows, the workgroup's threads and the
    parts of a row."""
    return program(tmp_path_factory, "distill", DISTILL)


@pytest.mark.parametrize("how", [0, 1, 2])
def test_as_many_rows_as_there_are(distill, how):
    """A row of a grid holds fewer than 2^32 threads, and the grid covers all rows: 2^31 - 1 short ones, too."""
    calls = [(n, b, min(k, b), dtype, indexed, how) for n in (1, 3, 255, 256, 5000, (1 << 22) + 1, (1 << 24) - 1, 1 << 24, (1 << 26) - 1, 1 << 26, (1 << 28) + 3, (1 << 31) - 1)
             for b, k, indexed in ((2, 2, 0), (9, 3, 1), (300, 200, 1), (1000, 1000, 0), (2100, 20, 1), (5000, 130, 1), (20_000, 7, 1), (70_000, 7, 1)) for dtype in (F32, F16) if n * b < 1 << 38]
    for call, r in zip(calls, distill(calls)):
        assert "error" not in r and len(r) in (5, 10), call
        for name, x, y, threads, pieces in zip(*(r[i::5] for i in range(5))):
            x, y, threads, pieces = int(x), int(y), int(threads), int(pieces)
            assert 0 < x * threads < 1 << 32 and y < 1 << 16, (call, name, x, y, threads)
            units = call[0] * (pieces if name == "stats" or how else 1)
            groups = -(-units // (x * y))  # of a workgroup, each with a row
            assert groups == 1 or threads // 64 >= groups, (call, name)


def test_parts_of_a_row_hold_their_sums(distill):
    """A gradient without a workspace passes every part's maximum and sum, 8 bytes, through the beginning of all parts of the row's gradient: the smallest part has room, wherever the row
    begins in 16 bytes."""
    calls = [(n, (32_768 * parts) // size + more, 1, dtype, 1, 2) for dtype, size in ((F32, 4), (F16, 2)) for n in (1, 2, 3, 7, 100, 255) for parts in (*range(1, 70), 127, 128, 511, 512, 513, 5000) for more in (0, 1, 8, 15)]
    split = 0
    for (n, b, _, dtype, *_), r in zip(calls, distill(calls)):
        pieces, v = int(r[4]), 4 if dtype == F32 else 8
        assert "error" not in r and pieces == int(r[-1])
        if pieces > 1:
            split += 1
            for head in range(v):
                every = (b - head) // v
                each = -(-every // pieces)
                assert 16 * (every - (pieces - 1) * each) >= 8 * pieces, (n, b, dtype, head)
        else:
            assert "stats" not in r
    assert split > 100
