"""Paged cache at the edges of its ranges, without a GPU."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

BOUND = r'''
#include <stdio.h>
#include <stdlib.h>
#include <algorithm>
#include <random>
#include <vector>
#include "vr_pages.h"
using namespace vr;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } } while (0)

static int64_t tiles_of(const std::vector<int32_t>& start, int T, int G, int Hg) {
    Sums s;
    for (size_t i = 0; i + 1 < start.size(); ++i) sum_up(s, seq_range(start[i], start[i + 1], 1000, T, 4096), G, Hg, 1, 0, costs_of(true));
    return s.units;
}
int main() {
    std::mt19937 gen(3);
    for (int round = 0; round < 2000; ++round) {
        const int S = 1 + (int)(gen() % 300), T = (int)(gen() % 5000), G = 1 + (int)(gen() % 8), Hg = 1 + (int)(gen() % 300);
        const int64_t most = max_units(T, S, G, Hg);
        std::vector<int32_t> start(S + 1);
        for (int& x : start) x = (int32_t)(gen() % (T + 1));
        const int64_t any = tiles_of(start, T, G, Hg);
        CHECK(units_of(any, most) <= most);
        std::sort(start.begin(), start.end());
        const int64_t rising = tiles_of(start, T, G, Hg);
        CHECK(units_of(rising, most) == rising);           // nothing of a proper call is left out
    }
    // 0, T, 0, T, ..: every second sequence has all rows
    std::vector<int32_t> start(65537);
    for (size_t i = 0; i < start.size(); ++i) start[i] = i & 1 ? 1 << 20 : 0;
    const int64_t all = tiles_of(start, 1 << 20, 8, 4), most = max_units(1 << 20, 65536, 8, 4);
    CHECK(all > 1000 * most && units_of(all, most) == 0);
    printf("ok\n");
    return 0;
}
'''


def run_host(tmp_path, source):
    from paper_2607_15498_amd import build as B
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(source)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-Wall", "-I", B.CSRC,
                    str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:]
    return r.stdout


def test_work_of_falling_starts_is_bounded(tmp_path):
    """Starts that rise have max_units tiles at most; of more, which only starts that fall have, none are computed."""
    assert run_host(tmp_path, BOUND).strip() == "ok"


# ---- the binding, on handles of host tensors (a call that gets as far as its launch fails otherwise) -----------------

@pytest.fixture
def host(monkeypatch):
    """(binding, pages, batch, q): handles that no device is needed for, and a launch that is never to be reached."""
    import torch
    import paper_2607_15498_amd as vr
    from paper_2607_15498_amd import _lib

    def launched(*args):
        raise AssertionError("launched")
    monkeypatch.setattr(vr, "_launch", launched)
    monkeypatch.setattr(vr, "_i32", lambda t, dim, name: t.data_ptr())
    kv = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    pages = vr.PagedCache.__new__(vr.PagedCache)
    pages._k, pages._v, pages.page, pages.G = kv, kv.clone(), 16, 2
    pages._c = _lib.PagesC(pages._k.data_ptr(), pages._v.data_ptr(), 4, 2, 128, 16, _lib.VARRATE_BF16)
    batch = vr.PagedBatch(torch.zeros((1, 4), dtype=torch.int32), torch.ones(1, dtype=torch.int32), torch.tensor([0, 1], dtype=torch.int32))
    return vr, pages, batch, torch.zeros((1, 4, 128), dtype=torch.bfloat16)


@pytest.mark.parametrize("window", [1 << 32, (1 << 32) + 5, -(1 << 32), 1 << 31, 1 << 70, 2.5])
def test_numbers_beyond_32_bits_raise(host, window):
    """A window of 2^32 + 5 is not one of 5."""
    vr, pages, batch, q = host
    with pytest.raises(vr.VarRateError):
        vr.paged_attn(pages, batch, q, window=window)
    for fine in (0, 5, 5.0, True):
        with pytest.raises(AssertionError, match="launched"):
            vr.paged_attn(pages, batch, q, window=fine)


def test_sizes_beyond_32_bits_raise(host):
    import torch
    vr, pages, batch, _ = host
    far = lambda n: torch.zeros(1, dtype=torch.int32).expand(n)            # no memory: one entry, read again and again
    S = (1 << 32) + 1
    with pytest.raises(vr.VarRateError):
        vr.PagedBatch(far(4).expand(S, 4), far(S), far(S + 1))
    with pytest.raises(vr.VarRateError):
        vr.PagedBatch(far(S)[None], far(1), far(2))
    with pytest.raises(vr.VarRateError):
        vr.paged_gather(pages, far(S), 3)


def test_import_needs_no_stream_handles():
    """The package imports, and the codec's part of it is there, with a torch that has no raw stream handles; they are asked for
    by the calls that use them."""
    code = ("import torch\n"
            "if hasattr(torch._C, '_cuda_getCurrentRawStream'): del torch._C._cuda_getCurrentRawStream\n"
            "import paper_2607_15498_amd as vr\n"
            "vr.library(); vr.Shape(n=64, G=1, H=2, w=32, r_min=16, kappa_pct=100).c()\n"
            "class S: cuda_stream = 7\n"
            "torch.cuda.current_stream = lambda i: S\n"
            "assert vr._raw_stream(0) == 7\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-2000:]


def test_tensors_of_no_dimension_raise(host):
    """A scalar tensor in the place of rows is refused as any other wrong shape."""
    import torch
    vr, pages, batch, q = host
    dot = torch.zeros((), dtype=torch.bfloat16)
    k = torch.zeros((1, 2, 128), dtype=torch.bfloat16)
    for call in (lambda: vr.paged_append(pages, batch, dot, k), lambda: vr.paged_append(pages, batch, k, dot),
                 lambda: vr.paged_attn(pages, batch, dot), lambda: vr.paged_attn(pages, batch, q, out=dot),
                 lambda: vr.paged_gather(pages, batch.table[0], 3, K=dot)):
        with pytest.raises(vr.VarRateError):
            call()


# ---- how the calls of paged_shapes.py are shared out -----------------------------------------------------------------

SPLIT = r'''
#include <stdio.h>
#include <stdlib.h>
#include "vr_pages.h"
using namespace vr;
int main(int, char** v) {                                  // bf16 G Hg causal window cap S, then the new and all tokens of each
    const int bf = atoi(v[1]), G = atoi(v[2]), Hg = atoi(v[3]), causal = atoi(v[4]), window = atoi(v[5]), cap = atoi(v[6]), S = atoi(v[7]);
    int T = 0, at = 0;
    for (int i = 0; i < S; ++i) T += atoi(v[8 + 2 * i]);
    const Costs c = costs_of(bf);
    Sums s;
    for (int i = 0; i < S; at += atoi(v[8 + 2 * i++])) sum_up(s, seq_range(at, at + atoi(v[8 + 2 * i]), atoi(v[9 + 2 * i]), T, cap), G, Hg, causal, window, c);
    const int n = max_groups(T, S, G, Hg, cap, c.lmin);
    const Split p = split_of(s, n, c);
    const double share = p.among ? s.total / p.among : 0;
    printf("%d %d %lld %d\n", p.among, p.same, (long long)((s.units + n - 1) / n), (int)((share - c.piece_many) / c.many));
    return 0;
}
'''


@pytest.fixture(scope="module")
def split_program(tmp_path_factory):
    from paper_2607_15498_amd import build as B
    d = tmp_path_factory.mktemp("split")
    (d / "split.cpp").write_text(SPLIT)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", B.CSRC, str(d / "split.cpp"), "-o", str(d / "split")], check=True)
    return str(d / "split")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("i", range(7))
def test_shapes_are_shared_out_as_named(split_program, dtype, i):
    from paged_shapes import SHAPES
    assert len(SHAPES) == 7
    s = SHAPES[i]
    args = [int(dtype == "bf16"), s.G, s.H // s.G, int(s.causal), s.window, s.width * s.page, len(s.q_len)]
    args += [x for pair in zip(s.q_len, s.kv_len) for x in pair]
    among, same, rounds, keys = map(int, subprocess.run([split_program, *map(str, args)], stdout=subprocess.PIPE, text=True, check=True).stdout.split())
    how, least = s.how[dtype]
    if how == "whole":
        assert among == 0 and rounds == least, s.name
    else:
        assert among > 0 and same == 0 and keys >= least, s.name
