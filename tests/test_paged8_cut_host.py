"""How calls of the attention over 8-bit pages are cut, without a GPU: the walks of the raw cache's cut with the 8-bit costs, and which calls
take one launch."""
import pytest

from test_paged8_host import batch, pages
from test_paged_edges_host import BOUND, run_host
from test_paged_host import WALK


@pytest.mark.parametrize("walk", [WALK, BOUND])
def test_cut_with_these_costs(tmp_path, walk):
    """Every new token meets every key that it sees exactly once, and proper calls are done whole, with these costs too."""
    assert "costs_of(" in walk
    assert run_host(tmp_path, walk.replace("costs_of(", "costs8_of(")).strip() == "ok"


ONE_LAUNCH = r'''
#include <stdio.h>
#include <stdlib.h>
#include <algorithm>
#include <random>
#include <vector>
#include "vr_pages.h"
using namespace vr;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } } while (0)
int main() {
    std::mt19937 gen(5);
    int one = 0, two = 0;
    for (int round = 0; round < 200000; ++round) {
        const int S = 1 + (int)(gen() % 80), Hg = 1 + (int)(gen() % 40), G = 1 + (int)(gen() % 8), cap = 32 * (1 + (int)(gen() % 64));
        const int64_t T = gen() % (gen() % 4 ? 2 * S : 600);
        const Costs c = costs8_of(gen() % 2);
        const int64_t rows = max_records8(T, S, G, Hg, cap, c.lmin);
        CHECK(rows == 0 || rows == max_records(T, S, G, Hg, cap, c.lmin));
        if (max_records(T, S, G, Hg, cap, c.lmin) == 0) continue;
        // single tokens over short tables, and calls that are one tile of few rows at most
        const bool short_one = cap <= 1024 && (T <= S || T * Hg <= ROWS_FEW);
        CHECK((rows == 0) == short_one);
        ++(rows ? two : one);
    }
    CHECK(one > 1000 && two > 1000);
    printf("ok\n");
    return 0;
}
'''


def test_one_launch(tmp_path):
    """Tiles are whole, and a call one launch, where the table is short and no sequence has more than single tokens' rows on average of
    every slot; a chunk in a batch whose other slots are empty may be cut."""
    assert run_host(tmp_path, ONE_LAUNCH).strip() == "ok"


def test_chunks_among_empty_slots_may_be_cut():
    from paper_2607_15498_amd import _lib
    L = _lib.load()
    need = lambda T, S, G=1, H=4, width=16, page=64, dtype=1: L.varrate_paged8_attn_workspace_bytes(pages(G=G, page=page), batch(T=T, S=S, width=width), dtype, H)
    assert need(512, 64) > 0 and need(65, 64) > 0 and need(512, 64, dtype=0) > 0    # a chunk in one of 64 slots
    assert need(64, 64) == 0 and need(1, 1) == 0 and need(1, 64) == 0               # single tokens
    assert need(8, 1) == 0 and need(9, 1) > 0                                        # one tile of 32 rows, and more
    assert need(64, 64, width=32) > 0 and need(1, 1, width=17) > 0                   # longer tables
