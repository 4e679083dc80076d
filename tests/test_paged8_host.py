"""The 8-bit paged cache without a GPU: the C ABI's refusals, the struct's layout, the binding's own checks, and the host
reference's codes against torch's conversion."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, EUNSUPPORTED = 0, -1, -3
A = 1 << 20                                                # addresses are never followed, so any aligned number serves


@pytest.fixture(scope="module")
def L():
    from paper_2607_15498_amd import _lib
    return _lib.load()


def test_struct_layout_matches_header(tmp_path):
    from paper_2607_15498_amd import _lib
    names = [n for n, _ in _lib.Pages8C._fields_]
    prog = tmp_path / "probe.c"
    prog.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "varrate.h"\nint main(void) {'
                    + 'printf("%zu\\n", sizeof(varrate_pages8));'
                    + "".join(f'printf("%zu\\n", offsetof(varrate_pages8, {n}));' for n in names) + "return 0; }")
    exe = tmp_path / "probe"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(prog)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(_lib.Pages8C)] + [getattr(_lib.Pages8C, n).offset for n in names]


def pages(**kw):
    from paper_2607_15498_amd import _lib
    f = dict(k=A, v=2 * A, k_scale=9 * A + 1, v_scale=10 * A + 3, n_pages=8, G=2, d=128, page=64, reserved=0)
    f.update(kw)
    return _lib.Pages8C(*(f[n] for n, _ in _lib.Pages8C._fields_))


def batch(**kw):
    from paper_2607_15498_amd import _lib
    f = dict(table=3 * A, kv_len=4 * A, q_start=5 * A, table_stride=4, T=5, S=2, width=4)
    f.update(kw)
    return _lib.BatchC(*(f[n] for n, _ in _lib.BatchC._fields_))


def append(L, pg=None, b=None, **kw):
    f = dict(dtype=1, k=6 * A, ks=256, v=7 * A, vs=256)
    f.update(kw)
    return L.varrate_paged8_append(pg or pages(), b or batch(), f["dtype"], f["k"], f["ks"], f["v"], f["vs"], None)


def attn(L, pg=None, b=None, **kw):
    f = dict(dtype=1, q=6 * A, q_stride=4 * 128, H=4, causal=1, window=0, scale=0.1, out=7 * A, out_stride=4 * 128, lse=11 * A,
             ws=8 * A, ws_bytes=1 << 40)
    f.update(kw)
    return L.varrate_paged8_attn(pg or pages(), b or batch(), f["dtype"], f["q"], f["q_stride"], f["H"], f["causal"], f["window"],
                                 f["scale"], f["out"], f["out_stride"], f["lse"], f["ws"], f["ws_bytes"], None)


def mass(lib, pg=None, b=None, **kw):
    f = dict(dtype=1, q=6 * A, q_stride=4 * 128, H=4, causal=1, window=0, scale=0.1, lse=11 * A, mass=12 * A, out=13 * A, L=300)
    f.update(kw)
    return lib.varrate_paged8_mass(pg or pages(), b or batch(), f["dtype"], f["q"], f["q_stride"], f["H"], f["causal"], f["window"],
                                 f["scale"], f["lse"], f["mass"], f["out"], f["L"], None)


def evict(lib, pg=None, **kw):
    f = dict(table=3 * A, ts=4, width=4, kv_len=4 * A, S=2, mass=12 * A, L=256, keep=100, first=4, recent=32, into=5 * A, into_s=2,
             into_w=2, index=14 * A, mass_out=15 * A, len_out=16 * A)
    f.update(kw)
    return lib.varrate_paged8_evict(pg or pages(), *f.values(), None)


def gather(L, pg=None, **kw):
    f = dict(table=3 * A, width=4, n=100, dtype=1, K=6 * A, V=7 * A)
    f.update(kw)
    return L.varrate_paged8_gather(pg or pages(), *f.values(), None)


BAD_PAGES = [
    (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(k_scale=None), EINVAL), (dict(v_scale=None), EINVAL),
    (dict(k=A + 8), EINVAL), (dict(v=A + 2), EINVAL), (dict(n_pages=0), EINVAL), (dict(n_pages=1 << 31), EINVAL),
    (dict(n_pages=-1), EINVAL), (dict(G=0), EINVAL), (dict(G=1025), EINVAL), (dict(d=64), EUNSUPPORTED),
    (dict(page=16), EUNSUPPORTED), (dict(page=96), EUNSUPPORTED), (dict(page=512), EUNSUPPORTED), (dict(page=0), EUNSUPPORTED),
    (dict(page=-64), EUNSUPPORTED), (dict(reserved=1), EINVAL),
]
BAD_BATCHES = [
    (dict(table=None), EINVAL), (dict(kv_len=None), EINVAL), (dict(q_start=None), EINVAL), (dict(table=A + 2), EINVAL),
    (dict(kv_len=A + 1), EINVAL), (dict(q_start=A + 3), EINVAL), (dict(S=0), EINVAL), (dict(S=65537), EINVAL),
    (dict(T=-1), EINVAL), (dict(width=0), EINVAL), (dict(width=(1 << 24) + 1), EINVAL), (dict(table_stride=-1), EINVAL),
    (dict(T=1 << 30), EUNSUPPORTED), (dict(T=(1 << 63) - 1), EUNSUPPORTED),
]


@pytest.mark.parametrize("kw,code", BAD_PAGES)
def test_pages_refused(L, kw, code):
    p = pages(**kw)
    for call in (append, attn, mass, evict, gather):
        assert call(L, p) == code and L.varrate_last_error(), call.__name__
    assert L.varrate_paged8_attn_workspace_bytes(p, batch(), 1, 4) == 0


@pytest.mark.parametrize("kw,code", BAD_BATCHES)
def test_batches_refused(L, kw, code):
    b = batch(**kw)
    for call in (append, attn, mass):
        assert call(L, None, b) == code and L.varrate_last_error(), call.__name__
    assert L.varrate_paged8_attn_workspace_bytes(pages(), b, 1, 4) == 0


ROWS = [(dict(dtype=2), EINVAL), (dict(dtype=-1), EINVAL)]
QUERIES = ROWS + [
    (dict(q=None), EINVAL), (dict(q=A + 8), EINVAL), (dict(q_stride=4), EINVAL), (dict(q_stride=-512), EINVAL), (dict(H=0), EINVAL),
    (dict(H=-2), EINVAL), (dict(H=3), EUNSUPPORTED), (dict(causal=2), EINVAL), (dict(causal=-1), EINVAL), (dict(window=-1), EINVAL),
    (dict(window=(1 << 30) + 1), EINVAL), (dict(causal=0, window=5), EUNSUPPORTED), (dict(scale=0.0), EINVAL),
    (dict(scale=-1.0), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(scale=1e38), EINVAL),
    (dict(lse=A + 2), EINVAL),
]


@pytest.mark.parametrize("kw,code", ROWS + [
    (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(k=A + 8), EINVAL), (dict(v=A + 8), EINVAL), (dict(ks=100), EINVAL),
    (dict(vs=-256), EINVAL), (dict(dtype=0, ks=258), EINVAL),
])
def test_append_refused(L, kw, code):
    assert append(L, **kw) == code and L.varrate_last_error()


@pytest.mark.parametrize("kw,code", QUERIES + [
    (dict(out=None), EINVAL), (dict(out=A + 8), EINVAL), (dict(out_stride=504), EINVAL), (dict(out_stride=0), EINVAL),
    (dict(out=6 * A), EINVAL), (dict(ws=None), EINVAL), (dict(ws_bytes=16), EINVAL), (dict(ws=A + 4), EINVAL),
])
def test_attn_refused(L, kw, code):
    assert attn(L, None, batch(width=32), **kw) == code and L.varrate_last_error()    # 2048 keys: may be cut


@pytest.mark.parametrize("kw,code", QUERIES + [
    (dict(lse=None), EINVAL), (dict(mass=None), EINVAL), (dict(out=None), EINVAL), (dict(mass=A + 1), EINVAL),
    (dict(out=A + 2), EINVAL), (dict(L=0), EINVAL), (dict(L=-1), EINVAL), (dict(L=(1 << 30) + 1), EINVAL),
])
def test_mass_refused(L, kw, code):
    assert mass(L, **kw) == code and L.varrate_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), EINVAL), (dict(table=A + 2), EINVAL), (dict(into=None), EINVAL), (dict(into=A + 1), EINVAL),
    (dict(kv_len=None), EINVAL), (dict(mass=None), EINVAL), (dict(index=None), EINVAL), (dict(mass_out=None), EINVAL),
    (dict(len_out=None), EINVAL), (dict(mass_out=A + 2), EINVAL), (dict(ts=-1), EINVAL), (dict(into_s=-4), EINVAL),
    (dict(width=0), EINVAL), (dict(into_w=0), EINVAL), (dict(width=1 << 30), EINVAL), (dict(S=0), EINVAL), (dict(S=65537), EINVAL),
    (dict(L=0), EINVAL), (dict(L=1 << 31), EINVAL), (dict(keep=0), EINVAL), (dict(keep=-5), EINVAL), (dict(keep=129), EINVAL),
    (dict(keep=1 << 40), EINVAL), (dict(first=-1), EINVAL), (dict(recent=-1), EINVAL), (dict(first=101), EINVAL),
    (dict(first=70, recent=31), EINVAL), (dict(recent=(1 << 63) - 1), EINVAL), (dict(mass_out=12 * A), EINVAL),
    (dict(len_out=4 * A), EINVAL),
])
def test_evict_refused(L, kw, code):
    assert evict(L, **kw) == code and L.varrate_last_error()


@pytest.mark.parametrize("kw,code", ROWS + [
    (dict(table=None), EINVAL), (dict(table=A + 2), EINVAL), (dict(width=0), EINVAL), (dict(n=-1), EINVAL), (dict(n=257), EINVAL),
    (dict(K=None), EINVAL), (dict(V=None), EINVAL), (dict(K=A + 8), EINVAL), (dict(V=A + 8), EINVAL),
])
def test_gather_refused(L, kw, code):
    assert gather(L, **kw) == code and L.varrate_last_error()


def test_nothing_to_do(L):
    b = batch(T=0)
    assert append(L, None, b, k=None, v=None) == OK
    assert attn(L, None, b, q=None, out=None, ws=None, ws_bytes=0, lse=None) == OK
    assert gather(L, n=0, K=None, V=None) == OK
    assert L.varrate_paged8_attn_workspace_bytes(pages(), b, 1, 4) == 0


def test_binding_refuses_before_the_library(L):
    import torch
    import paper_2607_15498_amd as vr
    code = lambda *shape: torch.zeros(shape, dtype=torch.uint8).view(torch.float8_e4m3fn)
    scale = lambda *shape: torch.zeros(shape, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    k, s = code(2, 1, 32, 128), scale(2, 1, 1)
    for args in ((k, k, s, s),                             # not on a device
                 (k, k[:1], s, s), (k[0], k[0], s, s), (k, k, s[:1], s), (k, k, s, s[0]), (k.view(torch.uint8), k.view(torch.uint8), s, s),
                 (k, k, s.view(torch.uint8), s), (k, k.view(torch.float8_e5m2), s, s)):
        with pytest.raises(vr.VarRateError):
            vr.PagedCache8(*args)
    with pytest.raises(vr.VarRateError):
        vr.new_pages8(2, 1, 32, device="cpu")


def test_reference_codes():
    """The reference rounds as torch's conversion does, and its scales are the smallest."""
    import torch
    import paged8_ref as R
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    assert torch.equal(R.nearest(every[~every.isnan()]).float(), every[~every.isnan()])
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(100000, generator=gen) * torch.exp2(torch.randint(-12, 9, (100000,), generator=gen))
    fine = every[:127]
    x = torch.cat([x.clamp(-448, 448), (fine[1:] + fine[:-1]) / 2])
    assert torch.equal(R.nearest(x).float(), x.to(torch.float8_e4m3fn).float())
    for most in (0.0, 1.0, 448.0, 448.0001, 449.0, 1e-40, 3e38, 2.0 ** 100, 1.75 * 2.0 ** -90):
        y = torch.full((1, 1), most, dtype=torch.float64)
        e = int(R.exponent(y))
        assert R.E_LO <= e <= R.E_HI
        assert most <= 448 * 2.0 ** e or e == R.E_HI
        assert e == R.E_LO or most > 448 * 2.0 ** (e - 1)


# ---- the generated code of the bf16 attention: as test_paged_host.py checks the raw cache's ------------------------------

@pytest.fixture(scope="module")
def coded_kernel(tmp_path_factory):
    import re
    import shutil
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc not available")
    from paper_2607_15498_amd import build as B
    from test_paged_host import _instructions
    out = tmp_path_factory.mktemp("asm") / "paged8_attn.s"
    cmd = ["hipcc", *B.FLAGS, *B.SOURCE_FLAGS["paged8_attn.hip"], "-S", "--offload-device-only", os.path.join(B.CSRC, "paged8_attn.hip"),
           "-o", str(out)]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-2000:]
    m = re.search(r"^(_ZN2vr17paged_attn_kernelINS_5CodedIt\w*):[^\n]*\n(.*?)\n\.Lfunc_end", out.read_text(), re.S | re.M)
    return _instructions(m.group(2))


def test_accumulators_are_private(coded_kernel):
    from test_paged_host import OWN_AGPRS
    own = {f"a{i}" for i in range(OWN_AGPRS)}
    for x in coded_kernel:
        assert x.asm or not own & (x.dst | x.src), x.text
    assert own <= set().union(*(x.dst | x.src for x in coded_kernel if x.asm))


def test_products_wait_for_their_operands(coded_kernel):
    """Decoded fragments are written by vector instructions: 2 states before the product that reads them."""
    from test_paged_host import _follow, _registers
    code, products = coded_kernel, [x for x in coded_kernel if x.asm and x.mfma]
    assert len(products) >= 90
    wanted = set().union(*(_registers(x.args[1]) | _registers(x.args[2]) for x in products))
    checked = 0
    for i, w in enumerate(code):
        if w.mfma or not w.op.startswith("v_") or not w.dst & wanted:
            continue
        checked += w.op.startswith("v_cvt_scalef32")

        def visit(x, t):
            if x.asm and x.mfma:
                assert not w.dst & (_registers(x.args[1]) | _registers(x.args[2])), f"{w.text} -> {x.text} after {t}"
            return False
        _follow(code, i, 3, visit)
    assert checked >= 128


def test_results_are_read_late_enough(coded_kernel):
    from test_paged_host import _follow, _registers
    code = coded_kernel
    for i, w in enumerate(code):
        if not (w.asm and w.mfma):
            continue

        def visit(x, t):
            if x.mfma:
                if x.asm and _registers(x.args[0]) == w.dst and _registers(x.args[3]) in (w.dst, set()):
                    return True
                hit = w.dst & (_registers(x.args[1]) | _registers(x.args[2]))
            else:
                hit = w.dst & (x.src | x.dst)
            assert not hit, f"{w.text} -> {x.text} after {t}"
            return False
        _follow(code, i, 12, visit)
