"""CPU checks of the operators without a context: every refusal of the C ABI (before anything
touches a GPU: the addresses here are never read), the workspace sizes, and the binding's checks
of tensors."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2509_04185_amd as P
from paper_2509_04185_amd import binding as Bd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, NO_MEMORY, UNSUPPORTED = 1, 4, 6
A = 0x1000   # an aligned address


@pytest.fixture(scope="module")
def lib():
    return P.load_library()


def refused(lib, status, st, text):
    assert st == status
    assert text in lib.sbd_last_error(None).decode()


def table(**kw):
    f = dict(batch=2, max_pages=8, n_pages=20, page_size=16, table=A, held=A, cached=A, free_list=A, free_count=A)
    f.update(kw)
    return ctypes.byref(Bd.PageTableArgs(*[f[n] for n, _ in Bd.PageTableArgs._fields_]))


def cache(**kw):
    f = dict(n_pages=20, page_size=16, n_kv_heads=2, head_dim=64, k_codes=A, v_codes=A, k_exp=A, v_exp=A)
    f.update(kw)
    return ctypes.byref(Bd.PagedKVArgs(*[f[n] for n, _ in Bd.PagedKVArgs._fields_]))


PAGE_SIZES = [0, 8, 24, 48, 512, -16]


@pytest.mark.parametrize("kw,text", [(dict(batch=0), "batch"), (dict(batch=65537), "batch"), (dict(n_pages=0), "n_pages"),
                                     (dict(n_pages=2 ** 27), "n_pages"), (dict(max_pages=0), "max_pages"),
                                     (dict(max_pages=2 ** 26 + 1), "max_pages")]
                         + [(dict(page_size=p), "page_size") for p in PAGE_SIZES]
                         + [({f: None}, "null") for f in ("table", "held", "cached", "free_list", "free_count")])
def test_plan_refuses_tables(lib, kw, text):
    refused(lib, INVALID, lib.sbd_paged_plan(None, table(**kw), A, None, 4, A, A, A, A), text)


def test_plan_refuses_arguments(lib):
    f = lib.sbd_paged_plan
    refused(lib, INVALID, f(None, None, A, None, 4, A, A, A, A), "null page table")
    refused(lib, INVALID, f(None, table(), A, None, -1, A, A, A, A), "rows")
    refused(lib, INVALID, f(None, table(), A, None, 2 ** 24 + 1, A, A, A, A), "rows")
    for i in range(5):
        args = [A] * 5
        args[i] = None
        refused(lib, INVALID, f(None, table(), args[0], None, 4, *args[1:]), "null")


@pytest.mark.parametrize("kw,status,text", [(dict(n_pages=0), INVALID, "n_pages"), (dict(n_pages=2 ** 27), INVALID, "n_pages"),
                                            (dict(n_kv_heads=0), INVALID, "n_kv_heads"),
                                            (dict(n_kv_heads=1025), INVALID, "n_kv_heads"),
                                            (dict(head_dim=96), UNSUPPORTED, "head_dim"),
                                            (dict(k_codes=A + 8), INVALID, "aligned"), (dict(v_codes=A + 1), INVALID, "aligned")]
                         + [(dict(page_size=p), INVALID, "page_size") for p in PAGE_SIZES]
                         + [({f: None}, INVALID, "null") for f in ("k_codes", "v_codes", "k_exp", "v_exp")])
def test_cache_refusals(lib, kw, status, text):
    refused(lib, status, lib.sbd_paged_append(None, cache(**kw), 0, 2, 4, A, A, A, 128, A, 128), text)
    refused(lib, status, lib.sbd_paged_attention(None, cache(**kw), 0, 2, 4, 4, A, A, A, 8, None, 1.0, 100, A, 256, A, 256,
                                                 A, 1 << 30), text)


def test_append_refuses_arguments(lib):
    def call(dtype=0, batch=2, rows=4, starts=A, slots=A, k=A, ks=128, v=A, vs=128):
        return lib.sbd_paged_append(None, cache(), dtype, batch, rows, starts, slots, k, ks, v, vs)
    refused(lib, INVALID, lib.sbd_paged_append(None, None, 0, 2, 4, A, A, A, 128, A, 128), "null paged cache")
    for kw, text in ((dict(dtype=2), "SBD_TYPE"), (dict(dtype=-1), "SBD_TYPE"), (dict(batch=0), "batch"), (dict(rows=-1), "rows"),
                     (dict(starts=None), "null"), (dict(slots=None), "null"), (dict(k=None), "k is null"),
                     (dict(v=None), "v is null"), (dict(k=A + 2), "k must be 16-byte"), (dict(v=A + 8), "v must be 16-byte"),
                     (dict(ks=120), "stride"), (dict(ks=132), "stride"), (dict(vs=0), "stride"), (dict(vs=-128), "stride")):
        refused(lib, INVALID, call(**kw), text)
    assert call(rows=0, slots=None, k=None, v=None) == 0     # nothing to write


def test_attention_refuses_arguments(lib):
    def call(dtype=0, batch=2, rows=4, nq=4, starts=A, kv=A, tab=A, width=8, scale=1.0, max_kv=100, q=A, qs=256, out=A,
             os_=256, ws=A, nb=1 << 30):
        return lib.sbd_paged_attention(None, cache(), dtype, batch, rows, nq, starts, kv, tab, width, None, scale, max_kv, q,
                                       qs, out, os_, ws, nb)
    nan, inf = float("nan"), float("inf")
    for kw, text in ((dict(dtype=2), "SBD_TYPE"), (dict(batch=65537), "batch"), (dict(rows=-3), "rows"), (dict(nq=3), "n_q_heads"),
                     (dict(nq=0), "n_q_heads"), (dict(nq=1026), "n_q_heads"), (dict(rows=2 ** 24, nq=512), "2^31"),
                     (dict(starts=None), "null"), (dict(kv=None), "null"), (dict(tab=None), "null"), (dict(width=0), "max_pages"),
                     (dict(width=2 ** 26 + 1), "max_pages"), (dict(scale=nan), "scale"), (dict(scale=inf), "scale"),
                     (dict(max_kv=0), "max_kv"), (dict(max_kv=129), "max_kv"), (dict(q=None), "q is null"),
                     (dict(out=None), "out is null"), (dict(q=A + 4), "q must"), (dict(out=A + 8), "out must"),
                     (dict(qs=248), "stride"), (dict(os_=257), "stride")):
        refused(lib, INVALID, call(**kw), text)
    assert call(rows=0, q=None, out=None, ws=None, nb=0) == 0
    long = dict(batch=1, rows=1, nq=2, width=1000, max_kv=16000, qs=128, os_=128)   # one row over many keys: split
    refused(lib, INVALID, call(ws=None, **long), "workspace")
    refused(lib, INVALID, call(ws=A + 4, **long), "workspace")
    refused(lib, NO_MEMORY, call(nb=64, **long), "need")


def test_attention_workspace(lib):
    n = ctypes.c_size_t(123)
    f = lib.sbd_paged_attention_workspace
    assert f(cache(k_codes=None, v_codes=None, k_exp=None, v_exp=None), 1, 16, 8, 2048, ctypes.byref(n)) == 0 and n.value > 0
    first = n.value
    assert f(cache(), 1, 16, 8, 32768, ctypes.byref(n)) == 0 and first <= n.value < 1 << 28
    # many rows fill the chip without splitting the keys
    assert f(cache(), 4, 20000, 64, 8192, ctypes.byref(n)) == 0 and n.value == 0
    refused(lib, INVALID, f(cache(), 1, 16, 8, 2048, None), "null bytes")
    refused(lib, INVALID, f(None, 1, 16, 8, 2048, ctypes.byref(n)), "null paged cache")
    refused(lib, INVALID, f(cache(), 1, 16, 7, 2048, ctypes.byref(n)), "n_q_heads")


def test_quantize_refusals(lib):
    def call(dtype=0, rows=4, cols=256, x=A, stride=256, br=1, codes=A, scales=A):
        return lib.sbd_scaled_quantize(None, dtype, rows, cols, x, stride, br, codes, scales)
    for kw, text in ((dict(dtype=3), "type"), (dict(dtype=-1), "type"), (dict(rows=-1), "rows"), (dict(cols=0), "cols"),
                     (dict(cols=100), "cols"), (dict(cols=8), "cols"), (dict(rows=2 ** 20, cols=2 ** 17, stride=2 ** 17), "2^36"), (dict(br=0), "block_rows"), (dict(br=64), "block_rows"),
                     (dict(x=None), "null"), (dict(codes=None), "null"), (dict(scales=None), "null"), (dict(x=A + 2), "aligned"),
                     (dict(codes=A + 8), "aligned"), (dict(stride=240), "stride"), (dict(stride=260), "stride"),
                     (dict(dtype=2, stride=258), "stride")):
        refused(lib, INVALID, call(**kw), text)
    assert call(rows=0, x=None, codes=None, scales=None) == 0


def test_matmul_refusals(lib):
    def call(m=4, n=256, k=256, a=A, sa=256, a_s=A, b=A, b_s=A, t=0, out=A, so=256, ws=None, nb=0):
        return lib.sbd_scaled_matmul(None, m, n, k, a, sa, a_s, b, b_s, t, out, so, ws, nb)
    for kw, text in ((dict(m=-1), "m "), (dict(m=2 ** 24 + 1), "m "), (dict(n=0), "n "), (dict(k=0), "k "), (dict(k=100), "k "),
                     (dict(k=8), "k "), (dict(t=3), "type"), (dict(a=None), "null"), (dict(a_s=None), "null"),
                     (dict(b=None), "null"), (dict(b_s=None), "null"), (dict(out=None), "null"), (dict(a=A + 8), "aligned"),
                     (dict(b=A + 4), "aligned"), (dict(sa=240), "stride"), (dict(sa=264), "stride"), (dict(so=255), "stride"),
                     (dict(k=2 ** 22 + 16), "k "), (dict(sa=2 ** 22 + 16), "stride"), (dict(m=2 ** 20, n=2 ** 16 + 1), "2^36"),
                     (dict(out=A + 1), "aligned"), (dict(out=A + 2, t=2), "aligned")):
        refused(lib, INVALID, call(**kw), text)
    assert call(m=0, a=None, out=None) == 0
    n = ctypes.c_size_t()
    refused(lib, INVALID, lib.sbd_scaled_matmul_workspace(4, 4, 100, ctypes.byref(n)), "k ")
    refused(lib, INVALID, lib.sbd_scaled_matmul_workspace(4, 4, 128, None), "null bytes")
    for m, nn, k in ((1, 64, 128), (16, 1024, 14336), (300, 130, 4096), (4096, 4096, 4096)):
        assert lib.sbd_scaled_matmul_workspace(m, nn, k, ctypes.byref(n)) == 0 and n.value < 1 << 30
        if n.value:
            big = dict(m=m, n=nn, k=k, sa=k, so=nn)
            refused(lib, INVALID, call(**big), "workspace")
            refused(lib, INVALID, call(ws=A + 4, nb=n.value, **big), "workspace")
            refused(lib, NO_MEMORY, call(ws=A, nb=n.value - 1, **big), "need")


def test_binding_refuses_tensors():
    """Tensors that are not on a GPU, or of another type or shape, never reach the library."""
    i, u = torch.int32, torch.uint8
    t = torch.zeros((2, 4), dtype=i)
    with pytest.raises(ValueError, match="table: expected a CUDA tensor"):
        P.PageTable(t, t[0], t[0], t[0], t[0, :1], 16)
    with pytest.raises(ValueError, match="CUDA"):
        P.PagedStep(t, t[0], t[0], t[0], 16)
    with pytest.raises(ValueError, match="k_codes"):
        P.PagedKV(torch.zeros((2, 2, 16), dtype=u), *[torch.zeros((2, 2), dtype=torch.int8)] * 3)
    with pytest.raises(ValueError, match="CUDA"):
        P.PagedKV(torch.zeros((2, 2, 16, 64), dtype=u), torch.zeros((2, 2, 64, 16), dtype=u),
                  *[torch.zeros((2, 2), dtype=torch.int8)] * 2)
    with pytest.raises(ValueError, match="x: expected a CUDA matrix"):
        P.scaled_quantize(torch.zeros((2, 128)))
    with pytest.raises(ValueError, match="a: expected a CUDA matrix"):
        P.scaled_matmul(torch.zeros((2, 128), dtype=u), torch.zeros((1, 2)), torch.zeros((2, 128), dtype=u), torch.zeros((1, 1)))


def test_structs_match_the_header():
    import re
    src = open(os.path.join(ROOT, "include", "sbd.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    for name, cls in (("sbd_page_table", Bd.PageTableArgs), ("sbd_paged_kv", Bd.PagedKVArgs)):
        body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", src).group(1)
        fields = re.findall(r"(\w+)\s*[,;]", body)
        assert [f for f, _ in cls._fields_] == fields


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_checks_under_sanitizers(tmp_path):
    """ops_api.cpp under AddressSanitizer and UndefinedBehaviorSanitizer against host-only stand-ins
    for the launchers: every size at the ends of its range, every refusal (ops_check.cpp)."""
    csrc = os.path.join(ROOT, "paper_2509_04185_amd", "csrc")
    exe = str(tmp_path / "ops_check")
    cmd = ["g++", "-std=c++17", "-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-I", os.path.join(csrc, "host_check"), "-I", os.path.join(ROOT, "include"), "-I", csrc]
    cmd += [os.path.join(csrc, f) for f in ("ops_api.cpp", "sbd_api.cpp", "host_check/hip_stub.cpp", "host_check/ops_check.cpp")]
    subprocess.run(cmd + ["-o", exe], check=True, capture_output=True, text=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    p = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert p.returncode == 0, p.stdout + p.stderr
    assert "operator checks passed" in p.stdout and "runtime error" not in p.stderr
