"""The serving operators' entry points where no GPU is needed: what the header declares is exported, and arguments that do not fit are refused before
anything is launched."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2604_12452_amd import lca, serve

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000            # an address that nothing reads


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lca.LIB_PATH):
        from paper_2604_12452_amd import build
        build.build(verbose=False)
    return serve.load()


def _declared():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lca_serve.h")).read(), flags=re.S)
    return re.findall(r"\blca_status\s+(\w+)\s*\(", text)


def test_every_declared_symbol_is_exported(lib, tmp_path):
    assert sorted(_declared()) == sorted(serve.EXPORTS)
    src = tmp_path / "use.c"
    src.write_text('#include "lca_serve.h"\nvoid *table[] = {' + ", ".join(f"(void *){n}" for n in _declared()) + "};\n"
                   "int main(void) { lca_serve_desc d; (void)d; return sizeof(table) + sizeof(lca_serve_desc) ? 0 : 1; }\n")
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-Wno-pedantic", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(tmp_path / "use.o")], check=True)


def test_the_descriptor_is_laid_out_as_the_header_says(tmp_path):
    src = tmp_path / "size.c"
    fields = [n for n, _ in serve._CDesc._fields_]
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "lca_serve.h"\nint main(void) {' +
                   "".join(f'printf("%zu ", offsetof(lca_serve_desc, {f}));' for f in fields) + 'printf("%zu\\n", sizeof(lca_serve_desc)); return 0; }\n')
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "size")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "size")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(serve._CDesc, f).offset for f in fields] + [ctypes.sizeof(serve._CDesc)]


def _desc(**kw):
    return serve.Desc(**{**dict(B=2, T=40, H=8, S=2, d_pool=64, d_sel=64, page=16, n_blocks=20, max_blocks=8), **kw})


ANY = [dict(B=0), dict(B=-1), dict(T=-1), dict(H=0), dict(S=0), dict(S=3), dict(dtype=3), dict(dtype=-1), dict(d_pool=0), dict(d_sel=12), dict(d_pool=1032), dict(window=-1),
       dict(scale=float("nan")), dict(scale=float("inf")), dict(softcap=float("nan")), dict(softcap=-1.0), dict(softcap=float("inf")), dict(softcap=1e-40), dict(softcap=3e38, dtype=lca.F32), dict(scale=3e38), dict(softcap=1025.0),
       dict(softcap=1025.0, dtype=lca.F16), dict(max_q=-1), dict(max_kv=-2),
       dict(T=1 << 28, H=8), dict(B=1 << 24), dict(q_row=8), dict(q_row=8 * 64 + 4), dict(sel_row=120), dict(pool_row=-128), dict(pool_row=1 << 33)]
PAGES = [dict(page=0), dict(page=8), dict(page=24), dict(page=2048), dict(n_blocks=0), dict(n_blocks=1 << 27), dict(max_blocks=0), dict(max_blocks=(1 << 26) + 1)]
CACHE = [dict(dtype=lca.F32), dict(d_pool=72), dict(d_sel=264), dict(d_sel=512)]


def _calls(lib, d):
    cd, ws = ctypes.byref(serve._c_desc(*d._key())), (A, 1 << 40)
    return {"tables": lambda: lib.lca_page_tables(cd, *[A] * 11, *ws, 0), "release": lambda: lib.lca_page_release(cd, *[A] * 5, 0),
            "store": lambda: lib.lca_page_store_q8(cd, *[A] * 6, 0), "paged": lambda: lib.lca_page_attn_q8(cd, *[A] * 11, *ws, 0),
            "packed": lambda: lib.lca_packed_attn(cd, *[A] * 8, *ws, 0)}


@pytest.mark.parametrize("kw", ANY + PAGES + CACHE, ids=str)
def test_descriptors_that_do_not_fit(lib, kw):
    hit = ("tables", "release", "store", "paged", "packed") if kw in ANY else ("tables", "release", "store", "paged") if kw in PAGES else ("store", "paged")
    for name in hit:
        assert _calls(lib, _desc(**kw))[name]() in (lca.ERR_INVALID_ARG, lca.ERR_UNSUPPORTED), (name, kw)
        assert lib.lca_last_error()
    if kw in ANY:
        with pytest.raises(lca.LcaError):
            serve.workspace_size(_desc(**kw))


@pytest.mark.parametrize("name,pointers,optional", [("lca_page_tables", 11, ()), ("lca_page_release", 5, ()), ("lca_page_store_q8", 6, ()), ("lca_page_attn_q8", 11, (3, 4, 10)),
                                                    ("lca_packed_attn", 8, (4, 5, 7))])
def test_pointers_that_are_missing_or_not_aligned(lib, name, pointers, optional):
    d = _desc()
    cd = ctypes.byref(serve._c_desc(*d._key()))
    rest = (A, 1 << 40, 0) if name in ("lca_page_tables", "lca_page_attn_q8", "lca_packed_attn") else (0,)
    for i in range(pointers):
        for bad in (0, A + 2):
            if bad == 0 and i in optional:
                continue
            args = [A] * pointers
            args[i] = bad
            assert getattr(lib, name)(cd, *args, *rest) == lca.ERR_INVALID_ARG, (name, i, bad)
    assert getattr(lib, name)(None, *[A] * pointers, *rest) == lca.ERR_INVALID_ARG


def test_float_arrays_need_four_bytes_of_alignment(lib):
    """(T = 0 ends behind the checks)"""
    cd = ctypes.byref(serve._c_desc(*_desc(T=0)._key()))
    assert lib.lca_page_store_q8(cd, A, A, A, A, A, A + 4, 0) == lca.OK
    assert lib.lca_page_attn_q8(cd, A, A, A, 0, A + 4, A, A, A, A + 4, A, A + 4, A, 1 << 40, 0) == lca.OK
    assert lib.lca_packed_attn(cd, A, A, A, A, 0, A + 4, A, A + 4, A, 1 << 40, 0) == lca.OK


def test_a_workspace_that_is_missing_or_too_small(lib):
    d = _desc(B=1000, max_q=1)
    need = serve.workspace_size(d)
    cd = ctypes.byref(serve._c_desc(*d._key()))
    assert need >= 4000
    assert lib.lca_page_tables(cd, *[A] * 11, 0, need, 0) == lca.ERR_WORKSPACE
    assert lib.lca_page_tables(cd, *[A] * 11, A + 4, need, 0) == lca.ERR_INVALID_ARG
    assert lib.lca_page_tables(cd, *[A] * 11, A, 3999, 0) == lca.ERR_WORKSPACE and b"needed" in lib.lca_last_error()


def test_the_largest_caps_are_taken(lib):
    for kw in (dict(softcap=1024.0), dict(softcap=1024.0, dtype=lca.F16), dict(softcap=1e30, dtype=lca.F32)):
        assert serve.workspace_size(_desc(**kw)) > 0


def test_no_rows_is_no_call(lib):
    """T = 0: nothing to write or attend, and empty tensors have no address."""
    cd = ctypes.byref(serve._c_desc(*_desc(T=0)._key()))
    assert lib.lca_page_store_q8(cd, 0, 0, 0, A, A, A, 0) == lca.OK
    assert lib.lca_page_attn_q8(cd, 0, A, A, 0, 0, A, A, A, A, 0, 0, 0, 0, 0) == lca.OK
    assert lib.lca_packed_attn(cd, 0, 0, 0, A, 0, 0, 0, 0, 0, 0, 0) == lca.OK


def test_tensors_that_do_not_fit(lib):
    import torch
    d = _desc()
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)      # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)        # noqa: E731
    ws, cache = torch.zeros(1 << 12, dtype=torch.uint8), [torch.zeros(20 * 2 * 16 * 64, dtype=torch.uint8)] * 2 + [torch.zeros(80)]
    Q, K, O = bf(40, 8, 64), bf(40, 2, 64), bf(40, 8, 64)
    wide = bf(40, 12 * 64)
    bad = [
        ("Q holds", lambda: serve.packed_attn(d, Q[:39], K, K, i32(3), None, None, O, None, ws)),
        ("SEL has dtype", lambda: serve.packed_attn(d, Q, K.float(), K, i32(3), None, None, O, None, ws)),
        ("doc_start holds", lambda: serve.packed_attn(d, Q, K, K, i32(2), None, None, O, None, ws)),
        ("prefix_len has dtype", lambda: serve.packed_attn(d, Q, K, K, i32(3), i32(2).long(), None, O, None, ws)),
        ("slopes holds", lambda: serve.packed_attn(d, Q, K, K, i32(3), None, torch.zeros(7), O, None, ws)),
        ("lse has dtype", lambda: serve.packed_attn(d, Q, K, K, i32(3), None, None, O, bf(40, 8), ws)),
        ("is not a device tensor", lambda: serve.packed_attn(d, Q, K, K, i32(3), None, None, O, None, ws)),
        ("is not a device tensor", lambda: serve.packed_attn(_desc(q_row=12 * 64), wide[:, :512].unflatten(1, (8, 64)), K, K, i32(3), None, None, O, None, ws)),
        ("q holds", lambda: serve.page_attn_q8(d, bf(39, 8, 64), i32(3), i32(2), None, None, i32(2, 8), *cache, O, None, ws)),
        ("block_table holds", lambda: serve.page_attn_q8(d, Q, i32(3), i32(2), None, None, i32(2, 7), *cache, O, None, ws)),
        ("slot has dtype", lambda: serve.page_store_q8(d, K, K, i32(40).long(), *cache)),
        ("sel_q8 has dtype", lambda: serve.page_store_q8(d, K, K, i32(40), cache[0].int(), *cache[1:])),
        ("scales holds", lambda: serve.page_store_q8(d, K, K, i32(40), *cache[:2], torch.zeros(79))),
        ("free_list holds", lambda: serve.page_tables(d, i32(2), i32(2), i32(19), i32(1), i32(1), i32(2, 8), i32(3), i32(2), i32(40), i32(40), i32(40), ws)),
        ("finished is required", lambda: serve.page_release(d, None, i32(2), i32(2, 8), i32(20), i32(1))),
    ]
    for needle, call in bad:
        with pytest.raises(ValueError) as e:
            call()
        assert needle in str(e.value), (needle, str(e.value))


class _Elsewhere:
    """A tensor on a device that is not the current one."""
    is_cuda, device = True, type("Device", (), {"index": 1, "__str__": lambda self: "cuda:1"})()


def test_a_tensor_on_another_device_is_refused(monkeypatch):
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="K is on cuda:1, the current device is cuda:0"):
        serve._same_device(Q=None, K=_Elsewhere())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    serve._same_device(K=_Elsewhere())


def test_every_tensor_of_a_call_is_held_to_the_current_device(lib, monkeypatch):
    """Each argument in turn on another device, the others as addresses."""
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(serve, "_bind", None)
    for name in ("_fit", "_fit_rows", "_fit_cache", "_fit_rule"):
        monkeypatch.setattr(serve, name, lambda *a: None)
    d = _desc()
    for call, n in ((serve.page_tables, 12), (serve.page_release, 5), (serve.page_store_q8, 6), (serve.page_attn_q8, 12), (serve.packed_attn, 9)):
        for i in range(n):
            args = [A] * n
            args[i] = _Elsewhere()
            with pytest.raises(ValueError, match="is on cuda:1, the current device is cuda:0"):
                call(d, *args)


def test_without_the_native_marshalling(lib, monkeypatch):
    """A module that does not know these calls, or does not fit, is left alone with a warning."""
    monkeypatch.setattr(serve, "_bind", None)

    class Older:
        pass
    with pytest.warns(RuntimeWarning, match="marshalled in Python"):
        serve._load_bind(serve.load(), Older)
    assert serve._bind is None


def test_strided_tensors_are_held_to_the_descriptor():
    import torch
    d = _desc(sel_row=160)

    class Strided:
        dtype, is_cuda = torch.bfloat16, True

        def __init__(self, shape, strides):
            self.shape, self.strides = shape, strides

        def stride(self, i=None):
            return self.strides if i is None else self.strides[i]

        def is_contiguous(self):
            return False

        def numel(self):
            return self.shape[0] * self.shape[1] * self.shape[2]

        def data_ptr(self):
            return A
    good = Strided((40, 2, 64), (160, 64, 1))
    serve._fit_rows(d, good, "SEL", 2, 64, d.sel_row)
    assert serve._row_ptr(good) == A
    for shape, strides in (((40, 2, 64), (128, 64, 1)), ((40, 2, 64), (160, 80, 1)), ((40, 2, 64), (160, 64, 2)), ((20, 4, 64), (160, 64, 1))):
        with pytest.raises(ValueError, match="elements apart"):
            serve._fit_rows(d, Strided(shape, strides), "SEL", 2, 64, d.sel_row)
