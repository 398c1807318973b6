"""What the serving entry points launch, on the CPU (tests/launches.py): which kernel, how many workgroups, and that the workspace holds what
they write."""
import ctypes
import re

import pytest

from paper_2604_12452_amd import lca, serve
from tests import launches as t

A = t.A


def _name(launch):
    """(kernel, element type, its numbers, its truth values); names with the bf16 type may come mangled."""
    k = launch.kernel
    if k.startswith("_Z"):
        kernel, rest = re.match(r"_ZN3lca12_GLOBAL__N_1\d\d([a-z_]+_kernel)(.*)", k).groups()
        return kernel, "bf16" if "DF16b" in rest else "f16", [int(x) for x in re.findall(r"Li(\d+)E", rest)], [x == "1" for x in re.findall(r"Lb([01])E", rest)]
    kernel, rest = re.match(r"([a-z_]+_kernel)(.*)", k).groups()
    return kernel, "f16" if "_Float16" in rest or "f16_t" in rest else "f32" if "float" in rest else "bf16", [int(x) for x in re.findall(r"\b(\d+)\b", rest)], re.findall(r"true|false", rest)


def _run(name, d, pointers, ws=True):
    lib = t._load()
    for n in serve.EXPORTS:
        getattr(lib, n).argtypes = getattr(serve.load(), n).argtypes
    lib.trace_reset()
    args = [A if p else None for p in pointers]
    status = getattr(lib, name)(ctypes.byref(serve._c_desc(*d._key())), *args, *((A, 1 << 40) if ws else ()), None)
    assert status == lca.OK, lib.lca_last_error().decode()
    return [t.Launch(k, int(g), int(b), int(s)) for k, g, b, s in (line.split("\t") for line in lib.trace_log().decode().splitlines())]


def _paged(d, slopes=False):
    return _run("lca_page_attn_q8", d, [1, 1, 1, 0, slopes, 1, 1, 1, 1, 1, 0])


def _packed(d, slopes=False):
    return _run("lca_packed_attn", d, [1, 1, 1, 1, 0, slopes, 1, 0])


def _desc(**kw):
    return serve.Desc(**{**dict(B=4, T=4, H=32, S=8, d_pool=128, d_sel=128, page=16, n_blocks=5000, max_blocks=4096), **kw})


@pytest.mark.parametrize("T,B,apart,grids", [(1, 1, 0, [1]), (256, 64, 1, [1]), (257, 64, 1, [1]), (4096, 2000, 0, [1]), (4096, 2000, 1, [4]), (4097, 10, 0, [1, 17]),
                                             (4097, 10, 1, [5]), (131072, 4096, 1, [128]), (131072, 4097, 1, [1, 512]), (0, 5000, 0, [1]), (0, 3, 0, [1])])
def test_tables(T, B, apart, grids):
    """One launch, every workgroup with all requests' sums; two where the stack's count is written in place and several would read it, or LDS holds no more requests."""
    lib = t._load()
    for n in serve.EXPORTS:
        getattr(lib, n).argtypes = getattr(serve.load(), n).argtypes
    lib.trace_reset()
    d = _desc(T=T, B=B, H=1, S=1)
    args = [A] * 11
    args[4] = A + 64 * apart
    assert lib.lca_page_tables(ctypes.byref(serve._c_desc(*d._key())), *args, A, 1 << 40, None) == lca.OK
    run = [line.split("\t") for line in lib.trace_log().decode().splitlines()]
    assert [int(r[1]) for r in run] == grids
    assert int(run[0][2]) == (64 if B <= 64 and T <= 256 else 1024)


@pytest.mark.parametrize("max_q,T,window", [(1, 32, 1), (8, 32, 2), (8, 4000, 16), (500, 2000, 16), (0, 8, 1), (0, 1000, 16), (0, 100000, 64)])
def test_store(max_q, T, window):
    """A wavefront's window is as long as the runs of tokens (4 requests), less where short ones may fill it."""
    (run,) = _run("lca_page_store_q8", _desc(T=T, max_q=max_q), [1] * 6, ws=False)
    assert run.grid == -(-(-(-T // window)) * 8 * 2 // 4)


@pytest.mark.parametrize("kw,kernels", [
    (dict(max_q=1, max_kv=1000), ["page_decode_kernel"]), (dict(max_q=1, max_kv=1100), ["page_decode_kernel", "page_merge_kernel"]),
    (dict(max_q=1, max_kv=4096, B=32, T=32), ["page_decode_kernel"]), (dict(max_q=1, max_kv=5000, B=32, T=32), ["page_decode_kernel", "page_merge_kernel"]),
    (dict(max_q=16, T=64, max_kv=1000), ["page_decode_kernel"]), (dict(max_q=17, T=64, max_kv=900), ["page_decode_kernel", "scored_tile_kernel"]),
    (dict(T=64, B=4, max_kv=9000), ["page_decode_kernel", "page_merge_kernel", "scored_tile_kernel", "scored_merge_kernel"]),
    (dict(max_q=1, max_kv=9000, window=500), ["page_decode_kernel"])])
def test_paged_kernels(kw, kernels):
    run = _paged(_desc(**kw))
    assert [_name(r)[0] for r in run] == kernels


@pytest.mark.parametrize("dtype", [lca.BF16, lca.F16])
@pytest.mark.parametrize("d_pool,d_sel,dk,dv", [(16, 64, 64, 64), (64, 80, 128, 128), (128, 128, 128, 128), (128, 144, 192, 128), (144, 16, 256, 256), (256, 256, 256, 256)])
def test_width_classes_and_lds(dtype, d_pool, d_sel, dk, dv):
    e = "bf16" if dtype == lca.BF16 else "f16"
    for d in (_desc(d_pool=d_pool, d_sel=d_sel, dtype=dtype, max_q=1, max_kv=500), _desc(d_pool=d_pool, d_sel=d_sel, dtype=dtype, T=400, max_kv=500)):
        for r in _paged(d):
            assert _name(r)[1] == e and (_name(r)[2][:2] == [dk, dv] or "merge" in r.kernel), r
    run = _packed(_desc(d_pool=d_pool, d_sel=d_sel, dtype=dtype, T=40000, B=3))
    assert len(run) == 1 and _name(run[0])[1:3] == (e, [dk, dv]) and run[0].lds == 2 * 64 * 2 * (dk + dv) <= (160 if dv == 256 else 80) * 1024


@pytest.mark.parametrize("kw", [dict(dtype=lca.F32), dict(d_pool=264), dict(d_sel=512), dict(sel_row=1 << 23), dict(pool_row=1 << 24)])
def test_what_no_matrix_kernel_takes_goes_row_by_row(kw):
    (run,) = _packed(_desc(T=100, **kw))
    assert _name(run)[0] == "scored_rows_kernel" and run.grid == 100 * 32 // 4


@pytest.mark.parametrize("d", [
    _desc(max_q=1, max_kv=60000), _desc(B=1, T=8, max_q=8, max_kv=60000), _desc(B=1, T=1, H=100, S=1, max_q=1, max_kv=30000), _desc(B=3, T=3, max_q=1, d_pool=256, d_sel=256),
    _desc(B=200, T=200, max_q=1), _desc(T=3000, B=2), _desc(T=70, B=1, max_kv=65536, d_pool=64, d_sel=64), _desc(T=500, B=1, H=2, S=2, max_blocks=0, n_blocks=0),
    _desc(T=9000, B=1, H=1, S=1, max_blocks=0, n_blocks=0), _desc(T=2000, B=30, H=4, S=4, d_pool=192, max_blocks=0, n_blocks=0)], ids=lambda d: f"B{d.B}-T{d.T}-H{d.H}-S{d.S}-{d.d_pool}")
def test_the_partial_results_fit_the_workspace(d):
    """A part's results are 16 NCT columns (decode) or as many as its workgroup has (32 per wavefront), the width and two numbers each; the tile kernels' lie in a slot
    for every 64 (row, head) pairs, KV head and part, whatever the number of requests."""
    have = serve.workspace_size(d)
    for run in ([_paged(d)] if d.max_blocks else []) + [_packed(d)]:
        for i, r in enumerate(run):
            if "merge" not in r.kernel:
                continue
            dv, columns = _name(run[i - 1])[2][1], 16 * _name(run[i - 1])[2][2] if "decode" in run[i - 1].kernel else run[i - 1].block // 2
            places = run[i - 1].grid
            if "decode" not in run[i - 1].kernel:
                pairs = d.T * d.H // d.S
                slots, items = pairs // 64 + 1, pairs // columns + d.B
                if _name(run[i - 1])[3][0] in (True, "true"):          # over the cache
                    items = min(items, slots)
                parts, rest = divmod(run[i - 1].grid, items * d.S)
                assert rest == 0 and parts > 1
                places = slots * d.S * parts
            assert places * columns * (dv + 2) * 4 <= have, (run[i - 1], have)


def test_the_workspace_does_not_grow_with_requests_of_one_token():
    """The chunk kernel's part of it (no hints: it is launched) is a matter of the rows."""
    small, large = (serve.workspace_size(_desc(T=256, B=b, max_kv=9000)) for b in (4, 256))
    assert large <= 3 * small and large < 1 << 29


def test_hints_never_make_a_grid_of_none():
    for kw in (dict(max_kv=1), dict(max_kv=0), dict(max_q=0), dict(max_q=10 ** 6, max_kv=10 ** 9), dict(window=1), dict(window=2 ** 31 - 1)):
        assert all(r.grid >= 1 for r in _paged(_desc(**kw)) + _packed(_desc(T=50, **kw)))
