"""The serving operators (include/lca_serve.h) on the GPU against their definitions in float64 (tests/serve_ref.py)."""
import numpy as np
import pytest

from tests import serve_ref as ref

pytestmark = pytest.mark.gpu

KIND = {"bf16": "bfloat16", "f16": "float16", "f32": "float32"}


def _api():
    import torch
    from paper_2604_12452_amd import lca, serve
    return torch, lca, serve


def _code(dtype):
    from paper_2604_12452_amd import lca
    return {"bf16": lca.BF16, "f16": lca.F16, "f32": lca.F32}[dtype]


def _i32(v):
    import torch
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _randn(rng, dtype, *shape, size=1.0):
    import torch
    return torch.tensor(rng.standard_normal(shape) * size, dtype=getattr(torch, KIND[dtype]), device="cuda")


def _f64(t):
    return t.double().cpu().numpy()


def _close(got, want, bound, what):
    bad = ~(np.abs(got - want) <= bound) & ~(got == want) & ~(np.isnan(got) & np.isnan(want))
    assert not bad.any(), (what, np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5], np.broadcast_to(bound, want.shape)[bad][:5])


# ---- block tables ----

def _run_tables(cached, new, free_list, free_count, table, T, page, alias=False):
    torch, lca, serve = _api()
    B = len(cached)
    d = serve.Desc(B=B, T=T, H=1, S=1, d_pool=16, d_sel=16, page=page, n_blocks=len(free_list), max_blocks=table.shape[1])
    dev = dict(table=_i32(table), count=_i32([free_count]), q_start=_i32(np.full(B + 1, -7)), seq_len=_i32(np.full(B, -7)))
    rows = {n: _i32(np.full(T, -7)) for n in ("slot", "position", "request")}
    left = dev["count"] if alias else _i32([-7])
    stack = _i32(free_list)
    serve.page_tables(d, _i32(cached), _i32(new), stack, dev["count"], left, dev["table"], dev["q_start"], dev["seq_len"], rows["slot"], rows["position"],
                      rows["request"], serve.alloc_workspace(d))
    torch.cuda.synchronize()
    assert stack.cpu().tolist() == list(free_list)
    got = dict(table=dev["table"], q_start=dev["q_start"], seq_len=dev["seq_len"], **rows)
    return {k: v.cpu().numpy() for k, v in got.items()} | {"left": int(left)}


@pytest.mark.parametrize("B,T,page,new,spare", [(1, 1, 16, 1, 5), (1, 0, 16, 1, 5), (3, 7, 16, 3, 0), (64, 64, 16, 1, 3), (65, 70, 32, 1, 100), (200, 300, 16, 4, 20),
                                                (200, 4096, 48, 60, 500), (1030, 4097, 16, 5, 300), (2500, 9000, 64, 9, 40), (4097, 3000, 16, 2, 900), (6000, 20000, 32, 6, 7000), (7, 20000, 16, 5000, 1000), (5, 30000, 1024, 9000, 4)])
def test_page_tables(B, T, page, new, spare):
    rng = np.random.default_rng(B * 7 + T)
    max_blocks = 3 + 4 * new // page
    cached = rng.integers(0, max_blocks * page + 1, B)
    cached[rng.random(B) < 0.1] = 0
    add = rng.integers(0, new + 1, B)
    have = [ref.blocks(c, page) for c in cached]
    ids = rng.permutation(sum(have) + spare)
    table = np.full((B, max_blocks), -1)
    at = 0
    for b, h in enumerate(have):
        table[b, :h] = ids[at:at + h]
        at += h
    free_list = np.concatenate([ids[at:], ids[:at]])
    want = ref.page_tables(cached, add, free_list, spare, table, T, page)
    for alias in (False, True):
        got = _run_tables(cached, add, free_list, spare, table, T, page, alias)
        for k in want:
            np.testing.assert_array_equal(got[k], want[k], err_msg=k)


def test_page_tables_of_numbers_that_make_no_sense():
    """Lengths below zero and beyond every limit, a free count beyond the pool, table entries that are no blocks: refused or skipped, nothing else touched."""
    big = 2 ** 31 - 1
    cached = [0, -5, 40, big, 3, 17, big - 3, 20]
    add = [3, 2, big, 1, -4, 2, 9, 1]
    table = np.full((8, 4), -1)
    table[4, 0], table[5, :2], table[7, :2] = 6, (9999, 5), (2, -3)
    for count in (big, -2, 5, 0):
        want = ref.page_tables(cached, add, list(range(10)), count, table, 12, 16)
        got = _run_tables(cached, add, list(range(10)), count, table, 12, 16)
        for k in want:
            if k == "position":
                ok = [r not in (1, 3, 6) for r in want["request"]]
                np.testing.assert_array_equal(got[k][ok], want[k][ok], err_msg=k)
            else:
                np.testing.assert_array_equal(got[k], want[k], err_msg=k)


def test_release_returns_what_was_taken():
    torch, lca, serve = _api()
    rng = np.random.default_rng(3)
    B, page, max_blocks, n_blocks = 130, 16, 1500, 60000
    d = serve.Desc(B=B, T=0, H=1, S=1, d_pool=16, d_sel=16, page=page, n_blocks=n_blocks, max_blocks=max_blocks)
    ids = rng.permutation(n_blocks)
    cached = np.where(rng.random(B) < 0.3, 0, rng.integers(1, 2000, B))
    cached[5] = max_blocks * page
    have = [ref.blocks(int(c), page) for c in cached]
    table = np.full((B, max_blocks), -1)
    at = 0
    for b, h in enumerate(have):
        table[b, :h] = ids[at:at + h]
        at += h
    table[7, 0] = n_blocks                                    # (no block: not returned)
    finished = (rng.random(B) < 0.5).astype(int)
    finished[[5, 7]] = 1
    stack, count = np.concatenate([ids[at:], np.full(at, -1)]), n_blocks - at
    dev = [_i32(x) for x in (finished, cached, table, stack, [count])]
    for _ in range(2):                                        # (the second time there is nothing left to return)
        serve.page_release(d, *dev)
    torch.cuda.synchronize()
    want_stack, want_table, want_cached = stack.copy(), table.copy(), cached.copy()
    for b in np.flatnonzero(finished):
        for c in range(have[b]):
            if 0 <= table[b, c] < n_blocks:
                want_stack[count] = table[b, c]
                want_table[b, c] = -1
                count += 1
        want_cached[b] = 0
    assert int(dev[4]) == count
    np.testing.assert_array_equal(dev[3].cpu().numpy()[:count], want_stack[:count])
    np.testing.assert_array_equal(dev[2].cpu().numpy(), want_table)
    np.testing.assert_array_equal(dev[1].cpu().numpy(), want_cached)


# ---- the store ----

def _cache(rng, n_blocks, S, page, d_sel, d_pool):
    """Codes of any value but NaN and scales of a few powers of two."""
    sel, pool = (rng.integers(0, 256, shape).astype(np.uint8) for shape in ((n_blocks, S, page, d_sel), (n_blocks, S, page // 16, d_pool, 16)))
    for x in (sel, pool):
        x[(x & 0x7F) == 0x7F] = 0
    return sel, pool, (2.0 ** rng.integers(-9, -5, (n_blocks, S, 2))).astype(np.float32)


def _same_codes(got, want, what):
    """Equal bytes; a NaN may have either sign."""
    got, want = (np.where((x & 0x7F) == 0x7F, 0x7F, x) for x in (got, want))
    np.testing.assert_array_equal(got, want, err_msg=what)


def _check_store(rng, SEL, POOL, slot, cache, dtype, max_q, **rows):
    torch, lca, serve = _api()
    sel, pool, scales = cache
    n_blocks, S, page, d_sel = sel.shape
    d = serve.Desc(B=1, T=len(slot), H=S, S=S, d_pool=pool.shape[3], d_sel=d_sel, page=page, n_blocks=n_blocks, max_blocks=1, dtype=_code(dtype), max_q=max_q, **rows)
    dev = [torch.tensor(x, device="cuda") for x in cache]
    serve.page_store_q8(d, SEL, POOL, _i32(slot), *dev)
    torch.cuda.synchronize()
    want = ref.store(sel, pool, scales, _f64(SEL), _f64(POOL), slot, dtype)
    np.testing.assert_array_equal(dev[2].cpu().numpy(), want[2])
    _same_codes(dev[0].cpu().numpy(), want[0], "keys")
    _same_codes(dev[1].cpu().numpy(), want[1], "values")


def _slots(rng, lens, page, n_blocks):
    """Slots of runs of tokens, each starting anywhere in a block of its own."""
    ids, out = list(rng.permutation(n_blocks)), []
    for off, n in lens:
        p, blk = off, ids.pop()
        for _ in range(n):
            if p == page:
                p, blk = 0, ids.pop()
            out.append(blk * page + p)
            p += 1
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page,S,d_sel,d_pool,lens", [
    (16, 1, 16, 16, [(0, 1)]), (16, 2, 128, 128, [(5, 1), (15, 1), (0, 1), (7, 1)]), (32, 4, 96, 64, [(0, 70), (31, 2), (17, 15), (16, 16), (1, 1)]),
    (64, 3, 64, 256, [(0, 200), (63, 1), (33, 31)]), (1024, 1, 32, 48, [(1000, 30), (3, 100)]), (48, 2, 256, 16, [(0, 48), (47, 49), (20, 5)])])
@pytest.mark.parametrize("max_q", [1, 0])
def test_store(dtype, page, S, d_sel, d_pool, lens, max_q):
    rng = np.random.default_rng(page + d_sel)
    n_blocks = 5 + sum(2 + n // page for _, n in lens)
    slot = _slots(rng, lens, page, n_blocks)
    T = len(slot)
    loud = 2.0 ** rng.integers(-3, 4, (T, S, 1))
    SEL, POOL = ((_randn(rng, "f32", T, S, d) * _i32(0).float().new_tensor(loud)).to(_randn(rng, dtype, 1).dtype) for d in (d_sel, d_pool))
    _check_store(rng, SEL, POOL, slot, _cache(rng, n_blocks, S, page, d_sel, d_pool), dtype, max_q)


def test_store_of_padded_rows_and_strides():
    """Slots of -1 and beyond the pool are skipped wherever they stand; tokens of a fused projection lie further apart than their heads."""
    torch, lca, serve = _api()
    rng = np.random.default_rng(1)
    page, S, d, n_blocks = 16, 2, 64, 12
    slot = _slots(rng, [(3, 30), (0, 1), (9, 4)], page, n_blocks)
    slot = [-1, -1] + slot[:13] + [n_blocks * page, 2 ** 31 - 1] + slot[13:] + [-1] * 70        # (a block's tokens stay together)
    fused = _randn(rng, "bf16", len(slot), 3 * S * d)
    SEL, POOL = fused[:, S * d:2 * S * d].unflatten(1, (S, d)), fused[:, 2 * S * d:].unflatten(1, (S, d))
    for max_q in (1, 0):
        _check_store(rng, SEL, POOL, slot, _cache(rng, n_blocks, S, page, d, d), "bf16", max_q, sel_row=3 * S * d, pool_row=3 * S * d)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_store_of_extremes(dtype):
    """Zeros, subnormals, the largest values, infinities, NaN, and values on the border between two codes."""
    torch, lca, serve = _api()
    rng = np.random.default_rng(2)
    page, d = 16, 32
    kind = getattr(torch, KIND[dtype])
    info = torch.finfo(kind)
    rows = [np.zeros(d), np.full(d, info.tiny), np.full(d, -info.max), np.linspace(-1, 1, d) * info.max, np.arange(d) * info.tiny / 8,
            np.where(np.arange(d) % 2, np.inf, 1.0), np.where(np.arange(d) % 3, np.nan, -2.0), np.full(d, np.nan), (np.arange(d) + 0.5) * 2.0 ** -4,
            448 + np.arange(d) - 16.0, -0.0 * np.ones(d), 2.0 ** -(np.arange(d) / 2.0)]
    x = torch.tensor(np.array(rows), dtype=kind, device="cuda")[:, None].contiguous()
    cache = _cache(rng, 20, 1, page, d, d)
    for start in (0, 4, 15):                                       # a block each, fresh and behind older tokens, then all in one block
        _check_store(rng, x, x.flip(2).contiguous(), [b * page + start for b in range(len(rows))], cache, dtype, 1)
    _check_store(rng, x, x.flip(2).contiguous(), list(range(2, 2 + len(rows))), cache, dtype, 0)


# ---- attention ----

RULES = {
    "plain": dict(), "cap": dict(softcap=5.0), "bias": dict(slopes=True), "window": dict(window=20), "prefix": dict(prefix=23),
    "all": dict(softcap=3.0, slopes=True, window=33, prefix=9), "window1": dict(window=1),
}


def _slopes(H, use):
    import torch
    return torch.tensor([2.0 ** (-1 - h) for h in range(H)], dtype=torch.float32, device="cuda") if use else None


def _check_packed(Q, SEL, POOL, starts, dtype, scale, rule, behind=0, **rows):
    """lca_packed_attn on documents starting at `starts` (the last entry: their end), the rows behind them left alone."""
    torch, lca, serve = _api()
    T, H, _ = Q.shape
    S, d_pool = POOL.shape[1:]
    B = len(starts) - 1
    rule = dict(rule)
    slopes, prefix = _slopes(H, rule.pop("slopes", False)), rule.pop("prefix", 0)
    d = serve.Desc(B=B, T=T, H=H, S=S, d_pool=d_pool, d_sel=Q.shape[2], dtype=_code(dtype), scale=scale, **rule, **rows)
    O = torch.full((T, H, d_pool), 77.0, dtype=Q.dtype, device="cuda")
    lse = torch.full((T, H), 77.0, device="cuda")
    serve.packed_attn(d, Q, SEL, POOL, _i32(starts), _i32([prefix] * B) if prefix else None, slopes, O, lse, serve.alloc_workspace(d))
    torch.cuda.synchronize()
    got, got_lse = _f64(O), _f64(lse)
    assert (got[starts[-1]:] == 77).all() and (got_lse[starts[-1]:] == 77).all()
    q, k, v = _f64(Q), _f64(SEL), _f64(POOL)
    for lo, hi in zip(starts[:-1], starts[1:]):
        for h in range(H):
            s = h // (H // S)
            want = ref.attend(q[lo:hi, h], k[lo:hi, s], v[lo:hi, s], np.arange(hi - lo), hi - lo, dtype, scale=scale, prefix=min(prefix, hi - lo),
                              slope=float(slopes[h]) if slopes is not None else 0.0, **rule)
            _close(got[lo:hi, h], want[0], want[2], (lo, hi, h, "O"))
            _close(got_lse[lo:hi, h], want[1], want[3], (lo, hi, h, "lse"))


WIDTHS = [(64, 64), (128, 128), (128, 192), (256, 256), (80, 96), (8, 24), (200, 136)]


@pytest.mark.parametrize("rule", list(RULES))
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d_pool,d_sel", WIDTHS[:2])
def test_packed_rules(rule, dtype, d_pool, d_sel):
    rng = np.random.default_rng(d_pool)
    starts = [0, 1, 1, 18, 83, 211, 212]
    x = [_randn(rng, dtype, 212, h, d) for h, d in ((4, d_sel), (2, d_sel), (2, d_pool))]
    _check_packed(*x, starts, dtype, d_sel ** -0.5, RULES[rule])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d_pool,d_sel", WIDTHS + [(1024, 520)])
def test_packed_widths(dtype, d_pool, d_sel):
    rng = np.random.default_rng(d_pool + 1)
    x = [_randn(rng, dtype, 150, h, d) for h, d in ((3, d_sel), (1, d_sel), (1, d_pool))]
    _check_packed(*x, [0, 20, 140], dtype, d_sel ** -0.5, RULES["all"])


@pytest.mark.parametrize("H,S", [(1, 1), (7, 1), (5, 5), (28, 4), (32, 2), (100, 1)])
def test_packed_heads(H, S):
    rng = np.random.default_rng(H)
    x = [_randn(rng, "bf16", 75, h, 64) for h in (H, S, S)]
    _check_packed(*x, [0, 9, 75], "bf16", 0.125, RULES["prefix"])


@pytest.mark.parametrize("starts", [[0, 1], [0, 0, 0], [0, 64], [0, 63, 128], [0, 65, 65, 65, 600], [0, 2, 515], [0, 1000]])
def test_packed_lengths(starts):
    rng = np.random.default_rng(len(starts))
    T = starts[-1] + 5
    x = [_randn(rng, "bf16", T, h, 128) for h in (2, 1, 1)]
    for rule in ("plain", "window"):
        _check_packed(*x, starts, "bf16", 0.1, RULES[rule])


def test_packed_prefix_longer_than_the_document_and_negative_scale():
    rng = np.random.default_rng(9)
    x = [_randn(rng, "bf16", 140, h, 64) for h in (2, 2, 2)]
    _check_packed(*x, [0, 40, 140], "bf16", -0.2, dict(prefix=90))
    _check_packed(*x, [0, 40, 140], "bf16", 0.0, dict(softcap=2.0))
    _check_packed(*x, [0, 40, 140], "bf16", 0.0, dict(window=7))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_packed_large_logits(dtype):
    """Logits of hundreds that grow along the keys, and rows whose first visible keys are far below later ones."""
    rng = np.random.default_rng(10)
    T = 300
    Q, SEL, POOL = (_randn(rng, dtype, T, h, 64) for h in (2, 1, 1))
    SEL *= 1 + 0.03 * _i32(np.arange(T))[:, None, None].to(SEL.dtype)
    _check_packed(Q, SEL, POOL, [0, T], dtype, 2.0, dict())
    _check_packed(Q, SEL.flip(0).contiguous(), POOL, [0, T], dtype, 2.0, dict())
    _check_packed(Q, SEL, POOL, [0, T], dtype, 2.0, dict(softcap=200.0, window=100))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_caps_far_above_the_scores_of_few_keys(dtype):
    """lse of rows that see up to three keys, scores of a hundredth of the cap: the bound is that of no cap (its slope is at most one), and 2^-20 of the logits for the
    series, its argument and the change of base, not 2^-22 of the cap."""
    rng = np.random.default_rng(9)
    torch, lca, serve = _api()
    T, cap = 48, 500.0
    Q, SEL, POOL = (_randn(rng, dtype, T, 2, 64) for _ in range(3))
    d = serve.Desc(B=16, T=T, H=2, S=2, d_pool=64, d_sel=64, dtype=_code(dtype), scale=0.125, softcap=cap)
    O, lse = torch.empty_like(Q), torch.empty(T, 2, device="cuda")
    serve.packed_attn(d, Q, SEL, POOL, _i32(range(0, T + 1, 3)), None, None, O, lse, serve.alloc_workspace(d))
    for h in range(2):
        q, k, v = _f64(Q)[:, h], _f64(SEL)[:, h], _f64(POOL)[:, h]
        for lo in range(0, T, 3):
            r = slice(lo, lo + 3)
            want = ref.attend(q[r], k[r], v[r], np.arange(3), 3, dtype, scale=0.125, softcap=cap)
            bound = ref.attend(q[r], k[r], v[r], np.arange(3), 3, dtype, scale=0.125)
            _close(_f64(lse)[r, h], want[1], bound[3] + 2.0 ** -20 * 0.125 * np.abs(q[r] @ k[r].T).max(), (lo, h, "lse"))


@pytest.mark.parametrize("softcap", [1024.0, 1e6])
def test_packed_fp32_caps_far_above_the_scores(softcap):
    """The cap bends scores of a few units by next to nothing and must not cost them its own 2^-24: the bound is that of no cap (its slope is at most one),
    and 2^-20 of the logits for the hyperbolic tangent, its argument and the change of base."""
    rng = np.random.default_rng(8)
    Q, SEL, POOL = (_randn(rng, "f32", 90, 2, 64) for _ in range(3))
    torch, lca, serve = _api()
    d = serve.Desc(B=1, T=90, H=2, S=2, d_pool=64, d_sel=64, dtype=lca.F32, scale=0.5, softcap=softcap)
    O, lse = torch.empty_like(Q), torch.empty(90, 2, device="cuda")
    serve.packed_attn(d, Q, SEL, POOL, _i32([0, 90]), None, None, O, lse, serve.alloc_workspace(d))
    for h in range(2):
        q, k, v = _f64(Q)[:, h], _f64(SEL)[:, h], _f64(POOL)[:, h]
        want = ref.attend(q, k, v, np.arange(90), 90, "f32", scale=0.5, softcap=softcap)
        bound = ref.attend(q, k, v, np.arange(90), 90, "f32", scale=0.5)
        logit = 2.0 ** -20 * 0.5 * np.abs(q @ k.T).max()
        _close(_f64(O)[:, h], want[0], bound[2] + 2 * logit * np.abs(v).max(), (h, "O"))
        _close(_f64(lse)[:, h], want[1], bound[3] + logit, (h, "lse"))


def test_packed_pieces_of_a_fused_projection():
    rng = np.random.default_rng(11)
    T, H, S, d = 130, 6, 2, 64
    row = (H + 2 * S) * d + 16
    fused = _randn(rng, "f16", T, row)
    Q, SEL, POOL = fused[:, :H * d].unflatten(1, (H, d)), fused[:, H * d:(H + S) * d].unflatten(1, (S, d)), fused[:, (H + S) * d:(H + 2 * S) * d].unflatten(1, (S, d))
    _check_packed(Q, SEL, POOL, [0, 50, 130], "f16", 0.125, RULES["all"], q_row=row, sel_row=row, pool_row=row)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("where", ["later", "window", "document", "behind"])
def test_packed_what_a_row_does_not_see_has_no_part_in_it(dtype, where):
    """Infinities and NaN in keys and values that are masked; in the rows that see one the result is no number (values) or the definition's."""
    torch, lca, serve = _api()
    rng = np.random.default_rng(12)
    T, H, S, d = 260, 4, 2, 64
    Q, SEL, POOL = (_randn(rng, dtype, T, h, d) for h in (H, S, S))
    rule = dict(window=16) if where == "window" else dict()
    starts = [0, 100, 250]
    bad = {"later": 77, "window": 77, "document": 99, "behind": 250}[where]
    clean = [x.clone() for x in (Q, SEL, POOL)]
    desc = dict(B=2, T=T, H=H, S=S, d_pool=d, d_sel=d, dtype=_code(dtype), scale=0.125, **rule)
    d_ = serve.Desc(**desc)
    outs = []
    for values in (None, float("nan"), float("inf"), float("-inf")):
        x = [t.clone() for t in clean]
        if values is not None:
            x[1][bad] = values
            x[2][bad] = values
        O, lse = torch.zeros((T, H, d), dtype=Q.dtype, device="cuda"), torch.zeros((T, H), device="cuda")
        serve.packed_attn(d_, *x, _i32(starts), None, None, O, lse, serve.alloc_workspace(d_))
        torch.cuda.synchronize()
        outs.append((_f64(O), _f64(lse)))
    t = np.arange(T)
    sees = (t >= bad) & (t < 100) & (t < (bad + 16 if where == "window" else T)) if where != "behind" else t < 0
    half = ref.HALF_STEP[dtype]
    for O, lse in outs[1:]:
        # (a row may be computed another way than without the value: off by the roundings of both)
        assert np.allclose(O[~sees], outs[0][0][~sees], rtol=8 * half, atol=16 * half) and np.allclose(lse[~sees], outs[0][1][~sees], rtol=1e-5, atol=1e-5)
    assert np.isnan(outs[1][0][sees]).all() and np.isnan(outs[2][0][sees]).all()


def _fill_cache(rng, lens, page, S, d_sel, d_pool, extra=3):
    owned = [ref.blocks(n, page) for n in lens]
    n_blocks = sum(owned) + extra
    ids, at = rng.permutation(n_blocks), 0
    table = np.full((len(lens), max(max(owned), 1) + 2), -1)
    for b, o in enumerate(owned):
        table[b, :o] = ids[at:at + o]
        at += o
    return _cache(rng, n_blocks, S, page, d_sel, d_pool), table


def _check_paged(rng, rows, lens, H, S, d_sel, d_pool, page, dtype, rule, max_q=0, max_kv=0, cache=None, lse=True, behind=3):
    torch, lca, serve = _api()
    B, T = len(lens), sum(rows) + behind
    (sel, pool, scales), table = cache if cache is not None else _fill_cache(rng, lens, page, S, d_sel, d_pool)
    rule = dict(rule)
    slopes, prefix = _slopes(H, rule.pop("slopes", False)), rule.pop("prefix", 0)
    scale = 0.02 / d_sel ** 0.5
    q = _randn(rng, dtype, T, H, d_sel)
    starts = np.concatenate([[0], np.cumsum(rows)])
    d = serve.Desc(B=B, T=T, H=H, S=S, d_pool=d_pool, d_sel=d_sel, page=page, n_blocks=len(sel), max_blocks=table.shape[1], dtype=_code(dtype), scale=scale, max_q=max_q,
                   max_kv=max_kv, **rule)
    O = torch.full((T, H, d_pool), 77.0, dtype=q.dtype, device="cuda")
    L = torch.full((T, H), 77.0, device="cuda") if lse else None
    dev = [torch.tensor(x, device="cuda") for x in (sel, pool, scales)]
    serve.page_attn_q8(d, q, _i32(starts), _i32(lens), _i32([prefix] * B) if prefix else None, slopes, _i32(table), *dev, O, L, serve.alloc_workspace(d))
    torch.cuda.synchronize()
    got, got_lse = _f64(O), _f64(L) if lse else None
    assert (got[starts[-1]:] == 77).all() and (not lse or (got_lse[starts[-1]:] == 77).all())
    qf = _f64(q)
    capacity = table.shape[1] * page
    for b in range(B):
        n, r = min(lens[b], capacity), slice(starts[b], starts[b + 1])
        for s in range(S):
            k, v, real = ref.gather(sel, pool, scales.astype(np.float64), table[b], n, s)
            for h in range(s * (H // S), (s + 1) * (H // S)):
                want = ref.attend(qf[r, h], k, v, n - rows[b] + np.arange(rows[b]), n, dtype, scale=scale, prefix=min(prefix, n), real=real,
                                  slope=float(slopes[h]) if slopes is not None else 0.0, **rule)
                _close(got[r, h], want[0], want[2], (b, h, "O"))
                if lse:
                    _close(got_lse[r, h], want[1], want[3], (b, h, "lse"))


@pytest.mark.parametrize("rule", list(RULES))
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,lens", [([1] * 6, [1, 16, 17, 63, 200, 129]), ([4, 1, 0, 3], [4, 77, 50, 130]), ([90, 1, 40], [90, 100, 300])])
def test_paged_rules(rule, dtype, rows, lens):
    rng = np.random.default_rng(sum(lens))
    _check_paged(rng, rows, lens, 6, 2, 64, 64, 16, dtype, RULES[rule], max_q=max(rows))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d_pool,d_sel", [(64, 64), (128, 128), (128, 192), (256, 256), (96, 80), (16, 48), (208, 240), (256, 64)])
@pytest.mark.parametrize("rows,lens", [([1, 1], [70, 150]), ([30, 2], [100, 90])])
def test_paged_widths(dtype, d_pool, d_sel, rows, lens):
    rng = np.random.default_rng(d_pool + d_sel)
    _check_paged(rng, rows, lens, 4, 1, d_sel, d_pool, 32, dtype, RULES["all"], max_q=max(rows))


@pytest.mark.parametrize("H,S", [(1, 1), (7, 1), (5, 5), (28, 4), (32, 2), (40, 1), (100, 1)])
@pytest.mark.parametrize("rows,lens", [([1, 1, 1], [140, 3, 64]), ([3, 1], [140, 30])])
def test_paged_heads(H, S, rows, lens):
    rng = np.random.default_rng(H)
    _check_paged(rng, rows, lens, H, S, 64, 64, 16, "bf16", RULES["prefix"], max_q=max(rows))


@pytest.mark.parametrize("page", [16, 32, 48, 64, 1024])
@pytest.mark.parametrize("max_q,max_kv", [(1, 0), (1, 50), (0, 0), (0, 2000)])
def test_paged_long_and_any_hint(page, max_q, max_kv):
    """Split over many workgroups, with hints that are right, absent and wrong."""
    rng = np.random.default_rng(page)
    _check_paged(rng, [1, 1, 2, 1], [2000, 1, 1025, 777], 4, 2, 64, 64, page, "bf16", dict(), max_q=max_q, max_kv=max_kv)
    _check_paged(rng, [70, 1], [900, 1500], 4, 1, 64, 64, page, "f16", RULES["all"], max_q=max_q, max_kv=max_kv, lse=False)


@pytest.mark.parametrize("rows", [[1] * 20 + [90] + [0, 1, 2] * 10 + [33, 34] + [1] * 5, [33, 200, 1, 40] + [1] * 60, [0] * 50 + [300] + [0] * 50 + [65, 33, 65]])
@pytest.mark.parametrize("max_kv", [0, 5000])
def test_paged_chunks_among_many_small_requests(rows, max_kv):
    """Work items are counted by rows where the requests are many; their parts lie by rows as well."""
    rng = np.random.default_rng(len(rows))
    lens = [n + int(rng.integers(1, 50)) + (1500 if n >= 90 else 0) for n in rows]
    _check_paged(rng, rows, lens, 4, 2, 64, 64, 16, "bf16", RULES["window" if max_kv else "plain"] if rows[0] else dict(slopes=True), max_kv=max_kv)


def test_packed_splits_among_many_small_documents():
    rng = np.random.default_rng(17)
    starts = np.cumsum([0] + [1, 0, 3] * 20 + [1200] + [2, 60] * 3 + [700] + [1] * 9).tolist()
    x = [_randn(rng, "bf16", starts[-1] + 2, h, 64) for h in (3, 1, 1)]
    _check_packed(*x, starts, "bf16", 0.125, RULES["plain"])


def test_paged_rows_that_see_nothing():
    """More rows than tokens, requests of no tokens (refused ones), tables of numbers that are no blocks, lengths beyond the table."""
    rng = np.random.default_rng(21)
    _check_paged(rng, [3, 2, 5, 1], [1, 0, 40, 0], 4, 2, 64, 64, 16, "bf16", RULES["prefix"], max_q=5)
    _check_paged(rng, [80, 2], [20, 0], 4, 2, 64, 64, 16, "bf16", dict(), max_q=80)
    for rows, lens in (([1, 2, 1], [100, 90, 33]), ([60, 2, 1], [100, 90, 33])):
        cache, table = _fill_cache(rng, lens, 16, 2, 64, 64)
        table[0, 2], table[0, 6], table[1, :] = 2 ** 31 - 1, -1, -5
        _check_paged(rng, rows, lens, 4, 2, 64, 64, 16, "f16", RULES["bias"], max_q=max(rows), cache=(cache, table))
        cache, table = _fill_cache(rng, lens, 16, 2, 64, 64)
        _check_paged(rng, rows, [2 ** 31 - 1, 90, 33], 4, 2, 64, 64, 16, "f16", RULES["window"], max_q=max(rows), cache=(cache, table))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [[1, 1], [3, 4], [70, 5]])
def test_paged_nan_behind_the_last_token_and_outside_the_window(dtype, rows):
    """Codes that are NaN in the free places of a request's last block, in blocks outside the window, and in tokens that only later rows see."""
    torch, lca, serve = _api()
    rng = np.random.default_rng(22)
    lens, page, S, H, d = [100, 77], 32, 2, 4, 64
    (sel, pool, scales), table = _fill_cache(rng, lens, page, S, d, d)
    for b, n in enumerate(lens):
        for j in list(range(n, ref.blocks(n, page) * page)) + list(range(0, 8)):
            sel[table[b, j // page], :, j % page] = 0x7F
            pool[table[b, j // page], :, j % page // 16, :, j % 16] = 0xFF
    _check_paged(rng, rows, lens, H, S, d, d, page, dtype, dict(window=20), max_q=max(rows), cache=((sel, pool, scales), table))
    last = lens[0] - 1                                    # the newest token: the rows in front of it do not see it
    pool[table[0, last // page], :, last % page // 16, :, last % 16] = 0x7F
    _check_paged(rng, rows, lens, H, S, d, d, page, dtype, dict(window=20), max_q=max(rows), cache=((sel, pool, scales), table))


# ---- together ----

def _decoded(sel, pool, scales):
    import torch
    k = sel.view(torch.float8_e4m3fn).float() * scales[..., 1, None, None]
    v = pool.view(torch.float8_e4m3fn).float() * scales[..., 0, None, None, None]
    return k.transpose(1, 2).flatten(0, 1), v.permute(0, 2, 4, 1, 3).flatten(0, 2)          # [slots, S, d]


@pytest.mark.parametrize("graph", [False, True])
def test_a_serving_loop(graph):
    """Requests that come, grow and leave: tables, store, attention over the cache and release, step after step (also recorded once into a graph and
    replayed on lengths that change), each step's attention checked against lca_packed_attn over the cache's values as they stand, and the first
    step's prompts with both calls."""
    torch, lca, serve = _api()
    rng = np.random.default_rng(30)
    B, H, S, d, page, max_blocks, n_blocks, T = 4, 4, 2, 64, 16, 20, 60, 170
    kind = torch.bfloat16
    desc = serve.Desc(B=B, T=T, H=H, S=S, d_pool=d, d_sel=d, page=page, n_blocks=n_blocks, max_blocks=max_blocks, scale=d ** -0.5, softcap=4.0, window=70, dtype=lca.BF16)
    sel, pool, scales = serve.alloc_cache(desc)
    free_list, count = _i32(rng.permutation(n_blocks)), _i32([n_blocks])
    table, cached, new = _i32(np.full((B, max_blocks), -1)), _i32([0] * B), _i32([0] * B)
    prefix, slopes, finished = _i32([6, 0, 3, 20]), _slopes(H, True), _i32([0] * B)
    q_start, seq_len = _i32([0] * (B + 1)), _i32([0] * B)
    slot, position, request = (_i32([0] * T) for _ in range(3))
    Q, SEL, POOL = (torch.zeros((T, h, d), dtype=kind, device="cuda") for h in (H, S, S))
    O, lse, ws = torch.zeros((T, H, d), dtype=kind, device="cuda"), torch.zeros((T, H), device="cuda"), serve.alloc_workspace(desc)

    def step():
        serve.page_release(desc, finished, cached, table, free_list, count)
        serve.page_tables(desc, cached, new, free_list, count, count, table, q_start, seq_len, slot, position, request, ws)
        serve.page_store_q8(desc, SEL, POOL, slot, sel, pool, scales)
        serve.page_attn_q8(desc, Q, q_start, seq_len, prefix, slopes, table, sel, pool, scales, O, lse, ws)

    run = step
    if graph:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()                                     # (no new tokens: changes nothing)
        torch.cuda.synchronize()
        recorded = torch.cuda.CUDAGraph()
        with torch.cuda.graph(recorded, stream=side):
            step()
        run = recorded.replay
    lens, shown = [0] * B, np.zeros(B, int)
    for k in range(8):
        gone = [int(k in (4, 6) and b == k % B) for b in range(B)]
        lens = [0 if g else n for g, n in zip(gone, lens)]
        add = [30 + 7 * b if k == 0 else 19 if lens[b] == 0 else (1, 1, 0, 4)[(b + k) % 4] for b in range(B)]
        finished.copy_(_i32(gone))
        new.copy_(_i32(add))
        for x in (Q, SEL, POOL):
            x.copy_(_randn(rng, "bf16", *x.shape, size=1 + k % 3))
        O.fill_(77)
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        total = [n + a for n, a in zip(lens, add)]
        assert seq_len.tolist() == total and q_start.tolist() == np.concatenate([[0], np.cumsum(add)]).tolist()
        used = table[table >= 0].tolist()
        assert len(set(used)) == len(used) == n_blocks - int(count) and set(used) | set(free_list[:int(count)].tolist()) == set(range(n_blocks))
        keys, values = _decoded(sel, pool, scales)
        rows, starts = sum(add), np.concatenate([[0], np.cumsum(total)])
        # the same rows by the packed call: every request is a document of all its tokens
        slots = torch.cat([(table[b, torch.arange(n, device="cuda") // page] * page + torch.arange(n, device="cuda") % page).long() for b, n in enumerate(total)])
        full = serve.Desc(B=B, T=int(starts[-1]), H=H, S=S, d_pool=d, d_sel=d, scale=d ** -0.5, softcap=4.0, window=70, dtype=lca.BF16)
        Qd = torch.zeros((full.T, H, d), dtype=kind, device="cuda")
        at = torch.tensor(np.concatenate([starts[b + 1] - add[b] + np.arange(add[b]) for b in range(B)]), device="cuda")
        Qd[at] = Q[:rows]
        Od, Ld = torch.zeros_like(Qd), torch.zeros((full.T, H), device="cuda")
        K, V = keys[slots].to(kind), values[slots].to(kind)
        assert torch.equal(K.float(), keys[slots]) and torch.equal(V.float(), values[slots])
        serve.packed_attn(full, Qd, K.contiguous(), V.contiguous(), _i32(starts), torch.minimum(prefix, seq_len), slopes, Od, Ld, serve.alloc_workspace(full))
        torch.cuda.synchronize()
        # both round their weights and outputs to bf16 (2^-8): off by at most four half steps of the largest value
        assert float((O[:rows].float() - Od[at].float()).abs().max()) <= 4 * 2.0 ** -8 * float(V.float().abs().max())
        # logits: 68 roundings of 2^-24 of sums of up to a few hundred times the scale, the cap's 2^-22 of 4
        assert float((lse[:rows] - Ld[at]).abs().max()) <= 1e-4
        assert (O[rows:] == 77).all()
        lens = total
        cached.copy_(seq_len)


# ---- where it can go wrong ----

def test_packed_many_documents_and_one_long_one():
    """More documents than lanes look at in one go, most of a token or two, some empty; one document split over its tiles."""
    rng = np.random.default_rng(40)
    lens = rng.choice([0, 1, 1, 2, 3], 5000)
    starts = np.concatenate([[0], np.cumsum(lens)]).tolist()
    x = [_randn(rng, "bf16", starts[-1], 1, 64) for _ in range(3)]
    torch, lca, serve = _api()
    d = serve.Desc(B=5000, T=starts[-1], H=1, S=1, d_pool=64, d_sel=64)
    O = torch.zeros((starts[-1], 1, 64), dtype=torch.bfloat16, device="cuda")
    serve.packed_attn(d, *x, _i32(starts), None, None, O, None, serve.alloc_workspace(d))
    q, k, v = (_f64(t)[:, 0] for t in x)
    got = _f64(O)[:, 0]
    for lo, hi in zip(starts[:-1], starts[1:]):
        want = ref.attend(q[lo:hi], k[lo:hi], v[lo:hi], np.arange(hi - lo), hi - lo, "bf16")
        _close(got[lo:hi], want[0], want[2], (lo, hi))
    x = [_randn(rng, "f16", 2600, 1, 64) for _ in range(3)]
    _check_packed(*x, [0, 2500], "f16", 0.125, dict())
    _check_packed(*x, [0, 30, 2600], "f16", 0.125, dict(window=900, prefix=100, slopes=True))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("jump", [8.0, 40.0, 300.0])
def test_packed_far_keys_with_larger_logits_than_near_ones(dtype, jump):
    """Keys are taken from the rows backwards: blocks of far keys whose logits exceed the near ones' by a few, by tens, and past either type's exponents."""
    torch, lca, serve = _api()
    rng = np.random.default_rng(41)
    T = 700
    Q, SEL, POOL = (_randn(rng, dtype, T, 1, 64) for _ in range(3))
    Q[:, :, 0] = 1.0
    SEL[:, :, 0] = 0.0
    for lo, hi, share in ((300, 310, 0.5), (130, 131, 1.0), (5, 70, 0.75)):
        SEL[lo:hi, :, 0] = jump * share
    _check_packed(Q, SEL, POOL, [0, T], dtype, 1.0, dict())


def test_store_and_attention_past_32_bits_of_offset():
    """A cache of more than 2^32 bytes of codes each: tokens stored in its last blocks, and attended to."""
    torch, lca, serve = _api()
    rng = np.random.default_rng(42)
    page, S, d, n_blocks = 64, 8, 128, 66000
    desc = serve.Desc(B=2, T=140, H=S, S=S, d_pool=d, d_sel=d, page=page, n_blocks=n_blocks, max_blocks=3, scale=d ** -0.5)
    sel, pool = (torch.empty(n_blocks * page * S * d, dtype=torch.uint8, device="cuda") for _ in range(2))
    scales = torch.zeros((n_blocks, S, 2), device="cuda")
    used = [65999, 3, 65536, 65535]
    slot = [65999 * page + i for i in range(64)] + [3 * page + i for i in range(6)] + [65536 * page + i for i in range(64)] + [65535 * page + i for i in range(6)]
    SEL, POOL, Q = (_randn(rng, "bf16", 140, S, d) for _ in range(3))
    serve.page_store_q8(desc, SEL, POOL, _i32(slot), sel, pool, scales)
    where = lambda t, shape: torch.stack([t.view(n_blocks, -1)[b].view(shape) for b in used]).cpu().numpy()      # noqa: E731
    cache = (where(sel, (S, page, d)), where(pool, (S, page // 16, d, 16)), scales[used].cpu().numpy())
    for i in (1, 3):                                              # (what lies behind the tokens of a block is not defined)
        cache[0][i][:, 6:] = 0
        cache[1][i][:, 1:] = 0
        cache[1][i][:, 0, :, 6:] = 0
    want = ref.store(*(np.zeros_like(c) for c in cache), _f64(SEL), _f64(POOL), list(range(64)) + list(range(64, 70)) + list(range(128, 192)) + list(range(192, 198)), "bf16")
    for got, w in zip(cache, want):
        np.testing.assert_array_equal(got, w)
    for rows in (1, 70):                                          # (both kernels; the second with every row of the batch)
        O = torch.zeros((140, S, d), dtype=torch.bfloat16, device="cuda")
        q_start = [0, rows, 2 * rows]
        serve.page_attn_q8(desc, Q, _i32(q_start), _i32([70, 70]), None, None, _i32([[65999, 3, -1], [65536, 65535, -1]]), sel, pool, scales, O, None, serve.alloc_workspace(desc))
        for b in range(2):
            for s in range(S):
                k, v, _ = ref.gather(cache[0], cache[1], cache[2].astype(np.float64), [2 * b, 2 * b + 1], 70, s)
                r = slice(q_start[b], q_start[b + 1])
                w = ref.attend(_f64(Q[r])[:, s], k, v, 70 - rows + np.arange(rows), 70, "bf16", scale=d ** -0.5)
                _close(_f64(O[r])[:, s], w[0], w[2], (rows, b, s))


@pytest.mark.parametrize("row", [1 << 22, (1 << 23) + 8])
def test_packed_tokens_far_apart(row):
    """Strides whose products pass 2^32 bytes: within what a buffer descriptor spans from tile to tile, and beyond it (row by row)."""
    torch, lca, serve = _api()
    rng = np.random.default_rng(43)
    T, d = 270, 64
    big = torch.empty((T - 1) * row + 3 * d, dtype=torch.float16, device="cuda")
    x = torch.as_strided(big, (T, 3, d), (row, d, 1))
    x.copy_(_randn(rng, "f16", T, 3, d))
    views = [x[:, i:i + 1] for i in range(3)]
    _check_packed(*views, [0, 200, 270], "f16", 0.125, RULES["prefix"], q_row=row, sel_row=row, pool_row=row)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attention_over_scales_at_the_ends_of_their_range(dtype):
    """Blocks whose scales are the smallest and the largest the store writes: every decoded value is one of the type, and so are the products' operands."""
    rng = np.random.default_rng(44)
    lens, page, d = [50, 130], 16, 64
    (sel, pool, scales), table = _fill_cache(rng, lens, page, 2, d, d)
    lo, hi = ref.RANGE[dtype]
    scales[..., 1] = 2.0 ** np.where(rng.random(scales.shape[:2]) < 0.5, lo, -8)       # keys: logits of ordinary size
    scales[..., 0] = 2.0 ** np.where(rng.random(scales.shape[:2]) < 0.5, lo, hi if dtype == "f16" else 100)
    sel[(sel & 0x7F) == 0x7F] = 0
    if dtype == "f16":                                                                  # (outputs of the largest scale end at 65504: smaller codes there)
        pool &= 0xBF
    for rows in ([1, 3], [40, 70]):
        _check_paged(rng, rows, lens, 4, 2, d, d, page, dtype, dict(), max_q=max(rows), cache=((sel, pool, scales), table))


def test_two_calls_at_once_and_on_other_streams():
    """The same inputs on the current stream, and on two streams at a time with workspaces of their own: the same bits, every time."""
    torch, lca, serve = _api()
    rng = np.random.default_rng(45)
    rows, lens = [1] * 5 + [80], [900, 40, 3000, 1, 2000, 700]
    (sel, pool, scales), table = _fill_cache(rng, lens, 32, 2, 128, 128)
    q, starts = _randn(rng, "bf16", sum(rows), 8, 128), _i32(np.concatenate([[0], np.cumsum(rows)]))
    d = serve.Desc(B=6, T=sum(rows), H=8, S=2, d_pool=128, d_sel=128, page=32, n_blocks=len(sel), max_blocks=table.shape[1], scale=0.005)
    dev = [torch.tensor(x, device="cuda") for x in (sel, pool, scales)]
    args = (d, q, starts, _i32(lens), None, _slopes(8, True), _i32(table), *dev)
    packed = serve.Desc(B=1, T=1500, H=2, S=1, d_pool=128, d_sel=128, scale=0.09, softcap=20.0)
    x = [_randn(rng, "bf16", 1500, h, 128) for h in (2, 1, 1)]

    def buffers():
        return (torch.empty_like(q), torch.empty((sum(rows), 8), device="cuda"), serve.alloc_workspace(d), torch.empty_like(x[0]), torch.empty((1500, 2), device="cuda"),
                serve.alloc_workspace(packed))

    def call(b, stream=None):
        serve.page_attn_q8(*args, *b[:3], stream=stream)
        serve.packed_attn(packed, *x, _i32([0, 1500]) if stream is None else start, None, None, *b[3:], stream=stream)
    first = buffers()
    call(first)
    start = _i32([0, 1500])
    torch.cuda.synchronize()
    streams, others = [torch.cuda.Stream() for _ in range(2)], [buffers() for _ in range(2)]
    for _ in range(5):
        for b, s in zip(others, streams):
            call(b, s)
        torch.cuda.synchronize()
        for b in others:
            for i in (0, 1, 3, 4):
                assert torch.equal(b[i].view(torch.uint8), first[i].view(torch.uint8))


def test_two_graphs_that_share_a_workspace():
    """Recorded with one workspace, replayed one after the other with other calls between: nothing of one call is left for the next."""
    torch, lca, serve = _api()
    rng = np.random.default_rng(46)
    runs = []
    for lens, H, d in (([2500, 33], 4, 64), ([700, 1900], 8, 128)):
        (sel, pool, scales), table = _fill_cache(rng, lens, 16, 2, d, d)
        desc = serve.Desc(B=2, T=2, H=H, S=2, d_pool=d, d_sel=d, page=16, n_blocks=len(sel), max_blocks=table.shape[1], scale=0.01, max_q=1)
        q, O = _randn(rng, "bf16", 2, H, d), torch.zeros((2, H, d), dtype=torch.bfloat16, device="cuda")
        runs.append((desc, [q, _i32([0, 1, 2]), _i32(lens), None, None, _i32(table), *(torch.tensor(x, device="cuda") for x in (sel, pool, scales)), O, None]))
    ws = torch.empty(max(serve.workspace_size(r[0]) for r in runs), dtype=torch.uint8, device="cuda")
    want, graphs, side = [], [], torch.cuda.Stream()
    for desc, args in runs:
        serve.page_attn_q8(desc, *args, ws)
        torch.cuda.synchronize()
        want.append(args[-2].clone())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            serve.page_attn_q8(desc, *args, ws)
        graphs.append(g)
    for _ in range(4):
        for g, (desc, args), w in zip(graphs, runs, want):
            args[-2].fill_(77)
            ws.fill_(0xFF)                                        # (NaN wherever something stale would be read)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(args[-2], w)
