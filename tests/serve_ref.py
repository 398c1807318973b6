"""The serving operators by their definitions in float64 (numpy), for the tests: block tables, the 8-bit store, scored attention with the
error that a kernel may make on each output."""
import math

import numpy as np

from oracle import q8

RANGE = {"bf16": (-100, 119), "f16": (-15, 7)}
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}     # relative, of one rounding to the type


def blocks(n, page):
    return -(-n // page)


def page_tables(cached, new, free_list, free_count, table, T, page):
    """Outputs of lca_page_tables as a dict; inputs are lists / arrays and are not changed."""
    B, max_blocks = table.shape
    table, n_blocks = table.copy(), len(free_list)
    stack = list(free_list[:max(0, min(free_count, n_blocks))])
    top = len(stack)
    out = dict(q_start=[0], seq_len=[], slot=np.full(T, -1), position=np.zeros(T, int), request=np.full(T, -1))
    row = wanted = got = 0
    for b in range(B):
        c, n = int(cached[b]), int(new[b])
        rows = max(n, 0)
        fits = c >= 0 and n >= 0 and row + rows <= T and c + n <= max_blocks * page
        have = blocks(c, page) if fits else 0
        need = blocks(c + n, page) - have if fits else 0
        wanted += need
        ok = fits and (need == 0 or wanted <= top)
        if ok:
            for r in range(need):
                table[b, have + r] = stack[top - 1 - (wanted - need) - r]
            got += need
        for i in range(rows):
            if row + i >= T:
                break
            p = max(c, 0) + i
            out["position"][row + i], out["request"][row + i] = p, b
            if ok and 0 <= table[b, p // page] < n_blocks:
                out["slot"][row + i] = table[b, p // page] * page + p % page
        row = min(row + rows, 1 << 40)
        out["q_start"].append(min(row, T))
        out["seq_len"].append(c + n if ok else 0)
    out.update(table=table, left=top - got)
    return out


def scale_exponent(amax, dtype):
    lo, hi = RANGE[dtype]
    if not amax > 0:
        return lo
    if amax == math.inf:
        return hi
    f, e = math.frexp(amax)
    return min(max(e - 9 if f <= 0.875 else e - 8, lo), hi)


def _encode(x):
    """E4M3 codes of float64 values, saturating, NaN as 0x7F."""
    return np.where(np.isnan(x), 0x7F, q8.e4m3_encode(np.where(np.isnan(x), 0.0, x))).astype(np.uint8)


def store(sel_q8, pool_q8, scales, SEL, POOL, slot, dtype):
    """lca_page_store_q8 on copies: (sel_q8, pool_q8, scales).  SEL, POOL float64 [T, S, d]."""
    sel_q8, pool_q8, scales = sel_q8.copy(), pool_q8.copy(), scales.astype(np.float64)
    n_blocks, S, page, _ = sel_q8.shape
    table = q8.e4m3_decode_table()
    T, t = len(slot), 0
    while t < T:
        first = int(slot[t])
        if not 0 <= first < n_blocks * page:
            t += 1
            continue
        block, off = divmod(first, page)
        n = 1
        while t + n < T and off + n < page and slot[t + n] == first + n:
            n += 1
        for s in range(S):
            for which, x in ((0, POOL), (1, SEL)):
                x = x[t:t + n, s]
                mags = np.abs(x[~np.isnan(x)])
                new = 2.0 ** scale_exponent(mags.max() if mags.size else 0.0, dtype)
                old = scales[block, s, which]
                scale = max(new, old) if off else new
                codes = sel_q8[block, s] if which else pool_q8[block, s].transpose(0, 2, 1).reshape(page, -1).copy()
                if off and scale > old:
                    codes[:off] = _encode(table[codes[:off]] * (old / scale))
                codes[off:off + n] = _encode(x / scale)
                if which == 0:
                    pool_q8[block, s] = codes.reshape(page // 16, 16, -1).transpose(0, 2, 1)
                scales[block, s, which] = scale
        t += n
    return sel_q8, pool_q8, scales


def gather(sel_q8, pool_q8, scales, blocks_of, n, s):
    """Keys [n, d_sel], values [n, d_pool] and a mask of tokens that exist, of one request (its row of the block table) and KV head."""
    n_blocks, _, page, d = sel_q8.shape
    decode = q8.e4m3_decode_table()
    k, v, real = np.zeros((n, d)), np.zeros((n, pool_q8.shape[3])), np.zeros(n, bool)
    for j in range(n):
        blk, at = int(blocks_of[j // page]), j % page
        if 0 <= blk < n_blocks:
            real[j] = True
            k[j] = decode[sel_q8[blk, s, at]] * scales[blk, s, 1]
            v[j] = decode[pool_q8[blk, s, at // 16, :, at % 16]] * scales[blk, s, 0]
    return k, v, real


def attend(q, k, v, pos, n, dtype, scale=1.0, softcap=0.0, slope=0.0, window=0, prefix=0, real=None):
    """One head: rows q [rows, d] at positions pos over keys k [n, d], values v [n, d'].  Returns (O, lse, bound on |dO|, bound on |dlse|).

    What a kernel may be off by: a logit is a sum of d products of fp32 (each rounding 2^-24 of the sum of magnitudes), then the score rule (2^-22 of the cap: an
    exponential and a reciprocal of one unit in the last place; the bias and the change to base 2 and back: 2^-22 of their size) and an exponential (2^-22).  A weight is rounded
    to the type once, which moves the output by half a step of sum p |v|; in fp16 weights of less than 2^-14 of a reference at most 2^8 below the largest
    have an absolute step of 2^-25; sums of n terms in fp32 add n 2^-24; the output is rounded once."""
    rows, S = len(pos), len(k)
    O, lse = np.zeros((rows, v.shape[1])), np.full(rows, -math.inf)
    dO, dL = np.zeros_like(O), np.zeros(rows)
    half = HALF_STEP[dtype]
    for r, i in enumerate(pos):
        j = np.arange(S)
        seen = (j < n) & (i >= 0) & (((j <= i) & ((i - j < window) if window else True)) | (j < prefix))
        if real is not None:
            seen &= real
        j = j[seen]
        if len(j) == 0:
            continue
        products = k[j] @ q[r]
        size = np.abs(k[j]) @ np.abs(q[r]) * abs(scale)
        a = products * scale
        if softcap:
            a = softcap * np.tanh(a / softcap)
        a = a - slope * np.abs(i - j)
        top = a.max()
        if top == -math.inf:
            continue
        w = np.exp(a - top)
        total = w.sum()
        O[r] = w @ v[j] / total
        lse[r] = top + math.log(total)
        logit = (k.shape[1] + 4) * 2.0 ** -24 * size.max() + 2.0 ** -22 * (softcap + slope * np.abs(i - j).max() + np.abs(a[w > 0]).max() + 2)
        A = w @ np.abs(v[j]) / total
        dO[r] = (half * 1.01 + 2 * logit + len(j) * 2.0 ** -23) * A + half * np.abs(O[r]) + 1e-30
        if dtype == "f16":
            dO[r] += len(j) * 2.0 ** -25 * 2.0 ** 8 * np.abs(v[j]).max() / max(total, 1.0) + 2.0 ** -25
        dL[r] = logit + len(j) * 2.0 ** -24 + 2.0 ** -22 * abs(lse[r])
    return O, lse, dO, dL
