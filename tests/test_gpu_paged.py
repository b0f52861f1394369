"""Rows written into pages, as they are and in 8 bits, and read back: every slot of the pools against plain indexing on the CPU."""
import pytest
import torch

import paper_2503_01840_amd as E

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROW = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.bfloat16}
CACHED = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.float8_e4m3fn}
INF, NAN = float("inf"), float("nan")
i32 = lambda v: torch.tensor(v, dtype=torch.int32)


def quantised(x):
    """(codes as bytes, exponent bytes) of bf16 rows, from the definition, in 64 bits on the CPU."""
    x = x.double()
    mag = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    e = torch.full_like(mag, -110)
    for _ in range(240):                                     # the smallest exponent that covers the row
        e = torch.where(mag > 448 * torch.exp2(e), e + 1, e)
    y = x / torch.exp2(e)[..., None]
    ok = torch.isfinite(y)
    z = torch.where(ok, y, torch.zeros_like(y))
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
    z = torch.round(z / step) * step                         # ties to even
    z = torch.where((e == 120)[..., None], z.clamp(-240, 240), z)            # 256 * 2^120 is no bf16 value; 240 is as near as half a step of 2^-4
    codes = z.float().to(torch.float8_e4m3fn).view(torch.uint8)
    codes = torch.where((z == 0) & torch.signbit(y), torch.full_like(codes, 0x80), codes)
    return torch.where(ok, codes, torch.full_like(codes, 0x7F)), (e + 127).to(torch.uint8)


def value(codes, exps):
    return codes.view(torch.float8_e4m3fn).double() * torch.exp2(exps.double() - 127)[..., None]


def make_cache(dtype, B, max_pages, page, Hkv, d, g, spare=3):
    """A pool filled with noise, its pages dealt to B sequences in random order."""
    n_pages = B * max_pages + spare
    table = torch.randperm(n_pages, generator=g)[:B * max_pages].view(B, max_pages).int()
    if dtype == "fp8":
        k, v = (torch.randint(0, 120, (n_pages, page, Hkv, d), generator=g, dtype=torch.uint8).view(torch.float8_e4m3fn).to(DEV) for _ in range(2))
        exps = [torch.randint(100, 140, (n_pages, page, Hkv), generator=g, dtype=torch.uint8).to(DEV) for _ in range(2)]
    else:
        k, v = (torch.randn(n_pages, page, Hkv, d, generator=g).to(ROW[dtype]).to(DEV) for _ in range(2))
        exps = [None, None]
    return E.PagedKVCache(k, v, table.to(DEV), *exps), table


def raw(t):
    return None if t is None else t.view(torch.uint8).cpu() if t.dtype == torch.float8_e4m3fn else t.cpu()


def pools(c):
    return [raw(t) for t in (c.k, c.v, c.k_exp, c.v_exp)]


def same(a, b):
    return a.dtype == b.dtype and torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# dtype, heads, dim, page size, pages a sequence, first tokens, rows of each sequence
CASES = [("bf16", 8, 128, 16, 9, [0, 130, 15, 16, 143], [1, 14, 1, 0, 1]),
         ("fp8", 8, 128, 16, 9, [0, 130, 15, 16, 143], [1, 14, 1, 0, 1]),
         ("fp32", 8, 128, 16, 9, [0, 130, 15, 16, 143], [1, 14, 1, 0, 1]),
         ("fp8", 1, 64, 1, 70, [3, 0], [66, 70]), ("bf16", 3, 64, 1, 70, [3, 0], [66, 70]), ("fp32", 3, 64, 7, 30, [20], [190]),
         ("fp8", 3, 64, 13, 30, [5, 1, 77], [200, 100, 313]), ("bf16", 5, 128, 100, 6, [1, 99], [599, 1]), ("fp8", 5, 128, 256, 3, [0, 511], [768, 257]),
         ("fp8", 8, 128, 64, 40, [17] * 4, [2500, 1, 64, 777]), ("fp8", 2, 128, 33, 1, [0], [1]), ("bf16", 40, 128, 32, 2, [31] * 70, [1] * 70),
         ("fp8", 40, 128, 32, 2, [31] * 70, [2] * 70)]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("packed", [False, True])
def test_append_and_read(case, packed):
    dtype, Hkv, d, page, max_pages, start, n = case
    B, g = len(n), torch.Generator().manual_seed(len(n) * 7 + d + page)
    c, table = make_cache(dtype, B, max_pages, page, Hkv, d, g)
    first, at = [], 2                                        # two rows that belong to no sequence, and one behind each
    for m in n:
        first.append(at)
        at += m + 1
    scale = torch.exp2(torch.randint(-20, 20, (at, 3 * Hkv, 1), generator=g).float())
    rows = (torch.randn(at, 3 * Hkv, d, generator=g) * scale).to(ROW[dtype])
    rows[2, 0] = 0                                           # a row of zeros
    k, v = rows[:, :Hkv], rows[:, 2 * Hkv:]
    dk, dv = (rows.to(DEV)[:, :Hkv], rows.to(DEV)[:, 2 * Hkv:]) if packed else (k.contiguous().to(DEV), v.contiguous().to(DEV))
    want = [t if t is None else t.clone() for t in pools(c)]
    E.eagle3_paged_append(c, dk, dv, i32(start).to(DEV), i32(n).to(DEV), rows=max(n), row_start=i32(first).to(DEV))
    sources = [(quantised(t) if dtype == "fp8" else (t, None)) for t in (k, v)]
    for b, m in enumerate(n):
        for j in range(m):
            p = start[b] + j
            s = (int(table[b, p // page]), p % page)
            for i in range(2):
                want[i][s] = sources[i][0][first[b] + j]
                if dtype == "fp8":
                    want[2 + i][s] = sources[i][1][first[b] + j]
    for got, w in zip(pools(c), want):
        assert (got is None and w is None) or same(got, w)
    # and back
    out = tuple(torch.full((at, Hkv * (2 if packed else 1), d), 3.0, dtype=ROW[dtype], device=DEV) for _ in range(2))
    E.eagle3_paged_read(c, i32(start).to(DEV), i32(n).to(DEV), rows=max(n), row_start=i32(first).to(DEV), out=tuple(o[:, :Hkv] for o in out))
    back = [torch.full((at, out[0].shape[1], d), 3.0, dtype=ROW[dtype]) for _ in range(2)]
    for b, m in enumerate(n):
        for i in range(2):
            x = sources[i][0][first[b]:first[b] + m]
            back[i][first[b]:first[b] + m, :Hkv] = value(x, sources[i][1][first[b]:first[b] + m]).to(ROW[dtype]) if dtype == "fp8" else x
    for got, w in zip(out, back):
        assert same(got.cpu(), w)


def test_eight_bits_of_every_bf16_value():
    """All 65536 bf16 bit patterns, each in a row whose largest magnitude puts it somewhere else in the codes' range; and the read-back is exact."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    g = torch.Generator().manual_seed(3)
    x = bits[torch.randperm(65536, generator=g)].view(64, 8, 128)
    x = torch.cat([x, bits.view(64, 8, 128)])                 # neighbours beside each other: rows of one magnitude
    c, table = make_cache("fp8", 1, 2, 64, 8, 128, g)
    E.eagle3_paged_append(c, x.to(DEV), x.flip(2).contiguous().to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV))
    (ck, ek), (cv, ev) = quantised(x), quantised(x.flip(2))
    t = table[0].long()
    pk, pv, pke, pve = pools(c)
    nan = lambda b: (b & 0x7F) == 0x7F
    for got, w, ge, we in ((pk[t], ck, pke[t], ek), (pv[t], cv, pve[t], ev)):
        assert torch.equal(ge.reshape(we.shape), we) and torch.equal(got.reshape(w.shape), w)
    k, _ = E.eagle3_paged_read(c, rows=128)
    ref = value(ck, ek)
    assert torch.equal(torch.isnan(k.cpu()), nan(ck))
    ok = ~nan(ck)
    assert torch.equal(k.cpu().double()[ok], ref[ok])
    # the error of a code: half a step relative to the value, or half the smallest step of the row's scale
    err = (ref - x.double()).abs()[ok]
    assert bool((err <= torch.maximum(2.0 ** -4 * x.double().abs(), 2.0 ** -10 * torch.exp2(ek.double() - 127)[..., None].expand_as(ref))[ok]).all())


def test_rows_that_have_no_place_are_dropped():
    """Positions before the first and behind the last page, pages outside the pool, source rows outside the array, counts beyond `rows`."""
    for dtype in ("bf16", "fp8", "fp32"):
        g = torch.Generator().manual_seed(5)
        B, page, max_pages, Hkv, d = 7, 4, 3, 2, 64
        c, table = make_cache(dtype, B, max_pages, page, Hkv, d, g)
        table[2, 1], table[3, 1] = -1, c.k.shape[0]
        c.page_table.copy_(table)
        start = i32([-2, 10, 2, 2, 0, 0, 2 ** 31 - 1])
        n = i32([5, 5, 5, 5, -3, 99, 5])
        row_start = i32([0, 5, 10, 15, 20, 28, 0])              # the sixth sequence's rows 28.. end at 30
        rows = torch.randn(30, Hkv, d, generator=g).to(ROW[dtype])
        want = [t if t is None else t.clone() for t in pools(c)]
        src = quantised(rows) if dtype == "fp8" else (rows, None)
        for b, cnt in enumerate([5, 5, 5, 5, 0, 5, 5]):
            for j in range(cnt):
                p, r = int(start[b]) + j, int(row_start[b]) + j
                if not (0 <= p < page * max_pages and 0 <= r < 30 and 0 <= int(table[b, p // page]) < c.k.shape[0]):
                    continue
                s = (int(table[b, p // page]), p % page)
                for i in range(2):
                    want[i][s] = src[0][r]
                    if dtype == "fp8":
                        want[2 + i][s] = src[1][r]
        E.eagle3_paged_append(c, rows.to(DEV), rows.to(DEV), start.to(DEV), n.to(DEV), rows=5, row_start=row_start.to(DEV))
        for got, w in zip(pools(c), want):
            assert (got is None and w is None) or same(got, w)
        out = tuple(torch.full((30, Hkv, d), 3.0, dtype=ROW[dtype], device=DEV) for _ in range(2))
        E.eagle3_paged_read(c, start.to(DEV), n.to(DEV), rows=5, row_start=row_start.to(DEV), out=out)
        kept = [1, 2, 3, 4, 7, 8, 9, 12, 13, 14, 17, 18, 19] + list(range(20, 28))   # in no place, on no page
        written = sorted(set(range(30)) - set(kept) - {0, 1})
        assert bool((out[0].cpu()[written] != 3.0).any(-1).all()) and bool((out[0].cpu()[20:28] == 3.0).all())
        assert bool((out[0].cpu()[[7, 8, 9, 12, 13, 14, 17, 18, 19]] == 3.0).all()) and bool((out[0].cpu()[:2] == 3.0).all())


def test_defaults_and_shared_pages():
    """No counts and no first rows: `rows` of every sequence, one behind the other; two sequences that share their first page read the same."""
    g = torch.Generator().manual_seed(6)
    c, table = make_cache("fp8", 3, 4, 8, 2, 128, g)
    x = torch.randn(3 * 5, 2, 128, generator=g).bfloat16()
    E.eagle3_paged_append(c, x.to(DEV), x.to(DEV), i32([0, 9, 27]).to(DEV))
    k, v = E.eagle3_paged_read(c, i32([0, 9, 27]).to(DEV), rows=5)
    want = value(*quantised(x)).bfloat16()
    assert same(k.cpu(), want) and same(v.cpu(), want)
    table[1, 0] = table[0, 0]
    c.page_table.copy_(table)
    k, _ = E.eagle3_paged_read(c, rows=8)
    assert same(k[:8], k[8:16]) and same(k[:5].cpu(), want[:5])


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_slots_behind_four_gigabytes(dtype):
    """Offsets that 32 bits do not hold: pools of more than 2^32 bytes, a sequence in their last pages."""
    Hkv, d, page = 8, 128, 64
    size = 2 if dtype == "bf16" else 1
    n_pages = (1 << 32) // (page * Hkv * d * size) + 5
    k, v = (torch.zeros(n_pages, page, Hkv, d, dtype=torch.uint8 if size == 1 else torch.bfloat16, device=DEV) for _ in range(2))
    exps = [torch.zeros(n_pages, page, Hkv, dtype=torch.uint8, device=DEV) for _ in range(2)] if size == 1 else [None, None]
    k, v = (t.view(torch.float8_e4m3fn) if size == 1 else t for t in (k, v))
    c = E.PagedKVCache(k, v, i32([[n_pages - 1, 0, n_pages - 2]]).to(DEV), *exps)
    x = torch.randn(150, Hkv, d, generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    E.eagle3_paged_append(c, x, x.flip(0), i32([10]).to(DEV))
    gk, gv = E.eagle3_paged_read(c, i32([10]).to(DEV), rows=150)
    want = x.cpu() if size == 2 else value(*quantised(x.cpu())).bfloat16()
    assert same(gk.cpu(), want) and same(gv.cpu(), want.flip(0))
    q = torch.randn(1, 32, d, generator=torch.Generator().manual_seed(2)).bfloat16().to(DEV)
    # the same sequence in a small pool
    small = torch.tensor([0, 1, 2])
    pages = c.page_table[0].long()
    s = E.PagedKVCache(k.view(torch.uint8)[pages].view(k.dtype) if size == 1 else k[pages], v.view(torch.uint8)[pages].view(v.dtype) if size == 1 else v[pages],
                       small.int()[None].to(DEV), *[None if e is None else e[pages] for e in exps])
    n = i32([160]).to(DEV)
    c.k[pages[0]].view(torch.uint8)[:10] = 0
    assert same(E.eagle3_paged_attention(c, q, n, 160), E.eagle3_paged_attention(s, q, n, 160))


def test_binding_refuses_what_does_not_fit():
    g = torch.Generator().manual_seed(8)
    c, _ = make_cache("bf16", 2, 3, 8, 2, 64, g)
    f, _ = make_cache("fp8", 2, 3, 8, 2, 64, g)
    x, s = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    bad = [lambda: E.eagle3_paged_append(c, x.float(), x.float(), s), lambda: E.eagle3_paged_append(c, x, x[:2], s),
           lambda: E.eagle3_paged_append(c, x[:3], x[:3], s), lambda: E.eagle3_paged_append(c, x, x, s.long()),
           lambda: E.eagle3_paged_append(c, x, x, s[:1]), lambda: E.eagle3_paged_append(c, x.cpu(), x.cpu(), s),
           lambda: E.eagle3_paged_append(c, x, x, s, rows=2, row_start=s[:1]), lambda: E.eagle3_paged_append(c, x[:, :1], x[:, :1], s),
           lambda: E.eagle3_paged_append(c, x, x, s, row_start=s), lambda: E.eagle3_paged_read(c), lambda: E.eagle3_paged_read(f, out=(x.float(), x.float())),
           lambda: E.eagle3_paged_append(c, x, torch.zeros(4, 4, 64, dtype=torch.bfloat16, device=DEV)[:, :2], s),
           lambda: E.PagedKVCache(c.k, c.v, c.page_table, f.k_exp, f.v_exp), lambda: E.PagedKVCache(f.k, f.v, f.page_table),
           lambda: E.PagedKVCache(c.k, c.v[:-1], c.page_table), lambda: E.PagedKVCache(c.k, c.v, c.page_table.long()),
           lambda: E.PagedKVCache(f.k, f.v, f.page_table, f.k_exp, f.v_exp[:-1]), lambda: E.PagedKVCache(c.k.half(), c.v.half(), c.page_table)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    odd = torch.zeros(4 * 2 * 64 + 8, dtype=torch.bfloat16, device=DEV)[1:1 + 4 * 2 * 64].view(4, 2, 64)
    for call in (lambda: E.eagle3_paged_append(c, odd, odd, s), lambda: E.eagle3_paged_append(c, x[:0], x[:0], s)):
        with pytest.raises(E.Eagle3Error):
            call()
