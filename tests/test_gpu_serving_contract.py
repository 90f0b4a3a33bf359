"""What the header promises of the serving operators where single cases could miss it: NaN that a row sees, batches whose
indices do not fit together, page tables that are columns of wider ones."""
import threading

import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2503_01483_b200 import kurtail
from test_gpu_serving import BF16, DEV, Seqs, close_attention, ctx, filled_cache, host, rand, rope_table  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------- NaN that a row sees
# rows and lengths of the sequences, query heads a key head, bits: blocks of 8 and 16 rows joined by a CTA a row, many blocks
# joined by a warp a row, a prompt in one piece, prompts in chunks
LAYOUTS = {"few": ([1], [897], 4, 4), "few16": ([4], [1000], 4, 8), "long": ([1], [20000], 2, 8), "short": ([1], [33], 4, 4),
           "many": ([1] * 21, [897] * 21, 4, 4), "prompt": ([40], [300], 4, 8), "chunks": ([40], [5000], 4, 4)}


def poisoned(layout, name, tokens, far, kind, seed=3):
    """A cache of two key heads; head 0 of the first sequence's `tokens` holds no number (NaN, or an infinity, in the keys' or
    the values' scale or shift); `far`: the keys of these tokens, but for one of those whose keys are broken, give scores more
    than 170 binary orders below the others'."""
    rows, lengths, group, bits = LAYOUTS[layout]
    sq = Seqs(rows, lengths, 32, seed=seed, pad=1)
    cache, _, _ = filled_cache(sq, 2, 128, bits, seed=seed, garbage=False)
    where = [sq.at(0, j) for j in tokens]
    p, o = torch.tensor([w[0] for w in where], device=DEV), torch.tensor([w[1] for w in where], device=DEV)
    if far:
        cache.k_codes[p, 0, o] = 0
        cache.k_steps[p, 0, o] = torch.tensor([0.1, -10.0], device=DEV)   # q.k <= -1280: a score of -113 and less
    steps = cache.k_steps if name == "k" else cache.v_steps
    which, value = {"scale": (0, float("nan")), "shift": (1, float("nan")), "inf": (1, float("inf"))}[kind]
    last = slice(-1, None) if far and name == "k" else slice(None)
    steps[p[last], 0, o[last], which] = value
    q = (1.0 + 0.1 * rand(seed + 1, sq.N, 2 * group * 128).abs()).to(BF16).to(DEV)
    return sq, cache, q, group, [j for j in tokens][last]


def token_sets(n):
    sets = {"newest": [n - 1], "last tiles": list(range(max(0, n - 104), n)), "first tiles": list(range(min(n, 128)))}
    if n > 600:
        sets["inside"] = list(range(384, 512))
    return sets


@pytest.mark.parametrize("layout,tokens", [(x, t) for x in LAYOUTS for t in token_sets(LAYOUTS[x][1][0])])
@pytest.mark.parametrize("name,kind", [("k", "scale"), ("k", "shift"), ("v", "scale"), ("v", "shift"), ("v", "inf")])
@pytest.mark.parametrize("far", [False, True])
def test_a_row_that_sees_what_is_no_number_gets_nan(ctx, layout, tokens, name, kind, far):  # noqa: F811
    n = LAYOUTS[layout][1][0]
    sq, cache, q, group, broken = poisoned(layout, name, token_sets(n)[tokens], far, kind)
    batch = sq.batch(ctx, cache, 2 * group)
    lse = torch.zeros(sq.N, 2 * group, device=DEV)
    out = ctx.kv_attend(cache, batch, q, out=torch.zeros_like(q), lse=lse)
    ctx.check()
    out, lse = out.view(sq.N, 2 * group, 128).cpu(), lse.cpu()
    sees = so.visible(sq.rows[0], n)[:, broken].any(1)
    for r in range(sq.N - sq.pad):
        nan = r < sq.rows[0] and bool(sees[r])
        assert bool(out[r, :group].isnan().all() if nan else out[r, :group].isfinite().all()), r
        assert bool(lse[r, :group].isnan().all() if nan else lse[r, :group].isfinite().all()), r
        assert bool(out[r, group:].isfinite().all()) and bool(lse[r, group:].isfinite().all())   # the other key head


@pytest.mark.parametrize("layout", ["few", "few16", "many", "chunks"])
def test_a_large_step_of_no_weight_beside_flat_values(ctx, layout):  # noqa: F811
    # all values are one number each (scale 0), but for a token of a large scale whose probability is 0 in float32
    sq, cache, q, group, _ = poisoned(layout, "v", [200], True, "shift")
    p, o = sq.at(0, 200)
    cache.v_steps[..., 0] = 0.0
    cache.v_steps[..., 1] = rand(5, *cache.v_steps.shape[:3]).to(DEV)
    batch = sq.batch(ctx, cache, 2 * group)
    want = ctx.kv_attend(cache, batch, q).clone()
    mid = 2.0 ** (cache.bits - 1)
    for big in (2.0**26, 2.0**40, 2.0**90):
        cache.v_steps[p, 0, o] = torch.tensor([big, -mid * big], device=DEV)
        got = ctx.kv_attend(cache, batch, q)
        ctx.check()
        sees = so.visible(sq.rows[0], sq.lengths[0])
        for r in range(sq.rows[0]):   # (the token's own row, in a prompt, gives it some weight)
            if sees[r].sum() > 300:
                assert torch.equal(got[r], want[r]), (big, r)
        assert torch.equal(got[sq.rows[0] :][: -sq.pad], want[sq.rows[0] :][: -sq.pad])


# ------------------------------------------------------------------------------------------------- host bounds
@pytest.mark.parametrize("max_rows,group,fits", [(2**28, 16, False), (2**30, 2, False), (2**30, 64, False), (2**27, 16, False),
                                                 (2**30, 1, True), (2**27, 15, True)])
def test_rows_of_a_key_head_are_counted_in_32_bits(ctx, max_rows, group, fits):  # noqa: F811
    sq = Seqs([1], [30], 16)
    cache = kurtail.KvCache.empty(sq.pages, 1, 16, 64, 4, DEV)
    if fits:
        assert sq.batch(ctx, cache, group, max_rows=max_rows).max_rows == max_rows   # (nothing is launched)
        return
    with pytest.raises(kurtail.KtError) as e:
        sq.batch(ctx, cache, group, max_rows=max_rows)
    assert e.value.status == 2


# ------------------------------------------------------------------------------------------------- row starts of an append
def test_append_skips_sequences_whose_rows_do_not_fit_and_says_so(ctx):  # noqa: F811
    # long sequences, so that a row that is taken for another one still has a position of the sequence
    hd, page, length = 64, 16, 300
    k = rand(1, 9, hd).to(BF16).to(DEV)
    q = rand(2, 9, 2 * hd).to(BF16).to(DEV)
    for starts, max_rows, skipped in (([0, 3, 6, 10], 5, [2]),        # past the matrices
                                      ([0, 3, 6, 9], 2, [0, 1, 2]),   # more rows than the bound
                                      ([0, 5, 7, 9], 4, [0]),
                                      ([-2, 3, 6, 9], 5, [0])):
        sq = Seqs([3, 3, 3], [length] * 3, page)
        cache = kurtail.KvCache.empty(sq.pages, 1, page, hd, 8, DEV)
        batch = sq.batch(ctx, cache, 2, max_rows=max_rows)
        batch.row_starts.copy_(torch.tensor(starts, dtype=torch.int32))
        out = torch.full_like(q, 55.0)
        ctx.kv_append(cache, batch, q, k, k, q_out=out)
        with pytest.raises(kurtail.KtError) as e:
            ctx.check()
        assert e.value.status == 12, starts
        left = torch.ones(9, dtype=torch.bool)
        for s in range(3):
            a, b = starts[s], starts[s + 1]
            written = [bool(cache.k_codes[p, 0, o].any()) for p, o in (sq.at(s, j) for j in range(length))]
            if s in skipped:
                assert not any(written), (starts, s)
            else:
                assert written == [False] * (length - b + a) + [True] * (b - a), (starts, s)
                left[a:b] = False
        assert bool((out.cpu()[left] == 55.0).all()) and bool((out.cpu()[~left] != 55.0).any(1).all()), starts


def test_append_says_so_where_starts_do_not_ascend(ctx):  # noqa: F811
    hd, page = 64, 16
    sq = Seqs([3, 3, 3], [300] * 3, page)
    cache = kurtail.KvCache.empty(sq.pages, 1, page, hd, 8, DEV)
    k = rand(1, 9, hd).to(BF16).to(DEV)
    for starts in ([0, 6, 3, 9], [0, 4, 2, 4]):   # (rows between two such starts have no owner, or two)
        batch = sq.batch(ctx, cache, 1, max_rows=9)
        batch.row_starts.copy_(torch.tensor(starts, dtype=torch.int32))
        ctx.kv_append(cache, batch, None, k, k)
        with pytest.raises(kurtail.KtError) as e:
            ctx.check()
        assert e.value.status == 12, starts


def test_rows_in_front_of_the_first_sequence_belong_to_none(ctx):  # noqa: F811
    hd, page = 64, 16
    sq = Seqs([2, 1], [40, 33], page)
    k, q = rand(1, 6, hd).to(BF16).to(DEV), rand(2, 6, 2 * hd).to(BF16).to(DEV)
    got = []
    for front in (0, 2):
        cache = kurtail.KvCache.empty(sq.pages, 1, page, hd, 8, DEV)
        batch = sq.batch(ctx, cache, 2)
        batch.row_starts.add_(front)
        out = torch.full_like(q, 55.0)
        shift = lambda t: t.roll(front, 0)  # noqa: E731
        ctx.kv_append(cache, batch, shift(q), shift(k), shift(k), q_out=out)
        ctx.kv_attend(cache, batch, out, out=out)
        ctx.check()
        assert bool((out[:front] == 55.0).all()) and bool((out[front + 3 :] == 55.0).all())
        got.append((out[front : front + 3].clone(), cache.k_codes))
    for a, b in zip(*got):
        assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------- page tables
@pytest.mark.parametrize("rows,group", [([2, 1], 4), ([70, 9], 4)])
def test_lengths_past_a_tables_own_columns_are_skipped(ctx, rows, group):  # noqa: F811
    hd, page = 64, 16
    sq = Seqs(rows, [90, 40], page)
    cache, _, _ = filled_cache(sq, 1, hd, 8, seed=8, garbage=False)
    q = rand(2, sq.N, group * hd).to(BF16).to(DEV)
    k = rand(3, sq.N, hd).to(BF16).to(DEV)
    batch = sq.batch(ctx, cache, group, max_length=1000)
    want = ctx.kv_attend(cache, batch, q).clone()
    n = sq.table.shape[1]
    wide = torch.zeros(2, n + 7, dtype=torch.int32, device=DEV)      # ids that a cache has, around the table
    wide[:, 5 : 5 + n] = batch.page_table
    part = ctx.kv_batch(cache, group, batch.row_starts, batch.lengths, wide[:, 5 : 5 + n], max(rows), 1000)
    assert torch.equal(ctx.kv_attend(cache, part, q), want)
    ctx.check()
    part.lengths[1] = n * page + 1                                    # one token behind the last row's own columns
    out = torch.full_like(q, 55.0)
    ctx.kv_attend(cache, part, q, out=out)
    with pytest.raises(kurtail.KtError) as e:
        ctx.check()
    assert e.value.status == 12
    assert torch.equal(out[: rows[0]], want[: rows[0]]) and bool((out[rows[0] :] == 55.0).all())
    qo = torch.full_like(q, 55.0)
    ctx.kv_append(cache, part, q, k, k, q_out=qo)
    with pytest.raises(kurtail.KtError) as e:
        ctx.check()
    assert e.value.status == 12
    assert bool((qo[: rows[0]] != 55.0).any(1).all()) and bool((qo[rows[0] :] == 55.0).all())
    other = kurtail.KvCache.empty(30, 1, 32, hd, 8, DEV)
    for call in (lambda: ctx.kv_attend(other, part, q), lambda: ctx.kv_append(other, part, q, k, k)):
        with pytest.raises(ValueError):
            call()


# ------------------------------------------------------------------------------------------------- single rows
def test_a_row_is_one_whatever_its_stride(ctx):  # noqa: F811
    hd = 64
    x = rand(1, 4 * hd, 1).to(BF16).to(DEV).t()                          # one row, contiguous, of stride 1
    assert x.stride(0) == 1
    c, s, v = ctx.rmsnorm_quant(x, residual=x, bits=8, values=torch.empty_like(x), codes=torch.empty(1, 4 * hd, dtype=torch.int8, device=DEV))
    wc, ws, wv = ctx.rmsnorm_quant(x.clone(memory_format=torch.contiguous_format).view(1, -1), residual=x.reshape(-1)[None], bits=8,
                                   values=torch.empty(1, 4 * hd, dtype=BF16, device=DEV),
                                   codes=torch.empty(1, 4 * hd, dtype=torch.int8, device=DEV))
    assert torch.equal(c, wc) and torch.equal(s, ws) and torch.equal(v, wv)
    sq = Seqs([1], [40], 16)
    caches = [kurtail.KvCache.empty(sq.pages, 1, 16, hd, 8, DEV) for _ in range(2)]
    outs = []
    for cache, q in zip(caches, (x, x.reshape(-1)[None])):
        batch = sq.batch(ctx, cache, 4)
        outs.append(ctx.kv_attend(cache, batch, ctx.kv_append(cache, batch, q, q[:, :hd], q[:, hd : 2 * hd])))
    ctx.check()
    assert torch.equal(*outs) and torch.equal(caches[0].k_codes, caches[1].k_codes)


# ------------------------------------------------------------------------------------------------- many sequences, many heads
@pytest.mark.parametrize("hd,bits,most_rows", [(64, 4, 2), (128, 8, 3), (64, 8, 40)])
def test_thousands_of_sequences(ctx, hd, bits, most_rows):  # noqa: F811
    # more than the attention's list keeps sums of, and three levels of the append's search
    g = np.random.RandomState(hd)
    n, heads, group = 4100, 1, 4
    rows = g.randint(0, most_rows + 1, n) * (g.rand(n) < 0.7)
    lengths = rows + np.where(g.rand(n) < 0.5, 0, g.randint(0, 60, n))
    lengths[g.rand(n) < 0.002] += 400
    sq = Seqs(rows, lengths, 16, seed=1, pad=5)
    cache, codes, steps = filled_cache(sq, heads, hd, bits, seed=2)
    q = rand(1, sq.N, heads * group * hd).to(BF16).to(DEV)
    batch = sq.batch(ctx, cache, heads * group)
    some = [s for s in [0, 1, 31, 32, 1023, 1024, 1025, n - 1, *np.argsort(-lengths)[:4], *g.randint(0, n, 60)]]
    close_attention(ctx, cache, codes, steps, sq, q, batch, hd, heads, group, hd**-0.5, True, 0, sequences=some)
    # each row of the append lands where a call for its sequence alone puts it
    k = rand(3, sq.N, hd).to(BF16).to(DEV)
    rope = rope_table(int(lengths.max()), hd)
    into = kurtail.KvCache.empty(sq.pages, 1, 16, hd, bits, DEV)
    ctx.kv_append(into, batch, None, k, k, rope=rope, hadamard=True)
    ctx.check()
    i32 = lambda a: torch.tensor(np.asarray(a, np.int32), device=DEV)  # noqa: E731
    alone = kurtail.KvCache.empty(sq.pages, 1, 16, hd, bits, DEV)
    for s in some:
        r = int(rows[s])
        one = ctx.kv_batch(alone, 1, i32([0, r]), i32([lengths[s]]), i32(sq.table[s : s + 1]), max(r, 1), max(int(lengths[s]), 1))
        part = k[int(sq.starts[s]) : int(sq.starts[s]) + r]
        ctx.kv_append(alone, one, None, part, part, rope=rope, hadamard=True)
        used = [p for p in sq.table[s, : -(-int(lengths[s]) // 16)]]
        for a, b in ((into.k_codes, alone.k_codes), (into.v_steps, alone.v_steps)):
            assert torch.equal(a[used], b[used]), s
    assert int((into.k_steps[..., 0] > 0).sum()) == int(rows.sum())
    ctx.check()


@pytest.mark.parametrize("group", [100, 128, 129, 200, 300])
def test_many_query_heads_on_one_key_head(ctx, group):  # noqa: F811
    sq = Seqs([1, 0, 1], [300, 10, 40], 32, pad=1)
    cache, codes, steps = filled_cache(sq, 1, 64, 4, seed=2)
    q = rand(1, sq.N, group * 64).to(BF16).to(DEV)
    close_attention(ctx, cache, codes, steps, sq, q, sq.batch(ctx, cache, group), 64, 1, group, 0.125, True, 0)


@pytest.mark.parametrize("rows,group", [([2, 3], 4), ([70, 9], 4)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_query_that_is_no_number_touches_its_own_row_only(ctx, rows, group, value):  # noqa: F811
    hd = 64
    sq = Seqs(rows, [r + 200 for r in rows], 32)
    cache, _, _ = filled_cache(sq, 2, hd, 8, seed=2)
    q = rand(1, sq.N, 2 * group * hd).to(BF16).to(DEV)
    batch = sq.batch(ctx, cache, 2 * group)
    lse = [torch.zeros(sq.N, 2 * group, device=DEV) for _ in range(2)]
    want = ctx.kv_attend(cache, batch, q, lse=lse[0]).clone()
    q[1, 3 * hd + 7] = value
    got = ctx.kv_attend(cache, batch, q, lse=lse[1])
    ctx.check()
    hit = torch.zeros(sq.N, 2 * group, dtype=torch.bool, device=DEV)
    hit[1, 3] = True
    got, want = got.view(sq.N, 2 * group, hd), want.view(sq.N, 2 * group, hd)
    assert torch.equal(got[~hit], want[~hit]) and torch.equal(lse[0][~hit], lse[1][~hit])
    assert bool(got[hit].isnan().all()) and bool(lse[1][hit].isnan().all())


# ------------------------------------------------------------------------------------------------- threads
def test_threads_with_a_context_each():
    """Calls of several shapes from three threads at once, the first of a shape among them, against calls in a row."""
    shapes = [(64, 4, [1, 1], 2), (64, 8, [3], 4), (128, 4, [2, 1], 8), (128, 8, [1], 3), (64, 4, [70], 2), (128, 8, [40, 1], 4)]
    cases = []
    for i, (hd, bits, rows, group) in enumerate(shapes):
        sq = Seqs(rows, [r + 500 for r in rows], 32, seed=i)
        cache, _, _ = filled_cache(sq, 2, hd, bits, seed=i, garbage=False)
        x = rand(i, sq.N, 2 * (group + 1) * hd).to(BF16).to(DEV)
        cases.append((sq, cache, x[:, : 2 * group * hd], x[:, 2 * group * hd :], 2 * group))
    torch.cuda.synchronize()
    results, errors = [None] * 4, []

    def work(n):
        try:
            c = kurtail.Context(DEV, stream=torch.cuda.Stream(DEV))
            got = []
            with torch.cuda.stream(c.stream):
                for sq, cache, q, k, heads in cases:
                    own = kurtail.KvCache(*(t.clone() for t in (cache.k_codes, cache.v_codes, cache.k_steps, cache.v_steps)), cache.bits)
                    batch = sq.batch(c, own, heads)
                    _, s, v = c.rmsnorm_quant(q, bits=8, values=torch.empty(q.shape, dtype=BF16, device=DEV))
                    qt = c.kv_append(own, batch, v, k, k, hadamard=True)
                    got.append((s, qt, c.kv_attend(own, batch, qt), own.k_codes))
                c.check()
            results[n] = got
            c.close()
        except Exception as e:   # (a thread's own failure would be lost)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(n,)) for n in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    work(3)
    assert not errors, errors
    for n in range(3):
        for a, b in zip(results[n], results[3]):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


# ------------------------------------------------------------------------------------------------- roundings of few rows
@pytest.mark.parametrize("rows,lengths,group", [([1] * 4, [1, 2, 3, 40], 4), ([3, 1, 2], [3, 70, 200], 4), ([1], [900], 8)])
@pytest.mark.parametrize("hd,bits", [(128, 4), (128, 8), (64, 4), (64, 8)])
def test_few_rows_round_products_to_float16_and_no_further(ctx, rows, lengths, group, hd, bits):  # noqa: F811
    """Values whose codes lie at one end of their range and whose shifts bring them near zero: the result is small beside the
    products p s u that it is summed from, so their rounding shows (with bf16 it is 8 times the bound).

    Keys are flat (scale 0), so a score is shift times sum(q), in float32: the sum of hd terms, at most hd / 4 + 2 of them one
    after another in a lane and across lanes, and four products, 2^-24 each; the exponential 2^-22 of itself.  With |score| <= S
    a probability is off by the factor exp(2 (hd / 4 + 6) 2^-24 S) and 2^-21.  p s: half a step of float16, 2^-11 of itself, and
    of float16's smallest step, 2^-25 against a largest of at least 2^2 (2^-27 of it; 2^-26 leaves room for a reference that
    moved).  Sums in float32: 2^-24 for each of the sequence's tokens and runs.  The result: half a step of bf16, 2^-8.  In norm
    that last error is uniform: 2^-8 / sqrt(3)."""
    mid = 2 ** (bits - 1)
    sq = Seqs(rows, lengths, 16, seed=bits)
    g = np.random.RandomState(hd + bits)
    shape = (sq.pages, 2, 16)
    u = {n: g.randint(2 * mid - mid // 4, 2 * mid, (*shape, hd)).astype(np.uint8) for n in "kv"}
    k_steps = np.stack((np.zeros(shape), g.uniform(-1.0, 1.0, shape)), -1).astype(np.float32)
    scale_v = g.uniform(0.5, 1.5, shape)
    v_steps = np.stack((scale_v, -scale_v * (2 * mid - mid / 8)), -1).astype(np.float32)
    dev = lambda a: torch.tensor(a, device=DEV)  # noqa: E731
    cache = kurtail.KvCache(dev(so.pack(u["k"], bits)), dev(so.pack(u["v"], bits)), dev(k_steps), dev(v_steps), bits)
    q = rand(bits, sq.N, 2 * group * hd).abs().to(BF16).to(DEV)
    out = ctx.kv_attend(cache, sq.batch(ctx, cache, 2 * group), q, scale=1.0 / hd)
    ctx.check()
    got, err, ref, rest = host(out).astype(np.float64), [], [], []
    for s, (r, n) in enumerate(zip(rows, lengths)):
        at = np.array([sq.at(s, j) for j in range(n)])
        at = (at[:, 0], at[:, 1])
        see = so.visible(r, n)
        for head in range(2 * group):
            kh = head // group
            cols, own = slice(head * hd, (head + 1) * hd), slice(sq.starts[s], sq.starts[s + 1])
            part = [a[at[0], kh, at[1]] for a in (u["k"], k_steps, u["v"], v_steps)]
            qq = host(q[own, cols])
            o, _, spread, size = so.attend(qq, *part, see, 1.0 / hd)
            S = np.abs(qq).astype(np.float64).sum(1).max() / hd
            moves = np.expm1(2 * (hd / 4 + 6) * 2.0**-24 * S) + 2.0**-21 + n * 2.0**-24
            # (a term p v enters as p s (u - middle) and p times the middle's value)
            parts = spread + np.abs(part[3][:, 0] * mid + part[3][:, 1]).max()
            low = 2.0**-26 * part[3][:, 0].max() * mid * n
            tol = (2.0**-11 * 1.001) * spread + 2 * moves * parts + low
            diff = np.abs(got[own, cols] - o)
            assert (diff <= 2.0**-8 * (np.abs(o) + tol) + tol).all(), np.max(diff / (2.0**-8 * np.abs(o) + tol))
            err.append(diff.ravel()), ref.append(o.ravel()), rest.append(tol.ravel())
    norm = lambda x: np.linalg.norm(np.concatenate(x))  # noqa: E731
    assert norm(err) <= 1.05 * 2.0**-8 / np.sqrt(3.0) * norm(ref) + norm(rest)


# ------------------------------------------------------------------------------------------------- the ends of float32
@pytest.mark.parametrize("asym", [True, False])
@pytest.mark.parametrize("bits", [4, 8])
def test_heads_whose_steps_pass_float32_are_no_numbers(ctx, asym, bits):  # noqa: F811
    # symmetric: the shift is -2^(bits - 1) times the scale, past float32 for a head that is within it
    hd = 64
    x = torch.zeros(4, hd, device=DEV)
    x[0], x[1, 3], x[2, 3], x[3, 5], x[3, 6] = 1.0, 3.4e38, 2.5e38, 3e38, -3e38
    cache = kurtail.KvCache.empty(1, 1, 16, hd, bits, DEV)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    batch = ctx.kv_batch(cache, 1, i32(0, 4), i32(4), i32(0)[None], 4, 4)
    values = torch.zeros(4, hd, dtype=BF16, device=DEV)
    ctx.kv_append(cache, batch, None, x, x, asymmetric=asym, v_values=values)
    ctx.check()
    with np.errstate(all="ignore"):
        _, s, b, _ = so.held(x.cpu().numpy()[:, None], bits, asym, np.float32(1.0))
    good = np.isfinite(s[:, 0]) & np.isfinite(b[:, 0])
    assert good[0] and good[2] and not good[3 if asym else 1]
    got = cache.v_steps[0, 0, :4].cpu().numpy()
    assert np.array_equal(got[good, 0], s[good, 0]) and np.array_equal(got[good, 1], b[good, 0])
    assert np.isnan(got[~good]).all() and bool(values[torch.tensor(~good)].isnan().all())
    assert int(cache.v_codes[0, 0, :4][torch.tensor(~good)].max()) == 0
