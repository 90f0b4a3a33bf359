"""What the header promises of the serving operators where single cases could miss it: NaN that a row sees, batches whose
indices do not fit together, page tables that are columns of wider ones."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2503_01483_b200 import kurtail
from test_gpu_serving import BF16, DEV, Seqs, ctx, filled_cache, rand  # noqa: F401

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


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("tokens", ["newest", "last tiles", "first tiles", "inside"])
@pytest.mark.parametrize("name,kind", [("k", "scale"), ("k", "shift"), ("v", "scale"), ("v", "shift"), ("v", "inf")])
@pytest.mark.parametrize("far", [False, True])
def test_a_row_that_sees_what_is_no_number_gets_nan(ctx, layout, tokens, name, kind, far):  # noqa: F811
    n = LAYOUTS[layout][1][0]
    if tokens not in token_sets(n):
        pytest.skip("the sequence is too short")
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
