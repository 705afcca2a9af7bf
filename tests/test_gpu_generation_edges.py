"""Generation from a paged cache where it is easily wrong: sizes at a limit of the launch, numbers that are not finite, weights far below a row's largest."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import generation_oracle as O
from tests.test_gpu_generation import BF16, E4M3, F16, ROUND, cosa, gpu, pools, tables, wide  # noqa: F401

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ---------------------------------------------------------------- page plan
PLANS = """
import numpy as np, paper_2607_25291_b200 as cosa
from oracle import generation_oracle as O
from tests.test_gpu_generation import check_plan
for batch in (3041, 3042, 3043, 3044, 3060, 3071, 3072, 3073, 4000):
    rng = np.random.default_rng(batch)
    lens, grow = rng.integers(0, 20, batch), rng.choice([-1, 0, 1, 9], batch)
    need = sum(O.pages_of(n + g, 8) - O.pages_of(n, 8) for n, g in zip(lens, grow) if g > 0)
    check_plan(cosa, lens, grow, 8, 5, need // 2, int(grow.clip(0).sum()) + 1, 7, rng)
    print("planned", batch)
"""


def test_page_plan_sizes_around_the_shared_memory_limit():
    """In a process of its own, smaller batches first: a larger one would have raised the kernel's limit for all."""
    run = subprocess.run([sys.executable, "-c", PLANS], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout[-500:] + run.stderr[-1500:]
    assert "planned 4000" in run.stdout


# ---------------------------------------------------------------- attention
def contents(lens, hq, hkv, d, page, dtype, cache, seed):
    """q, pools, scales and table of a call with ordinary numbers, and the place of a token in the pools."""
    rng, gen = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    table, pages, _ = tables(lens, page, rng, spare=1)
    k, v = ((torch.randn(pages, hkv, page, d, generator=gen, device="cuda") * (25.0 if cache is E4M3 else 1.0)).to(cache) for _ in range(2))
    ks, vs = (torch.rand(hkv, generator=gen, device="cuda") * 0.05 + 0.01 for _ in range(2)) if cache is E4M3 else (None, None)
    q = torch.randn(len(lens), hq, d, generator=gen, device="cuda").to(dtype)
    return q, k, v, ks, vs, table


def put(pool, table, page, b, h, tokens, channel, x):
    """Writes x into one channel of some tokens."""
    flat = pool.view(torch.uint8) if pool.dtype is E4M3 else pool
    x = torch.tensor(x, device="cuda").to(pool.dtype)
    x = x.view(torch.uint8) if pool.dtype is E4M3 else x
    t = torch.as_tensor(list(tokens), device="cuda")
    flat[gpu(table[b], torch.int64)[t // page], h, t % page, channel] = x


def attend(cosa, q, k, v, ks, vs, table, lens, route):
    handle = cosa.make_cache(k, v, gpu(table), k_scale=ks, v_scale=vs)
    out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:2], 9.0, device="cuda")
    opt = cosa.decode_options(impl=int(route == "check"), ctas=1 if route == "one CTA" else 0)
    if route == "workspace":      # the pieces are joined by a kernel of its own
        space = torch.empty(cosa.cosa_decode_workspace_bytes(1, handle, q.shape[0], q.shape[1]), dtype=torch.uint8, device="cuda")
        opt.workspace, opt.workspace_bytes = space.data_ptr(), space.numel()
    cosa.cosa_decode_attention(handle, q, gpu(lens), out, lse, opt=opt)
    assert cosa.cosa_device_status() == 0
    return out, lse


ROUTES = ["as usual", "one CTA", "workspace", "check"]


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F16, F16), (BF16, E4M3), (F16, E4M3)])
@pytest.mark.parametrize("lens", [[40, 3], [20000, 300]])
@pytest.mark.parametrize("route", ROUTES)
def test_logits_that_are_not_numbers_make_their_heads_nan(cosa, dtype, cache, lens, route):
    """NaN or +inf in a query, one key or a whole run of keys: outputs and lse of the heads that meet it are NaN, however the row is divided; all
    others are those of the call without it, bit by bit."""
    hq, hkv, d, page, n = 6, 2, 64, 16, lens[0]
    inputs = contents(lens, hq, hkv, d, page, dtype, cache, seed=n + d)
    q, k, v, ks, vs, table = inputs
    q[0, :, 3] = q[0, :, 3].abs() + 0.25
    right = attend(cosa, *inputs, lens, route)
    assert all(bool(torch.isfinite(x).all()) for x in right)

    def check(q, k, poisoned):
        out, lse = attend(cosa, q, k, v, ks, vs, table, lens, route)
        bad = torch.zeros(len(lens), hq, dtype=torch.bool, device="cuda")
        bad[0, poisoned] = True
        assert bool(out[bad].isnan().all()) and bool(lse[bad].isnan().all()), (out[bad], lse[bad])
        assert torch.equal(out[~bad], right[0][~bad]) and torch.equal(lse[~bad], right[1][~bad])

    for x in (math.nan, math.inf):
        other = q.clone()
        other[0, 4, 3] = x
        check(other, k, [4])
    some = range(n // 3, n // 3 + max(1, n // 2))
    for x, tokens in ((math.nan, [n - 1]), (math.nan, [0]), (math.nan, some), (math.nan, range(n)), (math.inf, [n // 2]), (math.inf, some)):
        if x == math.inf and cache is E4M3:
            continue      # (e4m3 has none)
        other = k.clone()
        put(other, table, page, 0, 1, tokens, 3, x)
        check(q, other, [3, 4, 5])


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F16, F16)])
@pytest.mark.parametrize("n", [40, 20000])
@pytest.mark.parametrize("route", ROUTES)
def test_logits_of_minus_infinity(cosa, dtype, cache, n, route):
    """Keys of -inf where the queries are positive: left out; a row that has no other is one without tokens."""
    hq, hkv, d, page = 4, 2, 64, 16
    q, k, v, ks, vs, table = contents([n], hq, hkv, d, page, dtype, cache, seed=n)
    q[0, :, 3] = q[0, :, 3].abs() + 0.25
    put(k, table, page, 0, 0, range(n), 3, -math.inf)
    put(k, table, page, 0, 1, range(n - 5), 3, -math.inf)
    out, lse = attend(cosa, q, k, v, ks, vs, table, [n], route)
    assert bool((out[0, :2] == 0).all()) and bool(torch.isneginf(lse[0, :2]).all())
    t = np.arange(n - 5, n)
    at, off = table[0][t // page], t % page
    want, want_lse, size = O.attention(wide(q[0, 2:]), wide(k)[at, 1, off], wide(v)[at, 1, off], d ** -0.5)
    top = np.abs(wide(v)[at, 1, off]).max()
    assert (np.abs(wide(out[0, 2:]) - want) <= ROUND[dtype] * np.abs(want) + (4 * 128 * 2.0 ** -24 * size + 2.0 ** -16) * top).all()
    assert np.abs(wide(lse[0, 2:]) - want_lse).max() <= 2 * 128 * 2.0 ** -24 * size + 4e-6 * max(1.0, np.abs(want_lse).max())


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F16, F16), (BF16, E4M3), (F16, E4M3)])
@pytest.mark.parametrize("n,d", [(40000, 64), (9001, 128)])
@pytest.mark.parametrize("gap", [10.0, 16.0, 18.0, 26.0])
@pytest.mark.parametrize("route", ["as usual", "one CTA", "check"])
def test_many_small_weights_behind_a_large_one(cosa, dtype, cache, n, d, gap, route):
    """One token's logit lies `gap` above all others, and its value is zero: the output is what the others' weights, e^-gap each, add up to."""
    q, k, v = torch.zeros(1, 2, d, device="cuda"), torch.zeros(1, 1, n, d, device="cuda"), torch.rand(1, 1, n, d, device="cuda") + 0.5
    q[0, :, 0] = 1.0
    k[0, 0, 7, 0], v[0, 0, 7] = gap, 0.0
    # (a multiple of 8 tokens a page, all in one order)
    page, count = 8, -(-n // 8)
    k, v = (torch.nn.functional.pad(x, (0, 0, 0, count * page - n)).view(count, page, 1, d).transpose(1, 2).to(cache).contiguous() for x in (k, v))
    q, ones = q.to(dtype), torch.ones(1, device="cuda") if cache is E4M3 else None
    handle = cosa.make_cache(k, v, gpu([range(count)]), k_scale=ones, v_scale=ones)
    out, lse = torch.empty_like(q), torch.empty(1, 2, device="cuda")
    cosa.cosa_decode_attention(handle, q, gpu([n]), out, lse, softmax_scale=1.0, opt=cosa.decode_options(impl=int(route == "check"), ctas=int(route == "one CTA")))
    want, want_lse, size = O.attention(wide(q[0]), wide(k).reshape(-1, d)[:n], wide(v).reshape(-1, d)[:n], 1.0)
    # every value is positive, so an error of the weights is one of the output: the outputs' rounding, logits as elsewhere, 2^-16 for the weights; and float32's own
    # sums, n additions of which the tensor cores may cut off
    loose = ROUND[dtype] + 4 * 128 * 2.0 ** -24 * size + 2.0 ** -16 + n / 32 * 2.0 ** -23
    assert (np.abs(wide(out[0]) - want) <= loose * want + 2.0 ** -25).all(), (np.abs(wide(out[0]) / want - 1).max(), loose)
    assert np.abs(wide(lse[0]) - want_lse).max() <= 2 * 128 * 2.0 ** -24 * size + 4e-6 * max(1.0, np.abs(want_lse).max())


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F16, F16), (BF16, E4M3), (F16, E4M3)])
@pytest.mark.parametrize("route", ROUTES)
def test_weights_are_not_rounded(cosa, dtype, cache, route):
    """Two tokens of opposite values, whose logits differ by little: the output is a small difference of the two weights, in which an error of
    either stands out."""
    hq, d, page = 64, 128, 8
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = torch.zeros(1, hq, d, device="cuda")
    q[0, :, 0] = torch.rand(hq, generator=gen, device="cuda") * 0.004 + 1e-4
    q[0, :, 1] = 1.0
    k, v = (torch.zeros(1, 1, page, d, device="cuda") for _ in range(2))
    k[0, 0, 0, 0] = 1.0
    v[0, 0, 0], v[0, 0, 1] = 1.0, -1.0
    q, k, v = q.to(dtype), k.to(cache), v.to(cache)
    ones = torch.ones(1, device="cuda") if cache is E4M3 else None
    out, lse = attend(cosa, q, k, v, ones, ones, np.zeros((1, 1), np.int64), [2], route)
    want, _, size = O.attention(wide(q[0]), wide(k)[0, 0, :2], wide(v)[0, 0, :2], d ** -0.5)
    # (the bound for two 16-bit terms, with values of 1)
    bad = np.abs(wide(out[0]) - want) - (ROUND[dtype] * np.abs(want) + 4 * 128 * 2.0 ** -24 * size + 2.0 ** -16 + 2.0 ** -25)
    assert bad.max() <= 0, float(bad.max())


@pytest.mark.parametrize("lens,hq,hkv,page", [([20000], 8, 2, 16), ([5000, 0, 1, 900], 32, 8, 64)])
def test_windows_of_any_size(cosa, lens, hq, hkv, page):
    """A window that no request fills is none: the same division of the work, the same bits."""
    q, k, v, _, _, table = contents(lens, hq, hkv, 128, page, BF16, BF16, seed=2)
    handle = cosa.make_cache(k, v, gpu(table))
    results = []
    for window in (0, 2 ** 31 - 1, 2 ** 31 - 9, 2 ** 30):
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        cosa.cosa_decode_attention(handle, q, gpu(lens), out, lse, window=window)
        results.append((out, lse))
    for out, lse in results[1:]:
        assert torch.equal(out, results[0][0]) and torch.equal(lse, results[0][1])


# ---------------------------------------------------------------- selection
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("pages", [[30], [3, 40, 41], [69], list(range(1, 70, 2)), list(range(70))])
@pytest.mark.parametrize("leaning", ["all", "one head", "none"])
def test_select_of_pages_with_infinite_scores(cosa, dtype, pages, leaning):
    """A page whose score is +inf holds that head's maximum and comes first, and of several the lowest indices; the other heads rank as ever."""
    page, n, hq, hkv, d = 16, 70, 6, 2, 128
    torch.manual_seed(len(pages))
    low = -torch.rand(n, hkv, d, device="cuda") - 0.1
    high = -low * torch.rand(n, hkv, d, device="cuda")
    high[pages, :, 5] = math.inf
    bounds = torch.stack([low, high], dim=2).to(dtype).contiguous()
    q = torch.randn(1, hq, d, device="cuda")
    towards = q[0, :, 5].abs() + 0.1
    q[0, :, 5] = towards if leaning == "all" else -towards
    if leaning == "one head":
        q[0, 1::3, 5] = towards[1::3]
    q = q.to(dtype)
    got, count = torch.empty(1, hkv, 12, dtype=torch.int32, device="cuda"), torch.empty(1, hkv, dtype=torch.int32, device="cuda")
    handle = cosa.make_cache(None, None, gpu([range(n)]), bounds=bounds, page_size=page)
    cosa.cosa_decode_select(handle, q, gpu([n * page]), 0.15, got, count)
    qs, bs = q.float().cpu().numpy(), bounds.float().cpu().numpy()
    for h in range(hkv):
        want = O.select(qs[0, h * 3:h * 3 + 3], bs[:, h, 0], bs[:, h, 1], 0.15)
        kept = got[0, h, :int(count[0, h])].tolist()
        assert kept == want.tolist() and len(kept) == 11
        if leaning != "none":
            # (beside them no more than a page of each other head's maximum, which ranks 0 as well)
            assert sum(j in pages for j in kept) >= min(len(pages), len(kept) - (0 if leaning == "all" else 2))
