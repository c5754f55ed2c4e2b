"""Roundings of the paged KV cache's operators, against the exact results: E4M3 codes
of the store at scales that are no powers of two, and the attention's weights."""
import numpy as np
import pytest
import torch

from gpu_helpers import DEV
from paper_2609_34380_amd import dps

pytestmark = pytest.mark.gpu

F16, BF16, E4M3 = torch.float16, torch.bfloat16, torch.float8_e4m3fn
# the values of the codes 0 .. 126, from the format: 4 exponent bits of bias 7, 3 mantissa bits
CODES = np.array([(c % 8) * 2.0 ** -9 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 7)
                  for c in range(127)])


def nearest(x):
    """E4M3 values nearest to x (float64), ties to the even code, clamped; NaN stays."""
    size = np.minimum(np.abs(x), 448.0)
    at = np.clip(np.searchsorted(CODES, size, side="right") - 1, 0, 125)
    mid = (CODES[at] + CODES[at + 1]) / 2       # exact, as the comparisons are
    up = (size > mid) | ((size == mid) & (at % 2 == 1))
    return np.where(np.isnan(x), np.nan, np.copysign(CODES[at + up], x))


# 16 / 17 and the like put quotients of FP16 values within 2^-25 of the middle of two
# codes: a quotient rounded to fp32 first would land on it
@pytest.mark.parametrize("scale", [0.03, 41.0, 47 / 1024, 16 / 17, 16 / 19, 16 / 31, 1 / 3, 7e-5,
                                   1.9, 3e38, 1.2e-38, 1e-30, 0.25])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_e4m3_codes_are_the_nearest_to_value_over_scale(dtype, scale):
    """Every 16-bit value, as key and as value.  A quotient of 8 or 11 bits by 24 that is
    not a code's middle is further from it than float64 resolves."""
    words = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
    rows, dim, tokens = 512, 128, 16
    x = words.view(rows, dim).repeat(1, 3)
    other = 2 * scale if scale < 1e38 else scale / 2
    pool = torch.zeros(rows // tokens * 2 * tokens * dim, dtype=torch.uint8, device=DEV)
    cache = dps.KvCache(pool, tokens, 1, dim, E4M3, k_scale=scale, v_scale=other)
    dps.kv_store(x.to(DEV), cache, torch.arange(rows, device=DEV), 1)
    got = pool.cpu().view(rows // tokens, 2, tokens * dim)
    k = got[:, 0].reshape(-1, dim // 64, tokens, 64).transpose(1, 2).reshape(-1)
    v = got[:, 1].reshape(-1)
    for code, s in ((k, scale), (v, other)):
        with np.errstate(over="ignore"):
            want = nearest(words.double().numpy() / np.float64(np.float32(s)))
        have = code.view(E4M3).double().numpy()
        bad = ~((have == want) | (np.isnan(have) & np.isnan(want)))
        assert not bad.any(), (s, int(bad.sum()), words.double().numpy()[bad][:4], have[bad][:4],
                               want[bad][:4])


@pytest.mark.parametrize("dtype,cdtype", [(BF16, BF16), (BF16, E4M3), (F16, F16)])
def test_attention_leans_to_no_side(dtype, cdtype):
    """Outputs of random weights over positive values: their errors, single roundings,
    cancel.  2^23 outputs near 1.5 round with a deviation of 2^-7 / sqrt(12) (BF16), so
    their mean relative error has one of 5e-7; a loss of weight shows as itself."""
    rows, heads, tokens, dim = 4096, 16, 64, 128
    gen = torch.Generator(device=DEV).manual_seed(11)
    rand = lambda *shape: torch.rand(*shape, generator=gen, device=DEV)
    k = (4 * rand(rows, tokens, dim) - 2).to(cdtype)
    v = (1 + rand(rows, tokens, dim)).to(cdtype)
    seg = 64 // cdtype.itemsize
    pool = torch.cat((k.view(rows, tokens, dim // seg, seg).transpose(1, 2).reshape(rows, -1)
                      .view(torch.uint8), v.view(rows, -1).view(torch.uint8)), 1).contiguous()
    cache = dps.KvCache(pool, tokens, 1, dim, cdtype)
    q = (2 * rand(rows, heads, dim) - 1).to(dtype)
    table = torch.arange(rows, dtype=torch.int32, device=DEV)[:, None].contiguous()
    got = dps.attn_decode(q, cache, table, torch.full_like(table[:, 0], tokens)).double()
    s = torch.matmul(q.double(), k.double().transpose(1, 2).contiguous()) * dim ** -0.5
    want = torch.matmul(torch.softmax(s, -1), v.double())
    lean = float(((got - want) / want).mean())
    assert abs(lean) <= (2.0 ** -18 if dtype == BF16 else 2.0 ** -21), lean


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("gap", [8.0, 17.0, 20.0])
@pytest.mark.parametrize("large", [0, 20002])
def test_small_weights_beside_a_large_one(dtype, gap, large):
    """One token e^gap above 20002 others, all of them in one wave's range of tiles (1100
    rows of one request, about one a wave).  The sum meets a rounding of 2^-24 of itself
    per tile of 32 tokens; FP16 terms lose up to 2^-30 of the largest weight a token,
    BF16 terms 2^-17 of a token's own."""
    n, dim, tokens, rows = 20003, 64, 16, 1100
    blocks = -(-n // tokens)
    k = torch.zeros(blocks * tokens, dim, dtype=dtype)
    v = torch.ones(blocks * tokens, dim, dtype=dtype)
    k[large, 0], v[large] = gap, 0.0
    k, v = (x.view(blocks, tokens, dim) for x in (k, v))
    pool = torch.cat((k.view(blocks, tokens, 2, 32).transpose(1, 2).reshape(blocks, -1),
                      v.reshape(blocks, -1)), 1).contiguous().to(DEV)
    q = torch.zeros(rows, 1, dim, dtype=dtype, device=DEV)
    q[..., 0] = 1.0
    i32 = lambda *shape, **kw: torch.zeros(*shape, dtype=torch.int32, device=DEV, **kw)
    lse = torch.empty(rows, 1, device=DEV)
    got = dps.attn_decode(q, dps.KvCache(pool, tokens, 1, dim, dtype),
                          torch.arange(blocks, dtype=torch.int32, device=DEV)[None],
                          i32(rows) + n, req=i32(rows), scale=1.0, lse=lse)
    small = (n - 1) * np.exp(-gap)
    drift = 2.0 ** -24 * (n // 32 + 2)
    err = float((lse.double() - (gap + np.log1p(small))).abs().max())
    assert err <= drift + 2.0 ** -18, err     # and lse's own rounding, at 16 to 32
    want = small / (1 + small)
    lost = (n - 1) * 2.0 ** -30 / (1 + small) if dtype == F16 else 2.0 ** -17 * want
    half = 2.0 ** -11 if dtype == F16 else 2.0 ** -8
    err = float((got.double() - want).abs().max())
    assert err <= lost + (half + 2 * drift) * want + (2.0 ** -25 if dtype == F16 else 0), err


@pytest.mark.parametrize("score", [-2.2e38, -2.3e38, 2.3e38])
def test_scores_near_the_ends_of_fp32(score):
    """Equal scores whose powers of two (log2(e) times them) are still finite: the mean of
    the values; one score far above them: its value alone."""
    n, dim, tokens = 300, 64, 16
    blocks = -(-n // tokens)
    k = torch.zeros(blocks * tokens, dim, dtype=BF16)
    k[:, 0] = score
    v = torch.randn(blocks * tokens, dim, generator=torch.Generator().manual_seed(3)).to(BF16)
    q = torch.zeros(2, 1, dim, dtype=BF16, device=DEV)
    q[..., 0] = 1.0
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    for best in (None, 7):
        if best is not None:
            k[:, 0] = min(score, score / 2)
            k[best, 0] = max(score, score / 2)
        pool = torch.cat((k.view(blocks, tokens, 2, 32).transpose(1, 2).reshape(blocks, -1),
                          v.view(blocks, -1)), 1).contiguous().to(DEV)
        lse = torch.empty(2, 1, device=DEV)
        got = dps.attn_decode(q, dps.KvCache(pool, tokens, 1, dim, BF16),
                              i32([list(range(blocks))]), i32([n, 10]), req=i32([0, 0]),
                              scale=1.0, lse=lse).cpu().double()
        for row, m in enumerate((n, 10)):
            want = v[:m].double().mean(0) if best is None else v[best].double()
            spread = v[:m].double().abs().mean(0) if best is None else want.abs()
            bound = 2.0 ** -8 * want.abs() + 2.0 ** -14 * spread
            assert bool(((got[row, 0] - want).abs() <= bound).all())
            top = float(k[:m, 0].double().max())
            assert abs(float(lse[row, 0]) - top) <= 2.0 ** -20 * abs(top)
