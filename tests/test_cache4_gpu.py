"""The K/V cache in 4 bits: append, read, attention, accumulated weights and eviction against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2602_01345_b200 as nova

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    return nova.Context(0)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _cu(counts):
    return _i32(np.concatenate([[0], np.cumsum(counts)]).tolist())


def _rows(seed, n, C, scale=1.0):
    g = torch.Generator(device="cpu").manual_seed(seed)
    x = torch.randn((n, C), generator=g) * torch.exp(0.5 * torch.randn((1, C), generator=g)) * scale
    return x.to(torch.bfloat16)


def _ref_quantise(x):
    """[n, C] bf16 CPU -> values float64, scales float64 [n, C/32], codes int [n, C], from the definition."""
    a = x.double().numpy().reshape(x.shape[0], x.shape[1] // 32, 32)
    top = np.abs(a).max(-1)
    m, e = np.frexp(top / 7.0)
    s = np.ldexp(np.ceil(m * 32.0) / 32.0, e)
    s = np.where(top > 0, np.maximum(s, 2.0 ** -120), 0.0)
    codes = np.rint(a / np.where(s > 0, s, 1.0)[..., None])
    return (codes * s[..., None]).reshape(x.shape), s, codes.reshape(x.shape).astype(np.int64)


def _unpack(packed):
    w = packed.cpu().contiguous().view(torch.int32).numpy().astype(np.int64) & 0xffffffff
    out = np.empty(w.shape[:-1] + (w.shape[-1] * 8,), dtype=np.int64)
    for i in range(4):
        out[..., 2 * i::8] = ((w >> (4 * i)) & 15) - 8
        out[..., 2 * i + 1::8] = ((w >> (16 + 4 * i)) & 15) - 8
    return out


def _garbage(cache):
    """What lies past kv_len must not matter: codes of all kinds and scales of NaN and infinity."""
    for t in (cache.k_codes, cache.v_codes):
        t.random_(0, 256)
    for i, t in enumerate((cache.k_scales, cache.v_scales)):
        t.fill_(float("nan") if i else float("inf"))


def _filled(ctx, lens, lmax, C, heads, seed):
    """A cache with rows appended in one call; returns it and the values it stands for, float64 per image."""
    cache = nova.Cache4.empty(len(lens), lmax, C, heads)
    _garbage(cache)
    n = sum(lens)
    k, v = _rows(seed, n, C), _rows(seed + 1, n, C)
    nova.nova_cache4_append(ctx, cache, k.to(DEV), v.to(DEV), _cu(lens))
    kr, vr = _ref_quantise(k)[0], _ref_quantise(v)[0]
    at = np.concatenate([[0], np.cumsum(lens)])
    return cache, [kr[at[b]:at[b + 1]] for b in range(len(lens))], [vr[at[b]:at[b + 1]] for b in range(len(lens))]


# ---- append and read ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("C,heads", [(64, 1), (192, 3), (1024, 16), (1920, 30), (2048, 16)])
@pytest.mark.parametrize("counts,lens", [([1], [0]), ([3, 0, 17], [5, 2, 0]), ([40, 1], [0, 63])])
def test_append_writes_the_defined_codes(ctx, C, heads, counts, lens):
    B, lmax = len(counts), 80
    cache = nova.Cache4.empty(B, lmax, C, heads)
    _garbage(cache)
    cache.kv_len.copy_(_i32(lens))
    before = [t.clone() for t in (cache.k_codes, cache.v_codes, cache.k_scales.view(torch.int16), cache.v_scales.view(torch.int16))]
    n = sum(counts)
    k, v = _rows(1, n, C), _rows(2, n, C, 1e-3)
    k[0, :32] = 0
    k[0, 32:40] = torch.tensor([7.0, 3.5, -3.5, 2.5, -2.5, 0.5, -7.0, 1.5]).to(torch.bfloat16)     # ties, when the rest is small
    k[0, 40:64] = 0
    wide = torch.zeros((n + 2, 3 * C), dtype=torch.bfloat16, device=DEV)      # rows apart, and two more than there are
    wide[:n, C:2 * C], wide[:n, 2 * C:] = k.to(DEV), v.to(DEV)
    wide[n:] = float("nan")
    nova.nova_cache4_append(ctx, cache, wide[:, C:2 * C], wide[:, 2 * C:], _cu(counts))
    assert ctx.device_status() == 0
    assert cache.kv_len.tolist() == [a + b for a, b in zip(lens, counts)]
    mask = torch.zeros((B, lmax), dtype=torch.bool)
    r = 0
    for name, x in (("k", k), ("v", v)):
        _, s, codes = _ref_quantise(x)
        got_c = _unpack(getattr(cache, name + "_codes"))
        got_s = getattr(cache, name + "_scales").double().cpu().numpy()
        r = 0
        for b, (n0, m) in enumerate(zip(lens, counts)):
            assert np.array_equal(got_c[b, n0:n0 + m], codes[r:r + m])
            assert np.array_equal(got_s[b, n0:n0 + m], s[r:r + m])
            mask[b, n0:n0 + m] = True
            r += m
    after = (cache.k_codes, cache.v_codes, cache.k_scales.view(torch.int16), cache.v_scales.view(torch.int16))
    for x, y in zip(before, after):                                            # nothing else was written
        assert torch.equal(x.cpu()[~mask], y.cpu()[~mask])


def test_append_without_advance_and_read_back(ctx):
    C, lens, counts = 1024, [7, 0], [9, 33]
    cache, kr, _ = _filled(ctx, lens, 64, C, 16, 3)
    k, v = _rows(5, sum(counts), C), _rows(6, sum(counts), C)
    nova.nova_cache4_append(ctx, cache, k.to(DEV), v.to(DEV), _cu(counts), advance=False)
    assert cache.kv_len.tolist() == lens
    out = torch.full((2, sum(counts) + 3, C), 7.0, dtype=torch.bfloat16, device=DEV)
    nova.nova_cache4_read(ctx, cache, _cu(counts), out[0], out[1], first=cache.kv_len)
    assert ctx.device_status() == 0
    assert np.array_equal(out[0, :42].double().cpu().numpy(), _ref_quantise(k)[0])
    assert np.array_equal(out[1, :42].double().cpu().numpy(), _ref_quantise(v)[0])
    assert (out[:, 42:] == 7.0).all()                                          # rows behind the last image
    nova.nova_cache4_read(ctx, cache, _cu([7, 0]), out[0, :7], out[1, :7])
    assert np.array_equal(out[0, :7].double().cpu().numpy(), kr[0])


def test_append_extreme_magnitudes(ctx):
    C = 64
    top = torch.tensor([2.0 ** 119, 2.0 ** -126, 2.0 ** -120 * 7, 2.0 ** -100, 1e-38, 3.0, -0.0, 2.0 ** 119 * 1.984375])
    k = torch.zeros((8, C))
    k[:, 3] = top
    k[:, 35] = -top
    k[:, 4] = top / 3
    k = k.to(torch.bfloat16)
    cache = nova.Cache4.empty(1, 8, C, 1)
    nova.nova_cache4_append(ctx, cache, k.to(DEV), k.to(DEV), _cu([8]))
    out = torch.empty((2, 8, C), dtype=torch.bfloat16, device=DEV)
    nova.nova_cache4_read(ctx, cache, _cu([8]), out[0], out[1])
    assert ctx.device_status() == 0
    ref = _ref_quantise(k)[0]
    assert np.array_equal(out[0].double().cpu().numpy(), ref) and np.array_equal(out[1].double().cpu().numpy(), ref)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 2.0 ** 120])
def test_append_nonfinite_group_reads_as_nan(ctx, bad):
    C = 128
    k = _rows(1, 3, C)
    v = k.clone()
    k[1, 70] = bad
    cache = nova.Cache4.empty(1, 8, C, 1)
    nova.nova_cache4_append(ctx, cache, k.to(DEV), v.to(DEV), _cu([3]))
    assert ctx.device_status() == 5
    out = torch.empty((2, 3, C), dtype=torch.bfloat16, device=DEV)
    nova.nova_cache4_read(ctx, cache, _cu([3]), out[0], out[1])
    got = out[0].double().cpu().numpy()
    ref = _ref_quantise(v)[0]
    hit = np.zeros((3, C), dtype=bool)
    hit[1, 64:96] = True
    assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], ref[~hit])
    assert np.array_equal(out[1].double().cpu().numpy(), ref)


def test_append_that_does_not_fit_leaves_the_image_alone(ctx):
    C = 64
    cache = nova.Cache4.empty(3, 10, C, 1)
    _garbage(cache)
    cache.kv_len.copy_(_i32([4, 6, 10]))
    before = cache.k_codes.clone()
    k = _rows(1, 12, C).to(DEV)
    nova.nova_cache4_append(ctx, cache, k, k, _cu([6, 5, 1]))
    assert ctx.device_status() == 2
    assert cache.kv_len.tolist() == [10, 6, 10]
    assert torch.equal(cache.k_codes[1:], before[1:]) and torch.equal(cache.k_codes[0, :4], before[0, :4])
    out = torch.full((2, 4, C), 3.0, dtype=torch.bfloat16, device=DEV)
    nova.nova_cache4_read(ctx, cache, _cu([4, 0, 0]), out[0], out[1], first=_i32([8, 0, 0]))
    assert ctx.device_status() == 2                                            # two of the four rows do not exist
    assert (out[:, 2:] == 3.0).all()


# ---- attention ------------------------------------------------------------------------------------------------
def _ref_attention(q, k, v, heads):
    """One image in 64 bits: o, lse [heads, n], bounds of the errors that a product of bf16 operands with sums in 32 bits may have.

    A score's sum of dh products, added in 32 bits in any order (truncated, as tensor cores do), is off by at most dh 2^-23 of the
    sum of magnitudes; the multiply-add that subtracts the maximum and the exponential by 2^-22 of the exponents' sizes. So a
    probability is off by delta relative, and so is a ratio of their sums by twice that. Rounding probabilities and o to bf16 adds
    2^-8 each (to the sum of |p v|, and to |o|). Exponentials below the smallest normal number, 2^-126, are taken as zero; as
    the tensor-core kernel scales them by 2^-48, a probability below 2^-78 of the highest, and of their sum, may be missing."""
    n, C = q.shape
    dh = C // heads
    o, lse = np.zeros((n, C)), np.full((heads, n), -np.inf)
    tol_o, tol_l = np.zeros((n, C)), np.zeros((heads, n))
    if len(k) == 0:
        return o, lse, tol_o, tol_l
    for h in range(heads):
        c = slice(h * dh, (h + 1) * dh)
        s = q[:, c] @ k[:, c].T / math.sqrt(dh)
        size = (np.abs(q[:, c]) @ np.abs(k[:, c]).T).max(1) / math.sqrt(dh)
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        tot = p.sum(1, keepdims=True)
        o[:, c] = p @ v[:, c] / tot
        lse[h] = (top + np.log(tot))[:, 0]
        delta = size * (dh * 2.0 ** -23) + (size + np.abs(top[:, 0])) * 2.0 ** -21 + 2.0 ** -20
        mass = p @ np.abs(v[:, c]) / tot
        tol_o[:, c] = 2.0 ** -8 * (mass + np.abs(o[:, c])) * 1.01 + 2.0 * delta[:, None] * mass + 2.0 ** -78 * np.abs(v[:, c]).sum(0)
        tol_l[h] = delta + np.abs(lse[h]) * 2.0 ** -22 + len(k) * 2.0 ** -24
    return o, lse, tol_o, tol_l


def _check_attention(ctx, lens, rows, C, heads, seed=0, lmax=None, q_scale=1.3, extra=0, stride=False):
    cache, k, v = _filled(ctx, lens, lmax or max(max(lens), 1) + 3, C, heads, seed)
    m = sum(rows)
    q = _rows(seed + 7, m + extra, C, q_scale)
    if extra:
        q[m:] = float("nan")
    qd = q.to(DEV)
    if stride:
        wide = torch.zeros((m + extra, C + 72), dtype=torch.bfloat16, device=DEV)
        wide[:, 8:8 + C] = qd
        qd = wide[:, 8:8 + C]
    ctx.ensure_cache4_workspace(cache, m + extra)
    o = torch.full((m + extra, C), 5.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((heads, m + extra), 5.0, dtype=torch.float32, device=DEV)
    nova.nova_cache4_attention(ctx, cache, qd, _cu(rows), o, lse=lse)
    assert ctx.device_status() == 0
    assert (o[m:] == 5.0).all() and (lse[:, m:] == 5.0).all()
    r0, qn = 0, q.double().numpy()
    for b, n in enumerate(rows):
        ref_o, ref_l, tol_o, tol_l = _ref_attention(qn[r0:r0 + n], k[b], v[b], heads)
        got_o = o[r0:r0 + n].double().cpu().numpy()
        got_l = lse[:, r0:r0 + n].double().cpu().numpy()
        assert np.all(np.abs(got_o - ref_o) <= tol_o), (b, np.max(np.abs(got_o - ref_o) - tol_o))
        fine = np.isfinite(ref_l)
        assert np.array_equal(fine, np.isfinite(got_l))
        assert np.all(np.abs(got_l[fine] - ref_l[fine]) <= tol_l[fine]), (b, np.max(np.abs(got_l[fine] - ref_l[fine]) - tol_l[fine]))
        r0 += n
    o2, lse2 = torch.zeros_like(o), torch.zeros_like(lse)
    nova.nova_cache4_attention(ctx, cache, qd, _cu(rows), o2, lse=lse2)          # the same bits again
    assert torch.equal(o[:m], o2[:m]) and torch.equal(lse[:, :m], lse2[:, :m])
    o3 = torch.zeros_like(o)
    nova.nova_cache4_attention(ctx, cache, qd, _cu(rows), o3)
    assert torch.equal(o[:m], o3[:m])
    return cache, qd, lse, k, v


SHAPES = [(64, 1), (128, 1), (192, 3), (384, 3), (1024, 16), (2048, 16)]


@pytest.mark.parametrize("C,heads", SHAPES)
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 127, 128, 129, 384, 385, 1000])
def test_attention_single_query(ctx, C, heads, n):
    _check_attention(ctx, [n], [1], C, heads, seed=n)


@pytest.mark.parametrize("C,heads", [(192, 3), (384, 3), (1024, 16)])
@pytest.mark.parametrize("rows", [2, 15, 16, 17, 33, 64, 128, 129, 200, 256, 257, 300])
def test_attention_row_counts(ctx, C, heads, rows):
    _check_attention(ctx, [417], [rows], C, heads, seed=rows, extra=3)


@pytest.mark.parametrize("C,heads", [(192, 3), (384, 3), (1920, 30), (2048, 16)])
@pytest.mark.parametrize("lens,rows", [([0, 5, 700], [3, 0, 1]), ([130, 0, 1, 64], [20, 9, 33, 0]), ([900, 40, 0, 0, 333], [1, 300, 2, 0, 140]),
                                       ([0, 0], [4, 1])])
def test_attention_ragged(ctx, C, heads, lens, rows):
    _check_attention(ctx, lens, rows, C, heads, seed=4, lmax=1000, extra=5, stride=True)


@pytest.mark.parametrize("rows", [1, 40, 300])
@pytest.mark.parametrize("C,heads", [(192, 3), (128, 1)])
def test_attention_many_images(ctx, C, heads, rows):
    rng = np.random.default_rng(rows)
    lens = rng.integers(0, 90, size=70).tolist()
    counts = (rng.integers(0, 2 * rows, size=70) * (rng.random(70) < 0.5)).tolist()
    _check_attention(ctx, lens, counts, C, heads, seed=2)


@pytest.mark.parametrize("C,heads,lens,rows", [(1920, 30, [1779] * 4, [563] * 4), (1920, 30, [1779, 1571, 1364, 1156], [366, 432, 497, 563]),
                                               (1920, 15, [1500] * 4, [700] * 4), (2048, 16, [900] * 30, [100] * 30), (2048, 16, [700] * 30, [9] * 30),
                                               (1536, 24, [640] * 30, [100] * 30)])
def test_attention_many_work_items(ctx, C, heads, lens, rows):
    """Several work items per CTA, one after the other, the same bits in every launch. (Against 64 bits on the device.)"""
    cache = nova.Cache4.empty(len(lens), max(lens), C, heads)
    g = torch.Generator(device=DEV).manual_seed(C + heads)
    k, v = ((torch.randn((sum(lens), C), generator=g, device=DEV) * torch.exp(0.4 * torch.randn((1, C), generator=g, device=DEV))).to(torch.bfloat16)
            for _ in range(2))
    nova.nova_cache4_append(ctx, cache, k, v, _cu(lens))
    kv = torch.empty((2, sum(lens), C), dtype=torch.bfloat16, device=DEV)
    nova.nova_cache4_read(ctx, cache, _cu(lens), kv[0], kv[1])
    m, dh = sum(rows), C // heads
    q = (1.3 * torch.randn((m, C), generator=g, device=DEV) * torch.exp(0.5 * torch.randn((m, 1), generator=g, device=DEV))).to(torch.bfloat16)
    ctx.ensure_cache4_workspace(cache, m)
    runs = []
    for _ in range(8):
        o, lse = torch.full((m, C), 5.0, dtype=torch.bfloat16, device=DEV), torch.full((heads, m), 5.0, device=DEV)
        nova.nova_cache4_attention(ctx, cache, q, _cu(rows), o, lse=lse)
        runs.append((o, lse))
    assert ctx.device_status() == 0
    at, r0 = 0, 0
    for n, r in zip(lens, rows):
        qh = q[r0:r0 + r].double().view(r, heads, dh).transpose(0, 1)
        kh, vh = (t[at:at + n].double().view(n, heads, dh).transpose(0, 1) for t in kv)
        s = qh @ kh.transpose(1, 2) / math.sqrt(dh)
        size = (qh.abs() @ kh.abs().transpose(1, 2)).amax(-1) / math.sqrt(dh)
        lse, p = torch.logsumexp(s, -1), torch.softmax(s, -1)
        # as in _ref_attention
        delta = size * (dh * 2.0 ** -23) + (size + s.amax(-1).abs()) * 2.0 ** -21 + 2.0 ** -20
        o, mass = p @ vh, p @ vh.abs()
        tol = 2.0 ** -8 * (mass + o.abs()) * 1.01 + 2.0 * delta[..., None] * mass + 2.0 ** -78 * vh.abs().sum(1, keepdim=True)
        got_o = runs[0][0][r0:r0 + r].double().view(r, heads, dh).transpose(0, 1)
        assert ((got_o - o).abs() <= tol).all()
        assert ((runs[0][1][:, r0:r0 + r].double() - lse).abs() <= delta + lse.abs() * 2.0 ** -22 + n * 2.0 ** -24).all()
        at, r0 = at + n, r0 + r
    for o, lse in runs[1:]:
        assert torch.equal(o, runs[0][0]) and torch.equal(lse, runs[0][1])


@pytest.mark.parametrize("rows", [1, 24, 200])
@pytest.mark.parametrize("C,heads", [(64, 1), (128, 1)])
def test_attention_long_cache(ctx, C, heads, rows):
    _check_attention(ctx, [20011], [rows], C, heads, seed=9)


@pytest.mark.parametrize("rows", [3, 150])
@pytest.mark.parametrize("C,heads", [(64, 1), (256, 2)])
def test_attention_scores_far_apart(ctx, C, heads, rows):
    """Scores of hundreds, with the highest anywhere among the keys."""
    _check_attention(ctx, [777], [rows], C, heads, seed=11, q_scale=40.0)


@pytest.mark.parametrize("rows", [2, 150])
def test_attention_highest_score_in_the_last_rows(ctx, rows):
    """The last keys' scores lie more than 2^128 (in probabilities) above all others."""
    C, heads, n = 256, 2, 900
    cache, k, v = _filled(ctx, [n - 2], n, C, heads, 21)
    big = (torch.ones((2, C)) * 30.0).to(torch.bfloat16)
    vv = _rows(5, 2, C)
    nova.nova_cache4_append(ctx, cache, big.to(DEV), vv.to(DEV), _cu([2]))
    q = torch.full((rows, C), 2.0).to(torch.bfloat16)
    q[::2] *= -1
    ctx.ensure_cache4_workspace(cache, rows)
    o = torch.empty((rows, C), dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((heads, rows), dtype=torch.float32, device=DEV)
    nova.nova_cache4_attention(ctx, cache, q.to(DEV), _cu([rows]), o, lse=lse)
    assert ctx.device_status() == 0
    kk = np.concatenate([k[0], _ref_quantise(big)[0]])
    vr = np.concatenate([v[0], _ref_quantise(vv)[0]])
    ref_o, ref_l, tol_o, tol_l = _ref_attention(q.double().numpy(), kk, vr, heads)
    assert np.all(np.abs(o.double().cpu().numpy() - ref_o) <= tol_o)
    assert np.all(np.abs(lse.double().cpu().numpy() - ref_l) <= tol_l)


def test_attention_nan_row_reaches_only_its_image(ctx):
    C, heads = 128, 1
    k = _rows(1, 60, C)
    k[45, 3] = float("nan")
    for rows in ([2, 2], [140, 140]):
        cache = nova.Cache4.empty(2, 40, C, heads)
        nova.nova_cache4_append(ctx, cache, k.to(DEV), k.to(DEV), _cu([30, 30]))
        assert ctx.device_status() == 5
        m = sum(rows)
        ctx.ensure_cache4_workspace(cache, m)
        o = torch.empty((m, C), dtype=torch.bfloat16, device=DEV)
        nova.nova_cache4_attention(ctx, cache, _rows(3, m, C).to(DEV), _cu(rows), o)
        assert torch.isfinite(o[:rows[0]].float()).all() and torch.isnan(o[rows[0]:].float()).all()
        ctx.device_status()


# ---- weights --------------------------------------------------------------------------------------------------
def _check_weights(ctx, lens, rows, C, heads, seed=0, lmax=None, extra=0):
    cache, qd, lse, k, _ = _check_attention(ctx, lens, rows, C, heads, seed=seed, lmax=lmax, extra=extra)
    B, L = cache.B, cache.Lmax
    g = torch.Generator(device="cpu").manual_seed(seed)
    w_in = torch.rand((B, L), generator=g).to(DEV)
    out = torch.full((B, L), 9.0, device=DEV)
    nova.nova_cache4_weights(ctx, cache, qd, lse, _cu(rows), out, weight_in=w_in)
    none = torch.full((B, L), 9.0, device=DEV)
    nova.nova_cache4_weights(ctx, cache, qd, lse, _cu(rows), none)
    inplace = w_in.clone()
    nova.nova_cache4_weights(ctx, cache, qd, lse, _cu(rows), inplace, weight_in=inplace)
    assert ctx.device_status() == 0
    dh, r0 = C // heads, 0
    qn, ln = qd.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, (n, r) in enumerate(zip(lens, rows)):
        assert (out[b, n:] == 9.0).all() and (none[b, n:] == 9.0).all() and torch.equal(inplace[b, n:], w_in[b, n:])
        ref, tol = np.zeros(n), np.zeros(n)
        for h in range(heads if n else 0):
            c = slice(h * dh, (h + 1) * dh)
            s = qn[r0:r0 + r, c] @ k[b][:, c].T / math.sqrt(dh)
            size = np.abs(qn[r0:r0 + r, c]) @ np.abs(k[b][:, c]).T / math.sqrt(dh)
            p = np.exp(s - ln[h, r0:r0 + r, None])
            # a score off by dh 2^-23 of its magnitudes, the exponent (score and lse in units of log2) by 2^-22 of its parts
            delta = size * (dh * 2.0 ** -23) + (size + np.abs(ln[h, r0:r0 + r, None])) * 2.0 ** -21 + 2.0 ** -20
            ref += p.sum(0)
            tol += (p * delta).sum(0)
        w0 = w_in[b, :n].double().cpu().numpy()
        tol += (ref + w0) * (heads * max(r, 1) + 4) * 2.0 ** -24
        assert np.all(np.abs(none[b, :n].double().cpu().numpy() - ref) <= tol)
        assert np.all(np.abs(out[b, :n].double().cpu().numpy() - ref - w0) <= tol + 2.0 ** -24 * (ref + w0))
        r0 += r
    assert torch.equal(torch.where(out == 9.0, w_in, out), inplace)


@pytest.mark.parametrize("C,heads", [(64, 1), (128, 1), (192, 3), (384, 3), (1024, 16)])
@pytest.mark.parametrize("n,rows", [(1, 1), (255, 1), (256, 8), (257, 31), (300, 32), (700, 33), (90, 130), (2000, 65)])
def test_weights_of_one_image(ctx, C, heads, n, rows):
    _check_weights(ctx, [n], [rows], C, heads, seed=n)


@pytest.mark.parametrize("C,heads", [(192, 3), (1920, 30), (2048, 16)])
def test_weights_ragged(ctx, C, heads):
    _check_weights(ctx, [130, 0, 1, 300, 77], [20, 9, 33, 0, 150], C, heads, seed=3, lmax=400, extra=4)


def test_weights_of_many_images(ctx):
    rng = np.random.default_rng(4)
    _check_weights(ctx, rng.integers(0, 7, size=1100).tolist(), rng.integers(0, 3, size=1100).tolist(), 64, 1, seed=2)


def test_weights_of_many_queries(ctx):
    _check_weights(ctx, [600, 1100], [900, 513], 256, 4, seed=5)
    _check_weights(ctx, [600, 1100], [900, 513], 256, 2, seed=6)


def test_weights_sum_to_the_number_of_queries(ctx):
    """Every query hands out a weight of one per head, whatever the heads' scores."""
    C, heads, rows = 1024, 16, 57
    cache, qd, lse, _, _ = _check_attention(ctx, [1300], [rows], C, heads, seed=8)
    out = torch.zeros((1, cache.Lmax), device=DEV)
    nova.nova_cache4_weights(ctx, cache, qd, lse, _cu([rows]), out)
    # each term is off by 2 delta of the attention's and this call's scores; 2^-10 holds both for sums of magnitudes below 30
    assert abs(out[0, :1300].double().sum().item() / (heads * rows) - 1.0) < 2.0 ** -10


def test_weights_ignore_rows_that_attended_to_nothing(ctx):
    C, heads = 128, 2
    cache, k, _ = _filled(ctx, [50], 60, C, heads, 1)
    q = _rows(2, 3, C).to(DEV)
    ctx.ensure_cache4_workspace(cache, 3)
    lse = torch.zeros((heads, 3), device=DEV)
    o = torch.empty_like(q)
    nova.nova_cache4_attention(ctx, cache, q, _cu([3]), o, lse=lse)
    lse[:, 1] = -math.inf
    out = torch.zeros((1, 60), device=DEV)
    nova.nova_cache4_weights(ctx, cache, q, lse, _cu([3]), out)
    two = torch.zeros((1, 60), device=DEV)
    keep = [0, 2]
    nova.nova_cache4_weights(ctx, cache, q[keep].contiguous(), lse[:, keep].contiguous(), _cu([2]), two)
    # the same terms, in another order of at most six per sum
    assert torch.allclose(out, two, rtol=8 * 2.0 ** -24, atol=0)


# ---- eviction ---------------------------------------------------------------------------------------------------
def _ref_evict(w, n, budget, recent):
    if n <= budget:
        return list(range(n))
    old = sorted(range(n - recent), key=lambda j: (-w[j], j))[:budget - recent]
    return sorted(old) + list(range(n - recent, n))


def _check_evict(ctx, lens, lmax, C, heads, budget, recent, weight, dst_max=None, seed=0):
    cache, _, _ = _filled(ctx, lens, lmax, C, heads, seed)
    B = len(lens)
    dst_max = dst_max or budget + 2
    dst = nova.Cache4.empty(B, dst_max, C, heads)
    _garbage(dst)
    kept_before = [t.clone() for t in (dst.k_codes, dst.v_codes, dst.k_scales.view(torch.int16), dst.v_scales.view(torch.int16))]
    ctx.ensure_cache4_workspace(cache, 1)
    w_out = torch.full((B, dst_max), 9.0, device=DEV)
    src = torch.full((B, budget), 77, dtype=torch.int32, device=DEV)
    nova.nova_cache4_evict(ctx, cache, weight, budget, recent, dst, weight_out=w_out, src_row=src)
    assert ctx.device_status() == 0
    dst2 = nova.Cache4.empty(B, dst_max, C, heads)
    nova.nova_cache4_evict(ctx, cache, weight, budget, recent, dst2)            # nothing but the cache
    wn = weight.double().cpu().numpy()
    got = [t.cpu() for t in (dst.k_codes, dst.v_codes, dst.k_scales.view(torch.int16), dst.v_scales.view(torch.int16))]
    got2 = [t.cpu() for t in (dst2.k_codes, dst2.v_codes, dst2.k_scales.view(torch.int16), dst2.v_scales.view(torch.int16))]
    old = [t.cpu() for t in (cache.k_codes, cache.v_codes, cache.k_scales.view(torch.int16), cache.v_scales.view(torch.int16))]
    assert cache.kv_len.tolist() == list(lens)
    assert dst.kv_len.tolist() == [min(n, budget) for n in lens] == dst2.kv_len.tolist()
    for b, n in enumerate(lens):
        rows = _ref_evict(wn[b], n, budget, recent)
        m = len(rows)
        assert src[b].tolist() == rows + [-1] * (budget - m)
        for x, x2, y, z in zip(got, got2, old, kept_before):
            assert torch.equal(x[b, :m], y[b, rows]) and torch.equal(x2[b, :m], y[b, rows])
            assert torch.equal(x[b, m:], z[b, m:].cpu())
        assert torch.equal(w_out[b, :m], weight[b, rows]) and (w_out[b, m:] == 0).all()


@pytest.mark.parametrize("C,heads", [(64, 1), (192, 3), (1920, 30), (2048, 16)])
@pytest.mark.parametrize("lens,budget,recent", [([10], 4, 2), ([10], 4, 4), ([10], 4, 0), ([9, 0, 1, 33], 8, 3), ([5, 8], 8, 8), ([7], 0, 0),
                                                ([300, 299, 5], 256, 100)])
def test_evict(ctx, C, heads, lens, budget, recent):
    g = torch.Generator(device="cpu").manual_seed(budget)
    w = torch.rand((len(lens), max(lens) + 5), generator=g).to(DEV)
    _check_evict(ctx, lens, max(lens) + 5, C, heads, budget, recent, w)


@pytest.mark.parametrize("kind", ["equal", "zeros", "two", "near", "signed", "wide"])
@pytest.mark.parametrize("lens", [[1023], [1024, 1025], [4097, 700, 4100], [9000], [20000, 13], [33000]])
def test_evict_weights_of_all_kinds(ctx, kind, lens):
    lmax, B = max(lens) + 1, len(lens)
    g = torch.Generator(device="cpu").manual_seed(len(kind))
    u = torch.rand((B, lmax), generator=g)
    w = {"equal": torch.full((B, lmax), 0.3), "zeros": torch.where(u < 0.7, torch.zeros(()), u), "two": torch.where(u < 0.5, 1.0, 2.0),
         "near": 1.0 + torch.floor(u * 40) * 2.0 ** -23, "signed": torch.where(u < 0.3, -torch.zeros(()), torch.randn((B, lmax), generator=g)),
         "wide": torch.exp(80 * (u - 0.5))}[kind]
    for b, n in enumerate(lens):
        w[b, n:] = float("nan")                          # past the rows: never looked at
    for budget, recent in ((max(lens) // 2, max(lens) // 7), (max(lens) - 1, 0), (1, 0)):
        _check_evict(ctx, lens, lmax, 64, 1, budget, recent, w.to(DEV))


def test_evict_infinite_weights(ctx):
    w = torch.tensor([[1.0, math.inf, -math.inf, 3.0, 0.0, math.inf, 2.0, -1.0]], device=DEV)
    _check_evict(ctx, [8], 8, 64, 1, 4, 1, w)


def test_evict_larger_budget_than_rows_without_a_list(ctx):
    cache, k, _ = _filled(ctx, [6, 9], 10, 64, 1, 2)
    dst = nova.Cache4.empty(2, 50, 64, 1)
    ctx.ensure_cache4_workspace(cache, 1)
    w = torch.rand((2, 10), device=DEV)
    w_out = torch.full((2, 50), 4.0, device=DEV)
    nova.nova_cache4_evict(ctx, cache, w, 40, 30, dst, weight_out=w_out)
    assert ctx.device_status() == 0 and dst.kv_len.tolist() == [6, 9]
    assert torch.equal(dst.k_codes[0, :6], cache.k_codes[0, :6]) and torch.equal(dst.v_scales[1, :9], cache.v_scales[1, :9])
    assert torch.equal(w_out[1, :9], w[1, :9]) and (w_out[0, 6:] == 0).all()


# ---- large offsets, graphs, refusals ------------------------------------------------------------------------------
def test_rows_past_32_bit_offsets(ctx):
    """Caches of more than 2^32 bytes: the last images' rows lie past every 32-bit offset."""
    B, lmax, C, heads = 36, 131072, 2048, 16
    cache = nova.Cache4.empty(B, lmax, C, heads)                                  # 2 x 4.8 GB of codes
    lens = [0] * (B - 1) + [lmax - 70]
    cache.kv_len.copy_(_i32(lens))
    k, v = _rows(1, 64, C), _rows(2, 64, C)
    counts = [0] * (B - 1) + [64]
    nova.nova_cache4_append(ctx, cache, k.to(DEV), v.to(DEV), _cu(counts))
    out = torch.empty((2, 64, C), dtype=torch.bfloat16, device=DEV)
    nova.nova_cache4_read(ctx, cache, _cu(counts), out[0], out[1], first=_i32(lens))
    assert np.array_equal(out[0].double().cpu().numpy(), _ref_quantise(k)[0])
    assert np.array_equal(out[1].double().cpu().numpy(), _ref_quantise(v)[0])
    # the 64 rows moved to the front of a small cache by their weight
    weight = torch.zeros((B, lmax), device=DEV)
    weight[-1, lmax - 70:lmax - 6] = 1.0
    dst = nova.Cache4.empty(B, 64, C, heads)
    ctx.ensure_cache4_workspace(dst, 64)
    src = torch.empty((B, 64), dtype=torch.int32, device=DEV)
    nova.nova_cache4_evict(ctx, cache, weight, 64, 0, dst, src_row=src)
    assert src[-1].tolist() == list(range(lmax - 70, lmax - 6))
    assert torch.equal(dst.k_codes[-1], cache.k_codes[-1, lmax - 70:lmax - 6]) and torch.equal(dst.v_codes[-1], cache.v_codes[-1, lmax - 70:lmax - 6])
    # attention and weights of a cache whose other rows are zeros: every one of them has the same score
    for t in (cache.k_codes, cache.v_codes):
        t[-1, :lmax - 70] = 0x88
    for t in (cache.k_scales, cache.v_scales):
        t[-1, :lmax - 70] = 0
    for rows in (2, 130):
        q = _rows(4, rows, C)
        ctx.ensure_cache4_workspace(cache, rows)
        o = torch.empty((rows, C), dtype=torch.bfloat16, device=DEV)
        lse = torch.empty((heads, rows), device=DEV)
        cu = _cu([0] * (B - 1) + [rows])
        nova.nova_cache4_attention(ctx, cache, q.to(DEV), cu, o, lse=lse)
        w_out = torch.zeros((B, lmax), device=DEV)
        nova.nova_cache4_weights(ctx, cache, q.to(DEV), lse, cu, w_out)
        assert ctx.device_status() == 0
        kr, vr = _ref_quantise(k)[0], _ref_quantise(v)[0]
        s = np.einsum("qhd,khd->hqk", q.double().numpy().reshape(rows, heads, 128), kr.reshape(64, heads, 128)) / math.sqrt(128)
        tot = np.exp(s).sum(-1) + (lmax - 70)
        ref_o = np.einsum("hqk,khd->qhd", np.exp(s) / tot[..., None], vr.reshape(64, heads, 128)).reshape(rows, -1)
        mass = np.einsum("hqk,khd->qhd", np.exp(s) / tot[..., None], np.abs(vr).reshape(64, heads, 128)).reshape(rows, -1)
        # as above, with scores below 40 and every probability at most one: delta < 40 (128 2^-23 + 2^-20) + 2^-20 < 2^-10
        assert np.all(np.abs(o.double().cpu().numpy() - ref_o) <= mass * (2.0 ** -7 * 1.01 + 2.0 ** -9))
        ref_w = np.exp(s - np.log(tot)[..., None]).sum((0, 1))
        got_w = w_out[-1, lmax - 70:lmax - 6].double().cpu().numpy()
        assert np.all(np.abs(got_w / ref_w - 1) <= 2.0 ** -9)


def test_calls_replay_from_a_graph(ctx):
    C, heads, lens, rows = 1024, 16, [500, 90], [3, 40]
    cache, _, _ = _filled(ctx, lens, 700, C, heads, 1)
    own = nova.Context(0)
    own.ensure_cache4_workspace(cache, 43)
    q, k, v = (_rows(i, 43, C).to(DEV) for i in (5, 6, 7))
    cu = _cu(rows)
    o, lse = torch.zeros_like(q), torch.zeros((heads, 43), device=DEV)
    w = torch.zeros((2, 700), device=DEV)
    dst, w_out = nova.Cache4.empty(2, 200, C, heads), torch.zeros((2, 200), device=DEV)

    def once():
        w.zero_()
        nova.nova_cache4_append(own, cache, k, v, cu)
        nova.nova_cache4_attention(own, cache, q, cu, o, lse=lse)
        nova.nova_cache4_weights(own, cache, q, lse, cu, w, weight_in=w)
        nova.nova_cache4_evict(own, cache, w, 200, 50, dst, weight_out=w_out)

    def state():
        return [t.clone() for t in (o, lse, w, dst.k_codes, dst.v_scales.view(torch.int16), dst.kv_len, w_out, cache.kv_len)]

    start = cache.kv_len.clone()
    once()
    want = state()
    cache.kv_len.copy_(start)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        once()
    torch.cuda.synchronize()
    for t in (o, lse, w_out):
        t.fill_(-1)
    for _ in range(2):
        cache.kv_len.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(state(), want):
            assert torch.equal(x, y)
    assert own.device_status() == 0
    # the next append goes behind these rows, eagerly and on another stream
    with torch.cuda.stream(side):
        nova.nova_cache4_append(own, cache, k, v, cu, stream=side)
    side.synchronize()
    assert cache.kv_len.tolist() == [506, 170]


@pytest.mark.parametrize("bad", [[0, 9, 4], [1, 4, 9], [0, 4, 11], [0, -3, 9]])
def test_debug_mode_refuses_bad_row_lists(bad):
    ctx = nova.Context(0)
    ctx.set_debug(True)
    C = 128
    cache, k, v = _filled(ctx, [5, 3], 20, C, 2, 1)
    before = [t.clone() for t in (cache.k_codes, cache.kv_len)]
    rows = _rows(2, 10, C).to(DEV)
    o, lse, w = torch.full_like(rows, 3.0), torch.full((2, 10), 3.0, device=DEV), torch.full((2, 20), 3.0, device=DEV)
    out = torch.full_like(rows, 3.0)
    ctx.ensure_cache4_workspace(cache, 10)
    for call in (lambda: nova.nova_cache4_append(ctx, cache, rows, rows, _i32(bad)), lambda: nova.nova_cache4_read(ctx, cache, _i32(bad), o, out),
                 lambda: nova.nova_cache4_attention(ctx, cache, rows, _i32(bad), o, lse=lse),
                 lambda: nova.nova_cache4_weights(ctx, cache, rows, lse, _i32(bad), w)):
        with pytest.raises(nova.NovaError) as e:
            call()
        assert e.value.status == 1
    assert torch.equal(cache.k_codes, before[0]) and torch.equal(cache.kv_len, before[1])
    for t in (o, out, lse, w):
        assert (t == 3.0).all()
    nova.nova_cache4_attention(ctx, cache, rows, _i32([0, 4, 10]), o, lse=lse)
    assert ctx.device_status() == 0 and torch.isfinite(o.float()).all()


def test_empty_calls_are_no_ops(ctx):
    C = 64
    cache = nova.Cache4.empty(2, 8, C, 1)
    nothing = torch.empty((0, C), dtype=torch.bfloat16, device=DEV)
    before = cache.kv_len.clone()
    nova.nova_cache4_append(ctx, cache, nothing, nothing, _cu([0, 0]))
    nova.nova_cache4_read(ctx, cache, _cu([0, 0]), nothing, nothing)
    nova.nova_cache4_attention(ctx, cache, nothing, _cu([0, 0]), nothing)
    w = torch.full((2, 8), 2.0, device=DEV)
    nova.nova_cache4_weights(ctx, cache, nothing, torch.empty((1, 0), device=DEV), _cu([0, 0]), w)
    assert torch.equal(cache.kv_len, before) and (w == 2.0).all()               # no rows in the cache: nothing to write
    cache.kv_len.fill_(3)
    nova.nova_cache4_weights(ctx, cache, nothing, torch.empty((1, 0), device=DEV), _cu([0, 0]), w)
    assert (w[:, :3] == 0).all() and (w[:, 3:] == 2.0).all()
    none = nova.Cache4.empty(0, 8, C, 1)
    nova.nova_cache4_attention(ctx, none, nothing, _cu([]), nothing)
    nova.nova_cache4_evict(ctx, none, torch.empty((0, 8), device=DEV), 4, 1, nova.Cache4.empty(0, 4, C, 1))
    flat = nova.Cache4.empty(1, 0, C, 1)
    q = _rows(1, 2, C).to(DEV)
    o = torch.full_like(q, 3.0)
    ctx.ensure_cache4_workspace(flat, 2)
    nova.nova_cache4_attention(ctx, flat, q, _cu([2]), o)
    assert (o == 0).all() and ctx.device_status() == 0


# ---- items shared by key ranges whose scores lie far apart ------------------------------------------------------------
def _apart(depth, C, n, half, zero):
    """Keys of one head of C channels, and a query's channels 0 and 32 with which their scores are, in units of log2, 0 for key `zero`, -1/2 for
    key `half` and -depth for all others."""
    k = torch.zeros((n, C))
    k[:, 0] = -7.0
    k[half, 0], k[half, 32] = 0.0, -7.0
    k[zero, 0] = 0.0
    unit = math.log(2.0) * math.sqrt(C) / 7.0
    return k.to(torch.bfloat16), depth * unit, 0.5 * unit


@pytest.mark.parametrize("C", [64, 128])
@pytest.mark.parametrize("rows", [24, 200, 300])
@pytest.mark.parametrize("depth", [60.0, 127.0, 140.0, 200.0])
@pytest.mark.parametrize("low_first", [True, False])
def test_attention_ranges_far_apart_share_a_row(ctx, C, rows, depth, low_first):
    """2500 keys are 20 tiles, shared by three CTAs (keys from 0, 768 and 1664): the range whose first tile lies `depth` below holds 0.41 of
    the weight, in a later key. Up to about 128 it does so against that tile, beyond it the item is run again."""
    n, heads = 2500, 1
    half, zero = (500, 770) if low_first else (1500, 5)
    k, q0, q32 = _apart(depth, C, n, half, zero)
    v = _rows(2, n, C)
    cache = nova.Cache4.empty(1, n, C, heads)
    nova.nova_cache4_append(ctx, cache, k.to(DEV), v.to(DEV), _cu([n]))
    q = _rows(3, rows, C)
    q[:, :64] = 0
    q[:, 0] = (q0 * (1.0 - 0.25 * (torch.arange(rows) % 4))).to(torch.bfloat16)
    q[:, 32] = q32
    ctx.ensure_cache4_workspace(cache, rows)
    o = torch.empty((rows, C), dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((heads, rows), device=DEV)
    nova.nova_cache4_attention(ctx, cache, q.to(DEV), _cu([rows]), o, lse=lse)
    assert ctx.device_status() == 0
    ref_o, ref_l, tol_o, tol_l = _ref_attention(q.double().numpy(), _ref_quantise(k)[0], _ref_quantise(v)[0], heads)
    assert np.all(np.abs(lse.double().cpu().numpy() - ref_l) <= tol_l)
    assert np.all(np.abs(o.double().cpu().numpy() - ref_o) <= tol_o)


@pytest.mark.parametrize("C", [64, 128])
@pytest.mark.parametrize("rows", [24, 200, 300])
@pytest.mark.parametrize("q_scale", [20.0, 40.0])
def test_attention_long_cache_scores_far_apart(ctx, C, rows, q_scale):
    """157 tiles shared by up to 26 CTAs, with scores of hundreds: the ranges' references lie far apart, and items are run again."""
    _check_attention(ctx, [20011], [rows], C, 1, seed=31, q_scale=q_scale)


@pytest.mark.parametrize("C,heads,rows", [(128, 2, 3), (128, 1, 70), (256, 2, 200)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 3e38])
def test_weights_of_queries_that_count_for_nothing(ctx, C, heads, rows, bad):
    """A query whose log-sum-exp is -inf adds nothing, whatever it holds, and not to a key that is NaN either."""
    n = 700
    cache, k, _ = _filled(ctx, [n], n + 20, C, heads, 1)
    q = _rows(2, rows, C).to(DEV)
    ctx.ensure_cache4_workspace(cache, rows)
    lse = torch.zeros((heads, rows), device=DEV)
    o = torch.empty_like(q)
    nova.nova_cache4_attention(ctx, cache, q, _cu([rows]), o, lse=lse)
    dead = list(range(1, rows, 3)) + [rows - 1]
    keep = [r for r in range(rows) if r not in dead]
    q_dead, lse_dead = q.clone(), lse.clone()
    q_dead[dead] = bad
    lse_dead[:, dead] = -math.inf
    out, two = (torch.zeros((1, n + 20), device=DEV) for _ in range(2))
    nova.nova_cache4_weights(ctx, cache, q_dead, lse_dead, _cu([rows]), out)
    nova.nova_cache4_weights(ctx, cache, q[keep].contiguous(), lse[:, keep].contiguous(), _cu([len(keep)]), two)
    # the same terms, all positive, in another order: at most rows * heads additions in each sum
    assert torch.allclose(out, two, rtol=2 * rows * heads * 2.0 ** -24, atol=0)
    cache.k_scales[0, 5] = float("nan")
    lse_dead.fill_(-math.inf)
    nova.nova_cache4_weights(ctx, cache, q_dead, lse_dead, _cu([rows]), out)
    assert (out == 0).all() and ctx.device_status() == 0
