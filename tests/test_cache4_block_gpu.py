"""The block and the scale runner on K/V caches in 4 bits: the calls on such a cache as they are used together."""
import math

import numpy as np
import pytest
import torch
import torch.nn.functional as F

import nova_synth as synth
import paper_2602_01345_b200 as nova
from paper_2602_01345_b200 import pipeline

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _cu(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV)


def _quantised(x):
    """bf16 rows as the cache holds them, float64."""
    g = x.double().cpu().reshape(x.shape[0], x.shape[1] // 32, 32).numpy()
    top = np.abs(g).max(-1, keepdims=True)
    m, e = np.frexp(top / 7.0)
    s = np.where(top > 0, np.ldexp(np.ceil(m * 32.0) / 32.0, e), 1.0)
    return torch.from_numpy((np.rint(g / s) * s).reshape(x.shape))


def _read(ctx, cache, counts, first=None):
    out = torch.empty((2, sum(counts), cache.C), dtype=torch.bfloat16, device=DEV)
    if sum(counts):
        nova.nova_cache4_read(ctx, cache, _cu(counts), out[0], out[1], first=first)
    return out[0].double().cpu(), out[1].double().cpu()


def _block64(wt, xc, k_old, v_old, k_new, v_new, heads, eps=1e-6):
    """One image in 64 bits, with the keys and values of the cache and of the new rows as they are held."""
    w = {n: t.double().cpu() for n, t in wt.tensors.items()}
    xc = xc.double().cpu()
    C = xc.shape[1]
    h = F.layer_norm(xc, (C,), w["ln1_g"], w["ln1_b"], eps)
    q = (F.linear(h, w["w_qkv"], w["b_qkv"])[:, :C]).view(-1, heads, C // heads)
    k = torch.cat((k_old, k_new)).view(-1, heads, C // heads)
    v = torch.cat((v_old, v_new)).view(-1, heads, C // heads)
    p = torch.softmax(torch.einsum("qhd,khd->hqk", q, k) / math.sqrt(C // heads), -1)
    o = torch.einsum("hqk,khd->qhd", p, v).reshape(-1, C)
    x1 = xc + F.linear(o, w["w_o"], w["b_o"])
    h2 = F.layer_norm(x1, (C,), w["ln2_g"], w["ln2_b"], eps)
    f = F.gelu(F.linear(h2, w["w_fc1"], w["b_fc1"]), approximate="tanh")
    return x1 + F.linear(f, w["w_fc2"], w["b_fc2"]), p.sum((0, 1))


def _case(C, heads, B, N, ks, lens, Lmax, seed):
    g = torch.Generator(device="cpu").manual_seed(seed)
    wt = nova.BlockWeights(synth.block_weights(C, 2 * C, seed, DEV), 1e-6)
    x = synth.activations(B, N, C, seed + 1, DEV)
    idx = torch.cat([torch.randperm(N, generator=g)[:k].sort().values for k in ks]).to(torch.int32).to(DEV)
    cache = nova.Cache4.empty(B, Lmax, C, heads)
    for t in (cache.k_codes, cache.v_codes):
        t.random_(0, 256)
    cache.k_scales.fill_(float("nan"))
    cache.v_scales.fill_(float("nan"))
    kv = torch.randn((2, sum(lens), C), generator=g).to(torch.bfloat16).to(DEV)
    return wt, x, idx, cache, kv


@pytest.mark.parametrize("C,heads,N,ks,lens", [(128, 2, 20, [7, 0, 20], [30, 4, 0]), (256, 2, 40, [40, 13], [200, 333]), (512, 8, 300, [290], [150]),
                                               (256, 2, 400, [390, 300], [500, 70])])
@pytest.mark.parametrize("on_device", [False, True])
def test_block_on_a_4_bit_cache(C, heads, N, ks, lens, on_device):
    ctx = nova.Context(0)
    B, M = len(ks), sum(ks)
    Lmax = max(a + b for a, b in zip(lens, ks)) + 2
    wt, x, idx, cache, kv = _case(C, heads, B, N, ks, lens, Lmax, 3)
    nova.nova_cache4_append(ctx, cache, kv[0], kv[1], _cu(lens))
    k_old, v_old = _read(ctx, cache, lens)
    cu = _cu(ks)
    bound = B * N if on_device else M
    shape = nova.BlockShape(B, N, C, heads, 2 * C, Lmax, bound)
    ctx.ensure_block_cache4_workspace(shape)
    if on_device:
        idx = torch.cat((idx, torch.zeros(bound - M, dtype=torch.int32, device=DEV)))
    weight = torch.zeros((B, Lmax), device=DEV)
    y = torch.full((bound, C), 7.0, dtype=torch.bfloat16, device=DEV)
    nova.nova_pruned_block_forward_cache4(ctx, wt, shape, x, idx, cu, cache, True, y, weight=weight, m_on_device=on_device)
    assert ctx.device_status() == 0
    assert (y[M:] == 7.0).all()
    assert cache.kv_len.tolist() == [a + b for a, b in zip(lens, ks)]
    # the new rows are those of the block on a bf16 cache, rounded
    k16 = torch.zeros((B, Lmax, C), dtype=torch.bfloat16, device=DEV)
    v16 = torch.zeros_like(k16)
    len16 = torch.tensor(lens, dtype=torch.int32, device=DEV)
    y16 = torch.empty_like(y)
    nova.nova_pruned_block_forward_ext(ctx, wt, None, None, shape, x, idx, cu, k16, v16, len16, False, y16, m_on_device=on_device)
    k_new, v_new = _read(ctx, cache, ks, first=torch.tensor(lens, dtype=torch.int32, device=DEV))
    rows = lambda t: torch.cat([t[b, n:n + k] for b, (n, k) in enumerate(zip(lens, ks))])  # noqa: E731
    assert torch.equal(k_new, _quantised(rows(k16))) and torch.equal(v_new, _quantised(rows(v16)))
    r0, o0 = 0, 0
    for b, (k, n) in enumerate(zip(ks, lens)):
        tokens = idx[r0:r0 + k].long()
        ref, w_ref = _block64(wt, x[b, tokens], k_old[o0:o0 + n], v_old[o0:o0 + n], k_new[r0:r0 + k], v_new[r0:r0 + k], heads)
        if k:
            # bf16 between the stages, as for the block on a bf16 cache: 2e-2 of the output's magnitude
            assert (y[r0:r0 + k].double().cpu() - ref).abs().max() <= 2e-2 * ref.abs().max()
            # h and q are rounded to bf16, 2^-8 relative each: a score moves by at most 2^-7 of the sum of its products' magnitudes
            # over sqrt(dh), which here is below 16, and a weight by that, relative
            got = weight[b, :n + k].double().cpu()
            assert (got - w_ref).abs().max() <= 2.0 ** -3 * w_ref.abs().max()
            assert abs(got.sum().item() / (heads * k) - 1) < 2.0 ** -10
        assert (weight[b, n + k:] == 0).all()
        r0, o0 = r0 + k, o0 + n


def test_block_without_append_leaves_lengths_and_equals_the_next_call():
    ctx = nova.Context(0)
    C, heads, N, ks, lens = 256, 4, 30, [30, 11], [64, 5]
    wt, x, idx, cache, kv = _case(C, heads, 2, N, ks, lens, 120, 5)
    nova.nova_cache4_append(ctx, cache, kv[0], kv[1], _cu(lens))
    shape = nova.BlockShape(2, N, C, heads, 2 * C, 120, sum(ks))
    ctx.ensure_block_cache4_workspace(shape)
    y, y2 = (torch.empty((sum(ks), C), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    nova.nova_pruned_block_forward_cache4(ctx, wt, shape, x, idx, _cu(ks), cache, False, y)
    assert cache.kv_len.tolist() == lens
    nova.nova_pruned_block_forward_cache4(ctx, wt, shape, x, idx, _cu(ks), cache, True, y2)
    assert cache.kv_len.tolist() == [94, 16] and torch.equal(y, y2) and ctx.device_status() == 0
    with pytest.raises(nova.NovaError):
        nova.nova_pruned_block_forward_cache4(ctx, wt, shape, x, idx, _cu(ks), cache, False, y, weight=torch.zeros((2, 120), device=DEV))
    small = nova.Context(0)
    with pytest.raises(nova.NovaError) as e:
        nova.nova_pruned_block_forward_cache4(small, wt, shape, x, idx, _cu(ks), cache, True, y)
    assert e.value.status == 4
    with pytest.raises(nova.NovaError) as e:
        nova.nova_pruned_block_forward_cache4(ctx, wt, nova.BlockShape(2, N, C, heads, 2 * C, 119, sum(ks)), x, idx, _cu(ks), cache, True, y)
    assert e.value.status == 1


def test_block_that_overflows_records_it():
    ctx = nova.Context(0)
    C, heads, N, ks, lens = 128, 2, 10, [10, 4], [20, 25]
    wt, x, idx, cache, kv = _case(C, heads, 2, N, ks, lens, 28, 6)
    nova.nova_cache4_append(ctx, cache, kv[0], kv[1], _cu(lens))
    cache.k_scales.nan_to_num_(0.0)
    cache.v_scales.nan_to_num_(0.0)
    shape = nova.BlockShape(2, N, C, heads, 2 * C, 28, sum(ks))
    ctx.ensure_block_cache4_workspace(shape)
    y = torch.empty((sum(ks), C), dtype=torch.bfloat16, device=DEV)
    nova.nova_pruned_block_forward_cache4(ctx, wt, shape, x, idx, _cu(ks), cache, True, y)
    assert ctx.device_status() == 2 and cache.kv_len.tolist() == lens


def test_block_with_the_parts_of_text_backbones():
    """Rotation, QK normalisation and cross-attention before and after the rounding: the new rows are again those of the bf16 block."""
    ctx = nova.Context(0)
    C, heads, N, ks, lens, Lc = 256, 2, 50, [50, 21], [40, 90], 24
    g = torch.Generator(device="cpu").manual_seed(9)
    wt, x, idx, cache, kv = _case(C, heads, 2, N, ks, lens, 160, 7)
    nova.nova_cache4_append(ctx, cache, kv[0], kv[1], _cu(lens))
    bf = lambda *s: (torch.randn(s, generator=g) * 0.05).to(torch.bfloat16).to(DEV)  # noqa: E731
    ang = torch.rand((N, C // heads // 2), generator=g).to(DEV)
    extras = dict(rope_cos=ang.cos(), rope_sin=ang.sin(), qk_gain_q=bf(C) + 2, qk_gain_k=bf(C) + 2, lnc_g=bf(C) + 1, lnc_b=bf(C), w_q2=bf(C, C),
                  b_q2=bf(C), w_o2=bf(C, C), b_o2=bf(C), cond_k=bf(2, Lc, C), cond_v=bf(2, Lc, C),
                  cond_len=torch.tensor([Lc, 3], dtype=torch.int32, device=DEV))
    mod = {"shift1": bf(2, C), "scale1": bf(2, C), "gate2": bf(2, C) + 1}
    shape = nova.BlockShape(2, N, C, heads, 2 * C, 160, sum(ks))
    ctx.ensure_block_cache4_workspace(shape)
    y, y16 = (torch.empty((sum(ks), C), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k_old, v_old = _read(ctx, cache, lens)
    nova.nova_pruned_block_forward_cache4(ctx, wt, shape, x, idx, _cu(ks), cache, True, y, modulation=mod, extras=extras)
    # the bf16 block on the rows that the cache stands for: the same up to the rounding of the new rows
    k16 = torch.zeros((2, 160, C), dtype=torch.bfloat16, device=DEV)
    v16 = torch.zeros_like(k16)
    at = np.concatenate([[0], np.cumsum(lens)])
    for b, n in enumerate(lens):
        k16[b, :n] = k_old[at[b]:at[b + 1]].to(torch.bfloat16).to(DEV)
        v16[b, :n] = v_old[at[b]:at[b + 1]].to(torch.bfloat16).to(DEV)
    len16 = torch.tensor(lens, dtype=torch.int32, device=DEV)
    nova.nova_pruned_block_forward_ext(ctx, wt, mod, extras, shape, x, idx, _cu(ks), k16, v16, len16, False, y16)
    assert ctx.device_status() == 0
    k_new, v_new = _read(ctx, cache, ks, first=torch.tensor(lens, dtype=torch.int32, device=DEV))
    rows = lambda t: torch.cat([t[b, n:n + k] for b, (n, k) in enumerate(zip(lens, ks))])  # noqa: E731
    assert torch.equal(k_new, _quantised(rows(k16))) and torch.equal(v_new, _quantised(rows(v16)))
    # new rows are off by at most half a step, 1/14 of their group's largest value, and weigh as the others: the attention's output, and with
    # weights of 0.02 the projection's, moves by less than 2^-4 of the block's output
    assert (y.double() - y16.double()).abs().max() <= 2.0 ** -4 * y16.double().abs().max()


@pytest.mark.parametrize("budget,recent", [(None, None), (40, None), (40, 0), (25, 25), (1000, 100)])
def test_generation_with_4_bit_caches(budget, recent):
    """All scales through MultiScaleRunner, every layer against 64 bits on the rows that its cache held, and the rows that stay
    against the definition."""
    ctx = nova.Context(0)
    C, heads, B, V, scales = 128, 2, 2, 64, (1, 2, 4, 6)
    weights = [synth.block_weights(C, 2 * C, 11 + j, DEV) for j in range(2)]
    run = pipeline.MultiScaleRunner(ctx, weights, heads, B, scales, cache_bits=4, cache_budget=budget, cache_recent=recent)
    sched = nova.SchedParams(force_act_scale=3, force_keep_ratio=0.6)
    g = torch.Generator(device="cpu").manual_seed(1)
    held = [[0] * B for _ in weights]
    for t, side in enumerate(scales, 1):
        N = side * side
        x = torch.randn((B, N, C), generator=g).to(torch.bfloat16).to(DEV)
        logits = [(torch.randn((B, N, V), generator=g) * 2).to(torch.bfloat16).to(DEV) for _ in range(3)]
        seen = {}

        def hook(stage, j, info):
            if stage == "before":
                seen["old"] = info["kv_len"].tolist()
                seen["kv"] = _read(ctx, info["cache4"], seen["old"])
                seen["weight"] = run.weights4[j].double().cpu() if run.weights4 else None
                return
            old, ks = seen["old"], info["keep"].tolist()
            assert old == held[j]
            k_new, v_new = _read(ctx, info["cache4"], ks, first=torch.tensor(old, dtype=torch.int32, device=DEV))
            assert info["kv_len"].tolist() == [a + b for a, b in zip(old, ks)]
            r0 = o0 = 0
            for b, (k, n) in enumerate(zip(ks, old)):
                tokens = info["keep_idx"][r0:r0 + k].long()
                ref, w_ref = _block64(run.block_weights[j], info["x_in"][b, tokens], seen["kv"][0][o0:o0 + n], seen["kv"][1][o0:o0 + n],
                                      k_new[r0:r0 + k], v_new[r0:r0 + k], heads)
                assert (info["x_out"][b, tokens].double().cpu() - ref).abs().max() <= 2e-2 * ref.abs().max()
                if run.weights4:
                    # as in the test of the block
                    got = run.weights4[j][b].double().cpu()
                    assert (got[:n + k] - seen["weight"][b, :n + k] - w_ref).abs().max() <= 2.0 ** -3 * w_ref.abs().max()
                    assert (got[n + k:] == 0).all()
                r0, o0 = r0 + k, o0 + n
                held[j][b] += k
            seen[j] = (run.weights4[j].clone() if run.weights4 else None, [_read(ctx, info["cache4"], held[j])])

        x_out, keeps, _ = run.run_scale(t, x, logits[0], logits[1:], sched, layer_hook=hook)
        assert ctx.device_status() == 0 and torch.isfinite(x_out.float()).all()
        for j in range(2):
            if budget is not None:
                w, [(k_all, v_all)] = seen[j]
                rec = min(N, budget) if recent is None else recent
                rows, o0 = [], 0
                for b, n in enumerate(held[j]):
                    keep = list(range(n))
                    if n > budget:
                        wb = w[b].tolist()
                        keep = sorted(sorted(range(n - rec), key=lambda i: (-wb[i], i))[:budget - rec]) + list(range(n - rec, n))
                    rows += [o0 + i for i in keep]
                    o0 += n
                    assert torch.equal(run.weights4[j][b, :len(keep)], w[b, keep]) and (run.weights4[j][b, len(keep):] == 0).all()
                    held[j][b] = len(keep)
                k_now, v_now = _read(ctx, run.caches4[j], held[j])
                assert torch.equal(k_now, k_all[rows]) and torch.equal(v_now, v_all[rows])
            assert run.caches4[j].kv_len.tolist() == held[j]


def test_generation_refuses_what_does_not_go_together():
    ctx = nova.Context(0)
    weights = [synth.block_weights(64, 128, 1, DEV)]
    for kw in (dict(cache_budget=5), dict(cache_bits=8), dict(cache_bits=4, on_device=True), dict(cache_bits=4, cache_budget=0),
               dict(cache_bits=4, cache_budget=5, cache_recent=6)):
        with pytest.raises(AssertionError):
            pipeline.MultiScaleRunner(ctx, weights, 1, 1, (1, 2), **kw)


@pytest.mark.parametrize("C,heads,N,ks,lens,Lmax", [(128, 2, 10, [10, 4], [20, 25], 30), (256, 2, 40, [40, 33, 17], [480, 90, 0], 520),
                                                     (128, 1, 300, [290, 300, 2], [20, 300, 598], 600), (256, 2, 300, [300, 280], [0, 360], 640)])
@pytest.mark.parametrize("refused", [0, 1])
def test_block_leaves_an_image_that_overflows_as_it_was(C, heads, N, ks, lens, Lmax, refused):
    """Its rows past kv_len hold codes of all kinds and scales of NaN: its queries attend to the rows that it has, its weights, rows and length stay, and the
    other images get what they get in a call in which nothing overflows."""
    ctx = nova.Context(0)
    B, M = len(ks), sum(ks)
    lens = list(lens)
    lens[refused] = Lmax - ks[refused] + 1
    wt, x, idx, cache, kv = _case(C, heads, B, N, ks, lens, Lmax, 6)
    nova.nova_cache4_append(ctx, cache, kv[0], kv[1], _cu(lens))
    fits = nova.Cache4.empty(B, Lmax, C, heads)       # the same rows, but for the last one of the image that is too long
    for a, b in zip((cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales), (fits.k_codes, fits.v_codes, fits.k_scales, fits.v_scales)):
        b.copy_(a)
    fits.kv_len.copy_(cache.kv_len)
    fits.kv_len[refused] -= 1
    shape = nova.BlockShape(B, N, C, heads, 2 * C, Lmax, M)
    ctx.ensure_block_cache4_workspace(shape)
    runs = []
    k_old, v_old = _read(ctx, cache, lens)
    for c in (cache, fits):
        before = [t.clone() for t in (c.k_codes, c.v_codes, c.k_scales.view(torch.int16), c.v_scales.view(torch.int16))]
        weight = torch.zeros((B, Lmax), device=DEV)
        for b in range(B):
            weight[b, :int(c.kv_len[b])] = 0.5
        y = torch.empty((M, C), dtype=torch.bfloat16, device=DEV)
        nova.nova_pruned_block_forward_cache4(ctx, wt, shape, x, idx, _cu(ks), c, True, y, weight=weight)
        assert ctx.device_status() == (2 if c is cache else 0)
        runs.append((y, weight, before))
    (y, weight, before), (y_fits, weight_fits, _) = runs
    at = np.concatenate([[0], np.cumsum(ks)])
    own = slice(at[refused], at[refused + 1])
    n = lens[refused]
    assert cache.kv_len.tolist() == [a + (k if b != refused else 0) for b, (a, k) in enumerate(zip(lens, ks))]
    assert (weight[refused, :n] == 0.5).all() and (weight[refused, n:] == 0).all()
    for t, old in zip((cache.k_codes, cache.v_codes, cache.k_scales.view(torch.int16), cache.v_scales.view(torch.int16)), before):
        assert torch.equal(t[refused], old[refused])
    o0 = sum(lens[:refused])
    none = torch.empty((0, C), dtype=torch.float64)
    ref, _ = _block64(wt, x[refused, idx[own].long()], k_old[o0:o0 + n], v_old[o0:o0 + n], none, none, heads)
    if n:
        assert (y[own].double().cpu() - ref).abs().max() <= 2e-2 * ref.abs().max()
    assert torch.isfinite(y.float()).all()
    for b in range(B):
        if b == refused:
            continue
        a, z = at[b], at[b + 1]
        # other images' sums may be cut into other parts: as in the test of the block
        if ks[b]:
            assert (y[a:z].double() - y_fits[a:z].double()).abs().max() <= 2e-2 * y_fits[a:z].double().abs().max()
        assert (weight[b] - weight_fits[b]).abs().max() <= 2.0 ** -10 * weight_fits[b].abs().max()
        assert (weight[b, lens[b] + ks[b]:] == 0).all()
        assert torch.equal(cache.k_codes[b, :lens[b] + ks[b]], fits.k_codes[b, :lens[b] + ks[b]])
        assert torch.equal(cache.v_codes[b, :lens[b] + ks[b]], fits.v_codes[b, :lens[b] + ks[b]])


def test_block_replays_from_a_graph():
    """Captured on a stream of its own and replayed: each replay appends and adds weights as another eager call does."""
    ctx = nova.Context(0)
    C, heads, N, ks, lens, Lmax = 256, 2, 40, [40, 13], [200, 333], 500
    wt, x, idx, cache, kv = _case(C, heads, 2, N, ks, lens, Lmax, 8)
    nova.nova_cache4_append(ctx, cache, kv[0], kv[1], _cu(lens))
    shape = nova.BlockShape(2, N, C, heads, 2 * C, Lmax, sum(ks))
    ctx.ensure_block_cache4_workspace(shape)
    weight = torch.zeros((2, Lmax), device=DEV)
    y = torch.empty((sum(ks), C), dtype=torch.bfloat16, device=DEV)
    cu, held = _cu(ks), (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales, cache.kv_len, weight)
    before = [t.clone() for t in held]

    def once():
        nova.nova_pruned_block_forward_cache4(ctx, wt, shape, x, idx, cu, cache, True, y, weight=weight)

    def state():
        n = cache.kv_len.tolist()
        rows = [t[b, :n[b]].view(torch.uint8).clone() for t in held[:4] for b in range(2)]
        return [n, y.clone(), weight.clone()] + rows

    eager = []
    for _ in range(3):
        once()
        eager.append(state())
    for t, b in zip(held, before):
        t.copy_(b)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        once()
    for ref in eager:
        graph.replay()
        got = state()
        assert got[0] == ref[0] and all(torch.equal(a, b) for a, b in zip(got[1:], ref[1:]))
    assert ctx.device_status() == 0
