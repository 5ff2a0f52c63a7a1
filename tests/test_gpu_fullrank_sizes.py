"""AdamW, its moments and the gradient norm at the sizes of real models, against their 64-bit forms: chunks of 4096 elements (from 1024 of them on), the norm's
chunks of 16384, more tensors and more gradients by rows than one launch takes, arrays beyond 2^31 elements and 2^32 bytes."""
import math

import numpy as np
import pytest

from tests import fullrank_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available()
    from paper_2602_04396_amd import lordo
    lordo.load()
    yield t
    t.cuda.empty_cache()


def _gen(torch, seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tensor(torch, gen, rows, cols, dtype, size, shift=0):
    flat = torch.empty(rows * cols + shift, dtype=dtype, device="cuda")
    flat.copy_(torch.randn(flat.shape, generator=gen, device="cuda") * size)
    return flat[shift:].view(rows, cols)


def _starts(shapes):
    out, at = [], 0
    for sh in shapes:
        out.append(at)
        at += (sh[0] * sh[1] + 127) // 128 * 128
    return out, at


def _np(t):
    return t.detach().double().cpu().numpy().reshape(-1)


def _compare(hp, q8, bf, t, lr, decay, w0, u0, v0, g, first, w1, u1, v1):
    """Elements from `first` of a tensor on, before and after step t."""
    wd = hp.weight_decay if decay else 0.0
    w, u, v, size = ref.adamw(w0, u0, v0, g, t, lr, hp.beta1, hp.beta2, hp.eps, wd, bool(hp.bias_correction))
    bw, bu, bv = ref.adamw_bounds(w, w0, hp.beta1 * np.abs(u0) + (1 - hp.beta1) * np.abs(g), v, size, lr, wd, bf)
    assert np.all(np.abs(w1 - w) <= bw)
    if q8:
        wu, wv = (x[first:] for x in ref.thresholds(t, first + w.size)) if first < 1 << 24 else _thresholds_from(t, first, w.size)
        assert np.array_equal(u1, ref.in_8_bits_of_many(u, wu, True).astype(np.float32))
        assert np.array_equal(v1, ref.in_8_bits_of_many(v, wv, False).astype(np.float32))
    else:
        assert np.all(np.abs(u1 - u) <= bu) and np.all(np.abs(v1 - v) <= bv)


def _thresholds_from(t, first, n):
    x = [((t * 0x9E3779B1) + i * 0xBB67AE85) & 0xFFFFFFFF for i in range(first, first + n)]
    x = [((a ^ a >> 15) * 0x6A09E667) & 0xFFFFFFFF for a in x]
    x = [a ^ a >> 14 for a in x]
    return np.array([a >> 15 for a in x]), np.array([a & 0x1FFFF for a in x])


SETS = {
    "odd": [(4099, 1031), (1, 777, 0), (3, 129), (1, 1)],                 # 1032 chunks of 4096, a ragged one, and three small tensors
    "border": [(1024, 4096)],                                             # exactly 1024 chunks
    "below": [(1023, 4096)],                                              # the largest set in chunks of 1024
    "many": [(1, 16400 + 37 * k, k % 2) for k in range(261)],             # more tensors than a launch, five or six chunks each
}


@pytest.mark.parametrize("which", sorted(SETS))
@pytest.mark.parametrize("state", ["f32", "q8"])
@pytest.mark.parametrize("w_bf16, g_bf16, shift", [(False, False, 0), (True, True, 0), (False, True, 1), (True, False, 3)])
def test_steps_of_large_sets(torch, which, state, w_bf16, g_bf16, shift):
    from paper_2602_04396_amd import lordo
    shapes, gen, types, q8 = SETS[which], _gen(torch, 5), [torch.float32, torch.bfloat16], state == "q8"
    hp = lordo.adamw_hparams(weight_decay=0.1, param_dtype=lordo.BF16 if w_bf16 else lordo.F32, state_dtype=lordo.Q8 if q8 else lordo.F32)
    opt = lordo.AdamW(shapes, hp, torch)
    starts, total = _starts(shapes)
    W = [_tensor(torch, gen, sh[0], sh[1], types[w_bf16], 0.02, shift) for sh in shapes]
    gap = np.ones(2 * total, dtype=bool)
    for k in range(2):
        G = [_tensor(torch, gen, sh[0], sh[1], types[g_bf16], 1e-3 * 8.0 ** k, shift) for sh in shapes]
        w0, m0 = [_np(w) for w in W], _np(opt.export_moments())
        opt.local_step(W, G, 1e-2, grad_scale=0.37)
        m1 = _np(opt.export_moments())
        for i, sh in enumerate(shapes):
            n, s = sh[0] * sh[1], starts[i]
            gap[s:s + n] = gap[total + s:total + s + n] = False
            _compare(hp, q8, w_bf16, k + 1, 1e-2, len(sh) < 3 or sh[2], w0[i], m0[s:s + n], m0[total + s:total + s + n], 0.37 * _np(G[i]), 0,
                     _np(W[i]), m1[s:s + n], m1[total + s:total + s + n])
        assert not m1[gap].any()
    opt.poll_status()


@pytest.mark.parametrize("which", ["odd", "many"])
def test_moments_of_large_sets(torch, which):
    """Out and in again: fp32 moments as they are, 8-bit ones on their grid and then the same; nothing between the tensors."""
    from paper_2602_04396_amd import lordo
    shapes, gen = SETS[which], _gen(torch, 7)
    starts, total = _starts(shapes)
    real = torch.zeros(total, dtype=torch.bool, device="cuda")
    for s, sh in zip(starts, shapes):
        real[s:s + sh[0] * sh[1]] = True
    src = torch.randn(2, total, generator=gen, device="cuda") * torch.exp2(torch.randn(2, total, generator=gen, device="cuda") * 6)
    src[1].abs_()
    half = np.full(total, 1 << 16)
    for q8 in (False, True):
        opt = lordo.AdamW(shapes, lordo.adamw_hparams(state_dtype=lordo.Q8 if q8 else lordo.F32), torch)
        opt.import_moments(src)
        out = opt.export_moments()
        assert not out[:, ~real].any()
        if not q8:
            assert torch.equal(out, src * real) and torch.equal(opt.sync_payload(), out)
            continue
        for row, signed in ((0, True), (1, False)):
            assert np.array_equal(out[row].cpu().numpy(), ref.in_8_bits_of_many(_np(src[row] * real), half, signed).astype(np.float32))
        opt.import_moments(out)
        assert torch.equal(opt.export_moments(), out)


def _by_rows(torch, lordo, gen, vocab, cols, slots, dtype, every):
    """(by rows, dense) of the same gradient; rows of data that hold nothing are NaN."""
    rows = _tensor(torch, gen, slots, cols, dtype, 1.0)
    held = torch.randperm(slots, generator=gen, device="cuda")[:len(range(0, vocab, every))]
    at = torch.arange(0, vocab, every, device="cuda")[:len(held)]
    index = torch.full((vocab + slots,), -1, dtype=torch.int32, device="cuda")
    index[at], index[vocab + held] = held.int(), at.int()
    dense = torch.zeros(vocab, cols, dtype=dtype, device="cuda")
    dense[at] = rows[held]
    rows[index[vocab:] < 0] = float("nan")
    return lordo.RowGrad(rows, index, vocab), dense


@pytest.mark.parametrize("vocab, cols", [(4099, 1031), (70001, 61)])
@pytest.mark.parametrize("g_bf16", [False, True])
@pytest.mark.parametrize("w_bf16", [False, True])
def test_large_gradient_by_rows_is_the_dense_one(torch, vocab, cols, g_bf16, w_bf16):
    """Bit for bit; the norm of the rows to what its order of summing leaves."""
    from paper_2602_04396_amd import lordo
    types, gen = [torch.float32, torch.bfloat16], _gen(torch, 9)
    by_rows, dense = _by_rows(torch, lordo, gen, vocab, cols, vocab // 2, types[g_bf16], 3)
    shapes = [(1, 50, 0), (vocab, cols), (1, 3)]
    extra = [torch.randn(sh[0], sh[1], generator=gen, device="cuda") for sh in (shapes[0], shapes[2])]
    for q8 in (False, True):
        hp = lordo.adamw_hparams(weight_decay=0.1, param_dtype=lordo.BF16 if w_bf16 else lordo.F32, state_dtype=lordo.Q8 if q8 else lordo.F32)
        results = []
        for g in (dense, by_rows):
            opt = lordo.AdamW(shapes, hp, torch)
            W = [_tensor(torch, _gen(torch, 10), sh[0], sh[1], types[w_bf16], 0.02) for sh in shapes]
            for _ in range(2):
                opt.local_step(W, [extra[0], g, extra[1]], 1e-2)
            results.append(W + [opt.export_moments()])
        assert all(torch.equal(a, b) for a, b in zip(*results))
    a, b = lordo.grad_norm([extra[0], dense, extra[1]], 1.0), lordo.grad_norm([extra[0], by_rows, extra[1]], 1.0)
    assert torch.isfinite(a).all() and torch.all((a - b).abs() <= 2 ** -23 * a.abs())


@pytest.mark.parametrize("count", [8, 9, 16, 17])
def test_many_gradients_by_rows(torch, count):
    """A launch takes eight gradients by rows; dense ones between them, and rows that hold nothing."""
    from paper_2602_04396_amd import lordo
    gen = _gen(torch, 11)
    shapes, G, dense = [], [], []
    for k in range(count):
        vocab, cols = 30 + k, 17 + 40 * k
        r, d = _by_rows(torch, lordo, gen, vocab, cols, 20, [torch.float32, torch.bfloat16][k % 2], 5 if k % 3 else 1000)
        if k % 7 == 6:
            r, d = lordo.RowGrad(r.rows[:0], r.index[:vocab].fill_(-1), vocab), torch.zeros_like(d)
        shapes += [(vocab, cols), (1, 33, 0)]
        small = torch.randn(1, 33, generator=gen, device="cuda")
        G += [r, small]
        dense += [d, small]
    want = math.sqrt(sum(float((d.double() ** 2).sum()) for d in dense))
    out = lordo.grad_norm(G, 0.5 * want)
    assert abs(float(out[0]) - want) <= 1.01 * ref.EPS32 * want and abs(float(out[1]) - 0.5) <= 1.01 * ref.EPS32
    for q8 in (False, True):
        results = []
        for grads in (dense, G):
            opt = lordo.AdamW(shapes, lordo.adamw_hparams(weight_decay=0.1, state_dtype=lordo.Q8 if q8 else lordo.F32), torch)
            W = [_tensor(torch, _gen(torch, 10 + i), sh[0], sh[1], torch.float32, 0.02) for i, sh in enumerate(shapes)]
            for _ in range(3):
                opt.local_step(W, grads, 1e-2)
            results.append(W + [opt.export_moments()])
        assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("sizes", [[17000001, 5, 100003], [320 * 16384], [319 * 16384], [319 * 16384 + 1], [1] * 319 + [16385], [1024 * 16384], [1023 * 16384 + 1], [3 + 31 * k % 977 for k in range(201)], [1 + 17 * k % 5001 for k in range(650)],
                                   [90000 + k for k in range(401)]])
@pytest.mark.parametrize("bf16, shift", [(False, 0), (True, 0), (False, 1), (True, 3)])
def test_norm_of_large_sets(torch, sizes, bf16, shift):
    from paper_2602_04396_amd import lordo
    gen = _gen(torch, 12)
    G = [_tensor(torch, gen, 1, n, torch.bfloat16 if bf16 else torch.float32, 1.0, shift) for n in sizes]
    want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in G))
    for _ in range(2):                                   # (the second call finds the sums of the first in whatever memory it gets)
        out = lordo.grad_norm(G, 0.5 * want)
        assert abs(float(out[0]) - want) <= 1.01 * ref.EPS32 * want and abs(float(out[1]) - 0.5) <= 1.01 * ref.EPS32
    for k in (0, len(G) - 1):                            # a value that is not finite in the first launch or in the last
        keep = G[k][0, 0].clone()
        G[k][0, 0] = float("nan")
        assert torch.isnan(lordo.grad_norm(G, 1.0)).all()
        G[k][0, 0] = keep


@pytest.mark.parametrize("vocab, cols, slots", [(9000, 2050, 8300), (60000, 300, 57000), (50, 5000, 3400)])
def test_norm_of_large_gradients_by_rows(torch, vocab, cols, slots):
    """Chunks of 16384 over rows longer and shorter than the width from which rows are taken one by one."""
    from paper_2602_04396_amd import lordo
    assert slots * cols >= 1024 * 16384
    gen = _gen(torch, 13)
    for dtype in (torch.float32, torch.bfloat16):
        r, d = _by_rows(torch, lordo, gen, vocab, cols, slots, dtype, 2)
        want = math.sqrt(float((d.double() ** 2).sum()))
        out = lordo.grad_norm([r], 0.5 * want)
        assert abs(float(out[0]) - want) <= 1.01 * ref.EPS32 * want and abs(float(out[1]) - 0.5) <= 1.01 * ref.EPS32


FAR = (524309, 4099)                                     # 2149142591 elements


@pytest.mark.parametrize("state", ["f32", "q8"])
def test_step_of_a_tensor_beyond_32_bits(torch, state):
    """Elements at the beginning, around 2^31 and at the end against the reference."""
    from paper_2602_04396_amd import lordo
    n, q8 = FAR[0] * FAR[1], state == "q8"
    assert n > 1 << 31
    hp = lordo.adamw_hparams(weight_decay=0.1, param_dtype=lordo.BF16, state_dtype=lordo.Q8 if q8 else lordo.F32)
    opt = lordo.AdamW([FAR], hp, torch)
    W, G = torch.zeros(FAR, dtype=torch.bfloat16, device="cuda"), torch.zeros(FAR, dtype=torch.bfloat16, device="cuda")
    spans = [(0, 5000), ((1 << 31) - 2560, (1 << 31) + 2560), (n // 128 * 128 - 1280, n)]
    gen, w, g = _gen(torch, 14), W.view(-1), G.view(-1)
    for a, b in spans:
        w[a:b] = torch.randn(b - a, generator=gen, device="cuda").bfloat16()
        g[a:b] = torch.randn(b - a, generator=gen, device="cuda").bfloat16()
    w0, g0 = [_np(w[a:b]) for a, b in spans], [_np(g[a:b]) for a, b in spans]
    want = math.sqrt(sum(float((x ** 2).sum()) for x in g0))
    out = lordo.grad_norm([G], 1.0)
    assert abs(float(out[0]) - want) <= 1.01 * ref.EPS32 * want
    opt.local_step([W], [G], 1e-2)
    m = opt.export_moments() if q8 else opt.sync_payload()
    for (a, b), x0, y in zip(spans, w0, g0):
        zero = np.zeros(b - a)
        _compare(hp, q8, True, 1, 1e-2, 1, x0, zero, zero, y, a, _np(w[a:b]), _np(m[0, a:b]), _np(m[1, a:b]))
    idle = slice(spans[0][1] + 128, spans[1][0] - 128)
    assert not w[idle].any() and not m[0, idle].any()


def test_gradient_by_rows_beyond_32_bits(torch):
    """Rows of data behind 2^31 elements belong to a small tensor."""
    from paper_2602_04396_amd import lordo
    slots, cols, vocab = FAR[0], FAR[1], 40
    rows = torch.zeros(slots, cols, dtype=torch.bfloat16, device="cuda")
    index = torch.full((vocab + slots,), -1, dtype=torch.int32, device="cuda")
    dense = torch.zeros(vocab, cols, dtype=torch.bfloat16, device="cuda")
    gen = _gen(torch, 15)
    for k in range(0, vocab, 3):
        slot = slots - 1 - 7 * k if k % 2 else 5 * k
        rows[slot] = torch.randn(cols, generator=gen, device="cuda").bfloat16()
        dense[k] = rows[slot]
        index[k], index[vocab + slot] = slot, k
    r = lordo.RowGrad(rows, index, vocab)
    results = []
    for g in (dense, r):
        opt = lordo.AdamW([(vocab, cols)], lordo.adamw_hparams(), torch)
        W = [torch.ones(vocab, cols, device="cuda")]
        opt.local_step(W, [g], 1e-2)
        results.append(W + [opt.export_moments()])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    want = math.sqrt(float((dense.double() ** 2).sum()))
    assert abs(float(lordo.grad_norm([r])[0]) - want) <= 1.01 * ref.EPS32 * want


@pytest.mark.parametrize("state", ["f32", "q8"])
def test_recorded_steps_of_large_sets(torch, state):
    """Many tensors in two launches, one of them by rows, with its norm: replays beside the same steps issued, synchronised in between."""
    from paper_2602_04396_amd import lordo
    shapes = [(1, 16400 + 37 * k, k % 2) for k in range(230)] + [(9001, 60)]
    gen = _gen(torch, 16)
    hp = lordo.adamw_hparams(weight_decay=0.1, param_dtype=lordo.BF16, state_dtype=lordo.Q8 if state == "q8" else lordo.F32)
    W = [_tensor(torch, gen, sh[0], sh[1], torch.bfloat16, 0.02) for sh in shapes]
    V = [w.clone() for w in W]
    G = [_tensor(torch, gen, sh[0], sh[1], torch.float32, 1.0) for sh in shapes[:-1]]
    ids, dy = torch.zeros(12000, dtype=torch.int64, device="cuda"), torch.zeros(12000, 60, device="cuda")
    eager, twin = lordo.AdamW(shapes, hp, torch), lordo.AdamW(shapes, hp, torch)
    PW, PV = eager.ptrs(W), twin.ptrs(V)

    def step(opt, weights):
        grads = G + [lordo.embed_gradient_rows(ids, dy, 9001)]
        clip = lordo.grad_norm(grads, 1.0)
        opt.local_step(weights, grads, 1e-2, clip=clip)
        return clip

    step(lordo.AdamW(shapes, hp, torch), [w.clone() for w in W])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step(twin, PV)
    for k in range(4):
        ids.copy_(torch.randint(-1, 9001, ids.shape, generator=gen, device="cuda"))
        dy.copy_(torch.randn(dy.shape, generator=gen, device="cuda"))
        for g in G:
            g.copy_(torch.randn(g.shape, generator=gen, device="cuda"))
        clip = step(eager, PW)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(clip, recorded) and all(torch.equal(a, b) for a, b in zip(W, V))
        assert torch.equal(eager.export_moments(), twin.export_moments()) and eager.steps_taken() == twin.steps_taken() == k + 1
    graph.reset()
