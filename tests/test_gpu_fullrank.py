"""AdamW over many tensors and the gradient norm against their 64-bit forms.  Every step is compared on its own: the reference starts from the
weights and moments that the library held before it."""
import ctypes as C
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
    return t


def _gen(torch, seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tensor(torch, gen, rows, cols, dtype, size, shift=0):
    """Contiguous random tensor that begins `shift` elements behind an aligned address."""
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


def _check_step(torch, opt, shapes, W, G, lr, scale=1.0, clip=None, dense=None):
    """One step of the library against the reference from the same start; `dense`: the gradients as plain tensors."""
    from paper_2602_04396_amd import lordo
    hp, q8, bf = opt.hp, opt.hp.state_dtype == lordo.Q8, opt.hp.param_dtype == lordo.BF16
    w0, m0 = [_np(w) for w in W], _np(opt.export_moments())
    t = opt.step + 1
    opt.local_step(W, G, lr, grad_scale=scale, clip=clip)
    m1 = _np(opt.export_moments())
    starts, total = _starts(shapes)
    coef = 1.0 if clip is None else float(clip[1])
    gap = np.ones(2 * total, dtype=bool)
    for i, sh in enumerate(shapes):
        n, s = sh[0] * sh[1], starts[i]
        gap[s:s + n] = gap[total + s:total + s + n] = False
        g = scale * coef * _np((dense or G)[i])
        u0, v0 = m0[s:s + n], m0[total + s:total + s + n]
        wd = hp.weight_decay if len(sh) < 3 or sh[2] else 0.0
        w, u, v, size = ref.adamw(w0[i], u0, v0, g, t, lr, hp.beta1, hp.beta2, hp.eps, wd, bool(hp.bias_correction))
        bw, bu, bv = ref.adamw_bounds(w, w0[i], hp.beta1 * np.abs(u0) + (1 - hp.beta1) * np.abs(g), v, size, lr, wd, bf)
        assert np.all(np.abs(_np(W[i]) - w) <= bw), f"weights of tensor {i} {sh}"
        gu, gv = m1[s:s + n], m1[total + s:total + s + n]
        if q8:
            wu, wv = ref.thresholds(t, n)
            assert np.array_equal(gu, ref.in_8_bits(u, wu, True).astype(np.float32)), f"u of tensor {i} {sh}"
            assert np.array_equal(gv, ref.in_8_bits(v, wv, False).astype(np.float32)), f"v of tensor {i} {sh}"
        else:
            assert np.all(np.abs(gu - u) <= bu), f"u of tensor {i} {sh}"
            assert np.all(np.abs(gv - v) <= bv), f"v of tensor {i} {sh}"
    assert not m1[gap].any()


SETS = {
    "lengths": [(1, n, n % 2) for n in (1, 2, 3, 4, 5, 127, 128, 129, 255, 1023, 1024, 1025, 4095, 4096, 4097, 8191)],
    "matrices": [(37, 129), (513, 1000), (1, 4099, 0), (300, 64)],
    "many": [(1, 1 + 7 * k % 300, k % 2) for k in range(251)],
    "long": [(1021, 1031), (3, 400000)],
}


@pytest.mark.parametrize("which", sorted(SETS))
@pytest.mark.parametrize("state", ["f32", "q8"])
@pytest.mark.parametrize("w_bf16, g_bf16, shift", [(False, False, 0), (True, True, 0), (False, True, 1), (True, False, 3)])
def test_steps(torch, which, state, w_bf16, g_bf16, shift):
    from paper_2602_04396_amd import lordo
    shapes = SETS[which]
    gen = _gen(torch, 5)
    types = [torch.float32, torch.bfloat16]
    hp = lordo.adamw_hparams(weight_decay=0.1, param_dtype=lordo.BF16 if w_bf16 else lordo.F32, state_dtype=lordo.Q8 if state == "q8" else lordo.F32)
    opt = lordo.AdamW(shapes, hp, torch)
    W = [_tensor(torch, gen, sh[0], sh[1], types[w_bf16], 0.02, shift) for sh in shapes]
    for k in range(3):
        G = [_tensor(torch, gen, sh[0], sh[1], types[g_bf16], 1e-3 * 8.0 ** k, shift) for sh in shapes]
        _check_step(torch, opt, shapes, W, G, 1e-2, scale=1.0 if k else 0.37)
    opt.poll_status()
    assert opt.step == 3


@pytest.mark.parametrize("state", ["f32", "q8"])
def test_options(torch, state):
    """eps = 0 where no gradient ever was, no bias correction, no decay, a far step count, values of all sizes in one block, a learning rate of zero."""
    from paper_2602_04396_amd import lordo
    shapes, gen = [(1, 700), (5, 128)], _gen(torch, 6)
    q = lordo.Q8 if state == "q8" else lordo.F32
    for kw, t0 in ((dict(eps=0.0), 0), (dict(eps=2.0 ** -100, beta2=1 - 2.0 ** -40), 0), (dict(eps=1e-13), 5), (dict(bias_correction=False, weight_decay=0.3), 0), (dict(beta1=0.0, beta2=0.0), 7), (dict(), 10 ** 9)):
        opt = lordo.AdamW(shapes, lordo.adamw_hparams(state_dtype=q, **kw), torch)
        opt.step = t0
        W = [_tensor(torch, gen, *sh, torch.float32, 0.02) for sh in shapes]
        for k in range(2):
            G = [_tensor(torch, gen, *sh, torch.float32, 1.0) for sh in shapes]
            G[0].mul_(torch.exp2(torch.randn(G[0].shape, generator=gen, device="cuda") * 12))
            if kw.get("eps", 1) < 1e-20:
                G[0][:, 100:] = 0
                G[1].zero_()
            _check_step(torch, opt, shapes, W, G, 1e-2 if k == 0 else 0.0)
            assert all(torch.isfinite(w).all() for w in W)


def test_not_finite_gradients_stay_where_they_are(torch):
    """fp32 moments: in their element; 8-bit ones: in the moments of their block of 128.  Other blocks and tensors go on."""
    from paper_2602_04396_amd import lordo
    for bad in (float("inf"), float("nan")):
        for q8 in (False, True):
            shapes = [(1, 300), (1, 40)]
            opt = lordo.AdamW(shapes, lordo.adamw_hparams(state_dtype=lordo.Q8 if q8 else lordo.F32), torch)
            W = [torch.ones(sh, device="cuda") for sh in shapes]
            G = [torch.ones(sh, device="cuda") for sh in shapes]
            G[0][0, 130] = bad
            opt.local_step(W, G, 1e-2)
            G[0][0, 130] = 1.0
            opt.local_step(W, G, 1e-2)
            ok = torch.isfinite(W[0][0])
            hit = torch.zeros(300, dtype=torch.bool, device="cuda")
            if q8:
                hit[128:256] = True
            hit[130] = True
            assert torch.equal(~ok, hit) and torch.isfinite(W[1]).all()
            m = opt.export_moments()
            assert torch.equal(torch.isfinite(m[0][:300]), ~hit) and torch.isfinite(m[:, 384:]).all()


def test_moments_in_and_out(torch):
    """What is exported comes back as it was; fp32 moments are the payload view; what is given between the tensors is not kept."""
    from paper_2602_04396_amd import lordo
    shapes, gen = [(1, 130), (7, 33), (1, 1)], _gen(torch, 7)
    starts, total = _starts(shapes)
    real = torch.zeros(total, dtype=torch.bool, device="cuda")
    for s, sh in zip(starts, shapes):
        real[s:s + sh[0] * sh[1]] = True
    src = torch.randn(2, total, generator=gen, device="cuda") * torch.exp2(torch.randn(2, total, generator=gen, device="cuda") * 6)
    src[1].abs_()
    for q8 in (False, True):
        opt = lordo.AdamW(shapes, lordo.adamw_hparams(state_dtype=lordo.Q8 if q8 else lordo.F32), torch)
        assert not opt.export_moments().any()
        opt.import_moments(src)
        out = opt.export_moments()
        assert not out[:, ~real].any()
        if not q8:
            assert torch.equal(out, src * real) and torch.equal(opt.sync_payload(), out)
        else:
            half = np.full(total, 1 << 16)
            for s, sh in zip(starts, shapes):
                n = sh[0] * sh[1]
                for row, signed in ((0, True), (1, False)):
                    want = ref.in_8_bits(_np(src[row][s:s + n]), half[:n], signed).astype(np.float32)
                    assert np.array_equal(out[row][s:s + n].cpu().numpy(), want)
            with pytest.raises(ValueError):
                opt.sync_payload()
            opt.import_moments(out)
            assert torch.equal(opt.export_moments(), out)


def test_moments_in_8_bits_follow_slow_changes(torch):
    """v of elements without a gradient shrinks by 1 - beta2 a step, far below half a step of the grid (1/16), beside one whose large gradient holds the
    exponent.  After 2000 steps its mean over 4064 elements is 0.135 of what it was: each step keeps the expectation, and the spread, sixteen or seventeen
    values further with a time on each as random as its mean, is at most 0.5 of the mean, 0.8 % of it for the mean of 4064; 5 % are six of those."""
    from paper_2602_04396_amd import lordo
    shapes = [(32, 128)]
    opt = lordo.AdamW(shapes, lordo.adamw_hparams(state_dtype=lordo.Q8), torch)
    W, G = [torch.zeros(shapes[0], device="cuda")], torch.zeros(shapes[0], device="cuda")
    start = torch.full((2, 32 * 128), 1e-4, device="cuda")
    start[1].view(32, 128)[:, 0] = 1.0
    opt.import_moments(start)
    v0 = opt.export_moments()[1].view(32, 128)[:, 1:].clone()
    G[:, 0] = 1.0
    for _ in range(2000):
        opt.local_step(W, [G], 0.0)
    ratio = (opt.export_moments()[1].view(32, 128)[:, 1:] / v0).double()
    assert abs(float(ratio.mean()) / 0.999 ** 2000 - 1) <= 0.05


def test_clip_and_steps_left_out(torch):
    from paper_2602_04396_amd import lordo
    for q8 in (False, True):
        shapes, gen = [(40, 65), (1, 9, 0)], _gen(torch, 8)
        opt = lordo.AdamW(shapes, lordo.adamw_hparams(weight_decay=0.1, state_dtype=lordo.Q8 if q8 else lordo.F32), torch)
        W = [_tensor(torch, gen, *sh[:2], torch.float32, 0.02) for sh in shapes]
        G = [_tensor(torch, gen, *sh[:2], torch.float32, 1.0) for sh in shapes]
        clip = lordo.grad_norm(G, 0.5)
        assert 0 < float(clip[1]) < 0.02
        _check_step(torch, opt, shapes, W, G, 1e-2, scale=2.0, clip=clip)
        opt.poll_status()
        before, m = [w.clone() for w in W], opt.export_moments()
        G[0][3, 4] = float("nan")
        opt.local_step(W, G, 1e-2, clip=lordo.grad_norm(G, 0.5))
        assert all(torch.equal(a, b) for a, b in zip(W, before)) and torch.equal(opt.export_moments(), m)
        with pytest.raises(lordo.LordoError) as e:
            opt.poll_status()
        assert e.value.code == lordo.ENUMERIC
        opt.poll_status()
        assert opt.step == 2                                     # issued; the device went on counting from one
        other = lordo.AdamW(shapes, opt.hp, torch)
        other.import_moments(m)
        other.step = 1
        W2 = [w.clone() for w in W]
        G[0][3, 4] = 1.0
        opt.local_step(W, G, 1e-2)
        other.local_step(W2, G, 1e-2)
        assert all(torch.equal(a, b) for a, b in zip(W, W2)) and torch.equal(opt.export_moments(), other.export_moments())


@pytest.mark.parametrize("cols", [1, 3, 64, 129, 5000])
@pytest.mark.parametrize("g_bf16", [False, True])
def test_gradient_by_rows_is_the_dense_one(torch, cols, g_bf16):
    """Bit for bit: the rows in any order, rows of data that hold nothing (NaN there), indices out of range."""
    from paper_2602_04396_amd import lordo
    vocab, slots, gen = 97, 40, _gen(torch, 9)
    dtype = torch.bfloat16 if g_bf16 else torch.float32
    rows = _tensor(torch, gen, slots, cols, dtype, 1.0)
    index = torch.full((vocab + slots,), -1, dtype=torch.int32, device="cuda")
    dense = torch.zeros(vocab, cols, dtype=dtype, device="cuda")
    for k, (row, slot) in enumerate(zip(range(0, vocab, 5), [7 * j % slots for j in range(1, 40, 2)])):
        index[row], index[vocab + slot] = slot, row
        dense[row] = rows[slot]
    for slot in range(slots):
        if index[vocab + slot] < 0:
            rows[slot] = float("nan")
    index[1], index[2] = slots, -7
    by_rows = lordo.RowGrad(rows, index, vocab)
    shapes = [(1, 50), (vocab, cols), (1, 3)]
    extra = [torch.randn(sh[0], sh[1], generator=gen, device="cuda") for sh in (shapes[0], shapes[2])]
    for q8 in (False, True):
        state = []
        for g in (dense, by_rows):
            hp = lordo.adamw_hparams(weight_decay=0.1, state_dtype=lordo.Q8 if q8 else lordo.F32)
            opt = lordo.AdamW(shapes, hp, torch)
            W = [_tensor(torch, _gen(torch, 10), *sh, torch.float32, 0.02) for sh in shapes]
            for _ in range(2):
                opt.local_step(W, [extra[0], g, extra[1]], 1e-2)
            state.append(W + [opt.export_moments()])
        assert all(torch.equal(a, b) for a, b in zip(*state))
    a, b = lordo.grad_norm([extra[0], dense, extra[1]], 1.0), lordo.grad_norm([extra[0], by_rows, extra[1]], 1.0)
    assert torch.isfinite(a).all() and torch.all((a - b).abs() <= 2 ** -23 * a.abs())
    none = lordo.RowGrad(rows[:0], index[vocab:].new_full((vocab,), -1), vocab)
    assert torch.equal(lordo.grad_norm([none, extra[0]]), lordo.grad_norm([extra[0]])) and float(lordo.grad_norm([none])[0]) == 0


@pytest.mark.parametrize("sizes", [[1], [3, 5], [1 << 20], [8191, 8192, 8193], [1 + 31 * k % 977 for k in range(200)], [3000000, 1, 777777]])
@pytest.mark.parametrize("bf16, shift", [(False, 0), (True, 0), (False, 1), (True, 3)])
def test_norm(torch, sizes, bf16, shift):
    """Products and sums in double: what is left is one rounding to fp32, and one of the coefficient."""
    from paper_2602_04396_amd import lordo
    gen = _gen(torch, 11)
    G = [_tensor(torch, gen, 1, n, torch.bfloat16 if bf16 else torch.float32, 1.0, shift) for n in sizes]
    want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in G))
    for most in (0.5 * want, 2 * want, float("inf")):
        out = lordo.grad_norm(G, most)
        assert abs(float(out[0]) - want) <= 1.01 * ref.EPS32 * want
        assert abs(float(out[1]) - min(1.0, most / want)) <= 1.01 * ref.EPS32
    assert torch.equal(lordo.grad_norm(G, 0.5 * want), lordo.grad_norm(lordo.grad_list(G), 0.5 * want))


def test_norm_of_extreme_values(torch):
    from paper_2602_04396_amd import lordo
    for x in (1e30, 1e-30, 3e38, 1e-44):
        g = torch.full((1, 4), x, device="cuda")
        assert abs(float(lordo.grad_norm([g])[0]) / (2 * float(g[0, 0])) - 1) <= 2 * ref.EPS32 or float(g[0, 0]) > 2e38
    out = lordo.grad_norm([torch.zeros(5, device="cuda")], 1.0)
    assert out.tolist() == [0.0, 1.0]
    for bad in (float("inf"), -float("inf"), float("nan")):
        out = lordo.grad_norm([torch.ones(5000, device="cuda"), torch.full((1,), bad, device="cuda")], 1.0)
        assert not math.isfinite(float(out[0])) and math.isnan(float(out[1]))


def test_on_another_stream_and_recorded(torch):
    """A recorded step counts its replays; eager work and synchronisation between them; a second recording shares nothing with the first."""
    from paper_2602_04396_amd import lordo
    shapes, gen = [(64, 257), (1, 33, 0)], _gen(torch, 12)
    for q8 in (False, True):
        hp = lordo.adamw_hparams(weight_decay=0.1, state_dtype=lordo.Q8 if q8 else lordo.F32)
        start = [_tensor(torch, gen, *sh[:2], torch.float32, 0.02) for sh in shapes]
        sets = [[_tensor(torch, gen, *sh[:2], torch.float32, 1.0) for sh in shapes] for _ in range(5)]
        W, V = [w.clone() for w in start], [w.clone() for w in start]
        eager, replayed = lordo.AdamW(shapes, hp, torch), lordo.AdamW(shapes, hp, torch)
        G = [g.clone() for g in sets[0]]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            replayed.local_step(V, G, 1e-2, clip=lordo.grad_norm(G, 1.0))
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            replayed.local_step(V, G, 1e-2, clip=lordo.grad_norm(G, 1.0))
        for k, new in enumerate(sets):
            if k:
                for g, x in zip(G, new):
                    g.copy_(x)
                graph.replay()
            eager.local_step(W, new, 1e-2, clip=lordo.grad_norm(new, 1.0))
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(W, V)) and torch.equal(eager.export_moments(), replayed.export_moments())
        graph.reset()


def test_factors_beyond_fp32_are_refused(torch):
    from paper_2602_04396_amd import lordo
    opt = lordo.AdamW([(4, 8)], lordo.adamw_hparams(weight_decay=1e3), torch)
    W, G = [torch.ones(4, 8, device="cuda")], [torch.ones(4, 8, device="cuda")]
    for lr, scale in ((1e39, 1.0), (1e-3, -1e39), (1e36, 1.0)):      # the last: lr times the decay
        with pytest.raises(lordo.LordoError):
            opt.local_step(W, G, lr, grad_scale=scale)
    assert torch.all(W[0] == 1.0) and opt.step == 0


def test_refusals_of_a_context(torch):
    from paper_2602_04396_amd import lordo
    lib = lordo.load()
    opt = lordo.AdamW([(4, 8)], lordo.adamw_hparams(), torch)
    W, G = [torch.zeros(4, 8, device="cuda")], [torch.zeros(4, 8, device="cuda")]
    for bad in ([torch.zeros(8, 4, device="cuda")], [torch.zeros(4, 8, device="cuda", dtype=torch.bfloat16)], [W[0], W[0]], [torch.zeros(8, 8, device="cuda")[:, :4].t()],
                [torch.zeros(4, 8)]):
        with pytest.raises(ValueError):
            opt.local_step(bad, G, 1e-3)
    for bad in ([torch.zeros(8, 4, device="cuda")], [G[0], G[0]], [torch.zeros(4, 8, device="cuda", dtype=torch.float16)]):
        with pytest.raises((ValueError, lordo.LordoError)):
            opt.local_step(W, bad, 1e-3)
    flat = torch.zeros(40, device="cuda")
    two = lordo.AdamW([(4, 8), (1, 8)], lordo.adamw_hparams(), torch)
    with pytest.raises(ValueError):                          # a tensor twice, or a part of it
        two.local_step([flat[:32].view(4, 8), flat[24:32]], [G[0], G[0][0]], 1e-3)
    both = two.ptrs([flat[:32].view(4, 8), flat[32:]])
    with pytest.raises(ValueError):
        opt.local_step(both, G, 1e-3)
    with pytest.raises(lordo.LordoError):
        opt.step = 2 ** 63 - 1
    with pytest.raises(lordo.LordoError):
        opt.local_step(W, G, float("nan"))
    with pytest.raises(lordo.LordoError):
        opt.local_step(W, G, 1e-3, grad_scale=float("inf"))
    with pytest.raises(ValueError):
        opt.local_step(W, G, 1e-3, clip=torch.ones(1, device="cuda"))
    with pytest.raises(ValueError):
        opt.import_moments(torch.zeros(2, 100, device="cuda"))
    with pytest.raises(lordo.LordoError):
        opt.step = -1
    arr = lordo.grad_list(G).arr
    null = (C.c_void_p * 1)(None)
    odd = (C.c_void_p * 1)(W[0].data_ptr() + 2)
    for w in (null, odd):
        assert lib.lordo_adamw_step(opt.ctx, w, arr, 1e-3, 1.0, None, None) == lordo.EINVAL
    assert not W[0].any() and opt.step == 0
    again = lordo.AdamW([(4, 8)], lordo.adamw_hparams(), torch)          # the same shapes: the list is good for both
    again.local_step(opt.ptrs(W), G, 1e-3)
