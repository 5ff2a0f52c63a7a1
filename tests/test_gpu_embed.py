"""Token embedding: lookup and gradient against their 64-bit forms, and the chain of gradient, norm and AdamW beside a low-rank step."""
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


def _ids(torch, kind, tokens, vocab, seed=3):
    """zipf: few frequent tokens; all: one token; distinct; mixed: padding of every sort among them; none: only padding."""
    rng = np.random.default_rng(seed)
    if kind == "zipf":
        ids = np.minimum((2.7 * ((vocab + 2.7) / 2.7) ** rng.random(tokens) - 2.7).astype(np.int64), vocab - 1)
    elif kind == "all":
        ids = np.full(tokens, vocab - 1)
    elif kind == "distinct":
        ids = rng.permutation(max(vocab, tokens))[:tokens] % vocab
    elif kind == "mixed":
        ids = rng.integers(-3, vocab + 3, tokens)
        ids[::7] = -100
        ids[3::11] = 2 ** 31 - 1
    else:
        ids = np.full(tokens, -1)
    return ids.astype(np.int64)


@pytest.mark.parametrize("tokens, vocab, cols", [(0, 5, 4), (1, 1, 1), (1, 32000, 4096), (7, 11, 3), (300, 50, 129), (64, 100, 1024), (33, 7, 1030), (5, 9, 5000)])
@pytest.mark.parametrize("w_bf16, out_bf16", [(False, False), (False, True), (True, False), (True, True)])
def test_lookup(torch, tokens, vocab, cols, w_bf16, out_bf16):
    """One product in fp32 and one rounding: the same bits."""
    from paper_2602_04396_amd import lordo
    types = [torch.float32, torch.bfloat16]
    table = torch.randn(vocab, cols, generator=torch.Generator().manual_seed(1)).to(types[w_bf16])
    for kind in ("zipf", "mixed", "none"):
        for wide in (True, False):
            ids = torch.tensor(_ids(torch, kind, tokens, vocab)).to(torch.int64 if wide else torch.int32)
            there = (ids >= 0) & (ids < vocab)
            want = torch.zeros(tokens, cols)
            want[there] = table.float()[ids[there].long()] * 0.3
            got = lordo.embed_lookup(table.cuda(), ids.cuda(), scale=0.3, dtype=types[out_bf16])
            assert torch.equal(got.cpu(), want.to(types[out_bf16]))


def test_lookup_of_a_batch_into_given_rows(torch):
    from paper_2602_04396_amd import lordo
    table, ids = torch.randn(20, 33, device="cuda"), torch.randint(0, 20, (3, 5), device="cuda")
    room = torch.full((17, 33), 7.0, device="cuda")
    out = lordo.embed_lookup(table, ids, out=room[1:16].view(3, 5, 33))
    assert torch.equal(out, table[ids]) and torch.equal(room[0], room[16]) and float(room[0, 0]) == 7.0


def _dense(torch, lordo, ids, dy, vocab, scale, pad_id, out_bf16, accumulate, shift):
    dtype = torch.bfloat16 if out_bf16 else torch.float32
    flat = torch.randn(vocab * dy.shape[1] + shift, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)).to(dtype)
    out = flat[shift:].view(vocab, dy.shape[1])
    old = out.double().cpu().numpy()
    lordo.embed_gradient(ids, dy, out, scale=scale, pad_id=pad_id, accumulate=accumulate)
    return out, old


CASES = [(0, 5, 4), (1, 1, 1), (2, 3, 5), (31, 4, 8), (32, 4, 8), (33, 4, 8), (64, 300, 129), (65, 3, 1024), (1000, 37, 1027), (777, 5000, 36), (4097, 60, 64)]


@pytest.mark.parametrize("tokens, vocab, cols", CASES)
@pytest.mark.parametrize("kind", ["zipf", "all", "distinct", "mixed", "none"])
@pytest.mark.parametrize("in_bf16, out_bf16, accumulate, shift", [(False, False, False, 0), (True, False, True, 1), (True, True, False, 3), (False, True, True, 0)])
def test_gradient(torch, tokens, vocab, cols, kind, in_bf16, out_bf16, accumulate, shift):
    from paper_2602_04396_amd import lordo
    ids = _ids(torch, kind, tokens, vocab)
    gen = torch.Generator(device="cuda").manual_seed(2)
    dy = torch.randn(tokens, cols, device="cuda", generator=gen).to(torch.bfloat16 if in_bf16 else torch.float32)
    pad_id = 2 if kind == "zipf" else -1
    dy[torch.tensor((ids < 0) | (ids >= vocab) | (ids == pad_id)).cuda()] = float("nan")      # what takes no part is not looked at
    dev = torch.tensor(ids).cuda().to(torch.int32 if shift else torch.int64)
    out, old = _dense(torch, lordo, dev, dy, vocab, 0.7, pad_id, out_bf16, accumulate, shift)
    total, size, count = ref.embed_gradient(ids, dy.double().cpu().numpy(), vocab, 0.7, pad_id)      # (leaves those tokens out)
    bound = ref.embed_bound(total, size, count, out_bf16, old if accumulate else None)
    want = total + old if accumulate else total
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= bound)
    idle = count == 0
    assert np.array_equal(got[idle], old[idle] if accumulate else np.zeros_like(old[idle]))
    again, _ = _dense(torch, lordo, dev, dy, vocab, 0.7, pad_id, out_bf16, accumulate, shift)
    assert torch.equal(again, out)


@pytest.mark.parametrize("tokens, vocab, cols", CASES)
@pytest.mark.parametrize("kind", ["zipf", "all", "distinct", "mixed", "none"])
def test_gradient_by_rows(torch, tokens, vocab, cols, kind):
    """The rows of the dense gradient, bit for bit; each id's row and each row's id point at each other; rows of no id stay as they were."""
    from paper_2602_04396_amd import lordo
    ids = torch.tensor(_ids(torch, kind, tokens, vocab)).cuda()
    dy = torch.randn(tokens, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    dense = lordo.embed_gradient(ids, dy, torch.empty(vocab, cols, device="cuda"), scale=0.7)
    for dtype in (torch.float32, torch.bfloat16):
        by_rows = lordo.embed_gradient_rows(ids, dy, vocab, scale=0.7, dtype=dtype)
        index = by_rows.index.cpu().numpy()
        slot, owner = index[:vocab], index[vocab:]
        there = np.unique(ids.cpu().numpy())
        there = there[(there >= 0) & (there < vocab)]
        assert np.array_equal(np.flatnonzero(slot >= 0), there) and np.array_equal(np.sort(owner[owner >= 0]), there)
        assert np.array_equal(owner[slot[there]], there)
        assert torch.equal(by_rows.rows[torch.tensor(slot[there]).cuda().long()], dense[torch.tensor(there).cuda().long()].to(dtype))
        assert by_rows.shape == (vocab, cols)
        again = lordo.RowGrad(torch.full_like(by_rows.rows, 7.0), torch.zeros_like(by_rows.index), vocab)      # rows of no id stay as they were
        assert lordo.embed_gradient_rows(ids, dy, vocab, scale=0.7, out=again) is again and torch.equal(again.index, by_rows.index)
        held = by_rows.index[vocab:] >= 0
        assert torch.equal(again.rows[held], by_rows.rows[held]) and torch.all(again.rows[~held] == 7.0)


@pytest.mark.parametrize("tokens, vocab, cols", [(8192, 300, 20), (8193, 300, 20), (20000, 70000, 20), (40000, 1000, 300), (70001, 32000, 20), (5000, (1 << 21) + 5, 2),
                                                 (9000, 1 << 22, 2), (600001, 5000, 1), (12000, 1, 5), (9001, 3000, 521)])
@pytest.mark.parametrize("kind", ["zipf", "all", "mixed"])
def test_gradient_of_many_tokens(torch, tokens, vocab, cols, kind):
    """Sums that cross many pieces, ids of up to 22 bits."""
    from paper_2602_04396_amd import lordo
    ids = _ids(torch, kind, tokens, vocab)
    dy = torch.randn(tokens, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    dev = torch.tensor(ids).cuda()
    out = lordo.embed_gradient(dev, dy, torch.full((vocab, cols), 9.0, device="cuda"))
    total, size, count = ref.embed_gradient(ids, dy.double().cpu().numpy(), vocab, 1.0)
    assert np.all(np.abs(out.double().cpu().numpy() - total) <= ref.embed_bound(total, size, count, False))
    assert torch.equal(lordo.embed_gradient(dev, dy, torch.empty_like(out)), out)
    low = torch.full((vocab * cols + 1,), 9.0, dtype=torch.bfloat16, device="cuda")
    assert torch.equal(lordo.embed_gradient(dev, dy, low[1:].view(vocab, cols)), out.bfloat16()) and float(low[0]) == 9.0
    by_rows = lordo.embed_gradient_rows(dev, dy, vocab)
    slot = by_rows.index[:vocab].long()
    assert torch.equal(by_rows.rows[slot[slot >= 0]], out[slot >= 0])


def test_outputs_just_above_whole_shares_are_filled_to_their_end(torch):
    """More than 8192 tokens: 64 KB pieces of the fill are spread over two launches a digit.  262146 bytes are four such pieces and one bf16 element
    (ids of 16 bits, two digits), 1572868 bytes are 24 and one int32 (ids of 19 bits, three digits): the last element is written too."""
    from paper_2602_04396_amd import lordo
    tokens, vocab, cols = 8193, 43691, 3
    assert vocab * cols * 2 == 4 * 65536 + 2
    ids = torch.arange(tokens, device="cuda")
    dy = torch.ones(tokens, cols, device="cuda")
    out = lordo.embed_gradient(ids, dy, torch.full((vocab, cols), 9.0, device="cuda", dtype=torch.bfloat16))
    assert torch.all(out[:tokens] == 1.0) and torch.all(out[tokens:] == 0.0)
    tokens, vocab = 93217, 300000
    assert 4 * (vocab + tokens) == 24 * 65536 + 4
    ids = torch.arange(tokens, device="cuda") // 2
    dy = torch.ones(tokens, 1, device="cuda")
    ids[-1] = ids[-2]                                    # (the last slot holds no row)
    got = lordo.RowGrad(torch.full((tokens, 1), 7.0, device="cuda"), torch.full((vocab + tokens,), 5, device="cuda", dtype=torch.int32), vocab)
    lordo.embed_gradient_rows(ids, dy, vocab, out=got)
    owner = got.index[vocab:]
    assert int((owner >= 0).sum()) == int(ids[-1]) + 1 and int(owner[-1]) == -1
    assert int((got.index[:vocab] >= 0).sum()) == int(ids[-1]) + 1


def test_refusals(torch):
    from paper_2602_04396_amd import lordo
    table, ids, dy = torch.zeros(8, 4, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(3, 4, device="cuda")
    for call in (lambda: lordo.embed_lookup(table.t(), ids), lambda: lordo.embed_lookup(table, ids.float()), lambda: lordo.embed_lookup(table.half(), ids),
                 lambda: lordo.embed_lookup(table, ids, out=torch.zeros(3, 5, device="cuda")), lambda: lordo.embed_lookup(table, ids.cpu()),
                 lambda: lordo.embed_gradient(ids, dy[:2], table), lambda: lordo.embed_gradient(ids, dy, table.t()),
                 lambda: lordo.embed_gradient(ids, dy, torch.zeros(8, 5, device="cuda")), lambda: lordo.embed_gradient(ids, dy.t().contiguous().t(), table),
                 lambda: lordo.embed_gradient_rows(ids, dy.cpu(), 8), lambda: lordo.embed_gradient_rows(ids, dy, 8, out=lordo.embed_gradient_rows(ids, dy, 9)),
                 lambda: lordo.embed_gradient_rows(ids, dy, 8, out=lordo.embed_gradient_rows(ids[:2], dy[:2], 8))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(lordo.LordoError):
        lordo.embed_gradient_rows(ids, dy, 0)


def test_training_steps_together(torch):
    """Lookup, gradient by rows, one norm over it, the norm weights and a projected matrix, AdamW and the low-rank step, four times: issued, and the full-rank
    part recorded, against 64 bits from the same start each time."""
    from paper_2602_04396_amd import lordo
    vocab, cols, batch = 50, 40, (4, 33)
    gen = torch.Generator(device="cuda").manual_seed(6)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    shapes = [(vocab, cols), (1, cols, 0)]
    hp = lordo.adamw_hparams(weight_decay=0.1)
    W = [randn(*sh[:2]) * 0.02 for sh in shapes]
    M = [randn(64, 96) * 0.02]
    low = lordo.Lordo([(64, 96, 8)], lordo.hparams(grad_dtype=lordo.F32, seed=1), M, torch)
    low.init_projection()
    full, twin = lordo.AdamW(shapes, hp, torch), lordo.AdamW(shapes, hp, torch)
    V = [w.clone() for w in W]
    ids, dy, gain, GM = torch.zeros(batch, dtype=torch.int64, device="cuda"), torch.zeros(*batch, cols, device="cuda"), torch.zeros(1, cols, device="cuda"), torch.zeros(64, 96, device="cuda")

    def step(opt, weights):
        rows = lordo.embed_gradient_rows(ids, dy, vocab, scale=6.0, pad_id=0)
        G = [rows, gain]
        clip = lordo.grad_norm(G + [GM], 1.0)
        opt.local_step(weights, G, 1e-2, clip=clip)
        return clip

    step(lordo.AdamW(shapes, hp, torch), [w.clone() for w in W])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step(twin, V)
    for k in range(4):
        ids.copy_(torch.randint(-1, vocab, batch, device="cuda", generator=gen))
        x = lordo.embed_lookup(W[0], ids, scale=6.0)
        assert torch.equal(x[ids < 0], torch.zeros_like(x[ids < 0]))
        dy.copy_(x + randn(*batch, cols) * 0.1)
        gain.copy_(randn(1, cols))
        GM.copy_(randn(64, 96))
        w0, m0 = [w.double().cpu().numpy().reshape(-1) for w in W], full.export_moments().double().cpu().numpy()
        clip = step(full, W)
        low.local_step(M, [GM], 1e-2, grad_scale=float(clip[1]))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(clip, recorded) and all(torch.equal(a, b) for a, b in zip(W, V))
        assert torch.equal(full.sync_payload(), twin.sync_payload())
        dw, size, count = ref.embed_gradient(ids.cpu().numpy(), dy.double().cpu().numpy(), vocab, 6.0, 0)
        g = [dw.reshape(-1), gain.double().cpu().numpy().reshape(-1)]
        norm = np.sqrt(sum((a ** 2).sum() for a in g) + float((GM.double() ** 2).sum()))
        # the rows' own error, at most 135 roundings of their terms, is part of the norm
        assert abs(float(clip[0]) - norm) <= (2 * ref.EPS32 + 135 * ref.EPS32 * np.linalg.norm(size) / norm) * norm
        at = 0
        for i, n in enumerate((vocab * cols, cols)):
            gi = float(clip[1]) * g[i]
            w, u, v, terms = ref.adamw(w0[i], m0[0, at:at + n], m0[1, at:at + n], gi, k + 1, 1e-2, hp.beta1, hp.beta2, hp.eps, 0.1 if i == 0 else 0.0)
            bw, _, _ = ref.adamw_bounds(w, w0[i], np.abs(u), v, terms, 1e-2, 0.1 if i == 0 else 0.0, False)
            got = W[i].double().cpu().numpy().reshape(-1)
            if i == 0:                                             # the gradient's error: a change of g moves the update by at most its share of the terms, twice
                eg = float(clip[1]) * ref.embed_bound(dw, size, count, False).reshape(-1)
                c1, c2 = 1 - hp.beta1 ** (k + 1), 1 - hp.beta2 ** (k + 1)
                den = np.sqrt(v / c2) + hp.eps
                bw = bw + 1e-2 * ((1 - hp.beta1) * eg / c1 / den + np.abs(u) / c1 / den ** 2 * (1 - hp.beta2) / c2 * np.abs(gi) * eg / np.maximum(den - hp.eps, 1e-30) * 2)
            assert np.all(np.abs(got - w) <= bw)
            at += (n + 127) // 128 * 128
    low.poll_status()
    full.poll_status()
    graph.reset()
