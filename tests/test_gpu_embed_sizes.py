"""Token embedding at the sizes of real batches: lookups of thousands of workgroups, tiles of 16 and 32 tokens in the gradient, arrays beyond 2^31 elements.
Gradients of whole numbers below 2^24 are summed exactly in fp32, so every form has to give the sum itself."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available()
    from paper_2602_04396_amd import lordo
    lordo.load()
    yield t
    t.cuda.empty_cache()


def _ids(torch, kind, tokens, vocab, gen):
    if kind == "all":
        return torch.full((tokens,), vocab - 1, device="cuda")
    if kind == "zipf":
        x = torch.rand(tokens, generator=gen, device="cuda", dtype=torch.float64)
        return (2.7 * ((vocab + 2.7) / 2.7) ** x - 2.7).long().clamp_(0, vocab - 1)
    if kind == "pairs":                                  # every id for two tiles of 32 and one token more
        return (torch.arange(tokens, device="cuda") // 65 % vocab)[torch.randperm(tokens, generator=gen, device="cuda")]
    ids = torch.randint(-3, vocab + 3, (tokens,), generator=gen, device="cuda")
    ids[::7] = -100
    return ids


# 2 to 32771 workgroups of 1 to 256 rows, ragged ones among them
@pytest.mark.parametrize("tokens, cols", [(4095, 2049), (4101, 2049), (2050, 8200), (8191, 1031), (16390, 1031), (262147, 5), (262147, 8), (524300, 20), (32771, 512)])
@pytest.mark.parametrize("w_bf16, out_bf16", [(False, False), (False, True), (True, False), (True, True)])
def test_lookup_of_large_batches(torch, tokens, cols, w_bf16, out_bf16):
    """One product in fp32 and one rounding: the same bits."""
    from paper_2602_04396_amd import lordo
    vocab, types, gen = 997, [torch.float32, torch.bfloat16], torch.Generator(device="cuda").manual_seed(1)
    table = torch.randn(vocab, cols, generator=gen, device="cuda").to(types[w_bf16])
    for kind, wide in (("mixed", True), ("zipf", False)):
        ids = _ids(torch, kind, tokens, vocab, gen).to(torch.int64 if wide else torch.int32)
        there = (ids >= 0) & (ids < vocab)
        want = table.float()[ids.long().clamp(0, vocab - 1)] * 0.3
        want[~there] = 0.0
        room = torch.full(((tokens + 2) * cols,), 7.0, dtype=types[out_bf16], device="cuda")
        out = room[cols:-cols].view(tokens, cols)
        lordo.embed_lookup(table, ids, scale=0.3, out=out)
        assert torch.equal(out, want.to(types[out_bf16]))
        assert torch.all(room[:cols] == 7.0) and torch.all(room[-cols:] == 7.0)


def _sum(torch, ids, dy, vocab):
    there = (ids >= 0) & (ids < vocab)
    out = torch.zeros(vocab, dy.shape[1], device="cuda", dtype=torch.float64)
    return out.index_add_(0, ids[there].long(), dy[there].double())


# 9000 x 1030: tiles of 8 (bf16) and 16 (fp32); 65539: 16; 131075: 32; 20000 x 2100: 32
@pytest.mark.parametrize("tokens, vocab, cols", [(9000, 400, 1030), (65539, 700, 20), (131075, 700, 20), (131075, 40000, 33), (140001, 5, 260), (20000, 300, 2100), (33000, 32000, 1024)])
@pytest.mark.parametrize("kind", ["zipf", "all", "pairs", "mixed"])
def test_gradient_of_large_batches(torch, tokens, vocab, cols, kind):
    from paper_2602_04396_amd import lordo
    gen = torch.Generator(device="cuda").manual_seed(2)
    ids = _ids(torch, kind, tokens, vocab, gen)
    whole = torch.randint(-8, 9, (tokens, cols), generator=gen, device="cuda")
    base = torch.randint(-100, 101, (vocab, cols), generator=gen, device="cuda").double()
    total = _sum(torch, ids, whole, vocab)
    none = torch.bincount(ids[(ids >= 0) & (ids < vocab)], minlength=vocab) == 0
    for dtype in (torch.float32, torch.bfloat16):
        dy = whole.to(dtype)
        dy[(ids < 0) | (ids >= vocab)] = float("nan")              # what takes no part is not looked at
        for out_type in (torch.float32, torch.bfloat16):
            # (scale 1/2: exact; bf16 outputs are rounded once)
            out = lordo.embed_gradient(ids, dy, torch.full((vocab, cols), 9.0, device="cuda", dtype=out_type), scale=0.5)
            assert torch.equal(out, (0.5 * total).float().to(out_type))
            out = lordo.embed_gradient(ids.int(), dy, base.to(out_type), scale=0.5, accumulate=True)
            assert torch.equal(out, (base + 0.5 * total).float().to(out_type))
        r = lordo.embed_gradient_rows(ids, dy, vocab, scale=0.5)
        slot, owner = r.index[:vocab].long(), r.index[vocab:].long()
        assert torch.equal(slot < 0, none) and int((owner >= 0).sum()) == int((~none).sum())
        there = torch.nonzero(~none).view(-1)
        assert torch.equal(owner[slot[there]], there) and torch.equal(r.rows[slot[there]], (0.5 * total[there]).float())


FAR = (524309, 4099)                                     # 2149142591 elements


def test_tables_and_outputs_beyond_32_bits(torch):
    from paper_2602_04396_amd import lordo
    vocab, cols = FAR
    table = torch.zeros(FAR, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.tensor([0, vocab - 1, vocab, vocab - 2, -1, 1, 523916, 523917, vocab - 1], device="cuda")
    rows = torch.unique(ids[(ids >= 0) & (ids < vocab)])
    table[rows] = torch.randn(len(rows), cols, generator=gen, device="cuda").bfloat16()
    out = lordo.embed_lookup(table, ids)
    for j, k in enumerate(ids.tolist()):
        assert torch.equal(out[j], table[k]) if 0 <= k < vocab else not out[j].any()
    # the gradient written over the table: zeros up to its end, added and by rows; then as many tokens, and a batch of as many rows
    dy = torch.randint(-8, 9, (len(ids), cols), generator=gen, device="cuda").float()
    table.fill_(3.0)
    lordo.embed_gradient(ids, dy, table)
    for k in rows.tolist():
        assert torch.equal(table[k], dy[ids == k].sum(0).bfloat16())
    table[rows] = 0
    assert not torch.any(table)
    table[rows] = 1.0
    lordo.embed_gradient(ids, dy, table, accumulate=True)
    for k in rows.tolist():
        assert torch.equal(table[k], (1 + dy[ids == k].sum(0)).bfloat16())
    table[rows] = 0
    assert not torch.any(table)


def test_batches_beyond_32_bits(torch):
    """Rows of dY, and rows looked up, behind 2^31 elements: whole numbers, exact sums."""
    from paper_2602_04396_amd import lordo
    tokens, cols = FAR
    vocab, gen = 1000, torch.Generator(device="cuda").manual_seed(4)
    small = torch.randint(-8, 9, (vocab, cols), generator=gen, device="cuda").bfloat16()
    ids = _ids(torch, "mixed", tokens, vocab, gen)
    dy = lordo.embed_lookup(small, ids)
    step = 1 << 16
    for at in range(0, tokens, step):
        part = ids[at:at + step]
        want = small[part.clamp(0, vocab - 1)]
        want[(part < 0) | (part >= vocab)] = 0
        assert torch.equal(dy[at:at + step], want)
    count = torch.bincount(ids[(ids >= 0) & (ids < vocab)], minlength=vocab).double()
    out = lordo.embed_gradient(ids, dy, torch.full((vocab, cols), 9.0, device="cuda"))
    assert torch.equal(out, (count[:, None] * small.double()).float())
    r = lordo.embed_gradient_rows(ids, dy, vocab)
    slot = r.index[:vocab].long()
    assert int(slot.min()) >= 0 and int(slot.max()) * cols > 1 << 30
    assert torch.equal(r.rows[slot], out)


@pytest.mark.parametrize("wide", [True, False])
def test_lookup_of_more_tokens_than_a_launch_takes(torch, wide):
    """Rows of more than 1024 columns are a workgroup each, 256 threads: 2^23 of them are one launch."""
    from paper_2602_04396_amd import lordo
    tokens, cols, vocab = (1 << 23) + 5, 1032, 50
    gen = torch.Generator(device="cuda").manual_seed(5)
    table = torch.randn(vocab, cols, generator=gen, device="cuda").bfloat16()
    ids = torch.randint(-1, vocab, (tokens,), generator=gen, device="cuda", dtype=torch.int64 if wide else torch.int32)
    out = torch.full((tokens, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    lordo.embed_lookup(table, ids, out=out)
    padded = torch.cat([table, torch.zeros(1, cols, dtype=torch.bfloat16, device="cuda")])      # (the row -1)
    step = 1 << 19
    for at in list(range(0, tokens, step)):
        assert torch.equal(out[at:at + step], padded[ids[at:at + step].long()])
