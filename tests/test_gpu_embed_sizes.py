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
    """Sums by differences of the running sum over the sorted ids, exact for whole numbers (adding by atomics to one id takes minutes)."""
    there = (ids >= 0) & (ids < vocab)
    keys, order = torch.sort(ids[there].long())
    run = torch.zeros(len(keys) + 1, dy.shape[1], dtype=torch.float64, device="cuda")
    torch.cumsum(dy[there].double()[order], 0, out=run[1:])
    ends = torch.searchsorted(keys, torch.arange(vocab + 1, device="cuda"))
    return run[ends[1:]] - run[ends[:-1]]


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
    none = torch.ones(vocab + 1, dtype=torch.bool, device="cuda")
    none[torch.where((ids >= 0) & (ids < vocab), ids, vocab)] = False
    none = none[:vocab]
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


@pytest.mark.parametrize("rows", [False, True])
@pytest.mark.parametrize("tokens, vocab, cols", [(300, 50, 40), (9001, 700, 130), (70001, 32000, 64)])
def test_recorded_gradients_follow_their_tokens(torch, tokens, vocab, cols, rows):
    """Recorded on a side stream, two graphs with their own workspaces, replayed in turn over new tokens: ranked in one launch, by digits, long runs and none."""
    from paper_2602_04396_amd import lordo
    gen = torch.Generator(device="cuda").manual_seed(6)
    state = []
    for k in range(2):
        s = dict(ids=torch.zeros(tokens, dtype=torch.int64, device="cuda"), dy=torch.zeros(tokens, cols, device="cuda"), out=torch.zeros(vocab, cols, device="cuda"))
        s["rows"] = lordo.RowGrad(torch.zeros(tokens, cols, device="cuda"), torch.zeros(vocab + tokens, dtype=torch.int32, device="cuda"), vocab)
        state.append(s)

    def call(s):
        if rows:
            lordo.embed_gradient_rows(s["ids"], s["dy"], vocab, out=s["rows"])
        else:
            lordo.embed_gradient(s["ids"], s["dy"], s["out"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for s in state:
            call(s)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                call(s)
            graphs.append(g)
    torch.cuda.current_stream().wait_stream(side)
    for kind in ("zipf", "all", "mixed", "pairs", "zipf"):
        want = []
        for s in state:
            s["ids"].copy_(_ids(torch, kind, tokens, vocab, gen))
            s["dy"].copy_(torch.randint(-8, 9, (tokens, cols), generator=gen, device="cuda"))
            want.append(_sum(torch, s["ids"], s["dy"], vocab).float())
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, w in zip(state, want):
            if rows:
                slot = s["rows"].index[:vocab].long()
                got = torch.where((slot >= 0)[:, None], s["rows"].rows[slot.clamp(min=0)], 0.0)
                there = torch.zeros(vocab + 1, dtype=torch.bool, device="cuda")
                there[torch.where((s["ids"] >= 0) & (s["ids"] < vocab), s["ids"], vocab)] = True
                there = there[:vocab]
                assert torch.equal(slot >= 0, there) and torch.equal(got, w)
            else:
                assert torch.equal(s["out"], w)
    for g in graphs:
        g.reset()


@pytest.mark.parametrize("kind", ["zipf", "all", "mixed"])
def test_the_most_tokens_and_the_largest_vocabulary(torch, kind):
    from paper_2602_04396_amd import lordo
    tokens, vocab, gen = lordo.MAX_TOKENS, lordo.MAX_VOCAB, torch.Generator(device="cuda").manual_seed(7)
    ids = _ids(torch, kind, tokens, vocab, gen)
    dy = torch.randint(0, 2, (tokens, 1), generator=gen, device="cuda").bfloat16()
    dy -= 0.5                                            # (halves: sums below 2^24 of them are exact)
    there = (ids >= 0) & (ids < vocab)
    want, held = _sum(torch, ids, dy, vocab)[:, 0].float(), torch.zeros(vocab, dtype=torch.bool, device="cuda")
    held[ids[there]] = True
    out = lordo.embed_gradient(ids, dy, torch.full((vocab, 1), 9.0, device="cuda"))
    assert torch.equal(out[:, 0], want)
    r = lordo.embed_gradient_rows(ids.int(), dy, vocab)
    slot = r.index[:vocab].long()
    assert torch.equal(slot >= 0, held)
    assert torch.equal(torch.where(slot >= 0, r.rows[slot.clamp(min=0), 0], 0.0), want)
    norm = float((want.double() ** 2).sum()) ** 0.5
    assert abs(float(lordo.grad_norm([r])[0]) - norm) <= 1.01 * 2.0 ** -24 * norm
    for bad in (ids.repeat(2)[:tokens + 1], ):
        with pytest.raises(lordo.LordoError):
            lordo.embed_gradient_rows(bad, torch.zeros(tokens + 1, 1, device="cuda"), vocab)
