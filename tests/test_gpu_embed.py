"""A table of embeddings (pp_embed_fwd, pp_embed_bwd) on the GPU.

Error bounds.  A feature is one fp32 product, rounded once to the output's type:
what torch computes, bit by bit.  A gradient is a sum of n fp32 values in some
order, n - 1 roundings of at most 2^-24 of the sum of magnitudes, then a product
and an addition; the bound is (n + 2) 2^-24 (|scale| sum |dy| + |add|) and half a
step of the output's type."""
import pytest
import torch

pp = pytest.importorskip("paper_2004_11250_amd")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
IGNORE = -100


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(seed, *shape, dtype="f32"):
    return torch.randn(shape, generator=rng(seed), device="cuda").to(DT[dtype])


def make_ids(seed, t, v, how="uniform", ignored=0.0):
    g = rng(seed)
    if how == "one":
        ids = torch.full((t,), v // 2, device="cuda")
    elif how == "heavy":        # half of all tokens are one row
        ids = torch.where(torch.rand(t, generator=g, device="cuda") < 0.5, v - 1, torch.randint(0, v, (t,), generator=g, device="cuda"))
    elif how == "sorted":
        ids = torch.randint(0, v, (t,), generator=g, device="cuda").sort()[0]
    else:
        ids = torch.randint(0, v, (t,), generator=g, device="cuda")
    drop = torch.rand(t, generator=g, device="cuda") < ignored
    return torch.where(drop, torch.full_like(ids, IGNORE), ids)


def ref_fwd(ids, w, scale, dtype, ignore=IGNORE):
    y = w[ids.clamp(0, w.shape[0] - 1)].float() * scale
    y[(ids < 0) | (ids >= w.shape[0])] = float("nan")
    y[ids == ignore] = 0.0
    return y.to(dtype)


def check_bwd(got, ids, dy, v, scale=1.0, add=None, ignore=IGNORE):
    live = (ids != ignore) & (ids >= 0) & (ids < v)
    at, x = ids[live], dy.reshape(-1, dy.shape[-1])[live.reshape(-1)].double()
    # (sorted, as differences of running sums: many additions to one row are slow in 64 bits)
    at, order = at.sort(stable=True)
    ends = torch.searchsorted(at, torch.arange(v + 1, device="cuda"))
    n = (ends[1:] - ends[:-1]).double()

    def rows(x):
        x = torch.cat([torch.zeros_like(x[:1]), x]).cumsum(0) if len(x) else torch.zeros(1, x.shape[1], dtype=x.dtype, device="cuda")
        return torch.where(n[:, None] > 0, x[ends[1:]] - x[ends[:-1]], 0.0)

    want, size = rows(x[order]) * scale, rows(x[order].abs()) * abs(scale)
    slack = x.abs().sum(0) * abs(scale) * 2.0 ** -44      # (of the running sums: at most 2^-53 of all, 2^9 times over)
    if add is not None:
        want, size = want + add.double(), size + add.double().abs()
    lim = (n[:, None] + 2) * 2.0 ** -24 * size + slack * (n[:, None] > 0)
    if got.dtype == torch.bfloat16:
        lim = lim + 2.0 ** -8 * (want.abs() + lim)
    bad = ~((got.double() - want).abs() <= lim)
    assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:3].tolist())


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("w,y", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("d", [1, 2, 7, 8, 9, 63, 64, 203, 256, 1030, 2048, 2056, 5000])
def test_lookup(w, y, d):
    for t, v in ((1, 1), (5, 3), (300, 77)):
        table, ids = normal(d, v, d, dtype=w), make_ids(d + t, t, v, ignored=0.2)
        got = pp.embed_fwd(ids, table, scale=1.7, dtype=DT[y])
        want = ref_fwd(ids, table, 1.7, DT[y])
        assert got.shape == want.shape and got.dtype == want.dtype and torch.equal(got, want)


def test_lookup_ids():
    table = normal(1, 10, 33)
    table[3] = float("inf")
    ids = torch.tensor([[0, 9, 10, -1], [-100, 3, 1 << 40, -(1 << 62)]], device="cuda")
    got = pp.embed_fwd(ids, table, scale=0.0)
    want = ref_fwd(ids, table, 0.0, torch.float32)
    assert got.shape == (2, 4, 33) and torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(5.0), want.nan_to_num(5.0))
    # an id of the table may be the ignored one: zeros, even of a row that is not finite
    got = pp.embed_fwd(ids, table, ignore_index=3)
    assert torch.equal(got.nan_to_num(5.0), ref_fwd(ids, table, 1.0, torch.float32, ignore=3).nan_to_num(5.0))
    assert bool((got[1, 1] == 0).all()) and bool(torch.isnan(got[1, 0]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,left,pitch", [(64, 0, 64), (64, 1, 67), (37, 3, 41), (40, 8, 56)])
def test_rows_apart(dtype, d, left, pitch):
    v, t = 50, 400
    wide = normal(3, v, pitch, dtype=dtype)
    table = wide[:, left:left + d]
    ids = make_ids(4, t, v, ignored=0.1)
    out = torch.full((t, pitch), 7.0, device="cuda", dtype=DT[dtype])
    got = pp.embed_fwd(ids, table, out=out[:, left:left + d])
    assert got.data_ptr() == out[:, left:].data_ptr() and torch.equal(got, ref_fwd(ids, table, 1.0, DT[dtype]))
    rest = torch.ones(pitch, dtype=torch.bool, device="cuda")
    rest[left:left + d] = False
    assert bool((out[:, rest] == 7.0).all())
    # the gradient: dy, add and out by rows inside wider ones
    dy = normal(5, t, pitch, dtype=dtype)[:, left:left + d]
    base = normal(6, v, pitch, dtype=dtype)
    keep = base.clone()
    dw = torch.full((v, pitch), 7.0, device="cuda", dtype=DT[dtype])
    pp.embed_bwd(ids, dy, v, scale=0.5, add=base[:, left:left + d], out=dw[:, left:left + d])
    check_bwd(dw[:, left:left + d], ids, dy, v, 0.5, add=keep[:, left:left + d])
    assert bool((dw[:, rest] == 7.0).all()) and torch.equal(base, keep)
    pp.embed_bwd(ids, dy, v, scale=0.5, add=base[:, left:left + d], out=base[:, left:left + d])
    assert torch.equal(base[:, left:left + d], dw[:, left:left + d]) and torch.equal(base[:, rest], keep[:, rest])


def test_same_results_however_called():
    ids, table, dy = make_ids(7, 300, 40, ignored=0.1).view(3, 100), normal(8, 40, 24), normal(9, 3, 100, 24)
    y, dw = pp.embed_fwd(ids, table, scale=0.5), pp.embed_bwd(ids, dy, 40, scale=0.5)
    assert torch.equal(y, ref_fwd(ids, table, 0.5, torch.float32)) and not y.requires_grad
    wide, wide_dy = torch.zeros(40, 30, device="cuda"), torch.zeros(3, 100, 30, device="cuda")
    wide[:, 3:27], wide_dy[..., 3:27] = table, dy
    half = torch.tensor(0.5, dtype=torch.float64).numpy()[()]
    for kw in (dict(scale=half), dict(scale=0.5, ignore_index=make_ids(1, 1, 9, "one").new_tensor(IGNORE)), dict(scale=torch.tensor(0.5))):
        assert torch.equal(pp.embed_fwd(ids, table, **kw), y) and torch.equal(pp.embed_bwd(ids, dy, 40, **kw), dw)
    assert torch.equal(pp.embed_fwd(ids, wide[:, 3:27], scale=0.5), y)
    assert torch.equal(pp.embed_bwd(ids, wide_dy[..., 3:27], 40, scale=0.5), dw)
    assert torch.equal(pp.embed_fwd(ids, table.requires_grad_(), scale=0.5), y)


def test_more_than_the_card_holds():
    ids = torch.zeros(1 << 20, dtype=torch.int64, device="cuda")
    with pytest.raises(torch.OutOfMemoryError):
        pp.embed_fwd(ids, torch.zeros(1, 1 << 20, device="cuda"))      # 4 TB
    assert torch.equal(pp.embed_fwd(ids[:2], torch.ones(1, 3, device="cuda")), torch.ones(2, 3, device="cuda"))


@pytest.mark.parametrize("w,y", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("d", [1, 8, 9, 63, 203, 256, 1030, 2056])
@pytest.mark.parametrize("how", ["uniform", "heavy"])
def test_gradient(w, y, d, how):
    for t, v in ((1, 1), (31, 4), (33, 1), (700, 90), (2500, 1000)):
        ids, dy = make_ids(d + t, t, v, how, ignored=0.2 if t > 1 else 0.0), normal(d + t, t, d, dtype=y)
        check_bwd(pp.embed_bwd(ids, dy, v, scale=0.3, dtype=DT[w]), ids, dy, v, 0.3)


@pytest.mark.parametrize("t", [0, 1, 32, 33, 64, 65, 1023, 1024, 1025, 4096, 32768, 32769, 70001])
@pytest.mark.parametrize("v,how", [(1, "one"), (2, "heavy"), (313, "heavy"), (313, "sorted"), (5000, "uniform"), (300000, "uniform"),
                                   (5000, "one")])
def test_token_counts(t, v, how):
    ids, dy = make_ids(t + v, t, v, how, ignored=0.1), normal(t + v, t, 24)
    add = normal(9, v, 24)
    check_bwd(pp.embed_bwd(ids, dy, v, scale=2.0), ids, dy, v, 2.0)
    got = pp.embed_bwd(ids, dy, v, add=add)
    check_bwd(got, ids, dy, v, add=add)
    # the same again, and in place: bit by bit
    assert same(got, pp.embed_bwd(ids, dy, v, add=add))
    assert same(got, pp.embed_bwd(ids, dy, v, add=add, out=add))


@pytest.mark.parametrize("v", [1023, 1024, 1025, 2047, 65536, 600000, 1 << 20, (1 << 20) + 1, 3000001])
@pytest.mark.parametrize("t", [2000, 16384, 16385, 65535, 65536, 200003])
def test_sorts(v, t):
    # one digit, two and three, the largest of each, and what lies beside them
    ids, dy = make_ids(t, t, v, "heavy" if v % 2 else "uniform", ignored=0.1), normal(t, t, 5)
    got = pp.embed_bwd(ids, dy, v, ignore_index=v // 2)
    check_bwd(got, ids, dy, v, ignore=v // 2)
    assert same(got, pp.embed_bwd(ids, dy, v, ignore_index=v // 2))
    add = normal(3, v, 5)
    got = pp.embed_bwd(ids, dy, v, ignore_index=v // 2, add=add)
    assert same(got, pp.embed_bwd(ids, dy, v, ignore_index=v // 2, add=add, out=add))


@pytest.mark.parametrize("t,v", [(1024, 300), (16384, 1024), (16385, 1024), (65535, 5000), (65536, 5000), (100003, 313), (200003, 313),
                                 (200003, 1025), (200003, 65537), (200003, (1 << 20) + 1), (70001, 3000001), (200003, 1)])
@pytest.mark.parametrize("how", ["one", "heavy", "two"])
@pytest.mark.parametrize("d", [5, 64, 200])
def test_long_rows_exactly(t, v, how, d):
    """Of whole numbers of at most 8, whose sums of up to 2^21 are exact in any order, in every sort: a row that all, or half of
    all tokens share, and two such rows beside each other."""
    if how == "two":
        ids = make_ids(t + v, t, v, "uniform")
        half = torch.rand(t, generator=rng(t), device="cuda")
        ids = torch.where(half < 0.4, v // 2, torch.where(half < 0.8, min(v // 2 + 1, v - 1), ids))
    else:
        ids = make_ids(t + v, t, v, how)
    ids = torch.where(torch.rand(t, generator=rng(v), device="cuda") < 0.1, torch.full_like(ids, IGNORE), ids)
    dy = torch.randint(-8, 9, (t, d), generator=rng(d), device="cuda").float()
    live = ids != IGNORE
    want = torch.zeros(v, d, device="cuda").index_add_(0, ids[live], dy[live])
    assert torch.equal(pp.embed_bwd(ids, dy, v), want)
    assert torch.equal(pp.embed_bwd(ids, dy.bfloat16(), v, dtype=torch.float32), want)
    base = torch.randint(-8, 9, (v, d), generator=rng(1), device="cuda").float()
    want += base
    assert torch.equal(pp.embed_bwd(ids, dy, v, add=base, out=base), want)


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("d", [1, 8, 16, 31, 32, 64, 128, 203, 256, 512, 1024])
@pytest.mark.parametrize("t", [900, 6000, 40000])
def test_runs_of_every_length(y, d, t):
    """Of whole numbers below 2^24 in all, whose sums are exact in any order; a row with infinities keeps them to itself."""
    g = torch.Generator().manual_seed(t + d)
    kinds = torch.tensor([1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 64, 65, 127, 130, 257, 511, 520, 1100])
    lens = kinds[torch.randint(0, len(kinds), (600,), generator=g)]
    lens = lens[:int((lens.cumsum(0) <= t).sum())]
    v = len(lens) + 3                   # (with rows that no token reaches)
    rows = torch.randperm(v, generator=g)[:len(lens)]
    ids = rows.repeat_interleave(lens)[torch.randperm(int(lens.sum()), generator=g)].cuda()
    dy = torch.randint(-8, 9, (len(ids), d), generator=g).cuda().to(DT[y])
    want = torch.zeros(v, d, dtype=torch.float64, device="cuda").index_add_(0, ids, dy.double())
    assert torch.equal(pp.embed_bwd(ids, dy, v, dtype=torch.float32).double(), want)
    wild = int(rows[0])
    dy[ids == wild] = float("inf")
    got = pp.embed_bwd(ids, dy, v, dtype=torch.float32).double()
    want[wild] = float("inf")
    assert torch.equal(got, want)


def test_ids_that_reach_no_row():
    ids = torch.tensor([-1, 10, 1 << 33, -100, 4, 4, 9, -(1 << 63), (1 << 63) - 1], device="cuda")
    dy = normal(2, 9, 40)
    dy[[0, 1, 2, 3, 7, 8]] = float("nan")
    check_bwd(pp.embed_bwd(ids, dy, 10), ids, torch.nan_to_num(dy), 10)
    got = pp.embed_bwd(ids, dy, 10, ignore_index=4)
    assert bool((got[:9] == 0).all()) and torch.equal(got[9], dy[6])
    none = torch.full((5000,), -100, device="cuda")
    assert bool((pp.embed_bwd(none, normal(2, 5000, 8), 10) == 0).all())


def test_long_rows_beside_each_other():
    # rows that end and begin inside a piece, are one piece exactly, or one token more
    counts = [32, 33, 64, 1, 31, 96, 65, 0, 128, 2, 200, 34, 32, 32]
    ids = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), torch.tensor(counts, device="cuda"))
    for seed in range(3):
        order = torch.randperm(len(ids), generator=rng(seed), device="cuda") if seed else torch.arange(len(ids), device="cuda")
        dy = normal(seed, len(ids), 72)
        check_bwd(pp.embed_bwd(ids[order], dy, len(counts)), ids[order], dy, len(counts))


def test_shapes():
    ids = make_ids(1, 60, 20).reshape(3, 4, 5)
    table, dy = normal(2, 20, 16), normal(3, 3, 4, 5, 16)
    assert pp.embed_fwd(ids, table).shape == (3, 4, 5, 16)
    check_bwd(pp.embed_bwd(ids, dy, 20), ids.reshape(-1), dy, 20)
    one = torch.tensor(7, device="cuda")
    assert torch.equal(pp.embed_fwd(one, table), table[7])
    check_bwd(pp.embed_bwd(one, dy[0, 0, 0], 20), one.reshape(1), dy[0, 0, 0], 20)
    empty = torch.zeros(0, 3, dtype=torch.int64, device="cuda")
    assert pp.embed_fwd(empty, table).shape == (0, 3, 16)


def test_offsets_past_32_bits():
    v, d = 270000, 8192                       # 2.2e9 elements
    table = torch.zeros(v, d, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([v - 1, 0, v - 2, v - 1], device="cuda")
    table[v - 2:] = normal(1, 2, d, dtype="bf16")
    assert torch.equal(pp.embed_fwd(ids, table), table[ids])
    dy = normal(2, 4, d, dtype="bf16")
    dw = pp.embed_bwd(ids, dy, v, out=table)
    assert torch.equal(dw[v - 2], dy[2]) and torch.equal(dw[0], dy[1])
    assert torch.equal(dw[v - 1], (dy[0].float() + dy[3].float()).bfloat16())
    assert not bool(dw[1:v - 2:997].any())
    ids = torch.zeros(v, dtype=torch.int64, device="cuda")
    ids[-1] = 1
    small = normal(3, 2, d, dtype="bf16")
    y = pp.embed_fwd(ids, small, out=table)
    assert torch.equal(y[-1], small[1]) and torch.equal(y[-2], small[0])
    check_bwd(pp.embed_bwd(ids[-3:], y[-3:], 2), ids[-3:], y[-3:], 2)


def test_lookups_of_more_than_one_launch():
    # 2^25 - 2 tokens are a launch where two lie in a workgroup
    t, d = (1 << 25) + 5, 513
    ids, table = torch.zeros(t, dtype=torch.int64, device="cuda"), normal(1, 3, d, dtype="bf16")
    ids[-9:] = torch.tensor([1, 2, 0, 1, 2, 2, IGNORE, 1, 2], device="cuda")
    ids[:3] = torch.tensor([2, IGNORE, 1], device="cuda")
    y = pp.embed_fwd(ids, table)
    want = ref_fwd(torch.arange(3, device="cuda"), table, 1.0, torch.bfloat16)
    assert torch.equal(y[-9:], ref_fwd(ids[-9:], table, 1.0, torch.bfloat16)) and torch.equal(y[:3], ref_fwd(ids[:3], table, 1.0, torch.bfloat16))
    for part in y[3:-9].split(1 << 21):
        assert bool((part == want[0]).all())


def test_streams_and_graphs():
    t, v, d = 3000, 400, 96
    ids, table, dy = make_ids(1, t, v, "heavy"), normal(2, v, d), normal(3, t, d)
    want = pp.embed_fwd(ids, table, scale=3.0), pp.embed_bwd(ids, dy, v, scale=3.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pp.embed_fwd(ids, table, scale=3.0, stream=side), pp.embed_bwd(ids, dy, v, scale=3.0, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    y, dw = torch.empty(t, d, device="cuda"), torch.empty(v, d, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pp.embed_fwd(ids, table, scale=3.0, out=y)
        pp.embed_bwd(ids, dy, v, scale=3.0, out=dw)
    for k in range(4):
        ids.copy_(make_ids(10 + k, t, v, "heavy", ignored=0.1))
        dy.copy_(normal(20 + k, t, d))
        graph.replay()
        assert torch.equal(y, ref_fwd(ids, table, 3.0, torch.float32))
        assert torch.equal(dw, pp.embed_bwd(ids, dy, v, scale=3.0))
        check_bwd(dw, ids, dy, v, 3.0)


def test_outputs_count_as_changed():
    ids, table = make_ids(1, 9, 4), normal(2, 4, 8)
    out, dw = torch.empty(9, 8, device="cuda"), torch.empty(4, 8, device="cuda")
    before = out._version, dw._version
    pp.embed_fwd(ids, table.requires_grad_(), out=out)
    pp.embed_bwd(ids, out, 4, out=dw)
    assert out._version > before[0] and dw._version > before[1] and not out.requires_grad
