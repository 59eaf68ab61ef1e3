"""Rows by token and their gradient against the definitions in 64 bits.

Tolerances.  lookup: one fp32 product (2^-24), one rounding to the output's type (eps / 2).  gradient: m rows added in fp32 in any
order are off by at most (m - 1) * 2^-24 of the sum of their magnitudes (first order; the factor 1.01 covers the rest), the
product with scale and the addition to the old value by 2^-24 of the result each, the rounding to the output's type by eps / 2."""
import numpy as np
import pytest
import torch

from oracle import ref
from paper_1804_08066_amd import mqgrad as mq
from paper_1804_08066_amd import workloads
from helpers import to_u32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]


def matrix(rows, dim, seed, dtype=F32, std=1.0):
    return workloads.normal(rows * dim, std, seed, DEV).view(rows, dim).to(dtype)


def host(t):
    return t.detach().cpu().to(torch.float64).numpy()


def some_tokens(kind, count, rows, seed=1):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    if kind == "spread":
        return torch.randint(0, rows, (count,), generator=g)
    if kind == "text":     # frequencies fall with the rank
        u = torch.rand(count, generator=g, dtype=torch.float64)
        return ((rows + 1.0) ** u - 1.0).long().clamp(0, rows - 1)
    if kind == "one":
        return torch.full((count,), rows - 1)
    if kind == "sorted":
        return torch.arange(count) * rows // max(1, count)
    if kind == "shards":   # every third belongs elsewhere, before and behind
        t = torch.randint(-rows, 2 * rows, (count,), generator=g)
        t[::7] = -1
        return t
    assert kind == "none"
    return torch.full((count,), rows)


KINDS = ["spread", "text", "one", "sorted", "shards", "none"]


def check_lookup(table, ids, out, scale, first_row=0):
    t, at = host(table), ids.cpu().reshape(-1).numpy().astype(np.int64) - first_row
    there = (at >= 0) & (at < t.shape[0])
    want = np.where(there[:, None], t[np.where(there, at, 0)], 0.0) * np.float64(np.float32(scale))
    got = host(out).reshape(want.shape)
    info = torch.finfo(out.dtype)
    tol = (2.0 ** -24 if scale not in (0.0, 1.0) else 0.0) + (info.eps / 2 if out.dtype != F32 else 0.0)
    assert np.all(np.abs(got - want) <= 1.01 * tol * np.abs(want) + info.smallest_normal * info.eps)
    assert not got[~there].any()


def check_grad(grad_out, ids, out, rows, scale, first_row=0, padding=None, old=None):
    g = host(grad_out).reshape(ids.numel(), -1)
    at = ids.cpu().reshape(-1).numpy().astype(np.int64)
    use = (at >= first_row) & (at < first_row + rows)
    if padding is not None:
        use &= at != padding
    at = at[use] - first_row
    order = np.argsort(at, kind="stable")
    count = np.bincount(at, minlength=rows)
    total, size = np.zeros((rows, g.shape[1])), np.zeros((rows, g.shape[1]))
    if len(at):
        named, starts = np.unique(at[order], return_index=True)
        total[named] = np.add.reduceat(g[use][order], starts, axis=0)
        size[named] = np.add.reduceat(np.abs(g[use][order]), starts, axis=0)
    s = np.float64(np.float32(scale))
    want = s * total + (host(old) if old is not None else 0.0)
    got = host(out)
    info = torch.finfo(out.dtype)
    tol = abs(s) * np.maximum(count - 1, 0)[:, None] * 2.0 ** -24 * size + 2.0 ** -24 * (np.abs(want) + np.abs(s * total))
    if out.dtype != F32:
        tol += info.eps / 2 * (np.abs(want) + tol)
    worst = np.abs(got - want) - 1.01 * tol - info.smallest_normal * info.eps
    assert np.all(worst <= 0), (worst.max(), np.unravel_index(worst.argmax(), worst.shape))
    untouched = count == 0
    if old is None:
        assert not got[untouched].any() and not np.signbit(got[untouched]).any()
    else:
        assert torch.equal(out.cpu()[torch.from_numpy(untouched)], old.cpu()[torch.from_numpy(untouched)])


# ---- lookup ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("index", [torch.int32, torch.int64], ids=str)
@pytest.mark.parametrize("out", TYPES, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_lookup_types(dtype, out, index):
    for dim, scale in ((64, 1.0), (131, -0.7), (4, 3.0)):
        table = matrix(77, dim, 1, dtype)
        ids = some_tokens("shards", 500, 77).to(DEV, index)
        got = mq.mqg_embedding(table, ids, scale=scale, out=torch.full((500, dim), 9.0, dtype=out, device=DEV))
        check_lookup(table, ids, got, scale)


@pytest.mark.parametrize("dim", [1, 2, 3, 7, 8, 9, 31, 255, 256, 257, 1023, 1024, 1025, 2048, 2049, 5000])
@pytest.mark.parametrize("tokens", [1, 2, 3, 65])
def test_lookup_sizes(tokens, dim):
    for dtype in (F32, BF16):
        table = matrix(11, dim, 2, dtype)
        ids = some_tokens("spread", tokens, 11).to(DEV)
        check_lookup(table, ids, mq.mqg_embedding(table, ids, scale=2.0), 2.0)


def test_lookup_shapes_strides_and_alignment():
    wide = matrix(40, 100, 3, BF16)
    table = wide[:, 3:90]                                   # rows at a stride, aligned to two bytes
    ids = some_tokens("spread", 24, 40).view(2, 3, 4).to(DEV)
    got = mq.mqg_embedding(table, ids)
    assert got.shape == (2, 3, 4, 87) and got.dtype == BF16
    check_lookup(table, ids, got, 1.0)
    frame = torch.full((24, 120), 5.0, dtype=F16, device=DEV)
    mq.mqg_embedding(table, ids.view(-1), out=frame[:, 7:94])
    check_lookup(table, ids, frame[:, 7:94], 1.0)
    assert (frame[:, :7] == 5.0).all() and (frame[:, 94:] == 5.0).all()
    one = matrix(1, 87, 4)
    check_lookup(one.expand(40, 87), ids, mq.mqg_embedding(one.expand(40, 87), ids), 1.0)   # one row for all tokens


def test_shards_add_up_to_the_table():
    table = matrix(100, 33, 5)
    ids = some_tokens("spread", 300, 100).to(DEV)
    whole = mq.mqg_embedding(table, ids, scale=0.5)
    parts = [mq.mqg_embedding(table[lo:lo + 25], ids, scale=0.5, first_row=lo) for lo in range(0, 100, 25)]
    assert torch.equal(sum(parts), whole)
    far = mq.mqg_embedding(table, ids + (1 << 40), first_row=1 << 40)
    assert torch.equal(far, mq.mqg_embedding(table, ids))
    edges = torch.tensor([-(1 << 63), (1 << 63) - 1, -1, 100, 0, 99], device=DEV)
    got = mq.mqg_embedding(table, edges)
    assert not got[:4].any() and torch.equal(got[4:], table[[0, 99]])


def test_lookup_of_nothing():
    table = matrix(10, 16, 6)
    assert mq.mqg_embedding(table, torch.empty(0, dtype=torch.int64, device=DEV)).shape == (0, 16)


def test_lookup_keeps_special_values():
    table = matrix(4, 16, 7)
    table[1, 3], table[1, 4], table[2, 5] = float("inf"), float("-inf"), float("nan")
    ids = torch.tensor([0, 1, 2, 7], device=DEV)
    got = mq.mqg_embedding(table, ids)
    assert torch.equal(got[0], table[0]) and torch.equal(got[1], table[1])
    assert torch.isnan(got[2, 5]) and torch.isfinite(got[2, :5]).all() and not got[3].any()
    big = torch.full((1, 4), 3e38, device=DEV)
    assert torch.isinf(mq.mqg_embedding(big, ids[:1], out=torch.empty(1, 4, dtype=F16, device=DEV))).all()   # as a conversion


# ---- gradient ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("out", TYPES, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_gradient_types(dtype, out, accumulate):
    for dim, rows, count, index in ((64, 50, 700, torch.int32), (37, 90, 3000, torch.int64), (520, 20, 90, torch.int64), (300, 60, 5000, torch.int32),
                                    (36, 70, 9000, torch.int64)):
        g = matrix(count, dim, 11, dtype)
        ids = some_tokens("shards", count, rows).to(DEV, index)
        old = matrix(rows, dim, 12, out)
        got = old.clone()
        back = mq.mqg_embedding_grad(g, ids, rows, scale=-0.3, padding_id=5, out=got, accumulate=accumulate)
        assert back is got
        check_grad(g, ids, got, rows, -0.3, padding=5, old=old if accumulate else None)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("count", [1, 2, 63, 64, 65, 200, 511, 513, 1024, 1025, 2047, 2049, 4096, 4097, 8192, 8193, 16_384, 16_385, 20_000])
def test_gradient_lengths(count, kind):
    for dim, rows in ((5, 300), (24, 7), (130, 1000)):
        g = matrix(count, dim, count, BF16)
        ids = some_tokens(kind, count, rows, seed=count).to(DEV)
        check_grad(g, ids, mq.mqg_embedding_grad(g, ids, rows, out=torch.full((rows, dim), 9.0, device=DEV)), rows, 1.0)


@pytest.mark.parametrize("dim", [1, 2, 3, 7, 8, 9, 31, 64, 255, 256, 257, 1023, 1025, 2048, 2049, 5000])
@pytest.mark.parametrize("dtype", [F32, F16], ids=str)
def test_gradient_widths(dtype, dim):
    for count, rows in ((50, 20), (700, 30), (3000, 40), (9000, 50)):
        g = matrix(count, dim, dim, dtype)
        ids = some_tokens("text", count, rows).to(DEV)
        check_grad(g, ids, mq.mqg_embedding_grad(g, ids, rows, scale=2.0, out=torch.full((rows, dim), 9.0, device=DEV)), rows, 2.0)


@pytest.mark.parametrize("rows", [1, 2, 255, 256, 257, 1023, 1024, 65_535, 65_536, (1 << 20) - 1, 1 << 20, (1 << 20) + 1])
def test_gradient_tables(rows):
    """One, two and three digits of the sort, and keys that fill them."""
    for count in (300, 9000):
        ids = some_tokens("spread", count, rows)
        ids[:3] = rows - 1
        ids[5] = rows
        ids = ids.to(DEV)
        g = matrix(count, 3, 13)
        check_grad(g, ids, mq.mqg_embedding_grad(g, ids, rows), rows, 1.0)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("rows", [511, 60_000, 65_281, 262_144, 262_145, 600_000])
@pytest.mark.parametrize("count", [5000, 16_384])
def test_gradient_where_the_remainders_by_256_are_few(count, rows, accumulate):
    """Rows that lie a multiple of 256 apart come together in the sort: all of them, none, and more than it compares with each other."""
    for used in ([7], [0, 255], [3, 4, 5, 200, 254]):
        quotients = some_tokens("text", count, (rows + 255) // 256, seed=count)
        ids = quotients * 256 + torch.tensor(used)[torch.arange(count) % len(used)]   # some behind the last row
        ids[::11] = -5
        ids = ids.to(DEV)
        g, old = matrix(count, 4, 14), matrix(rows, 4, 15)
        out = old.clone()
        mq.mqg_embedding_grad(g, ids, rows, scale=-1.5, out=out, accumulate=accumulate)
        check_grad(g, ids, out, rows, -1.5, old=old if accumulate else None)


@pytest.mark.parametrize("kind", KINDS)
def test_gradient_of_long_batches(kind):
    """More positions than the sort's workgroups take in one go."""
    for count, dim, rows in ((600_001, 2, 70_000), (70_000, 40, 3000)):
        g = matrix(count, dim, 14)
        ids = some_tokens(kind, count, rows).to(DEV)
        check_grad(g, ids, mq.mqg_embedding_grad(g, ids, rows), rows, 1.0)


@pytest.mark.parametrize("tokens", [9, 600, 30_000])
def test_gradient_equal_inputs_equal_bits(tokens):
    g = matrix(tokens, 72, 15)
    ids = some_tokens("text", tokens, 500).to(DEV)
    first = mq.mqg_embedding_grad(g, ids, 500)
    workspace = torch.full((mq.mqg_embedding_grad_workspace_bytes(tokens, 72, 500),), 255, dtype=torch.uint8, device=DEV)
    for index in (torch.int64, torch.int32):
        assert torch.equal(mq.mqg_embedding_grad(g, ids.to(index), 500, workspace=workspace), first)


@pytest.mark.parametrize("tokens", [40, 700, 5000, 9000])
def test_positions_that_add_to_no_row_are_not_read_into_any(tokens):
    """Infinite and missing values at padded and foreign positions stay out of every row."""
    ids = some_tokens("shards", tokens, 60).to(DEV)
    ids[3::5] = 0
    g = matrix(tokens, 48, 16)
    off = (ids <= 0) | (ids >= 60)
    g[off] = float("nan")
    g[3] = float("inf")
    got = mq.mqg_embedding_grad(g, ids, 60, padding_id=0)
    assert torch.isfinite(got).all() and not got[0].any()
    check_grad(torch.where(off[:, None], 0.0, g), ids, got, 60, 1.0, padding=0)
    at = int((~off).nonzero()[0])
    g[at, 7] = float("nan")
    got = mq.mqg_embedding_grad(g, ids, 60, padding_id=0)
    assert torch.isnan(got).sum() == 1 and torch.isnan(got[ids[at], 7])


@pytest.mark.parametrize("tokens", [20, 600, 5000, 12_000])
def test_gradient_strides_alignment_and_leading_dimensions(tokens):
    wide = matrix(tokens, 100, 17, BF16)
    g = wide[:, 5:66]
    ids = some_tokens("text", tokens, 90).to(DEV)
    frame = torch.full((92, 80), 5.0, dtype=BF16, device=DEV)
    out = frame[1:91, 3:64]
    mq.mqg_embedding_grad(g, ids, 90, out=out)
    check_grad(g, ids, out, 90, 1.0)
    keep = torch.ones_like(frame, dtype=torch.bool)
    keep[1:91, 3:64] = False
    assert (frame[keep] == 5.0).all()
    old = out.clone()
    mq.mqg_embedding_grad(g, ids, 90, scale=0.5, out=out, accumulate=True)
    check_grad(g, ids, out, 90, 0.5, old=old)
    assert (frame[keep] == 5.0).all()
    shaped = mq.mqg_embedding_grad(g.contiguous().view(4, tokens // 4, 61), ids.view(4, -1), 90)
    assert torch.equal(shaped, mq.mqg_embedding_grad(g, ids, 90))
    row = matrix(1, 61, 18)
    same = mq.mqg_embedding_grad(row.expand(tokens, 61), ids, 90)          # one gradient for all positions
    check_grad(row.expand(tokens, 61), ids, same, 90, 1.0)


def test_gradient_of_nothing():
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    g = torch.empty(0, 16, device=DEV)
    out = torch.full((30, 16), 4.0, device=DEV)
    mq.mqg_embedding_grad(g, none, 30, out=out, accumulate=True)
    assert (out == 4.0).all()
    mq.mqg_embedding_grad(g, none, 30, out=out)
    assert not out.any()


@pytest.mark.parametrize("tokens", [30, 3000])
def test_shards_gradients_are_slices_of_the_tables(tokens):
    g = matrix(tokens, 20, 19)
    ids = some_tokens("text", tokens, 400).to(DEV)
    for lo in range(0, 400, 100):
        check_grad(g, ids, mq.mqg_embedding_grad(g, ids, 100, first_row=lo), 100, 1.0, first_row=lo)
    base = 1 << 40
    far = mq.mqg_embedding_grad(g, ids + base, 400, first_row=base, padding_id=base + 3)
    check_grad(g, ids + base, far, 400, 1.0, first_row=base, padding=base + 3)


def test_gradient_against_differences():
    """The lookup is linear in the table: the loss sum(out * weight) changes by the gradient's element times the step, up to fp32
    roundings of the two lookups (each 2^-24 of a product below 8 in magnitude, 40 of them)."""
    table = matrix(12, 6, 20)
    ids = some_tokens("spread", 40, 12).to(DEV)
    weight = matrix(40, 6, 21)
    grad = mq.mqg_embedding_grad(weight, ids, 12, scale=1.5)
    for r, c in ((0, 0), (3, 5), (11, 2), (7, 4)):
        up, down = table.clone(), table.clone()
        up[r, c] += 0.5
        down[r, c] -= 0.5
        step = (up[r, c].double() - down[r, c].double())
        loss = [(mq.mqg_embedding(t, ids, scale=1.5).double() * weight.double()).sum() for t in (up, down)]
        assert abs((loss[0] - loss[1]) / step - grad[r, c].double()) <= 2 * 40 * 8 * 2.0 ** -24 * 3


@pytest.mark.parametrize("tokens", [7, 3000])
def test_memory_past_four_gigavalues(tokens):
    """Offsets of a table of 4.5 * 10^9 values: rows at its end are looked up, and added to, where they are."""
    rows, dim = 1_100_000, 4096
    table = torch.empty(rows, dim, dtype=BF16, device=DEV)
    ids = (rows - 1 - some_tokens("spread", tokens, 900)).to(DEV)
    ids[0] = rows - 1
    end = table[rows - 1000:]
    end.copy_(matrix(1000, dim, 22, BF16))
    near, old = ids - (rows - 1000), end.clone()
    assert torch.equal(mq.mqg_embedding(table, ids), mq.mqg_embedding(old, near))
    g = matrix(tokens, dim, 23, BF16)
    mq.mqg_embedding_grad(g, ids, rows, scale=-0.1, out=table, accumulate=True)
    check_grad(g, near, end, 1000, -0.1, old=old)


@pytest.mark.parametrize("tokens", [50, 1500, 5000, 9000])
def test_other_stream_and_replayed_graph(tokens):
    rows, dim = 700, 40
    g = matrix(tokens, dim, 24, BF16)
    table = matrix(rows, dim, 25)
    ids = some_tokens("text", tokens, rows).to(DEV)
    out = torch.zeros(rows, dim, device=DEV)
    got = torch.zeros(tokens, dim, dtype=BF16, device=DEV)
    workspace = torch.empty(mq.mqg_embedding_grad_workspace_bytes(tokens, dim, rows), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mq.mqg_embedding_grad(g, ids, rows, out=out, stream=side)
    mq.mqg_embedding(table, ids, out=got, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    check_grad(g, ids, out, rows, 1.0)
    check_lookup(table, ids, got, 1.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mq.mqg_embedding(table, ids, out=got)
        mq.mqg_embedding_grad(g, ids, rows, out=out, workspace=workspace)
        mq.mqg_embedding_grad(g, ids, rows, scale=-0.1, out=table, accumulate=True, workspace=workspace)
    for replay in range(4):
        ids.copy_(some_tokens(KINDS[replay], tokens, rows, seed=replay))
        g.copy_(matrix(tokens, dim, 30 + replay, BF16))
        old = table.clone()
        graph.replay()
        torch.cuda.synchronize()
        check_lookup(old, ids, got, 1.0)
        check_grad(g, ids, out, rows, 1.0)
        check_grad(g, ids, table, rows, -0.1, old=old)


def test_a_training_step_of_a_table():
    """Pull the rows, add up their gradient, clip it with the other layers' into one flat buffer, quantize, and let the server
    apply the exchanged mean of two workers; the same step in plain arithmetic on the host."""
    rows, dim, tokens, bits, bucket, lr, max_norm = 300, 24, 800, 6, 256, 0.5, 0.7
    n = rows * dim + 100
    params = workloads.uniform(n, -0.05, 0.05, 1, DEV)
    table = params[:rows * dim].view(rows, dim)
    streams, want = [], []
    for w in range(2):
        ids = some_tokens("text", tokens, rows, seed=w).to(DEV)
        x = mq.mqg_embedding(table, ids, scale=2.0, out=torch.empty(tokens, dim, dtype=BF16, device=DEV))
        g_table = mq.mqg_embedding_grad(x, ids, rows, scale=2.0, out=torch.empty(rows, dim, dtype=BF16, device=DEV))   # of half the squares' sum
        grads = [g_table.view(-1), workloads.normal(100, 0.1, w, DEV)]
        check_grad(x, ids, g_table, rows, 2.0)
        flat = torch.empty(n, device=DEV)
        _, norm = mq.mqg_clip_global_norm(grads, max_norm, outputs=list(flat.split([rows * dim, 100])))
        plain = np.concatenate([host(g) for g in grads])
        exact = float(np.sqrt(np.sum(plain ** 2)))
        assert abs(norm.item() - exact) <= 1e-13 * exact and exact > max_norm
        assert np.all(np.abs(host(flat) - plain * (max_norm / exact)) <= 2.0 ** -22 * np.abs(plain))
        streams.append(mq.mqg_quantize(flat, bits, bucket, seed=2, worker=w))
        want.append(ref.quantize(flat.cpu().numpy(), bits, bucket, 2, 0, w))
        assert np.array_equal(to_u32(streams[-1][0]), want[-1][0])
    before = params.cpu().numpy().copy()
    mq.mqg_aggregate_update([s[0] for s in streams], [s[1] for s in streams], n, bits, bucket, lr, params)
    assert np.array_equal(params.cpu().numpy(), ref.aggregate_update([s[0] for s in want], [s[1] for s in want], n, bits, bucket, lr, before))


def test_the_servers_update_from_rows():
    """W workers' rows pushed one after the other, applied in one call: parameters - lr / W * the sum of all rows by token."""
    rows, dim, W, lr = 200, 50, 3, 0.3
    params = matrix(rows, dim, 26)
    old = params.clone()
    ids = torch.cat([some_tokens("text", 150, rows, seed=w) for w in range(W)]).to(DEV)
    g = matrix(150 * W, dim, 27, BF16)
    mq.mqg_embedding_grad(g, ids, rows, scale=-lr / W, out=params, accumulate=True)
    check_grad(g, ids, params, rows, -lr / W, old=old)


@pytest.mark.parametrize("native", [True, False])
def test_binding_refusals(monkeypatch, native):
    mq.lib()
    if not native:
        monkeypatch.setattr(mq, "_marshal", mq._NoTables)
    table = matrix(10, 16, 1)
    ids = torch.zeros(4, dtype=torch.int64, device=DEV)
    g = matrix(4, 16, 2)
    for bad in (ids.float(), ids.to(torch.int16), ids.cpu(), torch.zeros(8, dtype=torch.int64, device=DEV)[::2]):
        with pytest.raises(TypeError):
            mq.mqg_embedding(table, bad)
        with pytest.raises(TypeError):
            mq.mqg_embedding_grad(g, bad, 10)
    with pytest.raises(TypeError):
        mq.mqg_embedding(table.double(), ids)
    with pytest.raises(TypeError):
        mq.mqg_embedding(table.t(), ids)
    with pytest.raises(TypeError):
        mq.mqg_embedding_grad(g.view(2, 2, 16).transpose(0, 1), ids, 10)
    for call in (lambda: mq.mqg_embedding(table, ids, out=torch.empty(4, 15, device=DEV)),
                 lambda: mq.mqg_embedding(table, ids, out=torch.empty(5, 16, device=DEV)),
                 lambda: mq.mqg_embedding(table, ids, first_row=-1),
                 lambda: mq.mqg_embedding_grad(g[:3], ids, 10),
                 lambda: mq.mqg_embedding_grad(g, ids, 10, accumulate=True),
                 lambda: mq.mqg_embedding_grad(g, ids, 10, out=torch.empty(9, 16, device=DEV)),
                 lambda: mq.mqg_embedding_grad(g, ids, 10, out=torch.empty(10, 17, device=DEV)),
                 lambda: mq.mqg_embedding_grad(g, ids, 10, padding_id=1 << 63),
                 lambda: mq.mqg_embedding_grad(matrix(40_000, 16, 3), torch.zeros(40_000, dtype=torch.int32, device=DEV), 10,
                                               workspace=torch.empty(64, dtype=torch.uint8, device=DEV))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(mq.MqgError):
        mq.mqg_embedding(table, ids, out=table[2:6])
    with pytest.raises(mq.MqgError):
        mq.mqg_embedding_grad(g, ids, 4, out=g)
    with pytest.raises(mq.MqgError):
        mq.mqg_embedding_grad(g, ids, 10, out=torch.empty(1, 16, device=DEV).expand(10, 16))


def test_every_form_of_argument_gives_the_same_results(monkeypatch):
    """Whole numbers for scale, parameters, buffers of the call's own or given, and the binding without its native tables."""
    table, ids, g = matrix(90, 40, 1), some_tokens("text", 2000, 90).to(DEV), matrix(2000, 40, 2)
    looked, grad = mq.mqg_embedding(table, ids, scale=2.0), mq.mqg_embedding_grad(g, ids, 90, scale=2.0, padding_id=1)
    for native in (True, False):
        if not native:
            monkeypatch.setattr(mq, "_marshal", mq._NoTables)
        for scale in (2, 2.0):
            assert torch.equal(mq.mqg_embedding(torch.nn.Parameter(table), ids, scale=scale), looked)
            assert torch.equal(mq.mqg_embedding(table, ids, scale=scale, out=torch.zeros_like(looked)), looked)
            assert torch.equal(mq.mqg_embedding_grad(g, ids, 90, scale=scale, padding_id=1), grad)
            workspace = torch.empty(mq.mqg_embedding_grad_workspace_bytes(2000, 40, 90) // 4, dtype=torch.int32, device=DEV)
            assert torch.equal(mq.mqg_embedding_grad(g, ids, 90, scale=scale, padding_id=1, out=torch.zeros_like(grad), workspace=workspace), grad)
