"""The norm, clipping and embedding calls refuse bad arguments before any launch (no GPU needed): sizes, types, alignment, matrices
whose rows overlap, and outputs that lie over what the call reads or writes elsewhere."""
import ctypes as C
import random

import pytest
import torch

from paper_1804_08066_amd import mqgrad as mq

F32, F16, BF16 = mq.MQG_FLOAT32, mq.MQG_FLOAT16, mq.MQG_BFLOAT16
SIZE = {F32: 4, F16: 2, BF16: 2}
A, B = 0x10000, 0x20000           # never dereferenced: every call here is refused, or has nothing to do


def items(*entries):
    table = (mq.ClipItem * max(1, len(entries)))()
    for k, e in enumerate(entries):
        table[k] = mq.ClipItem(*e)
    return table


def norm(table, count=None, workspace=A, out=B):
    return mq.lib().mqg_global_norm(table, len(table) if count is None else count, workspace, out, None)


def by_norm(table, count=None, at=0x8000, max_norm=1.0):
    return mq.lib().mqg_clip_by_norm(table, len(table) if count is None else count, at, max_norm, None)


def both(table, count=None, max_norm=1.0, workspace=0x1000000, out=0x8000):
    return mq.lib().mqg_clip_global_norm(table, len(table) if count is None else count, max_norm, workspace, out, None)


def test_workspace_sizes():
    assert mq.mqg_global_norm_workspace_bytes(0) == 0
    sizes = [mq.mqg_global_norm_workspace_bytes(k) for k in (1, 10, 200, 1000, 65536)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and sizes[-1] < 1 << 24
    assert mq.mqg_embedding_grad_workspace_bytes(0, 64, 100) == 0
    grown = [mq.mqg_embedding_grad_workspace_bytes(n, 64, 50000) for n in (1, 1000, 100_000, 10_000_000)]
    assert grown == sorted(grown) and all(b % 16 == 0 for b in grown)
    for bad in ((1 << 31, 64, 100), (10, 0, 100), (10, (1 << 20) + 1, 100), (10, 64, 0), (10, 64, 1 << 31)):
        assert mq.mqg_embedding_grad_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("call", [norm, by_norm, both])
def test_tensor_lists_are_checked(call):
    good = (A, B, 10, F32, F32)
    assert call(None, 1) == mq.MQG_EINVAL
    assert call(items(good), 65537) == mq.MQG_EINVAL
    assert call(items((None, B, 10, F32, F32))) == mq.MQG_EINVAL
    assert call(items((A, B, 10, 3, F32))) == mq.MQG_EINVAL
    assert call(items((A, B, 10, -1, F32))) == mq.MQG_EINVAL
    assert call(items((A, B, 1 << 60, F32, F32))) == mq.MQG_EINVAL
    assert call(items((A + 2, B, 10, F32, F32))) == mq.MQG_EALIGN
    assert call(items((A + 1, B, 10, F16, F32))) == mq.MQG_EALIGN
    assert call(items((A, B, 10, F32, F32), (A + 1, B, 10, BF16, F32))) == mq.MQG_EALIGN


def test_norm_and_its_places_are_checked():
    good = items((A, None, 10, F32, 7))   # neither `out` nor its type is read
    assert norm(good, workspace=None) == mq.MQG_EINVAL
    assert norm(good, out=None) == mq.MQG_EINVAL
    assert norm(good, out=B + 4) == mq.MQG_EALIGN
    assert norm(good, workspace=0x40004) == mq.MQG_EALIGN
    assert norm(good, workspace=A - 64) == mq.MQG_EINVAL                 # over the tensor
    assert norm(good, workspace=0x40000, out=A + 32) == mq.MQG_EINVAL
    assert norm(good, workspace=B - 64) == mq.MQG_EINVAL                 # over the norm
    clip = items((A, B, 10, F32, F32))
    assert by_norm(clip, at=None) == mq.MQG_EINVAL
    assert by_norm(clip, at=0x8004) == mq.MQG_EALIGN
    for call in (by_norm, both):
        for bad in (-1.0, -1e-300, float("nan")):
            assert call(clip, max_norm=bad) == mq.MQG_EINVAL
        assert call(items((A, None, 10, F32, F32))) == mq.MQG_EINVAL
        assert call(items((A, B, 10, F32, 4))) == mq.MQG_EINVAL
        assert call(items((A, B + 2, 10, F32, F32))) == mq.MQG_EALIGN
        assert call(items((A, B + 1, 10, F32, BF16))) == mq.MQG_EALIGN
    assert both(clip, workspace=None) == mq.MQG_EINVAL
    assert both(clip, out=None) == mq.MQG_EINVAL
    assert both(clip, workspace=0x40004) == mq.MQG_EALIGN
    assert by_norm(items((A, B, 0, F32, F32))) == mq.MQG_OK       # nothing to do
    assert by_norm(items(), 0) == mq.MQG_OK


@pytest.mark.parametrize("call", [by_norm, both])
def test_outputs_over_other_memory_are_refused(call):
    n = 100
    assert call(items((A, A, n, F32, BF16))) == mq.MQG_EINVAL                        # the same place, another type
    assert call(items((A, A + 4, n, F32, F32))) == mq.MQG_EINVAL                      # shifted by one value
    assert call(items((A, A, n, F32, F32), (A, A, n, F32, F32))) == mq.MQG_EINVAL      # one tensor twice, in place
    assert call(items((A, B, n, F32, F32), (A + 400, B + 396, n, F32, F32))) == mq.MQG_EINVAL   # outputs share a value
    assert call(items((A, B, n, F32, F32), (B + 200, 0x30000, n, F32, F32))) == mq.MQG_EINVAL   # an output over an input
    assert call(items((A, B, n, F32, F32)), **({"at": B + 8} if call is by_norm else {"out": B + 8})) == mq.MQG_EINVAL
    many = [(A + 512 * k, A + 512 * k, 128, F32, F32) for k in range(300)]
    random.Random(3).shuffle(many)
    assert call(items(*many, (A + 512 * 17 + 508, 0x40000, 1, F32, F32))) == mq.MQG_EINVAL
    if call is both:
        assert both(items((A, B, n, F32, F32)), workspace=B - 64) == mq.MQG_EINVAL
        assert both(items((A, B, n, F32, F32)), workspace=A - 64) == mq.MQG_EINVAL   # over an input
        assert both(items((A, B, n, F32, F32)), out=A + 8) == mq.MQG_EINVAL


def test_the_check_of_outputs_agrees_with_all_pairs():
    """Refused exactly where two spans collide: random lists against the definition.  A list that is not refused is made to fail
    on its last entry's type, so that nothing is launched."""
    rnd = random.Random(11)
    refused = 0
    for _ in range(4000):
        entries = []
        for _ in range(rnd.randint(1, 6)):
            n, dtype, out_dtype = rnd.randint(0, 6), rnd.choice([F32, F16, BF16]), rnd.choice([F32, F16, BF16])
            at = 0x10000 + 4 * rnd.randint(0, 60)
            out = at if rnd.random() < 0.4 else 0x10000 + 4 * rnd.randint(0, 60)
            entries.append((at, out, n, dtype, out_dtype))
        collide = False
        for k, (at, out, n, dtype, out_dtype) in enumerate(entries):
            if n == 0:
                continue
            end = out + n * SIZE[out_dtype]
            for j, (at2, out2, n2, dtype2, out_dtype2) in enumerate(entries):
                if n2 == 0:
                    continue
                over_in = out < at2 + n2 * SIZE[dtype2] and at2 < end
                over_out = out < out2 + n2 * SIZE[out_dtype2] and out2 < end
                if j == k:
                    collide |= over_in and not (at == out and dtype == out_dtype)
                else:
                    collide |= over_in or over_out
        # a norm at 0x8000 lies over nothing; at an output's first value it does
        st = by_norm(items(*entries, (0x90000, 0x90000, 1, F32, BF16)))   # the last entry collides by itself
        assert st == mq.MQG_EINVAL
        if collide:
            refused += 1
            assert by_norm(items(*entries)) == mq.MQG_EINVAL
        elif not torch.cuda.is_available() and any(e[2] for e in entries):
            assert by_norm(items(*entries)) == mq.MQG_ELAUNCH   # accepted: there is no GPU to launch on
    assert 1000 < refused < 3900


def rows(data=A, n=8, stride=16, dtype=F32):
    return C.byref(mq.Rows(data, n, stride, dtype))


def tokens(ids=0x1000, count=4, type=mq.MQG_INDEX32, first_row=0, padding=-1):
    return C.byref(mq.Tokens(ids, count, type, first_row, padding))


def lookup(table=rows(), ids=tokens(), dim=16, out=rows(B, 4)):
    return mq.lib().mqg_embedding(table, ids, dim, 1.0, out, None)


def grad(g=rows(A, 4), ids=tokens(), dim=16, out=rows(B), accumulate=0, workspace=0x100000):
    return mq.lib().mqg_embedding_grad(g, ids, dim, 1.0, out, accumulate, workspace, None)


def test_embedding_arguments_are_checked():
    for call in (lookup, grad):
        for dim in (0, (1 << 20) + 1):
            assert call(dim=dim) == mq.MQG_EINVAL
        assert call(ids=None) == mq.MQG_EINVAL
        assert call(out=None) == mq.MQG_EINVAL
        assert call(ids=tokens(None)) == mq.MQG_EINVAL
        assert call(ids=tokens(type=2)) == mq.MQG_EINVAL
        assert call(ids=tokens(count=1 << 31)) == mq.MQG_EINVAL
        assert call(ids=tokens(count=5)) == mq.MQG_EINVAL                # the other matrix has four rows
        assert call(ids=tokens(first_row=-1)) == mq.MQG_EINVAL
        assert call(ids=tokens(first_row=(1 << 62) + 1)) == mq.MQG_EINVAL
        assert call(ids=tokens(ids=0x1002)) == mq.MQG_EALIGN
        assert call(ids=tokens(ids=0x1004, type=mq.MQG_INDEX64)) == mq.MQG_EALIGN
    assert lookup(table=None) == mq.MQG_EINVAL
    assert lookup(table=rows(None)) == mq.MQG_EINVAL
    assert lookup(table=rows(n=0)) == mq.MQG_EINVAL
    assert lookup(table=rows(n=1 << 31)) == mq.MQG_EINVAL
    assert lookup(table=rows(stride=1 << 62)) == mq.MQG_EINVAL
    assert lookup(table=rows(dtype=3)) == mq.MQG_EINVAL
    assert lookup(table=rows(A + 2)) == mq.MQG_EALIGN
    assert lookup(out=rows(B, 4, 15)) == mq.MQG_EINVAL                   # its rows overlap
    assert lookup(out=rows(B + 1, 4, dtype=BF16)) == mq.MQG_EALIGN
    assert lookup(out=rows(A + 64, 4)) == mq.MQG_EINVAL                  # over the table
    assert lookup(out=rows(0xF04, 4)) == mq.MQG_EINVAL                   # over the tokens
    assert grad(g=None) == mq.MQG_EINVAL
    assert grad(g=rows(A, 3)) == mq.MQG_EINVAL
    assert grad(g=rows(A, 4, dtype=9)) == mq.MQG_EINVAL
    assert grad(g=rows(A + 2, 4)) == mq.MQG_EALIGN
    assert grad(out=rows(B, 0)) == mq.MQG_EINVAL
    assert grad(out=rows(B, 8, 15)) == mq.MQG_EINVAL
    assert grad(out=rows(A + 64)) == mq.MQG_EINVAL                       # over grad_out
    many = dict(g=rows(A, 5000), ids=tokens(count=5000), out=rows(0x200000))   # a few positions need no workspace
    assert mq.mqg_embedding_grad_workspace_bytes(5000, 16, 8) > 0
    assert grad(workspace=None, **many) == mq.MQG_EINVAL
    assert grad(workspace=0x300008, **many) == mq.MQG_EALIGN
    for over in (A, 0x1000, 0x200000):
        assert grad(workspace=over, **many) == mq.MQG_EINVAL
    assert lookup(ids=tokens(None, 0), out=rows(None, 0)) == mq.MQG_OK    # no tokens: nothing to do
    assert grad(g=rows(None, 0), ids=tokens(None, 0), accumulate=1, workspace=None) == mq.MQG_OK


def test_binding_refuses_what_the_calls_cannot_take():
    x = torch.zeros(4, 8)
    ids = torch.zeros(4, dtype=torch.int64)
    for call in (lambda: mq.mqg_global_norm([x]), lambda: mq.mqg_clip_global_norm([x], 1.0), lambda: mq.mqg_embedding(x, ids),
                 lambda: mq.mqg_clip_by_norm([x], torch.zeros(1, dtype=torch.float64), 1.0), lambda: mq.mqg_embedding_grad(x, ids, 10)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        mq.mqg_clip_by_norm([], torch.zeros(1, dtype=torch.float64), 1.0, outputs=[x])
