"""Gradients that share memory: refused at the C boundary, if and only if one is
written where another lies.  No call here reaches a device: its workspace is too
small, which is looked at last."""
import random

import pytest

from paper_2304_13724_amd import bgmf

A = 1 << 20  # an aligned address that no call may touch
F32, BF16 = 0, 1


def code(grads):
    """BGMF_E_ARG: shared memory was found; BGMF_E_BUDGET: none was."""
    table = (bgmf.Grad * len(grads))(*[bgmf.Grad(*g) for g in grads])
    with pytest.raises(bgmf.BgmfError) as e:
        bgmf.bgmf_clip_grad_norm(table, len(grads), 1.0, A, A, 0, 0)
    if e.value.code == bgmf.BGMF_E_ARG:
        assert "share memory" in str(e.value)
    return e.value.code


def elements(at, rows, cols, stride, size):
    return {at + r * stride * size + i for r in range(rows) for i in range(cols * size)}


def overlaps(grads):
    """By the bytes themselves."""
    sets = []
    for g in grads:
        at, out, rows, cols, in_stride, out_stride, type_ = g
        size = 4 if type_ == F32 else 2
        sets.append((elements(at, rows, cols, in_stride, size),
                     elements(out, rows, cols, out_stride, size), at == out))
    for i, (_, out, same) in enumerate(sets):
        for j, (other_in, other_out, _) in enumerate(sets):
            if i == j:
                if not same and out & other_in:
                    return True
            elif out & other_in or out & other_out:
                return True
    return False


@pytest.mark.parametrize("grads,shared", [
    ([(A, A, 1, 5, 5, 5, F32)] * 2, True),                                    # the same twice
    ([(A, A, 1, 5, 5, 5, F32), (A + 16, A + 16, 1, 3, 3, 3, F32)], True),      # one element
    ([(A, A, 1, 5, 5, 5, F32), (A + 20, A + 20, 1, 3, 3, 3, F32)], False),     # neighbours
    ([(A + 20, A + 20, 1, 3, 3, 3, F32), (A, A, 1, 5, 5, 5, F32)], False),     # in another order
    ([(A, A + 4, 1, 5, 5, 5, F32)], True),                                    # moved by one
    ([(A, A, 50, 3, 9, 9, F32), (A + 12, A + 12, 50, 6, 9, 9, F32)], False),   # columns
    ([(A, A, 50, 3, 9, 9, F32), (A + 12, A + 12, 50, 7, 9, 9, F32)], True),
    ([(A, 2 * A, 1, 5, 5, 5, F32), (A, 3 * A, 1, 5, 5, 5, F32)], False),       # one input, two outs
    ([(A, 2 * A, 1, 5, 5, 5, F32), (3 * A, A + 8, 1, 5, 5, 5, F32)], True),
    ([(A, 2 * A, 0, 5, 5, 5, F32), (A, 2 * A, 1, 0, 5, 5, F32), (A, 2 * A, 1, 5, 5, 5, F32)], False),
    ([(A, A, 1 << 20, 1, 1 << 19, 1 << 19, F32), (A + 4, A + 4, 1 << 20, 2, 1 << 19, 1 << 19, F32)],
     False)])
def test_gradients_that_share_memory(grads, shared):
    assert code(grads) == (bgmf.BGMF_E_ARG if shared else bgmf.BGMF_E_BUDGET)


@pytest.mark.parametrize("seed", range(8))
def test_against_the_bytes(seed):
    rng = random.Random(seed)
    found = [0, 0]
    for _ in range(400):
        grads = []
        for _ in range(rng.randint(1, 4)):
            type_ = rng.choice([F32, BF16])
            size = 4 if type_ == F32 else 2
            rows, cols = rng.randint(0, 6), rng.randint(0, 4)
            strides = [cols + rng.choice([0, 0, 1, 3, 7]) for _ in range(2)]
            at, out = (A + size * rng.randint(0, rng.choice([12, 60, 200])) for _ in range(2))
            if rng.random() < 0.6:
                out, strides[1] = at, strides[0]
            elif out == at and strides[0] != strides[1]:
                continue
            if rng.random() < 0.5 and grads:  # as wide apart as the one before
                strides = [max(s, cols) for s in grads[-1][4:6]]
                if out == at:
                    strides[1] = strides[0]
            grads.append((at, out, rows, cols, *strides, type_))
        if grads:
            shared = overlaps(grads)
            found[shared] += 1
            assert code(grads) == (bgmf.BGMF_E_ARG if shared else bgmf.BGMF_E_BUDGET), grads
    assert min(found) > 40, found
