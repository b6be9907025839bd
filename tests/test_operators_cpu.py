"""Operators around the step: what is refused before any CUDA call, and the layouts that the Python names accept."""
import ctypes

import pytest
import torch

import paper_2505_22549_b200 as d
from paper_2505_22549_b200 import binding as B
from paper_2505_22549_b200 import module


def _logprobs(outer=2, inner=3, vocab=8, logits=None, tokens=None, top=0, logp=16, lse=16, entropy=0, ids=0, tlp=0, device=0):
    logits = B.rows(64, d.DESLOC_F32, 24, 8) if logits is None else logits
    tokens = B.rows(64, d.DESLOC_I64, 3, 1) if tokens is None else tokens
    return lambda: B.desloc_token_logprobs(outer, inner, vocab, logits, tokens, top, logp, lse, entropy, ids, tlp, device)


def _grad(outer=2, inner=3, vocab=8, logits=None, tokens=None, out=None, lse=16, dlogp=16, entropy=0, dentropy=0, device=0):
    logits = B.rows(64, d.DESLOC_F32, 24, 8) if logits is None else logits
    tokens = B.rows(64, d.DESLOC_I64, 3, 1) if tokens is None else tokens
    out = B.rows(64, d.DESLOC_F32, 24, 8) if out is None else out
    return lambda: B.desloc_token_logprobs_grad(outer, inner, vocab, logits, tokens, lse, dlogp, entropy, dentropy, out, device)


REFUSED = [
    (_logprobs(outer=-1), d.DESLOC_E_RANGE),
    (_logprobs(inner=-1), d.DESLOC_E_RANGE),
    (_logprobs(vocab=0), d.DESLOC_E_RANGE),
    (_logprobs(vocab=(1 << 30) + 1), d.DESLOC_E_RANGE),
    (_logprobs(outer=1 << 20, inner=1 << 20), d.DESLOC_E_RANGE),
    (_logprobs(top=-1), d.DESLOC_E_RANGE),
    (_logprobs(top=d.DESLOC_MAX_TOP + 1, ids=16, tlp=16), d.DESLOC_E_RANGE),
    (_logprobs(device=-1), d.DESLOC_E_RANGE),
    (_logprobs(logits=B.rows(64, 2, 24, 8)), d.DESLOC_E_INVALID),
    (_logprobs(logits=B.rows(66, d.DESLOC_F32, 24, 8)), d.DESLOC_E_INVALID),
    (_logprobs(tokens=B.rows(64, 7, 3, 1)), d.DESLOC_E_INVALID),
    (_logprobs(tokens=B.rows(68, d.DESLOC_I64, 3, 1)), d.DESLOC_E_INVALID),
    (_logprobs(logits=B.rows(0, d.DESLOC_F32, 24, 8)), d.DESLOC_E_NULL),
    (_logprobs(tokens=B.rows(0, d.DESLOC_I64, 3, 1)), d.DESLOC_E_NULL),
    (_logprobs(logp=0), d.DESLOC_E_NULL),
    (_logprobs(lse=0), d.DESLOC_E_NULL),
    (_logprobs(top=1, ids=16), d.DESLOC_E_NULL),
    (_logprobs(top=1, tlp=16), d.DESLOC_E_NULL),
    (_grad(vocab=0), d.DESLOC_E_RANGE),
    (_grad(device=-1), d.DESLOC_E_RANGE),
    (_grad(out=B.rows(64, d.DESLOC_BF16, 24, 8)), d.DESLOC_E_INVALID),
    (_grad(out=B.rows(65, d.DESLOC_F32, 24, 8)), d.DESLOC_E_INVALID),
    (_grad(out=B.rows(0, d.DESLOC_F32, 24, 8)), d.DESLOC_E_NULL),
    (_grad(lse=0), d.DESLOC_E_NULL),
    (_grad(dlogp=0), d.DESLOC_E_NULL),
    (_grad(dentropy=16), d.DESLOC_E_NULL),
]


@pytest.mark.parametrize("k", range(len(REFUSED)))
def test_logprobs_refused_before_any_cuda_call(k):
    call, status = REFUSED[k]
    with pytest.raises(d.DeslocError) as e:
        call()
    assert e.value.status == status


def test_no_rows_is_no_work():
    _logprobs(outer=0, logits=B.rows(0, d.DESLOC_F32, 0, 0), tokens=B.rows(0, d.DESLOC_I64, 0, 0), logp=0, lse=0)()
    _grad(inner=0, logits=B.rows(0, d.DESLOC_F32, 0, 0), tokens=B.rows(0, d.DESLOC_I64, 0, 0), lse=0, dlogp=0)()


def test_calls_with_a_context_refuse_none():
    L, none = d.raw_lib(), B.rows(64, 0, 1, 1)
    assert L.desloc_embed(None, 0, 8, none, 1, 1.0, none, None) == d.DESLOC_E_NULL
    assert L.desloc_embed_grad(None, 0, 8, none, 1, none, 1.0, 0, None, None, 0, None) == d.DESLOC_E_NULL
    assert L.desloc_embed_grad_bytes(None, 0, 8, 1) == d.DESLOC_E_NULL
    assert L.desloc_clip_grads(None, 1.0, 0, None, 0, None, None, None, None, 0, None) == d.DESLOC_E_NULL
    assert L.desloc_clip_grads_bytes(None) == d.DESLOC_E_NULL
    assert L.desloc_token_logprobs(1, 1, 1, None, None, 0, None, None, None, None, None, 0, None) == d.DESLOC_E_NULL
    assert L.desloc_token_logprobs_grad(1, 1, 1, none, none, None, None, None, None, None, 0, None) == d.DESLOC_E_NULL


def test_rows_struct_is_the_headers():
    assert ctypes.sizeof(B.DeslocRows) == 32
    assert (B.DeslocRows.data.offset, B.DeslocRows.dtype.offset, B.DeslocRows.stride.offset) == (0, 8, 16)


def test_host_tensors_are_refused():
    x, t = torch.zeros(2, 3, 8), torch.zeros(2, 3, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA"):
        d.token_logprobs(x, t)
    with pytest.raises(ValueError, match="CUDA"):
        d.token_logprobs_grad(x, t, torch.zeros(2, 3), torch.zeros(2, 3))


def _reach(t, split):
    """Element offsets of a tensor's rows from its outer and inner strides."""
    outer, inner, strides = split
    a, b = strides[t]
    return [i * a + j * b for i in range(outer) for j in range(inner)]


@pytest.mark.parametrize("make", [
    lambda x: x, lambda x: x[:, :-1], lambda x: x[1:], lambda x: x[:, 1:3], lambda x: x[::2], lambda x: x[:, ::2], lambda x: x[0],
    lambda x: x[:1], lambda x: x[:, :1], lambda x: x[0, 0], lambda x: x.transpose(0, 1), lambda x: x[:0], lambda x: x.unsqueeze(1),
    lambda x: x.unsqueeze(0), lambda x: x.expand(2, 4, 5, 6), lambda x: x.view(2, 2, 5, 6)])
def test_two_strides_reach_every_row(make):
    x = make(torch.arange(4 * 5 * 6).view(4, 5, 6))
    lead = tuple(x.shape[:-1])
    split = module._split(lead, [x, torch.zeros(x.shape)])
    assert split is not None
    want = (x[..., 0] - x.storage_offset() * (x.numel() > 0)).reshape(-1).tolist() if x.numel() else []
    assert _reach(0, split) == want


def test_three_strides_are_more_than_two():
    x = torch.arange(4 * 5 * 4 * 6).view(4, 5, 4, 6)[:, ::2, ::2]
    assert module._split(tuple(x.shape[:-1]), [x]) is None


@pytest.mark.parametrize("outer, inner, strides, overlap", [
    (2, 3, (24, 8), False), (2, 3, (8, 16), False), (3, 2, (8, 24), False), (2, 3, (-24, -8), False), (1, 3, (0, 8), False), (2, 1, (8, 0), False),
    (1, 1, (0, 0), False), (2, 3, (0, 8), True), (2, 3, (24, 0), True), (2, 3, (24, 7), True), (2, 3, (23, 8), True), (2, 3, (8, 15), True),
    (2, 3, (8, 8), True), (1, 3, (100, 4), True), (2, 1, (7, 100), True), (2, 3, (-24, -7), True)])
def test_written_rows_that_overlap_are_refused(outer, inner, strides, overlap):
    reached = sorted(i * strides[0] + j * strides[1] for i in range(outer) for j in range(inner))
    assert overlap == any(b - a < 8 for a, b in zip(reached, reached[1:]))
    if overlap:     # (what is not refused would run)
        with pytest.raises(d.DeslocError) as e:
            _grad(outer=outer, inner=inner, out=B.rows(1 << 20, d.DESLOC_F32, *strides))()
        assert e.value.status == d.DESLOC_E_INVALID


def test_the_device_of_bound_gradients():
    rows = [[torch.zeros(3), torch.zeros(2)] for _ in range(2)]
    assert module.BoundGrads((ctypes.c_void_p * 4)(), rows).device() == -1


def _engine(M, numel, grad_dtype, index=0):
    eng = d.DesLoc.__new__(d.DesLoc)                       # no context: marshalling only
    eng.ctx, eng.M, eng.numel, eng.grad_dtype, eng._index = None, M, numel, grad_dtype, index
    eng._tables()
    return eng


@pytest.mark.parametrize("M, numel, kind", [(2, [4, 6], d.DESLOC_BF16), (2, [4, 5], d.DESLOC_F32), (2, [6, 4], d.DESLOC_F32), (1, [4, 6, 4, 6], d.DESLOC_F32),
                                            (4, [10], d.DESLOC_F32), (1, [4, 6], d.DESLOC_F32), (3, [4, 6], d.DESLOC_F32)])
def test_gradients_bound_for_other_tensors_are_refused(M, numel, kind):
    """A handle stands for what it was checked as: workers, sizes and type."""
    eng, other = _engine(2, [4, 6], d.DESLOC_F32), _engine(M, numel, kind)
    dtype = torch.bfloat16 if kind == d.DESLOC_BF16 else torch.float32
    bound = other.bind_grads([[torch.zeros(n, dtype=dtype) for n in numel] for _ in range(M)])
    bound._device = eng._index                             # (as if it lay on the device)
    assert other._bound(bound) == other._grad_address(bound) == bound.address
    for call in (eng._bound, eng._grad_address, lambda b: eng._list_of(eng._table, b), eng.bind_grads):
        with pytest.raises(ValueError, match="gradient tensor"):
            call(bound)


def test_gradients_bound_for_equal_tensors_are_taken():
    eng, other = _engine(2, [4, 6], d.DESLOC_F32), _engine(2, [4, 6], d.DESLOC_F32)
    bound = other.bind_grads([[torch.zeros(4), torch.zeros(6)] for _ in range(2)])
    bound._device = eng._index
    assert eng._bound(bound) == eng._grad_address(bound) == bound.address and eng.bind_grads(bound) is bound
    eng.M = 3                                              # other workers from here on
    eng._tables()
    with pytest.raises(ValueError, match="gradient tensor"):
        eng._grad_address(bound)


def test_a_handle_keeps_the_tensors_that_it_was_made_from():
    """Whatever becomes of the lists: a generator is used up, a list may hold another tensor later."""
    import gc
    import weakref
    eng = _engine(2, [4, 6], d.DESLOC_F32)
    lists = [[torch.zeros(4), torch.zeros(6)] for _ in range(2)]
    seen = [weakref.ref(t) for row in lists for t in row]
    for given in (lists, (row for row in [list(row) for row in lists])):
        bound = eng.bind_grads(given)
    assert [t.data_ptr() for row in bound._keep for t in row] == list(bound.array) == [r().data_ptr() for r in seen]
    lists[0][1] = torch.zeros(6)
    del lists[1], given
    gc.collect()
    assert all(r() is not None for r in seen)
    eng.bind_grads([[torch.zeros(4), torch.zeros(6)] for _ in range(2)])
    assert [t.data_ptr() for row in bound._keep for t in row] == list(bound.array)


def _shares(numel, grads_size, grads, out_size, out):
    """Byte for byte."""
    nt, spans = len(numel), []
    for i, (a, b) in enumerate(zip(grads, out)):
        spans.append((set(range(a, a + grads_size * numel[i % nt])), set(range(b, b + out_size * numel[i % nt]))))
    for i, (_, w) in enumerate(spans):
        for j, (r, v) in enumerate(spans):
            if i != j and w & (r | v):
                return True
        if w & spans[i][0] and (grads[i] != out[i] or grads_size != out_size):
            return True
    return False


@pytest.mark.parametrize("M, numel, grads, out, types, shares", [
    (3, [4], [100, 200, 300], [100, 200, 300], (0, 0), False),              # in place
    (3, [4], [100, 200, 100], [100, 200, 100], (0, 0), True),               # the first and the third worker the same
    (3, [4], [100, 100, 100], [200, 300, 400], (0, 0), False),              # read by all of them
    (3, [4], [100, 200, 300], [400, 500, 400], (0, 0), True),
    (2, [4, 4], [100, 100, 200, 216], [100, 100, 200, 216], (0, 0), True),  # a tensor listed twice
    (2, [4, 4], [100, 116, 200, 216], [116, 100, 200, 216], (0, 0), True),  # two tensors for one another
    (2, [4, 4], [100, 116, 200, 216], [300, 316, 400, 412], (0, 0), True),  # four bytes of each
    (2, [4, 4], [100, 116, 200, 216], [300, 316, 400, 416], (0, 0), False),
    (2, [4], [100, 200], [100, 200], (0, 1), True),                         # in place, another type
    (2, [4], [100, 200], [116, 216], (0, 1), False),
    (2, [4], [100, 200], [112, 216], (0, 1), True),
    (2, [4], [100, 200], [200, 100], (0, 0), True),                         # the workers' for one another
    (2, [4], [100, 200], [300, 200], (0, 0), False),                        # one of them in place
    (2, [8], [100, 200], [104, 300], (0, 0), True),                         # its own, shifted
    (2, [8], [100, 200], [92, 300], (0, 0), True),
])
def test_lists_that_share_memory(M, numel, grads, out, types, shares):
    size = [2 if t == d.DESLOC_BF16 else 4 for t in types]
    assert _shares(numel, size[0], grads, size[1], out) == shares
    assert B.desloc_testing_clip_shares(numel, M, types[0], grads, types[1], out) == shares


def test_lists_that_share_memory_or_nearly_do():
    import random
    rng, seen = random.Random(5), [0, 0]
    for _ in range(4000):
        M, numel, types = rng.randint(1, 4), [rng.randint(1, 6) for _ in range(rng.randint(1, 4))], (rng.randint(0, 1), rng.randint(0, 1))
        size = [2 if t == d.DESLOC_BF16 else 4 for t in types]
        n, room = M * len(numel), rng.choice([200, 1000, 4000])
        lists = []
        for k in range(2):
            at, flat = 4096 + 4 * rng.randint(0, room // 4), []
            for i in range(n):
                flat.append(at if rng.random() < 0.7 else 4096 + 4 * rng.randint(0, room // 4))
                at = flat[-1] + size[k] * numel[i % len(numel)] + 2 * rng.randint(0, 3)
            lists.append(flat)
        if rng.random() < 0.4:
            lists[1] = [a if rng.random() < 0.9 else b for a, b in zip(*lists)]
        want = _shares(numel, size[0], lists[0], size[1], lists[1])
        seen[want] += 1
        assert B.desloc_testing_clip_shares(numel, M, types[0], lists[0], types[1], lists[1]) == want
    assert min(seen) > 300


@pytest.mark.parametrize("top", [-1, -(1 << 40), d.DESLOC_MAX_TOP + 1, 1 << 40])
def test_a_number_of_alternatives_out_of_range_is_the_librarys_refusal(top):
    """Before anything is allocated for it."""
    for shape in ((2, 3), (2, 2, 2, 2)):
        with pytest.raises(d.DeslocError) as e:
            d.token_logprobs(torch.zeros(*shape, 8), torch.zeros(shape, dtype=torch.int64), top=top)
        assert e.value.status == d.DESLOC_E_RANGE
