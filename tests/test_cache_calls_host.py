"""What the cache and log-probability calls promise and refuse beyond single bad
arguments: workspaces kept for many calls, types of tensors, host lists, buffers
that share memory.  Nothing reaches a GPU; addresses are made up and every check
fails first."""

import ctypes as C

import pytest
import torch

import paper_2608_01821_amd as dv

EINVAL, ESHAPE, EDTYPE, ENOMEM = -1, -2, -3, -4
A = 1 << 20                                    # an aligned made-up address


@pytest.mark.parametrize("top", [0, 1, 5, 64])
@pytest.mark.parametrize("vocab", [1000, 16384, 32003, 126464, 1 << 24])
def test_a_log_probability_workspace_for_every_count_of_rows(vocab, top):
    """The header's bound for up to N rows, though fewer rows may need more."""
    most = 0
    for rows in range(1, 600):
        most = max(most, dv.davet_logprobs_workspace_bytes(rows, vocab, top))
        assert most <= (min(rows, 255) + 255) * (8 * top + 12)
    assert dv.davet_logprobs_workspace_bytes(1 << 22, vocab, top) <= most


def test_fewer_rows_than_the_workspace_was_asked_for():
    """255 rows are refused with what 256 need, which is nothing."""
    def f(rows, nb):
        return dv.raw().davet_token_logprobs(
            rows, 126464, A, dv.DAVET_F32, 126464, -1, A, A, None, 5, A, A, A, nb,
            None)
    assert dv.davet_logprobs_workspace_bytes(256, 126464, 5) == 0
    need = dv.davet_logprobs_workspace_bytes(255, 126464, 5)
    assert f(255, need - 1) == ENOMEM
    assert "%d bytes" % need in dv.raw().davet_last_error().decode()


# ------------------------------------------------------------- types of tensors --

K16 = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
TABLE = torch.zeros(2, 3, dtype=torch.int32)
Q16 = torch.zeros(3, 256, dtype=torch.float16)
F = torch.zeros(3, 256)
I = torch.zeros(3, 256, dtype=torch.int32)
CHUNK = ([0, 3], [3])


def _wrong_types():
    c = dv.KvCache(K16, K16, TABLE, dv.DAVET_F16)
    qkv = torch.zeros(3, 512, dtype=torch.float16)
    b = torch.bfloat16

    def append(x=qkv, q=Q16, **kw):
        return lambda: dv.davet_cache_append(c, *CHUNK, x, 4, q, **kw)

    def attend(q=Q16, out=Q16, **kw):
        return lambda: dv.davet_cache_attention(c, *CHUNK, q, 4, out, **kw)

    def weigh(q=Q16, lse=F, w=F, **kw):
        return lambda: dv.davet_cache_weights(c, *CHUNK, q, 4, lse, w, **kw)

    def select(w=F, kept=I, **kw):
        return lambda: dv.davet_evict_select([5], [2], w, kept, **kw)

    def score(x=F, dt=dv.DAVET_F32, **kw):
        return lambda: dv.davet_token_logprobs(x, dt, **kw)
    return [
        lambda: dv.KvCache(K16.to(b), K16, TABLE, dv.DAVET_F16),
        lambda: dv.KvCache(K16, K16.to(b), TABLE, dv.DAVET_F16),
        lambda: dv.KvCache(K16, K16, TABLE, dv.DAVET_BF16),
        lambda: dv.KvCache(K16, K16, TABLE.float(), dv.DAVET_F16),
        append(qkv.to(b)), append(q=Q16.to(b)), append(pos=F), append(q_gain=I),
        append(k_gain=I),
        attend(Q16.to(b)), attend(out=Q16.to(b)), attend(lse=I),
        weigh(Q16.to(b)), weigh(lse=I), weigh(w=I), weigh(prev=I),
        select(I), select(kept=F), select(weights_out=I),
        lambda: dv.davet_cache_gather(c, F, [2], TABLE),
        lambda: dv.davet_cache_gather(c, I, [2], TABLE.float()),
        score(I), score(Q16, dv.DAVET_BF16), score(targets=F, logp=F),
        score(targets=I, logp=I), score(entropy=I),
        score(top_logp=I, top_ids=I), score(top_logp=F, top_ids=F),
    ]


@pytest.mark.parametrize("i", range(28))
def test_a_tensor_of_another_type_of_the_same_width_is_refused(i):
    calls = _wrong_types()
    assert len(calls) == 28
    with pytest.raises(ValueError, match="is of torch"):
        calls[i]()


def test_sixteen_bits_may_come_as_bit_patterns():
    """As elsewhere in the binding; these get as far as the check of the device."""
    bits = K16.view(torch.int16)
    for dt in (dv.DAVET_F16, dv.DAVET_BF16):
        c = dv.KvCache(bits, bits, TABLE, dt)
        with pytest.raises(ValueError, match="on a GPU"):
            dv.davet_cache_attention(c, *CHUNK, Q16.view(torch.int16), 4,
                                     Q16.view(torch.int16))
    with pytest.raises(dv.DavetError) as e:
        dv.KvCache(K16, K16, TABLE, 7)
    assert e.value.status == EDTYPE


# ----------------------------------------------------------------- host lists --

@pytest.mark.parametrize("bad", [2 ** 32 + 3, 2 ** 31, -2 ** 31 - 1, -2 ** 32 + 3,
                                 3.0, None])
@pytest.mark.parametrize("n", [1, 2, 64, 65, 100])
def test_lengths_beyond_32_bits_are_refused(bad, n):
    """Not taken modulo 2^32, whatever the list's length."""
    with pytest.raises(ValueError, match="32-bit"):
        dv._lib._ints([3] * (n - 1) + [bad])
    if n <= 64:
        table = TABLE[:1].expand(n, 3).contiguous()
        c = dv.KvCache(K16, K16, table, dv.DAVET_F16)
        with pytest.raises(ValueError, match="32-bit"):
            dv.davet_cache_attention(c, [0] * n + [3], [3] * (n - 1) + [bad], Q16, 4,
                                     Q16)


def test_lists_reach_the_library_whole():
    for vals in ([], [5], list(range(-3, 62)), list(range(100))):
        got = dv._lib._ints(vals)
        assert isinstance(got, C.Array) and list(got) == vals
        assert dv._lib._ints(got) is got


def test_sizes_of_tensors_beyond_32_bits_are_refused():
    """Not taken modulo 2^32: a vocabulary of 2^32 + 3 is not one of 3."""
    big, f16, i = 2 ** 32 + 3, torch.float16, torch.int32

    def of(*shape, dtype=f16):
        return torch.empty(shape, dtype=dtype, device="meta")
    c = dv.KvCache(K16, K16, TABLE, dv.DAVET_F16)
    k, one = of(4, 2, 16, 64), torch.zeros(2, dtype=i)
    s, turns = of(3, 2, dtype=torch.float32), of(1, dtype=torch.float64)
    ids, h = of(3, 2, dtype=i), dv.DAVET_F16
    for call in (
            lambda: dv.KvCache(k, k, of(1, big, dtype=i), h),
            lambda: dv.KvCache(of(big, 2, 16, 64), None, of(1, 4, dtype=i), h),
            lambda: dv.davet_token_logprobs(of(1, big), h),
            lambda: dv.davet_token_logprobs(of(big, 1), h),
            lambda: dv.davet_token_logprobs(of(1, 9), h, top_ids=of(1, big, dtype=i),
                                            top_logp=of(1, big, dtype=torch.float32)),
            lambda: dv.davet_cache_gather(c, I, [2], of(1, big, dtype=i)),
            lambda: dv.davet_cache_reorder(c, [1, 1], one, one, of(2, big, dtype=i)),
            lambda: dv.davet_cache_page_select(c, *CHUNK, Q16, 4,
                                               torch.zeros(4, 2, 2, 64, dtype=f16),
                                               of(3, 2, big, dtype=i)),
            lambda: dv.davet_cache_page_attention(c, *CHUNK, Q16, 4,
                                                  of(3, 2, big, dtype=i), Q16),
            lambda: dv.davet_beam_select(of(3, big), h, s, 1, s, ids, ids),
            lambda: dv.davet_beam_select(of(big, 1), h, of(big, dtype=torch.float32), 1,
                                         of(big, 2, dtype=torch.float32),
                                         of(big, 2, dtype=i), of(big, 2, dtype=i)),
            lambda: dv.davet_beam_select(of(3, 9), h, s, 1,
                                         of(3, big, dtype=torch.float32),
                                         of(3, big, dtype=i), of(3, big, dtype=i)),
            lambda: dv.davet_rotary(of(big, 64), 1, 64, turns, of(big, 64), h),
            lambda: dv.davet_rotary(of(3, 64), 1, 64, of(2 ** 31 + 1,
                                                         dtype=torch.float64),
                                    of(3, 64), h)):
        with pytest.raises(ValueError, match="32-bit"):
            call()


@pytest.mark.parametrize("name", [
    "davet_cache_append", "davet_cache_attention", "davet_cache_weights",
    "davet_tree_plan", "davet_cache_tree_attention", "davet_cache_page_bounds",
    "davet_cache_page_select", "davet_cache_page_attention", "davet_cache_reorder",
    "davet_evict_select", "davet_cache_gather"])
def test_raw_calls_take_lists_of_int32_alone(name):
    """An array of other integers would be read as int32, a number as an address."""
    f = getattr(dv.raw(), name)
    lists = [i for i, t in enumerate(f.argtypes) if t is C.POINTER(C.c_int32)]
    assert len(lists) == {"davet_tree_plan": 3, "davet_cache_reorder": 1,
                          "davet_cache_gather": 1}.get(name, 2)
    i32 = (C.c_int32 * 3)(0, 0, 0)
    for at in lists:
        for bad in ((C.c_int64 * 3)(0, 0, 0), (C.c_float * 3)(), A, b"\0" * 12):
            args = [i32 if i in lists else None if t is C.POINTER(dv.KvCacheT) else
                    t(0) for i, t in enumerate(f.argtypes)]
            assert f(*args) < 0                 # no cache, or no sequence
            args[at] = bad
            with pytest.raises(C.ArgumentError):
                f(*args)


def test_streams_by_public_names(monkeypatch):
    """A torch without the short cuts that the binding takes."""
    class Stream:
        cuda_stream = 77
    monkeypatch.delattr(torch._C, "_cuda_getDevice", raising=False)
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev: Stream())
    try:
        dv._lib._load_torch()
        calls = []
        for stream in (None, 5, Stream()):
            dv._lib._launch(3, stream, lambda *a: calls.append(a) or 0, 1, 2)
        assert calls == [(1, 2, 77), (1, 2, 5), (1, 2, 77)]
    finally:
        monkeypatch.undo()
        dv._lib._load_torch()


# ------------------------------------------------------------- memory in common --

def _attend(q, ldq, out, ldo, n=3):
    cache = dv.KvCacheT(A, A << 4, A << 8, 8, 32, 16, 2, 64, dv.DAVET_F16)
    f = dv.raw().davet_cache_attention
    return f(C.byref(cache), 1, (C.c_int32 * 2)(0, n), (C.c_int32 * 1)(10), q, ldq, 4,
             0.0, 0, out, ldo, None, A << 3, 1 << 30, None)


def test_rows_that_share_memory_are_refused():
    """Of 256 fp16 elements (512 bytes) each: columns that meet, rows that run into
    the next ones, strides that differ."""
    x = A << 1
    for d in (0, 256, 496, 528 - 1024, -496, 1024, 1024 + 16, 1024 * 2 - 16, 528):
        assert _attend(x, 512, x + d, 512) == EINVAL, d     # 1024-byte rows
    assert _attend(x, 512, x + 512, 520) == EINVAL          # drift into each other
    assert _attend(x, 256, x + 512, 256) == EINVAL          # one row on
    assert _attend(x, 256, x + 256, 256, n=1) == EINVAL
    # what stays of weights beside them, too wide by one
    i = lambda *v: (C.c_int32 * len(v))(*v)
    for d in (0, 9, 27, 30):
        assert dv.raw().davet_evict_select(2, i(10, 8), i(4, 3), A, 30, 0, 0, A << 1,
                                           8, A + 4 * d, 30, None) == EINVAL, d


def test_arrays_are_aligned_to_their_elements():
    """Every float32 and int32 argument, off by two bytes."""
    L, cache = dv.raw(), dv.KvCacheT(A, A << 4, A << 8, 8, 32, 16, 2, 64, dv.DAVET_F16)
    c, i = C.byref(cache), lambda *v: (C.c_int32 * len(v))(*v)
    cu, kv = i(0, 3), i(10)

    def attend(lse):
        return L.davet_cache_attention(c, 1, cu, kv, A << 1, 256, 4, 0.0, 0, A << 2,
                                       256, lse, A << 3, 1 << 30, None)

    def weigh(lse=A, prev=A, w=A):
        return L.davet_cache_weights(c, 1, cu, kv, A << 1, 256, 4, 0.0, 0, lse, prev,
                                     w, 16, A << 3, 1 << 30, None)

    def select(w=A, kept=A << 1, out=A << 2):
        return L.davet_evict_select(1, i(10), i(4), w, 16, 0, 0, kept, 8, out, 8, None)

    def gather(kept=A, dst=A):
        return L.davet_cache_gather(c, 1, i(4), kept, 8, dst, 2, None)

    def score(tgt=A, lp=A, en=A, tl=A, ti=A):
        return L.davet_token_logprobs(2, 100, A, dv.DAVET_F16, 100, -1, tgt, lp, en, 2,
                                      tl, ti, None, 0, None)
    b = A + 2
    for call in (lambda: attend(b), lambda: weigh(lse=b), lambda: weigh(prev=b),
                 lambda: weigh(w=b), lambda: select(w=b), lambda: select(kept=b),
                 lambda: select(out=b), lambda: gather(kept=b), lambda: gather(dst=b),
                 lambda: score(tgt=b), lambda: score(lp=b), lambda: score(en=b),
                 lambda: score(tl=b), lambda: score(ti=b)):
        assert call() == EINVAL
        assert "4-byte aligned" in L.davet_last_error().decode()


def test_selection_of_nothing_and_strides_past_any_memory():
    """Nothing kept shares no memory with the weights; a stride whose last row's
    address would not fit 64 bits is refused before it is computed."""
    i = lambda *v: (C.c_int32 * len(v))(*v)

    def select(keep, ldw=16, ldk=8, ldo=16):
        return dv.raw().davet_evict_select(2, i(10, 10), i(keep, keep), A, ldw, 0, 0,
                                           A << 1, ldk, A, ldo, None)
    assert select(0) == 0
    assert select(4) == EINVAL
    for kw in (dict(ldw=2 ** 62), dict(ldk=2 ** 62), dict(ldo=2 ** 62),
               dict(ldw=2 ** 62, ldo=2 ** 62), dict(ldw=2 ** 40)):
        assert select(4, **kw) == ESHAPE, kw


@pytest.mark.parametrize("bad", [2 ** 32, 2 ** 32 + 1, -2 ** 32, 2 ** 31])
def test_integers_beyond_32_bits_are_refused(bad):
    """exclude 2^32 is not token 0, block 2^32 not the bidirectional mask."""
    c = dv.KvCache(K16, K16, TABLE, dv.DAVET_F16)
    qkv = torch.zeros(3, 512, dtype=torch.float16)
    for call in (
            lambda: dv.davet_cache_append(c, *CHUNK, qkv, bad + 4, Q16),
            lambda: dv.davet_cache_attention(c, *CHUNK, Q16, bad + 4, Q16),
            lambda: dv.davet_cache_weights(c, *CHUNK, Q16, bad + 4, F, F),
            lambda: dv.davet_cache_attention(c, *CHUNK, Q16, 4, Q16, block=bad),
            lambda: dv.davet_cache_weights(c, *CHUNK, Q16, 4, F, F, block=bad),
            lambda: dv.davet_evict_select([5], [2], F, I, first=bad),
            lambda: dv.davet_evict_select([5], [2], F, I, last=bad),
            lambda: dv.davet_token_logprobs(F, dv.DAVET_F32, exclude=bad),
            lambda: dv.davet_cache_workspace_bytes(4, 64, bad),
            lambda: dv.davet_cache_workspace_bytes(bad + 4, 64, 1),
            lambda: dv.davet_logprobs_workspace_bytes(bad + 2, 50000, 5),
            lambda: dv.davet_logprobs_workspace_bytes(2, bad + 50000, 5)):
        with pytest.raises(ValueError, match="32-bit"):
            call()
