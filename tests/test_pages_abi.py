"""Refusals of the shared-cache entry points (prompt attention, append, fork, compact): bad arguments end
in SD2_EINVAL with a reason before any device work, and no call falls back to anything else."""
import ctypes

import pytest
import torch

from paper_2511_09844_gb300 import build, sd2

P = ctypes.c_void_p(1 << 20)          # stand-in addresses: every call fails a host check before using them
Q = ctypes.c_void_p(1 << 21)
U = ctypes.c_void_p((1 << 20) + 4)


@pytest.fixture(scope="module")
def L():
    build.build()
    return sd2.load_library()


def refused(L, st, word):
    return st == sd2.SD2_EINVAL and word in L.sd2_last_error(None)


def test_prompt_attention_refuses(L):
    assert L.sd2_attention_prompt_workspace_bytes(0, 1, 8, 2, 64, 10) == 0
    assert L.sd2_attention_prompt_workspace_bytes(5, 1, 8, 3, 64, 10) == 0
    need = L.sd2_attention_prompt_workspace_bytes(7, 2, 32, 8, 128, 65536)
    assert need > 0 and need % 256 == 0

    def call(q=P, ldq=4096, M=7, H=32, Hkv=8, hd=128, pool=P, nb=64, table=P, stride=8, layer=0, cu=P, kv=P, n_seq=2,
             max_kv=65536, out=P, work=P, nbytes=need):
        return L.sd2_attention_prompt(q, ldq, M, H, Hkv, hd, pool, nb, table, stride, layer, cu, kv, n_seq, max_kv, out, None,
                                      work, nbytes, None, None)
    for name in ("q", "pool", "table", "cu", "kv", "out", "work"):
        assert refused(L, call(**{name: None}), b"null"), name
    for kw in (dict(hd=96), dict(H=30), dict(H=129 * 8, ldq=129 * 8 * 128), dict(Hkv=0), dict(M=-1)):
        assert refused(L, call(**kw), b"bad attention shape"), kw
    for kw in (dict(nb=0), dict(stride=0), dict(n_seq=0), dict(layer=-1), dict(max_kv=0), dict(stride=(1 << 26) + 1)):
        assert refused(L, call(**kw), b"need n_blocks"), kw
    assert refused(L, call(nb=1 << 28), b"31 bits")
    for kw in (dict(ldq=4088), dict(ldq=4100), dict(q=U), dict(pool=U), dict(out=U)):
        assert refused(L, call(**kw), b"16-byte"), kw
    assert refused(L, call(nbytes=need - 1), b"workspace too small")
    assert refused(L, call(work=U), b"256-byte")
    assert call(M=0) == sd2.SD2_OK


def test_append_refuses(L):
    def call(k=P, ldk=1024, v=P, ldv=1024, dtype=sd2.DTYPE_BF16, M=7, Hkv=8, hd=128, pool=P, nb=64, table=P, stride=8,
             layer=0, cu=P, kv=P, n_seq=2):
        return L.sd2_pages_append(k, ldk, v, ldv, dtype, M, Hkv, hd, pool, nb, table, stride, layer, cu, kv, n_seq, None, None)
    for name in ("k", "v", "pool", "table", "cu", "kv"):
        assert refused(L, call(**{name: None}), b"null"), name
    assert refused(L, call(dtype=2), b"dtype")
    for kw in (dict(M=-1), dict(stride=0), dict(n_seq=0), dict(layer=-1)):
        assert refused(L, call(**kw), b"need M"), kw
    for kw in (dict(nb=0), dict(Hkv=0), dict(hd=12), dict(hd=0)):
        assert refused(L, call(**kw), b"need L"), kw
    assert refused(L, call(pool=U), b"pool not 16-byte")
    for kw in (dict(ldk=1016), dict(ldv=1028), dict(k=U), dict(v=U)):
        assert refused(L, call(**kw), b"rows of k and v"), kw
    assert call(M=0) == sd2.SD2_OK


def test_fork_refuses(L):
    assert L.sd2_pages_fork_workspace_bytes(0, 9) == 0 and L.sd2_pages_fork_workspace_bytes(9, 0) == 0
    need = L.sd2_pages_fork_workspace_bytes(4, 64)
    assert need % 256 == 0 and need >= 4 * 16 + 64 * 12

    def call(pool=P, layers=2, nb=64, Hkv=8, hd=128, table=P, stride=8, ln=P, n_seq=2, parent=P, n_out=4, t2=Q, l2=Q, p2=Q,
             r2=Q, work=P, nbytes=need, pinned=None):
        return L.sd2_pages_fork(pool, layers, nb, Hkv, hd, table, stride, ln, n_seq, parent, None, None, pinned, n_out, t2, l2,
                                p2, r2, work, nbytes, None, None)
    for name in ("pool", "table", "ln", "parent", "t2", "l2", "p2", "r2", "work"):
        assert refused(L, call(**{name: None}), b"null"), name
    for kw in (dict(layers=0), dict(nb=0), dict(hd=4)):
        assert refused(L, call(**kw), b"need L"), kw
    assert refused(L, call(layers=1 << 30), b"page too large")
    for kw in (dict(n_seq=0), dict(n_out=0), dict(stride=0)):
        assert refused(L, call(**kw), b"need n_seq"), kw
    for kw in (dict(t2=P), dict(l2=P), dict(pinned=Q)):
        assert refused(L, call(**kw), b"outputs must not"), kw
    assert refused(L, call(nbytes=need - 1), b"workspace too small")
    assert refused(L, call(work=U), b"256-byte")


def test_compact_refuses(L):
    assert L.sd2_pages_compact_workspace_bytes(0) == 0
    need = L.sd2_pages_compact_workspace_bytes(64)
    assert need % 256 == 0 and need >= 64 * 12

    def call(pool=P, layers=2, nb=64, Hkv=8, hd=128, table=P, stride=8, pages=P, n_seq=2, ref=P, t2=Q, r2=Q, m2=Q, n2=Q,
             work=P, nbytes=need):
        return L.sd2_pages_compact(pool, layers, nb, Hkv, hd, table, stride, pages, n_seq, ref, t2, r2, m2, n2, work, nbytes,
                                   None, None)
    for name in ("pool", "table", "pages", "ref", "t2", "r2", "m2", "n2", "work"):
        assert refused(L, call(**{name: None}), b"null"), name
    assert refused(L, call(layers=0), b"need L")
    for kw in (dict(n_seq=0), dict(stride=0)):
        assert refused(L, call(**kw), b"need n_seq"), kw
    assert refused(L, call(r2=P), b"outputs must not")
    assert refused(L, call(nbytes=need - 1), b"workspace too small")
    assert refused(L, call(work=U), b"256-byte")


def test_binding_refuses_other_tensors(L):
    """Tensors the C ABI cannot judge: host memory is refused, not computed some other way."""
    pool = torch.zeros(1, 4, 2, 2, 16, 64, dtype=torch.bfloat16)
    i = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    kv = torch.zeros(3, 2, 64)
    table = torch.zeros(1, 2, dtype=torch.int32)
    for call in (lambda: sd2.attention_prompt(q, pool, table, 0, i(0, 3), i(3)),
                 lambda: sd2.pages_append(kv, kv, pool, table, 0, i(0, 3), i(3)),
                 lambda: sd2.pages_fork(pool, table, i(3), i(0)),
                 lambda: sd2.pages_compact(pool, table, i(1), i(1, 0, 0, 0))):
        with pytest.raises(sd2.SD2Error, match="EINVAL.*pool must be"):
            call()


def test_fork_refuses_tables_beyond_31_bits(L):
    need = L.sd2_pages_fork_workspace_bytes(1 << 16, 64)

    def call(n_out, stride):
        return L.sd2_pages_fork(P, 2, 64, 8, 128, P, stride, P, 2, P, None, None, None, n_out, Q, Q, Q, Q, U, need, None, None)
    assert refused(L, call(1 << 16, 1 << 15), b"n_out * bt_stride")
    assert refused(L, call(1 << 16, (1 << 15) - 1), b"256-byte")
    assert refused(L, call(1, (1 << 26) + 1), b"bt_stride <= 2^26")


class _Recorded(torch.Tensor):
    """A tensor that notes the streams it is said to be used on."""

    def record_stream(self, stream):
        self.__dict__.setdefault("streams", []).append(stream)


def _host_calls(monkeypatch, current):
    """The four calls of the binding on host tensors and a library that does nothing: (calls by name, the stream that was
    current at each allocation, the handles that the library got). `current` is a one-element list, the current stream."""
    made, handles = [], []

    class Lib:
        def __getattr__(self, name):
            if name.endswith("workspace_bytes"):
                return lambda *a: 4096
            return lambda *a: handles.append(a[-1]) or 0

    class Use:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            self.before, current[0] = current[0], self.stream

        def __exit__(self, *a):
            current[0] = self.before

    def empty(*a, **kw):
        made.append(current[0])
        return host_empty(*a, **kw).as_subclass(_Recorded)

    host_empty = torch.empty
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "stream", Use)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current[0])
    monkeypatch.setattr(sd2, "_raw_stream", None)
    monkeypatch.setattr(sd2, "load_library", lambda: Lib())
    monkeypatch.setattr(sd2, "_pool_shape", lambda pool: (1, 4, 2, 64, -1))
    monkeypatch.setattr(sd2, "_prompt_workspace_bytes", lambda *a: 4096)
    i = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    pool = torch.zeros(1, 4, 2, 2, 16, 64, dtype=torch.bfloat16)
    table, kv = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(3, 2, 64)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    calls = {"attention": lambda **kw: sd2.attention_prompt(q, pool, table, 0, i(0, 3), i(3), return_lse=True, **kw),
             "append": lambda **kw: sd2.pages_append(kv, kv, pool, table, 0, i(0, 3), i(3), **kw),
             "fork": lambda **kw: sd2.pages_fork(pool, table, i(3), i(0), **kw),
             "compact": lambda **kw: sd2.pages_compact(pool, table, i(1), i(1, 0, 0, 0), **kw)}
    return calls, made, handles


class _Stream:
    device = None

    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.mark.parametrize("name,n_out,n_made", [("attention", 2, 3), ("append", 0, 0), ("fork", 4, 5), ("compact", 4, 5)])
def test_memory_comes_from_the_stream_that_uses_it(monkeypatch, name, n_out, n_made):
    """What a call allocates for work on a given stream is that stream's memory: a block of the caller's stream may
    still be written by work that is pending there. The outputs are noted as used on the caller's stream."""
    caller, side = _Stream(3), _Stream(7)
    current = [caller]
    calls, made, handles = _host_calls(monkeypatch, current)
    out = calls[name](stream=side)
    assert handles == [7] and made == [side] * n_made and current == [caller]
    outs = list(out) if out is not None else []
    assert len(outs) == n_out and all(t.streams == [caller] for t in outs)
    del made[:], handles[:]
    calls[name]()
    assert handles == [3] and made == [caller] * n_made


def test_a_given_workspace_is_kept_for_its_stream(monkeypatch):
    caller, side = _Stream(3), _Stream(7)
    calls, made, handles = _host_calls(monkeypatch, [caller])
    ws = torch.zeros(4096, dtype=torch.uint8).as_subclass(_Recorded)
    calls["fork"](stream=side, workspace=ws)
    assert len(made) == 4 and ws.streams == [side]


def test_binding_refuses_a_pool_on_another_device(monkeypatch):
    """The library launches on the current device: tensors of another one are refused."""
    class Pool:
        is_cuda, dtype, shape, device = True, torch.bfloat16, (1, 4, 2, 2, 16, 64), torch.device("cuda", 1)

        def is_contiguous(self):
            return True

        def get_device(self):
            return 1

        def data_ptr(self):
            return 1 << 20

    i = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    q, kv, table = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64), torch.zeros(1, 2, dtype=torch.int32)
    pool = Pool()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for call in (lambda: sd2.attention_prompt(q, pool, table, 0, i(0, 3), i(3)),
                 lambda: sd2.pages_append(kv, kv, pool, table, 0, i(0, 3), i(3)),
                 lambda: sd2.pages_fork(pool, table, i(3), i(0)),
                 lambda: sd2.pages_compact(pool, table, i(1), i(1, 0, 0, 0))):
        with pytest.raises(sd2.SD2Error, match="EINVAL.*current device"):
            call()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    assert sd2._pool_shape(pool) == (1, 4, 2, 64, 1)
