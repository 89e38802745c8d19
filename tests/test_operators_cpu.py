"""Refusals of the operators around the linear layers: every argument is checked before any HIP call, the
same with and without a GPU.  (A call whose only fault is the missing context ends with -1.)"""
import numpy as np
import pytest

import paper_2602_05754_amd as tf

A = 1 << 20          # fake, aligned "device pointers", 1 MB apart: never dereferenced
INVALID, SHAPE, DTYPE, ALIGN, WORKSPACE, ALIAS = -1, -2, -3, -4, -5, -8
F32, BF16 = tf.TF_F32, tf.TF_BF16


def code(fn, *a, **k):
    try:
        fn(*a, **k)
    except tf.TfError as e:
        return e.code
    return 0


def caller(fn, names, defaults):
    def call(**kw):
        assert not set(kw) - set(names), kw
        return code(fn, None, *[kw.get(n, d) for n, d in zip(names, defaults)], **{"workspace": kw["workspace"]} if "workspace" in kw and "workspace" not in names else {})
    return call


def test_norm_forward_refusals():
    names = "T d io x weight bias eps center y mean rstd".split()
    call = caller(tf.tf_norm_forward, names, [8, 16, F32, A, 2 * A, 3 * A, 1e-5, 1, 4 * A, 5 * A, 6 * A])
    assert call() == INVALID and call(bias=None) == INVALID and call(center=0, mean=None) == INVALID
    for bad in (dict(T=0), dict(T=-1), dict(d=0), dict(d=16385), dict(T=1 << 31)):
        assert call(**bad) == SHAPE
    assert call(io=2) == DTYPE and call(io=-1) == DTYPE
    for bad in (dict(center=2), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(weight=None),
                dict(y=None), dict(mean=None), dict(rstd=None)):
        assert call(**bad) == INVALID
    for n in ("x", "weight", "bias", "y", "mean", "rstd"):
        assert call(**{n: 7 * A + 4}) == ALIGN
    assert call(center=0, mean=7 * A + 4) == INVALID                  # not looked at
    assert call(y=A) == ALIAS and call(y=A + 8 * 16 * 4 - 16) == ALIAS and call(y=A + 8 * 16 * 4) == INVALID
    assert call(rstd=5 * A) == ALIAS and call(y=2 * A) == ALIAS and call(mean=3 * A) == ALIAS
    assert call(x=2 * A) == INVALID                                   # inputs may overlap


def test_norm_backward_refusals():
    names = "T d io x weight dy mean rstd center dx dweight dbias dw accumulate".split()
    base = [8, 16, BF16, A, 2 * A, 3 * A, 4 * A, 5 * A, 1, 6 * A, 7 * A, 8 * A, BF16, False]

    def call(workspace=9 * A, **kw):
        return code(tf.tf_norm_backward, None, *[kw.get(n, d) for n, d in zip(names, base)], workspace=workspace)
    assert call() == INVALID and call(dweight=None) == INVALID and call(dweight=None, dbias=None, workspace=None) == INVALID
    assert call(T=0) == SHAPE and call(d=16385) == SHAPE and call(io=5) == DTYPE and call(dw=5) == DTYPE
    assert call(io=F32) == DTYPE and call(accumulate=True) == DTYPE and call(accumulate=True, dw=F32) == INVALID
    assert call(mean=None) == INVALID and call(mean=None, center=0) == INVALID and call(rstd=None) == INVALID and call(dx=None) == INVALID
    for n in ("x", "weight", "dy", "mean", "rstd", "dx", "dweight", "dbias", "workspace"):
        assert call(**{n: 10 * A + 8}) == ALIGN, n
    assert call(dx=A) == ALIAS and call(dx=3 * A) == ALIAS and call(dweight=8 * A) == ALIAS and call(workspace=A) == ALIAS
    small = np.zeros(1, np.uint8)
    lib = tf.load_library()
    need = tf.tf_norm_workspace(8, 16)
    raw = lambda n: lib.tf_norm_backward(None, None, 8, 16, BF16, A, 2 * A, 3 * A, 4 * A, 5 * A, 1, 6 * A, 7 * A, 8 * A, BF16, 0, 9 * A, n)
    assert raw(need) == INVALID and raw(need - 1) == WORKSPACE and raw(0) == WORKSPACE and raw(-5) == WORKSPACE and small.size
    assert lib.tf_norm_backward(None, None, 8, 16, F32, A, 2 * A, 3 * A, 4 * A, 5 * A, 1, 6 * A, 7 * A, 8 * A, F32, 2, 9 * A, need) == INVALID


def test_embedding_refusals():
    fwd = caller(tf.tf_embedding_forward, "T rows d io ids table scale out".split(), [8, 32, 16, F32, A, 2 * A, 1.0, 3 * A])
    assert fwd() == INVALID
    for bad in (dict(T=0), dict(rows=0), dict(d=0), dict(rows=1 << 31), dict(T=1 << 31), dict(d=(1 << 20) + 1)):
        assert fwd(**bad) == SHAPE
    assert fwd(io=3) == DTYPE and fwd(scale=float("inf")) == INVALID and fwd(scale=float("nan")) == INVALID
    assert fwd(ids=None) == INVALID and fwd(table=None) == INVALID and fwd(out=None) == INVALID
    assert fwd(ids=A + 4) == ALIGN and fwd(table=A + 4) == ALIGN and fwd(out=A + 4) == ALIGN
    assert fwd(out=A) == ALIAS and fwd(out=2 * A + 32 * 16 * 4 - 16) == ALIAS

    names, base = "T rows d io ids dout scale dtable dw accumulate".split(), [8, 32, 16, BF16, A, 2 * A, 1.0, 3 * A, BF16, False]

    def bwd(workspace=4 * A, **kw):
        return code(tf.tf_embedding_backward, None, *[kw.get(n, d) for n, d in zip(names, base)], workspace=workspace)
    assert bwd() == INVALID and bwd(dw=F32, accumulate=True) == INVALID
    assert bwd(rows=-4) == SHAPE and bwd(io=F32) == DTYPE and bwd(accumulate=True) == DTYPE and bwd(dw=9) == DTYPE
    assert bwd(ids=None) == INVALID and bwd(dout=None) == INVALID and bwd(dtable=None) == INVALID and bwd(workspace=None) == INVALID
    assert bwd(dtable=A + 4) == ALIGN and bwd(workspace=A + 8) == ALIGN
    assert bwd(dtable=2 * A) == ALIAS and bwd(workspace=A) == ALIAS and bwd(workspace=3 * A) == ALIAS
    lib = tf.load_library()
    need = tf.tf_embedding_workspace(8, 32, 16)
    raw = lambda n: lib.tf_embedding_backward(None, None, 8, 32, 16, BF16, A, 2 * A, 1.0, 3 * A, BF16, 0, 4 * A, n)
    assert raw(need) == INVALID and raw(need - 1) == WORKSPACE
    for bad in ((0, 5, 5), (5, 0, 5), (5, 5, 0), (5, 5, (1 << 20) + 1)):
        assert code(tf.tf_embedding_workspace, *bad) == SHAPE
    assert code(tf.tf_norm_workspace, 0, 5) == SHAPE and code(tf.tf_norm_workspace, 5, 16385) == SHAPE


def test_distill_refusals():
    names = "T V K io logits ids teacher weight temperature scale loss dlogits".split()
    call = caller(tf.tf_distill_loss, names, [4, 50, 3, F32, A, 2 * A, 3 * A, 4 * A, 1.0, 1.0, 5 * A, 6 * A])
    assert call() == INVALID and call(weight=None) == INVALID and call(dlogits=None) == INVALID
    for bad in (dict(T=0), dict(V=0), dict(K=0), dict(K=1025), dict(V=1 << 31), dict(T=1 << 31)):
        assert call(**bad) == SHAPE
    assert call(io=2) == DTYPE
    for bad in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(scale=float("nan")),
                dict(logits=None), dict(ids=None), dict(teacher=None), dict(loss=None)):
        assert call(**bad) == INVALID
    for n in ("logits", "ids", "teacher", "weight", "loss", "dlogits"):
        assert call(**{n: 7 * A + 4}) == ALIGN
    assert call(dlogits=A) == ALIAS and call(loss=A) == ALIAS and call(loss=6 * A) == ALIAS and call(dlogits=4 * A) == ALIAS


def test_the_wrappers_look_at_their_tensors():
    import torch
    x, w = torch.zeros(8, 16), torch.zeros(16)
    ok = dict(io=F32, x=x, weight=w, y=torch.zeros(8, 16), rstd=torch.zeros(8))

    def norm(**kw):
        a = dict(ok, **kw)
        tf.tf_norm_forward(None, 8, 16, a["io"], a["x"], a["weight"], None, 1e-5, False, a["y"], None, a["rstd"])
    with pytest.raises(tf.TfError):
        norm()                                        # only the missing context
    for bad in (dict(io=BF16), dict(x=x[:7]), dict(x=torch.zeros(16, 8).T), dict(weight=w.double()), dict(rstd=torch.zeros(7)), dict(y=torch.zeros(8, 15))):
        with pytest.raises(ValueError):
            norm(**bad)
    with pytest.raises(ValueError):
        tf.tf_embedding_forward(None, 4, 8, 16, F32, torch.zeros(4, dtype=torch.int64), x, 1.0, torch.zeros(4, 16))
    with pytest.raises(ValueError):
        tf.tf_distill_loss(None, 4, 8, 3, F32, torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 3), None, 1.0, 1.0, torch.zeros(4), None)


def test_attention_refusals():
    """Sizes 10 x (4 heads, 2 of keys and values) x 32, fp32: q, o 5 KB, k, v 2.5 KB."""
    names = "starts T hq hkv d io q k v scale o lse".split()
    base = [[0, 4, 10], 10, 4, 2, 32, F32, A, 2 * A, 3 * A, 0.2, 4 * A, 5 * A]
    call = caller(tf.tf_attention_forward, names, base)
    assert call() == INVALID and call(starts=[0]) == INVALID and call(starts=[0, 0, 10, 10]) == INVALID and call(k=A, v=A) == INVALID
    for bad in (dict(starts=[1, 10]), dict(starts=[0, 11]), dict(starts=[0, 5, 4]), dict(starts=[0, -1]), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(lse=None)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(T=0), dict(T=1 << 31), dict(hq=0), dict(hkv=0), dict(hq=3), dict(hkv=3), dict(hkv=8), dict(d=0), dict(d=8), dict(d=72), dict(d=144),
                dict(T=1 << 30, starts=[0, 1 << 30])):
        assert call(**bad) == SHAPE, bad
    assert call(io=4) == DTYPE
    for n in ("q", "k", "v", "o", "lse"):
        assert call(**{n: 7 * A + 8}) == ALIGN, n
    for bad in (dict(o=A), dict(o=2 * A), dict(o=A + 5120 - 16), dict(lse=3 * A), dict(lse=4 * A)):
        assert call(**bad) == ALIAS, bad
    assert call(o=A + 5120) == INVALID

    lib = tf.load_library()
    st = np.array([0, 10], np.int64)

    def raw(fn="tf_attention_forward", n_seqs=1, starts=st.ctypes.data, q=(A, 128), k=(2 * A, 64), v=(3 * A, 64), o=(4 * A, 128)):
        return lib.tf_attention_forward(None, None, n_seqs, starts, 10, 4, 2, 32, F32, *q, *k, *v, 0.2, *o, 5 * A)
    assert raw() == INVALID and raw(starts=None) == INVALID and raw(n_seqs=-1) == INVALID
    for bad in (dict(q=(A, 127)), dict(k=(2 * A, 63)), dict(q=(A, 0)), dict(o=(4 * A, (1 << 24) + 4)), dict(v=(3 * A, -64))):
        assert raw(**bad) == SHAPE, bad
    assert raw(q=(A, 130)) == ALIGN
    # views of one buffer of 256 columns: beside each other, touching, crossing the row's end
    assert raw(q=(A, 256), o=(A + 128 * 4, 256)) == INVALID and raw(q=(A, 256), o=(A + 127 * 4 - 12, 256)) == ALIAS
    assert raw(q=(A + 128 * 4, 256), o=(A, 256)) == INVALID and raw(q=(A, 256), o=(A + 132 * 4, 256)) == ALIAS
    assert raw(q=(A, 256), o=(A + 256 * 4 * 10, 256)) == INVALID and raw(q=(A, 256), o=(A + 128 * 4, 264)) == ALIAS

    names = "starts T hq hkv d io q k v o lse do scale dq dk dv".split()
    back = [[0, 4, 10], 10, 4, 2, 32, F32, A, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A, 0.2, 7 * A, 8 * A, 9 * A]

    def bwd(workspace=10 * A, **kw):
        return code(tf.tf_attention_backward, None, *[kw.get(n, d) for n, d in zip(names, back)], workspace=workspace)
    assert bwd() == INVALID
    for n in ("q", "k", "v", "o", "lse", "do", "dq", "dk", "dv", "workspace"):
        assert bwd(**{n: None}) == INVALID and bwd(**{n: 11 * A + 4}) == ALIGN, n
    for bad in (dict(dq=A), dict(dk=2 * A), dict(dv=8 * A), dict(dq=6 * A), dict(workspace=5 * A), dict(workspace=9 * A), dict(dk=3 * A)):
        assert bwd(**bad) == ALIAS, bad
    assert bwd(d=20) == SHAPE and bwd(io=9) == DTYPE and bwd(starts=[0, 12]) == INVALID and bwd(scale=0.0) == INVALID
    need = tf.tf_attention_workspace(10, 4, 2, 32, F32)
    full = lambda n: lib.tf_attention_backward(None, None, 1, st.ctypes.data, 10, 4, 2, 32, F32, A, 128, 2 * A, 64, 3 * A, 64, 4 * A, 128, 5 * A, 6 * A, 0.2,
                                               7 * A, 8 * A, 9 * A, 10 * A, n)
    assert full(need) == INVALID and full(need - 1) == WORKSPACE
    assert code(tf.tf_attention_workspace, 0, 4, 2, 32, F32) == SHAPE and code(tf.tf_attention_workspace, 10, 4, 2, 32, 7) == DTYPE


def test_the_attention_wrappers_look_at_their_tensors():
    import torch
    new = lambda *s: torch.zeros(*s)

    def call(**kw):
        a = dict(q=new(10, 4, 32), k=new(10, 2, 32), v=new(10, 64), o=new(10, 128), lse=new(10, 4), **{k: v for k, v in kw.items() if k == "io"})
        a.update(kw)
        tf.tf_attention_forward(None, [0, 10], 10, 4, 2, 32, a.get("io", F32), a["q"], a["k"], a["v"], 0.2, a["o"], a["lse"])
    with pytest.raises(tf.TfError):
        call()
    with pytest.raises(tf.TfError):
        call(q=new(10, 200)[:, 40:168])               # a view of a wider buffer
    for bad in (dict(q=new(9, 4, 32)), dict(q=new(10, 4, 31)), dict(k=new(10, 4, 32)), dict(q=new(4, 10, 32).transpose(0, 1)), dict(lse=new(9, 4)),
                dict(io=BF16), dict(v=new(10, 128)[:, ::2]), dict(q=new(10, 4, 32).double())):
        with pytest.raises(ValueError):
            call(**bad)


@pytest.mark.parametrize("asked,current,want", [(None, 0, 0), (None, 7, 7), (0, 0, 0), (0, 7, 0), (7, 0, 7), (9, 7, 9), ("default", 7, 0), ("side", 0, 5), ("side", 5, 5)])
def test_a_workspace_comes_from_the_pool_of_the_calls_stream(monkeypatch, asked, current, want):
    """Whichever stream is current: torch hands its memory out again in that stream's order."""
    import contextlib
    import types
    import torch
    from paper_2602_05754_amd import binding
    stream = lambda handle: types.SimpleNamespace(cuda_stream=handle)
    now, made, empty = [current], [], torch.empty

    @contextlib.contextmanager
    def inside(s):
        now.append(s.cuda_stream)
        yield
        now.pop()

    def new(*a, device, **k):
        assert device == "cuda:3"
        made.append(now[-1])
        return empty(*a, **k)
    monkeypatch.setattr(torch, "empty", new)
    for name, value in (("current_stream", lambda device=None: stream(now[-1])), ("default_stream", lambda device=None: stream(0)), ("stream", inside),
                        ("ExternalStream", lambda handle, device=None: stream(handle)), ("current_device", lambda: 3)):
        monkeypatch.setattr(torch.cuda, name, value)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: now[-1], raising=False)
    asked = {"default": stream(0), "side": stream(5)}.get(asked, asked) if isinstance(asked, str) else asked
    ctx = types.SimpleNamespace(device_id=3)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 3)
    keep, address, n = binding._workspace(ctx, None, 64, asked)
    assert made == [want] and now == [current] and n == 64 and address == keep.data_ptr()
    assert binding._stream_handle(asked) == (want or None)             # where the kernels go


def test_a_workspace_does_for_all_smaller_calls():
    for d in (1, 64, 1000, 1024, 1500, 2731, 4096, 8192, 16384):
        sizes = [tf.tf_norm_workspace(T, d) for T in list(range(1, 1100)) + [2047, 2048, 2049, 4097, 5000, 1 << 20, (1 << 31) - 4096]]
        assert sizes == sorted(sizes), d
        # what a call is given is what it asks for
        lib = tf.load_library()
        raw = lambda T, n: lib.tf_norm_backward(None, None, T, d, BF16, A, A << 20, A << 21, A << 22, A << 23, 1, A << 24, A << 25, A << 26, BF16, 0, A << 27, n)
        assert raw(300, tf.tf_norm_workspace(300, d)) == INVALID and raw(300, sizes[-1]) == INVALID and raw(300, 4 * d) == WORKSPACE
    lengths = list(range(1, 600)) + [8191, 8192, 8193, 16384, 16385, 30000, 1 << 20, (1 << 31) - 4096]
    for d in (1, 7, 8, 4096):
        sizes = [tf.tf_embedding_workspace(T, 1000, d) for T in lengths]
        assert sizes == sorted(sizes), d
    for hq, hkv, d in ((1, 1, 16), (32, 8, 128), (3, 1, 48)):
        sizes = [tf.tf_attention_workspace(T, hq, hkv, d, BF16) for T in lengths]
        assert sizes == sorted(sizes)


REFUSING = """
#include <cstdlib>
#include <new>
static bool refuse = false;
extern "C" void refuse_memory(int on) { refuse = on; }
void* operator new(std::size_t n) { if (!refuse) if (void* p = std::malloc(n ? n : 1)) return p; throw std::bad_alloc(); }
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }
"""
CALLS = """
import ctypes, sys
from ctypes import c_float as f, c_int64 as i, c_void_p
memory, lib = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL), ctypes.CDLL(sys.argv[2])
p = lambda n: c_void_p(n << 20)
starts = (i * 3)(0, 4, 10)
rows = [p(1), i(128), p(2), i(64), p(3), i(64)]
calls = {
    "norm_forward": (i(8), i(16), 0, p(1), p(2), p(3), f(1e-5), 1, p(4), p(5), p(6)),
    "norm_backward": (i(8), i(16), 0, p(1), p(2), p(3), p(4), p(5), 1, p(6), p(7), p(8), 0, 0, p(9), i(1 << 20)),
    "embedding_forward": (i(8), i(32), i(16), 0, p(1), p(2), f(1), p(3)),
    "embedding_backward": (i(8), i(32), i(16), 0, p(1), p(2), f(1), p(3), 0, 0, p(4), i(1 << 20)),
    "distill_loss": (i(4), i(50), i(3), 0, p(1), p(2), p(3), p(4), f(1), f(1), p(5), p(6)),
    "attention_forward": (2, starts, i(10), 4, 2, 32, 0, *rows, f(0.2), p(4), i(128), p(5)),
    "attention_backward": (2, starts, i(10), 4, 2, 32, 0, *rows, p(4), i(128), p(5), p(6), f(0.2), p(7), p(8), p(9), p(10), i(1 << 20)),
}
for name, args in calls.items():
    call = lambda: getattr(lib, "tf_" + name)(None, None, *args)
    before = call()
    memory.refuse_memory(1)
    code = call()
    memory.refuse_memory(0)
    print(name, before, code, call(), flush=True)
"""


def test_no_exception_leaves_a_call_without_memory(tmp_path):
    """Host memory that cannot be had is an error code, or none where the call needs none; in a process of its own."""
    import subprocess
    import sys
    from paper_2602_05754_amd import binding
    tf.load_library()
    source, shim = tmp_path / "refusing.cpp", tmp_path / "refusing.so"
    source.write_text(REFUSING)
    subprocess.run(["g++", "-shared", "-fPIC", str(source), "-o", str(shim)], check=True)
    res = subprocess.run([sys.executable, "-c", CALLS, str(shim), binding._LIB_PATH], capture_output=True, text=True, timeout=100)
    assert res.returncode == 0, res.stdout + res.stderr
    lines = [line.split() for line in res.stdout.splitlines()]
    assert len(lines) == 7
    for name, before, refused, after in lines:
        assert int(before) == int(after) == INVALID, name                  # only the missing context
        assert int(refused) in (INVALID, WORKSPACE), name
    assert any(int(refused) == WORKSPACE for _, _, refused, _ in lines)    # the memory was refused


def test_distill_refuses_a_temperature_whose_inverse_is_infinite():
    call = lambda tau: code(tf.tf_distill_loss, None, 4, 50, 3, F32, A, 2 * A, 3 * A, None, tau, 1.0, 4 * A, None)
    lib = tf.load_library()
    assert call(1e-39) == call(1e-45) == INVALID
    # (without a context those are -1 in any case: a misaligned tensor, which is looked at later, tells them apart)
    raw = lambda tau, ids: lib.tf_distill_loss(None, None, 4, 50, 3, F32, A, ids, 3 * A, None, tau, 1.0, 4 * A, None)
    assert raw(1e-39, A + 4) == INVALID and raw(2.0 ** -126, A + 4) == ALIGN and raw(1e-30, A + 4) == ALIGN
