"""The norms, the embedding and the distillation loss through the C ABI, against the oracle's fp64
definitions on the same inputs, at the sizes and values where they can go wrong.  Bounds per element are
gpu_util's: one rounding of an fp32 result."""
import numpy as np
import pytest
import torch

import workloads as wl
import paper_2602_05754_amd as tf
from gpu_util import CODE, TDT, assert_elementwise, canary, dev, host64, raw_bytes
from oracle import operators as op

pytestmark = pytest.mark.gpu
TYPES = ("f32", "bf16")


@pytest.fixture(scope="module")
def ctx():
    c = tf.Context(0)
    yield c
    c.close()


def stored(a, io):
    """The values that `a` has in storage type io, and the device tensor of them."""
    t = dev(np.asarray(a, np.float32), io)
    return host64(t), t


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


# ---------------------------------------------------------------------------------------------
# norms
# ---------------------------------------------------------------------------------------------
# one element; a piece and its neighbours; a wave's row and its neighbours; each wider shape; the widest row
WIDTHS = [1, 3, 8, 63, 511, 513, 1000, 1024, 2048, 2731, 4096, 6001, 8192, 16384]


@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_forward(ctx, d, center, io):
    rs = np.random.default_rng(d)
    for T in (1, 2, 37):
        x, gx = stored(rs.standard_normal((T, d)) * 2 + 0.7, io)
        w, gw = stored(1 + 0.3 * rs.standard_normal(d), io)
        b, gb = stored(rs.standard_normal(d), io)
        for bias in (None, b):
            y, mean, rstd = canary((T, d), TDT[io]), canary((T,), torch.float32), canary((T,), torch.float32)
            before = raw_bytes(mean)
            tf.tf_norm_forward(ctx, T, d, CODE[io], gx, gw, None if bias is None else gb, 1e-3, center, y, mean if center else None, rstd)
            ey, em, er = op.norm_forward(x, w, bias, float(np.float32(1e-3)), center)
            assert_elementwise(host64(y), ey, io, f"y T={T}")
            assert_elementwise(host64(rstd), er, "f32", "rstd")
            if center:
                assert_elementwise(host64(mean), em, "f32", "mean")
            else:
                assert raw_bytes(mean) == before


@pytest.mark.parametrize("io,dw", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_backward(ctx, d, center, io, dw):
    rs = np.random.default_rng(d + 1)
    for T in (1, 5, 2300) if d <= 1024 else (1, 5, 300):                  # more rows than blocks take at once
        x, gx = stored(rs.standard_normal((T, d)) + 0.3, io)
        w, gw = stored(1 + 0.3 * rs.standard_normal(d), io)
        dy, gdy = stored(rs.standard_normal((T, d)), io)
        eps = 1e-2                                    # (a row of one element, centred, has nothing but eps)
        _, mean, rstd = op.norm_forward(x, w, None, eps, center)
        ex, ew, eb = op.norm_backward(x, w, dy, eps, center)
        gm, gr = (f32(mean) if center else None), f32(rstd)
        dx, gdw, gdb = canary((T, d), TDT[io]), canary((d,), TDT[dw]), canary((d,), TDT[dw])
        tf.tf_norm_backward(ctx, T, d, CODE[io], gx, gw, gdy, gm, gr, center, dx, gdw, gdb, CODE[dw])
        # dx is a difference of three values of order rstd |dy w|: where they cancel, the bound is theirs
        scale = float(np.abs(rstd).max() * np.sqrt((dy * w) ** 2).mean())
        if dw != "bf16" or d > 1:
            got, tiny = host64(dx), 2e-6 * scale
            assert_elementwise(np.where(np.abs(got - ex) <= tiny, ex, got), ex, io, f"dx T={T}")
        # sums over T rows of products with xh: 32-bit, error below T^0.5 2^-24 of a term's size
        for got, want, what in ((gdw, ew, "dw"), (gdb, eb, "db")):
            got, tiny = host64(got), 4e-7 * np.sqrt(T) * 4
            assert_elementwise(np.where(np.abs(got - want) <= tiny, want, got), want, dw, f"{what} T={T}")


def test_norm_backward_of_frozen_parameters_and_accumulation(ctx):
    rs = np.random.default_rng(9)
    T, d = 70, 300
    x, gx = stored(rs.standard_normal((T, d)), "bf16")
    w, gw = stored(1 + 0.3 * rs.standard_normal(d), "bf16")
    dy, gdy = stored(rs.standard_normal((T, d)), "bf16")
    _, mean, rstd = op.norm_forward(x, w, None, 1e-5, True)
    _, ew, eb = op.norm_backward(x, w, dy, 1e-5, True)
    call = lambda dx, dw, db, **kw: tf.tf_norm_backward(ctx, T, d, tf.TF_BF16, gx, gw, gdy, f32(mean), f32(rstd), True, dx, dw, db, tf.TF_F32, **kw)
    new = lambda: torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    all_dx, dx, dw, db = new(), new(), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    call(all_dx, dw, db)
    for pair in ((None, None), (dw, None), (None, db)):                     # what is frozen changes nothing else
        was = [None if t is None else t.clone() for t in pair]
        call(dx.fill_(7), *pair)
        assert torch.equal(dx, all_dx) and all(t is None or torch.equal(t, v) for t, v in zip(pair, was))
    old = torch.randn(d, device="cuda")
    sums = [old.clone(), old.clone()]
    call(dx, *sums, accumulate=True)
    assert torch.equal(sums[0], old + dw) and torch.equal(sums[1], old + db)


def test_norm_of_rows_with_infinities_stays_in_its_row(ctx):
    x = np.random.default_rng(1).standard_normal((9, 100)).astype(np.float32)
    clean = x.copy()
    x[4, 50], x[6, 3] = np.inf, np.nan
    out = []
    for a in (x, clean):
        y, rstd, mean = torch.empty((9, 100), device="cuda"), torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
        tf.tf_norm_forward(ctx, 9, 100, tf.TF_F32, f32(a), f32(np.ones(100)), None, 1e-5, True, y, mean, rstd)
        out.append(y.cpu().numpy())
    keep = [i for i in range(9) if i not in (4, 6)]
    assert np.array_equal(out[0][keep], out[1][keep]) and np.isnan(out[0][4]).any() and np.isnan(out[0][6]).all()


# ---------------------------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------------------------
def ids_of(kind, T, V, rs):
    if kind == "one":
        return np.full(T, V // 2)                     # every token the same row: whole windows, long runs
    if kind == "all":
        return rs.permutation(max(T, V))[:T] % V
    ids = np.minimum((V * rs.random(T) ** 4).astype(np.int64), V - 1)      # few rows often, most never
    if kind == "padded":
        ids[rs.random(T) < 0.3] = -1
        ids[rs.random(T) < 0.1] = V
        ids[-1] = np.iinfo(np.int32).min
    return ids


@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (1, 700, 8), (3, 5, 7), (100, 17, 300), (2049, 1000, 96), (5000, 333, 2049)])
def test_embedding_forward(ctx, T, V, d, io):
    rs = np.random.default_rng(T + d)
    table, gt = stored(rs.standard_normal((V, d)), io)
    ids = ids_of("padded" if T > 1 else "all", T, V, rs)
    out = canary((T, d), TDT[io])
    tf.tf_embedding_forward(ctx, T, V, d, CODE[io], torch.from_numpy(ids.astype(np.int32)).cuda(), gt, 0.75, out)
    assert_elementwise(host64(out), op.embedding_forward(ids, table, 0.75), io, "out")


@pytest.mark.parametrize("io,dw", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("kind", ["one", "all", "text", "padded"])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (1, 700, 8), (63, 5, 7), (65, 200, 300), (2048, 50, 33), (2049, 1000, 96), (6500, 4001, 2056)])
def test_embedding_backward(ctx, T, V, d, kind, io, dw):
    rs = np.random.default_rng(T + d)
    ids = ids_of(kind, T, V, rs)
    gids = torch.from_numpy(ids.astype(np.int32)).cuda()
    dout, gd = stored(rs.standard_normal((T, d)), io)
    want = op.embedding_backward(ids, dout, 1.25, V)
    out = canary((V, d), TDT[dw])
    tf.tf_embedding_backward(ctx, T, V, d, CODE[io], gids, gd, 1.25, out, CODE[dw])
    # sums of up to T values of order 1 in 32 bits: their rounding is below T^0.5 2^-24 of the sum's own size sqrt(T)
    tiny = 6e-8 * T if kind != "all" else 0.0
    check = lambda got, label: assert_elementwise(np.where(np.abs(got - want) <= tiny, want, got), want, dw, label)
    check(host64(out), "dtable")
    again = canary((V, d), TDT[dw])
    tf.tf_embedding_backward(ctx, T, V, d, CODE[io], gids, gd, 1.25, again, CODE[dw])
    assert torch.equal(out, again)                    # the same bits
    if dw == "f32":
        old = torch.randn((V, d), device="cuda")
        untouched = [v for v in range(V) if v not in set(ids.tolist())]
        sums = old.clone()
        sums[untouched] = float("nan")                # rows without tokens are left alone, whatever they hold
        tf.tf_embedding_backward(ctx, T, V, d, CODE[io], gids, gd, 1.25, sums, CODE[dw], accumulate=True)
        hit = sorted(set(ids.tolist()) & set(range(V)))
        assert torch.isnan(sums[untouched]).all()
        # (the scaling may join the addition in one rounding there)
        assert torch.allclose(sums[hit], old[hit] + out[hit], rtol=3e-7, atol=3e-7 * max(1.0, T ** 0.5))


@pytest.mark.parametrize("io,dw", [("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("kind", ["one", "text", "padded"])
@pytest.mark.parametrize("T,V,d", [(16, 3, 8), (17, 2, 5), (128, 9, 24), (257, 40, 8), (512, 100, 520), (513, 100, 8), (8192, 77, 12), (8193, 500, 8), (30000, 900, 20)])
def test_embedding_backward_windows(ctx, T, V, d, kind, io, dw):
    """Lengths around those of a window, of the sort by counting and of a chunk; runs over many windows and chunks."""
    test_embedding_backward(ctx, T, V, d, kind, io, dw)


# ---------------------------------------------------------------------------------------------
# distillation loss
# ---------------------------------------------------------------------------------------------
def distill(ctx, z, ids, teacher, weight, tau, scale, io, grad=True):
    T, V = z.shape
    loss = canary((T,), torch.float32)
    dz = canary((T, V), TDT[io]) if grad else None
    tf.tf_distill_loss(ctx, T, V, ids.shape[1], CODE[io], z, torch.from_numpy(ids.astype(np.int32)).cuda(), f32(teacher),
                       None if weight is None else f32(weight), tau, scale, loss, dz)
    return host64(loss), None if dz is None else host64(dz)


def check_distill(ctx, rs, T, V, K, tau, io, ids=None, weight=None):
    z, gz = stored(rs.standard_normal((T, V)) * 3, io)
    ids = np.stack([rs.permutation(max(V, K))[:K] for _ in range(T)]) if ids is None else ids
    teacher = (rs.standard_normal((T, K)) * 2).astype(np.float32)
    tau, scale = float(np.float32(tau)), float(np.float32(0.37))
    loss, dz = distill(ctx, gz, ids, teacher, weight, tau, scale, io)
    el, ez = op.distill_loss(z, ids, teacher, weight, tau, scale)
    # log q is a difference of numbers up to |z| / tau + log V: 4 roundings of those in the sum of p (log p - log q)
    assert np.abs(loss - el).max() <= 4 * 2.0 ** -24 * tau ** 2 * (15 / tau + 12) * (1 if weight is None else max(1, np.abs(weight).max())) + 1e-30
    # q - p where they cancel: the bound is theirs, exp of an argument up to 30 / tau rounded to 24 bits
    tiny = scale * tau * 3e-6
    assert_elementwise(np.where(np.abs(dz - ez) <= tiny * (np.abs(ez) / (scale * tau) + (ez <= 0) + 1e-3), ez, dz), ez, io, f"dz T={T} V={V} K={K}")
    alone, _ = distill(ctx, gz, ids, teacher, weight, tau, scale, io, grad=False)
    assert np.array_equal(alone, loss)


# each number of pieces and of threads, their last element and the next; beyond: rows that are read twice
@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("V", [1, 2, 7, 130, 4096, 4097, 5003, 8192, 8200, 16385, 32768, 32771, 65536, 65537, 131072, 131079, 160001])
def test_distill_widths(ctx, V, io):
    check_distill(ctx, np.random.default_rng(V), 3, V, min(V, 5), 1.0, io)


@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("K,tau", [(1, 1.0), (1, 3.0), (63, 2.0), (64, 0.5), (65, 4.0), (1000, 2.0), (1024, 1.0)])
def test_distill_entries_and_temperatures(ctx, K, tau, io):
    check_distill(ctx, np.random.default_rng(K), 5, 1500, K, tau, io)


@pytest.mark.parametrize("io", TYPES)
def test_distill_names_absent_twice_and_not_at_all(ctx, io):
    rs = np.random.default_rng(7)
    V = 333
    ids = rs.integers(-40, V + 40, (40, 50))
    ids[3], ids[4], ids[5] = -1, V, 17                # none; none; one id fifty times
    weight = np.where(rs.random(40) < 0.3, 0, rs.random(40)).astype(np.float32)
    check_distill(ctx, rs, 40, V, 50, 2.0, io, ids, weight)


@pytest.mark.parametrize("V", [50, 300000])           # held in registers; read twice
def test_distill_rows_that_are_not_read_and_masked_words(ctx, V):
    rs = np.random.default_rng(8)
    z = rs.standard_normal((6, V)).astype(np.float32)
    ids, teacher = np.tile(np.arange(4), (6, 1)), rs.standard_normal((6, 4)).astype(np.float32)
    weight = np.array([1, 0, 1, 1, 1, 1], np.float32)
    z[1] = np.nan                                     # weight 0: not looked at
    z[2, 10:20] = -np.inf                             # words that cannot be: q = 0
    z[3] = np.finfo(np.float32).min                   # all words equally impossible but one
    z[3, 2] = 0
    teacher[4] = -np.inf                              # a teacher without an opinion
    teacher[5, 1] = -np.inf                           # one of its words ruled out, by the student too
    z[5, 1] = -np.inf
    z[4] = np.nan
    loss, dz = distill(ctx, f32(z), ids, teacher, weight, 1.0, 1.0, "f32")
    with np.errstate(all="ignore"):
        clean = z.copy()
        clean[1] = clean[4] = 0
        el, ez = op.distill_loss(clean, ids, teacher, weight, 1.0, 1.0)
    assert loss[1] == loss[4] == 0 and not dz[1].any() and not dz[4].any()
    assert not dz[2, 10:20].any() and dz[5, 1] == 0
    assert np.isfinite(dz).all() and np.abs(dz - ez).max() < 3e-6
    good = [0, 1, 2, 4, 5]
    assert np.abs(loss - el)[good].max() < 2e-5 and abs(loss[3] / el[3] - 1) < 1e-5
    z[0, 7] = np.nan                                  # a NaN that is read is passed on, within its row
    loss, dz = distill(ctx, f32(z), ids, teacher, weight, 1.0, 1.0, "f32")
    assert np.isnan(loss[0]) and np.isnan(dz[0]).all() and np.isfinite(dz[1:]).all()


@pytest.mark.parametrize("tau", [0.01, 0.25, 0.5, 0.99, 1.0])
@pytest.mark.parametrize("io", TYPES)
def test_distill_of_a_word_with_the_lowest_value(ctx, io, tau):
    """A word that the teacher names and the student's mask rules out: log q = z / tau is beyond 32 bits, the loss tau^2 p log q is not.
    Of the sum only that word's term is left, its factors rounded a few times each; the gradient does not see how low the word is."""
    rs = np.random.default_rng(5)
    lowest = float(torch.finfo(TDT[io]).min)
    z = rs.standard_normal((4, 60))
    z[:, 7] = lowest
    z[2] = lowest                                      # all but one
    z[2, 30] = 1.0
    z, gz = stored(z, io)
    ids, teacher = np.tile([7, 9, 11], (4, 1)), rs.standard_normal((4, 3)).astype(np.float32)
    teacher[3, 0] = -np.inf                            # there the teacher has ruled it out too
    tau = float(np.float32(tau))
    loss, dz = distill(ctx, gz, ids, teacher, None, tau, 1.0, io)
    el, ez = op.distill_loss(z, ids, teacher, None, tau, 1.0)
    assert np.isfinite(el).all() and np.all(np.abs(loss - el) <= 1e-4 * np.abs(el)), (loss, el)
    # exp of up to 10 / tau, rounded to 24 bits as the arguments are; bf16: the result's rounding
    assert np.all(np.abs(dz - ez) <= (2.0 ** -8 if io == "bf16" else 0) * np.abs(ez) + tau * (20 / tau) * 2.0 ** -22)


@pytest.mark.parametrize("tau", [2.0 ** -126, 2.0 ** -100, 2.0 ** -40])
def test_distill_at_the_smallest_temperatures(ctx, tau):
    """p and q have one word each: the loss is tau times the difference of two logits, the gradient tau at the two words."""
    rs = np.random.default_rng(6)
    z, teacher = rs.standard_normal((5, 300)).astype(np.float32), rs.standard_normal((5, 4)).astype(np.float32)
    ids = np.tile([7, 9, 11, 250], (5, 1))
    loss, dz = distill(ctx, f32(z), ids, teacher, None, tau, 1.0, "f32")
    el, ez = op.distill_loss(z, ids, teacher, None, tau, 1.0)
    assert np.all(np.abs(loss - el) <= 1e-5 * el) and np.array_equal(dz, ez) and (ez != 0).any()


def test_distill_of_the_widest_rows(ctx):
    """V = 2^31 - 4096, where a row's last step of 8192 words ends behind 2^31: a row that is read, between one without weight and one
    without a teacher's word.  All logits are 0, so q = 1 / V and the sum of V ones in 32 bits is exact."""
    V, T, room = (1 << 31) - 4096, 3, 8192
    z = torch.zeros((T, V), dtype=torch.bfloat16, device="cuda")
    buf = torch.full((room + T * V + room,), 3.0, dtype=torch.bfloat16, device="cuda")
    dz = buf[room:room + T * V].view(T, V)
    ids = torch.tensor([[V - 1], [V - 1], [V]], dtype=torch.int32, device="cuda")
    loss = canary((T,), torch.float32)
    tf.tf_distill_loss(ctx, T, V, 1, tf.TF_BF16, z, ids, torch.zeros((T, 1), device="cuda"), f32([0, 1, 1]), 1.0, 1024.0, loss, dz)
    loss = host64(loss)
    assert loss[0] == loss[2] == 0 and abs(loss[1] - np.log(V)) < 1e-5
    every = lambda x, value: all(bool((part == value).all()) for part in x.split(1 << 28))
    assert every(buf[:room], 3.0) and every(buf[room + T * V:], 3.0)
    assert every(dz[0], 0.0) and every(dz[2], 0.0)
    # (2^10 / V is 2^-21 within 2^-19 of it)
    assert every(dz[1, :V - 1], 2.0 ** -21) and float(dz[1, V - 1]) == -1024.0


# ---------------------------------------------------------------------------------------------
# streams, graphs
# ---------------------------------------------------------------------------------------------
def test_calls_on_another_stream_and_in_a_graph(ctx):
    rs = np.random.default_rng(3)
    T, d, V = 200, 520, 90
    _, x = stored(rs.standard_normal((T, d)), "bf16")
    _, w = stored(rs.standard_normal(d), "bf16")
    _, dy = stored(rs.standard_normal((T, d)), "bf16")
    ids = torch.from_numpy(ids_of("text", T, V, rs).astype(np.int32)).cuda()
    _, z = stored(rs.standard_normal((T, V)), "f32")
    tids, tl = torch.randint(0, V, (T, 6), device="cuda", dtype=torch.int32), torch.randn((T, 6), device="cuda")
    y, rstd, mean = torch.empty_like(x), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    dtable, loss, dz = torch.empty((V, d), device="cuda"), torch.empty(T, device="cuda"), torch.empty((T, V), device="cuda")
    ws = torch.empty(max(tf.tf_norm_workspace(T, d), tf.tf_embedding_workspace(T, V, d)), dtype=torch.uint8, device="cuda")

    def step(workspace=ws):
        tf.tf_norm_forward(ctx, T, d, tf.TF_BF16, x, w, None, 1e-5, True, y, mean, rstd)
        tf.tf_norm_backward(ctx, T, d, tf.TF_BF16, x, w, dy, mean, rstd, True, dx, dw, db, tf.TF_F32, workspace=workspace)
        tf.tf_embedding_backward(ctx, T, V, d, tf.TF_BF16, ids, dx, 2.0, dtable, tf.TF_F32, workspace=workspace)
        tf.tf_distill_loss(ctx, T, V, 6, tf.TF_F32, z, tids, tl, None, 2.0, 0.1, loss, dz)
    outs = [y, mean, rstd, dx, dw, db, dtable, loss, dz]
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    for workspace in (ws, None):
        for t in outs:
            t.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(workspace)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        for t in outs:
            t.fill_(i)
        ws.fill_(255)                                 # nothing is kept there from one call to the next
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("default", [0, "stream"])
def test_a_call_on_the_default_stream_while_another_is_current(ctx, default):
    """Its workspace is not the other stream's memory, which that stream's work would get next."""
    from paper_2602_05754_amd import binding
    stream = 0 if default == 0 else torch.cuda.default_stream()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.empty(5 << 20, dtype=torch.uint8, device="cuda")             # the side stream's pool has memory of that size
        keep, address, n = binding._workspace(ctx, None, 5 << 20, stream)
        del keep
        again = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
        assert all(t.data_ptr() != address for t in again)
    keep, address, n = binding._workspace(ctx, None, 5 << 20, side)
    del keep
    with torch.cuda.stream(side):
        assert torch.empty(n, dtype=torch.uint8, device="cuda").data_ptr() == address


def test_the_default_stream_gives_the_same_gradients_while_another_is_current(ctx):
    rs = np.random.default_rng(4)
    T, V, d = 900, 60, 264
    _, dout = stored(rs.standard_normal((T, d)), "bf16")
    ids = torch.from_numpy(ids_of("text", T, V, rs).astype(np.int32)).cuda()
    want, got = torch.empty((V, d), device="cuda"), torch.empty((V, d), device="cuda")
    tf.tf_embedding_backward(ctx, T, V, d, tf.TF_BF16, ids, dout, 1.0, want, tf.TF_F32)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for _ in range(20):
            tf.tf_embedding_backward(ctx, T, V, d, tf.TF_BF16, ids, dout, 1.0, got, tf.TF_F32, stream=0)
            torch.empty(tf.tf_embedding_workspace(T, V, d), dtype=torch.uint8, device="cuda").fill_(255)       # the current stream's own work
        torch.cuda.synchronize()
    assert torch.equal(got, want)
