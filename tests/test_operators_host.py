"""Refusals of the operators around the head's logits (int8 head, sampling,
distillation): reported before anything is enqueued, so they need no GPU."""
import ctypes as C

import pytest
import torch

from paper_2608_27460_amd import vie

L = vie.lib
P = C.c_void_p(4096)      # never dereferenced: every call below fails its checks first
ODD = C.c_void_p(4097)
PRM = vie.SamplingParams(1.0, 1.0, 0.0, 0)
BIG = 1 << 40


def _int8(q=P, scale=P, V=100, d=64, h=P, ht=vie.BF16, B=40, out=C.c_void_p(1 << 20), ot=vie.F32, ld=100, ws=P, n=BIG):
    return L.vie_int8_logits(q, scale, V, d, h, ht, B, out, ot, ld, ws, n, None)


@pytest.mark.parametrize("change", [
    {"q": None}, {"scale": None}, {"h": None}, {"out": None}, {"V": 0}, {"V": 1 << 31, "ld": 1 << 31}, {"d": 0}, {"d": 8193},
    {"B": 0}, {"B": 65536}, {"ht": 2}, {"ot": -1}, {"ld": 99}, {"ws": None}, {"ws": C.c_void_p(4096 + 128)}, {"n": 10},
    {"h": ODD}, {"out": C.c_void_p((1 << 20) + 1)}, {"scale": ODD},
    {"out": P}, {"out": C.c_void_p(4096 + 6396)}, {"h": C.c_void_p((1 << 20) + 15996)}, {"scale": C.c_void_p((1 << 20) - 4)},  # overlaps
])
def test_int8_logits_refuses(change):
    assert _int8(**change) == vie.EINVAL
    assert vie.lib.vie_last_error()


def _sample(ids=P, lg=P, B=2, k=5, prm=C.byref(PRM), u=P, tok=P):
    return L.vie_sample(ids, lg, B, k, prm, u, tok, None, None, None)


@pytest.mark.parametrize("change", [{"ids": None}, {"lg": None}, {"B": 0}, {"B": 65536}, {"k": 0}, {"k": 2049},
                                    {"prm": None}, {"u": None}, {"tok": None}])
def test_sample_refuses(change):
    assert _sample(**change) == vie.EINVAL


def _rows(lg=P, dt=vie.BF16, V=100, ld=100, B=2, prm=C.byref(PRM), u=P, tok=P, ws=P, n=BIG):
    return L.vie_sample_rows(lg, dt, V, ld, B, prm, u, tok, None, None, ws, n, None)


@pytest.mark.parametrize("change", [{"lg": None}, {"lg": ODD}, {"dt": 7}, {"V": 0}, {"ld": 99}, {"B": 0}, {"prm": None},
                                    {"u": None}, {"tok": None}])
def test_sample_rows_refuses(change):
    assert _rows(**change) == vie.EINVAL


def _loss(lg=P, dt=vie.BF16, N=2, V=100, ld=100, ids=P, t=P, k=5, tau=1.0, loss=P, stats=P, ws=P, n=BIG):
    return L.vie_distill(lg, dt, N, V, ld, ids, t, k, tau, loss, stats, ws, n, None)


def _grad(lg=P, dt=vie.BF16, N=2, V=100, ld=100, ids=P, t=P, k=5, tau=1.0, stats=P, grad=C.c_void_p(1 << 20), gld=100):
    return L.vie_distill_grad(lg, dt, N, V, ld, ids, t, k, tau, stats, None, 1.0, grad, gld, None)


def _step(lg=P, dt=vie.BF16, N=2, V=100, ld=100, ids=P, t=P, k=5, tau=1.0, loss=P, grad=C.c_void_p(1 << 20), gld=100,
          ws=P, n=BIG):
    return L.vie_distill_step(lg, dt, N, V, ld, ids, t, k, tau, None, 1.0, loss, grad, gld, ws, n, None)


@pytest.mark.parametrize("call", [_loss, _grad, _step])
@pytest.mark.parametrize("change", [{"lg": None}, {"lg": ODD}, {"dt": 3}, {"N": 0}, {"N": 65536}, {"V": 0}, {"ld": 99},
                                    {"ids": None}, {"t": None}, {"k": 0}, {"k": 2049}, {"tau": 0.0}, {"tau": -1.0},
                                    {"tau": float("nan")}, {"tau": 2e4}])
def test_distill_refuses(call, change):
    assert call(**change) == vie.EINVAL


def test_distill_refuses_results_and_overlaps():
    assert _loss(loss=None) == vie.EINVAL
    assert _loss(stats=None) == vie.EINVAL
    assert _step(loss=None) == vie.EINVAL
    for call in (_grad, _step):
        assert call(grad=None) == vie.EINVAL
        assert call(gld=99) == vie.EINVAL
        assert call(grad=C.c_void_p(4096 + 200)) == vie.EINVAL  # one row further: overlaps
        assert call(grad=C.c_void_p(4096 - 2)) == vie.EINVAL
        assert call(grad=P, gld=101) == vie.EINVAL  # in place, another stride
        assert b"in place" in L.vie_last_error()
    assert _grad(stats=None) == vie.EINVAL


def test_outputs_that_overlap_are_refused():
    """Every output against every other argument, by its last byte and by its first."""
    at = {name: (i + 1) << 20 for i, name in enumerate(("a", "b", "c", "d", "e", "f", "g", "h", "i", "j"))}
    B, V, k = 3, 50, 5

    def sample_prm(x):
        return vie.SamplingParams(1.0, 1.0, 0.0, 0, x["g"], x["h"], x["i"], x["j"])

    def lists(x):
        return L.vie_sample(x["a"], x["b"], B, k, C.byref(sample_prm(x)), x["c"], x["d"], x["e"], x["f"], None)

    def rows(x):
        return L.vie_sample_rows(x["a"], vie.F32, V, V, B, C.byref(sample_prm(x)), x["c"], x["d"], x["e"], x["f"], P, BIG, None)

    def loss(x):
        return L.vie_distill(x["a"], vie.F32, B, V, V, x["b"], x["c"], k, 1.0, x["d"], x["e"], P, BIG, None)

    def grad(x):
        return L.vie_distill_grad(x["a"], vie.F32, B, V, V, x["b"], x["c"], k, 1.0, x["e"], x["f"], 1.0, x["d"], V, None)

    def step(x):
        return L.vie_distill_step(x["a"], vie.F32, B, V, V, x["b"], x["c"], k, 1.0, x["f"], 1.0, x["e"], x["d"], V, P, BIG, None)

    four, lst, row = 4 * B, 4 * B * k, 4 * B * V
    settings = {n: four for n in "ghij"}
    for call, outs, sizes in ((lists, "def", {"a": lst, "b": lst, "c": four, "d": four, "e": four, "f": four, **settings}),
                              (rows, "def", {"a": row, "c": four, "d": four, "e": four, "f": four, **settings}),
                              (loss, "de", {"a": row, "b": lst, "c": lst, "d": four, "e": 2 * four}),
                              (grad, "d", {"a": row, "b": lst, "c": lst, "d": row, "e": 2 * four, "f": four}),
                              (step, "de", {"a": row, "b": lst, "c": lst, "d": row, "e": four, "f": four})):
        for o in outs:
            for other, n in sizes.items():
                if other == o:
                    continue
                for where in (at[other] + n - 4, at[other] - sizes[o] + 4):
                    assert call({**at, o: where}) == vie.EINVAL, (call.__name__, o, other)
                    assert b"overlap" in L.vie_last_error()


def test_workspace_queries():
    n = C.c_size_t()
    assert L.vie_int8_logits_workspace(1000, 64, 40, C.byref(n)) == vie.OK and n.value >= 40 * 64
    assert L.vie_int8_logits_workspace(1000, 64, 3, C.byref(n)) == vie.OK and n.value == 0
    assert L.vie_sample_rows_workspace(1000, 3, C.byref(n)) == vie.OK
    assert L.vie_distill_workspace(1000, 3, C.byref(n)) == vie.OK
    for f, args in ((L.vie_int8_logits_workspace, (0, 64, 3)), (L.vie_int8_logits_workspace, (10, 0, 3)),
                    (L.vie_int8_logits_workspace, (10, 4, 0)), (L.vie_sample_rows_workspace, (0, 3)),
                    (L.vie_sample_rows_workspace, (10, 0)), (L.vie_distill_workspace, (10, 65536))):
        assert f(*args, C.byref(n)) == vie.EINVAL
        assert f(*args, None) == vie.EINVAL


def test_binding_refuses_host_tensors_types_and_shapes():
    f, i = torch.zeros(2, 5), torch.zeros(2, 5, dtype=torch.int32)
    u = torch.zeros(2)
    with pytest.raises(ValueError, match="device tensor"):
        vie.Int8Head(torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4))
    with pytest.raises(TypeError, match="int8"):
        vie.Int8Head(f, u)
    with pytest.raises(ValueError, match="device tensor"):
        vie.sample(i, f, u)
    with pytest.raises(TypeError, match="int32"):
        vie.sample(i.long(), f, u)
    with pytest.raises(ValueError, match="device tensor"):
        vie.sample_rows(f, u)
    for call in (lambda: vie.distill(f, i, f), lambda: vie.distill_step(f, i, f),
                 lambda: vie.distill_grad(f, i, f, torch.zeros(2, 2))):
        with pytest.raises(ValueError, match="device tensor"):
            call()


def test_a_teacher_that_requires_a_gradient_is_refused():
    f, i = torch.zeros(2, 5), torch.zeros(2, 5, dtype=torch.int32)
    with pytest.raises(ValueError, match="detach"):
        vie.distill(f, i, f.clone().requires_grad_())


def test_arrays_that_are_not_aligned_are_refused():
    """Every array of 4-byte values, one and two bytes past its place."""
    at = {name: (i + 1) << 20 for i, name in enumerate("abcdefghij")}
    B, V, k = 3, 50, 5

    def prm(x):
        return C.byref(vie.SamplingParams(1.0, 1.0, 0.0, 0, x["g"], x["h"], x["i"], x["j"]))

    calls = {
        "abcdefghij": lambda x: L.vie_sample(x["a"], x["b"], B, k, prm(x), x["c"], x["d"], x["e"], x["f"], None),
        "acdefghij": lambda x: L.vie_sample_rows(x["a"], vie.F32, V, V, B, prm(x), x["c"], x["d"], x["e"], x["f"], P, BIG, None),
        "abcde": lambda x: L.vie_distill(x["a"], vie.F32, B, V, V, x["b"], x["c"], k, 1.0, x["d"], x["e"], P, BIG, None),
        "abcdef": lambda x: L.vie_distill_grad(x["a"], vie.F32, B, V, V, x["b"], x["c"], k, 1.0, x["e"], x["f"], 1.0, x["d"], V, None),
        "fabcde": lambda x: L.vie_distill_step(x["a"], vie.F32, B, V, V, x["b"], x["c"], k, 1.0, x["f"], 1.0, x["e"], x["d"], V, P,
                                               BIG, None),
        "abc": lambda x: L.vie_int8_logits(P, x["a"], V, 8, x["b"], vie.F32, B, x["c"], vie.F32, V, P, BIG, None),
    }
    for names, call in calls.items():
        for name in names:
            for off in (1, 2):
                assert call({**at, name: at[name] + off}) == vie.EINVAL, (names, name, off)
                assert b"aligned" in L.vie_last_error(), (names, name, off)


def test_sampling_workspace_is_what_the_rows_need():
    """Little for short rows, whatever their number, and enough for fewer rows and shorter ones."""
    def need(V, B):
        n = C.c_size_t()
        assert L.vie_sample_rows_workspace(V, B, C.byref(n)) == vie.OK
        return n.value

    assert need(40, 1024) <= 1024 * 256 and need(4096, 65535) <= 65535 * 256
    sizes = [1, 40, 4096, 4097, 16384, 16385, 16896, 16897, 20000, 50257, 81920, 81921, 128256, 262144, 1 << 24, (1 << 31) - 1]
    rows = [*range(1, 140), 255, 256, 257, 1023, 1024, 1025, 65535]
    for V in sizes:
        assert all(need(V, a) <= need(V, b) for a, b in zip(rows, rows[1:])), V
    for B in rows:
        assert all(need(a, B) <= need(b, B) for a, b in zip(sizes, sizes[1:])), B
    assert need(262144, 1024) <= 128 * 120000


def test_workspaces_that_overlap_are_refused():
    """A workspace over any other argument, by its first byte and by its last 256."""
    at = {name: (i + 1) << 24 for i, name in enumerate("abcdefghij")}
    B, V, k = 40, 70000, 5
    n = C.c_size_t()

    def prm(x):
        return C.byref(vie.SamplingParams(1.0, 1.0, 0.0, 0, x["g"], x["h"], x["i"], x["j"]))

    four, lst, row = 4 * B, 4 * B * k, 4 * B * V
    for query, sizes, names, call in (
            (lambda: L.vie_sample_rows_workspace(V, B, C.byref(n)), (V, B), "acdefghij",
             lambda x, ws: L.vie_sample_rows(x["a"], vie.F32, V, V, B, prm(x), x["c"], x["d"], x["e"], x["f"], ws, BIG, None)),
            (lambda: L.vie_distill_workspace(V, B, C.byref(n)), (V, B), "abcde",
             lambda x, ws: L.vie_distill(x["a"], vie.F32, B, V, V, x["b"], x["c"], k, 1.0, x["d"], x["e"], ws, BIG, None)),
            (lambda: L.vie_distill_workspace(V, B, C.byref(n)), (V, B), "abcdef",
             lambda x, ws: L.vie_distill_step(x["a"], vie.F32, B, V, V, x["b"], x["c"], k, 1.0, x["f"], 1.0, x["e"], x["d"], V, ws,
                                              BIG, None)),
            (lambda: L.vie_int8_logits_workspace(V, 33, B, C.byref(n)), (V, B), "abcd",
             lambda x, ws: L.vie_int8_logits(x["a"], x["b"], V, 33, x["c"], vie.F32, B, x["d"], vie.F32, V, ws, BIG, None))):
        assert query() == vie.OK and n.value >= 256
        for name in names:
            for ws in (at[name], at[name] - (n.value - 4) // 256 * 256):
                assert call(at, C.c_void_p(ws)) == vie.EINVAL, (names, name)
                assert b"overlap" in L.vie_last_error(), (names, name, L.vie_last_error())


def test_a_workspace_serves_fewer_rows():
    """What a call asks for never grows as its rows become fewer."""
    n = C.c_size_t()
    rows = [*range(1, 70), 127, 128, 129, 255, 256, 257, 258, 300, 1000, 1024, 1025, 40000, 65535]
    queries = [lambda V, B: L.vie_sample_rows_workspace(V, B, C.byref(n)), lambda V, B: L.vie_distill_workspace(V, B, C.byref(n))]
    queries += [lambda V, B, d=d: L.vie_int8_logits_workspace(V, d, B, C.byref(n))
                for d in (1, 15, 16, 256, 1000, 1024, 2047, 2048, 2049, 2064, 4096, 8191, 8192)]
    for query in queries:
        for V in (1, 7, 1000, 17000, 50257, 262144):
            need = []
            for B in rows:
                assert query(V, B) == vie.OK
                need.append(n.value)
            assert need == sorted(need), V


def test_matrices_that_share_rows_of_one_buffer():
    """Halves of wider rows do not overlap, but any byte of the other half does, and so do other strides."""
    B, V, ld, k = 4, 50, 128, 5
    at = (1 << 20)
    lists = (C.c_void_p(1 << 24), C.c_void_p(1 << 25))

    def grad(logits, out, gld=ld, stats=C.c_void_p(1 << 26)):
        return L.vie_distill_grad(C.c_void_p(logits), vie.F32, B, V, ld, *lists, k, 1.0, stats, None, 1.0, C.c_void_p(out), gld, None)

    for off in (4, 4 * 49, 4 * (128 - 49), 4 * 127, 4 * 128, 4 * 129, 4 * 3 * 128, -4, -4 * 49, -4 * 128, -4 * (128 + 79)):
        assert grad(at, at + off) == vie.EINVAL, off
        assert b"overlap" in L.vie_last_error()
    assert grad(at, at + 4 * 64, ld + 1) == vie.EINVAL                       # rows of another stride meet them somewhere
    for off in (-4, 4 * 49, 4 * 128 - 28, 4 * 128 + 40, 4 * (3 * 128 + 49)):  # 32 bytes of statistics, gaps of 200 to 512
        assert grad(1 << 27, at, stats=C.c_void_p(at + off)) == vie.EINVAL, off
