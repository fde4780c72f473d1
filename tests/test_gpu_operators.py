"""Operators on rows of logits on the GPU against their definitions in 64 bits (tests/logits_ref.py)."""
import math
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import logits_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
INF = math.inf


@pytest.fixture(scope="module")
def B():
    from paper_1801_03138_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.lib()
    return binding


def table(rng, rows, n, dtype, pad=0, sigma=1.5, masked=0.0, shift=0.0):
    """rows x n logits on the GPU as a view into a wider table, and the same values in 64 bits."""
    x = rng.normal(shift, sigma, (rows, n + pad)).astype(np.float32)
    if masked:
        x[rng.random(x.shape) < masked] = -INF
    t = torch.from_numpy(x).to(DT[dtype]).cuda()
    view = t[:, :n]
    return view, view.float().cpu().double().numpy()


# --------------------------------------------------------------------------------------- choose
def check_choice(x, u, how, index, logp):
    """Every row's choice is the definition's; where u falls within a hair of a border, either neighbour.
    Sums are off by less than half a unit of 2^-44 (of the best action's weight) per action, and by a few
    2^-53 of themselves; the log-probability is rounded to 32 bits once."""
    index, logp = index.cpu().numpy(), logp.cpu().double().numpy()
    for r in range(len(x)):
        row_how = {k: float(v[r]) if isinstance(v, np.ndarray) else v for k, v in how.items()}
        row_how["top_k"] = int(row_how.get("top_k", 0))
        want = ref.choose(x[r], float(u[r]), **row_how)
        if want is None:
            assert index[r] == -1 and logp[r] == 0, r
            continue
        ids, c, at = want
        hair = len(x[r]) * 2.0 ** -44 + 2.0 ** -40 * c[-1]
        drawn = max(float(u[r]), 0.0) * c[-1]
        near = [at]
        if at > 0 and drawn - c[at - 1] < hair:
            near.append(at - 1)
        if at + 1 < len(c) and c[at] - drawn < hair:
            near.append(at + 1)
        assert index[r] in ids[near], (r, index[r], ids[near], row_how, float(u[r]))
        got = int(np.nonzero(ids == index[r])[0][0])
        w = c[got] - (c[got - 1] if got else 0.0)
        exact = math.log(w / c[-1]) if row_how.get("temperature", 1.0) > 0 else 0.0
        assert abs(logp[r] - exact) <= 2.0 ** -23 * abs(exact) + 2 * hair / w, (r, logp[r], exact)


def draw_u(rng, rows):
    u = rng.random(rows).astype(np.float32)
    edge = np.array([0.0, np.float32(1 - 2.0 ** -24), 0.5], np.float32)
    u[:min(rows, 3)] = edge[:min(rows, 3)]
    return u


SHAPES = [(1, 1), (3, 2), (130, 30), (5, 63), (5, 64), (5, 65), (7, 257), (4, 1000), (3, 2049), (9, 4099), (2, 20_011),
          (1, 131_072), (3, 70_001)]
HOWS = [{"temperature": 0.8}, {"temperature": 1.3, "top_k": 7}, {"top_p": 0.9}, {"top_p": 0.7, "min_p": 0.01, "top_k": 50},
        {"min_p": 0.2}, {"temperature": 0.0}, {"top_k": 1}, {"top_p": 0.0}, {"temperature": 0.7, "top_k": 1500, "top_p": 0.97},
        {"temperature": 4.0, "top_k": 1024}]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_choice_is_the_definitions(B, rows, n, dtype):
    rng = np.random.default_rng(rows * 1000 + n)
    for i, how in enumerate(HOWS):
        g, x = table(rng, rows, n, dtype, pad=[0, 1, 2, 5][i % 4], sigma=[0.3, 1.5, 3.0][i % 3], masked=[0.0, 0.4][i % 2],
                     shift=[0.0, -7.0, 40.0][(i // 2) % 3])
        u = draw_u(rng, rows)
        index, logp = B.choose_actions(g, torch.from_numpy(u).cuda(), **how)
        check_choice(x, u, how, index, logp)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(200, 30), (40, 700), (24, 5003), (9, 33_333)])
def test_every_row_has_its_own_settings(B, rows, n, dtype):
    rng = np.random.default_rng(n)
    g, x = table(rng, rows, n, dtype, pad=3, sigma=2.0, masked=0.2)
    how = {"temperature": rng.choice([-1.0, 0.0, 0.5, 1.0, 2.5, 1e-30, 1e30], rows).astype(np.float32),
           "top_k": rng.choice([-3, 0, 1, 2, 20, 300, 1024, 1025, n, n + 1], rows).astype(np.int32),
           "top_p": rng.choice([-1.0, 0.0, 0.1, 0.5, 0.95, 1.0, 2.0], rows).astype(np.float32),
           "min_p": rng.choice([-1.0, 0.0, 0.001, 0.3, 1.0, 1.5], rows).astype(np.float32)}
    u = draw_u(rng, rows)
    index, logp = B.choose_actions(g, torch.from_numpy(u).cuda(), **{k: torch.from_numpy(v).cuda() for k, v in how.items()})
    check_choice(x, u, how, index, logp)


SPECIAL = {
    "nothing allowed": lambda n: [-INF] * n,
    "only NaN": lambda n: [math.nan] * n,
    "one allowed": lambda n: [-INF] * (n - 1) + [-3.0],
    "NaN among others": lambda n: [math.nan, 1.0] + [0.5] * (n - 2),
    "infinities": lambda n: [0.0, INF, 5.0, INF] + [-INF] * (n - 4),
    "all equal": lambda n: [0.25] * n,
    "both zeros": lambda n: [0.0, -0.0] * (n // 2) + [0.0] * (n % 2),
    "lowest values": lambda n: [-3.3895313892515355e38] * (n - 2) + [0.0, -1.0],
    "only lowest values": lambda n: [-3.3895313892515355e38] * n,
    "highest and lowest": lambda n: [3.3895313892515355e38] * 2 + [-3.3895313892515355e38] * (n - 2),
    "two levels": lambda n: [1.0] * (n // 2) + [2.0] * (n - n // 2),
    "a far tail": lambda n: [30.0] + [0.0] * (n - 1),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [6, 30, 64, 65, 1000, 6001, 150_001])
def test_choice_from_special_rows(B, n, dtype):
    names = list(SPECIAL)
    g = torch.tensor([SPECIAL[k](n) for k in names], dtype=torch.float32).to(DT[dtype]).cuda()
    x = g.float().cpu().double().numpy()
    for u0 in (0.0, 0.25, 0.5, 1 - 2.0 ** -24):
        u = np.full(len(names), u0, np.float32)
        for how in ({}, {"top_k": 3}, {"top_k": 1000}, {"top_k": 1500}, {"top_p": 0.5}, {"min_p": 0.5}, {"temperature": 0.0},
                    {"temperature": INF}, {"temperature": math.nan}, {"top_p": math.nan, "min_p": math.nan}):
            index, logp = B.choose_actions(g, torch.from_numpy(u).cuda(), **how)
            check_choice(np.where(np.isnan(x), -INF, x), u, how, index, logp)


def test_random_numbers_outside_the_unit_interval_are_its_ends(B):
    g, x = table(np.random.default_rng(1), 1, 40, "f32")
    c = lambda v: int(B.choose_actions(g, torch.tensor([v], device="cuda"))[0])
    first, last = c(0.0), ref.order(x[0])[-1]
    assert first == ref.order(x[0])[0]
    assert c(-1.0) == first and c(math.nan) == first and c(1.0) == last and c(7.0) == last


@pytest.mark.parametrize("n", [30, 6007])
def test_choices_have_the_softmax_frequencies(B, n):
    """Evenly spaced random numbers hit every action as often as its probability says, to one draw."""
    rng = np.random.default_rng(5)
    g, x = table(rng, 1, n, "f32", sigma=2.0)
    draws = 20_000
    u = ((np.arange(draws) + 0.5) / draws).astype(np.float32)
    index = B.choose_actions(g.expand(draws, n), torch.from_numpy(u).cuda())[0].cpu().numpy()
    p = np.exp(x[0] - ref.log_sum_exp(x[0]))
    # (u is rounded to 2^-24: a draw moves by less than 2^-24 * draws of a place)
    assert np.abs(np.bincount(index, minlength=n) - p * draws).max() <= 1.01


# ------------------------------------------------------------------------------------------ top
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_top_actions(B, rows, n, dtype):
    rng = np.random.default_rng(rows * 77 + n)
    for i, k in enumerate(sorted({1, 2, 8, 64, 100, 500, 1000, 1024, n})):
        if k > min(n, 1024):
            continue
        g, x = table(rng, rows, n, dtype, pad=i % 3, sigma=[0.3, 2.0][i % 2], masked=[0.0, 0.5, 0.0, 0.97][i % 4])
        t = [1.0, 0.7, 3.0][i % 3]
        check_top(x, k, t, *B.top_actions(g, k, temperature=t))


def check_top(x, k, t, values, index, lse):
    values, index, lse = values.float().cpu().numpy(), index.cpu().numpy(), lse.cpu().numpy()
    for r in range(len(x)):
        ids = ref.order(x[r])[:k]
        assert np.array_equal(index[r], np.concatenate([ids, np.full(k - len(ids), -1)])), r
        assert np.array_equal(values[r], np.concatenate([x[r][ids], np.full(k - len(ids), -INF)])), r
        if len(ids) and x[r][ids[0]] == INF:
            assert lse[r] == INF
            continue
        want = ref.log_sum_exp(x[r], t)
        if want == -INF:
            assert lse[r] == -INF
            continue
        # the sum's relative error (see ref.distill), and the rounding of the result
        assert abs(lse[r] - want) <= 2.0 ** -22 * (math.log(x.shape[1]) + 4) + 2.0 ** -23 * abs(want), (r, lse[r], want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [6, 30, 64, 65, 1000, 6001, 150_001])
def test_top_actions_of_special_rows(B, n, dtype):
    names = list(SPECIAL)
    g = torch.tensor([SPECIAL[k](n) for k in names], dtype=torch.float32).to(DT[dtype]).cuda()
    x = g.float().cpu().double().numpy()
    for k in {1, 5, min(n, 700), min(n, 1024)}:
        check_top(np.where(np.isnan(x), -INF, x), k, 1.0, *B.top_actions(g, k))


# -------------------------------------------------------------------------------------- distill
def entries(rng, x, k, dtype, short=0.2, repeated=False, noise=1.0):
    """A teacher's entries for rows x: the top k of noisy logits, some missing; its log-sum-exp at 0.9."""
    rows, n = x.shape
    t = 0.7 * np.where(np.isfinite(x), x, 0.0) + rng.normal(0, noise, x.shape)
    t = torch.from_numpy(t.astype(np.float32)).to(DT[dtype]).double().numpy()
    index = np.argsort(-t, axis=1, kind="stable")[:, :k].astype(np.int32)
    if k > n:
        index = np.concatenate([index, np.full((rows, k - n), -1, np.int32)], axis=1)
    value = np.take_along_axis(t, np.maximum(index, 0), 1)
    lse = np.array([ref.log_sum_exp(r, 0.9) for r in t], np.float32)
    index[rng.random(index.shape) < short] = rng.choice([-1, n, n + 5, -(2 ** 31), 2 ** 31 - 1])
    if repeated and k > 1:
        index[:, -1] = index[:, 0]
        index[::2, k // 2] = index[::2, 0]
        lse += 0.5   # (so that the entries' mass stays below 1)
    return value, index, lse


def check_distill(B, g, x, value, index, weight, lse, tdtype, dtype, ts=1.1, tt=0.9):
    tv = torch.from_numpy(value.astype(np.float32)).to(DT[tdtype])
    value = tv.double().numpy()
    kw = dict(weight=None if weight is None else torch.from_numpy(weight).cuda(),
              teacher_lse=None if lse is None else torch.from_numpy(lse).cuda(), student_temperature=ts,
              teacher_temperature=tt)
    idx = torch.from_numpy(index).cuda()
    only = B.distill_loss(g, tv.cuda(), idx, **kw)
    loss, grad = B.distill_grad(g, tv.cuda(), idx, **kw)
    own = g.clone()
    own_loss, own_grad = B.distill_grad(own, tv.cuda(), idx, out=(torch.empty_like(loss), own), **kw)
    assert own_grad.data_ptr() == own.data_ptr()
    assert torch.equal(own_loss, loss) and torch.equal(own_grad.float().nan_to_num(7.0), grad.float().nan_to_num(7.0))
    grad, loss, only = grad.double().cpu().numpy(), loss.double().cpu().numpy(), only.double().cpu().numpy()
    half = torch.finfo(DT[dtype]).eps / 2
    tiny = float(torch.finfo(DT[dtype]).tiny)
    for r in range(len(x)):
        want, dwant, slack, dslack = ref.distill(x[r], value[r], index[r], 1.0 if weight is None else float(weight[r]),
                                                 None if lse is None else float(lse[r]), ts, tt)
        for got in (loss[r], only[r]):
            assert got == want or abs(got - want) <= slack + 1e-12, (r, got, want, slack)
        off = np.abs(grad[r] - dwant) - (dslack + (half + 2.0 ** -23) * np.abs(dwant) + tiny)
        assert (off <= 0).all(), (r, int(off.argmax()), grad[r][off.argmax()], dwant[off.argmax()], float(off.max()))


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype,tdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,n,k", [(1, 1, 1), (3, 2, 1), (130, 30, 8), (5, 64, 64), (5, 65, 3), (7, 257, 300), (4, 1000, 1000),
                                      (3, 2049, 17), (9, 4099, 64), (2, 20_011, 1024), (1, 131_072, 50), (3, 70_001, 333),
                                      (600, 1031, 5)])
def test_distillation(B, rows, n, k, dtype, tdtype, rest):
    rng = np.random.default_rng(rows + n + k)
    for i in range(2):
        g, x = table(rng, rows, n, dtype, pad=[0, 3][i], sigma=[2.0, 0.2][i], shift=[0.0, 20.0][i])
        value, index, lse = entries(rng, x, k, tdtype, short=[0.0, 0.3][i])
        weight = rng.choice([0.0, 1.0, -0.5, 1.0 / rows], rows).astype(np.float32) if i else None
        check_distill(B, g, x, value, index, weight, lse if rest else None, tdtype, dtype)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("n,k", [(30, 7), (5000, 40), (90_001, 1000)])
def test_distillation_with_an_action_in_several_entries(B, n, k, rest):
    rng = np.random.default_rng(n)
    g, x = table(rng, 5, n, "f32")
    value, index, lse = entries(rng, x, k, "f32", short=0.1, repeated=True)
    check_distill(B, g, x, value, index, None, lse if rest else None, "f32", "f32")


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("n", [30, 1500, 80_000])
def test_distillation_of_masked_rows(B, n, rest):
    """Student's actions that are not allowed, teachers without entries, rows without either."""
    rng = np.random.default_rng(n)
    g, x = table(rng, 6, n, "f32")
    value, index, lse = entries(rng, x, 5, "f32", short=0.0)
    outside = [a for a in range(n) if a not in index[0]][:3]
    g[0, outside] = -INF                      # masked where the teacher names nothing
    g[1] = -INF                               # nothing allowed
    index[2] = -1                             # no entry
    value[3, 1:] = -INF                       # entries of no weight
    mask = np.ones(n, bool)
    mask[index[4]] = False
    g[4, torch.from_numpy(mask).cuda()] = -INF   # the student has nothing outside the entries
    g[5, int(index[5, 0])] = -INF             # no student mass where the teacher has some: loss infinite
    x = g.double().cpu().numpy()
    with np.errstate(divide="ignore"):
        check_distill(B, g, x, value, index, None, lse if rest else None, "f32", "f32")
    loss, grad = B.distill_grad(g, torch.from_numpy(value.astype(np.float32)).cuda(), torch.from_numpy(index).cuda(),
                                teacher_lse=torch.from_numpy(lse).cuda() if rest else None)
    assert loss[1] == 0 and not grad[1].any() and loss[2] == 0 and not grad[2].any()
    assert loss[5] == INF and torch.isfinite(grad).all() and (grad[0, outside] == 0).all()


@pytest.mark.parametrize("n", [30, 1500, 80_000])
def test_rows_of_weight_zero_are_not_read_and_nan_stays_in_its_row(B, n):
    rng = np.random.default_rng(n)
    g, x = table(rng, 4, n, "f32")
    value, index, lse = entries(rng, x, 5, "f32", short=0.0)
    clean = B.distill_grad(g, torch.from_numpy(value.astype(np.float32)).cuda(), torch.from_numpy(index).cuda())
    g[1] = math.nan
    g[2, n // 2] = math.nan
    weight = torch.tensor([1.0, 0.0, 1.0, 1.0], device="cuda")
    loss, grad = B.distill_grad(g, torch.from_numpy(value.astype(np.float32)).cuda(), torch.from_numpy(index).cuda(),
                                weight=weight)
    assert loss[1] == 0 and not grad[1].any()
    assert torch.isnan(loss[2]) and torch.isnan(grad[2]).all()
    for r in (0, 3):
        assert loss[r] == clean[0][r] and torch.equal(grad[r], clean[1][r])
    g[2] = g[0]
    g[2, 3] = INF
    loss, grad = B.distill_grad(g, torch.from_numpy(value.astype(np.float32)).cuda(), torch.from_numpy(index).cuda(),
                                weight=weight)
    assert torch.isnan(loss[2]) and torch.isnan(grad[2]).all()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,n,k", [(2, 30, 6), (2, 300, 20)])
def test_distillation_gradient_against_differences(B, rows, n, k, rest):
    """The gradient is the slope of the 64-bit loss: central differences with step h, whose error is h^2 / 6 of a
    third derivative of at most 2 / ts^3 and 2^-50 / h of rounding."""
    rng = np.random.default_rng(9)
    g, x = table(rng, rows, n, "f32")
    value, index, lse = entries(rng, x, k, "f32", short=0.0)
    value = value.astype(np.float32).astype(np.float64)
    _, grad = B.distill_grad(g, torch.from_numpy(value.astype(np.float32)).cuda(), torch.from_numpy(index).cuda(),
                             teacher_lse=torch.from_numpy(lse).cuda() if rest else None, student_temperature=1.1,
                             teacher_temperature=0.9)
    grad, h = grad.double().cpu().numpy(), 1e-4
    for r in range(rows):
        slack = ref.distill(x[r], value[r], index[r], 1.0, float(lse[r]) if rest else None, 1.1, 0.9)[3]
        for i in range(n):
            ends = []
            for sign in (1, -1):
                y = x[r].copy()
                y[i] += sign * h
                ends.append(ref.distill(y, value[r], index[r], 1.0, float(lse[r]) if rest else None, 1.1, 0.9)[0])
            slope = (ends[0] - ends[1]) / (2 * h)
            assert abs(grad[r, i] - slope) <= h * h / 2 + 2.0 ** -46 / h + slack[i] + 2.0 ** -22 * abs(slope), (r, i)


# ------------------------------------------------------------------------------------- as called
def test_nothing_is_done_for_no_rows(B):
    x = torch.empty((0, 30), device="cuda")
    index, logp = B.choose_actions(x, torch.empty(0, device="cuda"))
    assert len(index) == 0
    values, index, lse = B.top_actions(x, 4)
    assert values.shape == (0, 4)
    loss, grad = B.distill_grad(x, values, index)
    assert grad.shape == (0, 30) and len(loss) == 0


def test_rows_and_columns_beside_the_given_ones_are_left_as_they_were(B):
    rng = np.random.default_rng(2)
    for dtype in ("f32", "bf16"):
        for rows, n, k in ((5, 30, 4), (3, 777, 9), (2, 40_001, 33)):
            wide, _ = table(rng, rows + 2, n + 7, dtype)
            before = wide.clone()
            g = wide[1:-1, 3:n + 3]
            value, index, lse = B.top_actions(g, k)
            out = torch.full((rows + 2, n + 7), 5.0, dtype=DT[dtype], device="cuda")
            B.distill_grad(g, value, index, teacher_lse=lse, out=(torch.empty(rows, device="cuda"), out[1:-1, 3:n + 3]))
            assert torch.equal(wide, before)
            out[1:-1, 3:n + 3] = 5.0
            assert (out == 5.0).all()
            B.distill_grad(g, value, index, teacher_lse=lse, out=(torch.empty(rows, device="cuda"), g))
            wide[1:-1, 3:n + 3] = before[1:-1, 3:n + 3]
            assert torch.equal(wide, before)


def test_teacher_to_student_to_choice_captured_and_replayed(B):
    """A teacher's top actions distilled into a student and an action drawn from it, as one graph on a stream of
    its own, replayed over changing inputs with eager work in between, against eager calls."""
    torch.manual_seed(0)
    for rows, n, k, dtype in ((64, 30, 6, "f32"), (3, 60_001, 100, "bf16"), (300, 2001, 20, "f32")):
        teacher = torch.randn((rows, n), device="cuda").to(DT[dtype])
        student = torch.randn((rows, n), device="cuda").to(DT[dtype])
        u = torch.rand(rows, device="cuda")

        def calls(stream=None):
            value, index, lse = B.top_actions(teacher, k, temperature=0.5, stream=stream)
            loss, grad = B.distill_grad(student, value, index, teacher_lse=lse, teacher_temperature=0.5, stream=stream)
            act, logp = B.choose_actions(student, u, top_k=n // 2, top_p=0.9, stream=stream)
            act2, logp2 = B.choose_actions(student, u, temperature=0.8, stream=stream)
            return value, index, lse, loss, grad, act, logp, act2, logp2

        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = calls()
        for _ in range(4):
            teacher.copy_(torch.randn((rows, n), device="cuda"))
            student.copy_(torch.randn((rows, n), device="cuda"))
            u.copy_(torch.rand(rows, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            kept = [t.clone() for t in got]
            want = calls()
            side.wait_stream(torch.cuda.current_stream())
            other = calls(side)
            torch.cuda.synchronize()
            for a, b, c in zip(kept, want, other):
                assert torch.equal(a, b) and torch.equal(a, c)


def test_two_streams_at_once_do_not_disturb_each_other(B):
    torch.manual_seed(1)
    xs = [torch.randn((2, 90_000 + 100 * i), device="cuda") for i in range(2)]
    us = [torch.rand(2, device="cuda") for _ in range(2)]
    calls = lambda i, s: (*B.choose_actions(xs[i], us[i], top_p=0.9, stream=s), *B.top_actions(xs[i], 200, stream=s))
    want = [calls(i, None) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [calls(i, streams[i]) for i in range(2)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_the_same_call_gives_the_same_bits(B):
    torch.manual_seed(2)
    for rows, n, k in ((300, 5000, 200), (2, 131_072, 700)):
        x = torch.randn((rows, n), device="cuda")
        u = torch.rand(rows, device="cuda")
        value, index, lse = B.top_actions(x, k)
        y = torch.randn((rows, n), device="cuda")
        calls = lambda: (*B.choose_actions(x, u, top_p=0.9), *B.choose_actions(x, u), *B.top_actions(x, k),
                         *B.distill_grad(y, value, index, teacher_lse=lse))
        want = calls()
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(calls(), want))


def test_extreme_temperatures(B):
    """At the ends of the allowed range: the teacher's and the student's best actions alone, or all alike."""
    rng = np.random.default_rng(4)
    for n in (30, 3000, 50_000):
        g, x = table(rng, 3, n, "f32")
        value, index, _ = entries(rng, x, 4, "f32", short=0.0)
        tv, idx = torch.from_numpy(value.astype(np.float32)).cuda(), torch.from_numpy(index).cuda()
        loss, grad = B.distill_grad(g, tv, idx, student_temperature=1e30, teacher_temperature=1e30)
        # (uniform over the entries against uniform over n; the gradient, of size 1e-30, is a number)
        assert np.abs(loss.cpu().numpy() - math.log(n / 4)).max() <= 2.0 ** -22 * (math.log(n) + 4) and torch.isfinite(grad).all()
        loss, grad = B.distill_grad(g, tv, idx, student_temperature=1.0, teacher_temperature=1e-30)
        first = np.array([ref.log_sum_exp(r) - r[i] for r, i in zip(x, index[:, 0])])
        assert np.abs(loss.cpu().numpy() - first).max() <= 2.0 ** -22 * (math.log(n) + 4 + np.abs(first).max())
        # the student at its coldest: no loss where it agrees with a single entry, else the difference / 1e-30
        for at in (x.argmax(1), x.argmin(1)):
            loss, grad = B.distill_grad(g, tv[:, :1].contiguous(), torch.from_numpy(at.astype(np.int32))[:, None].cuda(),
                                        student_temperature=1e-30)
            far = (x.max(1) - x[np.arange(3), at]) / 1e-30
            assert np.abs(loss.double().cpu().numpy() - far).max() <= 2.0 ** -23 * far.max()
        for t in (1e-30, 1e30):
            _, top, lse = B.top_actions(g, 3, temperature=t)
            best = x.max(1)
            if t == 1e30:
                assert np.abs(lse.cpu().numpy() - math.log(n)).max() <= 2.0 ** -22 * (math.log(n) + 4)
            else:
                assert np.abs(lse.double().cpu().numpy() / (best / t) - 1).max() <= 2.0 ** -23
        for t in (1e-300, 1e-40, 1e40, 1e300):
            u = draw_u(rng, 3)
            index2, logp = B.choose_actions(g, torch.from_numpy(u).cuda(), temperature=t)
            check_choice(x, u, {"temperature": t}, index2, logp)


def test_settings_may_be_numbers_of_other_kinds(B):
    g, x = table(np.random.default_rng(3), 2, 40, "f32")
    u = torch.rand(2, device="cuda")
    a = B.choose_actions(g, u, temperature=1, top_k=np.int32(5), top_p=np.float32(0.5), min_p=0)
    b = B.choose_actions(g, u, temperature=1.0, top_k=5, top_p=0.5)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("rows,n", [(300_001, 30), (70_003, 70), (66_001, 300)])
def test_more_rows_than_a_launch_has_workgroups_in_a_row(B, rows, n):
    """Rows on both sides of 2^16 (and of 4 * 2^16, where a workgroup takes four): every row is done, and done as it would
    be on its own."""
    torch.manual_seed(n)
    x = torch.randn((rows, n), device="cuda")
    u = torch.rand(rows, device="cuda")
    some = torch.tensor([0, 1, 65_535, 65_536, 65_537, rows // 2, rows - 2, rows - 1], device="cuda")
    index, logp = B.choose_actions(x, u, top_p=0.9)
    value, top, lse = B.top_actions(x, 5)
    y = torch.randn((rows, n), device="cuda")
    loss, grad = B.distill_grad(y, value, top, teacher_lse=lse)
    pick = lambda t: t[some].contiguous()
    for got, want in ((index, B.choose_actions(pick(x), pick(u), top_p=0.9)[0]), (top, B.top_actions(pick(x), 5)[1]),
                      (grad, B.distill_grad(pick(y), pick(value), pick(top), teacher_lse=pick(lse))[1])):
        assert torch.equal(got[some], want)
    assert ((index >= 0) & (index < n)).all() and torch.equal(top[:, 0].long(), x.argmax(1))
    # (rows of a gradient sum to zero: n products of 32 bits, each off by some 2^-21 of itself)
    assert (grad.sum(1).abs() <= 2.0 ** -20 * grad.abs().sum(1) + 2.0 ** -21).all() and (loss > 0).all()


def test_a_table_beyond_4_gib(B):
    """Offsets of the last rows pass 32 bits, in elements and in bytes."""
    n = 262_144
    rows = (1 << 32) // n + 3
    x = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    x.normal_()
    u = torch.rand(rows, device="cuda")
    index, logp = B.choose_actions(x, u, top_k=20)
    i2, l2 = B.choose_actions(x, u, top_p=0.8)
    value, top, lse = B.top_actions(x, 16)
    last = slice(rows - 3, rows)
    few = x[last].clone()
    for how, got in (({"top_k": 20}, index), ({"top_p": 0.8}, i2)):
        assert torch.equal(B.choose_actions(few, u[last].clone(), **how)[0], got[last])
    check_choice(few.double().cpu().numpy(), u[last].cpu().numpy(), {"top_k": 20}, index[last], logp[last])
    check_choice(few.double().cpu().numpy(), u[last].cpu().numpy(), {"top_p": 0.8}, i2[last], l2[last])
    check_top(few.double().cpu().numpy(), 16, 1.0, value[last], top[last], lse[last])
    loss, grad = B.distill_grad(x, value, top, teacher_lse=lse, student_temperature=2.0)
    a, b = B.distill_grad(few, value[last].clone(), top[last].clone(), teacher_lse=lse[last].clone(), student_temperature=2.0)
    assert torch.equal(loss[last], a) and torch.equal(grad[last], b)


# ------------------------------------------------------------------------- on a trainer's own network
def trainer(B, dtype="f32", D=27, H=64, G=0, A=30, batch=64, dueling=False, layered=False, opt=None, seed=3, **kw):
    from paper_1801_03138_amd import synth
    st = B.RP_F32 if dtype == "f32" else B.RP_BF16
    ring = B.Replay(512, D, st, seed=seed)
    rows = synth.experiences(512, D, A, 0.02, seed=seed, state_dtype=dtype)
    ring.append(rows["s"], rows["s_next"], rows["a"], rows["r"], rows["term"])
    p = synth.init_params(D, H, A + (1 if dueling else 0), seed, hidden2=G or None)
    return B.Trainer(ring, H, A, batch, param_dtype=st, opt=B.RP_SGD if opt is None else opt, lr=1e-2, appends_per_step=0,
                     dueling=dueling, layered=layered, hidden2=G, init_params=p, **kw)


def network(params, D, H, G, A, dueling, X):
    """Q(s, .) with 64-bit torch tensors; params in the trainer's order, requiring gradients."""
    G, O = G or H, A + (1 if dueling else 0)
    at, parts = 0, []
    for shape in ((D, H), (H,), (H, G), (G,), (G, O), (O,)):
        n = int(np.prod(shape))
        parts.append(params[at:at + n].view(shape))
        at += n
    W1, b1, W2, b2, W3, b3 = parts
    h = torch.relu(torch.relu(X @ W1 + b1) @ W2 + b2)
    if not dueling:
        return h @ W3 + b3
    v = h[:, :G // 2] @ W3[:G // 2, :1] + b3[:1]
    a = h[:, G // 2:] @ W3[G // 2:, 1:] + b3[1:]
    return v + a - a.mean(dim=1, keepdim=True)


@pytest.mark.parametrize("dtype,H,G,A,dueling,layered", [
    ("f32", 64, 0, 30, False, False), ("f32", 128, 256, 30, True, False), ("f32", 320, 0, 100, False, False),
    ("f32", 64, 0, 5, True, True), ("bf16", 128, 0, 30, False, False), ("bf16", 64, 0, 30, True, True)])
def test_a_trainer_acts_with_its_network(B, dtype, H, G, A, dueling, layered):
    """Q-values to the rounding of the products (contractions of up to 320 terms in 32 bits, three of them: 2^-24 a term
    and product relative to the largest sum of magnitudes, here under 8 times the largest Q), choices as the
    definition has them on those Q-values, and nothing of the trainer changed."""
    tr = trainer(B, dtype, H=H, G=G, A=A, dueling=dueling, layered=layered, target_sync=3)
    for _ in range(4):
        tr.step()
    p, last = tr.params(), tr.last()
    rng = np.random.default_rng(0)
    for rows in (1, 3, 64, 517):
        s = torch.from_numpy(rng.normal(size=(rows, 27)).astype(np.float32)).to(DT[dtype]).cuda()
        u = draw_u(rng, rows)
        q = torch.empty((rows, A), device="cuda")
        how = {"temperature": 0.5, "top_k": 4, "top_p": 0.9}
        action, logp = tr.act(s, torch.from_numpy(u).cuda(), q=q, **how)
        again, _ = tr.act(s, torch.from_numpy(u).cuda(), **how)
        want = network(torch.from_numpy(p).double(), 27, H, G, A, dueling, s.double().cpu()).numpy()
        got = q.double().cpu().numpy()
        assert np.abs(got - want).max() <= 8 * 2.0 ** -24 * (27 + H + (G or H)) * np.abs(want).max()
        check_choice(got, u, how, action, logp)
        assert torch.equal(action, again)
        best, _ = tr.act(s, torch.from_numpy(u).cuda(), temperature=0.0)
        assert np.array_equal(best.cpu().numpy(), got.argmax(1))
    assert np.array_equal(tr.params(), p)
    now = tr.last()
    assert all(np.array_equal(now[k], last[k]) for k in ("Q", "y", "delta", "idx")) and now["loss"] == last["loss"]


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype,G,A,dueling", [("f32", 0, 30, False), ("f32", 128, 30, True), ("f32", 0, 300, False),
                                               ("bf16", 0, 30, False)])
def test_a_step_on_a_teachers_actions(B, dtype, G, A, dueling, rest):
    """The step's gradient against automatic differentiation of the same loss in 64 bits, its update against that gradient.
    Sums of up to D + H + G + B terms in 32 bits: 2^-24 a term, relative to sums of magnitudes of up to 4 times the largest
    entry.  bf16: six roundings to 2^-8 on the way (states' and weights' are in the reference too), twice that for units
    at the kink."""
    D, H, batch, k = 27, 64, 64, 6
    tr = trainer(B, dtype, G=G, A=A, dueling=dueling, layered=True)
    rng = np.random.default_rng(A)
    s = torch.from_numpy(rng.normal(size=(batch, D)).astype(np.float32)).to(DT[dtype]).cuda()
    t = rng.normal(0, 1, (batch, A)).astype(np.float32)
    index = np.argsort(-t, axis=1)[:, :k].astype(np.int32)
    index[::7, -1] = -1
    value = np.take_along_axis(t, np.maximum(index, 0), 1)
    lse = np.array([ref.log_sum_exp(r, 0.5) for r in t], np.float32)
    weight = rng.uniform(0.5, 1.5, batch).astype(np.float32)
    weight[5] = 0.0
    p0 = tr.params()
    cuda = lambda v: torch.from_numpy(v).cuda()
    tr.distill_batch(s, cuda(value), cuda(index), weight=cuda(weight), teacher_lse=cuda(lse) if rest else None,
                     student_temperature=0.7, teacher_temperature=0.5)
    # the reference
    p = torch.from_numpy(p0)
    p = (p.to(torch.bfloat16) if dtype == "bf16" else p).double().requires_grad_()
    z = network(p, D, H, G, A, dueling, s.double().cpu()) / 0.7
    log_p = torch.log_softmax(z, dim=1)
    there = torch.from_numpy(index >= 0)
    tt = torch.from_numpy(value).double() / 0.5
    tt = torch.where(there, tt, -INF)
    log_q = tt - torch.from_numpy(lse).double()[:, None] if rest else torch.log_softmax(tt, dim=1)
    q = log_q.exp()
    at = torch.from_numpy(np.maximum(index, 0)).long()
    picked = torch.gather(log_p, 1, at)
    loss = torch.where(there, q * (torch.where(there, log_q, 0.0) - picked), 0.0).sum(1)
    if rest:
        q_rest = 1 - q.sum(1)
        p_rest = 1 - torch.where(there, picked.exp(), 0.0).sum(1)
        loss = loss + q_rest * (q_rest.log() - p_rest.log())
    loss = (loss * torch.from_numpy(weight).double()).mean()
    loss.backward()
    want, got = p.grad.numpy(), tr.grads()
    tol = 4 * 2.0 ** -24 * (D + H + (G or H) + batch + A) if dtype == "f32" else 12 * 2.0 ** -8
    assert np.abs(got - want).max() <= tol * np.abs(want).max()
    last = tr.last()
    # (32 bits: each row's loss to 2^-22 (log A + 4) of its size and the Q-values' error of before)
    q_off = 8 * 2.0 ** -24 * (D + H + (G or H)) if dtype == "f32" else 6 * 2.0 ** -8
    assert abs(last["loss"] - loss.item()) <= 2.0 ** -22 * (math.log(A) + 4) + 4 * q_off * np.abs(last["Q"]).max() / 0.7
    step = np.float32(1e-2) * got
    assert np.abs(tr.params() - (p0 - step)).max() <= 2.0 ** -23 * np.abs(p0).max()
    assert tr.opt_state()[2:] == (1, 1)
    # the trainer goes on: a TD step after it counts on
    assert tr.step() == 0 and tr.opt_state()[2:] == (2, 2)


def test_adam_on_a_teachers_actions_counts_its_steps(B):
    """Two steps of Adam from its own definition on the gradients the trainer reports."""
    tr = trainer(B, layered=True, opt=B.RP_ADAM)
    s = torch.randn((64, 27), device="cuda")
    value, index, lse = B.top_actions(torch.randn((64, 30), device="cuda"), 5)
    m = v = 0.0
    p = tr.params().astype(np.float64)
    for t in (1, 2):
        tr.distill_batch(s, value, index, teacher_lse=lse)
        g = tr.grads().astype(np.float64)
        m, v = 0.9 * m + 0.1 * g, 0.999 * v + 0.001 * g * g
        step = 1e-2 * (m / (1 - 0.9 ** t)) / (np.sqrt(v / (1 - 0.999 ** t)) + 1e-8)
        # (moments, corrections, root and quotient in 32 bits: under 16 roundings of the step, and 1 - 0.999 in
        # 32 bits is 0.001 to 2^-24 / 0.001 of itself, under the root)
        assert np.abs(tr.params() - (p - step)).max() <= 1e-2 * (16 * 2.0 ** -24 + 2.0 ** -24 / 0.001) * 1.01 + 2.0 ** -24 * np.abs(p).max()
        p = tr.params().astype(np.float64)
        assert tr.opt_state()[2] == t


def test_teacher_and_student_together(B):
    """A teacher acts on states drawn from its replay, its top actions train a student, which acts in turn: each loss is
    the operator's on the student's Q-values of before, to the rounding of those."""
    teacher = trainer(B, H=128, seed=1)
    student = trainer(B, H=64, layered=True, seed=2)
    for _ in range(10):
        teacher.step()
    u = torch.rand(64, device="cuda")
    for step in range(5):
        _, (s, *_) = teacher.replay.sample_gather(step, 64)
        q, z = torch.empty((64, 30), device="cuda"), torch.empty((64, 30), device="cuda")
        teacher.act(s, u, q=q)
        value, index, lse = B.top_actions(q, 8, temperature=0.3)
        before, _ = student.act(s, u, q=z)
        want = B.distill_loss(z, value, index, teacher_lse=lse, teacher_temperature=0.3).mean().item()
        student.distill_batch(s, value, index, teacher_lse=lse, teacher_temperature=0.3)
        scale = 1 + z.abs().max().item()
        assert abs(student.last()["loss"] - want) <= 16 * 2.0 ** -24 * (27 + 64 + 64) * scale
        action, logp = student.act(s, u, temperature=0.3, top_k=8)
        assert ((action >= 0) & (action < 30)).all() and (logp <= 0).all()


def test_paths_refuse_what_they_cannot_do(B):
    fast, slow = trainer(B), trainer(B, layered=True)
    s = torch.randn((64, 27), device="cuda")
    value, index, lse = B.top_actions(torch.randn((64, 30), device="cuda"), 5)
    with pytest.raises(B.ReplayError, match="LAYERED"):
        fast.distill_batch(s, value, index)
    before = slow.params()
    for bad in (dict(s=s[:63]), dict(s=s.double()), dict(index=index[:63]), dict(index=index.long()), dict(teacher=value.half()),
                dict(weight=torch.ones(63, device="cuda")), dict(teacher_lse=lse.double())):
        with pytest.raises(ValueError):
            slow.distill_batch(**{"s": s, "teacher": value, "index": index, **bad})
    for bad in (dict(student_temperature=0.0), dict(teacher_temperature=math.nan)):
        with pytest.raises(B.ReplayError):
            slow.distill_batch(s, value, index, **bad)
    u = torch.rand(64, device="cuda")
    for bad in (dict(s=s[:63]), dict(s=s.bfloat16()), dict(q=torch.empty((64, 29), device="cuda")),
                dict(temperature=torch.ones(63, device="cuda"))):
        with pytest.raises(ValueError):
            slow.act(**{"s": s, "u": u, **bad})
    with pytest.raises(B.ReplayError):
        slow.act(s[:0], u[:0])
    assert np.array_equal(slow.params(), before) and slow.opt_state()[2:] == (0, 0)


# ------------------------------------------------------------------------- lengths where a row is just not cut
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(1, 8193), (2, 10_001), (128, 12_289), (129, 10_001), (3, 16_383), (3, 16_385), (2, 32_767)])
def test_rows_next_to_the_lengths_where_they_are_cut(B, rows, n, dtype):
    rng = np.random.default_rng(n + rows)
    g, x = table(rng, rows, n, dtype, pad=1, sigma=2.0, masked=0.1)
    u = draw_u(rng, rows)
    for how in ({"top_p": 0.9, "min_p": 0.001}, {"top_k": 40, "temperature": 0.7}, {"temperature": 0.0}):
        check_choice(x, u, how, *B.choose_actions(g, torch.from_numpy(u).cuda(), **how))
    check_top(x, 33, 0.7, *B.top_actions(g, 33, temperature=0.7))


@pytest.mark.parametrize("n", [20_000, 262_144])
def test_nothing_is_done_for_no_long_rows(B, n):
    x = torch.empty((0, n), device="cuda")
    assert len(B.choose_actions(x, torch.empty(0, device="cuda"))[0]) == 0
    value, index, lse = B.top_actions(x, 4)
    assert len(B.distill_loss(x, value, index, teacher_lse=lse)) == 0
    assert B.distill_grad(x, value, index)[1].shape == (0, n)


# ----------------------------------------------------------------- a student that is sure of the teacher's actions
def far_rows(rng, rows, n, k, dtype, ts, gap, mass):
    """A student whose logits at the k named actions lie around `gap` temperatures above the others; a teacher with
    about `mass` of its own on them."""
    x = rng.normal(0, 1, (rows, n)) * min(1.0, 5 * ts)
    index = np.stack([rng.permutation(n)[:k] for _ in range(rows)]).astype(np.int32)
    np.put_along_axis(x, index, np.take_along_axis(x, index, 1) + gap * ts, 1)
    g = torch.from_numpy(x.astype(np.float32)).to(DT[dtype]).cuda()
    t = rng.normal(0, 1, (rows, k)).astype(np.float32)
    lse = np.array([ref.log_sum_exp(r, 0.9) - math.log(mass) for r in t], np.float32)
    return g, g.double().cpu().numpy(), t, index, lse


def check_far(B, g, x, t, index, lse, dtype, ts, weight=None, tt=0.9):
    cuda = lambda v: None if v is None else torch.from_numpy(v).cuda()
    kw = dict(weight=cuda(weight), teacher_lse=cuda(lse), student_temperature=ts, teacher_temperature=tt)
    only = B.distill_loss(g, cuda(t), cuda(index), **kw)
    loss, grad = B.distill_grad(g, cuda(t), cuda(index), **kw)
    own = g.clone()
    own_loss, _ = B.distill_grad(own, cuda(t), cuda(index), out=(torch.empty_like(loss), own), **kw)
    assert torch.isfinite(grad).all() and torch.equal(own, grad) and torch.equal(own_loss, loss)
    loss, only, grad = loss.double().cpu().numpy(), only.double().cpu().numpy(), grad.double().cpu().numpy()
    half, tiny = torch.finfo(DT[dtype]).eps / 2, float(torch.finfo(DT[dtype]).tiny)
    for r in range(len(x)):
        want, dwant, slack, dslack = ref.distill_rest(x[r], t[r], index[r], float(lse[r]), ts, tt,
                                                      1.0 if weight is None else float(weight[r]))
        assert max(abs(loss[r] - want), abs(only[r] - want)) <= slack, (r, loss[r], only[r], want, slack)
        off = np.abs(grad[r] - dwant) - (dslack + (half + 2.0 ** -23) * np.abs(dwant) + tiny)
        assert (off <= 0).all(), (r, int(off.argmax()), grad[r][off.argmax()], dwant[off.argmax()], float(off.max()))


FAR_SHAPES = [(3, 30, 8), (3, 200, 20), (40, 1500, 20), (3, 5000, 1000), (33, 20_011, 64), (2, 30_000, 50), (130, 70_001, 9),
              (3, 80_000, 300)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,k", FAR_SHAPES)
def test_the_rest_far_below_the_entries(B, rows, n, k, dtype):
    """On both sides of the distances at which sums start anew, 32 bits end, and numbers below the normal ones."""
    rng = np.random.default_rng(n)
    for i, gap in enumerate((-20, 0, 30, 44, 60, 86, 90, 104, 300, 680) if rows * n < 2 ** 20 else (44, 60, 90, 680)):
        ts = [1.1, 0.1, 0.01][i % 3]
        g, x, t, index, lse = far_rows(rng, rows, n, k, dtype, ts, gap, [0.6, 0.95, 0.05, 1.2][i % 4])
        weight = None if i % 2 else rng.choice([1.0, -0.5, 1.0 / rows], rows).astype(np.float32)
        check_far(B, g, x, t, index, lse, dtype, ts, weight)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [30, 1500, 80_000])
def test_a_cold_student_of_ordinary_logits(B, n, dtype):
    """Unit normal logits at low temperatures, entries anywhere among them."""
    rng = np.random.default_rng(n + 1)
    g, x = table(rng, 40 if n < 10_000 else 4, n, dtype, sigma=1.0)
    index = np.argsort(-x + rng.normal(0, 0.3, x.shape), axis=1)[:, :4].astype(np.int32)
    t = rng.normal(0, 1, index.shape).astype(np.float32)
    lse = np.array([ref.log_sum_exp(r, 0.9) + 0.3 for r in t], np.float32)
    for ts in (0.1, 0.02, 0.01):
        check_far(B, g, x, t, index, lse, dtype, ts)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_cold_student_trains(B, dtype):
    """A layered step whose Q-values span some 600 student temperatures, the teacher's actions the best of them, backward
    from the gradient that these very Q-values have by definition: to the tolerances of the step's products, and in mixed
    precision of its roundings."""
    D, H, batch, A, k = 27, 64, 64, 30, 6
    tr = trainer(B, dtype, layered=True)
    rng = np.random.default_rng(8)
    s = torch.from_numpy(rng.normal(size=(batch, D)).astype(np.float32)).to(DT[dtype]).cuda()
    t = rng.normal(0, 1, (batch, k)).astype(np.float32)
    lse = np.array([ref.log_sum_exp(r, 0.5) + 0.5 for r in t], np.float32)
    p0, cuda = tr.params(), lambda v: torch.from_numpy(v).cuda()
    q = torch.empty((batch, A), device="cuda")
    tr.act(s, torch.rand(batch, device="cuda"), q=q)
    ts = float((q.max(1).values - q.min(1).values).max()) / 600
    index = B.top_actions(q, k)[1].cpu().numpy()
    tr.distill_batch(s, cuda(t), cuda(index), teacher_lse=cuda(lse), student_temperature=ts, teacher_temperature=0.5)
    q = np.asarray(tr.last()["Q"], np.float64).reshape(-1, A)[:batch]
    rows = [ref.distill_rest(q[i], t[i], index[i], float(lse[i]), ts, 0.5) for i in range(batch)]
    p = torch.from_numpy(p0)
    p = (p.to(torch.bfloat16) if dtype == "bf16" else p).double().requires_grad_()
    z = network(p, D, H, 0, A, False, s.double().cpu())
    (z * torch.from_numpy(np.stack([r[1] for r in rows]) / batch)).sum().backward()
    got, want = tr.grads(), p.grad.numpy()
    assert np.isfinite(got).all() and np.isfinite(tr.params()).all()
    tol = 4 * 2.0 ** -24 * (D + 2 * H + batch + A) if dtype == "f32" else 12 * 2.0 ** -8
    assert np.abs(got - want).max() <= tol * np.abs(want).max()
    loss = np.mean([r[0] for r in rows])
    assert abs(tr.last()["loss"] - loss) <= max(r[2] for r in rows) + 2.0 ** -22 * abs(loss)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,k", FAR_SHAPES)
def test_a_rest_below_the_numbers_of_64_bits(B, rows, n, k, dtype):
    """The student's probability of the rest is no number any more; its logarithm is, and pulls."""
    rng = np.random.default_rng(n + 2)
    for i, (ts, gap) in enumerate(((1.1, 740), (0.01, 800), (1e-3, 5000), (1e-3, 1e5))):
        g, x, t, index, lse = far_rows(rng, rows, n, k, dtype, ts, gap, [0.6, 0.95, 0.05, 1.2][i])
        check_far(B, g, x, t, index, lse, dtype, ts)
    g, x, t, index, lse = far_rows(rng, rows, n, k, dtype, 1.0, 3, 0.7)
    check_far(B, g, x, t, index, lse, dtype, 1e-30)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [40, 65, 5000, 12_000, 50_000])
def test_random_numbers_outside_the_unit_interval_are_its_ends_at_every_length(B, n, dtype):
    """No number and negative ones choose the first action, one and more the last that stays, however small its weight."""
    rng = np.random.default_rng(n)
    u = np.array([math.nan, -1.0, 0.0, 1.0, 7.0, INF], np.float32)
    for i, how in enumerate(({}, {"top_p": 0.9}, {"min_p": 0.02}, {"top_p": 0.6, "min_p": 0.02}, {"top_k": 7}, {"top_k": 1500},
                             {"top_k": 1500, "top_p": 0.9, "min_p": 0.001}, {"temperature": 0.05}, {"temperature": 1e-3, "top_p": 0.99},
                             {"temperature": 50.0, "min_p": 0.9}, {"temperature": 0.0})):
        g, x = table(rng, len(u), n, dtype, pad=1, sigma=[2.0, 0.4][i % 2], masked=[0.0, 0.3][i % 2])
        index, logp = B.choose_actions(g, torch.from_numpy(u).cuda(), **how)
        for r in range(len(u)):
            ids, c, at = ref.choose(x[r], float(u[r]), **how)
            assert at == (len(ids) - 1 if u[r] >= 1 else 0) and int(index[r]) == ids[at], (how, r, int(index[r]), ids[at])
        assert torch.isfinite(logp).all()


def test_tables_of_another_shape_are_refused(B):
    x = torch.randn((6, 30), device="cuda")
    value, index, lse = B.top_actions(x, 4)
    flip = lambda t: t.reshape(4, 6)
    for call in (lambda: B.distill_loss(x, flip(value), index), lambda: B.distill_grad(x, flip(value), index),
                 lambda: B.distill_loss(x, value, flip(index)), lambda: B.top_actions(x, 4, out=(flip(value), index, lse)),
                 lambda: B.top_actions(x, 4, out=(value, flip(index), lse))):
        with pytest.raises(ValueError):
            call()
    tr = trainer(B, layered=True)
    s, u = torch.randn((6, 27), device="cuda"), torch.rand(6, device="cuda")
    with pytest.raises(ValueError):
        tr.act(s, u, q=torch.empty((30, 6), device="cuda"))
    flat = B.top_actions(x, 4, out=(torch.empty(24, device="cuda"), torch.empty(24, dtype=torch.int32, device="cuda"), lse))
    assert torch.equal(flat[0].view(6, 4), value) and torch.equal(flat[1].view(6, 4), index)


def test_logits_that_autograd_watches(B):
    """They are taken by their values: what comes back takes no part in automatic differentiation."""
    x = torch.randn((5, 300), device="cuda")
    value, index, lse = B.top_actions(x, 4)
    y = torch.randn((5, 300), device="cuda")
    want = B.distill_grad(y, value, index, teacher_lse=lse)
    y.requires_grad_()
    loss, grad = B.distill_grad(y, value, index, teacher_lse=lse)
    assert not loss.requires_grad and not grad.requires_grad and torch.equal(loss, want[0]) and torch.equal(grad, want[1])
    assert not B.distill_loss(y, value, index, teacher_lse=lse).requires_grad
    y.backward(grad)   # as a program hands it on
    assert torch.equal(y.grad, grad)


@pytest.mark.parametrize("n", [30, 1500, 80_000])
def test_a_cold_teacher(B, n):
    """A log-sum-exp of thousands, in 32 bits: the loss and the gradient are those of this very number, of which the rest
    is a small remainder."""
    rng = np.random.default_rng(n + 3)
    x, xs = table(rng, 6, n, "f32", sigma=1.0, shift=20.0)
    g, gs = table(rng, 6, n, "f32", sigma=1.0)
    for tt in (0.1, 0.01):
        value, index, lse = B.top_actions(x, 8, temperature=tt)
        for r in range(6):
            assert abs(float(lse[r]) - ref.log_sum_exp(xs[r], tt)) <= 2.0 ** -23 * float(lse[r]) + 2.0 ** -22 * (math.log(n) + 4)
        check_far(B, g, gs, value.cpu().numpy(), index.cpu().numpy(), lse.cpu().numpy(), "f32", 1.0, tt=tt)


@pytest.mark.parametrize("dtype,H,G,A,batch,dueling,kw", [
    ("f32", 64, 0, 30, 64, True, {}), ("f32", 256, 0, 30, 128, True, {"target_sync": 2}), ("f32", 256, 0, 30, 128, False, {}),
    ("f32", 128, 1024, 31, 32, False, {"target_sync": 3}), ("bf16", 128, 0, 30, 64, True, {"target_sync": 2}),
    ("bf16", 256, 128, 40, 512, False, {}), ("f32", 64, 0, 1, 64, False, {}), ("f32", 64, 0, 4096, 16, False, {})])
def test_a_trainer_acts_after_a_run_of_steps(B, dtype, H, G, A, batch, dueling, kw):
    """Q-values of the weights that the trainer reports, after single steps and after a run of them in one call, on a stream
    of its own too; the bounds are those of test_a_trainer_acts_with_its_network."""
    tr = trainer(B, dtype, H=H, G=G, A=A, batch=batch, dueling=dueling, **kw)
    side = torch.cuda.Stream()
    rng = np.random.default_rng(H + A)
    for count in (1, 7, 40):
        if count == 1:
            assert tr.step() == 0
        else:
            assert tr.steps(count) == count
        torch.cuda.synchronize()
        s = torch.from_numpy(rng.normal(size=(130, 27)).astype(np.float32)).to(DT[dtype]).cuda()
        u = torch.from_numpy(draw_u(rng, 130)).cuda()
        q = torch.empty((130, A), device="cuda")
        torch.cuda.synchronize()
        action, logp = tr.act(s, u, temperature=0.3, q=q, stream=side)
        torch.cuda.synchronize()
        p = tr.params()
        want = network(torch.from_numpy(p).double(), 27, H, G, A, dueling, s.double().cpu()).numpy()
        got = q.double().cpu().numpy()
        assert np.abs(got - want).max() <= 8 * 2.0 ** -24 * (27 + H + (G or H)) * np.abs(want).max()
        check_choice(got, u.cpu().numpy(), {"temperature": 0.3}, action, logp)


def test_a_run_of_steps_after_steps_on_a_teachers_actions(B):
    """Steps on a teacher's actions between runs of TD steps in one call: sampling and optimizer go on where single steps
    would, to the same weights."""
    value, index, lse = B.top_actions(torch.randn((64, 30), device="cuda"), 5)
    s = torch.randn((64, 27), device="cuda")
    ends = []
    for one_call in (False, True):
        tr = trainer(B, layered=True, opt=B.RP_ADAM, target_sync=3)
        for _ in range(2):
            if one_call:
                assert tr.steps(5) == 5
            else:
                for _ in range(5):
                    assert tr.step() == 0
            tr.distill_batch(s, value, index, teacher_lse=lse)
        assert tr.opt_state()[2:] == (12, 12)
        ends.append((tr.params(), tr.target()))
    assert np.array_equal(ends[0][0], ends[1][0]) and np.array_equal(ends[0][1], ends[1][1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_top_p_of_equal_logits_ends_where_it_should(B, dtype):
    """A constant row (an untrained network's): whole numbers, a nucleus of exactly p n actions, with and without actions
    that are not allowed or 60 temperatures below."""
    last = torch.tensor([1 - 2.0 ** -24, 0.0, 0.5], device="cuda")
    for n in (30, 64, 66, 100, 160, 1000, 2048, 2052, 10_000, 60_000):
        for value in (0.0, -3.7, 1.25, 1e6):
            x = torch.full((3, n), value, device="cuda").to(DT[dtype])
            for how, kept in (({"top_p": 0.5}, (n + 1) // 2), ({"top_p": 0.25, "temperature": 0.7}, (n + 3) // 4),
                              ({"top_p": 0.75, "min_p": 0.5}, (3 * n + 3) // 4), ({"min_p": 1.0}, n), ({"min_p": 1.5}, 1), ({}, n)):
                index, logp = B.choose_actions(x, last, **how)
                assert index.tolist() == [kept - 1, 0, kept // 2 if kept > 1 else 0], (n, value, how)
                assert (logp.double() + math.log(kept)).abs().max().item() <= 2.0 ** -23 * math.log(kept) + 1e-12
            for off in (-INF, value - 60 - abs(value) * 0.1):
                y = x.clone()
                y[:, ::2] = off
                kept = (n // 2 + 1) // 2
                index, _ = B.choose_actions(y, last, top_p=0.5)
                assert index.tolist() == [2 * kept - 1, 1, 2 * (kept // 2) + 1 if kept > 1 else 1], (n, value, off)


def test_settings_of_rows_that_go_in_several_launches(B):
    """More rows than the workspace has pieces for at once: each with its own settings, on both sides of the cut, as on its own."""
    rows, n = 2800, 40_001
    torch.manual_seed(11)
    x, u = torch.randn((rows, n), device="cuda").mul_(2.0), torch.rand(rows, device="cuda")
    pick = lambda v, dtype=torch.float32: torch.tensor(v, dtype=dtype, device="cuda")[torch.randint(0, len(v), (rows,), device="cuda")]
    how = {"temperature": pick([0.0, 0.7, 1.0, 1.5]), "top_k": pick([0, 0, 3, 40, 900], torch.int32),
           "top_p": pick([0.5, 0.9, 1.0]), "min_p": pick([0.0, 0.01, 0.1])}
    index, logp = B.choose_actions(x, u, **how)
    value, top, lse = B.top_actions(x, 7)
    some = torch.cat([torch.arange(0, 5), torch.arange(2700, 2760), torch.arange(rows - 5, rows)]).cuda()
    part = {k: v[some].contiguous() for k, v in how.items()}
    few = x[some].contiguous()
    check_choice(few.double().cpu().numpy(), u[some].cpu().numpy(), {k: v.cpu().numpy() for k, v in part.items()}, index[some], logp[some])
    check_top(few.double().cpu().numpy(), 7, 1.0, value[some], top[some], lse[some])
