"""What the operators on rows of logits refuse, before anything is launched.  Runs without a GPU."""
import ctypes as C
import math

import pytest
import torch

from paper_1801_03138_amd import binding as B

EINVAL = B.RP_EINVAL
P = 0x1000   # an address that is never followed: every call below is refused first


def rows(**kw):
    d = dict(data=P, rows=4, stride=30, n=30, dtype=B.RP_F32)
    d.update(kw)
    return B.LogitRows(d["data"], d["rows"], d["stride"], d["n"], d["dtype"])


def teacher(**kw):
    d = dict(value=P, index=P, lse=None, weight=None, k=8, dtype=B.RP_F32, temperature=1.0, student_temperature=1.0)
    d.update(kw)
    return B.Teacher(*(d[f] for f, _ in B.Teacher._fields_))


BAD_ROWS = [dict(n=0), dict(n=262_145), dict(rows=2 ** 24 + 1), dict(dtype=B.RP_U8), dict(dtype=7), dict(stride=2 ** 41)]


def choose(x, how=True, u=P, index=P):
    how = B.Choice(1.0, 1.0, 0.0, 0, None, None, None, None) if how else None
    return B.lib().rp_choose_actions(C.byref(x) if x else None, C.byref(how) if how else None, u, index, None, None, 0, None)


def top(x, k=4, temperature=1.0, values=P, index=P):
    return B.lib().rp_top_actions(C.byref(x) if x else None, k, temperature, values, index, None, None, 0, None)


def loss(x, t, out=P):
    return B.lib().rp_distill_loss(C.byref(x) if x else None, C.byref(t) if t else None, out, None, 0, None)


def grad(x, t, out=P, g=0x100000, stride=30):
    return B.lib().rp_distill_grad(C.byref(x) if x else None, C.byref(t) if t else None, out, g, stride, None, 0, None)


@pytest.mark.parametrize("bad", BAD_ROWS + [dict(data=None), dict(data=P + 2)])
def test_rows_that_cannot_be_read_are_refused(bad):
    for st in (choose(rows(**bad)), top(rows(**bad)), loss(rows(**bad), teacher()), grad(rows(**bad), teacher())):
        assert st == EINVAL
    assert b"rp_distill_grad" in B.lib().rp_last_error()


@pytest.mark.parametrize("bad", BAD_ROWS)
def test_invalid_rows_have_no_workspace_size(bad):
    x = rows(**bad)
    none = C.c_size_t(-1).value
    lib = B.lib()
    assert lib.rp_choose_workspace_bytes(C.byref(x)) == none
    assert lib.rp_top_workspace_bytes(C.byref(x), 4) == none
    assert lib.rp_distill_workspace_bytes(C.byref(x), 4) == none
    good = rows()
    assert lib.rp_choose_workspace_bytes(C.byref(good)) != none
    for k, ok in ((0, False), (1, True), (30, True), (31, False), (1025, False)):
        assert (lib.rp_top_workspace_bytes(C.byref(good), k) != none) == ok
    for k, ok in ((0, False), (1, True), (31, True), (1024, True), (1025, False)):
        assert (lib.rp_distill_workspace_bytes(C.byref(good), k) != none) == ok


def test_null_arguments_are_refused():
    assert choose(None) == EINVAL and choose(rows(), how=False) == EINVAL and choose(rows(), u=None) == EINVAL
    assert choose(rows(), index=None) == EINVAL
    assert top(None) == EINVAL and top(rows(), values=None) == EINVAL and top(rows(), index=None) == EINVAL
    assert loss(None, teacher()) == EINVAL and loss(rows(), None) == EINVAL and loss(rows(), teacher(), out=None) == EINVAL
    assert loss(rows(), teacher(value=None)) == EINVAL and loss(rows(), teacher(index=None)) == EINVAL
    assert grad(rows(), teacher(), g=None) == EINVAL


def test_settings_out_of_range_are_refused():
    for k in (0, 31, 1025):
        assert top(rows(), k=k) == EINVAL
    assert top(rows(n=4000, stride=4000), k=1025) == EINVAL
    for t in (0.0, -1.0, math.inf, math.nan, 1e-31, 1e31):
        assert top(rows(), temperature=t) == EINVAL
        assert loss(rows(), teacher(temperature=t)) == EINVAL
        assert grad(rows(), teacher(student_temperature=t)) == EINVAL
    for bad in (dict(k=0), dict(k=1025), dict(dtype=B.RP_U8)):
        assert loss(rows(), teacher(**bad)) == EINVAL and grad(rows(), teacher(**bad)) == EINVAL


def test_gradients_that_would_overwrite_something_else_are_refused():
    x, t = rows(data=0x10000, rows=4, stride=32), teacher()
    bytes_ = ((4 - 1) * 32 + 30) * 4
    assert grad(x, t, g=0x10000 + 4, stride=32) == EINVAL            # shifted against the logits
    assert grad(x, t, g=0x10000, stride=40) == EINVAL                # in place, another stride
    assert grad(x, t, g=0x10000 + bytes_ - 4, stride=32) == EINVAL   # its first element on the logits' last
    assert grad(x, t, g=0x10000 - bytes_ + 4, stride=32) == EINVAL
    assert grad(x, t, stride=29) == EINVAL                           # rows of the gradient overlap
    assert grad(x, t, g=0x100002) == EINVAL                          # not aligned
    assert grad(x, t, stride=2 ** 41) == EINVAL
    assert grad(rows(data=0x10000, stride=0), t, g=0x10000, stride=30) == EINVAL   # in place of a broadcast row


def test_no_rows_are_no_work():
    assert choose(rows(rows=0, data=None)) == 0 and top(rows(rows=0, data=None)) == 0
    assert loss(rows(rows=0, data=None), teacher()) == 0 and grad(rows(rows=0, data=None), teacher()) == 0


def test_the_binding_checks_tensors():
    x = torch.zeros(4, 30)
    with pytest.raises(ValueError, match="not on the GPU"):
        B.choose_actions(x, torch.zeros(4))
    for bad in (torch.zeros(30), torch.zeros(4, 30, dtype=torch.float64), torch.zeros(4, 30, dtype=torch.float16),
                torch.zeros(30, 4).t(), torch.zeros(4, 60)[:, ::2], None):
        with pytest.raises(ValueError):
            B.check_rows(bad, "t", "cpu")
    for good in (x, torch.zeros(4, 32)[:, 1:31], torch.zeros(1, 30).expand(4, 30), torch.zeros(30, 1), torch.zeros(8, 30)[::2],
                 x.bfloat16()):
        B.check_rows(good, "t", "cpu")
    cpu = torch.device("cpu")
    assert B.check_setting(0.5, torch.float32, 4, cpu, "t") == (0.5, None)
    v = torch.zeros(4)
    assert B.check_setting(v, torch.float32, 4, cpu, "t") == (None, v)
    for bad in (torch.zeros(3), torch.zeros(4, dtype=torch.float64), torch.zeros(8)[::2]):
        with pytest.raises(ValueError):
            B.check_setting(bad, torch.float32, 4, cpu, "t")


def test_a_workspace_that_is_too_small_is_refused():
    lib = B.lib()
    x = rows(rows=2, n=200_000, stride=200_000)
    how = B.Choice(1.0, 1.0, 0.0, 0, None, None, None, None)
    for need, call in ((lib.rp_choose_workspace_bytes(C.byref(x)),
                        lambda ws, b: lib.rp_choose_actions(C.byref(x), C.byref(how), P, P, None, ws, b, None)),
                       (lib.rp_top_workspace_bytes(C.byref(x), 8),
                        lambda ws, b: lib.rp_top_actions(C.byref(x), 8, 1.0, P, P, None, ws, b, None)),
                       (lib.rp_distill_workspace_bytes(C.byref(x), 8),
                        lambda ws, b: lib.rp_distill_loss(C.byref(x), C.byref(teacher()), P, ws, b, None)),
                       (lib.rp_distill_workspace_bytes(C.byref(x), 8),
                        lambda ws, b: lib.rp_distill_grad(C.byref(x), C.byref(teacher()), P, 0x10000000, 200_000, ws, b, None))):
        assert need > 0
        assert call(None, 0) == B.RP_ENOMEM and call(0x1000, need - 1) == B.RP_ENOMEM and call(None, need) == B.RP_ENOMEM
        assert call(0x1010, need) == B.RP_ENOMEM and b"aligned" in lib.rp_last_error()


def test_the_trainers_paths_check_their_arguments():
    lib = B.lib()
    cfg = B.TrainConfig(27, 256, 30, 128, B.RP_F32, 0, 1, 1, 1e-4, 0.99, 0.9, 0.999, 1e-8, 1)
    size = lambda c, n: lib.train_act_workspace_bytes(C.byref(c), n)
    assert size(cfg, 1) >= (256 + 256 + 30) * 4 and size(cfg, 1000) >= 1000 * (256 + 256 + 30) * 4
    assert size(cfg, 0) == 0 and size(cfg, 2 ** 20 + 1) == 0
    bad = B.TrainConfig(27, 100, 30, 128, B.RP_F32, 0, 1, 1, 1e-4, 0.99, 0.9, 0.999, 1e-8, 1)
    assert size(bad, 4) == 0
    how = B.Choice(1.0, 1.0, 0.0, 0, None, None, None, None)
    assert lib.train_act(None, 4, P, C.byref(how), P, P, None, None, P, 1 << 20, None) == EINVAL
    assert lib.train_distill_batch(None, P, C.byref(teacher()), None) == EINVAL


def piece_lengths():
    """Row lengths around everything that decides how a row is cut, and all of those of one or two pieces."""
    around = {b + d for b in range(8192, 262_145, 8192) for d in (-65, -64, -63, -1, 0, 1, 63, 64, 65)}
    return sorted({n for n in around if n <= 262_144} | set(range(1, 130)) | set(range(8000, 17_000)))


@pytest.mark.parametrize("dtype", [B.RP_F32, B.RP_BF16])
@pytest.mark.parametrize("rows_", [1, 4, 32, 100, 128, 129, 1000, 2 ** 24])
def test_every_row_length_has_a_workspace_size(rows_, dtype):
    """Of at most 8,192 pieces with 2,048 words and a head each, and none where a workgroup holds the row and there are
    rows for all compute units."""
    lib, held = B.lib(), 32_768 if dtype == B.RP_BF16 else 16_384
    for n in piece_lengths():
        x = rows(rows=rows_, n=n, stride=n, dtype=dtype)
        need = lib.rp_choose_workspace_bytes(C.byref(x))
        assert need == lib.rp_top_workspace_bytes(C.byref(x), 1), n
        assert need <= 8192 * (2048 * 8 + 32), n
        if n <= 8192 or (n <= held and rows_ > 128):
            assert need == 0, n
        if n > held:
            assert need >= min(rows_, 100) * 2 * (2048 * 8 + 32), n


@pytest.mark.parametrize("dtype", [B.RP_F32, B.RP_BF16])
def test_no_rows_of_any_length_are_no_work(dtype):
    lib = B.lib()
    for n in piece_lengths():
        x = rows(rows=0, data=None, n=n, stride=n, dtype=dtype)
        assert lib.rp_choose_workspace_bytes(C.byref(x)) == 0 and lib.rp_top_workspace_bytes(C.byref(x), 1) == 0
        assert lib.rp_distill_workspace_bytes(C.byref(x), 4) == 0
        assert choose(x) == 0 and top(x, k=1) == 0 and loss(x, teacher()) == 0 and grad(x, teacher(), stride=n) == 0


@pytest.mark.parametrize("dtype", [B.RP_F32, B.RP_BF16])
@pytest.mark.parametrize("rows_", [1, 4, 32, 33, 128, 129, 2 ** 24])
def test_every_row_length_has_a_workspace_size_for_distillation(rows_, dtype):
    """Of at most 64 pieces a row, 24 bytes each, and the entries' logits, each rounded up to 256 bytes."""
    for n in piece_lengths():
        x = rows(rows=rows_, n=n, stride=n, dtype=dtype)
        need = B.lib().rp_distill_workspace_bytes(C.byref(x), 7)
        cut = n > 16_384 and rows_ <= (128 if n > 32_768 else 32)
        assert (need > 0) == cut, n
        assert need <= rows_ * 64 * 24 + 256 + rows_ * 7 * 4 + 256, n


def test_the_binding_checks_shapes():
    """A transposed table has as many elements as the right one."""
    cpu = torch.device("cpu")
    index = torch.zeros(4, 3, dtype=torch.int32)
    take = lambda t: B._teacher(4, cpu, t, index, None, None, 1.0, 1.0, "t")
    for good in (torch.zeros(4, 3), torch.zeros(12), torch.zeros(4, 3).bfloat16()):
        take(good)
    for bad in (torch.zeros(3, 4), torch.zeros(2, 6), torch.zeros(4, 4)[:, :3], torch.zeros(11), torch.zeros(4, 3).half()):
        with pytest.raises(ValueError):
            take(bad)


def test_a_step_on_a_teachers_actions_runs_on_its_tensors_device(monkeypatch):
    """The step's launches, and the stream it takes where none is given, belong to the device of its tensors, whichever is
    the current one."""
    from types import SimpleNamespace
    seen = []

    class On:
        def __init__(self, device, stream):
            self.device = device

        def __enter__(self):
            seen.append(("enter", self.device))

        def __exit__(self, *error):
            seen.append(("exit", self.device))

    monkeypatch.setattr(B, "_on", On)
    monkeypatch.setattr(B, "_stream_ptr", lambda stream=None: seen.append("stream"))
    monkeypatch.setattr(B, "lib", lambda: SimpleNamespace(train_distill_batch=lambda *a: seen.append("call") or 0))
    cpu = torch.device("cpu")
    tr = object.__new__(B.Trainer)
    tr._h = None
    tr.cfg = SimpleNamespace(batch=4)
    tr.replay = SimpleNamespace(cfg=SimpleNamespace(state_dim=27, state_dtype=B.RP_F32), device=cpu)
    assert tr.distill_batch(torch.zeros(4, 27), torch.zeros(4, 3), torch.zeros(4, 3, dtype=torch.int32)) == 0
    assert seen == [("enter", cpu), "stream", "call", ("exit", cpu)]
