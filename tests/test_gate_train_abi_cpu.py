"""Host-side checks of the calls that train a gate: nothing is launched here."""
import os

import pytest

from paper_2603_06350_amd import binding as B

ONE = 0x1000          # an aligned address that no case below gets to use
BIG = 1 << 40


def addresses(*there):
    """Addresses far enough from each other for one argument each; None for those that are not there."""
    return [ONE + (i + 1) * (1 << 36) if t else None for i, t in enumerate(there)]


def put(args, i, a):
    """Argument i: None, a small number, or its own address moved by as much as a differs from ONE."""
    args[i] = args[i] + a - ONE if a is not None and a >= ONE else a


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not os.path.exists(B.lib_path()):
        from paper_2603_06350_amd import build
        build.build()
    B.load()


def code_of(call):
    with pytest.raises(B.MoeError) as err:
        call()
    return err.value.code


SH = B.make_shape(64, 128, 8, 2, 256, B.MOE_BF16, 1)


@pytest.mark.parametrize("i,a", [(0, None), (1, None), (3, None), (4, None), (5, None), (6, None), (0, ONE + 4), (1, ONE + 2),
                                 (3, ONE + 1), (4, ONE + 2), (5, ONE + 2), (6, ONE + 8)])
def test_balance_loss_refuses(i, a):
    args = addresses(1, 1, 1, 1, 1, 1, 1)
    put(args, i, a)
    assert code_of(lambda: B.moe_balance_loss(SH, *args, BIG)) == -1


@pytest.mark.parametrize("i,a", [(0, None), (1, None), (6, None), (0, ONE + 4), (1, ONE + 2), (2, ONE + 2), (3, ONE + 2), (6, ONE + 8),
                                 (7, 2), (7, -1)])
def test_route_backward_refuses(i, a):
    args = addresses(1, 1, 1, 1, 1, 0, 1, 1)
    args[4], args[7] = 1.0, 0
    put(args, i, a)
    assert code_of(lambda: B.moe_route_backward(SH, *args)) == -1


def test_route_backward_needs_one_of_its_parts():
    assert code_of(lambda: B.moe_route_backward(SH, ONE, ONE, None, None, 1.0, None, ONE)) == -1


@pytest.mark.parametrize("i,a", [(0, None), (1, None), (4, None), (7, None), (0, ONE + 4), (1, ONE + 4), (4, ONE + 1), (5, ONE + 4), (6, 2),
                                 (7, ONE + 4)])
def test_gate_distill_refuses(i, a):
    args = addresses(1, 1, 0, 1, 1, 1, 1, 1)
    args[3], args[6] = 1.0, 0
    put(args, i, a)
    assert code_of(lambda: B.moe_gate_distill(SH, *args, BIG)) == -1


@pytest.mark.parametrize("i,a", [(0, None), (1, None), (2, None), (8, None), (0, ONE + 8), (1, ONE + 8), (2, ONE + 8), (4, ONE + 8), (5, ONE + 2),
                                 (6, ONE + 8), (7, 4), (7, -1), (8, ONE + 8)])
def test_gate_backward_refuses(i, a):
    args = addresses(1, 1, 1, 0, 1, 1, 1, 1, 1)
    args[7] = 0
    put(args, i, a)
    assert code_of(lambda: B.moe_gate_backward(SH, *args, BIG)) == -1


@pytest.mark.parametrize("inside", [0, 16])
@pytest.mark.parametrize("out,read", [("d_x", "x"), ("d_x", "w_gate"), ("d_x", "d_scores"), ("d_w_gate", "x"), ("d_w_gate", "w_gate"),
                                      ("d_w_gate", "d_scores"), ("d_w_gate", "d_x")])
def test_gate_backward_refuses_outputs_that_are_read(out, read, inside):
    names = ("x", "w_gate", "d_scores", "mask", "d_w_gate", "d_gate_bias", "d_x", "accumulate", "workspace")
    args = dict(zip(names, addresses(1, 1, 1, 0, 1, 1, 1, 1, 1)), accumulate=0)
    args[out] = args[read] + inside
    assert code_of(lambda: B.moe_gate_backward(SH, *args.values(), BIG)) == -1


@pytest.mark.parametrize("inside", [-16, 0, 16])
def test_score_gradients_are_not_written_over_what_is_read(inside):
    scores, idx, dw, counts, target, loss, ws = addresses(1, 1, 1, 1, 1, 1, 1)
    for read in (scores, dw, idx):
        assert code_of(lambda: B.moe_route_backward(SH, scores, idx, dw, counts, 1.0, None, read + inside)) == -1
    for read in (scores, target):
        assert code_of(lambda: B.moe_gate_distill(SH, scores, target, None, 1.0, loss, read + inside, 0, ws, BIG)) == -1


@pytest.mark.parametrize("dtype,d", [(B.MOE_BF16, 2 ** 23 + 8), (B.MOE_F32, 2 ** 22 + 4), (B.MOE_BF16, 2 ** 24)])
def test_gate_backward_refuses_rows_that_its_offsets_do_not_reach(dtype, d):
    args = addresses(1, 1, 1, 0, 1, 1, 1, 1, 1)
    args[7] = 0
    assert code_of(lambda: B.moe_gate_backward(B.make_shape(2, d, 2, 1, 8, dtype, 0), *args, BIG)) == -2


def test_gate_backward_needs_an_output():
    assert code_of(lambda: B.moe_gate_backward(SH, ONE, ONE, ONE, None, None, None, None, 0, ONE, BIG)) == -1


def test_workspaces():
    sizes = [B.moe_train_workspace_bytes(B.make_shape(T, d, E, 1, 8, B.MOE_BF16, 0))
             for T, d, E in ((0, 8, 1), (1, 8, 1), (64, 128, 8), (4096, 4096, 8), (65536, 2048, 64), (2 ** 27, 4096, 256))]
    assert all(n >= 256 and n % 256 == 0 for n in sizes) and sizes[-1] < 2 ** 31
    nb = B.moe_train_workspace_bytes(SH)
    for call in (lambda: B.moe_balance_loss(SH, ONE, ONE, None, ONE, ONE, ONE, ONE, 16),
                 lambda: B.moe_gate_distill(SH, ONE, ONE, None, 1.0, ONE, ONE, 0, ONE, nb - 1),
                 lambda: B.moe_gate_backward(SH, ONE, ONE, ONE, None, ONE, None, None, 0, ONE, nb - 1)):
        assert code_of(call) == -3
    assert nb < 1 << 24
    with pytest.raises(B.MoeError):
        B.moe_train_workspace_bytes(B.make_shape(64, 124, 8, 2, 256, B.MOE_BF16, 1))
    for call in (lambda s: B.moe_balance_loss(s, ONE, ONE, None, ONE, ONE, ONE, ONE, BIG),
                 lambda s: B.moe_route_backward(s, ONE, ONE, ONE, ONE, 1.0, None, ONE),
                 lambda s: B.moe_gate_distill(s, ONE, ONE, None, 1.0, ONE, ONE, 0, ONE, BIG),
                 lambda s: B.moe_gate_backward(s, ONE, ONE, ONE, None, ONE, ONE, ONE, 0, ONE, BIG)):
        assert code_of(lambda: call(B.make_shape(64, 128, 8, 9, 256, B.MOE_BF16, 1))) == -1
        assert code_of(lambda: call(B.make_shape(64, 128, 300, 2, 256, B.MOE_BF16, 1))) == -2


def raw_list(*tensors):
    """A GradList of plain addresses: (data, out, elements, type)."""
    lst = B.GradList([])
    lst.array = (B.MoeTensor * max(1, len(tensors)))(*[B.MoeTensor(d, o, n, t, 0) for d, o, n, t in tensors])
    lst.grads = list(tensors)
    return lst


@pytest.mark.parametrize("tensor,code", [((None, ONE, 5, 0), -1), ((ONE + 2, ONE, 5, 0), -1), ((ONE + 1, ONE, 5, 1), -1), ((ONE, ONE, -1, 0), -1),
                                         ((ONE, ONE, 5, 2), -1), ((ONE, ONE, 2 ** 40 + 1, 1), -2), ((ONE, None, 5, 0), -1), ((ONE, ONE + 2, 5, 0), -1)])
def test_gradient_lists_refuse(tensor, code):
    lst = raw_list((ONE, ONE, 16, 0), tensor)
    assert code_of(lambda: B.moe_clip_grads(lst, 1.0, ONE, ONE, BIG)) == code
    if tensor[1] == ONE:                   # outputs are not looked at by the norm
        assert code_of(lambda: B.moe_grad_norm(lst, ONE, ONE, BIG)) == code
        assert code_of(lambda: B.moe_grad_workspace_bytes(lst)) == code


def test_norm_and_clip_refuse():
    lst = raw_list((ONE, ONE, 16, 0))
    assert code_of(lambda: B.moe_clip_grads(lst, -1.0, ONE, ONE, BIG)) == -1
    assert code_of(lambda: B.moe_clip_grads(lst, float("nan"), ONE, ONE, BIG)) == -1
    for call in (B.moe_grad_norm, lambda lst, *a: B.moe_clip_grads(lst, 1.0, *a)):
        assert code_of(lambda: call(lst, None, ONE, BIG)) == -1
        assert code_of(lambda: call(lst, ONE + 2, ONE, BIG)) == -1
        assert code_of(lambda: call(lst, ONE, None, BIG)) == -1
        assert code_of(lambda: call(lst, ONE, ONE + 8, BIG)) == -1
        assert code_of(lambda: call(lst, ONE, ONE, 255)) == -3
    sizes = [B.moe_grad_workspace_bytes(raw_list(*[(ONE, ONE, n, 0)] * c)) for n, c in ((1, 1), (1, 3000), (2 ** 30, 4), (2 ** 40, 1))]
    assert all(nb % 256 == 0 for nb in sizes) and sizes[-1] <= 1 << 16


def test_tensors_on_the_host_are_refused():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        B.moe_balance_loss(SH, torch.zeros(64, 8), ONE, None, ONE, ONE, ONE, ONE, BIG)
    with pytest.raises(ValueError):
        B.GradList([torch.zeros(5)])
