"""Refusals of the binding of the operators around the layer: device tensors that differ from an
accepted call in one property. Every refusal comes before a launch."""
import pytest
import torch

pytestmark = pytest.mark.gpu

b = pytest.importorskip("paper_2603_23198_amd.binding")

T, D, E, K = 6, 40, 8, 2


def new(*shape, dt=torch.float32):
    return torch.zeros(shape, dtype=dt, device="cuda")


def norm_forward():
    t = {n: new(T, D, dt=torch.bfloat16) for n in ("X", "Y", "X_out", "N")}
    t.update(w_pre=new(D), w_post=new(D), gate_c=new(D), gate_t=new(T))
    return t, lambda X, **kw: b.sfl_norm_forward(X, **kw)


def norm_backward():
    t = {n: new(T, D, dt=torch.bfloat16) for n in ("X_out", "Y", "dX_out", "dN", "dX", "dY")}
    t.update(w_pre=new(D), w_post=new(D), gate_c=new(D), gate_t=new(T), dw_pre=new(D), dw_post=new(D), dgate_c=new(D),
             dgate_t=new(T))
    t["workspace"] = new(b.sfl_norm_workspace_size(T, D, "bf16"), dt=torch.uint8)
    return t, lambda X_out, Y, dX_out, dN, **kw: b.sfl_norm_backward(X_out, Y, dX_out, dN, **kw)


def route_forward():
    return (dict(logits=new(T, E), expert=new(T, K, dt=torch.int32), weight=new(T, K)),
            lambda logits, expert, weight: b.sfl_route_forward(logits, expert, weight))


def route_backward():
    return (dict(logits=new(T, E), expert=new(T, K, dt=torch.int32), dweight=new(T, K), dlogits=new(T, E)),
            lambda logits, expert, dweight, dlogits: b.sfl_route_backward(logits, expert, dweight, dlogits))


def dispatch():
    return (dict(expert=new(T, K, dt=torch.int32), pos=new(T, K, dt=torch.int32), offsets=new(E + 1, dt=torch.int32),
                 X=new(T, D, dt=torch.bfloat16), Xs=new(T * K, D, dt=torch.bfloat16)),
            lambda expert, pos, offsets, **kw: b.sfl_expert_dispatch(expert, E, pos, offsets, **kw))


def combine():
    return (dict(Ys=new(T * K, D), pos=new(T, K, dt=torch.int32), Y=new(T, D), weight=new(T, K)),
            lambda Ys, pos, Y, weight: b.sfl_expert_combine(Ys, pos, Y, weight=weight))


def combine_backward():
    t = dict(dY=new(T, D), Ys=new(T * K, D), pos=new(T, K, dt=torch.int32), weight=new(T, K), dYs=new(T * K, D),
             dweight=new(T, K))
    return t, lambda dY, Ys, pos, weight, **kw: b.sfl_expert_combine_backward(dY, Ys, pos, weight, **kw)


def gradients():
    t = dict(first=new(T, D), second=new(K, dt=torch.bfloat16), sumsq=new(1, dt=torch.float64), norm=new(1))

    def call(first, second, sumsq, norm):
        # both in place and into outputs that fit the accepted call
        for out in (None, [new(T, D), new(K, dt=torch.bfloat16)]):
            l = b.grad_list([first, second], out)
            b.sfl_grad_sumsq(l, sumsq, workspace=new(b.sfl_grad_workspace_size(l), dt=torch.uint8))
            b.sfl_grad_clip(l, sumsq, 1.0, norm)

    return t, call


CALLS = [norm_forward, norm_backward, route_forward, route_backward, dispatch, combine, combine_backward, gradients]
# A call takes its sizes and its type from these, so that another size of theirs makes the others wrong.
GIVES_SIZES = {"X", "X_out", "logits", "expert", "Ys", "Xs", "dY", "pos", "first", "second"}


def strided(t):
    """The same shape and values, every second element of a buffer."""
    wide = torch.zeros((*t.shape, 2), dtype=t.dtype, device="cuda")
    return wide.select(-1, 0)


@pytest.mark.parametrize("make", CALLS, ids=lambda f: f.__name__)
def test_one_wrong_tensor(make):
    tensors, call = make()
    call(**tensors)  # accepted as it is
    torch.cuda.synchronize()
    for name, t in tensors.items():
        if name == "workspace":
            continue
        wrong = {"type": t.to(torch.float16), "contiguity": strided(t), "device": t.cpu()}
        if name not in GIVES_SIZES:
            wrong["elements"] = new(t.numel() + 1, dt=t.dtype)
        for what, bad in wrong.items():
            if what == "contiguity" and t.numel() == 1:
                continue  # a single element is contiguous whatever its stride
            assert not (what == "contiguity" and bad.is_contiguous())
            with pytest.raises(ValueError):
                call(**{**tensors, name: bad})
                pytest.fail(f"{make.__name__} took a wrong {name}: {what}")
        with pytest.raises((TypeError, AttributeError)):
            call(**{**tensors, name: 7})
    call(**tensors)
    torch.cuda.synchronize()


def test_a_refusal_says_what_it_wanted():
    x, n = new(T, D), new(T, D)
    for bad, says in [(new(T, D, dt=torch.bfloat16), "contiguous float32 tensor .* got BFloat16"),
                      (new(T, D - 1), f"tensor of {T * D} elements .* of {T * (D - 1)}"),
                      (strided(x), "not contiguous"), (x.cpu(), "on the CPU")]:
        with pytest.raises(ValueError, match=says):
            b.sfl_norm_forward(x, bad, X_out=x, N=n)
    b.sfl_norm_forward(x, new(T, D), X_out=x, N=n)


@pytest.mark.parametrize("make", CALLS[:-1], ids=lambda f: f.__name__)
def test_rows_of_another_width(make):
    """As many elements, in rows of another width: [d][T] is not [T][d]. Rows that are
    counted or divided by several dimensions and flat buffers have the same order in memory and are taken."""
    tensors, call = make()
    for name, t in tensors.items():
        if t.dim() != 2 or (name in GIVES_SIZES and (make, name) != (dispatch, "pos")):
            continue
        for bad in (t.view(t.shape[1], t.shape[0]), t.view(2, -1, t.shape[1] // 2), t.view(1, -1)):
            with pytest.raises(ValueError):
                call(**{**tensors, name: bad})
                pytest.fail(f"{make.__name__} took {name} as {tuple(bad.shape)}")
        for good in (t.view(2, -1, t.shape[1]), t.view(t.shape[0], 2, -1), t.view(-1)):
            call(**{**tensors, name: good})
    torch.cuda.synchronize()
