"""Argument checks of the operators for many routed experts in 8 bits that need no GPU: they are made
before any launch, in C for sizes and pointers and in the binding for tensors."""
import ctypes

import pytest
import torch

from paper_2603_23198_amd import binding as b

P = 0x1000  # a pointer that is never followed
lib = b._lib
ARG, UNSUPPORTED, OK = b.SFL_E_ARG, b.SFL_E_UNSUPPORTED, b.SFL_OK


def refused(call, cases, code=ARG):
    for kw in cases:
        assert call(**kw) == code, kw


def filled(kind, defaults):
    def make(**kw):
        a = kind()
        for n, v in {**defaults, **kw}.items():
            setattr(a, n, v)
        return a
    return make


def test_structures_are_the_headers():
    sizes = {b.RouteGroupsArgs: 80, b.RouteGroupsBwdArgs: 64, b.QuantArgs: 88, b.Adamw: 80, b.AdamwCfg: 80}
    for kind, size in sizes.items():
        assert ctypes.sizeof(kind) == size, kind


def test_route_groups():
    make = filled(b.RouteGroupsArgs, dict(T=4, E=16, k=2, groups=4, group_k=2, group_top=2, normalise=1, scale=1.0,
                                          logits=P, expert=P, weight=P))

    def f(**kw):
        return lib.sfl_route_groups_forward(make(**kw), None)

    refused(f, [dict(dtype=2), dict(score=2), dict(score=-1), dict(T=-1), dict(E=0), dict(k=0), dict(k=17), dict(groups=0),
                dict(groups=3), dict(groups=-4), dict(group_k=0), dict(group_k=5), dict(group_top=0), dict(group_top=3),
                dict(k=9), dict(normalise=2), dict(logits=None), dict(expert=None), dict(weight=None)])
    refused(f, [dict(E=1028), dict(E=512, k=65), dict(T=1 << 31)], UNSUPPORTED)
    assert f(T=0, logits=None, expert=None, weight=None) == OK
    assert lib.sfl_route_groups_forward(None, None) == ARG
    back = filled(b.RouteGroupsBwdArgs, dict(T=4, E=16, k=2, normalise=1, scale=1.0, logits=P, expert=P, dweight=P,
                                             dlogits=P))

    def g(**kw):
        return lib.sfl_route_groups_backward(back(**kw), None)

    refused(g, [dict(dtype=-1), dict(score=7), dict(T=-1), dict(E=0), dict(k=0), dict(k=17), dict(normalise=-1),
                dict(logits=None), dict(expert=None), dict(dweight=None), dict(dlogits=None)])
    refused(g, [dict(E=1028), dict(E=512, k=65), dict(T=1 << 31)], UNSUPPORTED)
    assert g(T=0, logits=None) == OK and lib.sfl_route_groups_backward(None, None) == ARG


def test_quant_rows():
    make = filled(b.QuantArgs, dict(E=1, T=4, d=64, columns=512, X=P, Q=P, S=P, Qt=P, St=P))

    def f(**kw):
        return lib.sfl_quant_rows(make(**kw), None)

    refused(f, [dict(dtype=9), dict(T=-1), dict(d=0), dict(E=0), dict(E=2), dict(X=None), dict(Q=None), dict(S=None),
                dict(Qt=None), dict(St=None), dict(Q=None, S=None, Qt=None, St=None), dict(Q=P + 8), dict(Qt=P + 1),
                dict(S=P + 2), dict(St=P + 1), dict(columns=0), dict(columns=500), dict(T=400, columns=256),
                dict(T=600, columns=512), dict(columns=1 << 31)])
    refused(f, [dict(E=1025, offsets=P), dict(d=(1 << 20) + 1), dict(T=(1 << 31) - 1)], UNSUPPORTED)
    assert f(T=0, X=None) == OK and lib.sfl_quant_rows(None, None) == ARG


def test_quant_columns_never_shrink():
    rng = __import__("random").Random(1)
    for _ in range(2000):
        T, E = rng.randint(0, 5000), rng.randint(1, 64)
        n = b.sfl_quant_columns(T, E)
        assert n % 512 == 0 and n <= b.sfl_quant_columns(T + rng.randint(0, 300), E + rng.randint(0, 9))
        cuts = sorted(rng.randint(0, T) for _ in range(E - 1))
        runs = [y - x for x, y in zip([0] + cuts, cuts + [T])]
        assert sum(-(-r // 128) * 128 for r in runs) <= n
    for E in (1, 3, 64):  # the worst runs: one token in each but one
        T = 1000
        assert sum(-(-r // 128) * 128 for r in [T - E + 1] + [1] * (E - 1)) <= b.sfl_quant_columns(T, E)
    out = ctypes.c_int64(0)
    assert lib.sfl_quant_columns(4, 1, None) == ARG and lib.sfl_quant_columns(-1, 1, out) == ARG
    assert lib.sfl_quant_columns(4, 0, out) == ARG and lib.sfl_quant_columns(4, 1025, out) == UNSUPPORTED


def test_quant_weights():
    def f(W=P, dtype=0, E=2, R=64, C=64, Q=P, S=P, Qt=P, St=P):
        return lib.sfl_quant_weights(W, dtype, E, R, C, Q, S, Qt, St, None)

    refused(f, [dict(W=None), dict(dtype=4), dict(E=0), dict(R=0), dict(C=0), dict(Q=None), dict(St=None),
                dict(Q=None, S=None, Qt=None, St=None), dict(Q=P + 4), dict(Qt=P + 8), dict(S=P + 1), dict(St=P + 2)])
    refused(f, [dict(E=1025), dict(R=(1 << 20) + 1), dict(C=(1 << 20) + 1)], UNSUPPORTED)


def test_products():
    def f(Q=P, S=P, rows=4, K=128, W=P, Ws=P, E=2, N=64, offsets=P, dtype=1, Y=P):
        return lib.sfl_quant_product(Q, S, rows, K, W, Ws, E, N, offsets, dtype, Y, None)

    refused(f, [dict(rows=-1), dict(K=0), dict(K=64), dict(K=192), dict(E=0), dict(N=0), dict(offsets=None), dict(dtype=5),
                dict(Q=None), dict(S=None), dict(W=None), dict(Ws=None), dict(Y=None), dict(Q=P + 8), dict(W=P + 4),
                dict(S=P + 1), dict(Ws=P + 2), dict(Y=P + 1)])
    refused(f, [dict(E=1025), dict(rows=(1 << 31) - 1), dict(N=(1 << 31) - 1), dict(K=(1 << 20) + 128)], UNSUPPORTED)
    assert f(rows=0, Q=None, S=None, Y=None) == OK

    def g(Yt=P, Ys=P, N=64, Xt=P, Xs=P, K=64, rows=512, columns=512, offsets=P, E=2, dtype=0, dW=P):
        return lib.sfl_quant_product_weights(Yt, Ys, N, Xt, Xs, K, rows, columns, offsets, E, dtype, dW, None)

    refused(g, [dict(N=0), dict(K=0), dict(rows=-1), dict(rows=513), dict(columns=500), dict(columns=0), dict(E=0),
                dict(offsets=None), dict(dtype=3), dict(dW=None), dict(dW=P + 2), dict(Yt=None), dict(Ys=None),
                dict(Xt=None), dict(Xs=None), dict(Yt=P + 8), dict(Xt=P + 1), dict(Ys=P + 1), dict(Xs=P + 2),
                ])
    refused(f, [dict(E=1024, rows=(1 << 28) + 128)], UNSUPPORTED)
    refused(g, [dict(E=1025), dict(N=(1 << 20) + 1), dict(K=(1 << 20) + 1), dict(columns=(1 << 22) + 512)], UNSUPPORTED)


def test_adamw():
    tensor = filled(b.Adamw, dict(param=P, grad=P, m=P, v=P, n=10))
    cfg = filled(b.AdamwCfg, dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, max_norm=1.0, step=P))

    def f(n=1, t={}, **kw):
        a = (b.Adamw * 1)(tensor(**t))
        return lib.sfl_adamw_step(a, n, cfg(**kw), None)

    nan = float("nan")
    refused(f, [dict(n=-1), dict(step=None), dict(lr=-1.0), dict(lr=nan), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
                dict(beta2=nan), dict(eps=0.0), dict(eps=-1e-8), dict(eps=nan), dict(eps=1e-39),
                dict(sumsq=P, max_norm=-1.0), dict(sumsq=P, max_norm=nan), dict(norm=P)])
    refused(f, [dict(t=t) for t in (dict(n=-1), dict(n=(1 << 40) + 1), dict(param=None), dict(grad=None), dict(m=None),
                                    dict(v=None), dict(param_dtype=2), dict(grad_dtype=-1), dict(moments=2),
                                    dict(moments=1), dict(moments=1, m_scale=P), dict(m_scale=P), dict(v_scale=P),
                                    dict(weight_decay=-0.1), dict(weight_decay=nan), dict(param_dtype=1, half=P))])
    assert lib.sfl_adamw_step(None, 1, cfg(), None) == ARG and lib.sfl_adamw_step(None, 0, None, None) == ARG
    assert lib.sfl_adamw_step(None, 0, cfg(), None) == OK
    assert f(t=dict(n=0, param=None, grad=None, m=None, v=None)) == OK


def test_the_binding_refuses_tensors_on_the_cpu_and_of_other_types():
    f32 = torch.zeros((4, 8))
    with pytest.raises(ValueError, match="on the CPU"):
        b.sfl_route_groups_forward(f32, torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2)))
    with pytest.raises(ValueError, match="unknown score"):
        b.sfl_route_groups_forward(f32, torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2)), score="tanh")
    with pytest.raises(ValueError):
        b.sfl_quant_rows(f32.half())
    for kind, name in ((4, "float8_e4m3fn"), (5, "uint8"), (6, "int64")):
        with pytest.raises(ValueError, match=name):
            b._buf(f32, kind, 32)
    with pytest.raises(ValueError, match="unknown kind"):
        b._buf(f32, 7, 32)


def test_the_binding_of_products_checks_the_experts():
    Q, S = torch.zeros((4, 128), dtype=torch.float8_e4m3fn), torch.zeros((4, 4), dtype=torch.uint8)
    W, Ws = torch.zeros((2, 64, 128), dtype=torch.float8_e4m3fn), torch.zeros((2, 1, 4), dtype=torch.uint8)
    with pytest.raises(ValueError, match="offsets of 2 experts"):
        b.sfl_quant_product(Q, S, W, Ws, torch.zeros((4, 64)), offsets=torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="rows or offsets"):
        b.sfl_quant_product_weights(torch.zeros((64, 512)), None, torch.zeros((64, 512)), None, torch.zeros((1, 64, 64)))


def test_lists_of_adamw(monkeypatch):
    monkeypatch.setattr(b, "_buf", lambda t, *_: None if t is None else P)
    z = torch.zeros
    a = b.adamw_list([z(3), z(5, dtype=torch.bfloat16)], [z(3), z(5)], [z(3), z(5, dtype=torch.float8_e4m3fn)],
                     [z(3), z(5, dtype=torch.float8_e4m3fn)], m_scales=[None, z(1, dtype=torch.uint8)],
                     v_scales=[None, z(1, dtype=torch.uint8)], weight_decay=[0.0, 0.5])
    assert [(t.n, t.param_dtype, t.moments, t.weight_decay) for t in a] == [(3, 0, 0, 0.0), (5, 1, 1, 0.5)]
    with pytest.raises(ValueError, match="one entry"):
        b.adamw_list([z(3)], [z(3), z(3)], [z(3)], [z(3)])
    with pytest.raises(ValueError, match="no scales"):
        b.adamw_list([z(3)], [z(3)], [z(3)], [z(3)], m_scales=[z(1)], v_scales=[z(1)])
    assert len(b.adamw_list([], [], [], [])) == 0


def test_fast_products_are_asked_for_and_have_bf16_results():
    fast = b.SFL_BF16_FAST

    def f(dtype=fast, rows=0, Y=P):
        return lib.sfl_quant_product(P, P, rows, 128, P, P, 2, 64, P, dtype, Y, None)

    def g(dtype=fast, dW=P, K=64):
        return lib.sfl_quant_product_weights(P, P, 64, P, P, K, 512, 512, P, 2, dtype, dW, None)

    assert f() == OK and f(Y=P + 2) == OK and f(dtype=0, Y=P + 2) == ARG
    refused(f, [dict(dtype=0x100), dict(dtype=0x102), dict(Y=P + 1)])
    refused(g, [dict(dtype=0x100), dict(dtype=0x102), dict(dW=P + 1), dict(dtype=0, dW=P + 2)])
    assert g(K=(1 << 20) + 1) == UNSUPPORTED
    # no other call takes it
    assert lib.sfl_quant_weights(P, fast, 2, 64, 64, P, P, P, P, None) == ARG
    a = b.QuantArgs(fast, 1, 4, 64, 512, P, None, None, P, P, P, P)
    assert lib.sfl_quant_rows(a, None) == ARG
    Q, S, W, Ws = torch.zeros((4, 128)), None, torch.zeros((64, 128)), None
    with pytest.raises(ValueError, match="bf16 results"):
        b.sfl_quant_product(Q, S, W, Ws, torch.zeros((4, 64)), fast=True)
    with pytest.raises(ValueError, match="bf16 results"):
        b.sfl_quant_product_weights(torch.zeros((64, 512)), None, W, None, torch.zeros((1, 64, 64)), rows=4, fast=True)


def test_a_step_by_the_norm_says_what_it_clips_to(monkeypatch):
    """Whoever gives the norm, were it to have it written or looked at alone, has to say the largest one: a
    default of zero would clip every gradient to nothing."""
    monkeypatch.setattr(b, "_buf", lambda t, *_: None if t is None else P)
    seen = []
    monkeypatch.setattr(b, "_lib", type("Lib", (), dict(sfl_adamw_step=lambda _, lst, n, cfg, stream: seen.append(cfg) or 0))())
    monkeypatch.setattr(b, "_stream", lambda stream: None)
    step = torch.tensor([1])
    with pytest.raises(ValueError, match="max_norm"):
        b.sfl_adamw_step(b.adamw_list([], [], [], []), step, lr=1.0, sumsq=torch.zeros(1))
    assert not seen
    b.sfl_adamw_step(b.adamw_list([], [], [], []), step, lr=1.0)
    for most in (0.0, 1.0, float("inf")):
        b.sfl_adamw_step(b.adamw_list([], [], [], []), step, lr=1.0, sumsq=torch.zeros(1), max_norm=most)
        assert seen[-1].max_norm == most
