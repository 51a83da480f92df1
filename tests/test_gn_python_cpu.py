"""The Python binding of the group-norm and dropout calls reads the types of the
tensors it is given (CPU; the library is a recorder)."""
import pytest
import torch

K = pytest.importorskip("paper_1604_06174_amd.ckpt")

F32, BF16 = torch.float32, torch.bfloat16


class Recorder:
    def __init__(self, monkeypatch):
        self.calls = []
        monkeypatch.setattr(K, "_lib", self)

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def lib(monkeypatch):
    return Recorder(monkeypatch)


def drop():
    return K.dropout(torch.zeros(2, dtype=torch.int64), 0.1)


# --------------------------------------------------------------- defaults --
@pytest.mark.parametrize("xt,yt", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
def test_dropout_takes_the_tensors_types(lib, xt, yt):
    x, y = torch.zeros(4, 8, dtype=xt), torch.zeros(4, 8, dtype=yt)
    K.op_dropout(4, 8, x, y, drop(), res=torch.zeros(4, 8, dtype=yt))
    (name, a), = lib.calls
    assert name == "op_dropout" and a[2] == K.type_of(x) and a[7] == K.type_of(y)


def test_dropout_of_addresses_stays_bf16_by_default(lib):
    K.op_dropout(4, 8, 4096, 8192, drop())
    K.op_dropout(4, 8, 4096, 8192, drop(), xtype=K.TYPE_F32)
    assert [(a[2], a[7]) for _, a in lib.calls] == [(K.TYPE_BF16,) * 2, (K.TYPE_F32,) * 2]


def test_parameters_count_as_tensors(lib):
    K.op_dropout(4, 8, torch.nn.Parameter(torch.zeros(4, 8)), torch.zeros(4, 8), drop())
    assert lib.calls[0][1][2] == K.TYPE_F32


# --------------------------------------------------------------- refusals --
def tensors(n=2, hw=4, c=16, groups=4, x=BF16, g=None, d=None):
    e = lambda t: torch.zeros(n * hw, c, dtype=t)
    return dict(x=e(x), y=e(x), g=e(g or x), d=e(d or x), gamma=torch.zeros(c), beta=torch.zeros(c),
                st=torch.zeros(2 * n * groups), dgamma=torch.zeros(c), dbeta=torch.zeros(c))


def forward(d, t):
    K.op_gn_forward(d, t["x"], t["gamma"], t["beta"], t["y"], t["st"])


def apply(d, t):
    K.op_gn_apply(d, t["x"], t["st"], t["gamma"], t["beta"], t["y"])


def backward(d, t):
    K.op_gn_backward(d, t["g"], t["x"], t["st"], t["gamma"], t["beta"], t["d"], t["dgamma"], t["dbeta"])


CALLS = {forward: ["x", "y", "gamma", "beta", "st"], apply: ["x", "y", "gamma", "beta", "st"],
         backward: ["x", "g", "d", "gamma", "beta", "st", "dgamma", "dbeta"]}


@pytest.mark.parametrize("call,name", [(f, k) for f, names in CALLS.items() for k in names])
def test_a_tensor_of_another_type_is_refused(lib, call, name):
    d = K.gn_desc(2, 4, 16, 4)
    call(d, tensors())
    assert len(lib.calls) == 1
    for wrong in {F32, BF16, torch.float16, torch.float64} - {tensors()[name].dtype}:
        t = tensors()
        t[name] = t[name].to(wrong)
        with pytest.raises(K.CkptError) as e:
            call(d, t)
        assert e.value.code == K.E_INVALID and name in str(e.value) and len(lib.calls) == 1
    # raw memory and addresses carry no type
    for raw in (4096, torch.zeros(4096, dtype=torch.uint8)):
        call(d, {**tensors(), name: raw})
    assert len(lib.calls) == 3


def test_mixed_types_as_described(lib):
    backward(K.gn_desc(2, 4, 16, 4, gtype=K.TYPE_F32), tensors(g=F32))
    backward(K.gn_desc(2, 4, 16, 4, dtype=K.TYPE_F32), tensors(d=F32))
    forward(K.gn_desc(2, 4, 16, 4, xtype=K.TYPE_F32), tensors(x=F32))
    assert len(lib.calls) == 3


@pytest.mark.parametrize("kw", [dict(xtype=1, ytype=0), dict(xtype=0, ytype=1), dict(ytype=1)])
def test_dropout_types_that_do_not_fit_are_refused(lib, kw):
    x, y = torch.zeros(4, 8), torch.zeros(4, 8)
    with pytest.raises(K.CkptError) as e:
        K.op_dropout(4, 8, x, y, drop(), **kw)
    assert e.value.code == K.E_INVALID and not lib.calls


def test_dropout_residual_of_another_type_is_refused(lib):
    with pytest.raises(K.CkptError) as e:
        K.op_dropout(4, 8, torch.zeros(4, 8), torch.zeros(4, 8), drop(), res=torch.zeros(4, 8, dtype=BF16))
    assert e.value.code == K.E_INVALID and "res" in str(e.value) and not lib.calls


@pytest.mark.parametrize("x,y", [(torch.float16, F32), (F32, torch.float64)])
def test_dropout_of_unknown_types_is_refused(lib, x, y):
    with pytest.raises(K.CkptError) as e:
        K.op_dropout(4, 8, torch.zeros(4, 8, dtype=x), torch.zeros(4, 8, dtype=y), drop())
    assert e.value.code == K.E_UNSUPPORTED and not lib.calls


@pytest.mark.parametrize("rng", [torch.zeros(1, dtype=torch.int64), torch.zeros(2, dtype=torch.int32),
                                 torch.zeros(2), torch.zeros(2, dtype=torch.float64),
                                 torch.zeros(4, dtype=torch.int64)[::2]])
def test_generator_state_is_two_words_of_64_bits(rng):
    with pytest.raises(K.CkptError) as e:
        K.dropout(rng, 0.1)
    assert e.value.code == K.E_INVALID


# ---------------------------------------------------- fields of fixed width --
@pytest.mark.parametrize("kw", [dict(n=2 - (1 << 64)), dict(hw=-(1 << 64) + 1), dict(c=16 - (1 << 32)),
                                dict(groups=4 - (1 << 32)), dict(act=1 << 32), dict(act=2 - (1 << 32)),
                                dict(xtype=(1 << 32) + 1), dict(gtype=1 << 32), dict(dtype=-(1 << 32)),
                                dict(ldx=16 - (1 << 64)), dict(ldd=1 << 64)])
def test_descriptor_values_do_not_wrap(kw):
    """Values that a narrower field would turn into valid ones."""
    a = dict(n=2, hw=4, c=16, groups=4)
    a.update(kw)
    with pytest.raises(K.CkptError) as e:
        K.gn_desc(**a)
    assert e.value.code in (K.E_INVALID, K.E_UNSUPPORTED)


@pytest.mark.parametrize("rows,cols,kw", [((1 << 64) + 4, 8, {}), (4 - (1 << 64), 8, {}), (4, (1 << 64) + 8, {}),
                                          (4, 8, dict(ldx=1 << 64)), (4, 8, dict(ldr=8 - (1 << 64))),
                                          (4, 8, dict(ldy=1 << 65)), (4, 8, dict(xtype=1 << 32)),
                                          (4, 8, dict(ytype=(1 << 32) + 1))])
def test_dropout_sizes_do_not_wrap(lib, rows, cols, kw):
    with pytest.raises(K.CkptError) as e:
        K.op_dropout(rows, cols, 4096, 8192, drop(), **kw)
    assert e.value.code in (K.E_INVALID, K.E_UNSUPPORTED) and not lib.calls


@pytest.mark.parametrize("nbytes", [-1, 16 - (1 << 64), 1 << 64])
def test_workspace_sizes_do_not_wrap(lib, nbytes):
    d = K.gn_desc(2, 1 << 20, 16, 4)
    for call in (lambda: K.op_gn_forward(d, *(4096,) * 5, 4096, nbytes),
                 lambda: K.op_gn_backward(d, *(4096,) * 8, 4096, nbytes)):
        with pytest.raises(K.CkptError) as e:
            call()
        assert e.value.code == K.E_INVALID and not lib.calls
