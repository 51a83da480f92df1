"""Python's calls of the token models' operators read vectors and statistics as values side by side, and
memory by the type that the description says: tensors that are neither are refused (no GPU)."""
import pytest

K = pytest.importorskip("paper_1604_06174_amd.ckpt")
torch = pytest.importorskip("torch")

A = 0x1000  # an aligned address that nothing reads
F = torch.zeros(64)
STRIDED = {"steps": F[::2], "column": F.view(32, 2)[:, 0], "transposed": F.view(8, 8).T, "narrow": F.view(8, 8)[:, :4]}


def calls():
    """(name, call, its arguments, which of them are dense fp32)"""
    r, r8, e, a = (K.rms_desc(4, 16), K.rms_desc(4, 16, ytype=K.TYPE_E4M3, gtype=K.TYPE_BF16), K.embed_desc(5, 9, 16),
                   K.attn_desc(10, 12, 2, 4, 2, 16))
    yield "rms_forward", K.op_rms_forward, [r8, A, A, A, A, None, None, A], {2: "w", 4: "st", 7: "ys"}
    yield "rms_apply", K.op_rms_apply, [r8, A, A, A, A, A], {2: "st", 3: "w", 5: "ys"}
    yield "rms_backward", K.op_rms_backward, [r, A, A, A, A, A, A, A, 1 << 20], {3: "st", 4: "w", 6: "dw"}
    yield "attn_forward", K.op_attn_forward, [a, A, A, A, A, A, A, A], {7: "lse"}
    yield "attn_backward", K.op_attn_backward, [a] + [A] * 11 + [A, 1 << 20], {6: "lse"}


CASES = [(name, k, arg) for name, _, _, dense in calls() for k, arg in dense.items()]


def refusal(name, k, bad):
    for n, call, args, _ in calls():
        if n == name:
            args[k] = bad
            with pytest.raises(K.CkptError) as e:
                call(*args)
            assert e.value.code == K.E_INVALID
            return str(e.value)


@pytest.mark.parametrize("name,k,arg", CASES)
@pytest.mark.parametrize("how", STRIDED)
def test_strided_vectors(name, k, arg, how):
    assert f"op_{name}({arg})" in (m := refusal(name, k, STRIDED[how])) and "contiguous" in m


@pytest.mark.parametrize("name,k,arg", CASES)
def test_vectors_side_by_side_are_looked_at_further(name, k, arg):
    """Contiguous ones get as far as their device."""
    assert "current device" in refusal(name, k, F) and "current device" in refusal(name, k, F.view(1, 64)[:, 8:])


@pytest.mark.parametrize("name,k,arg", CASES)
@pytest.mark.parametrize("t", [torch.int64, torch.int16])
def test_integers_of_another_size(name, k, arg, t):
    assert f"op_{name}({arg})" in (m := refusal(name, k, torch.zeros(64, dtype=t))) and "described as" in m


@pytest.mark.parametrize("t,ok", [(torch.int16, True), (torch.uint8, True), (torch.int8, True), (torch.int32, False),
                                  (torch.int64, False)])
def test_integers_as_memory_of_16_bits(t, ok):
    """Bits of the type's own size, or bytes, are memory; other integers are a mistake."""
    z = torch.zeros(64, dtype=t)
    for name, k in (("rms_forward", 1), ("rms_backward", 1), ("attn_forward", 1), ("attn_backward", 9)):
        assert ("current device" if ok else "described as") in refusal(name, k, z)
    for args in ((A, z, A), (A, A, z)):
        with pytest.raises(K.CkptError) as e:
            K.op_embed_forward(K.embed_desc(5, 9, 16), *args)
        assert ("current device" if ok else "described as") in str(e.value)


@pytest.mark.parametrize("ws", [torch.zeros(1 << 10, dtype=torch.uint8)[::2], torch.zeros(64, 64).T])
def test_strided_workspaces(ws):
    for name, k in (("rms_backward", 7), ("attn_backward", 12)):
        assert "contiguous" in refusal(name, k, ws)
