"""Attention over packed sequences (op_attn_*) of more sequences than a wavefront has lanes, where a tile is found
by the offsets alone: every form, groups of query heads, rows of no sequence, empty sequences, split keys.
Against the float64 oracle, whose bounds of rounding are the bars."""
import numpy as np
import pytest

from test_gpu_attn import SAME, Case

pytestmark = pytest.mark.gpu
pytest.importorskip("torch")

MANY = {
    "65": SAME(*[(0, 1, 129, 300, 40)[k % 5] for k in range(65)]),
    "100": SAME(*[(300, 0, 1, 129, 5, 64)[k % 6] for k in range(100)]),
    "after_earlier": [((k * 7) % 140, (k * 7) % 140 + (k * 13) % 90) for k in range(90)],
    "fewer_keys": [((k * 11) % 150, (k * 5) % 70) for k in range(80)],
}


@pytest.mark.parametrize("name", MANY)
@pytest.mark.parametrize("heads,kv", [(9, 3), (16, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_more_than_64_sequences(name, heads, kv, causal):
    dim = 64 if kv == 3 else 24
    t = Case(MANY[name], heads, kv, dim, causal, before=3, after=70, seed=heads)
    t.check()


@pytest.mark.parametrize("causal", [True, False])
def test_more_than_64_tokens_with_split_keys(causal):
    t = Case([(1, (k * 397) % 1500) for k in range(70)], 4, 2, 128, causal, before=2, after=5)
    assert t.workspace(False)[1] > 0
    t.check()


@pytest.mark.parametrize("seqs", [64, 65, 4096, 4097, 5000])
def test_thousands_of_sequences(seqs):
    rng = np.random.default_rng(seqs)
    lq = rng.integers(0, 3, seqs)
    lk = lq + rng.integers(0, 2, seqs)
    Case(list(zip(lq.tolist(), lk.tolist())), 2, 1, 16, before=1, after=40).check()
