"""Random geometries, batches and masks through gk_append and gk_attention, against the same 64-bit definitions and within the same
bounds as their own tests."""
import random

import pytest

pytestmark = pytest.mark.gpu

import test_gpu_append
import test_gpu_attention
from seq_reference import Layout


def _layout(r):
    fp8 = r.random() < 0.5
    D = r.choice([16, 32, 64, 64, 80, 128, 128, 128, 208, 256])
    H = r.choice([1, 2, 3, 4]) if not fp8 else r.choice([2, 4])
    return Layout(H, D, r.choice([1, 5, 8, 16, 16, 24, 32, 64, 100, 128, 256]), fp8, r.choice([1, 2]), r.random() < 0.4, 2,
                  16 * r.randint(0, 3), r.randint(0, 4))


def _lengths(r, step):
    n = r.choice([1, 2, 5, 17])
    kv, new = [], []
    for _ in range(n):
        past = r.choice([0, r.randint(0, 40), r.randint(0, 700), r.randint(0, 3000)])
        q = 1 if step else r.choice([0, 1, r.randint(1, 9), r.randint(1, 200), r.randint(1, 500)])
        kv.append(past + q)
        new.append(q)
    if sum(new) == 0:
        kv[0], new[0] = kv[0] + 3, 3
    return kv, new


@pytest.mark.parametrize("case", range(40))
def test_attention(case):
    r = random.Random(4100 + case)
    step = r.random() < 0.4
    kv, new = _lengths(r, step)
    test_gpu_attention.run(_layout(r), kv, new, G=r.choice([1, 2, 4, 5, 8, 12]), window=r.choice([0, 0, 0, 1, 77, 512]),
                           causal=r.random() < 0.8, seed=case, step_form=step, layer=r.randint(0, 1))


@pytest.mark.parametrize("case", range(40))
def test_append(case):
    r = random.Random(5200 + case)
    step = r.random() < 0.4
    lay = _layout(r)
    kv, new = _lengths(r, step)
    R = r.choice([lay.D, lay.D, 16, 0])
    axes = r.choice([1, 1, 2, 3]) if R >= 32 else 1
    test_gpu_append.run(lay, kv, new, G=r.choice([1, 4, 7]), R=R, axes=axes, interleaved=r.random() < 0.3, positions=r.random() < 0.5,
                        seed=case, step_form=step, queries=r.random() < 0.8)
