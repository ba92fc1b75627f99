"""Drawn calls of the operators of positions and cross attention: forms, pages, dimensions, head layouts and
ragged lengths that no other test puts together, against the same references."""
import random

import numpy as np
import pytest

from tests import cache_ref as ref
from tests.test_gpu_cross import run_cross
from tests.test_gpu_positions import run_append, run_move

pytestmark = pytest.mark.gpu


def drawn(seed):
    """The random numbers of a case, a cache's form and page, and a way to draw lengths."""
    r = random.Random(seed)
    form = r.choice(["bf16", "head", 16, 32, 64, 128])
    page = form * r.choice([1, 2, 3, 4]) if isinstance(form, int) else r.choice([1, 5, 8, 16, 24, 48, 64, 128])

    def lengths(n, most, least=0):
        return [least if r.random() < 0.2 else int(np.exp(r.uniform(0, np.log(most)))) for _ in range(n)]

    return r, form, page, lengths


@pytest.mark.parametrize("seed", range(24))
def test_append(seed):
    r, form, page, lengths = drawn(seed)
    most = [1, 2, 3, 5, 8, 9, 16, 20, 32, 33, 150, 400][seed % 12]
    new = lengths(r.choice([1, 3, 9] if most > 40 else [2, 9, 33, 70]), most + 1) + [most]
    lens = [m + x for m, x in zip(new, lengths(len(new), 200))]
    hkv = r.choice([1, 2, 3, 5, 8, 9])
    run_append(lens, new, form, page, r.choice([2, 4, 16, 18, 50, 64, 96, 100, 126, 128]), r.random() < 0.5, hkv=hkv,
               hq=hkv * r.choice([1, 2, 4, 8]), at=r.choice([None, 5, -90, 1 << 20]), codes=r.random() < 0.4, seed=seed,
               part=r.random() < 0.5, spread=r.choice([0.1, 1.0, 2.5]))


@pytest.mark.parametrize("seed", range(100, 116))
def test_move(seed):
    r, form, page, lengths = drawn(seed)
    here = seed % 2 == 0
    run_move(form, page, r.choice(["one", "heads", "tokens", "each"] + ["copy"] * (not here)),
             r.choice([2, 4, 16, 18, 50, 64, 96, 100, 126, 128]), r.random() < 0.5, in_place=here, seed=seed,
             lens=lengths(r.choice([1, 3, 9]), 400) + [77])


@pytest.mark.parametrize("seed", range(200, 232))
def test_cross(seed):
    r, form, page, lengths = drawn(seed)
    hkv, g = r.choice([1, 2, 3, 5]), r.choice([1, 2, 4, 8])
    few = seed % 2 == 0
    new = lengths(r.choice([1, 5, 40] if few else [1, 3, 7]), 64 // g + 1 if few else 400) + [3 if few else 90]
    lens = lengths(len(new) - 1, r.choice([60, 800, 2500])) + [r.choice([40, 1700])]
    run_cross(ref.Cache(lens, hkv, form, page, seed=seed, spread=1.0), hkv * g, new, splits=r.choice([0, 0, 0, 1, 3, 7]),
              seed=seed, scale=r.choice([0.0, 0.3]))
