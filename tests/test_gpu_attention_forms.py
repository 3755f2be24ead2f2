"""hb_attention in every form that its choice by size takes: all keys, ragged ones, masked ones, both, and NaN where nothing is visible."""
import numpy as np
import pytest

from attentiontest import FORMS
from test_gpu_attention import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Lq,Lk,Hq,Hkv,D", FORMS)
def test_form(B, Lq, Lk, Hq, Hkv, D):
    rng = np.random.default_rng(Lk + D)
    lens, mask, nan = [Lk, 65, 0][:B], rng.random((B, Lk)) < 0.5, (np.nan, np.nan)
    run("hb_attention", B, Lq, Lk, Hq, Hkv, D, vmean=0.5, pads=(8, 16, 24))
    run("hb_attention", B, Lq, Lk, Hq, Hkv, D, lens=lens, hidden=nan, vmean=0.5)
    run("hb_attention", B, Lq, Lk, Hq, Hkv, D, mask=mask, hidden=(np.inf, np.nan))
    run("hb_attention", B, Lq, Lk, Hq, Hkv, D, lens=[Lk - 1, 64, 1][:B], mask=mask, hidden=nan, scale=-1.0)
    mask[:] = False
    mask[B - 1, Lk - 1] = True                            # one key, the last one of all
    run("hb_attention", B, Lq, Lk, Hq, Hkv, D, mask=mask, hidden=(np.nan, np.inf))
