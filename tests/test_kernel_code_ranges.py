"""The built dk/dv kernels of attention over key ranges of head dimension 128 keep the distances of their accumulators, as
test_kernel_code.py checks them for the causal one."""
import os

import pytest

import test_kernel_code as K

SYMBOLS = [f"_ZN12_GLOBAL__N_118range_flash_dkv128ILb{c}ELb{b}EEEv9RangeArgs" for c in (0, 1) for b in (0, 1)]


@pytest.mark.skipif(not (os.path.exists(K.LIB) and os.path.exists(K.OBJDUMP)), reason="needs the built library and llvm-objdump")
@pytest.mark.parametrize("symbol", SYMBOLS)
def test_accumulators_keep_their_distances(symbol, monkeypatch, tmp_path):
    monkeypatch.setattr(K, "SYMBOL", symbol)
    K.test_dkv128_accumulators_keep_their_distances(tmp_path)
