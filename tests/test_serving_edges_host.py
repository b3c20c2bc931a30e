"""Host side of the calls that a server makes around the 8-bit cache: what the binding takes, and what it refuses."""
import numpy as np
import pytest
import torch

from paper_2609_14717_b200 import binding, synth


def _cfg(S=2, W=4, layers=2, n_pages=5, width=3, kv8=True, carry_rounds=1):
    sh = synth.DrafterShape(dtype="bf16", d_target=8, n_cap=1, d_model=256, n_layers=layers, n_q=2, n_kv=1, hd=128, vocab=64, W=W,
                            page=16, kv8=kv8, carry_rounds=carry_rounds)
    return binding.make_config(sh, S, width, n_pages)


@pytest.mark.parametrize("kv8", [True, False])
def test_a_state_takes_the_tensors_that_its_caller_has(kv8):
    cfg = _cfg(kv8=kv8, carry_rounds=2)
    table, lens = np.arange(6, dtype=np.int64).reshape(2, 3), [4, 5]
    own = {"kv_pool": torch.empty((2, 5, 1, 2, 16, 128), dtype=torch.float8_e4m3fn if kv8 else torch.bfloat16),
           "kv_scale": torch.empty((2, 5, 1, 2)), "carry_kv": torch.empty((2, 2, 1, 2, 8, 128), dtype=torch.bfloat16),
           "carry_len": torch.ones(2, dtype=torch.int32), "carry_hist": torch.ones((2, 2), dtype=torch.int32)}
    st = binding.State(cfg, "bf16", 2, table, lens, device="cpu", **own)
    for k, v in own.items():
        assert getattr(st, k) is (v if kv8 or k != "kv_scale" else None), k
    assert st.block_table.tolist() == table.tolist() and st.committed_len.tolist() == lens
    fresh = binding.State(cfg, "bf16", 2, table, lens, device="cpu")
    for k, v in own.items():
        if kv8 or k != "kv_scale":
            assert getattr(fresh, k).shape == v.shape and getattr(fresh, k).dtype == v.dtype and not getattr(fresh, k).float().any()
    for k, v in own.items():
        if kv8 or k != "kv_scale":
            for bad in (v[:1], v.double()):
                with pytest.raises(ValueError, match=k):
                    binding.State(cfg, "bf16", 2, table, lens, device="cpu", **{k: bad})
