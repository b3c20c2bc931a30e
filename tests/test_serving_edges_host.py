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


def _tables(S=3, rows=20, **kw):
    cfg = _cfg(S=S, carry_rounds=2)
    st = binding.State(cfg, "bf16", S, np.zeros((S, 3), np.int32), np.zeros(S, np.int32), device="cpu")
    return cfg, binding.Pages(cfg, S, device="cpu"), st, binding.RowPlan(S, rows, device="cpu")


def test_page_table_calls_take_larger_tensors_and_refuse_smaller_ones():
    """The library writes row_off[S], held[S - 1] and so on: a tensor that ends before that is refused (device -1 is the host's)."""
    cfg, pages, st, plan = _tables()

    def marshal(pages, st, plan, S=3, device=-1):
        sizes = binding._Sizes(cfg, device)
        return st.table_struct(sizes, S), pages.struct(sizes, S), plan.struct(sizes, S)

    a, b, c = marshal(pages, st, plan)
    assert (a.block_table, a.carry_hist, b.held, c.row_seq, c.max_rows) == (
        st.block_table.data_ptr(), st.carry_hist.data_ptr(), pages.held.data_ptr(), plan.row_seq.data_ptr(), 20)
    marshal(pages, st, plan, S=2)
    none = _tables()
    none[2].carry_hist, none[3].row_pos = None, None            # what may be NULL is left to the library
    a, _, c = marshal(*none[1:])
    assert a.carry_hist is None and c.row_pos is None
    small = _cfg(S=2, carry_rounds=2)
    cases = [("held", binding.Pages(cfg, 2, device="cpu"), st, plan), ("row_off", pages, st, binding.RowPlan(2, 20, device="cpu")),
             ("block_table", pages, binding.State(small, "bf16", 2, np.zeros((2, 3), np.int32), np.zeros(2, np.int32), device="cpu"), plan)]
    for obj, name, value in [(0, "free_list", pages.free_list[1:]), (0, "n_free", pages.n_free[1:]), (0, "free_list", pages.free_list.long()),
                             (1, "block_table", st.block_table.view(1, 9)), (1, "block_table", torch.zeros((3, 4), dtype=torch.int32)[:, :3]),
                             (1, "committed_len", st.committed_len[:2]), (1, "committed_len", torch.zeros(6, dtype=torch.int32)[::2]),
                             (1, "carry_len", st.carry_len[:2]), (1, "carry_hist", st.carry_hist[:2]), (1, "block_table", st.block_table.float()),
                             (2, "slot", plan.slot[1:]), (2, "row_pos", plan.row_pos[1:]), (2, "row_seq", plan.row_seq[1:])]:
        objs = list(_tables()[1:])
        setattr(objs[obj], name, value)
        cases.append((name, *objs))
    for name, *objs in cases:
        with pytest.raises(ValueError, match=name):
            marshal(*objs)
    with pytest.raises(ValueError, match="device 0"):
        marshal(pages, st, plan, device=0)


@pytest.mark.parametrize("kv8", [True, False])
def test_a_cache_of_another_size_type_or_device_is_refused(kv8):
    cfg = _cfg(kv8=kv8)
    st = binding.State(cfg, "bf16", 2, np.zeros((2, 3), np.int32), np.zeros(2, np.int32), device="cpu")
    assert st.cache_struct(binding._Sizes(cfg, -1)).kv_pool == st.kv_pool.data_ptr()
    for other in (_cfg(kv8=not kv8), _cfg(kv8=kv8, n_pages=6), _cfg(kv8=kv8, layers=3)):
        with pytest.raises(ValueError, match="kv_pool"):
            st.cache_struct(binding._Sizes(other, -1))
    with pytest.raises(ValueError, match="kv_pool"):
        st.cache_struct(binding._Sizes(cfg, 0))
    if kv8:
        st.kv_scale = st.kv_scale[:1]
        with pytest.raises(ValueError, match="kv_scale"):
            st.cache_struct(binding._Sizes(cfg, -1))
