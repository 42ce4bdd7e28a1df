"""The counter table that bench.py reports beside the training step's rate is of the kernels that are there: it is ignored when their
sources have changed since, and then the figure is lost without a word."""
import bench


def test_the_counter_table_is_of_the_present_kernels():
    table, where = bench.measured_traffic("c2")
    assert table is not None, where
    assert set(table) >= {"proj_qkv", "attn_fwd_bf16", "attn_bwd_dkv_bf16"} and all(v > 0 for v in table.values())
