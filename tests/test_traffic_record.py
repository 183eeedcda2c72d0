"""The measured HBM traffic that bench.py reports belongs to the attention kernels as they are: host files only."""
import pytest

import bench
import dream_inputs as di
import paper_2505_19201_amd as dream


@pytest.mark.parametrize("name", sorted(bench.PAPER_TAU))
def test_the_committed_figure_is_not_stale(name):
    """The file was measured on the kernel that the launch plan names, built from the sources as they are.  What only other kernels use has no place in the headers they share: a line
    there loses the figures of kernels that it does not change.  (After a change to those sources the traffic is measured again.)"""
    cfg = di.CONFIGS[name]
    rows = cfg.prefix + cfg.n_tree
    plan = dream.dream_attn_plan_describe(dream.attn_desc(cfg.batch, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, dream.BF16, rows), cfg.n_tree, rows)
    traffic, source = bench.read_traffic(name, plan)
    assert traffic is not None, source
