"""bench.py --run: the chains of a searched workload."""
import os
import subprocess
import sys

import pytest

import mmee_inputs as mi
import paper_2604_03446_b200 as mm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("args", [["--workload", "reconfig"], ["--impl", "reference"]])
def test_run_is_refused_where_nothing_would_be_run(args):
    done = subprocess.run([sys.executable, os.path.join(ROOT, "bench.py"), "--run"] + args, capture_output=True, text=True)
    assert done.returncode == 2 and "--run" in done.stderr


@pytest.mark.gpu
def test_a_line_says_which_products_were_searched_and_which_run():
    """The gated block has three, the two-GEMM chain whose mapping was searched two; attention has the two that were searched."""
    import bench
    cfg = mi.config1()
    h = mm.mmee_create(cfg["workload"], cfg["arch"], cfg["searches"][0])
    best, _ = mm.mmee_search_host(h)
    mm.mmee_destroy(h)
    (line,) = bench.run_chains("tiny", [(cfg, cfg["searches"][0])], [best], steps=1)
    assert line["products"] == dict(searched=2, run=2)
    chain = [c for c in mi.beyond_attention_configs() if c["name"] == "mlp_768_64_384_64"][0]
    (line,) = bench.run_chains("beyond", [(chain, chain["searches"][0])], [best], steps=1)
    assert line["products"] == dict(searched=2, run=3)
    w = chain["workload"]
    assert abs(line["tflops"] * line["ms"] * 1e9 - 2 * w["seq_q"] * w["seq_kv"] * (2 * w["d_qk"] + w["d_v"])) < 1e3
