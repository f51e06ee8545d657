"""Pools' formats on the host side, without a GPU: the byte counts that the benchmark
reports, and its command line."""
import os
import subprocess
import sys

import pytest

from paper_2607_17299_amd import harness, synth, war

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("cfg", [synth.TINY, synth.LARGE])
def test_a_tokens_bytes_are_those_of_a_pool(cfg, fmt):
    pages = 7
    pool = war.lib().war_kv_pool_bytes(war.config_struct(cfg, 1), pages, war.KV_FORMATS[fmt])
    assert pool == cfg.n_layers * pages * cfg.page_size * harness.kv_token_bytes(cfg, fmt)


def test_a_pool_of_another_format_has_no_size():
    for pages, fmt in ((0, 0), (7, 2), (7, -1)):
        assert war.lib().war_kv_pool_bytes(war.config_struct(synth.TINY, 1), pages, fmt) == -1


def test_another_format_is_refused_by_name():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "bench.py"), "--kv-format", "int8"], capture_output=True,
                       text=True, timeout=60, cwd=ROOT)
    assert r.returncode == 2 and "kv-format" in r.stderr
    with pytest.raises(ValueError):
        war.Pool(synth.TINY, 4, 1, 4, device="cpu", kv_format="int8")


def test_a_line_over_8_bit_pools_does_not_call_itself_bf16():
    import bench
    assert bench.result_dtype("bf16") == "bf16"
    assert bench.result_dtype("e4m3") != "bf16" and "e4m3" in bench.result_dtype("e4m3")


def test_the_sweep_refuses_a_format_it_does_not_measure():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "bench.py"), "--sweep", "--kv-format", "e4m3"], capture_output=True,
                       text=True, timeout=60, cwd=ROOT)
    assert r.returncode == 2 and "--kv-format" in r.stderr
