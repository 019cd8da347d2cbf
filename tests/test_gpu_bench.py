"""bench.py on a small workload whose workers take their gradients themselves."""
import json
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_layer_workload_steps_start_with_a_flushed_cache(monkeypatch, capsys):
    # the gradients leave rows in the memory-side cache; like that of every workload
    # below 1 GiB, the timed step is not to find them there
    import bench
    from paper_2507_07114_amd import probe
    from workloads.device import DeviceState
    calls = []

    def spy(owner, name):
        real = getattr(owner, name)

        def call(*args, **kw):
            calls.append(name)
            return real(*args, **kw)
        monkeypatch.setattr(owner, name, call)

    spy(DeviceState, "local_gradients")
    spy(DeviceState, "fused")
    spy(probe, "hbm_probe_read")
    monkeypatch.setattr(bench, "hbm_copy_probe", lambda: 1.0)
    monkeypatch.setattr(bench, "hbm_probes", lambda *a: {"copy_16B": 1.0})
    monkeypatch.setattr(sys, "argv", ["bench.py", "--workload", "n8_layer16m_bf16_adam",
                                      "--steps", "3", "--warmup", "1", "--no-cpu-baseline"])
    bench.main()
    line = json.loads(capsys.readouterr().out)
    # the buffers' first gradients, the warmup, and the timed steps
    assert calls == (["local_gradients", "fused"]
                     + 3 * ["local_gradients", "hbm_probe_read", "fused"])
    assert line["config"]["mall_flush_between_steps"] == "read"
    assert line["steps"] == 3 and line["value"] > 0
    assert line["ms_per_step"] == pytest.approx(line["roofline"]["launch_ms"], abs=1e-3)
    assert 0 < line["local_gradients_ms"]["min"] <= line["local_gradients_ms"]["max"]
