"""What bench.py prints: one short JSON line on stdout, the long tables on stderr, nothing lost between them."""
import json


def test_result_is_one_short_line_and_the_rest_is_on_stderr(capsys):
    import bench
    line = {"metric": "bitlinear_prefill_tops_7b", "value": 2424.123456789, "unit": "TOPS", "n_gpus": 1, "steps": 20, "warmup": 5,
            "ms_per_step": 58.8, "config": {"workload": "x" * 200}, "clocks": {"sm_mhz": 1500.0}, "roofline": {"achieved": 1.0 / 3},
            "e2e": {"value": 108.0}, "gpu_launches": 4620, "cpu_baseline": None, "decode": {"tokens_1": {"us": 1.0 / 7}}, "block": {"ms": 2.0}}
    tables = {k: {"points": [{"us": i / 3.0} for i in range(300)]} for k in bench.LONG_KEYS}
    bench.print_line(dict(line, **tables))
    out, err = capsys.readouterr()
    assert out.count("\n") == 1 and len(out) < 4096
    assert json.loads(out) == line
    assert err.count("\n") == 1 and json.loads(err) == {"metric": line["metric"], "legs": tables}
    bench.print_line(dict(line, sweep=None))  # legs that were not run
    out, err = capsys.readouterr()
    assert json.loads(out) == line and err == ""
