"""The bench prints one line that is short enough to be kept whole; the rows of the other workloads go to stderr."""
import json

import pytest


@pytest.fixture
def rows():
    return [{"workload": "w%d" % i, "step_us": {"median": 1.0 / 3, "blocks": [1.0 / 7] * 10}} for i in range(60)]


def test_the_line_is_short_and_the_rows_go_to_stderr(rows, capsys):
    import bench
    out = {"metric": bench.METRIC, "value": 1.5, "workloads": rows, "small": rows, "clocks": {"sm_mhz": 1965}}
    bench.print_line(dict(out), whole=False)
    caught = capsys.readouterr()
    line = json.loads(caught.out)
    assert caught.out.count("\n") == 1 and line == {"metric": bench.METRIC, "value": 1.5, "clocks": {"sm_mhz": 1965}}
    assert json.loads(caught.err) == {"workloads": rows, "small": rows}


def test_the_whole_line_where_it_is_asked_for(rows, capsys):
    import bench
    out = {"metric": bench.METRIC, "value": 1.5, "workloads": rows, "small": rows}
    bench.print_line(dict(out), whole=True)
    caught = capsys.readouterr()
    assert json.loads(caught.out) == out and caught.err == ""


def test_no_rows_no_second_line(capsys):
    import bench
    bench.print_line({"value": 2.0}, whole=False)
    caught = capsys.readouterr()
    assert json.loads(caught.out) == {"value": 2.0} and caught.err == ""
