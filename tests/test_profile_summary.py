"""Summaries of profiler output, from files like the profiler's."""
import csv

import profile_summary


def test_a_kernel_that_a_pass_launches_twice_counts_twice(tmp_path, capsys):
    """1000 passes of two calls with two kernels each: 4 and 2 us a launch, 12 a pass."""
    (tmp_path / "case").mkdir()
    with open(tmp_path / "case" / "kt_kernel_trace.csv", "w", newline="") as f:
        rows = csv.writer(f)
        rows.writerow(["Kernel_Name", "Start_Timestamp", "End_Timestamp"])
        for i in range(2000):
            for k, (name, us) in enumerate((("quoka::first(int)", 4), ("quoka::second(int)", 2))):
                rows.writerow([name, 20000 * i + 9000 * k, 20000 * i + 9000 * k + 1000 * us])
    profile_summary.cases(str(tmp_path), "more_operators")
    out = capsys.readouterr().out
    assert "## case: 12.0 us in kernels per pass" in out
    lines = [line.split() for line in out.splitlines()]
    assert ["first", "2", "4.00", "4.00", "4.00"] in lines and ["second", "2", "2.00", "2.00", "2.00"] in lines
