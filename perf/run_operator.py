"""Runs listed cases of operators.py on the framework's own calls, for a profiler:
python3 perf/run_operator.py CASE[,CASE...] [CALLS]"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import torch  # noqa: E402

from perf import operators  # noqa: E402

operators.own = True
calls = int(sys.argv[2]) if len(sys.argv) > 2 else 20
cases = {c["name"]: c for c in operators.listed()}
for name in sys.argv[1].split(","):
    states = [operators.prepare(cases[name], seed) for seed in (0, 1)]
    for i in range(calls):
        operators.run(states[i % 2])
    torch.cuda.synchronize()
    print(name, calls, flush=True)
