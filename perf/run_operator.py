"""Runs listed cases of operators.py and more_operators.py on the framework's own calls, for a profiler:
python3 perf/run_operator.py CASE[,CASE...] [CALLS]"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import torch  # noqa: E402

from perf import more_operators, operators  # noqa: E402

calls = int(sys.argv[2]) if len(sys.argv) > 2 else 20
cases = {}
for module in (operators, more_operators):
    module.own = True
    cases |= {c["name"]: (module, c) for c in module.listed()}
for name in sys.argv[1].split(","):
    module, case = cases[name]
    states = [module.prepare(case, seed) for seed in (0, 1)]
    for i in range(calls):
        module.run(states[i % 2])
    torch.cuda.synchronize()
    print(name, calls, flush=True)
