"""Times the cases of operators.py, or of another file of cases beside it, on the current GPU:
python3 perf/time_operators.py [--cases more_operators] [--only NAME,NAME] [--own N]

For every case the plain form and the entry points in turn, nine times each over inputs of three seeds: the median time of a pass among
others, in microseconds.  --own N makes N passes of every case through the entry points and times nothing (for a profiler)."""
import argparse
import importlib
import os
import statistics
import sys

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path[:0] = [os.path.dirname(HERE), HERE]

SEEDS = 3
RUN_US = 20000                                       # of the passes timed together, about


def time_of(operators, states, own, passes):
    operators.own = own
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for x in range(passes):
        operators.run(states[x % SEEDS])
    end.record()
    torch.cuda.synchronize()
    return begin.elapsed_time(end) / passes * 1e3


def main():
    args = argparse.ArgumentParser()
    args.add_argument("--cases", default="operators", choices=["operators", "more_operators"])
    args.add_argument("--only", default="")
    args.add_argument("--own", type=int, default=0)
    args = args.parse_args()
    operators = importlib.import_module(args.cases)
    only = set(filter(None, args.only.split(",")))
    for case in operators.listed():
        if only and case["name"] not in only:
            continue
        states = [operators.prepare(case, seed) for seed in range(1, 2 if args.own else 1 + SEEDS)]
        if args.own:
            operators.own = True
            for _ in range(args.own):
                operators.run(states[0])
            torch.cuda.synchronize()
            print(case["name"], flush=True)
            continue
        passes, times = {}, {False: [], True: []}
        for own in times:
            time_of(operators, states, own, SEEDS)
            passes[own] = max(SEEDS, min(300, int(RUN_US / time_of(operators, states, own, SEEDS))))
        for _ in range(9):
            for own in times:
                times[own].append(time_of(operators, states, own, passes[own]))
        plain, kernels = (sorted(times[own]) for own in (False, True))
        print(f"{case['name']:20s} plain {statistics.median(plain):9.1f}  kernels {statistics.median(kernels):8.1f} ({kernels[0]:.1f} .. {kernels[-1]:.1f})", flush=True)


if __name__ == "__main__":
    main()
