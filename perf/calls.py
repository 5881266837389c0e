"""Calls of the listed cases of operators.py, for a profiler.

    python3 perf/calls.py [NAME,NAME...] [calls of each case] [inputs of each case]

Every case (or those whose names begin so) is prepared from as many seeds as it has inputs and
called on one after the other.  Prints the time of a call: of the host alone, and with the GPU.
"""
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import perf.operators as operators  # noqa: E402


def main(names=(), calls=20, inputs=3):
    operators.own = True
    for case in operators.listed():
        if names and not case["name"].startswith(tuple(names)):
            continue
        states = [operators.prepare(case, seed + 1) for seed in range(inputs)]
        for state in states:
            operators.run(state)
        torch.cuda.synchronize()
        start = time.perf_counter()
        for i in range(calls):
            operators.run(states[i % inputs])
        host = time.perf_counter() - start
        torch.cuda.synchronize()
        both = time.perf_counter() - start
        print(f"{case['name']:28s} host {1e6 * host / calls:8.2f} us  call {1e6 * both / calls:8.2f} us", flush=True)


if __name__ == "__main__":
    main([n for n in (sys.argv[1] if len(sys.argv) > 1 else "").split(",") if n], *map(int, sys.argv[2:4]))
