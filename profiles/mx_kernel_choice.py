"""How the built-in choice of a kernel of the MX product (csrc/mx_matmul.hip: the smallest of fitted estimates) compares with the fastest kernel, over the
times in mx_kernel_choice_times.csv: per kind of activations the mean and the largest ratio of the chosen kernel's time to the fastest one's, the worst
products, the relative error of the estimates, and the mean without each of the kernels in the tables.

    python3 profiles/mx_kernel_choice.py
"""
import csv
import math
import os
import re

HERE = os.path.dirname(os.path.abspath(__file__))
SOURCE = os.path.join(HERE, "..", "paper_2310_15929_amd", "csrc", "mx_matmul.hip")
CUTS = (1, 2, 3, 4, 6, 8)
COMPUTE_UNITS = 256


def ceil_div(a, b):
    return -(-a // b)


def table(source, kind, act):
    """{(kind, the kernel's numbers): its constants}"""
    lines = re.search(r"#define MX_%s_%s\(X\)((?: *\\\n  X\([^)]*\))*)" % (kind.upper() + ("S" if kind == "tile" else ""), act.upper()), source).group(1)
    rows = [[float(v) for v in x.split(",")] for x in re.findall(r"X\(([^)]*)\)", lines)]
    n = 4 if kind == "rows" else 6
    return {(kind,) + tuple(int(v) for v in r[:n]): r[n:] for r in rows}


def estimate(kernel, constants, M, N, K, cut):
    steps, row_tiles = ceil_div(K, 128), ceil_div(N, 64) * 4
    if kernel[0] == "rows":
        (t0, c, b, d), (token_tiles, rows) = constants, kernel[1:3]
        groups = ceil_div(row_tiles, rows) * ceil_div(M, 16 * token_tiles)
        filled = min(M, 16 * token_tiles) / (16 * token_tiles)
        return t0 + steps * (c * ceil_div(groups, COMPUTE_UNITS) + b * groups / COMPUTE_UNITS) * (1 - d + d * filled)
    t0, e, c, u, r0, r = constants
    per = ceil_div(steps, cut)
    pieces = ceil_div(steps, per)
    load = ceil_div(ceil_div(row_tiles * 16, kernel[1] * kernel[3] * 16) * ceil_div(M, kernel[2] * kernel[4] * 16) * pieces, COMPUTE_UNITS)
    return t0 + e * load + c * per * max(1, u * load) + (r0 + pieces * M * row_tiles * 64e-6 * r if pieces > 1 else 0)


def choose(kernels, M, N, K):
    """(kernel, cut) as the library chooses among those that it offers for a size"""
    steps, row_tiles = ceil_div(K, 128), ceil_div(N, 64) * 4
    offers = []
    for kernel, constants in kernels.items():
        if kernel[0] == "rows":
            t = kernel[1]
            if (8 * t if t > 1 else 0) < M <= (128 if t == 4 else 16 * t):
                offers.append((kernel, 1))
        elif M > 16:
            tokens = kernel[2] * kernel[4] * 16
            if tokens <= 64 or M > tokens // 2:
                offers += [(kernel, cut) for cut in CUTS if cut == 1 or (steps >= 2 * cut and cut * M * row_tiles * 64 <= 256 << 20)]
    return min(offers, key=lambda o: estimate(o[0], kernels[o[0]], M, N, K, o[1]))


def read_times():
    """{act: {(M, N, K): {(kernel, cut): us}}}"""
    times, names = {}, []
    for line in csv.reader(l for l in open(os.path.join(HERE, "mx_kernel_choice_times.csv")) if not l.startswith("#")):
        if line[0] == "activations":
            names = [tuple(n.split()[:1]) + tuple(int(v) for v in n.split()[1:]) for n in line[4:]]
            continue
        cells = {}
        for name, cell in zip(names, line[4:]):
            cells.update({(name, cut): float(us) for cut, us in zip(CUTS, cell.split()) if us != "-"})
        times.setdefault(line[0], {})[tuple(int(v) for v in line[1:4])] = cells
    return times


def ratios(cases, kernels):
    """(ratio to the fastest of all kernels, product, chosen, its time, the fastest time), largest first"""
    out = []
    for product, cells in cases.items():
        chosen = choose(kernels, *product)
        if chosen not in cells:  # (without one of the kernels, a cut of K that was not timed)
            chosen = min((k for k in cells if k[0] in kernels), key=lambda k: estimate(k[0], kernels[k[0]], *product, k[1]))
        best = min(cells.values())
        out.append((cells[chosen] / best, product, chosen, cells[chosen], best))
    return sorted(out, reverse=True)


def mean(values):
    values = list(values)
    return sum(values) / len(values)


def main():
    source = open(SOURCE).read()
    for act, cases in read_times().items():
        kernels = {**table(source, "rows", act), **table(source, "tile", act)}
        r = ratios(cases, kernels)
        measured = {k[0] for cells in cases.values() for k in cells}
        assert set(kernels) <= measured, "a kernel of the tables has no times"
        errors = [math.log(estimate(k[0], kernels[k[0]], *p, k[1]) / us) for p, cells in cases.items() for k, us in cells.items() if k[0] in kernels and us <= 1.3 * min(cells.values())]
        print(f"{act}: {len(cases)} products, {len(kernels)} kernels in the tables of {len(measured)} measured: {mean(x[0] for x in r):.4f} of the fastest on average, {r[0][0]:.3f} at most; "
              f"estimates within 1.3 of the fastest are off by {mean(abs(e) for e in errors):.3f} on average")
        for ratio, product, (kernel, cut), us, best in r[:3]:
            print(f"   {ratio:.3f}  {' x '.join(map(str, product))}: {' '.join(map(str, kernel))} cut {cut} {us} us, fastest {best}")
        for kernel in kernels:
            rest = {k: v for k, v in kernels.items() if k != kernel}
            print(f"   without {' '.join(map(str, kernel)):22} {mean(x[0] for x in ratios(cases, rest)):.4f}")


if __name__ == "__main__":
    main()
