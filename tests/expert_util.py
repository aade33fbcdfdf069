"""Helpers for the tests of the experts' operators: choices of experts and, from the definition, the order of the rows that they make; which kernels
and tiles the library takes for a product."""
import ctypes
import functools
import os
import subprocess
import tempfile

import torch


def choices(tokens, experts, chosen, seed, how="some"):
    """[tokens, chosen], different experts for each token, int32 on the host.  `how`: "some" are more popular; "even"; "one": all tokens at the first ones; "first" tokens
    alone have any (a padded batch); "holes": each choice may be missing; "none"."""
    g = torch.Generator().manual_seed(seed)
    popular = torch.randn(experts, generator=g) * {"even": 0.0}.get(how, 1.0)
    if how == "one":
        popular = -100.0 * torch.arange(experts)
    u = torch.rand(tokens, experts, generator=g).clamp(1e-7, 1 - 1e-7)
    index = (popular - torch.log(-torch.log(u))).argsort(dim=1, descending=True)[:, :chosen]
    if how == "first":
        index[(tokens + 1) // 2:] = -1
    elif how == "holes":
        index[torch.rand(index.shape, generator=g) < 0.3] = -1
    elif how == "none":
        index[:] = -1
    return index.int().contiguous()


def tables(index, experts):
    """slots, source and offsets of the definition, int32 on the host: one choice after the other."""
    tokens, chosen = index.shape
    rows = [[] for _ in range(experts)]
    flat = index.flatten().tolist()
    for i, e in enumerate(flat):
        if 0 <= e < experts:
            rows[e].append(i)
    slots, source, offsets = [-1] * len(flat), [-1] * len(flat), [0]
    for e in range(experts):
        offsets.append(offsets[e] + len(rows[e]))
    order = [i for r in rows for i in r]
    for row, i in enumerate(order):
        slots[i], source[row] = row, i // chosen
    ints = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return ints(slots).view(tokens, chosen), ints(source), ints(offsets)


def plan_on_device(experts_module, index, experts):
    """The plan of the definition in device memory, and its groups: (expert, first row, end)."""
    slots, source, offsets = tables(index, experts)
    plan = experts_module.Plan(index.cuda(), slots.cuda(), source.cuda(), offsets.cuda())
    o = offsets.tolist()
    return plan, [(e, o[e], o[e + 1]) for e in range(experts)], source


_WAYS = """
#include "expert_rules.h"
extern "C" int few_rows(int pair, uint64_t rows, uint64_t experts, uint64_t n, uint64_t k, int width) { return btb::few_rows(pair != 0, rows, experts, n, k, width); }
extern "C" int size_of(int kind, uint64_t rows, uint64_t experts, uint64_t m, uint64_t n, uint64_t k, uint64_t outputs, int width) {
    return btb::size_of((btb::Kind)kind, rows, experts, m, n, k, outputs, width);
}
extern "C" unsigned most_parts(int kind, int size, uint64_t rows, uint64_t experts, uint64_t m, uint64_t n, uint64_t k, uint64_t outputs, int width) {
    return btb::parts_of((btb::Kind)kind, (btb::Size)size, rows, experts, m, n, k, outputs, width).most;
}
"""
PAIR, PLAIN, BACK, BACK_PAIR, WEIGHTS = range(5)                   # csrc/expert_rules.h, as are the sizes
SMALL, MIDDLE, LARGE = range(3)


@functools.lru_cache(None)
def rules():
    """The rules by which a product's kernel and tiles are chosen, as the library has them."""
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2110_15362_amd", "csrc")
    with tempfile.TemporaryDirectory() as tmp:
        source, lib = os.path.join(tmp, "ways.cpp"), os.path.join(tmp, "ways.so")
        with open(source, "w") as f:
            f.write(_WAYS)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fPIC", "-shared", "-I", csrc, source, "-o", lib], check=True)
        L = ctypes.CDLL(lib)
    u64, ci = ctypes.c_uint64, ctypes.c_int
    L.few_rows.argtypes = [ci] + [u64] * 4 + [ci]
    L.size_of.argtypes = [ci] + [u64] * 6 + [ci]
    L.most_parts.argtypes, L.most_parts.restype = [ci, ci] + [u64] * 6 + [ci], ctypes.c_uint
    return L


def takes_few_rows(kind, rows, experts, d, f, width):
    """Whether a forward product with weights [experts, f, d] reads them straight to registers."""
    return bool(rules().few_rows(kind == PAIR, rows, experts, f, d, width))


def tiles_of(kind, groups, rows, experts, d, f, width):
    """(size of the tiles, how many of them there are, and of those the whole ones and into how many parts each of the rest goes) for a product of weights [experts, f, d] whose operands are
    fetched straight to LDS; groups: (expert, first row, end)."""
    m, n, k, outputs = {PAIR: (0, f, d, 0), PLAIN: (0, f, d, 0), BACK: (0, d, f, 0), BACK_PAIR: (0, d, f, 0)}[kind]
    size = rules().size_of(kind, rows, experts, m, n, k, outputs, width)
    side, slots = (64, 128, 256)[size], (1024, 512, 256)[size]
    last = groups[-1][2]
    count = sum(-(-(b - a) // side) for a, b in [g[1:] for g in groups] + [(last, rows)]) * -(-n // (side // 2 if kind == PAIR else side))
    most, splits, full = rules().most_parts(kind, size, rows, experts, m, n, k, outputs, width), 1, count // slots * slots
    while splits < most and (count - full) * splits * 2 <= slots:
        splits *= 2
    return size, count, full, splits
