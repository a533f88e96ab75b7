"""The plans of the library's matrix products, printed by a host program built from the library's own header."""
import os
import subprocess
import tempfile

from paper_2605_01989_b200 import build as lib_build

PROGRAM = r"""
#include <stdio.h>
#include "product_plan.h"

using namespace dblp;

int main()
{
    unsigned M, N, K, batch, terms, few, symmetric, a_mn, b_mn, whole;
    while (scanf("%u %u %u %u %u %u %u %u %u %u", &M, &N, &K, &batch, &terms, &few, &symmetric, &a_mn, &b_mn, &whole) == 10) {
        Product p{};
        auto operand = [&](bool mn, uint32_t rows) {                // padded rows, or (whole = 0) rows off 16 bytes
            const uint32_t inner = mn ? rows : K;
            const int64_t stride = whole ? (inner + 15) / 16 * 16 : inner | 1;
            return Operand{(const void*)4096, nullptr, stride, stride * (mn ? K : rows), mn};
        };
        p.a = operand(a_mn, M);
        p.b = operand(b_mn, N);
        p.M = M;
        p.N = N;
        p.K = K;
        p.batch = batch;
        p.dtype = 1;
        p.terms = (int)terms;
        p.few = few;
        p.symmetric = symmetric;
        const ProductPlan r = plan_product(p);
        printf("%d %d %u %u %u %u %u %u %u %d %d %d %u\n", (int)rows_take(p), r.cg, r.bn, r.tiles, r.whole, r.rest, r.parts, r.per, r.items, (int)r.turned,
               (int)r.several, (int)(r.copy_a || r.copy_b), r.longest);
    }
}
"""
FIELDS = ("rows_take", "cg", "bn", "tiles", "whole", "rest", "parts", "per", "items", "turned", "several", "copies", "longest")
_folder, _program = None, None


def plans(products):
    """A dict per product; a product is a dict of M, N, K and, where they differ from 1, 1, 0, 0, 0, 0, 1: batch, terms, few, symmetric,
    a_mn, b_mn (the rows of an operand are contiguous, not the summed dimension) and whole (rows on 16 bytes)."""
    global _folder, _program
    if _program is None:
        _folder = tempfile.TemporaryDirectory()
        source, _program = os.path.join(_folder.name, "plans.cpp"), os.path.join(_folder.name, "plans")
        with open(source, "w") as f:
            f.write(PROGRAM)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", lib_build.CSRC, "-o", _program, source], check=True)
    default = dict(batch=1, terms=1, few=0, symmetric=0, a_mn=0, b_mn=0, whole=1)
    text = "".join("%d %d %d %d %d %d %d %d %d %d\n" % tuple({**default, **p}[k] for k in (
        "M", "N", "K", "batch", "terms", "few", "symmetric", "a_mn", "b_mn", "whole")) for p in products)
    out = subprocess.run([_program], input=text, capture_output=True, text=True, check=True).stdout
    return [dict(zip(FIELDS, map(int, line.split()))) for line in out.splitlines()]


def forward(n, i, o, turned=False):
    return dict(M=n, N=o, K=i, few=1, b_mn=not turned)


def grad_x(n, i, o, turned=False):
    return dict(M=n, N=i, K=o, few=1, b_mn=turned)


def grad_w(n, i, o, turned=False):
    return dict(M=o if turned else i, N=i if turned else o, K=n, a_mn=1, b_mn=1)


def update(b, m, n, precise):
    """X X^T (of the shorter side), A A, B X."""
    low, high, tall, terms = min(m, n), max(m, n), m > n, 3 if precise else 1
    return [dict(M=low, N=low, K=high, batch=b, terms=terms, symmetric=1, a_mn=tall, b_mn=tall),
            dict(M=low, N=low, K=low, batch=b, terms=terms, symmetric=1), dict(M=m, N=n, K=low, batch=b, terms=terms, b_mn=not tall)]
