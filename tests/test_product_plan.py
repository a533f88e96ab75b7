"""How products are cut, on the CPU: every tile and every stage once, within the device's multiprocessors and the kernels' limits."""
import random

import plans as pl


def cases():
    rng = random.Random(5)
    size = lambda: int(2 ** rng.uniform(0, 14))
    found = []
    for _ in range(300):
        n, i, o, turned = size(), size(), size(), rng.random() < 0.5
        found += [pl.forward(n, i, o, turned), pl.grad_x(n, i, o, turned), pl.grad_w(n, i, o, turned)]
        found += pl.update(rng.choice([1, 1, 3, 8]), min(n, 4000), min(i, 4000), rng.random() < 0.5)
    return [dict(p, whole=rng.random() < 0.7) for p in found]


def test_every_tile_and_stage_is_done_once():
    products = cases()
    for p, r in zip(products, pl.plans(products)):
        M, N = (p["N"], p["M"]) if r["turned"] else (p["M"], p["N"])
        tm, bn, batch, slots = 128 * r["cg"], r["bn"], p.get("batch", 1), 148 // r["cg"]
        mt, nt = -(-M // tm), -(-N // bn)
        want = sum(nt - i * tm // bn for i in range(mt)) if p.get("symmetric") else mt * nt
        assert r["tiles"] == want and r["whole"] + r["rest"] == want * batch
        steps = -(-p["K"] // 64) * p.get("terms", 1)
        assert r["parts"] * r["per"] >= steps > (r["parts"] - 1) * r["per"]          # no part is empty
        assert r["items"] == r["whole"] + r["rest"] * r["parts"] and (r["parts"] > 1) == (r["rest"] > 0)
        assert r["rest"] == 0 or r["whole"] % slots == 0                             # only the last round is cut
        assert bn in (64, 128, 256) if not r["turned"] else N <= bn <= 128 and r["cg"] == 1
        assert not r["several"] or r["items"] > slots


def test_rows_off_sixteen_bytes_are_copied():
    a, b = pl.plans([dict(pl.forward(777, 1601, 1999), whole=w) for w in (1, 0)])
    assert not a["copies"] and b["copies"]
