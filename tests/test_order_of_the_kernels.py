"""The order in which work-groups take tiles of packed sequences, and the dealing of a cache's keys, asked of the kernels' own functions (compiled for
the host, tests/host_runtime/order.cpp): every tile has one rank, heavier tiles come first, pieces cover every run, parts have slots of their own."""
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("order")
    csrc = os.path.join(ROOT, "paper_2301_08984_amd", "csrc")
    obj, exe = str(d / "order.o"), str(d / "order")
    src = os.path.join(ROOT, "tests", "host_runtime", "order.cpp")
    r = subprocess.run(["hipcc", "-x", "hip", "--cuda-host-only", "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", csrc, "-c", src, "-o", obj],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    subprocess.check_call(["g++", obj, "-o", exe, "-no-pie", "-Wl,--unresolved-symbols=ignore-all"])

    def f(questions):
        r = subprocess.run([exe], input="\n".join(questions), capture_output=True, text=True, timeout=60)
        assert r.returncode == 0
        out = r.stdout.split("\n")[:-1]
        assert len(out) == len(questions)
        return [[int(x) for x in line.split()] for line in out]
    return f


def pairs(x):
    return list(zip(x[::2], x[1::2]))


def test_every_rank_and_head_has_one_work_group(ask):
    heads = list(range(1, 40)) + [64, 96, 100]
    for HK, got in zip(heads, ask([f"p {48 * HK} {HK}" for HK in heads])):
        assert sorted(pairs(got)) == [(r, h) for r in range(48) for h in range(HK)], HK


@pytest.mark.parametrize("keys,sh", [(0, 7), (1, 5), (1, 6), (1, 7)])
@pytest.mark.parametrize("G", [1, 2, 3, 5, 8, 40])
def test_every_tile_has_one_rank_and_heavy_ones_come_first(ask, keys, sh, G):
    rng = np.random.default_rng(100 * keys + 10 * sh + G)
    batches = []
    for i in range(40):
        n_seq = int(rng.integers(1, 65)) if i % 2 else int(rng.integers(1, 4))
        most = int(rng.choice([3, 40, 300, 1500]))
        n = rng.integers(0, most, n_seq)
        m = n if i % 4 == 0 else n + rng.integers(0, 500, n_seq) if i % 4 == 1 else rng.integers(0, most, n_seq)
        batches.append([(int(a), int(b)) for a, b in zip(n, m)])
    batches += [[(0, 0)], [(0, 300)], [(300, 0)], [(1, 1)], [(700, 1)], [(1, 700)], [(0, 0), (5, 0), (0, 5)]]
    got = ask([f"t {keys} {sh} {G} {len(b)} " + " ".join(f"{n} {m}" for n, m in b) for b in batches])
    for batch, line in zip(batches, got):
        want, steps = [], {}
        for b, (n, m) in enumerate(batch):
            for t in range(-(-(m if keys else n * G) // (1 << sh))):
                want.append((b, t))
                if keys:  # rows of 32 (token, head) pairs that see the tile's first key, or later ones
                    first = max((t << sh) - (m - n), 0)
                    steps[b, t] = -(-max(n - first, 0) * G // 32)
                else:  # blocks of 64 keys that the tile's last row sees
                    last = min((t + 1 << sh) - 1, n * G - 1) // G
                    steps[b, t] = -(-max(last + m - n + 1, 0) // 64)
        order = pairs(line)
        assert sorted(order) == want, batch
        heavy = [steps[x] for x in order]
        assert heavy == sorted(heavy, reverse=True), batch


@pytest.mark.parametrize("seed", range(6))
def test_pieces_cover_the_line_and_parts_have_slots_of_their_own(ask, seed):
    rng = np.random.default_rng(seed)
    for _ in range(12):
        G, n_seq, pieces = int(rng.integers(1, 20)), int(rng.integers(1, 40)), int(rng.integers(1, 65))
        lens, new = rng.integers(0, 4000, n_seq) * rng.integers(0, 2, n_seq), rng.integers(0, 40, n_seq)
        runs = []
        for b, (many, units, n_runs) in enumerate(ask([f"c 0 {n} {G} {x}" for n, x in zip(new, lens)])):
            assert many == (new[b] * G > 64) and n_runs == (0 if not new[b] else -(-int(new[b]) * G // 128) if many else 1)
            assert units == max(1, -(-int(lens[b]) // (64 if many else 128)))
            runs += [(b, g, units) for g in range(n_runs)]
        total = sum(u for _, _, u in runs)
        if not total:
            continue
        each = ask([f"e 2 {total} {pieces}"])[0][0]
        assert each >= 2 and each * pieces >= total and (each == 2 or (each - 1) * pieces < total)
        starts = list(np.cumsum([0] + [u for _, _, u in runs[:-1]]))
        parts, questions = [], []
        for piece in range(pieces):  # as the attention's kernels go
            u, stop = piece * each, min(piece * each + each, total)
            while u < stop:
                i = max(k for k, s in enumerate(starts) if s <= u)
                take = min(runs[i][2] - (u - starts[i]), stop - u)
                if take < runs[i][2]:
                    parts.append((i, u - starts[i], take))
                    questions.append(f"s {piece} {each} {starts[i]}")
                u += take
        slots = [x[0] for x in ask(questions)] if questions else []
        assert len(set(slots)) == len(slots) and all(0 <= s < 2 * pieces for s in slots)
        written = dict(zip(slots, parts))
        for i, (_, _, units) in enumerate(runs):  # as the joining kernel finds them
            begin = int(starts[i])
            piece, n = begin // each, (begin + units - 1) // each - begin // each + 1
            if n == 1:
                assert all(w[0] != i for w in written.values())
                continue
            found = [x[0] for x in ask([f"s {piece} {each} {begin}", f"s {piece + 1} {each} {begin}"])]
            got = [written.pop(s) for s in [found[0]] + [found[1] + 2 * x for x in range(n - 1)]]
            assert [w[0] for w in got] == [i] * n and sum(w[2] for w in got) == units
            assert [w[1] for w in got] == list(np.cumsum([0] + [w[2] for w in got[:-1]]))
        assert not written
