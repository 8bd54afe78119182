"""Where tensors lie and whether they meet (csrc/launch_plan.h), compiled for the host, against sets of bytes."""
import random

from test_launch_plan_cpu import run


def bytes_of(at, size, dims):
    out = {at}
    for n, step in dims:
        out = {x + i * step for x in out for i in range(n)}
    return {x + i for x in out for i in range(size)}


def place(at, size, dims):
    return "ra::place_of(base + %d, %d%s)" % (at, size, "".join(", {%d, %d}" % d for d in dims))


def test_places_meet_where_their_bytes_do(tmp_path):
    """Random layouts: nested ones, parts of one buffer with the same steps, steps that do not nest, zero and negative."""
    rng = random.Random(1)
    cases = []
    for k in range(3000):
        steps = [rng.choice([0, 2, 4, 6, 8, 12, 16, 24, 30, 48, 64, 96, -8]) for _ in range(3)]
        pair = []
        for _ in range(2):
            dims = [(rng.choice([1, 1, 2, 3, 4]), s if k % 2 else rng.choice([0, 2, 6, 8, 10, 16, 40, 64, -16])) for s in steps]
            if rng.random() < 0.3:
                rng.shuffle(dims)
            pair.append((rng.randrange(0, 120, 2), rng.choice([2, 4, 6, 8]), dims))
        cases.append(pair)
    flat = lambda t: "%d,%d,%s" % (t[0], t[1], ",".join("%d,%d" % d for d in t[2]))  # noqa: E731
    body = """const char* base = reinterpret_cast<const char*>(1 << 20);
      static const int t[][16] = {%s};
      auto place = [&](const int* v) { return ra::place_of(base + v[0], v[1], {v[2], v[3]}, {v[4], v[5]}, {v[6], v[7]}); };
      for (auto& v : t) {
        const ra::Place a = place(v), b = place(v + 8);
        printf("%%d%%d%%d ", int(ra::meet(ra::merged(a), ra::merged(b))), int(ra::meet(a, b)), int(ra::meets_itself(a)));
      }""" % ",\n".join("{%s,%s}" % (flat(a), flat(b)) for a, b in cases)
    for (a, b), got in zip(cases, run(tmp_path, body)):
        A = bytes_of(*a)
        want = not A.isdisjoint(bytes_of(*b))
        count = a[1]
        for n, step in a[2]:
            count *= n if step else 1  # a step of zero is one place
        assert got == "%d%d%d" % (want, want, len(A) < count), (a, b, got)


def test_places_of_large_tensors_take_few_steps(tmp_path):
    """q, k and v side by side in one buffer, slots of a cache and whole tensors; the answer comes within the steps
    allowed (it would be no otherwise), and nowhere is not met."""
    B, H, n, d = 8, 32, 100000, 128
    row = 3 * H * d * 2
    side = [(i * H * d * 2, d * 2, [(B, n * row), (H, d * 2), (n, row)]) for i in range(3)]
    slots = [(off * d * 2, d * 2, [(B, H * n * d * 2), (H, n * d * 2), (m, d * 2)]) for off, m in ((0, 40000), (40000, 60000))]
    shifted = (H * d * 2 + d * 2 - 16, d * 2, side[0][2])  # the last bytes of k's first head
    body = "const char* base = reinterpret_cast<const char*>(1ll << 30);\nra::Place t[] = {%s};\nfor (auto& a : t) a = ra::merged(a);\n" % \
        ", ".join(place(*x) for x in side + slots + [shifted, (H * d * 2 * 2 + 5 * row - 16, 32, []), (row * 7 + 16, 16, []),
                                                     (0, 0, []), (0, 16, [(0, 16)])])
    body += "for (auto& a : t) for (auto& b : t) printf(\"%d\", int(ra::meet(a, b)));\n"
    got = run(tmp_path, body)[0]
    t = [got[10 * i:10 * i + 10] for i in range(10)]
    assert t[0][:3] == "100" and t[1][:3] == "010" and t[2][:3] == "001"
    assert t[3][3:5] == "10" and t[4][3:5] == "01" and t[5][1] == "1"
    assert t[6][:3] == "011" and t[7][:3] == "100"  # an interval across the border of two parts, one inside a part
    assert t[8] == "0" * 10 and t[9] == "0" * 10
