"""Host checks of the attention's plan (no GPU): the pieces of the schedule
cover every visible (query, key) pair once, the parts of split rows lie in
slots of their own in the order of their keys, each output row is written once,
and every row and key index that a piece leads to lies in its sequence.  And
the refusals of geocache_plan_attention and geocache_attention."""
import ctypes

import numpy as np
import pytest

from paper_2608_13255_gb300 import build as gbuild


@pytest.fixture(scope="module")
def gc():
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


def _parse(info, schedule):
    raw = schedule.numpy()
    at = (info.n_ctas + 1 + 15) // 16 * 16
    ptr = raw[:info.n_ctas + 1]
    items = raw[at:at + 16 * info.n_items].reshape(-1, 16)
    joins = raw[at + 16 * info.n_items:].reshape(-1, 8)
    assert len(joins) == info.n_joins
    assert ptr[0] == 0 and ptr[-1] == info.n_items and (np.diff(ptr) >= 0).all()
    return ptr, items, joins


def _check(gc, q, k, Hq, Hk, D, causal, n_ctas):
    info, schedule = gc.plan_attention_host(q, k, Hq, Hk, D, causal, n_ctas)
    ptr, items, joins = _parse(info, schedule)
    q_at, k_at = np.concatenate([[0], np.cumsum(q)]), np.concatenate([[0], np.cumsum(k)])
    tok = 128 // info.pack
    assert (Hq // Hk) % info.pack == 0 and info.q_tokens == q_at[-1] and info.k_tokens == k_at[-1]
    slot_bytes = 128 * D * 4 + 128 * 4
    n_slots = info.workspace_bytes // slot_bytes
    assert info.workspace_bytes == n_slots * slot_bytes
    seen = {}      # (token, head) -> end of the keys covered so far, in the sequence's own count
    written = {}   # (token, head) -> times the output is written
    parts = {}     # slot -> (first token, tokens, head, first key)
    for it in items:
        q_row, head, hk, kv_row, n_keys, sees, t0, t1, n0, n1, s0, s1 = (int(x) for x in it[:12])
        s = int(np.searchsorted(q_at, q_row, side="right")) - 1
        assert hk == head // (Hq // Hk) and (head % (Hq // Hk)) % info.pack == 0
        key0 = kv_row - int(k_at[s])
        assert key0 % 128 == 0 and 0 <= key0 <= k[s] and n_keys == k[s] - key0
        for t, (n_tok, n_kv, slot) in enumerate(((t0, n0, s0), (t1, n1, s1))):
            assert n_tok >= 0 and n_kv >= 0 and n_tok <= tok
            if not n_tok:
                assert n_kv == 0 and slot == -1
                continue
            first = q_row + t * tok
            assert first + n_tok <= q_at[s + 1]
            assert max(0, n_kv - 1) * 128 <= max(0, n_keys - 1)  # the last key tile begins inside the sequence
            for i in range(n_tok):
                own = first + i - int(q_at[s])
                visible = min(n_keys, sees + t * tok + i) if causal else n_keys
                assert (visible + key0 == max(0, min(k[s], own + 1 + k[s] - q[s]))) or (visible <= 0 and causal) or not causal
                end = key0 + max(0, min(visible, n_kv * 128))
                for h in range(head, head + info.pack):
                    r = (first + i, h)
                    if r in seen:
                        assert seen[r][1] == key0  # this part begins where the last one ended
                    else:
                        assert key0 == 0
                    if visible <= 0 and key0:
                        end = seen[r][0]  # a row of the tile that sees none of this part's keys
                    seen[r] = (end, key0 + n_kv * 128)
                    if slot < 0:
                        written[r] = written.get(r, 0) + 1
            if slot >= 0:
                assert 0 <= slot < n_slots and slot not in parts
                parts[slot] = (first, n_tok, head, key0)
    assert len(parts) == n_slots
    used = set()
    for j in joins:
        q_row, n_tok, head, slot, n_parts = (int(x) for x in j[:5])
        assert n_parts > 1
        keys = []
        for x in range(slot, slot + n_parts):
            assert x not in used
            used.add(x)
            assert parts[x][:3] == (q_row, n_tok, head)
            keys.append(parts[x][3])
        assert keys == sorted(set(keys)) and keys[0] == 0
        for i in range(n_tok):
            for h in range(head, head + info.pack):
                written[(q_row + i, h)] = written.get((q_row + i, h), 0) + 1
    assert used == set(parts)
    # every row is written once and has seen all of its keys
    assert len(written) == q_at[-1] * Hq and set(written.values()) <= {1}
    for s in range(len(q)):
        for i in range(q[s]):
            visible = max(0, min(k[s], i + 1 + k[s] - q[s])) if causal else k[s]
            for h in range(Hq):
                assert seen[(int(q_at[s]) + i, h)][0] == visible, (s, i, h)
    return info


@pytest.mark.parametrize("n_ctas", [1, 7, 152])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q,k,Hq,Hk", [
    ([1], [1], 1, 1), ([0], [5], 2, 1), ([3], [0], 2, 2), ([], [], 4, 4),
    ([512], [512], 2, 2), ([129, 0, 256, 1], [300, 7, 0, 1500], 3, 1), ([300], [4000], 6, 2),
    ([1, 1, 1], [5000, 1, 129], 8, 1), ([17, 5], [9000, 8999], 4, 4), ([700, 64, 2, 0, 33, 200], [520, 5, 409, 30, 0, 200], 12, 2),
    ([40], [2000], 130, 1), ([257, 128, 127], [257, 128, 127], 5, 5),
], ids=str)
def test_schedule_covers_every_pair_once(gc, q, k, Hq, Hk, causal, n_ctas):
    _check(gc, q, k, Hq, Hk, 64, causal, n_ctas)


def test_random_schedules(gc):
    rng = np.random.default_rng(5)
    split = 0
    for _ in range(40):
        n = int(rng.integers(1, 6))
        q = [int(x) for x in rng.integers(0, 400, n)]
        k = [int(x) for x in rng.integers(0, 3000, n)]
        Hk = int(rng.choice([1, 2, 3]))
        info = _check(gc, q, k, Hk * int(rng.choice([1, 2, 5, 8])), Hk, int(rng.choice([40, 128])), bool(rng.integers(2)),
                      int(rng.choice([3, 33, 152])))
        split += info.n_joins > 0
    assert split > 5  # both ways of dividing the work came up


def test_plan_checks_arguments(gc):
    L = gc.load()
    q, k = (ctypes.c_int32 * 2)(10, 20), (ctypes.c_int32 * 2)(10, 20)
    info = gc.AttentionPlanInfo()

    def call(q=q, k=k, n=2, Hq=4, Hk=2, D=64, ctas=8, plan=None, schedule=None, nbytes=0):
        return L.geocache_plan_attention(q, k, n, Hq, Hk, D, 0, ctas, ctypes.byref(info) if plan is None else None,
                                         schedule, nbytes)

    assert call() == gc.OK and info.n_items > 0
    assert call(q=None) == gc.EINVAL and call(k=None) == gc.EINVAL and call(plan=0) == gc.EINVAL
    assert call(schedule=8, nbytes=1 << 20) == gc.EINVAL  # not 16-byte aligned
    buf = (ctypes.c_char * 4096)()
    at = ctypes.addressof(buf) + -ctypes.addressof(buf) % 16
    assert call(schedule=at, nbytes=8) == gc.EINVAL and "takes" in gc.last_error()
    assert call(n=-1) == gc.ESHAPE and call(Hq=3) == gc.ESHAPE and call(Hk=0) == gc.ESHAPE and call(Hq=1) == gc.ESHAPE
    for d in (0, 4, 60, 136, -8):
        assert call(D=d) == gc.ESHAPE
    assert call(ctas=-1) == gc.ESHAPE
    assert call(q=(ctypes.c_int32 * 2)(-1, 5)) == gc.ESHAPE
    big = (ctypes.c_int32 * 2)(2 ** 31 - 1, 2 ** 31 - 1)
    assert call(q=(ctypes.c_int32 * 2)(1, 1), k=big) == gc.ESHAPE
    many = (ctypes.c_int32 * 2)(2 ** 30 - 1024, 2 ** 30 - 1024)
    assert call(q=many, k=many, Hq=4096, Hk=4096) == gc.ESHAPE and "pieces" in gc.last_error()
    # offsets near 2^31: one row against the largest cache
    assert call(q=(ctypes.c_int32 * 1)(1), k=(ctypes.c_int32 * 1)(2 ** 31 - 1024), n=1) == gc.OK


def test_attention_checks_arguments(gc):
    L = gc.load()
    info, _ = gc.plan_attention_host([100, 40], [300, 4000], 4, 2, 64, False, 152)
    assert info.workspace_bytes > 0
    M = 1 << 24

    def heads(data, ts=None, hs=64, H=4):
        return gc.Heads(data, H * 64 if ts is None else ts, hs)

    def call(plan=info, schedule=M, q=None, k=None, v=None, out=None, lse=None, dtype=1, scale=0.125, ws=6 * M, nbytes=None):
        x = (plan, q or heads(2 * M), k or heads(3 * M, H=2), v or heads(4 * M, H=2), out or heads(5 * M))
        plan, q, k, v, out = map(ctypes.byref, x)
        return L.geocache_attention(plan, schedule, q, k, v, out, lse, dtype, scale, ws,
                                    info.workspace_bytes if nbytes is None else nbytes, None)

    assert L.geocache_attention(None, M, M, M, M, M, None, 1, 0.1, None, 0, None) == gc.EINVAL
    assert call(dtype=0) == gc.EDTYPE and call(dtype=3) == gc.EDTYPE
    for s in (0.0, -1.0, float("inf"), float("nan"), 1e-60, 1e60):
        assert call(scale=s) == gc.EINVAL
    assert call(schedule=None) == gc.EINVAL and call(schedule=M + 8) == gc.EINVAL
    assert call(ws=None) == gc.EINVAL and call(nbytes=info.workspace_bytes - 1) == gc.EINVAL and call(ws=6 * M + 4) == gc.EINVAL and call(ws=6 * M + 16) == gc.EINVAL
    assert call(lse=7 * M + 2) == gc.EINVAL
    assert call(q=heads(2 * M + 8)) == gc.EINVAL and call(k=heads(3 * M, hs=68, H=2)) == gc.EINVAL
    assert call(v=heads(4 * M, ts=132)) == gc.EINVAL and call(out=heads(None)) == gc.EINVAL
    assert call(q=heads(2 * M, ts=-64)) == gc.ESHAPE
    assert call(out=heads(2 * M)) == gc.EALIAS and call(out=heads(3 * M + 128, H=2, ts=256)) == gc.EALIAS
    assert call(out=heads(5 * M, ts=0)) == gc.EALIAS
    assert call(ws=4 * M) == gc.EALIAS and call(lse=6 * M) == gc.EALIAS and call(lse=5 * M) == gc.EALIAS
    assert call(schedule=6 * M) == gc.EALIAS
    # a struct that no plan call filled
    for field, value in (("Hq", 3), ("D", 200), ("pack", 0), ("n_ctas", 0), ("n_items", 0), ("workspace_bytes", 8),
                         ("schedule_bytes", 64), ("q_tokens", -1)):
        bad = gc.AttentionPlanInfo.from_buffer_copy(info)
        setattr(bad, field, value)
        assert call(plan=bad) == gc.ESHAPE, field
    assert gc.last_launches() == 0
    # no queries at all: nothing to do
    none, _ = gc.plan_attention_host([0], [10], 4, 2, 64, False, 8)
    assert call(plan=none, schedule=None) == gc.OK and gc.last_launches() == 0


def test_binding_checks(gc):
    import torch
    with pytest.raises(ValueError):
        gc.plan_attention_host([1, 2], [1], 1, 1, 64, n_ctas=1)
    with pytest.raises(ValueError):
        gc.plan_attention_host([2 ** 31], [1], 1, 1, 64, n_ctas=1)
    with pytest.raises(TypeError):
        gc.plan_attention_host([1.5], [1], 1, 1, 64, n_ctas=1)
    info, schedule = gc.plan_attention_host([4], [4], 1, 1, 64, n_ctas=1)
    plan = gc.AttentionPlan(info, schedule, None)
    x = torch.zeros((4, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        gc.attention(plan, x, x, x, out=x)  # not on a CUDA device
    with pytest.raises(TypeError):
        gc.attention(plan, x.float(), x, x)
