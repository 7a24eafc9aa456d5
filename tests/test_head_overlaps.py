"""Outputs and workspaces of the calls at the end of a section that overlap something else are turned down before anything is launched: none of this needs a GPU."""
import ctypes as C

import pytest

from paper_2605_10501_amd import binding as B

N, V, D, K = 32, 1024, 128, 8
STEP = 1 << 28                                        # nobody follows these; each is far from the others
WS_BYTES = STEP


def _config(at):
    return C.byref(B._HeadCfg(V, D, B.MS_BF16, 0, 1.0, 1.0, at["w"]))


def top(a):
    return B._fn("ms_top_logits")(_config(a), N, a["h"], K, a["values"], a["ids"], a["lse"], a["ws"], WS_BYTES, None)


def tkd(a):
    return B._fn("ms_topk_kd_loss_forward_backward")(_config(a), N, a["h"], K, a["top_ids"], a["top_logits"], a["lse_teacher"], a["loss"], a["kl_tok"], a["d_h"], a["d_w"], a["ws"], WS_BYTES, None)


def logp(a):
    return B._fn("ms_token_logprobs")(_config(a), N, a["h"], a["labels"], a["logp"], a["ws"], WS_BYTES, None)


def back(a):
    return B._fn("ms_token_logprobs_backward")(_config(a), N, a["h"], a["labels"], a["d_logp"], a["logp"], a["d_h"], a["d_w"], a["ws"], WS_BYTES, None)


def policy(a):
    pc = B._PolicyCfg(0.2, 0.2, 0.1)
    return B._fn("ms_policy_loss_forward_backward")(_config(a), C.byref(pc), N, a["h"], a["labels"], a["old_logp"], a["ref_logp"], a["advantages"], a["weights"], a["loss"], a["loss_tok"], a["logp"],
                                                    a["d_h"], a["d_w"], a["ws"], WS_BYTES, None)


def pref(a):
    host = (C.c_int32 * 3)(0, 20, N)
    b, pc = B.BatchC(N, 2, C.c_void_p(a["cu"]), host), B._PreferenceCfg(0.1, 0.0)
    return B._fn("ms_preference_loss_forward_backward")(_config(a), C.byref(pc), C.byref(b), a["h"], a["labels"], a["ref_logp"], a["loss"], a["margin"], a["logp"], a["d_h"], a["d_w"], a["ws"], WS_BYTES,
                                                        None)


SIZE = dict(h=N * D * 2, w=V * D * 2, d_h=N * D * 2, d_w=V * D * 4, ws=64, values=N * K * 4, ids=N * K * 4, top_ids=N * K * 4, top_logits=N * K * 4, loss=4, margin=4, cu=12)      # the rest: 4 N
CALLS = {top: (["h", "w"], ["values", "ids", "lse", "ws"]), tkd: (["h", "w", "top_ids", "top_logits", "lse_teacher"], ["loss", "kl_tok", "d_h", "d_w", "ws"]),
         logp: (["h", "w", "labels"], ["logp", "ws"]), back: (["h", "w", "labels", "d_logp"], ["logp", "d_h", "d_w", "ws"]),
         policy: (["h", "w", "labels", "old_logp", "ref_logp", "advantages", "weights"], ["loss", "loss_tok", "logp", "d_h", "d_w", "ws"]),
         pref: (["h", "w", "labels", "ref_logp", "cu"], ["loss", "margin", "logp", "d_h", "d_w", "ws"])}
PAIRS = [(f, x, y) for f, (reads, writes) in CALLS.items() for i, x in enumerate(writes) for y in reads + writes[:i] if (x, y) != ("d_h", "h")]


@pytest.mark.parametrize("call,written,other", PAIRS, ids=[f"{f.__name__}-{x}-{y}" for f, x, y in PAIRS])
def test_an_output_over_something_else(call, written, other):
    reads, writes = CALLS[call]
    at = {name: (i + 4) * STEP for i, name in enumerate(reads + writes)}
    starts = {at[other]}                                                            # at its first byte, over its first and its last (d_h, d_w and the workspace: whole 16 bytes)
    size = {name: SIZE.get(name, 4 * N) for name in (written, other)}
    starts.add(at[other] + (size[other] - 1) // 16 * 16)
    starts.add(at[other] - (size[written] - 1) // 16 * 16)
    for start in starts:
        assert call({**at, written: start}) != 0
        assert "overlap" in B.lib().ms_last_error().decode()
