"""Calls whose bias gradient is tested against the narrow bounds: tiles of each kind, borders near and far, short and long sequences."""
import paper_2506_21411_amd as dchag

LOG = dchag.log_borders(8, 32)

CASES = {
    "64": dict(dtype="bf16", heads=16, kv=16, d=64, ql=[129, 257, 1, 190] * 9, borders=LOG, seed=61),
    "128": dict(dtype="bf16", heads=16, kv=16, d=128, ql=[200, 77, 130, 65] * 9, borders=[1, 4, 60], seed=62),
    "32 causal": dict(dtype="bf16", heads=32, kv=16, d=32, ql=[200, 77, 130, 65] * 9, causal=True, borders=LOG, seed=63),
    "64 long": dict(dtype="bf16", heads=32, kv=8, d=64, ql=[1100, 1030], borders=[1, 2, 70, 300], seed=64),
    "128 long": dict(dtype="bf16", heads=32, kv=32, d=128, ql=[1100, 1030], borders=[2, 3, 100], seed=65),
    "128 long causal": dict(dtype="bf16", heads=32, kv=16, d=128, ql=[1100, 1030], causal=True, borders=LOG, seed=66),
    "128 far": dict(dtype="bf16", heads=32, kv=32, d=128, ql=[1100, 1100], borders=[1, 2, 500, 700, 1024], seed=67),
    "few rows": dict(dtype="bf16", heads=2, kv=1, d=128, ql=[300, 1200], borders=[1, 2, 500, 1023], seed=68),
    "more keys": dict(dtype="bf16", heads=4, kv=2, d=64, ql=[100, 37, 5], kl=[700, 300, 900], borders=LOG, seed=69),
    "counted keys": dict(dtype="bf16", heads=4, kv=2, d=64, ql=[100, 37], kl=[700, 300], used=[411, 300], causal=True, borders=LOG, seed=70),
    "f32": dict(dtype="f32", heads=16, kv=8, d=64, ql=[129, 257, 1, 190] * 5, borders=LOG, seed=71),
    "f32 128": dict(dtype="f32", heads=2, kv=2, d=128, ql=[300, 700], borders=[1, 2, 500, 1023], seed=72),
}
