// The calling thread's last error (tg_last_error): keeps the message, returns the code.
#pragma once
int tg_fail(int code, const char* fmt, ...);
